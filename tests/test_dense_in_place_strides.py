"""In place the residual and the added gradient are read where the result is written: with another row stride than the result's a
row would be read after another block has written it.  Refused before anything runs; no GPU is needed."""
import ctypes as C

import pytest

EINVAL = -1


@pytest.fixture(scope="module")
def kb():
    from paper_2201_02791_amd import binding
    binding.load()
    return binding


@pytest.mark.parametrize("dtype", [0, 1])
def test_strides_of_results_in_place(kb, dtype):
    lib, d = kb.load(), kb._Dense(8, 8, 1, dtype, 1 << 12, None)
    X, Y, Z, G = (C.c_void_p((k + 1) << 12) for k in range(4))
    none, n = C.c_void_p(0), C.c_int64(5)
    at = lambda x: C.c_int64(x)  # noqa: E731
    for ldr, ldy in ((16, 8), (8, 16), (9, 8)):
        assert lib.kge_dense_forward(C.byref(d), n, X, at(8), Y, at(ldr), Y, at(ldy), none, at(0), none) == EINVAL
        assert b"row stride" in lib.kge_last_error()
        assert lib.kge_dense_backward(C.byref(d), n, X, at(8), Z, at(8), G, at(8), Y, at(ldr), Y, at(ldy), none, none, none, C.c_size_t(0), none) == EINVAL
        assert b"row stride" in lib.kge_last_error()
