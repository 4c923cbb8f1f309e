"""Lists of tensors whose arrays overlap: an AdamW step would write one of them twice, in no order."""
import pytest


@pytest.fixture(scope="module")
def kb():
    from paper_2201_02791_amd import binding
    return binding


def made(kb, rows=4, d=300, bits=32):
    import torch
    p = torch.zeros(rows, d)
    return dict(param=p, grad=torch.zeros(rows, d), **kb.adamw_state(p, bits))


@pytest.mark.parametrize("bits", [32, 8])
def test_the_same_parameter_twice(kb, bits):
    a, b = made(kb, bits=bits), made(kb, bits=bits)
    with pytest.raises(kb.KgeError, match="overlaps"):
        kb.AdamWTensors([a, b, a])
    with pytest.raises(kb.KgeError, match="overlaps"):
        kb.AdamWTensors([a, dict(b, param=a["param"])])
    for k in ("m", "v", "m_scale", "v_scale"):
        if a[k] is not None:
            with pytest.raises(kb.KgeError, match="overlaps"):
                kb.AdamWTensors([a, dict(b, **{k: a[k]})])
    kb.AdamWTensors([a, b])


def test_arrays_of_one_tensor_and_parts_of_others(kb):
    import torch
    a, b = made(kb), made(kb)
    whole = torch.zeros(9, 300)
    for bad in ([dict(a, grad=a["param"])], [dict(a, m=a["v"])], [dict(a, param=whole[:4]), dict(b, param=whole[3:7])],
                [dict(a, grad=whole[:4]), dict(b, param=whole[3:7])], [dict(a, param=whole[3:7]), dict(b, grad=whole[:4])],
                [dict(a, param=whole[:4], grad=whole[4:8]), dict(b, m=whole[1:5])]):
        with pytest.raises(kb.KgeError, match="overlaps") as e:
            kb.AdamWTensors(bad)
        assert e.value.status == -1
    copy = torch.zeros(4, 300, dtype=torch.bfloat16)
    with pytest.raises(kb.KgeError, match="overlaps"):
        kb.AdamWTensors([dict(a, copy=copy), dict(b, copy=copy)])


def test_what_is_only_read_may_be_shared(kb):
    import torch
    a, b = made(kb), made(kb)
    mask, whole = torch.ones(4, dtype=torch.uint8), torch.zeros(12, 300)
    kb.AdamWTensors([dict(a, rows="mask", row_mask=mask), dict(b, rows="mask", row_mask=mask.data_ptr())])
    kb.AdamWTensors([a, dict(b, grad=a["grad"])])
    kb.AdamWTensors([dict(a, param=whole[:4], grad=whole[4:8]), dict(b, param=whole[8:])])         # side by side
    empty = torch.zeros(0, 300)
    kb.AdamWTensors([a, b, dict(param=empty, grad=empty, m=empty, v=empty), dict(param=empty, grad=empty, m=empty, v=empty)])
