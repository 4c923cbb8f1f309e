// The input gradient of long matrices of narrow rows: one kernel per type, activation, width class and added gradient.
#include "dense_rows.h"

namespace dense {

namespace {
template <class T>
int by_act(const Args<T> &a, int act, hipStream_t st)
{
    if (act == KGE_ACT_SILU) return launch_shape<INPUT, T, KGE_ACT_SILU>(a, act, st);
    if (act == KGE_ACT_RELU) return launch_shape<INPUT, T, KGE_ACT_RELU>(a, act, st);
    return launch_shape<INPUT, T, KGE_ACT_IDENTITY>(a, act, st);
}
}  // namespace

template <>
int launch_rows<INPUT, float>(const Args<float> &a, int act, hipStream_t st) { return by_act(a, act, st); }
template <>
int launch_rows<INPUT, uint16_t>(const Args<uint16_t> &a, int act, hipStream_t st) { return by_act(a, act, st); }

}  // namespace dense
