// The forward product of long matrices of narrow rows: one kernel per type, width class and what its epilogue reads and writes.
#include "dense_rows.h"

namespace dense {

template <>
int launch_rows<FORWARD, float>(const Args<float> &a, int act, hipStream_t st) { return launch_shape<FORWARD, float, KGE_ACT_IDENTITY>(a, act, st); }
template <>
int launch_rows<FORWARD, uint16_t>(const Args<uint16_t> &a, int act, hipStream_t st) { return launch_shape<FORWARD, uint16_t, KGE_ACT_IDENTITY>(a, act, st); }

}  // namespace dense
