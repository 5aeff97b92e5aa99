// Attention of one new token per sequence, rows that begin alike, bf16 caches.
#include "attend_parts_kernels.hpp"

template int parse::pt_width<uint16_t, false>(const PtArgs &, int64_t, hipStream_t);
