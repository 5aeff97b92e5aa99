// Attention of one new token per sequence, rows that begin alike, fp32 caches.
#include "attend_parts_kernels.hpp"

template int parse::pt_width<float, false>(const PtArgs &, int64_t, hipStream_t);
