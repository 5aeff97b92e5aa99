// Attention of one new token per sequence, listed pages, fp32 caches.
#include "attend_parts_kernels.hpp"

template int parse::pt_width<float, true>(const PtArgs &, int64_t, hipStream_t);
