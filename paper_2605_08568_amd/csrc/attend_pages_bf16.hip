// Attention of one new token per sequence, listed pages, bf16 caches.
#include "attend_parts_kernels.hpp"

template int parse::pt_width<uint16_t, true>(const PtArgs &, int64_t, hipStream_t);
