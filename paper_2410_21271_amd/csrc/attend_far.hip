// Attention of one new token per request over the last tokens of its pages and some first ones: the kernel of attend.inc with a second stretch of tokens,
// and with a scale for each block of the cache.  Bound by memory as that one: a block's power of two goes into the conversion of its codes to fp16, which stays exact, and first tokens are more tiles in
// front of the run.  64 / 8 heads of 128, scales by block, 160 requests to 8192 tokens (1081 MB): 199 us, 5.4 TB/s, as with scales by head (197.5).  32 / 8 heads, 64 requests of 1 to 8192 tokens, a
// window of 2048 and 16 first tokens (72 MB): 28.7 us; 13 / 13 heads of 64 in fp16, 37 requests, a window of 1000 and 37 first tokens (32 MB): 19.2, both mostly the start and the joins.
#include "attend.inc"

namespace eora {
namespace {
template <int DIM>
hipError_t start(AttendArgs& a, hipStream_t stream)
{
    if (a.bits == 16) return start<DIM, 16, true, false>(a, stream);
    return a.k_scales ? start<DIM, 8, true, true>(a, stream) : start<DIM, 8, true, false>(a, stream);
}
}  // namespace

hipError_t launch_attend_far(AttendArgs a, hipStream_t stream)
{
    set_blocks(a);
    return a.dim == 64 ? start<64>(a, stream) : (a.dim == 128 ? start<128>(a, stream) : start<256>(a, stream));
}

}  // namespace eora
