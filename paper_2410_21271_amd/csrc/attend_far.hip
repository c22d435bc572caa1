// Attention of one new token per request over the last tokens of its pages and some first ones: the kernel of attend.inc with a second stretch of tokens,
// and with a scale for each block of the cache.
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
