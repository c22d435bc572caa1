// Attention of one new token per request over the last tokens of its pages: the kernel of attend.inc with one stretch of tokens, scales by head.
#include "attend.inc"

namespace eora {

size_t attend_workspace_bytes(int heads, int kv, int dim)
{
    AttendArgs a{};
    a.heads = heads;
    a.kv = kv;
    set_blocks(a);
    // two partial results a wavefront that a launch may have (a workspace for wide heads also serves narrower ones, of which there are more at a time)
    size_t row = CUS * residents<64>() * (64 + 2);
    if (dim >= 128 && row < CUS * residents<128>() * (128 + 2)) row = CUS * residents<128>() * (128 + 2);
    if (dim >= 256 && row < CUS * residents<256>() * (256 + 2)) row = CUS * residents<256>() * (256 + 2);
    return ((size_t)COUNTERS + 2 * NW * row * a.rows) * sizeof(float);
}

namespace {
template <int DIM>
hipError_t start(AttendArgs& a, hipStream_t stream)
{
    return a.bits == 8 ? start<DIM, 8, false, false>(a, stream) : start<DIM, 16, false, false>(a, stream);
}
}  // namespace

hipError_t launch_attend(AttendArgs a, hipStream_t stream)
{
    set_blocks(a);
    return a.dim == 64 ? start<64>(a, stream) : (a.dim == 128 ? start<128>(a, stream) : start<256>(a, stream));
}

}  // namespace eora
