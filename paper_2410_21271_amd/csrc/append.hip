// Head norms, position rotations and the store into the paged cache, in one pass over q, k and v.
//
//      n = x * rsqrt(mean(x^2) + eps) * w          (per head; without a weight n = x)
//      (a, b) -> (a c - b s, b c + a s)            (a, b): columns (i, i + rot/2) or (2i, 2i + 1), (c, s) of the token's position
//      q -> q_out (fp16), k and v -> the token's slot of the cache (fp16, or e4m3 of value / scale of the head)
//
// Bound by memory: every value is read once and written once.  A head is held by dim / 8 lanes, 16 bytes each, so that its sum of squares
// is a few lane exchanges, its store one contiguous piece, and the partner column of a rotation sits in another lane of the same
// wavefront (one exchange of the raw 16 bytes; rot/2 is a whole number of lanes).  A workgroup belongs to one token and keeps the
// token's (cos, sin) in registers over all heads that it passes; few tokens are cut over several workgroups.  All arithmetic is in fp32; a value is
// rounded once, when it is stored.
#include "serving.hpp"
#include "tiles.hpp"

namespace eora {
namespace {

constexpr int THREADS = 256;

template <int DIM, bool Q8>
__global__ __launch_bounds__(THREADS) void append_kernel(const AppendArgs a)
{
    constexpr int LPH = DIM / 8;                          // lanes per head
    constexpr int PER = THREADS / LPH;                    // heads at a time
    const int token = blockIdx.x / a.slices, slice = blockIdx.x - token * a.slices;
    const int c = threadIdx.x % LPH, mine = threadIdx.x / LPH, col = 8 * c;
    const int total = a.heads + 2 * a.kv;

    // (cos, sin) of this lane's columns; a position outside the table has none: the rotated columns become NaN
    float cs[8], sn[8];
    const bool turns = col < a.rot;
    if (turns) {
        const int pos = a.positions[token];
        const bool known = (unsigned)pos < (unsigned)a.n_positions;
        const float* row = a.rotations + (size_t)(known ? pos : 0) * a.rot;
        const int half = a.rot / 2;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = a.interleaved ? (col + e) / 2 : (col < half ? col + e : col + e - half);
            const float2 v = *(const float2*)(row + 2 * i);
            const bool second = a.interleaved ? e & 1 : col >= half;
            cs[e] = known ? v.x : __builtin_nanf("");
            sn[e] = second ? v.y : -v.y;                  // a c - b s, b c + a s
        }
    }
    const int partner = turns && !a.interleaved ? (col < a.rot / 2 ? c + a.rot / 16 : c - a.rot / 16) : c;
    const int from = (threadIdx.x & 63) - c + partner;    // the lane that holds the partner columns
    const long long slot = a.slots[token];
    const bool stored = slot >= 0 && slot < (long long)a.n_slots;
    const unsigned page = stored ? (unsigned)slot / (unsigned)a.page : 0, place = stored ? (unsigned)slot % (unsigned)a.page : 0;

    for (int h0 = slice * PER; h0 < total; h0 += a.slices * PER) {
        const int h = h0 + mine;
        const bool live = h < total;
        const int kind = !live || h < a.heads ? 0 : (h < a.heads + a.kv ? 1 : 2), hk = h - a.heads - (kind == 2 ? a.kv : 0);
        const _Float16* src = kind == 0 ? a.q + (size_t)token * a.q_stride + (size_t)(live ? h : 0) * DIM
                                        : (kind == 1 ? a.k + (size_t)token * a.k_stride : a.v + (size_t)token * a.v_stride) + (size_t)hk * DIM;
        Frag raw;
        raw.v = *(const h8*)(src + col);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)raw.v[e];
        const _Float16* weight = kind == 0 ? a.q_weight : a.k_weight;
        const bool normed = kind != 2 && weight;
        float rstd = 1.f;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
#pragma unroll
        for (int o = 1; o < LPH; o <<= 1) sum += __shfl_xor(sum, o, 64);
        if (normed) {
            rstd = rsqrtf(sum * (1.f / DIM) + a.eps);
            const h8 w = *(const h8*)(weight + col);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = x[e] * rstd * (float)w[e];
        }
        if (a.rot > 0) {
            float other[8];
            if (a.interleaved) {
#pragma unroll
                for (int e = 0; e < 8; ++e) other[e] = x[e ^ 1];
            } else {
                Frag p;
#pragma unroll
                for (int u = 0; u < 4; ++u) p.u[u] = __shfl(raw.u[u], from, 64);
#pragma unroll
                for (int e = 0; e < 8; ++e) other[e] = (float)p.v[e];
                if (normed) {
                    const h8 w = *(const h8*)(weight + 8 * partner);
#pragma unroll
                    for (int e = 0; e < 8; ++e) other[e] = other[e] * rstd * (float)w[e];
                }
            }
            if (turns && kind != 2) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] * cs[e] + other[e] * sn[e];
            }
        }
        if (!live) continue;
        if (kind == 0) {
            h8 y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (_Float16)x[e];
            *(h8*)(a.q_out + ((size_t)token * a.heads + h) * DIM + col) = y;
        } else if (stored) {
            const size_t at = (((size_t)page * a.kv + hk) * a.page + place) * DIM + col;
            void* pages = kind == 1 ? a.pages_k : a.pages_v;
            if constexpr (Q8) {
                const float scale = (kind == 1 ? a.k_scale : a.v_scale)[hk];
                // nearest-even to e4m3, saturating; NaN stays NaN
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = x[e] / scale;
                    x[e] = v != v ? v : fminf(fmaxf(v, -448.f), 448.f);
                }
                int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], 0, false);
                lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
                hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], hi, true);
                *(int2*)((char*)pages + at) = make_int2(lo, hi);
            } else {
                h8 y;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = (_Float16)x[e];
                *(h8*)((_Float16*)pages + at) = y;
            }
        }
    }
}

template <int DIM>
hipError_t start(const AppendArgs& a, unsigned grid, hipStream_t stream)
{
    if (a.bits == 8) append_kernel<DIM, true><<<grid, THREADS, 0, stream>>>(a);
    else append_kernel<DIM, false><<<grid, THREADS, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendArgs& args, hipStream_t stream)
{
    AppendArgs a = args;
    const int per = THREADS / (a.dim / 8), total = a.heads + 2 * a.kv, most = (total + per - 1) / per;
    constexpr int LAUNCH = 1 << 20;                       // tokens of a launch
    for (int m0 = 0; m0 < args.M; m0 += LAUNCH) {
        a.M = args.M - m0 < LAUNCH ? args.M - m0 : LAUNCH;
        // few tokens: a workgroup for every `per` heads; many: one for all heads of a token, whose rotations it then reads once
        a.slices = (1024 + a.M - 1) / a.M;
        a.slices = a.slices > most ? most : a.slices;
        a.q = args.q + (size_t)m0 * a.q_stride;
        a.k = args.k + (size_t)m0 * a.k_stride;
        a.v = args.v + (size_t)m0 * a.v_stride;
        a.q_out = args.q_out + (size_t)m0 * a.heads * a.dim;
        a.positions = args.positions ? args.positions + m0 : nullptr;
        a.slots = args.slots + m0;
        const unsigned grid = (unsigned)a.M * (unsigned)a.slices;
        const hipError_t e = a.dim == 64 ? start<64>(a, grid, stream) : (a.dim == 128 ? start<128>(a, grid, stream) : start<256>(a, grid, stream));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace eora
