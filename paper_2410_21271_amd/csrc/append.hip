// Head norms, position rotations and the store into the paged cache, in one pass over q, k and v.
//
//      n = x * rsqrt(mean(x^2) + eps) * w          (per head; without a weight n = x)
//      (a, b) -> (a c - b s, b c + a s)            (a, b): columns (i, i + rot/2) or (2i, 2i + 1), (c, s) of the token's position
//      q -> q_out (fp16), k and v -> the token's slot of the cache (fp16, or e4m3 of value / scale of the head)
//
// Bound by memory where nothing is turned (8192 tokens, 64 + 8 + 8 heads of 128 into 8 bits: 62 us, 5.2 TB/s; with norms and rotations 68 us).  A head is held by
// dim / 8 lanes, two groups of four columns each: where pairs are (i, i + rot/2), the groups are partners, so that a lane has both columns of its pairs, four (cos, sin) and no
// exchange (with eight neighbouring columns a lane, the partners fetched from another one and the sum over LDS, the instructions of a value bound it: 96 us).  The sum of squares is three to five
// exchanges within a row of lanes.  A workgroup belongs to one token and keeps the token's (cos, sin) and the weights in registers over all heads that it
// passes; few tokens are cut over several workgroups.  All arithmetic is in fp32; a value is rounded once, when it is stored.
#include "serving.hpp"
#include "tiles.hpp"

namespace eora {
namespace {

constexpr int THREADS = 256;

// v plus the value of another lane of its row of 16
template <int CTRL>
__device__ __forceinline__ float plus_dpp(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
// sum over the LPH lanes of a head, in all of them
template <int LPH>
__device__ __forceinline__ float sum_of_head(float v)
{
    v = plus_dpp<0xB1>(v);                                // lanes 1, 0, 3, 2 of each four
    v = plus_dpp<0x4E>(v);                                // lanes 2, 3, 0, 1
    v = plus_dpp<0x141>(v);                               // the eight lanes mirrored: the other four
    if constexpr (LPH >= 16) v = plus_dpp<0x140>(v);      // the sixteen mirrored: the other eight
    if constexpr (LPH >= 32) v += __shfl_xor(v, 16, 64);
    return v;
}

typedef _Float16 h4 __attribute__((ext_vector_type(4)));

template <int DIM, bool Q8, bool INTERLEAVED>
__global__ __launch_bounds__(THREADS) void append_kernel(const AppendArgs a)
{
    constexpr int LPH = DIM / 8;                          // lanes per head
    constexpr int PER = THREADS / LPH;                    // heads at a time
    const int token = blockIdx.x / a.slices, slice = blockIdx.x - token * a.slices;
    const int c = threadIdx.x % LPH, mine = threadIdx.x / LPH;
    const int total = a.heads + 2 * a.kv, half = a.rot / 2;
    // this lane's columns: col0 .. col0 + 3 and col1 .. col1 + 3
    const bool turns = 8 * c < a.rot;
    const int col0 = !INTERLEAVED && turns ? 4 * c : 8 * c, col1 = !INTERLEAVED && turns ? half + 4 * c : 8 * c + 4;

    // (cos, sin) of its four pairs; a position outside the table has none: the rotated columns become NaN
    float co[4] = {1.f, 1.f, 1.f, 1.f}, si[4] = {0.f, 0.f, 0.f, 0.f};
    if (turns) {
        const int pos = a.positions[token];
        const bool known = (unsigned)pos < (unsigned)a.n_positions;
        const f4* at = (const f4*)(a.rotations + (size_t)(known ? pos : 0) * a.rot + 8 * c);
        const f4 lo = at[0], hi = at[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            co[e] = known ? (e < 2 ? lo[2 * e] : hi[2 * e - 4]) : __builtin_nanf("");
            si[e] = e < 2 ? lo[2 * e + 1] : hi[2 * e - 3];
        }
    }
    const long long slot = a.slots[token];
    const bool stored = slot >= 0 && slot < (long long)a.n_slots;
    const unsigned page = stored ? (unsigned)slot / (unsigned)a.page : 0, place = stored ? (unsigned)slot % (unsigned)a.page : 0;

    // weights of this lane's columns, those of the kind of head that comes next
    float w[8];
    auto weights = [&](const _Float16* from) {
        if (!from) return;
        const h4 lo = *(const h4*)(from + col0), hi = *(const h4*)(from + col1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = (float)lo[e];
            w[4 + e] = (float)hi[e];
        }
    };
    auto fetch = [&](const _Float16* head, float (&x)[8]) {
        const h4 lo = *(const h4*)(head + col0), hi = *(const h4*)(head + col1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = (float)lo[e];
            x[4 + e] = (float)hi[e];
        }
    };
    auto norm = [&](float (&x)[8]) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
        const float rstd = rsqrtf(sum_of_head<LPH>(sum) * (1.f / DIM) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * rstd * w[e];
    };
    auto turn = [&](float (&x)[8]) {
        if (!turns) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float &p = INTERLEAVED ? x[2 * e] : x[e], &q = INTERLEAVED ? x[2 * e + 1] : x[4 + e];
            const float was = p;
            p = was * co[e] - q * si[e];
            q = q * co[e] + was * si[e];
        }
    };
    auto put16 = [&](_Float16* head, const float (&x)[8]) {
        h4 lo, hi;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            lo[e] = (_Float16)x[e];
            hi[e] = (_Float16)x[4 + e];
        }
        *(h4*)(head + col0) = lo;
        *(h4*)(head + col1) = hi;
    };
    auto store = [&](void* pages, int h, const float* scales, float (&x)[8]) {
        if (!stored) return;
        const size_t head = (((size_t)page * a.kv + h) * a.page + place) * DIM;
        if constexpr (Q8) {
            // nearest-even to e4m3, saturating; NaN stays NaN
            const float scale = scales[h];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = x[e] / scale;
                x[e] = v != v ? v : fminf(fmaxf(v, -448.f), 448.f);
            }
            int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], 0, false);
            *(int*)((char*)pages + head + col0) = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
            *(int*)((char*)pages + head + col1) = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], hi, true);
        } else {
            put16((_Float16*)pages + head, x);
        }
    };

    // Heads in one row, q's, k's and v's.  (The lanes of a head take every branch together, and exchange only among themselves.)
    const int first = slice * PER + mine, step = a.slices * PER;
    int h = first;
    weights(a.q_weight);
    for (; h < a.heads; h += step) {
        float x[8];
        fetch(a.q + (size_t)token * a.q_stride + (size_t)h * DIM, x);
        if (a.q_weight) norm(x);
        turn(x);
        put16(a.q_out + ((size_t)token * a.heads + h) * DIM, x);        // (in place: these lanes have read all of it)
    }
    if (h < a.heads + a.kv) weights(a.k_weight);
    for (; h < a.heads + a.kv; h += step) {
        float x[8];
        fetch(a.k + (size_t)token * a.k_stride + (size_t)(h - a.heads) * DIM, x);
        if (a.k_weight) norm(x);
        turn(x);
        store(a.pages_k, h - a.heads, a.k_scale, x);
    }
    for (; h < total; h += step) {
        float x[8];
        fetch(a.v + (size_t)token * a.v_stride + (size_t)(h - a.heads - a.kv) * DIM, x);
        store(a.pages_v, h - a.heads - a.kv, a.v_scale, x);
    }
}

template <int DIM>
hipError_t start(const AppendArgs& a, unsigned grid, hipStream_t stream)
{
    if (a.interleaved) {
        if (a.bits == 8) append_kernel<DIM, true, true><<<grid, THREADS, 0, stream>>>(a);
        else append_kernel<DIM, false, true><<<grid, THREADS, 0, stream>>>(a);
    } else {
        if (a.bits == 8) append_kernel<DIM, true, false><<<grid, THREADS, 0, stream>>>(a);
        else append_kernel<DIM, false, false><<<grid, THREADS, 0, stream>>>(a);
    }
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
