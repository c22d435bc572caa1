// New tokens into a paged cache of e4m3 codes with a power of two for each 16 tokens of a head, and tokens of a cache back as fp16.
//
//      n = x rsqrt(mean(x^2) + eps) w,   (a, b) -> (a c - b s, b c + a s)          (queries and keys, as eora_cache_append())
//      2^e: the least of 2^-15 .. 2^8 with |x| <= 448 2^e for all finite x of the block, and not below what the block has, unless it is begun anew
//      code = e4m3(x / 2^e)
//
// A power of two, so that a block whose values grow can take a larger one: codes that it has are divided by a power of two, which is exact but for those
// that become subnormal.  From 2^-15 on every code stands for a number that fp16 holds (the least step is 2^-24), up to 2^8 as well with codes to 240 there: whatever reads
// the cache converts without a rounding, and no scale has to be carried through a sum.
//
// Bound by memory for many tokens, by the time of its dependent reads (slots, rows, the block's scale) for few: 8192 tokens of 64 + 8 + 8 heads of 128, with norm, stored and read back
// (373 MB) in 78.7 us, 4.7 TB/s, as a copy; one token in 12 (two launches).  Queries: a workgroup for a token, as where nothing is scaled by blocks, behind all keys and
// values, whose chains are longer (85.4 us with them last).
// Keys and values: a wavefront for a block of a head, in registers (8 to 64 values a lane), so that the block's largest value is known before anything is stored and every value is read once.
// Who handles a block: the first of its rows, which are among 16 consecutive rows of the call; a wavefront looks through some rows for first ones (one row where there
// are few, so that requests with one new token each run side by side; up to 16, a block of a prompt).
#include "heads.hpp"
#include "serving.hpp"

namespace eora {
namespace {

constexpr int THREADS = 256, NW = THREADS / 64;
constexpr int LOOK = BLOCK_TOKENS - 1;                    // rows before the first that one of its block may be

__device__ __forceinline__ float power(int e) { return __uint_as_float((unsigned)(127 + e) << 23); }

// what a lane holds of a head: columns col0 .. col0 + 3 and col1 .. col1 + 3, both columns of its pairs
template <int DIM, bool INTERLEAVED>
struct Columns {
    static constexpr int LPH = DIM / 8;                   // lanes per head
    int c, col0, col1;
    bool turns;
    __device__ __forceinline__ Columns(int lane, int rot)
    {
        c = lane % LPH;
        turns = 8 * c < rot;
        col0 = !INTERLEAVED && turns ? 4 * c : 8 * c;
        col1 = !INTERLEAVED && turns ? rot / 2 + 4 * c : 8 * c + 4;
    }
    __device__ __forceinline__ void fetch(const _Float16* head, float (&x)[8]) const
    {
        const h4 lo = *(const h4*)(head + col0), hi = *(const h4*)(head + col1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = (float)lo[e];
            x[4 + e] = (float)hi[e];
        }
    }
    // (cos, sin) of the pairs at a token's position; a position outside the table has none: the rotated columns become NaN
    __device__ __forceinline__ void angles(const BlocksArgs& a, int token, float (&co)[4], float (&si)[4]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            co[e] = 1.f;
            si[e] = 0.f;
        }
        if (!turns) return;
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
    __device__ __forceinline__ void turn(float (&x)[8], const float (&co)[4], const float (&si)[4]) const
    {
        if (!turns) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float &p = INTERLEAVED ? x[2 * e] : x[e], &q = INTERLEAVED ? x[2 * e + 1] : x[4 + e];
            const float was = p;
            p = was * co[e] - q * si[e];
            q = q * co[e] + was * si[e];
        }
    }
    // all lanes of a head together
    __device__ __forceinline__ static void norm(float (&x)[8], const float (&w)[8], float eps)
    {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
        const float rstd = rsqrtf(sum_of_head<LPH>(sum) * (1.f / DIM) + eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * rstd * w[e];
    }
};

// queries of a token: workgroup `slice` of a.slices
template <int DIM, bool INTERLEAVED>
__device__ __forceinline__ void queries(const BlocksArgs& a, int token, int slice)
{
    typedef Columns<DIM, INTERLEAVED> C;
    constexpr int PER = THREADS / C::LPH;                 // heads at a time
    const C col((int)threadIdx.x, a.rot);
    float co[4], si[4], w[8];
    col.angles(a, token, co, si);
    if (a.q_weight) col.fetch(a.q_weight, w);
    for (int h = slice * PER + (int)threadIdx.x / C::LPH; h < a.heads; h += a.slices * PER) {
        float x[8];
        col.fetch(a.q + (size_t)token * a.q_stride + (size_t)h * DIM, x);
        if (a.q_weight) C::norm(x, w, a.eps);
        col.turn(x, co, si);
        h4 lo, hi;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            lo[e] = (_Float16)x[e];
            hi[e] = (_Float16)x[4 + e];
        }
        _Float16* to = a.q_out + ((size_t)token * a.heads + h) * DIM;           // (in place: these lanes have read all of it)
        *(h4*)(to + col.col0) = lo;
        *(h4*)(to + col.col1) = hi;
    }
}

// the nearest codes of four values / 2^e (by = 2^-e), saturating at `top`; NaN stays NaN
__device__ __forceinline__ int four_codes(const float* x, float by, float top)
{
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = x[e] * by;
        v[e] = v[e] != v[e] ? v[e] : fminf(fmaxf(v[e], -top), top);
    }
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
}
// four codes' values, code * 2^e (scale = 2^e): fp16 holds them
__device__ __forceinline__ void four_values(unsigned w, float scale, float* x)
{
    const h2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true);
    x[0] = (float)lo[0];
    x[1] = (float)lo[1];
    x[2] = (float)hi[0];
    x[3] = (float)hi[1];
}

// Blocks whose first row is one of a.look from r0 on, in kv head h: their keys, or values.  One wavefront.
template <int DIM, bool INTERLEAVED>
__device__ __forceinline__ void blocks_of(const BlocksArgs& a, int r0, int h, bool values)
{
    typedef Columns<DIM, INTERLEAVED> C;
    constexpr int SUBS = 64 / C::LPH, TPS = BLOCK_TOKENS / SUBS;                // tokens at a time; tokens that a lane has columns of
    const int lane = threadIdx.x & 63, sub = lane / C::LPH;
    const C col(lane, values ? 0 : a.rot);
    const _Float16* weight = values ? nullptr : a.k_weight;
    const _Float16* x_rows = values ? a.v : a.k;
    const size_t stride = values ? a.v_stride : a.k_stride;
    char* codes = (char*)(values ? a.pages_v : a.pages_k);
    uint8_t* scales = values ? a.v_scales : a.k_scales;

    // lane LOOK + i has row r0 + i
    const int row = r0 - LOOK + lane;
    const long long slot = row >= 0 && row < a.M && lane < a.look + 2 * LOOK ? a.slots[row] : -1;
    const int block = slot >= 0 && slot < (long long)a.n_slots ? (int)(slot / BLOCK_TOKENS) : -1, place = (int)(slot & (BLOCK_TOKENS - 1));
    float w[8];
    if (weight) col.fetch(weight, w);
    for (int i = LOOK; i < LOOK + a.look; ++i) {
        if (r0 - LOOK + i >= a.m0 + a.tokens) break;                            // (of the next launch)
        const int b = __builtin_amdgcn_readlane(block, i);
        if (b < 0) continue;
        const unsigned long long same = __ballot(block == b);
        if (same >> (i - LOOK) & ((1u << LOOK) - 1)) continue;                  // an earlier row handles it
        const bool in = block == b && lane >= i && lane <= i + LOOK;
        const bool begun = __ballot(in && place == 0) != 0;
        // lane t: 1 + the lane whose row goes to place t, 0: none (lane 63 takes what belongs nowhere)
        const int from = __builtin_amdgcn_ds_permute(4 * (in ? place : 63), in ? lane + 1 : 0);
        const unsigned page = (unsigned)b * BLOCK_TOKENS / (unsigned)a.page, first = (unsigned)b * BLOCK_TOKENS % (unsigned)a.page;
        const size_t at = ((size_t)page * a.kv + h) * a.page + first;           // token 0 of the block
        int old = (int)scales[at / BLOCK_TOKENS] - 127;
        old = old < SCALE_LEAST ? SCALE_LEAST : (old > SCALE_MOST ? SCALE_MOST : old);

        float x[TPS][8], most = 0.f;
        bool has[TPS];
#pragma unroll
        for (int t = 0; t < TPS; ++t) {
            const int lane_of = __shfl(from, sub + SUBS * t, 64);
            has[t] = lane_of > 0;
            if (__ballot(has[t]) == 0) continue;                                // (single tokens: 1024 requests 13.3 us, without this 22.5)
            const int token = has[t] ? r0 - LOOK + lane_of - 1 : r0 - LOOK + i;
            col.fetch(x_rows + (size_t)token * stride + (size_t)h * DIM, x[t]);
            if (weight) C::norm(x[t], w, a.eps);
            if (!values) {
                float co[4], si[4];
                col.angles(a, token, co, si);
                col.turn(x[t], co, si);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = fabsf(x[t][e]);
                most = fmaxf(most, has[t] && v < INFINITY ? v : 0.f);
            }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
        // most = 1.f 2^p: 448 is 1.75 2^8
        const unsigned bits = __float_as_uint(most);
        int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
        e = e < SCALE_LEAST ? SCALE_LEAST : (e > SCALE_MOST ? SCALE_MOST : e);
        if (!begun && old > e) e = old;
        e = __builtin_amdgcn_readfirstlane(e);
        const bool again = !begun && e != old;
        const float by = power(-e), top = e == SCALE_MOST ? 240.f : 448.f;      // (240 2^8 = 61440, the last that fp16 holds)
#pragma unroll
        for (int t = 0; t < TPS; ++t) {
            char* to = codes + (at + sub + SUBS * t) * DIM;
            if (!has[t]) {
                if (!again) continue;
                four_values(*(const unsigned*)(to + col.col0), power(old), x[t]);
                four_values(*(const unsigned*)(to + col.col1), power(old), x[t] + 4);
            }
            *(int*)(to + col.col0) = four_codes(x[t], by, top);
            *(int*)(to + col.col1) = four_codes(x[t] + 4, by, top);
        }
        if (lane == 0) scales[at / BLOCK_TOKENS] = (uint8_t)(127 + e);
    }
}

// (Seven wavefronts a SIMD: reads of a block's rows on their way together take registers of which only three are left, 8192 tokens 78.7 -> 97 us; six 81.)
template <int DIM, bool INTERLEAVED>
__global__ __launch_bounds__(THREADS, DIM == 256 ? 4 : 7) void append_blocks_kernel(const BlocksArgs a)
{
    const unsigned groups = (unsigned)((a.tokens + a.look - 1) / a.look), first = (groups * 2u * (unsigned)a.kv + NW - 1) / NW;       // workgroups of keys and values
    if (blockIdx.x >= first) {
        const unsigned id = blockIdx.x - first, token = id / (unsigned)a.slices;
        queries<DIM, INTERLEAVED>(a, a.m0 + (int)token, (int)(id - token * (unsigned)a.slices));
        return;
    }
    const unsigned unit = blockIdx.x * NW + (unsigned)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), heads = 2u * (unsigned)a.kv;
    const unsigned group = unit / heads, h = unit - group * heads;
    if (group >= groups) return;
    blocks_of<DIM, INTERLEAVED>(a, a.m0 + (int)group * a.look, (int)(h % (unsigned)a.kv), h >= (unsigned)a.kv);
}

// Eight values of a token's key and of its value a thread.  FORM: 0 fp16, 1 codes with a scale a head, 2 codes with a scale a block
template <int FORM>
__global__ __launch_bounds__(THREADS) void read_kernel(const ReadArgs a)
{
    const unsigned per = (unsigned)a.kv * (unsigned)(a.dim / 8);                // pieces of a row
    const size_t id = (size_t)blockIdx.x * THREADS + threadIdx.x;
    const size_t row = id / per;
    if (row >= (size_t)a.M) return;
    const unsigned piece = (unsigned)(id - row * per), h = piece / (unsigned)(a.dim / 8), c = piece - h * (unsigned)(a.dim / 8);
    const long long slot = a.slots[row];
    const bool there = slot >= 0 && slot < (long long)a.n_slots;
    const unsigned page = there ? (unsigned)slot / (unsigned)a.page : 0, place = there ? (unsigned)slot % (unsigned)a.page : 0;
    const size_t token = ((size_t)page * a.kv + h) * a.page + place;
#pragma unroll
    for (int values = 0; values < 2; ++values) {
        const char* pages = (const char*)(values ? a.pages_v : a.pages_k);
        Frag f;
        f.q = u4{0, 0, 0, 0};
        if (there) {
            if constexpr (FORM == 0) {
                f.q = *(const u4*)(pages + (token * a.dim + 8 * c) * 2);
            } else {
                const uint2 w = *(const uint2*)(pages + token * a.dim + 8 * c);
                float scale = 1.f;
                if constexpr (FORM == 2) scale = power_of(((const uint8_t*)(values ? a.v_scale : a.k_scale))[token / BLOCK_TOKENS]);
                float x[8];
                four_values(w.x, scale, x);
                four_values(w.y, scale, x + 4);
                const float by = FORM == 1 ? ((const float*)(values ? a.v_scale : a.k_scale))[h] : 1.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) f.v[e] = (_Float16)(x[e] * by);
            }
        }
        *(u4*)((values ? a.v : a.k) + row * (size_t)a.kv * a.dim + 8 * (size_t)piece) = f.q;
    }
}

template <int DIM>
hipError_t start(const BlocksArgs& a, unsigned grid, hipStream_t stream)
{
    if (a.interleaved) append_blocks_kernel<DIM, true><<<grid, THREADS, 0, stream>>>(a);
    else append_blocks_kernel<DIM, false><<<grid, THREADS, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append_blocks(BlocksArgs a, hipStream_t stream)
{
    const int per = THREADS / (a.dim / 8), most = (a.heads + per - 1) / per;
    constexpr int LAUNCH = 1 << 18;                       // tokens of a launch (a block whose rows two launches share is handled by its first row's)
    for (a.m0 = 0; a.m0 < a.M; a.m0 += LAUNCH) {
        a.tokens = a.M - a.m0 < LAUNCH ? a.M - a.m0 : LAUNCH;
        a.slices = (1024 + a.tokens - 1) / a.tokens;
        a.slices = a.slices > most ? most : a.slices;
        // wavefronts enough for the chip, then rows for each (32 + 8 + 8 heads of 128, prompts of 1024, 2048, 4096 tokens: with 8192 wavefronts 16.6, 18.0, 28.2 us, with 4096 10.9, 13.7,
        // 22.7, with 2048 10.3, 12.5, 23.5, but a token of each of 1024 requests then 19.8, not 13.4)
        const size_t look = (size_t)a.tokens * 2 * a.kv / 4096;
        a.look = look < 1 ? 1 : (look > BLOCK_TOKENS ? BLOCK_TOKENS : (int)look);
        const size_t units = (size_t)((a.tokens + a.look - 1) / a.look) * 2 * a.kv, grid = (size_t)a.tokens * a.slices + (units + NW - 1) / NW;
        if (grid > 0x7fffffff) return hipErrorInvalidConfiguration;
        const hipError_t e = a.dim == 64 ? start<64>(a, (unsigned)grid, stream) : (a.dim == 128 ? start<128>(a, (unsigned)grid, stream) : start<256>(a, (unsigned)grid, stream));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_read(const ReadArgs& args, hipStream_t stream)
{
    const size_t per = (size_t)args.kv * (args.dim / 8);
    const int rows = per > (1u << 30) ? 1 : (int)((1u << 30) / per);            // rows of a launch
    for (int m0 = 0; m0 < args.M;) {
        ReadArgs a = args;
        a.M = args.M - m0 < rows ? args.M - m0 : rows;
        a.slots = args.slots + m0;
        a.k = args.k + (size_t)m0 * a.kv * a.dim;
        a.v = args.v + (size_t)m0 * a.kv * a.dim;
        const unsigned grid = (unsigned)((a.M * per + THREADS - 1) / THREADS);
        if (a.bits == 16) read_kernel<0><<<grid, THREADS, 0, stream>>>(a);
        else if (a.blocks) read_kernel<2><<<grid, THREADS, 0, stream>>>(a);
        else read_kernel<1><<<grid, THREADS, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        m0 += a.M;
    }
    return hipSuccess;
}

}  // namespace eora
