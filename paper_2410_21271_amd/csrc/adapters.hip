// Low-rank pairs of many requests beside a shared projection:
//
//      y[m] = base[m] + s_a (x[m] A_a^T) B_a^T            a = adapter of row m, from a pool of any size
//
// Two launches: t = x A^T (fp32 partial sums of ranges of the contraction), then y from t and B.  Only the pairs that rows select are read,
// each once per window of 64 rows, in the stored tiles of the layer kernels.
//
// Bound by memory at a few rows per pair (4 r flops a row against 2 bytes of a factor's element): the rows of a pair are the 16 columns (or rows)
// of the matrix instructions, mostly empty, and a wavefront's work is to keep tiles in flight.  With many rows of one pair, y's own traffic bounds it.
//
// Rows are grouped without sorting: a window of 64 rows is one adapter index a lane, the rows of a pair are a ballot, and the workgroup whose row
// comes first among them (the leader) does the work for all.  Prompts have long runs of one pair; a batch of decoding requests has as many leaders as rows.
//
// t is not rounded to fp16: each row's t is scaled by a power of two to a largest value in [256, 512) and split in two fp16 (22 bits, whatever the
// size of t), both are multiplied with B's tile, and the sum is scaled back in fp32.  y is rounded once.
#include "serving.hpp"
#include "segments.hpp"

namespace eora {
namespace {

constexpr int NW = 4, THREADS = 64 * NW;
constexpr int WINDOW = 64;

// the adapter of lane's row of a window (-1: none; -2: no row)
__device__ __forceinline__ int adapter_of(const AdapterArgs& a, int row0, int lane)
{
    const int row = row0 + lane;
    if (row >= a.M) return -2;
    const int id = a.ids[row];
    return (unsigned)id < (unsigned)a.n ? id : -1;
}

// rank of a pair in whole k-tiles of B
__device__ __forceinline__ int rank_of(const AdapterArgs& a, int id, int step)
{
    if (id < 0) return 0;
    if (!a.ranks) return a.r;
    const int v = a.ranks[id];
    const int up = v <= 0 ? 0 : (v + step - 1) / step * step;
    return v > a.r || up > a.r ? a.r : up;
}

// list[s] = place (in the window) of the s-th of the rows in `rows`
__device__ __forceinline__ void list_rows(unsigned long long rows, int* list)
{
    const int lane = threadIdx.x & 63;
    if (threadIdx.x < 64 && rows >> lane & 1) list[__popcll(rows & ((1ull << lane) - 1))] = lane;
}

// First launch.  A workgroup: 16 RB ranks of the leaders' pairs x one range of the contraction, whose chunks of 128 columns its
// wavefronts share.
template <int FA, int TB, int RB>
__device__ __forceinline__ void down_tile(const AdapterArgs& a, int id, int rank, int row0, const int* list, int count, int rg, int ks, float* red)
{
    constexpr int WORDS = Fmt<FA>::WORDS, KT = Fmt<FA>::KT, TPC = 128 / KT;      // tiles of a chunk
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, j = lane >> 4;
    const int chunks = a.d_in / 128, c0 = chunks * ks / a.ksplit, c1 = chunks * (ks + 1) / a.ksplit;
    const int rb0 = rg * RB, blocks = (rank / 16 - rb0) < RB ? rank / 16 - rb0 : RB;
    const size_t pair = (size_t)id * a.r * a.d_in / KT * (64 * WORDS / 16);      // words before this pair's tiles
    const uint32_t* tiles = (const uint32_t*)a.A + pair;
    const _Float16* px[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        const int s = 16 * b + n;
        px[b] = a.x + (size_t)(row0 + list[s < count ? s : 0]) * a.d_in;
    }
    f4 acc[TB][RB];
#pragma unroll
    for (int b = 0; b < TB; ++b)
#pragma unroll
        for (int q = 0; q < RB; ++q) acc[b][q] = f4{0.f, 0.f, 0.f, 0.f};
    for (int c = c0 + wave; c < c1; c += NW) {
        uint32_t w[RB][TPC][WORDS];
        float sc[RB];
#pragma unroll
        for (int q = 0; q < RB; ++q) {
            const int rb = rb0 + (q < blocks ? q : 0);    // (blocks beyond the rank read the first one again and are not stored)
            const size_t tile = (size_t)rb * (a.d_in / KT) + (size_t)c * TPC;
#pragma unroll
            for (int t = 0; t < TPC; ++t) load_words<WORDS>(w[q][t], tiles + ((tile + t) * 64 + lane) * WORDS);
            if constexpr (FA != S_F16) sc[q] = (float)a.A_scales[((size_t)id * a.r + 16 * rb + n) * chunks + c];
        }
        h8 x[TB][4];
#pragma unroll
        for (int b = 0; b < TB; ++b)
#pragma unroll
            for (int t = 0; t < 4; ++t) x[b][t] = *(const h8*)(px[b] + 128 * c + (FA == S_F16 ? 32 * t + 8 * j : 32 * j + 8 * t));
#pragma unroll
        for (int q = 0; q < RB; ++q) {
            h8 f[4];
            if constexpr (FA == S_F16) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    Frag g;
#pragma unroll
                    for (int u = 0; u < 4; ++u) g.u[u] = w[q][t][u];
                    f[t] = g.v;
                }
            } else {
                decode_tile<FA>(w[q][0], 8u, f);
            }
#pragma unroll
            for (int b = 0; b < TB; ++b) {
                if constexpr (FA == S_F16) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) acc[b][q] = mfma16(x[b][t], f[t], acc[b][q]);
                } else {
                    f4 part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int t = 0; t < 4; ++t) part = mfma16(x[b][t], f[t], part);
                    acc[b][q] += sc[q] * part;
                }
            }
        }
    }
    // sum over the wavefronts, in order
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        if (16 * b >= count) break;
#pragma unroll
        for (int q = 0; q < RB; ++q) *(f4*)(red + ((wave * RB + q) * 64 + lane) * 4) = acc[b][q];
        __syncthreads();
        for (int e = threadIdx.x; e < RB * 256; e += THREADS) {
            // consecutive threads: consecutive ranks of one row
            const int col = e % 16, q = e / 16 % RB, slot = e / (16 * RB), l = 16 * (slot / 4) + col, i = slot % 4;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) sum += red[((w * RB + q) * 64 + l) * 4 + i];
            const int s = 16 * b + slot;
            if (s < count && q < blocks) a.t[((size_t)ks * a.M + row0 + list[s]) * a.r + 16 * (rb0 + q) + col] = sum;
        }
        __syncthreads();
    }
}

template <int FA, int RB>
__global__ __launch_bounds__(THREADS) void down_kernel(const AdapterArgs a, int step)
{
    __shared__ int list[WINDOW];
    __shared__ __attribute__((aligned(16))) float red[NW * RB * 256];
    int at = blockIdx.x;
    const int rg = at % a.rgroups;
    at /= a.rgroups;
    const int ks = at % a.ksplit;
    at /= a.ksplit;
    const int row0 = at / a.leaders * WINDOW, lane = threadIdx.x & 63;
    const int ids = adapter_of(a, row0, lane);
    for (int first = at % a.leaders; first < WINDOW; first += a.leaders) {
        const int id = __builtin_amdgcn_readlane(ids, first);
        if (id < 0) continue;
        const unsigned long long rows = __ballot(ids == id);
        if (rows & ((1ull << first) - 1)) continue;       // an earlier row leads
        const int rank = rank_of(a, id, step), count = __popcll(rows);
        if (16 * RB * rg >= rank) continue;
        __syncthreads();
        list_rows(rows, list);
        __syncthreads();
        if (count <= 16) down_tile<FA, 1, RB>(a, id, rank, row0, list, count, rg, ks, red);
        else down_tile<FA, 4, RB>(a, id, rank, row0, list, count, rg, ks, red);
    }
}

// Second launch.  A workgroup: the leaders' rows x a slab of outputs.  t goes to LDS as (high, low) fp16 pairs, one word an element, rows of r + 4 words.
template <int FE, int TB>
__device__ __forceinline__ void up_tile(const AdapterArgs& a, int id, int rank, int row0, const int* list, int count, int slab, const uint32_t* t, const float* back)
{
    constexpr int WORDS = Fmt<FE>::WORDS, KT = Fmt<FE>::KT, NF = KT / 32, PAIR = 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, j = lane >> 4;
    const int ntk = a.r / KT, nk = rank / KT, ld = a.r + 4;
    const int blocks = a.d_out / 16, first = slab * a.slab, last = first + a.slab < blocks ? first + a.slab : blocks;
    const size_t pair = id < 0 ? 0 : (size_t)id * a.d_out * a.r / KT * (64 * WORDS / 16);
    const uint32_t* tiles = (const uint32_t*)a.B + pair;
    for (int rb = first + PAIR * wave; rb < last; rb += PAIR * NW) {
        f4 acc[PAIR][TB];
#pragma unroll
        for (int p = 0; p < PAIR; ++p)
#pragma unroll
            for (int b = 0; b < TB; ++b) acc[p][b] = f4{0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < nk; ++k) {
            uint32_t w[PAIR][WORDS];
            f4 sc[PAIR];
#pragma unroll
            for (int p = 0; p < PAIR; ++p) {
                const int R = rb + p < last ? rb + p : rb;
                load_words<WORDS>(w[p], tiles + (((size_t)R * ntk + k) * 64 + lane) * WORDS);
                if constexpr (FE != S_F16) {
                    const _Float16* s = a.B_scales + ((size_t)id * a.d_out + 16 * R + 4 * j) * ntk + k;
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[p][i] = (float)s[(size_t)i * ntk];
                }
            }
            h8 f[PAIR][NF];
#pragma unroll
            for (int p = 0; p < PAIR; ++p) decode_tile<FE>(w[p], 8u, f[p]);
#pragma unroll
            for (int b = 0; b < TB; ++b) {
                f4 part[PAIR];
#pragma unroll
                for (int p = 0; p < PAIR; ++p) part[p] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int q = 0; q < NF; ++q) {
                    const uint32_t* src = t + (16 * b + n) * ld + k * KT + (KT / 4) * j + 8 * q;
                    const u4 lo4 = *(const u4*)src, hi4 = *(const u4*)(src + 4);
                    Frag high, low;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        high.u[u] = __builtin_amdgcn_perm(lo4[2 * u + 1], lo4[2 * u], 0x05040100u);
                        low.u[u] = __builtin_amdgcn_perm(lo4[2 * u + 1], lo4[2 * u], 0x07060302u);
                        high.u[2 + u] = __builtin_amdgcn_perm(hi4[2 * u + 1], hi4[2 * u], 0x05040100u);
                        low.u[2 + u] = __builtin_amdgcn_perm(hi4[2 * u + 1], hi4[2 * u], 0x07060302u);
                    }
#pragma unroll
                    for (int p = 0; p < PAIR; ++p) {
                        f4& to = FE == S_F16 ? acc[p][b] : part[p];
                        to = mfma16(f[p][q], high.v, to);
                        to = mfma16(f[p][q], low.v, to);
                    }
                }
                if constexpr (FE != S_F16) {
#pragma unroll
                    for (int p = 0; p < PAIR; ++p) acc[p][b] += sc[p] * part[p];
                }
            }
        }
#pragma unroll
        for (int b = 0; b < TB; ++b) {
            const int s = 16 * b + n;
            if (s >= count) continue;
            const size_t row = (size_t)(row0 + list[s]) * a.d_out;
            const float f = back[s];
#pragma unroll
            for (int p = 0; p < PAIR; ++p) {
                if (rb + p >= last) continue;
                const size_t at = row + 16 * (rb + p) + 4 * j;
                typedef _Float16 h4 __attribute__((ext_vector_type(4)));
                h4 y;
                if (a.base) {
                    const h4 v = *(const h4*)(a.base + at);
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = (_Float16)((float)v[i] + (rank ? acc[p][b][i] * f : 0.f));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = (_Float16)(rank ? acc[p][b][i] * f : 0.f);
                }
                *(h4*)(a.y + at) = y;
            }
        }
    }
}

template <int FE>
__global__ __launch_bounds__(THREADS) void up_kernel(const AdapterArgs a, int slabs)
{
    __shared__ int list[WINDOW];
    __shared__ unsigned top[WINDOW];
    __shared__ float back[WINDOW];
    uint32_t* t = (uint32_t*)eora_smem;                   // (rows of the largest group) x (r + 4)
    int at = blockIdx.x;
    const int slab = at % slabs;
    at /= slabs;
    const int row0 = at / a.leaders * WINDOW, lane = threadIdx.x & 63, ld = a.r + 4;
    const int ids = adapter_of(a, row0, lane);
    for (int first = at % a.leaders; first < WINDOW; first += a.leaders) {
        const int id = __builtin_amdgcn_readlane(ids, first);
        if (id == -2) continue;
        const unsigned long long rows = __ballot(ids == id);
        if (rows & ((1ull << first) - 1)) continue;
        const int rank = rank_of(a, id, Fmt<FE>::KT), count = __popcll(rows);
        if (rank == 0 && a.base == a.y) continue;         // nothing to add
        __syncthreads();
        list_rows(rows, list);
        if (threadIdx.x < WINDOW) top[threadIdx.x] = 0;
        __syncthreads();
        const int slots = count <= 16 ? 16 : 64;
        if (rank) {
            const float scaling = a.scalings ? a.scalings[id] : 1.f;
            const int quads = rank / 4;
            for (int e = threadIdx.x; e < slots * quads; e += THREADS) {
                const int s = e / quads, c = 4 * (e - s * quads);
                f4 sum = {0.f, 0.f, 0.f, 0.f};
                if (s < count) {
                    const float* src = a.t + (size_t)(row0 + list[s]) * a.r + c;
                    for (int ks = 0; ks < a.ksplit; ++ks) sum += *(const f4*)(src + (size_t)ks * a.M * a.r);
                    sum *= scaling;
                    float big = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) big = fmaxf(big, fabsf(sum[i]));
                    atomicMax(&top[s], __float_as_uint(big));         // (non-negative floats order as their bits)
                }
                *(f4*)(t + s * ld + c) = sum;
            }
            __syncthreads();
            for (int e = threadIdx.x; e < slots * quads; e += THREADS) {
                const int s = e / quads, c = 4 * (e - s * quads);
                int ex = (int)(top[s] >> 23) - 127;       // exponent of the row's largest value
                ex = top[s] == 0u ? 8 : (ex < -110 ? -110 : (ex > 127 ? 127 : ex));
                const float to = __uint_as_float((unsigned)(127 + 8 - ex) << 23);
                if (c == 0) back[s] = __uint_as_float((unsigned)(127 - 8 + ex) << 23);
                const f4 v = *(const f4*)(t + s * ld + c);
                u4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = v[i] * to;
                    const _Float16 high = (_Float16)x, low = (_Float16)(fabsf(x) == INFINITY ? 0.f : x - (float)high);
                    w[i] = (uint32_t)__builtin_bit_cast(uint16_t, high) | (uint32_t)__builtin_bit_cast(uint16_t, low) << 16;
                }
                *(u4*)(t + s * ld + c) = w;
            }
        } else if (threadIdx.x < WINDOW) {
            back[threadIdx.x] = 0.f;
        }
        __syncthreads();
        if (count <= 16) up_tile<FE, 1>(a, id, rank, row0, list, count, slab, t, back);
        else up_tile<FE, 4>(a, id, rank, row0, list, count, slab, t, back);
    }
}

constexpr int MAX_KSPLIT = 8;

template <int FA, int RB>
hipError_t start_down(const AdapterArgs& a, unsigned grid, int step, hipStream_t stream)
{
    down_kernel<FA, RB><<<grid, THREADS, 0, stream>>>(a, step);
    return hipGetLastError();
}

template <int FA>
hipError_t start_down(const AdapterArgs& a, unsigned grid, int rblocks, int step, hipStream_t stream)
{
    return rblocks == 1 ? start_down<FA, 1>(a, grid, step, stream) : start_down<FA, 4>(a, grid, step, stream);
}

template <int FE>
hipError_t start_up(const AdapterArgs& a, int windows, hipStream_t stream)
{
    const int blocks = a.d_out / 16, slabs = (blocks + a.slab - 1) / a.slab;
    const size_t lds = (size_t)(a.M <= 16 ? 16 : WINDOW) * (a.r + 4) * 4;
    const auto kern = up_kernel<FE>;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    kern<<<(unsigned)(windows * a.leaders) * slabs, THREADS, lds, stream>>>(a, slabs);
    return hipGetLastError();
}

}  // namespace

size_t adapters_workspace_bytes(int M, int d_in, int d_out, int r) { return (size_t)MAX_KSPLIT * M * r * sizeof(float); }

hipError_t launch_adapters(AdapterArgs args, int fa, int fe, hipStream_t stream)
{
    constexpr int LAUNCH = 1 << 16;                       // rows of a launch
    for (int m0 = 0; m0 < args.M; m0 += LAUNCH) {
        AdapterArgs a = args;
        a.M = args.M - m0 < LAUNCH ? args.M - m0 : LAUNCH;
        a.x += (size_t)m0 * a.d_in;
        a.ids += m0;
        a.y += (size_t)m0 * a.d_out;
        if (a.base) a.base += (size_t)m0 * a.d_out;
        const int windows = (a.M + WINDOW - 1) / WINDOW, chunks = a.d_in / 128, nr = a.r / 16;
        // a workgroup for each row that may lead; where there are many windows (prompts) few rows lead
        a.leaders = windows == 1 ? a.M : (windows <= 8 ? WINDOW : 4);
        const int groups = windows * (windows <= 8 ? a.leaders : 1);
        int rblocks = groups * ((nr + 3) / 4) * (chunks < 16 ? 1 : 4) >= 256 && nr >= 4 ? 4 : 1;
        a.rgroups = (nr + rblocks - 1) / rblocks;
        a.ksplit = 1;
        while (a.ksplit < MAX_KSPLIT && a.ksplit * 2 * NW <= chunks && groups * a.rgroups * a.ksplit < 512) a.ksplit *= 2;
        const int step = fe == S_F16 ? 32 : (fe == S_Q4S64 ? 64 : 128);
        const unsigned grid = (unsigned)(windows * a.leaders) * a.rgroups * a.ksplit;
        hipError_t e = fa == S_F16 ? start_down<S_F16>(a, grid, rblocks, step, stream)
                                   : (fa == S_Q4S128 ? start_down<S_Q4S128>(a, grid, rblocks, step, stream) : start_down<S_Q3S128>(a, grid, rblocks, step, stream));
        if (e != hipSuccess) return e;
        // slabs of outputs: enough workgroups to fill the chip, two row blocks a wavefront at least
        const int blocks = a.d_out / 16;
        int slabs = (1024 + groups - 1) / groups;
        a.slab = (blocks + slabs - 1) / slabs;
        a.slab = a.slab < 2 * NW ? 2 * NW : (a.slab + 2 * NW - 1) / (2 * NW) * (2 * NW);
        e = fe == S_F16 ? start_up<S_F16>(a, windows, stream)
                        : (fe == S_Q4S64 ? start_up<S_Q4S64>(a, windows, stream)
                                         : (fe == S_Q4S128 ? start_up<S_Q4S128>(a, windows, stream) : start_up<S_Q3S128>(a, windows, stream)));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace eora
