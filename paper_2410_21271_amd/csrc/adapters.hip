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

// The pairs of a window, one after the other: calls work(id, rows, first) for those that are `mine`.  With a workgroup for each row that may lead,
// the one whose row leads; else the leaders are counted.
template <typename F>
__device__ __forceinline__ void for_pairs(const AdapterArgs& a, int ids, int mine, F work)
{
    if (a.leaders >= WINDOW || a.leaders >= a.M) {
        const int id = __builtin_amdgcn_readlane(ids, mine);
        const unsigned long long rows = __ballot(ids == id);
        if (id != -2 && !(rows & ((1ull << mine) - 1))) work(id, rows);
        return;
    }
    int k = 0;
    for (unsigned long long left = __ballot(ids != -2); left;) {
        const int id = __builtin_amdgcn_readlane(ids, __ffsll(left) - 1);
        const unsigned long long rows = __ballot(ids == id);
        left &= ~rows;
        if (k++ % a.leaders == mine) work(id, rows);
    }
}

// list[s] = place (in the window) of the s-th of the rows in `rows`; one list a wavefront
__device__ __forceinline__ void list_rows(unsigned long long rows, int lane, int* list)
{
    if (rows >> lane & 1) list[__popcll(rows & ((1ull << lane) - 1))] = lane;
}

// Wavefronts of a workgroup: `blocks` of them (1, 2 or 4) have a block of 16 rows each, the others share their work
__device__ __forceinline__ int row_blocks(int count) { return count <= 16 ? 1 : (count <= 32 ? 2 : 4); }

// First launch.  A workgroup: 16 RB ranks of the leaders' pairs x one range of the contraction, in chunks of 128 columns.
template <int FA, int RB>
struct Chunk {
    static constexpr int WORDS = Fmt<FA>::WORDS, TPC = 128 / Fmt<FA>::KT;        // tiles of a chunk
    uint32_t w[RB][TPC][WORDS];
    _Float16 sc[RB];
    h8 x[4];
};

template <int FA, int RB>
__global__ __launch_bounds__(THREADS, 2) void down_kernel(const AdapterArgs a, int step)
{
    constexpr int WORDS = Fmt<FA>::WORDS, KT = Fmt<FA>::KT, TPC = 128 / KT;
    __shared__ int lists[NW][WINDOW];
    __shared__ __attribute__((aligned(16))) float red[NW * RB * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, j = lane >> 4;
    int at = blockIdx.x;
    const int rg = at % a.rgroups;
    at /= a.rgroups;
    const int ks = at % a.ksplit;
    at /= a.ksplit;
    const int row0 = at / a.leaders * WINDOW;
    int* list = lists[wave];
    const int chunks = a.d_in / 128, c0 = chunks * ks / a.ksplit, c1 = chunks * (ks + 1) / a.ksplit, rb0 = rg * RB;
    const int ids = adapter_of(a, row0, lane);
    for_pairs(a, ids, at % a.leaders, [&](int id, unsigned long long rows) {
        if (id < 0) return;
        const int rank = rank_of(a, id, step), count = __popcll(rows);
        if (16 * rb0 >= rank) return;
        const int blocks = rank / 16 - rb0 < RB ? rank / 16 - rb0 : RB;
        const int tbs = row_blocks(count), phases = NW / tbs, tb = wave % tbs, phase = wave / tbs;
        list_rows(rows, lane, list);
        const int s = 16 * tb + n;
        const _Float16* px = a.x + (size_t)(row0 + list[s < count ? s : 0]) * a.d_in;
        const uint32_t* tiles = (const uint32_t*)a.A + (size_t)id * a.r * a.d_in / KT * (64 * WORDS / 16) + (size_t)lane * WORDS;
        auto load = [&](Chunk<FA, RB>& k, int c) {
#pragma unroll
            for (int q = 0; q < RB; ++q) {
                const int rb = rb0 + (q < blocks ? q : 0);               // (blocks beyond the rank read the first one again and are not stored)
#pragma unroll
                for (int t = 0; t < TPC; ++t) load_words<WORDS>(k.w[q][t], tiles + ((size_t)rb * (a.d_in / KT) + (size_t)c * TPC + t) * (64 * WORDS));
                if constexpr (FA != S_F16) k.sc[q] = a.A_scales[((size_t)id * a.r + 16 * rb + n) * chunks + c];
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) k.x[t] = *(const h8*)(px + 128 * c + (FA == S_F16 ? 32 * t + 8 * j : 32 * j + 8 * t));
        };
        f4 acc[RB];
#pragma unroll
        for (int q = 0; q < RB; ++q) acc[q] = f4{0.f, 0.f, 0.f, 0.f};
        auto add = [&](const Chunk<FA, RB>& k) {
#pragma unroll
            for (int q = 0; q < RB; ++q) {
                h8 f[4];
                if constexpr (FA == S_F16) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        Frag g;
#pragma unroll
                        for (int u = 0; u < 4; ++u) g.u[u] = k.w[q][t][u];
                        f[t] = g.v;
                    }
#pragma unroll
                    for (int t = 0; t < 4; ++t) acc[q] = mfma16(k.x[t], f[t], acc[q]);
                } else {
                    decode_tile<FA>(k.w[q][0], 8u, f);
                    f4 part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int t = 0; t < 4; ++t) part = mfma16(k.x[t], f[t], part);
                    acc[q] += (float)k.sc[q] * part;
                }
            }
        };
        // two chunks at a time in registers; no request behind a branch
        const int mine = c1 - c0 > phase ? (c1 - c0 - phase + phases - 1) / phases : 0, first = c0 + phase;
        if (mine > 0) {
            Chunk<FA, RB> even, odd;
            load(even, first);
            int i = 0;
            for (; i + 2 < mine; i += 2) {
                load(odd, first + (i + 1) * phases);
                add(even);
                load(even, first + (i + 2) * phases);
                add(odd);
            }
            if (i + 1 < mine) {
                load(odd, first + (i + 1) * phases);
                add(even);
                add(odd);
            } else {
                add(even);
            }
        }
        if (phases == 1) {
#pragma unroll
            for (int q = 0; q < RB; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int slot = 16 * tb + 4 * j + i;
                    if (slot < count && q < blocks) a.t[((size_t)ks * a.M + row0 + list[slot]) * a.r + 16 * (rb0 + q) + n] = acc[q][i];
                }
            return;
        }
        // sum over the wavefronts of a block of rows, in order
        __syncthreads();                                  // (the last pair's sums have been read)
#pragma unroll
        for (int q = 0; q < RB; ++q) *(f4*)(red + ((wave * RB + q) * 64 + lane) * 4) = acc[q];
        __syncthreads();
        for (int e = threadIdx.x; e < tbs * RB * 256; e += THREADS) {
            // consecutive threads: consecutive ranks of one row
            const int col = e % 16, q = e / 16 % RB, slot = e / (16 * RB), b = slot / 16, l = 16 * (slot % 16 / 4) + col, i = slot % 4;
            if (slot >= count || q >= blocks) continue;
            float sum = 0.f;
            for (int p = 0; p < phases; ++p) sum += red[(((p * tbs + b) * RB + q) * 64 + l) * 4 + i];
            a.t[((size_t)ks * a.M + row0 + list[slot]) * a.r + 16 * (rb0 + q) + col] = sum;
        }
    });
}

// Second launch.  A workgroup: the leaders' rows x a slab of outputs.  A wavefront keeps t of its 16 rows in registers, as the second operand (NK fragments of 32 ranks, high
// and low halves), and takes 16 PB outputs at a time: B's tiles are the first operand.  The products pass through LDS (a part of its own for each
// wavefront, no barrier) so that base and y are moved 16 bytes a lane, consecutive lanes along a row: straight from the products' registers they are 16 rows an instruction, 64
// accesses of the L1 instead of 16 (2048 rows, 4096 -> 14336, rank 128: 131 us this launch, 38 now).
template <int FE, int NK>
__global__ __launch_bounds__(THREADS, NK <= 8 ? 2 : 1) void up_kernel(const AdapterArgs a, int slabs)
{
    constexpr int WORDS = Fmt<FE>::WORDS, KT = Fmt<FE>::KT, NF = KT / 32, TILES = NK / NF;
    constexpr int PB = NK <= 4 || (FE != S_F16 && NK <= 8) ? 4 : 2;       // blocks of 16 outputs at a time
    constexpr int LPR = 2 * PB, RPI = 64 / LPR, INS = (16 + RPI - 1) / RPI;      // lanes of a row, rows of an instruction, instructions
    constexpr int LD = 16 * PB + 4;
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    __shared__ int lists[NW][WINDOW];
    __shared__ __attribute__((aligned(16))) float turn[NW][16 * LD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, j = lane >> 4;
    int at = blockIdx.x;
    const int slab = at % slabs;
    at /= slabs;
    const int row0 = at / a.leaders * WINDOW;
    int* list = lists[wave];
    float* mine = turn[wave];
    const int ids = adapter_of(a, row0, lane);
    for_pairs(a, ids, at % a.leaders, [&](int id, unsigned long long rows) {
        const int rank = rank_of(a, id, KT), count = __popcll(rows), ntk = a.r / KT, nt = rank / KT;
        if (rank == 0 && a.base == a.y) return;           // nothing to add
        const int tbs = row_blocks(count), phases = NW / tbs, tb = wave % tbs, phase = wave / tbs, here = count - 16 * tb < 16 ? count - 16 * tb : 16;
        list_rows(rows, lane, list);
        const bool live = n < here;
        const size_t row = (size_t)(row0 + list[live ? 16 * tb + n : 0]);
        const int blocks = a.d_out / 16, end = (slab + 1) * a.slab < blocks ? (slab + 1) * a.slab : blocks;
        int rb = slab * a.slab + PB * phase;
        if (rb >= end || here <= 0) return;
        // the rows that this lane moves
        const int piece = lane % LPR;
        size_t moved[INS];
#pragma unroll
        for (int i = 0; i < INS; ++i) {
            const int r = lane / LPR + RPI * i;
            moved[i] = (size_t)(row0 + list[r < here ? 16 * tb + r : 0]) * a.d_out;
        }

        uint32_t w[PB][TILES][WORDS];
        h4 sc[PB][TILES];                                 // of rows 4 j .. 4 j + 3, TILES tiles each
        h8 base[INS];
        const _Float16* from = a.base ? a.base : a.y;     // (requested either way: no branch around a request)
        const uint32_t* tiles = (const uint32_t*)a.B + (id < 0 ? 0 : (size_t)id * a.d_out * a.r / KT * (64 * WORDS / 16)) + (size_t)lane * WORDS;
        auto load = [&](int first) {
#pragma unroll
            for (int p = 0; p < PB; ++p) {
                const int R = first + p < end ? first + p : end - 1;
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    const size_t tile = (size_t)R * ntk + (t < nt ? t : (nt ? nt - 1 : 0));     // (beyond the rank: the last tile again, times zeros)
                    load_words<WORDS>(w[p][t], tiles + tile * (64 * WORDS));
                }
                if constexpr (FE != S_F16) {
                    const _Float16* src = a.B_scales + ((size_t)(id < 0 ? 0 : id) * a.d_out + 16 * R + 4 * j) * TILES;
#pragma unroll
                    for (int t = 0; t < TILES; ++t) sc[p][t] = *(const h4*)(src + 4 * t);
                }
            }
            const int c = 16 * first + 8 * piece, last = 16 * end - 8;
#pragma unroll
            for (int i = 0; i < INS; ++i) base[i] = *(const h8*)(from + moved[i] + (c < last ? c : last));
        };
        load(rb);

        // t of this lane's row, its k-slots: sums of the ranges in order
        float t[NK][8];
        float big = 0.f;
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) t[k][e] = 0.f;
        constexpr int ROUND = NK <= 4 ? 2 : 1;            // ranges requested at a time
#pragma clang loop unroll(disable)
        for (int k0 = 0; k0 < a.ksplit; k0 += ROUND) {
            f4 in[ROUND][NK][2];
#pragma unroll
            for (int q = 0; q < ROUND; ++q) {
                const float* src = a.t + ((size_t)(k0 + q < a.ksplit ? k0 + q : k0) * a.M + row) * a.r + KT / 4 * j;
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    const float* at = src + (k / NF < nt ? k / NF * KT : 0) + 8 * (k % NF);
                    in[q][k][0] = *(const f4*)at;
                    in[q][k][1] = *(const f4*)(at + 4);
                }
            }
#pragma unroll
            for (int q = 0; q < ROUND; ++q)
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    const bool there = live && k / NF < nt && k0 + q < a.ksplit;
#pragma unroll
                    for (int e = 0; e < 8; ++e) t[k][e] += there ? in[q][k][e / 4][e % 4] : 0.f;
                }
        }
        const float scaling = a.scalings && id >= 0 ? a.scalings[id] : 1.f;
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                t[k][e] *= scaling;
                big = fmaxf(big, fabsf(t[k][e]));
            }
        big = fmaxf(big, __shfl_xor(big, 16, 64));
        big = fmaxf(big, __shfl_xor(big, 32, 64));
        int ex = (int)(__float_as_uint(big) >> 23) - 127; // exponent of the row's largest value
        ex = big == 0.f ? 8 : (ex < -110 ? -110 : (ex > 127 ? 127 : ex));
        const float to = __uint_as_float((unsigned)(127 + 8 - ex) << 23), back = rank ? __uint_as_float((unsigned)(127 - 8 + ex) << 23) : 0.f;
        h8 high[NK], low[NK];
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = t[k][e] * to;
                high[k][e] = (_Float16)v;
                low[k][e] = (_Float16)(fabsf(v) == INFINITY ? 0.f : v - (float)high[k][e]);
            }

        for (;;) {
#pragma unroll
            for (int p = 0; p < PB; ++p) {
                f4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int q = 0; q < TILES; ++q) {
                    h8 f[NF];
                    decode_tile<FE>(w[p][q], 8u, f);
                    f4 part = {0.f, 0.f, 0.f, 0.f};
                    f4& sum = FE == S_F16 ? acc : part;
#pragma unroll
                    for (int i = 0; i < NF; ++i) {
                        sum = mfma16(f[i], high[q * NF + i], sum);
                        sum = mfma16(f[i], low[q * NF + i], sum);
                    }
                    if constexpr (FE != S_F16) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[i] += (float)sc[p][(i * TILES + q) / 4][(i * TILES + q) % 4] * part[i];
                    }
                }
                // (without a pair the tiles are another's: whatever they give, nothing is added)
                *(f4*)(mine + n * LD + 16 * p + 4 * j) = rank ? acc * back : f4{0.f, 0.f, 0.f, 0.f};
            }
            h8 y[INS];
#pragma unroll
            for (int i = 0; i < INS; ++i) {
                const float* src = mine + (lane / LPR + RPI * i) * LD + 8 * piece;
                const f4 lo = *(const f4*)src, hi = *(const f4*)(src + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[i][e] = (_Float16)((a.base ? (float)base[i][e] : 0.f) + (e < 4 ? lo[e] : hi[e - 4]));
            }
            const int col = 16 * rb + 8 * piece;
            rb += PB * phases;
            const bool more = rb < end;
            if (more) load(rb);
#pragma unroll
            for (int i = 0; i < INS; ++i)
                if (lane / LPR + RPI * i < here && col < 16 * end) *(h8*)(a.y + moved[i] + col) = y[i];
            if (!more) break;
        }
    });
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

template <int FE, int NK>
hipError_t start_up(const AdapterArgs& a, int windows, hipStream_t stream)
{
    const int slabs = (a.d_out / 16 + a.slab - 1) / a.slab;
    up_kernel<FE, NK><<<(unsigned)(windows * a.leaders) * slabs, THREADS, 0, stream>>>(a, slabs);
    return hipGetLastError();
}

template <int FE>
hipError_t start_up(const AdapterArgs& a, int windows, hipStream_t stream)
{
    if constexpr (FE == S_Q4S64) {
        return start_up<FE, 2>(a, windows, stream);
    } else {
        if (a.r <= 128) return start_up<FE, 4>(a, windows, stream);
        if (a.r <= 256) return start_up<FE, 8>(a, windows, stream);
        return a.r <= 384 ? start_up<FE, 12>(a, windows, stream) : start_up<FE, 16>(a, windows, stream);
    }
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
        a.leaders = windows == 1 ? a.M : (windows <= 8 ? WINDOW : 2);
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
        // slabs of outputs: enough workgroups to fill the chip, a step of each wavefront at least
        const int blocks = a.d_out / 16, least = (a.r <= 128 || (fe != S_F16 && a.r <= 256) ? 4 : 2) * NW;
        int slabs = (512 + groups - 1) / groups;
        if (windows > 8) slabs = (slabs + 7) / 8 * 8;     // slab s of every window then runs on the same XCD, whose L2 keeps its tiles
        a.slab = (blocks + slabs - 1) / slabs;
        a.slab = windows > 8 ? (a.slab + 3) / 4 * 4 : (a.slab + least - 1) / least * least;
        e = fe == S_F16 ? start_up<S_F16>(a, windows, stream)
                        : (fe == S_Q4S64 ? start_up<S_Q4S64>(a, windows, stream)
                                         : (fe == S_Q4S128 ? start_up<S_Q4S128>(a, windows, stream) : start_up<S_Q3S128>(a, windows, stream)));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace eora
