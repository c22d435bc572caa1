// Low-rank pairs of many requests beside a shared projection:
//
//      y[m] = base[m] + s_a (x[m] A_a^T) B_a^T            a = adapter of row m, from a pool of any size
//
// Two parts: t = x A^T (fp32 partial sums of ranges of the contraction), then y from t and B.  One launch for up to 64 rows, where each of two would be half the time
// (1 row 1024 -> 1024, rank 64: 7.2 us in one, 9.8 in two; 64 of 256 pairs 4096 -> 4096, rank 128: 20.3, 22.3), two beyond.  Only the pairs that rows select are read, in the stored tiles of the layer kernels.
//
// Bound by memory at a few rows per pair (4 r flops a row against 2 bytes of a factor's element): the rows of a pair are the 16 columns (or rows)
// of the matrix instructions, mostly empty, and a wavefront's work is to keep tiles in flight (64 requests, 4096 -> 4096, rank 128: 76 MB in 20.3 us).  With many rows of one pair, y's
// own traffic bounds it (2048 rows, 4096 -> 14336: 158 MB in 68 us).
//
// Rows by pairs: below 512 rows without sorting, in windows of 64 rows, an adapter index a lane; as many ballots as an index has bits give each lane the rows of its pair, and
// the first row of each pair (its leader) its place among the window's pairs.  Every window has the same number of workgroups, which share its pairs out:
// a pair's work is cut into as many parts as there are workgroups for it.  So long runs of one pair (prompts) and a pair for each row (a batch of decoding requests) both fill the chip.
// From 512 rows on they are put in the order of their pairs first (see Order).
//
// t is not rounded to fp16: each row's t is scaled by a power of two to a largest value in [256, 512) and split in two fp16 (20.7 bits, whatever the
// size of t), both are multiplied with B's tile, and the sum is scaled back in fp32.  The first is cut off from a little below, so that both have t's sign: an infinite
// element of B then gives an infinity, which halves of zero or of two signs would make a NaN.  y is rounded once.
#include "serving.hpp"
#include "segments.hpp"

#include <type_traits>

namespace eora {
namespace {

constexpr int NW = 4, THREADS = 64 * NW;
constexpr int WINDOW = 64;

// A window's rows: lane's adapter (-1: none), the rows of the same one, and the first row of each
struct Window {
    int row0, id;
    unsigned long long same, leaders;
};
__device__ __forceinline__ Window window_of(const AdapterArgs& a, int row0, bool with_none)
{
    const int lane = threadIdx.x & 63, row = row0 + lane;
    const bool there = row < a.M;
    Window w;
    w.row0 = row0;
    w.id = there ? a.ids[row] : -1;
    w.id = (unsigned)w.id < (unsigned)a.n ? w.id : -1;
    w.same = __ballot(there);
    const unsigned key = (unsigned)(w.id + 1);             // 0 .. n
    for (int bit = 0; bit < 32 - __clz(a.n); ++bit) {
        const unsigned long long ones = __ballot(key >> bit & 1);
        w.same &= key >> bit & 1 ? ones : ~ones;
    }
    w.leaders = __ballot(there && (with_none || w.id >= 0) && !(w.same & ((1ull << lane) - 1)));
    return w;
}
// row of the p-th leader
__device__ __forceinline__ int leader_at(const Window& w, int p)
{
    const int lane = threadIdx.x & 63;
    return __ffsll(__ballot((w.leaders >> lane & 1) && __popcll(w.leaders & ((1ull << lane) - 1)) == p)) - 1;
}
__device__ __forceinline__ unsigned long long rows_at(const Window& w, int first)
{
    const unsigned lo = __builtin_amdgcn_readlane((unsigned)w.same, first), hi = __builtin_amdgcn_readlane((unsigned)(w.same >> 32), first);
    return (unsigned long long)hi << 32 | lo;
}

// Ranges of the contraction in the first part, for a window with so many pairs: as many as there are workgroups for, of a chunk a wavefront at least, and four at most where
// pairs have more than a few rows (the second part reads the parts of t of every row once a slab).
constexpr int MAX_KSPLIT = 8;
__device__ __forceinline__ int ranges_of(const AdapterArgs& a, int pairs)
{
    const int rows = a.M < WINDOW ? a.M : WINDOW, most = rows > 8 * pairs ? MAX_KSPLIT / 2 : MAX_KSPLIT;
    int ks = 1;
    while (2 * ks <= most && 2 * ks * NW <= a.d_in / 128 && 2 * ks * pairs * a.rgroups <= a.down_wgs) ks *= 2;
    return ks;
}

// Both parts in one launch, for up to a window of rows: the workgroups of the second part request their first tiles of B and then wait for t, which the first part
// (lower indices, and it never waits) hands over past the caches of an XCD, eight bytes at a time (relaxed, agent scope), with a count of its finished units for each pair (at the
// pair's first row).  The last wavefront to have read a pair's t clears its counts.
constexpr int READY = 64, TAKEN = 1, LINE = 32, HEADER = READY + LINE * WINDOW;       // words before t (word HDR_ERROR: a wait expired); a pair's two counts in a line of their own
__device__ __forceinline__ void put_t(float* p, float x, float y)
{
    const unsigned long long v = (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x);
    __hip_atomic_store((unsigned long long*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_t(const float* p)
{
    const unsigned long long v = __hip_atomic_load((const unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}
__device__ __forceinline__ unsigned add_one(unsigned* p) { return __hip_atomic_fetch_add(p, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// rank of a pair in whole k-tiles of B
__device__ __forceinline__ int rank_of(const AdapterArgs& a, int id, int step)
{
    if (id < 0) return 0;
    if (!a.ranks) return a.r;
    const int v = a.ranks[id];
    const int up = v <= 0 ? 0 : (v + step - 1) / step * step;
    return v > a.r || up > a.r ? a.r : up;
}

// list[s] = place (in the window) of the s-th of the rows in `rows`; one list a wavefront
__device__ __forceinline__ void list_rows(unsigned long long rows, int lane, int* list)
{
    if (rows >> lane & 1) list[__popcll(rows & ((1ull << lane) - 1))] = lane;
}

// Wavefronts of a workgroup: `blocks` of them (1, 2 or 4) have a block of 16 rows each, the others share their work
__device__ __forceinline__ int row_blocks(int count) { return count <= 16 ? 1 : (count <= 32 ? 2 : 4); }

// First part.  A workgroup: 16 RB ranks of the rows of a pair x one range of the contraction, in chunks of 128 columns.  x passes through LDS (a part of its own for each
// wavefront) so that its rows are read 256 bytes at a time.
template <int FA, int RB>
struct Chunk {
    static constexpr int WORDS = Fmt<FA>::WORDS, TPC = 128 / Fmt<FA>::KT;        // tiles of a chunk
    uint32_t w[RB][TPC][WORDS];
    _Float16 sc[RB];
    h8 x[4];
};

template <int RB>
struct DownSpace {
    static constexpr int XLD = 128 + 8;
    int lists[NW][WINDOW];
    __attribute__((aligned(16))) _Float16 xs[NW][16 * XLD];
    __attribute__((aligned(16))) float red[NW * RB * 256];
};

// One unit: `count` rows (row0 + list[..]) of pair id, group rg of its ranks, range ks of kss.  first_row: the pair's counts (ONE)
template <int FA, int RB, bool ONE>
struct Down {
    static constexpr int WORDS = Fmt<FA>::WORDS, KT = Fmt<FA>::KT, TPC = 128 / KT, XLD = DownSpace<RB>::XLD;
    static __device__ __forceinline__ void run(const AdapterArgs& a, int id, int rank, int row0, const int* list, int count, int rg, int ks, int kss, int first_row, DownSpace<RB>& space)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, j = lane >> 4;
        _Float16* xw = space.xs[wave];
        float* red = space.red;
        const int chunks = a.d_in / 128, c0 = chunks * ks / kss, c1 = chunks * (ks + 1) / kss, rb0 = rg * RB;
        const int blocks = rank / 16 - rb0 < RB ? rank / 16 - rb0 : RB;
        const int tbs = row_blocks(count), phases = NW / tbs, tb = wave % tbs, phase = wave / tbs;
        // the rows of x that this lane moves, 16 bytes of each
        const _Float16* px[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = 16 * tb + 4 * i + lane / 16;
            px[i] = a.x + (size_t)(row0 + list[s < count ? s : 0]) * a.d_in + 8 * n;
        }
        const uint32_t* tiles = (const uint32_t*)a.A + (size_t)id * a.r * a.d_in / KT * (64 * WORDS / 16) + (size_t)lane * WORDS;
        auto load = [&](Chunk<FA, RB>& k, int c) {
#pragma unroll
            for (int i = 0; i < 4; ++i) k.x[i] = *(const h8*)(px[i] + 128 * c);
#pragma unroll
            for (int q = 0; q < RB; ++q) {
                const int rb = rb0 + (q < blocks ? q : 0);               // (blocks beyond the rank read the first one again and are not stored)
#pragma unroll
                for (int t = 0; t < TPC; ++t) load_words<WORDS>(k.w[q][t], tiles + ((size_t)rb * (a.d_in / KT) + (size_t)c * TPC + t) * (64 * WORDS));
                if constexpr (FA != S_F16) k.sc[q] = a.A_scales[((size_t)id * a.r + 16 * rb + n) * chunks + c];
            }
        };
        f4 acc[RB];
#pragma unroll
        for (int q = 0; q < RB; ++q) acc[q] = f4{0.f, 0.f, 0.f, 0.f};
        auto add = [&](const Chunk<FA, RB>& k) {
            h8 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) *(h8*)(xw + (4 * i + lane / 16) * XLD + 8 * n) = k.x[i];
#pragma unroll
            for (int t = 0; t < 4; ++t) x[t] = *(const h8*)(xw + n * XLD + (FA == S_F16 ? 32 * t + 8 * j : 32 * j + 8 * t));
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
                    for (int t = 0; t < 4; ++t) acc[q] = mfma16(x[t], f[t], acc[q]);
                } else {
                    decode_tile<FA>(k.w[q][0], 8u, f);
                    f4 part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int t = 0; t < 4; ++t) part = mfma16(x[t], f[t], part);
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
            // (fences: the compiler would otherwise multiply first and request afterwards)
            for (; i + 2 < mine; i += 2) {
                load(odd, first + (i + 1) * phases);
                __builtin_amdgcn_sched_barrier(0);
                add(even);
                load(even, first + (i + 2) * phases);
                __builtin_amdgcn_sched_barrier(0);
                add(odd);
            }
            if (i + 1 < mine) {
                load(odd, first + (i + 1) * phases);
                __builtin_amdgcn_sched_barrier(0);
                add(even);
                add(odd);
            } else {
                add(even);
            }
        }
        if (!ONE && phases == 1) {
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
        __syncthreads();                                  // (the last unit's sums have been read)
#pragma unroll
        for (int q = 0; q < RB; ++q) *(f4*)(red + ((wave * RB + q) * 64 + lane) * 4) = acc[q];
        __syncthreads();
        for (int e = threadIdx.x; e < tbs * RB * 128; e += THREADS) {
            // consecutive threads: consecutive pairs of ranks of one row
            const int col = 2 * (e % 8), q = e / 8 % RB, slot = e / (8 * RB), b = slot / 16, l = 16 * (slot % 16 / 4) + col, i = slot % 4;
            if (slot >= count || q >= blocks) continue;
            float sum = 0.f, sum1 = 0.f;
            for (int p = 0; p < phases; ++p) {
                const float* src = red + (((p * tbs + b) * RB + q) * 64 + l) * 4 + i;
                sum += src[0];
                sum1 += src[4];
            }
            float* dst = a.t + ((size_t)ks * a.M + row0 + list[slot]) * a.r + 16 * (rb0 + q) + col;
            if constexpr (ONE) put_t(dst, sum, sum1);
            else *(float2*)dst = make_float2(sum, sum1);
        }
        if constexpr (ONE) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (threadIdx.x == 0) add_one(a.header + READY + LINE * first_row);
        }
    }
};

// Many rows: batches of up to 2048 of them in the order of their pairs (stable), cut into units of up to 64 rows of one pair.  Rows without one come first.  In the
// caller's order B is read again for each 64 rows that hold one of a pair's.  Each workgroup of the first launch finds the order itself (5 us of 256 threads; a launch of its own would
// cost as much), and one of a batch leaves it for the second.
constexpr int BATCH = 2048, NOWHERE = 2 * 4 * 64, ORDER = 4 + 4 * (BATCH + 1) + BATCH + NOWHERE;       // words of a batch in the workspace; the last are for stores of no use
struct Order {
    int keys[BATCH];                           // pair + 1, 0: none
    unsigned short rows[2][BATCH], starts[BATCH + 1];
    int digits[64 * NW];
    int sums[NW];
    int units, none;                           // units in all, without a pair
};

// sum (maximum) of v over the threads before this one; all: over all
template <bool MAX>
__device__ __forceinline__ int before_me(int v, int* sums, int& all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto join = [](int x, int y) { return MAX ? (x > y ? x : y) : x + y; };
    const int none = MAX ? -1 : 0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int w = __shfl_up(v, o, 64);
        v = join(v, lane >= o ? w : none);
    }
    if (lane == 63) sums[wave] = v;
    int mine = __shfl_up(v, 1, 64);
    if (lane == 0) mine = none;
    __syncthreads();
    all = none;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wave) mine = join(mine, sums[w]);
        all = join(all, sums[w]);
    }
    __syncthreads();
    return mine;
}

// All threads; returns the rows in order.  By up to six bits of the key at a time, lowest first.
__device__ __forceinline__ const unsigned short* order_rows(const AdapterArgs& a, int row0, int m, Order& o)
{
    static_assert(64 * NW == THREADS, "a digit's counts by wavefronts: one a thread");
    constexpr int EACH = BATCH / THREADS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = (m + THREADS - 1) / THREADS, place = wave * 64 * per + lane;         // places of a wavefront: `per` times 64
    int row[EACH], key[EACH], from = 0;
#pragma unroll
    for (int c = 0; c < EACH; ++c) {
        row[c] = place + 64 * c;
        key[c] = a.ids[row0 + (row[c] < m ? row[c] : 0)];
    }
#pragma unroll
    for (int c = 0; c < EACH; ++c) {
        key[c] = (unsigned)key[c] < (unsigned)a.n ? key[c] + 1 : 0;
        if (c < per && row[c] < m) o.keys[row[c]] = key[c];
    }
    const int bits = 32 - __clz(a.n);
    for (int shift = 0; shift < bits; shift += 6, from ^= 1) {
        const int width = bits - shift < 6 ? bits - shift : 6;
        o.digits[threadIdx.x] = 0;
        __syncthreads();
        if (shift > 0) {
#pragma unroll
            for (int c = 0; c < EACH; ++c) {
                const int p = place + 64 * c;
                row[c] = o.rows[from][p < m ? p : 0];
            }
#pragma unroll
            for (int c = 0; c < EACH; ++c) key[c] = o.keys[row[c]];
        }
        // how many of each digit; then where they go: a wavefront's counts in the order of its places
        unsigned long long same[EACH];
#pragma unroll
        for (int c = 0; c < EACH; ++c) {
            if (c >= per) break;
            const bool there = place + 64 * c < m;
            same[c] = __ballot(there);
            for (int bit = shift; bit < shift + width; ++bit) {
                const unsigned long long ones = __ballot(key[c] >> bit & 1);
                same[c] &= key[c] >> bit & 1 ? ones : ~ones;
            }
            if (there && !(same[c] & ((1ull << lane) - 1))) atomicAdd(&o.digits[(key[c] >> shift & 63) * NW + wave], __popcll(same[c]));
        }
        __syncthreads();
        int all;
        const int before = before_me<false>(o.digits[threadIdx.x], o.sums, all);
        o.digits[threadIdx.x] = before;
        __syncthreads();
        int to[EACH];
#pragma unroll
        for (int c = 0; c < EACH; ++c) {
            to[c] = 0;
            if (c < per && place + 64 * c < m && !(same[c] & ((1ull << lane) - 1))) to[c] = atomicAdd(&o.digits[(key[c] >> shift & 63) * NW + wave], __popcll(same[c]));
        }
#pragma unroll
        for (int c = 0; c < EACH; ++c) {
            if (c >= per) break;
            const int first = __shfl(to[c], __ffsll(same[c]) - 1, 64);
            if (place + 64 * c < m) o.rows[from ^ 1][first + __popcll(same[c] & ((1ull << lane) - 1))] = (unsigned short)row[c];
        }
        __syncthreads();
    }
    const unsigned short* rows = o.rows[from];
    // units: every 64 places of a run of equal keys
    int start[EACH], last = -1, all;
    const int p0 = EACH * (int)threadIdx.x, previous = o.keys[rows[p0 > 0 && p0 <= m ? p0 - 1 : 0]];
#pragma unroll
    for (int e = 0; e < EACH; ++e) row[e] = rows[p0 + e < m ? p0 + e : 0];
#pragma unroll
    for (int e = 0; e < EACH; ++e) key[e] = o.keys[row[e]];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int p = p0 + e;
        if (p < m && (p == 0 || key[e] != (e ? key[e ? e - 1 : 0] : previous))) last = p;
        start[e] = last;
    }
    const int run = before_me<true>(last, o.sums, all);
    int count = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int p = p0 + e;
        start[e] = p < m && ((p - (start[e] < 0 ? run : start[e])) & 63) == 0;
        count += start[e] ? (key[e] ? 1 : 1 + (1 << 16)) : 0;
    }
    int at = before_me<false>(count, o.sums, all) & 0xffff;
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        if (start[e]) o.starts[at++] = (unsigned short)(p0 + e);
    if (threadIdx.x == 0) {
        o.units = all & 0xffff;
        o.none = all >> 16;
        o.starts[all & 0xffff] = (unsigned short)m;
    }
    __syncthreads();
    return rows;
}

// Work of a unit in the second launch: up to 16 rows, which all wavefronts have, or a block for each
__device__ __forceinline__ int weight_of(int count) { return count > 16 ? 4 : 1; }

// For the second launch: units and units without a pair, then of each unit its first place, the weights before it and its pair, then the rows in order
__device__ __forceinline__ void leave_order(const AdapterArgs& a, int batch, int m, const Order& order, const unsigned short* rows, int* sums)
{
    int* to = a.order + (size_t)batch * ORDER;
    constexpr int EACH = BATCH / THREADS;
    int weight = 0, all;
    for (int e = 0; e < EACH; ++e) {
        const int u = EACH * (int)threadIdx.x + e;
        if (u < order.units) weight += weight_of(order.starts[u + 1] - order.starts[u]);
    }
    int before = before_me<false>(weight, sums, all);
    for (int e = 0; e < EACH; ++e) {
        const int u = EACH * (int)threadIdx.x + e;
        if (u >= order.units) break;
        const int first = order.starts[u];
        ((int4*)to)[1 + u] = make_int4(first, before, order.keys[rows[first]] - 1, 0);
        before += weight_of(order.starts[u + 1] - first);
    }
    if (threadIdx.x == 0) {
        ((int4*)to)[0] = make_int4(order.units, order.none, 0, 0);
        ((int4*)to)[1 + order.units] = make_int4(m, all, -1, 0);
    }
    for (int e = threadIdx.x; e < m; e += THREADS) to[4 + 4 * (BATCH + 1) + e] = rows[e];
}
// ranges of the contraction where a batch has so many units with a pair
__device__ __forceinline__ int ranges_of_batch(const AdapterArgs& a, int m, int units)
{
    const int most = m > 8 * units ? MAX_KSPLIT / 2 : MAX_KSPLIT, fair = units ? a.down_wgs / (units * a.rgroups) : 1, chunks = a.d_in / 128 / NW;
    const int ks = fair < most ? fair : most;
    return ks <= 1 ? 1 : (ks < chunks ? ks : (chunks < 1 ? 1 : chunks));
}

template <int FA, int RB>
__global__ __launch_bounds__(THREADS, 1) void down_ordered_kernel(const AdapterArgs a, int step)
{
    __shared__ DownSpace<RB> space;
    __shared__ Order order;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int batch = blockIdx.x / a.down_wgs, g = blockIdx.x - batch * a.down_wgs, row0 = batch * BATCH, m = a.M - row0 < BATCH ? a.M - row0 : BATCH;
    int* list = space.lists[wave];
    const unsigned short* rows = order_rows(a, row0, m, order);
    if (g == a.down_wgs - 1) leave_order(a, batch, m, order, rows, order.sums);        // (often one without a unit)
    const int none = order.none, kss = ranges_of_batch(a, m, order.units - none), slices = a.rgroups * kss;
    for (int unit = g; unit < (order.units - none) * slices; unit += a.down_wgs) {
        const int u = none + unit / slices, slice = unit % slices, rg = slice % a.rgroups;
        const int first = __builtin_amdgcn_readfirstlane(order.starts[u]), count = __builtin_amdgcn_readfirstlane(order.starts[u + 1]) - first;
        const int id = __builtin_amdgcn_readfirstlane(order.keys[rows[first]]) - 1, rank = rank_of(a, id, step);
        if (16 * RB * rg >= rank) continue;
        list[lane] = rows[first + (lane < count ? lane : 0)];
        Down<FA, RB, false>::run(a, id, rank, row0, list, count, rg, slice / a.rgroups, kss, 0, space);
    }
}

// Rows in the caller's order: workgroup g of the a.down_wgs of a window
template <int FA, int RB, bool ONE>
__device__ __forceinline__ void down_window(const AdapterArgs& a, int step, int window, int g, DownSpace<RB>& space)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int* list = space.lists[wave];
    const Window win = window_of(a, window * WINDOW, false);
    const int pairs = __popcll(win.leaders), kss = ranges_of(a, pairs);
    for (int unit = g; unit < pairs * a.rgroups * kss; unit += a.down_wgs) {
        const int rg = unit % a.rgroups, ks = unit / a.rgroups % kss, first_row = leader_at(win, unit / (a.rgroups * kss));
        const int id = __builtin_amdgcn_readlane(win.id, first_row);
        const unsigned long long rows = rows_at(win, first_row);
        const int rank = rank_of(a, id, step);
        if (16 * RB * rg >= rank) continue;
        list_rows(rows, lane, list);
        Down<FA, RB, ONE>::run(a, id, rank, win.row0, list, __popcll(rows), rg, ks, kss, first_row, space);
    }
}

template <int FA, int RB>
__global__ __launch_bounds__(THREADS, 1) void down_kernel(const AdapterArgs a, int step)
{
    __shared__ DownSpace<RB> space;
    const int window = blockIdx.x / a.down_wgs;
    down_window<FA, RB, false>(a, step, window, blockIdx.x - window * a.down_wgs, space);
}

// Waits for, and gives up, t of the pair that row `first` leads; need: the units that make it up, readers: the wavefronts that read it
struct Wait {
    int first;
    unsigned need, readers;
    __device__ __forceinline__ void ready(const AdapterArgs& a) const
    {
        bool there = need == 0;
        for (int spins = 0; !there && spins <= a.spin_limit; ++spins) {
            unsigned v = 0;
            if ((threadIdx.x & 63) == 0) v = ld_relaxed(a.header + READY + LINE * first);
            there = (unsigned)__builtin_amdgcn_readfirstlane(v) >= need;
            if (!there) __builtin_amdgcn_s_sleep(20);        // (looking more often delays the counting: 1 row 4096 -> 14336 13.5 us with 2, 10.2)
        }
        if (!there && (threadIdx.x & 63) == 0) __hip_atomic_store(a.header + HDR_ERROR, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("" ::: "memory");                    // nothing of t is requested before
    }
    __device__ __forceinline__ void taken(const AdapterArgs& a) const
    {
        if (need == 0 || (threadIdx.x & 63) != 0) return;
        asm volatile("" ::: "memory");
        unsigned* counts = a.header + READY + LINE * first;
        if (add_one(counts + TAKEN) + 1 < readers) return;
        __hip_atomic_store(counts, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(counts + TAKEN, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
};

// Second part.  A workgroup: the leaders' rows x a slab of outputs.  A wavefront keeps t of its 16 rows in registers, as the second operand (NK fragments of 32
// ranks, high and low halves), and takes 16 PB outputs at a time: B's tiles are the first operand.  What is row-major (t on its way in, base and y) passes through LDS, a part of
// its own for each wavefront and no barrier, so that it is moved 16 bytes a lane, consecutive lanes along a row: straight to and from the operands' places it is
// 16 rows an instruction, 64 accesses of the L1 instead of 16.
//
// SHARE (rows in order): the wavefronts have a block of rows each and all outputs of the slab, so that B's tiles are requested once a workgroup, a quarter by each, and pass through LDS
// too, two steps of them (requested by every wavefront they are 470 MB from L2 for 2048 rows, 4096 -> 14336, rank 128).
template <int FE, int NK, bool SHARE, bool ONE>
struct Up {
    static constexpr int WORDS = Fmt<FE>::WORDS, KT = Fmt<FE>::KT, NF = KT / 32, TILES = NK / NF;
    static constexpr int PB = NK <= 4 || (FE != S_F16 && NK <= 8) ? 4 : 2;       // blocks of 16 outputs at a time
    static constexpr int LPR = 2 * PB, RPI = 64 / LPR, INS = (16 + RPI - 1) / RPI;       // lanes of a row, rows of an instruction, instructions of a block of rows
    static constexpr int LD = 16 * PB + 4, COLS = NK * 32 < 128 ? NK * 32 : 128, TLD = COLS + 4;
    static constexpr int LDS = 16 * (LD > TLD ? LD : TLD);                       // floats of a wavefront
    static constexpr int STEP = PB * TILES, HELD = SHARE ? (STEP + NW - 1) / NW : STEP;      // tiles of a step, of them in this wavefront's registers
    static constexpr int STAGE = SHARE ? 2 * STEP * 64 * WORDS : 1;                          // words of the workgroup
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));

    // tb: this wavefront's first block of rows; it takes every `phases`-th step of 16 PB outputs from `phase` on
    static __device__ __forceinline__ void run(const AdapterArgs& a, int id, int rank, int row0, const int* list, int count, int tb, int phase, int phases, int first_block, int end, int kss, float* mine, uint32_t* stage, const Wait& wait)
    {
        const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
        const int ntk = a.r / KT, nt = rank / KT, here = count - 16 * tb;
        int rb = first_block + PB * phase;
        if (!SHARE && (rb >= end || here <= 0)) {
            if constexpr (ONE) wait.taken(a);
            return;
        }
        const int wave = SHARE ? tb : 0;
        // The rows that this lane moves.  Lanes beyond the last row or column have the last one's, and store the same there; a wavefront without rows (SHARE) stores to where nothing
        // reads: a store behind a branch would make the next step's wait for its requests one for the stores too (2048 rows, 4096 -> 14336, 74.7 us, 72.3).
        const int piece = lane % LPR, last_row = here > 0 ? here - 1 : 0;
        size_t moved[INS];
#pragma unroll
        for (int i = 0; i < INS; ++i) {
            const int r = lane / LPR + RPI * i;
            moved[i] = (size_t)(row0 + list[here > 0 ? 16 * tb + (r < last_row ? r : last_row) : 0]) * a.d_out;
        }

        static_assert(INS <= 2, "what NOWHERE has room for");
        _Float16* const nowhere = (_Float16*)(a.order + ORDER - NOWHERE) + 8 * lane;
        uint32_t w[HELD][WORDS];
        h4 sc[PB][TILES];                                 // of rows 4 j .. 4 j + 3, TILES tiles each
        h8 base[INS];
        const _Float16* from = a.base ? a.base : a.y;     // (requested either way: no branch around a request)
        const uint32_t* tiles = (const uint32_t*)a.B + (id < 0 ? 0 : (size_t)id * a.d_out * a.r / KT * (64 * WORDS / 16)) + (size_t)lane * WORDS;
        auto load_tiles = [&](int first) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const int k = SHARE ? wave + NW * i : i, p = k / TILES, t = k % TILES, R = first + p < end ? first + p : end - 1;
                const size_t tile = (size_t)R * ntk + (t < nt ? t : (nt ? nt - 1 : 0));      // (beyond the rank: the last tile again)
                load_words<WORDS>(w[i], tiles + tile * (64 * WORDS));
            }
        };
        auto load_scales = [&](int first) {
#pragma unroll
            for (int p = 0; p < PB; ++p) {
                if constexpr (FE != S_F16) {
                    const int R = first + p < end ? first + p : end - 1;
                    const _Float16* src = a.B_scales + ((size_t)(id < 0 ? 0 : id) * a.d_out + 16 * R + 4 * j) * TILES;
#pragma unroll
                    for (int t = 0; t < TILES; ++t) sc[p][t] = *(const h4*)(src + 4 * t);
                }
            }
        };
        auto load_base = [&](int first) {
            const int c = 16 * first + 8 * piece, last = 16 * end - 8;
#pragma unroll
            for (int i = 0; i < INS; ++i) base[i] = *(const h8*)(from + moved[i] + (c < last ? c : last));
        };
        auto put_tiles = [&](int buffer) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                if (STEP % NW && wave + NW * i >= STEP) break;
                uint32_t* dst = stage + ((size_t)(buffer * STEP + wave + NW * i) * 64 + lane) * WORDS;
#pragma unroll
                for (int v = 0; v < WORDS; ++v) dst[v] = w[i][v];
            }
        };
        load_tiles(rb);
        load_scales(rb);
        if constexpr (!SHARE) load_base(rb);
        __builtin_amdgcn_sched_barrier(0);

        if constexpr (ONE) wait.ready(a);
        // t of the rows, summed over the ranges in order, COLS columns at a time
        h8 high[NK], low[NK];
        float t[NK][8], big = 0.f;
        constexpr int TL = COLS / 4, TRI = 64 / TL, TIN = 16 / TRI;              // lanes of a row, rows of an instruction, instructions
        const float scaling = a.scalings && id >= 0 ? a.scalings[id] : 1.f;
#pragma unroll
        for (int c = 0; c < NK * 32 / COLS; ++c) {
            f4 sum[TIN];
#pragma unroll
            for (int i = 0; i < TIN; ++i) sum[i] = f4{0.f, 0.f, 0.f, 0.f};
            const int col = c * COLS + 4 * (lane % TL);
            auto fetch = [&](int ks, int r) {
                const float* src = a.t + ((size_t)ks * a.M + row0 + list[r < here ? 16 * tb + r : 0]) * a.r + (col < rank ? col : 0);
                if constexpr (ONE) {
                    const float2 lo = get_t(src), hi = get_t(src + 2);
                    return f4{lo.x, lo.y, hi.x, hi.y};
                } else {
                    return *(const f4*)src;
                }
            };
            if (ONE && here <= TRI) {
                // one instruction a range: all of them at a time
                f4 in[MAX_KSPLIT];
#pragma unroll
                for (int ks = 0; ks < MAX_KSPLIT; ++ks) in[ks] = fetch(ks < kss ? ks : 0, lane / TL);
#pragma unroll
                for (int ks = 0; ks < MAX_KSPLIT; ++ks) sum[0] += ks < kss ? in[ks] : f4{0.f, 0.f, 0.f, 0.f};
            } else {
#pragma clang loop unroll(disable)
                for (int ks = 0; ks < kss; ++ks) {
                    f4 in[TIN];
#pragma unroll
                    for (int i = 0; i < TIN; ++i) in[i] = fetch(ks, lane / TL + TRI * i);
#pragma unroll
                    for (int i = 0; i < TIN; ++i) sum[i] += in[i];
                }
            }
#pragma unroll
            for (int i = 0; i < TIN; ++i) {
                const int r = lane / TL + TRI * i;
                *(f4*)(mine + r * TLD + 4 * (lane % TL)) = r < here && col < rank ? sum[i] * scaling : f4{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int k = 0; k < COLS / 32; ++k) {
                const float* src = mine + n * TLD + k / NF * KT + KT / 4 * j + 8 * (k % NF);
                const f4 lo = *(const f4*)src, hi = *(const f4*)(src + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = e < 4 ? lo[e] : hi[e - 4];
                    t[c * (COLS / 32) + k][e] = v;
                    big = fmaxf(big, fabsf(v));
                }
            }
        }
        if constexpr (ONE) wait.taken(a);                 // (t is in LDS)
        big = fmaxf(big, __shfl_xor(big, 16, 64));
        big = fmaxf(big, __shfl_xor(big, 32, 64));
        int ex = (int)(__float_as_uint(big) >> 23) - 127;  // exponent of the row's largest value
        ex = big == 0.f ? 8 : (ex < -110 ? -110 : (ex > 127 ? 127 : ex));
        const float to = __uint_as_float((unsigned)(127 + 8 - ex) << 23), below = to * (1.f - 0x1p-12f), back = rank ? __uint_as_float((unsigned)(127 - 8 + ex) << 23) : 0.f;
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const h2 cut = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(t[k][e] * below, t[k][e + 1] * below));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    high[k][e + i] = cut[i];
                    low[k][e + i] = (_Float16)fminf(t[k][e + i] * to - (float)cut[i], 512.f);        // (of an infinity 512, not NaN)
                }
            }

        if constexpr (SHARE) {
            __syncthreads();                              // (the last unit's tiles have been read)
            put_tiles(0);
            // as in every step, stores among it: what is under way at the loop's beginning in whatever order decides how little its waits may leave (72.3, 71.3)
            load_tiles(rb + PB < end ? rb + PB : rb);
            load_base(rb);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < INS; ++i) *(h8*)(nowhere + 512 * i) = h8{};
            __builtin_amdgcn_sched_barrier(0);
            __syncthreads();
        }
        for (int buffer = 0;; buffer ^= 1) {
            f4 acc[PB];
#pragma unroll
            for (int p = 0; p < PB; ++p) acc[p] = f4{0.f, 0.f, 0.f, 0.f};
            // Tiles of B behind the pair's rank are left out: with zeros of t, infinities in the tile that stands for them and scales of anything, NaN among it, would
            // make NaN.  (In a copy of the loop of their own: 2048 rows of full rank take 1 % longer with a branch for each tile.)
            auto multiply = [&](auto some) {
#pragma unroll
                for (int q = 0; q < TILES; ++q) {
                    if (decltype(some)::value && q >= nt) break;
#pragma unroll
                    for (int p = 0; p < PB; ++p) {
                        uint32_t now[WORDS];
                        if constexpr (SHARE) {
                            const uint32_t* src = stage + ((size_t)(buffer * STEP + p * TILES + q) * 64 + lane) * WORDS;
#pragma unroll
                            for (int v = 0; v < WORDS; ++v) now[v] = src[v];
                        } else {
#pragma unroll
                            for (int v = 0; v < WORDS; ++v) now[v] = w[p * TILES + q][v];
                        }
                        h8 f[NF];
                        decode_tile<FE>(now, 8u, f);
                        f4 part = {0.f, 0.f, 0.f, 0.f};
                        f4& sum = FE == S_F16 ? acc[p] : part;
#pragma unroll
                        for (int i = 0; i < NF; ++i) {
                            sum = mfma16(f[i], high[q * NF + i], sum);
                            sum = mfma16(f[i], low[q * NF + i], sum);
                        }
                        if constexpr (FE != S_F16) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[p][i] += (float)sc[p][(i * TILES + q) / 4][(i * TILES + q) % 4] * part[i];
                        }
                    }
                }
            };
            if (nt < TILES) multiply(std::true_type{});
            else multiply(std::false_type{});
            const int most = 2 * (end - rb) - 1, at = piece < most ? piece : most, col = 16 * rb + 8 * at;
            // (without a pair the tiles are another's: whatever they give, -0 is added, which leaves base as it is)
#pragma unroll
            for (int p = 0; p < PB; ++p) *(f4*)(mine + n * LD + 16 * p + 4 * j) = rank ? acc[p] * back : f4{-0.f, -0.f, -0.f, -0.f};
            h8 y[INS];
#pragma unroll
            for (int i = 0; i < INS; ++i) {
                const int r = lane / LPR + RPI * i;
                const float* src = mine + (r < last_row ? r : last_row) * LD + 8 * at;
                const f4 lo = *(const f4*)src, hi = *(const f4*)(src + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[i][e] = (_Float16)((a.base ? (float)base[i][e] : 0.f) + (e < 4 ? lo[e] : hi[e - 4]));
            }
            auto store = [&] {
#pragma unroll
                for (int i = 0; i < INS; ++i) {
                    _Float16* to = a.y + moved[i] + col;
                    if constexpr (SHARE) to = here > 0 ? to : nowhere + 512 * i;
                    // (many rows: past L2, which has B's tiles and base to hold: 2048 rows, 4096 -> 14336, 71.1 us, 68.1; 30000 rows 1024 -> 2048 118.5, 115; followed by a reader of y the
                    // same as without)
                    if constexpr (SHARE) __builtin_nontemporal_store(y[i], (h8*)to);
                    else *(h8*)to = y[i];
                }
            };
            rb += PB * phases;
            if (rb >= end) {
                store();
                break;
            }
            if constexpr (SHARE) {
                put_tiles(buffer ^ 1);
                load_tiles(rb + PB < end ? rb + PB : rb);
            } else {
                load_tiles(rb);
            }
            load_scales(rb);
            load_base(rb);
            __builtin_amdgcn_sched_barrier(0);
            store();
            if constexpr (SHARE) __syncthreads();
        }
    }
};

template <int FE, int NK, bool SHARE>
struct UpSpace {
    int lists[NW][WINDOW];
    __attribute__((aligned(16))) float space[NW][Up<FE, NK, SHARE, false>::LDS];
    __attribute__((aligned(16))) uint32_t stage[Up<FE, NK, SHARE, false>::STAGE];
};

// Rows in the caller's order: workgroup g of the a.up_wgs of a window; rb_ranks: ranks of a unit of the first part (ONE)
template <int FE, int NK, bool ONE>
__device__ __forceinline__ void up_window(const AdapterArgs& a, int window, int g, int rb_ranks, UpSpace<FE, NK, false>& s)
{
    typedef Up<FE, NK, false, ONE> Rows;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int* list = s.lists[wave];
    // (rows without a pair have nothing to add; with y apart from base they are copied)
    const Window win = window_of(a, window * WINDOW, a.base != a.y);
    const int pairs = __popcll(win.leaders), kss = ranges_of(a, __popcll(win.leaders & __ballot(win.id >= 0)));
    // slabs of outputs: as many as there are workgroups for, a step of each wavefront at least for the largest pair (with no more than a small pair has steps for: 256 rows of one
    // pair, 4096 -> 4096, 22 us, 18)
    const int rows_here = __popcll(win.same);
    const bool four = __ballot(rows_here > 32) & win.leaders, two = __ballot(rows_here > 16) & win.leaders;
    const int blocks = a.d_out / 16, steps = (blocks + Rows::PB - 1) / Rows::PB, most = four ? steps : (two ? (steps + 1) / 2 : (steps + 3) / 4);
    const int each = pairs ? a.up_wgs / pairs : 1, slabs = each < 1 ? 1 : (each < most ? each : most), size = (blocks + slabs - 1) / slabs;
    for (int unit = g; unit < pairs * slabs; unit += a.up_wgs) {
        const int slab = unit % slabs, first_row = leader_at(win, unit / slabs);
        const int id = __builtin_amdgcn_readlane(win.id, first_row);
        const unsigned long long rows = rows_at(win, first_row);
        const int rank = rank_of(a, id, Fmt<FE>::KT), count = __popcll(rows), first = slab * size, end = first + size < blocks ? first + size : blocks;
        const Wait wait{first_row, (unsigned)((rank + rb_ranks - 1) / rb_ranks * kss), (unsigned)(slabs * NW)};
        if ((rank == 0 && a.base == a.y) || (!ONE && first >= end)) continue;      // (ONE: every wavefront of a pair's units gives its t up)
        list_rows(rows, lane, list);
        const int tbs = row_blocks(count);
        Rows::run(a, id, rank, win.row0, list, count, wave % tbs, wave / tbs, NW / tbs, first, end, kss, s.space[wave], s.stage, wait);
    }
}

template <int FE, int NK>
__global__ __launch_bounds__(THREADS, NK <= 8 ? 2 : 1) void up_kernel(const AdapterArgs a)
{
    __shared__ UpSpace<FE, NK, false> space;
    const int window = blockIdx.x / a.up_wgs;
    up_window<FE, NK, false>(a, window, blockIdx.x - window * a.up_wgs, 1, space);
}

// Rows in order: the outputs are cut into up to eight column groups, one for the workgroups of each XCD (whose L2 then holds its columns of B once), and the units of a batch, as
// they follow one another, for each group into runs of equal weight: a workgroup ends one unit and begins another.
template <int FE, int NK>
__global__ __launch_bounds__(THREADS, NK <= 8 ? 2 : 1) void up_ordered_kernel(const AdapterArgs a)
{
    __shared__ UpSpace<FE, NK, true> s;
    typedef Up<FE, NK, false, false> Rows;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int batch = blockIdx.x / a.up_wgs, g = blockIdx.x - batch * a.up_wgs, row0 = batch * BATCH, m = a.M - row0 < BATCH ? a.M - row0 : BATCH;
    const int4* units = (const int4*)(a.order + (size_t)batch * ORDER) + 1;
    const int* rows = (const int*)(units + BATCH + 1);
    int* list = s.lists[wave];
    const int n_units = __builtin_amdgcn_readfirstlane(units[-1].x), none = __builtin_amdgcn_readfirstlane(units[-1].y);
    const int u0 = a.base == a.y ? none : 0;              // (rows without a pair have nothing to add; with y apart from base they are copied)
    const int kss = ranges_of_batch(a, m, n_units - none), blocks = a.d_out / 16;
    int groups = 8;
    while (groups > 1 && (groups > a.up_wgs || blocks < groups * 4 * NW * Rows::PB)) groups /= 2;
    const int per = (blocks + groups - 1) / groups, group = g % groups, first = group * per, end = first + per < blocks ? first + per : blocks;
    // a unit of weight w has w q places, of NW / w steps of PB blocks
    const int q = (per + NW * Rows::PB - 1) / (NW * Rows::PB), before = __builtin_amdgcn_readfirstlane(units[u0].y);
    const unsigned total = (unsigned)(__builtin_amdgcn_readfirstlane(units[n_units].y) - before) * (unsigned)q, n = (unsigned)(a.up_wgs / groups), i = (unsigned)(g / groups);
    if (i >= n) return;
    unsigned at = (unsigned)((unsigned long long)total * i / n);
    const unsigned stop = (unsigned)((unsigned long long)total * (i + 1) / n);
    if (at >= stop) return;
    int u = u0;
    for (int range = n_units - u0; range > 1;) {          // the last unit that begins at or before `at`
        const int stride = (range + 63) / 64, mine = u + lane * stride, past = u + range;
        const bool here = mine < past && (unsigned)(units[mine < past ? mine : past - 1].y - before) * (unsigned)q <= at;
        u += (__popcll(__ballot(here)) - 1) * stride;
        range = past - u < stride ? past - u : stride;
    }
    u = __builtin_amdgcn_readfirstlane(u);
    for (; at < stop; ++u) {
        const int4 unit = units[u], after = units[u + 1];
        const int start = __builtin_amdgcn_readfirstlane(unit.x), count = __builtin_amdgcn_readfirstlane(after.x) - start, id = __builtin_amdgcn_readfirstlane(unit.z);
        const unsigned begins = (unsigned)(__builtin_amdgcn_readfirstlane(unit.y) - before) * (unsigned)q, ends = (unsigned)(__builtin_amdgcn_readfirstlane(after.y) - before) * (unsigned)q;
        const int weight = weight_of(count), place = NW / weight * Rows::PB, from = first + (int)(at - begins) * place, to = first + (int)((stop < ends ? stop : ends) - begins) * place;
        at = ends;
        const int rank = rank_of(a, id, Fmt<FE>::KT), last = to < end ? to : end;
        if (from >= last || (rank == 0 && a.base == a.y)) continue;
        list[lane] = rows[start + (lane < count ? lane : 0)];
        const Wait wait{0, 0, 0};
        if (weight == 4) Up<FE, NK, true, false>::run(a, id, rank, row0, list, count, wave, 0, 1, from, last, kss, s.space[wave], s.stage, wait);
        else Rows::run(a, id, rank, row0, list, count, 0, wave, NW, from, last, kss, s.space[wave], s.stage, wait);
    }
}

template <int FA, int RB, int FE, int NK>
__global__ __launch_bounds__(THREADS, NK <= 8 ? 2 : 1) void adapters_kernel(const AdapterArgs a, int step)
{
    __shared__ union Space {
        DownSpace<RB> first;
        UpSpace<FE, NK, false> second;
        __device__ Space() {}
    } space;
    const int g = blockIdx.x;
    if (g < a.down_wgs) down_window<FA, RB, true>(a, step, 0, g, space.first);
    else up_window<FE, NK, true>(a, 0, g - a.down_wgs, 16 * RB, space.second);
}

// How a call goes: in one launch, in two by windows of 64 rows, in two by batches of 2048 in order.  Ordering costs 4 to 6 us and saves B's being read in every window (4096 -> 4096,
// by windows and in order: 1024 rows of 64 pairs in turn, rank 64, 83 and 31 us; rank 128, 512 rows of 16 pairs in turn 21.9 and 22.8, of one pair 18.9 and 22.0, 256 rows of 16 in turn 17.1 and
// 23.0; 8192 rows of 16 pairs in turn 280 and 84.5, in runs of 60 134 and 116, of one pair 94 and 81).  By the number of rows alone: what the indices are the host does not know.
enum Form { ONE_LAUNCH, WINDOWS, ORDERED };
constexpr int MANY = 512;                      // rows from which they are put in order

template <int FA, int RB>
hipError_t start_down(const AdapterArgs& a, Form form, unsigned grid, int step, hipStream_t stream)
{
    if (form == ORDERED) down_ordered_kernel<FA, RB><<<grid, THREADS, 0, stream>>>(a, step);
    else down_kernel<FA, RB><<<grid, THREADS, 0, stream>>>(a, step);
    return hipGetLastError();
}

template <int FA>
hipError_t start_down(const AdapterArgs& a, Form form, unsigned grid, int rblocks, int step, hipStream_t stream)
{
    if constexpr (FA == S_F16)                            // (codes have ranks of 64 or more)
        if (rblocks == 1) return start_down<FA, 1>(a, form, grid, step, stream);
    return start_down<FA, 4>(a, form, grid, step, stream);
}

template <int FE, int NK>
hipError_t start_up(const AdapterArgs& a, Form form, unsigned grid, int rblocks, int step, hipStream_t stream)
{
    if (form == ONE_LAUNCH) {
        constexpr int FA = FE == S_Q4S64 ? S_Q4S128 : FE;
        if constexpr (NK <= 4)
            if (rblocks == 1) {
                adapters_kernel<FA, 1, FE, NK><<<a.down_wgs + a.up_wgs, THREADS, 0, stream>>>(a, step);
                return hipGetLastError();
            }
        adapters_kernel<FA, 4, FE, NK><<<a.down_wgs + a.up_wgs, THREADS, 0, stream>>>(a, step);
    } else if (form == WINDOWS) {
        up_kernel<FE, NK><<<grid, THREADS, 0, stream>>>(a);
    } else {
        up_ordered_kernel<FE, NK><<<grid, THREADS, 0, stream>>>(a);
    }
    return hipGetLastError();
}

template <int FE>
hipError_t start_up(const AdapterArgs& a, Form form, unsigned grid, int rblocks, int step, hipStream_t stream)
{
    if constexpr (FE == S_Q4S64) {
        return start_up<FE, 2>(a, form, grid, rblocks, step, stream);
    } else {
        if (a.r <= 128) return start_up<FE, 4>(a, form, grid, rblocks, step, stream);
        if (a.r <= 256) return start_up<FE, 8>(a, form, grid, rblocks, step, stream);
        return a.r <= 384 ? start_up<FE, 12>(a, form, grid, rblocks, step, stream) : start_up<FE, 16>(a, form, grid, rblocks, step, stream);
    }
}

}  // namespace

size_t adapters_workspace_bytes(int M, int d_in, int d_out, int r)
{
    return (HEADER + (size_t)((M + BATCH - 1) / BATCH) * ORDER) * sizeof(uint32_t) + (size_t)MAX_KSPLIT * M * r * sizeof(float);
}

hipError_t launch_adapters(AdapterArgs args, int fa, int fe, hipStream_t stream)
{
    constexpr int LAUNCH = 1 << 16;                       // rows of a launch
    for (int m0 = 0; m0 < args.M; m0 += LAUNCH) {
        AdapterArgs a = args;
        a.M = args.M - m0 < LAUNCH ? args.M - m0 : LAUNCH;
        const Form form = a.M <= WINDOW ? ONE_LAUNCH : (a.M < MANY ? WINDOWS : ORDERED);
        const int of = form == ORDERED ? BATCH : WINDOW, parts = (a.M + of - 1) / of, nr = a.r / 16, rblocks = nr < 4 || (a.M == 1 && nr <= 8) ? 1 : 4;
        a.order = (int*)(a.header + HEADER);
        a.t = (float*)(a.order + (form == ORDERED ? (size_t)parts * ORDER : 0));
        a.x += (size_t)m0 * a.d_in;
        a.ids += m0;
        a.y += (size_t)m0 * a.d_out;
        if (a.base) a.base += (size_t)m0 * a.d_out;
        a.rgroups = (nr + rblocks - 1) / rblocks;
        const int step = fe == S_F16 ? 32 : (fe == S_Q4S64 ? 64 : 128);
        if (form == ONE_LAUNCH) {
            // one workgroup a compute unit for either part, and no more than the rows have work for
            const int down = a.M * a.rgroups * MAX_KSPLIT, up = a.M * ((a.d_out / 16 + 7) / 8);
            a.down_wgs = down < 256 ? down : 256;
            a.up_wgs = up < 256 ? up : 256;
        } else {
            // First: one workgroup a compute unit, with two chunks in its registers (two: 2048 rows 68.1 us, 71.9), but with more batches 128 each while that is no more than four a
            // compute unit (8192 rows of one pair, 4096 -> 4096, with 64 each 83.3 us, 80.7; in runs of 60 119, 116; of 16 in turn 82.1, 84.5).  Second: two.
            a.down_wgs = form == WINDOWS || parts == 1 ? 256 / parts : (parts < 8 ? 128 : 1024 / parts);
            a.up_wgs = 512 / parts;
            const unsigned grid = (unsigned)parts * a.down_wgs;
            const hipError_t e = fa == S_F16 ? start_down<S_F16>(a, form, grid, rblocks, step, stream)
                                             : (fa == S_Q4S128 ? start_down<S_Q4S128>(a, form, grid, rblocks, step, stream) : start_down<S_Q3S128>(a, form, grid, rblocks, step, stream));
            if (e != hipSuccess) return e;
        }
        const unsigned grid = (unsigned)parts * a.up_wgs;
        const hipError_t e = fe == S_F16 ? start_up<S_F16>(a, form, grid, rblocks, step, stream)
                                         : (fe == S_Q4S64 ? start_up<S_Q4S64>(a, form, grid, rblocks, step, stream)
                                                          : (fe == S_Q4S128 ? start_up<S_Q4S128>(a, form, grid, rblocks, step, stream) : start_up<S_Q3S128>(a, form, grid, rblocks, step, stream)));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace eora
