// Attention of many new tokens per request (a prompt, a piece of one, some drafted tokens) over a paged key-value cache.
//
//      s_rt = scale q_r . k_t,   out_r = sum_t 2^(s_rt log2 e - m) v_t / sum_t 2^(s_rt log2 e - m)      t <= p_r, and t > p_r - window or t < sinks
//
// Row r of a request's n sits at p_r = length - n + r.  Bound by the matrix instructions: 4 dim flops for each pair of a query head's row and a token.
//
// Tile: 128 pairs of a row and a query head of one kv head (32 a wavefront) by 64 keys.  A column of the matrix instructions is a pair, all query heads of a kv head share the keys.
// S^T = K Q^T (32 x 32 x 16): a lane holds one pair's scores of 16 keys of 32, so that softmax needs no exchange between lanes but one of the largest score, and the scores are,
// as fp16 weights, the second operand of O^T = V^T P^T, if that takes its keys in the order in which they lie: 8 (e / 4) + 4 half + e % 4 of 16.
// K and V lie in LDS as fp16 rows, in two stages; V's operand is read transposed (ds_read_tr16_b64: four keys of a column a lane).  Pieces of a row are
// moved around by the row's number, so that the lanes that read at a time meet different banks.  Codes of a cache in 8 bits become fp16, exactly, once, on their way to LDS.
//
// Two teams of four wavefronts work on the same 128 pairs, on every other tile of keys, and add up in LDS at the end: so there is one unit a compute unit at a time, of all its
// wavefronts, and units in the order of falling work even out.  (Heads of 256: one team.)
//
// Softmax: as for single tokens, m is a reference (LOWER below the largest score when it is set, raised when a score has risen by RAISE more), the largest weight 2^11 to 2^15.  A weight meets
// V as one fp16, rounded to nearest: off by 2^-12 of itself at most, which in a sum over tokens stays below the result's own rounding; two of them, as for single
// tokens, would take half as long again.  Scores, sums and O are fp32.
//
// What rows may not see: a tile that all rows of a wavefront see as a whole takes no test.  Tokens that no row of the tile sees are zeros in LDS; where some rows see a token and others do not, a value
// that is not finite would spoil a product with weights of 0: then the tile takes a slower way, in which such values are added to the rows that see them one by one.
//
// Split: tiles with more than their share of all work are cut along the keys, into equal parts by a rule on the lengths of all requests; the last part to
// arrive adds up the results of all, in the order of the keys.
#include "heads.hpp"
#include "serving.hpp"

namespace eora {
namespace {

constexpr int RG = 4, TQ = 32 * RG;            // wavefronts of a team, pairs of a tile
constexpr int KT = 64;                         // keys of a tile
constexpr int CUS = 256;
constexpr int WANT = 2 * CUS;                  // parts that all tiles together are cut into at least, where they have the work
constexpr int LEAST_PART = 4;                  // tiles of keys of a part
constexpr int MAX_PARTS = 2 * WANT;            // partial results: see unit_of()
constexpr int COUNTERS = ATTEND_COUNTERS;      // words before the partial results: the first of them one for each tile that is cut
static_assert(MAX_PARTS <= COUNTERS, "a counter for each tile that is cut");
constexpr float RAISE = 4.f, LOWER = 11.f;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

template <int DIM>
constexpr int teams() { return DIM == 256 ? 1 : 2; }

typedef float f16x __attribute__((ext_vector_type(16)));
typedef __fp16 tr4 __attribute__((__vector_size__(8)));
typedef __attribute__((address_space(3))) tr4* tr4_lds;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ f16x mfma32(h8 a, h8 b, f16x c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
// the larger of a value and that of the lane 32 further on
__device__ __forceinline__ float max_of_halves(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A request as the kernel takes it: n tokens, rows [first, first + rows), tiles of its pairs, tiles of keys of its longest tile at most, parts a tile is cut into
struct Request {
    int n, first, rows, tiles, cost;
};
__device__ __forceinline__ Request request_of(const PromptArgs& a, int b)
{
    Request r;
    const int most = a.width * a.page, group = a.heads / a.kv;
    int n = a.lengths[b], s = a.starts[b], e = a.starts[b + 1];
    r.n = n < 0 ? 0 : (n > most ? most : n);
    s = s < 0 ? 0 : (s > a.M ? a.M : s);
    e = e < s ? s : (e > a.M ? a.M : e);
    r.first = s;
    r.rows = e - s;
    r.tiles = (int)(((long long)r.rows * group + TQ - 1) / TQ);
    r.cost = (r.n + KT - 1) / KT;
    if (a.window > 0) {
        const long long near = ((long long)a.window + (TQ - 1) / group + 1) / KT + 2 + (a.sinks + KT - 1) / KT;
        r.cost = near < r.cost ? (int)near : r.cost;
    }
    r.cost = r.cost < 1 ? 1 : r.cost;
    return r;
}

// What a workgroup does: part `part` of `parts` of a tile.  place: its partial results' number; of its tile's first part.
struct Unit {
    int b, h, tile, part, parts;
    int place, first;
};
// All threads.  Tiles of a request are cut into ceil(cost / share) parts, share = a WANT-th of all work: with parts > 1 a request has less than 2 cost / share, so all of them have less
// than 2 WANT parts.
template <int THREADS>
__device__ __forceinline__ bool unit_of(const PromptArgs& a, unsigned id, Unit& u, int* scratch)
{
    constexpr int NW = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned long long* sums = (unsigned long long*)scratch;                    // NW
    int* found = scratch + 2 * NW;                                              // b, id within the request, parts before
    int* totals = found + 4;                                                    // 2 NW
    unsigned long long work = 0;
    for (int b = threadIdx.x; b < a.B; b += THREADS) {
        const Request r = request_of(a, b);
        work += (unsigned long long)r.tiles * r.cost;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) work += __shfl_xor(work, o, 64);
    if (lane == 0) sums[wave] = work;
    if (threadIdx.x == 0) found[0] = -1;
    __syncthreads();
    work = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) work += sums[w];
    unsigned long long share = (work * (unsigned)a.kv + WANT - 1) / WANT;
    share = share < LEAST_PART ? LEAST_PART : share;
    unsigned before = 0, cut_before = 0;
    for (int b0 = 0; b0 < a.B; b0 += THREADS) {
        const int b = b0 + (int)threadIdx.x;
        unsigned units = 0, cut = 0;
        if (b < a.B) {
            const Request r = request_of(a, b);
            const unsigned parts = r.cost <= share ? 1u : (unsigned)((r.cost + share - 1) / share);
            units = (unsigned)r.tiles * parts * (unsigned)a.kv;
            cut = parts > 1 ? units : 0;
        }
        unsigned v = units, c = cut;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const unsigned x = __shfl_up(v, o, 64), y = __shfl_up(c, o, 64);
            v += lane >= o ? x : 0;
            c += lane >= o ? y : 0;
        }
        if (lane == 63) {
            totals[2 * wave] = (int)v;
            totals[2 * wave + 1] = (int)c;
        }
        __syncthreads();
        unsigned sum = 0, cut_sum = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            v += w < wave ? (unsigned)totals[2 * w] : 0;
            c += w < wave ? (unsigned)totals[2 * w + 1] : 0;
            sum += (unsigned)totals[2 * w];
            cut_sum += (unsigned)totals[2 * w + 1];
        }
        v += before;
        c += cut_before;
        if (id >= v - units && id < v) {
            found[0] = b;
            found[1] = (int)(id - (v - units));
            found[2] = (int)(c - cut);
        }
        before += sum;
        cut_before += cut_sum;
        __syncthreads();
        if (id < before) break;
    }
    u.b = __builtin_amdgcn_readfirstlane(found[0]);
    if (u.b < 0) return false;
    const Request r = request_of(a, u.b);
    const int local = __builtin_amdgcn_readfirstlane(found[1]), cut = __builtin_amdgcn_readfirstlane(found[2]);
    u.parts = r.cost <= share ? 1 : (int)((r.cost + share - 1) / share);
    const int rest = local / a.kv, tile = rest / u.parts;
    u.h = local - rest * a.kv;
    u.part = rest - tile * u.parts;
    u.tile = r.tiles - 1 - tile;               // (the last rows see most)
    u.first = cut + (tile * u.parts) * a.kv + u.h;
    u.place = u.first + u.part * a.kv;
    return true;
}

// Stores and loads of partial results go past the caches of an XCD, eight bytes each (relaxed, agent scope).
__device__ __forceinline__ void put2(float* p, float x, float y)
{
    const unsigned long long v = (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x);
    __hip_atomic_store((unsigned long long*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float* p)
{
    const unsigned long long v = __hip_atomic_load((const unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}
__device__ __forceinline__ float factor(float m, float to) { return m == -INFINITY ? 0.f : exp2_(m - to); }

// a partial result: RG wavefronts x (DIM / 2 + 1) x 64 lanes x two words, the last pair (m, sum)
template <int DIM>
constexpr size_t part_words() { return (size_t)RG * (DIM / 4 + 1) * 128; }

template <int DIM, int BITS, bool BLOCKS>
__global__ __launch_bounds__(64 * RG * teams<DIM>(), teams<DIM>()) void prompt_kernel(const PromptArgs a)
{
    constexpr int TEAMS = teams<DIM>(), THREADS = 64 * RG * TEAMS, TEAM = 64 * RG;
    constexpr int ROW = 2 * DIM;               // bytes of a row in LDS
    constexpr int STAGE = 2 * KT * ROW;        // keys, then values
    constexpr int NK = DIM / 16, ND = DIM / 32;                   // k-steps of the first product, blocks of O^T
    constexpr int PER = 16 / (BITS / 8);       // elements of a 16-byte piece in memory
    constexpr int PIECES = KT * DIM / PER / TEAM;                 // pieces of K (of V) a thread moves
    constexpr int PR = DIM / PER;              // pieces of a row
    constexpr int VX = DIM == 64 ? 3 : 7;      // how many units of 32 bytes of V's rows change places

    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ int scratch[2 * 8 + 4 + 2 * 8];
    __shared__ int marks[2][2];                // (team, stage): the step whose values have one that is not finite
    __shared__ int last;

    Unit u;
    if (!unit_of<THREADS>(a, blockIdx.x, u, scratch)) return;
    const Request r = request_of(a, u.b);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave / RG, rg = wave % RG;
    const int tt = threadIdx.x % TEAM, col = lane & 31, half = lane >> 5;
    const int group = a.heads / a.kv, pairs = r.rows * group, from = r.n - r.rows;             // from: position of row 0 (below 0: rows that see nothing)
    const int pair0 = u.tile * TQ, pair1 = pair0 + TQ < pairs ? pair0 + TQ : pairs;

    // tiles of keys that some row of the tile sees
    const int low = from + pair0 / group, high = from + (pair1 - 1) / group;                   // positions of its first and last row
    const int hi = high + 1 < 0 ? 0 : high + 1;
    int lo = a.window > 0 && low - a.window + 1 > 0 ? low - a.window + 1 : 0;
    if (lo <= a.sinks) lo = 0;
    const int sinks = lo > 0 ? a.sinks : 0;
    const int first = lo / KT;
    int head = (sinks + KT - 1) / KT;
    head = head < first ? head : first;
    const int tiles = (hi + KT - 1) / KT - first + head > 0 ? (hi + KT - 1) / KT - first + head : 0;
    auto key_of = [&](int i) { return (i < head ? i : i - head + first) * KT; };
    int parts = (tiles + LEAST_PART - 1) / LEAST_PART;
    parts = parts < 1 ? 1 : (parts < u.parts ? parts : u.parts);
    if (u.part >= parts) return;
    const int k0 = (int)((long long)tiles * u.part / parts), k1 = (int)((long long)tiles * (u.part + 1) / parts);
    const int steps = (k1 - k0 + TEAMS - 1) / TEAMS, mine = (k1 - k0 - team + TEAMS - 1) / TEAMS;

    // this lane's pair, and the positions that this wavefront's pairs have
    const int pair = pair0 + 32 * rg + col;
    const bool there = pair < pair1;
    const int row = there ? pair / group : 0, qh = u.h * group + (there ? pair - row * group : 0);
    const int pos = there ? from + row : -1;
    const int w0 = pair0 + 32 * rg, w1 = w0 + 32 < pair1 ? w0 + 32 : pair1;                    // (w1 <= w0: no pair)
    const int wlow = from + w0 / group, whigh = w1 > w0 ? from + (w1 - 1) / group : -1;
    const bool all = w1 - w0 == 32;

    // Rows of the next 64 groups of 16 keys of this team: lane 4 i + g has group g of its tile i (-1: no page, or no key that a row sees)
    long long rows_of = -1;
    uint32_t bytes_of = 0;
    const int* table = a.table + (size_t)u.b * a.width;
    auto look = [&](int i0) {
        const int i = i0 + (lane >> 2), key = i < mine ? key_of(k0 + team + TEAMS * i) + 16 * (lane & 3) : hi;
        rows_of = -1;
        bytes_of = 0;
        if (key < hi) {
            const int p = key / a.page, page = table[p];
            if ((unsigned)page < (unsigned)a.n_pages) {
                rows_of = ((long long)page * a.kv + u.h) * a.page + (key - p * a.page);
                if constexpr (BLOCKS) bytes_of = a.k_scales[rows_of / BLOCK_TOKENS] | (uint32_t)a.v_scales[rows_of / BLOCK_TOKENS] << 8;
            }
        }
    };
    auto row_at = [&](int i, int g) {
        const int from_lane = 4 * (i & 15) + g;
        const unsigned l = __builtin_amdgcn_readlane((unsigned)rows_of, from_lane), h = __builtin_amdgcn_readlane((unsigned)(rows_of >> 32), from_lane);
        return (long long)((unsigned long long)h << 32 | l);
    };
    // Pieces on their way from memory to LDS: piece tt + TEAM i of the tile's, keys' and values'
    u4 mk[PIECES], mv[PIECES];
    uint32_t mbytes[PIECES];
    int mgone = 0;                             // bit i: no page
    auto load = [&](int i) {
        mgone = 0;
#pragma unroll
        for (int e = 0; e < PIECES; ++e) {
            const int piece = __builtin_amdgcn_readfirstlane((tt & ~63) + TEAM * e), g = piece / PR / 16;       // (a wavefront's pieces lie in one group)
            const long long at = row_at(i, g);
            if constexpr (BLOCKS) mbytes[e] = __builtin_amdgcn_readlane(bytes_of, 4 * (i & 15) + g);
            mgone |= (at < 0) << e;
            const size_t base = (size_t)((at < 0 ? 0 : at) + piece / PR % 16) * (DIM * BITS / 8);
            const unsigned off = 16u * lane;
            mk[e] = *(const u4*)((const char*)a.pages_k + base + off);
            mv[e] = *(const u4*)((const char*)a.pages_v + base + off);
        }
    };
    auto store = [&](int i, int stage) {
        const int key0 = key_of(k0 + team + TEAMS * i);
        // tokens that no row sees are zeros: those behind the last, those between the first ones and the window, those without a page
        const bool clean = key0 + KT <= hi && (key0 >= lo || key0 + KT <= sinks) && mgone == 0;
        // whether some rows see one and others do not
        const bool torn = key0 + KT > low + 1 || (a.window > 0 && key0 <= high - a.window && key0 + KT > sinks);
        unsigned char* to = smem + (team * 2 + stage) * STAGE;
        bool odd = false;
#pragma unroll
        for (int e = 0; e < PIECES; ++e) {
            const int piece = tt + TEAM * e, key = piece / PR, c = piece - key * PR;
            Frag k[PER / 8], v[PER / 8];
            if constexpr (BITS == 16) {
                k[0].q = mk[e];
                v[0].q = mv[e];
            } else {
                const float ks = BLOCKS ? power_of(mbytes[e] & 255) : 1.f, vs = BLOCKS ? power_of(mbytes[e] >> 8) : 1.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    k[w / 2].p[2 * (w % 2)] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(mk[e][w], ks, false);
                    k[w / 2].p[2 * (w % 2) + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(mk[e][w], ks, true);
                    v[w / 2].p[2 * (w % 2)] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(mv[e][w], vs, false);
                    v[w / 2].p[2 * (w % 2) + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(mv[e][w], vs, true);
                }
            }
            if (!clean) {
                const int at = key0 + key;
                const bool seen = at < hi && (at >= lo || at < sinks) && !(mgone >> e & 1);
#pragma unroll
                for (int w = 0; w < PER / 8; ++w) {
                    v[w].q = seen ? v[w].q : u4{0, 0, 0, 0};
                }
            }
#pragma unroll
            for (int w = 0; w < PER / 8; ++w) {
                const int chunk = c * (PER / 8) + w;                    // of 16 bytes in the row
                *(u4*)(to + key * ROW + 16 * (chunk ^ (key & 7))) = k[w].q;
                *(u4*)(to + KT * ROW + key * ROW + 16 * (chunk ^ (2 * (key & VX)))) = v[w].q;
                if (torn) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) odd |= (v[w].u[q] & 0x7c00u) == 0x7c00u || (v[w].u[q] & 0x7c000000u) == 0x7c000000u;
                }
            }
        }
        if (torn && __any(odd) && lane == 0) marks[team][stage] = i + 1;
    };

    // q, its sign that of the scale
    const float scale = a.scale * LOG2E * (BITS == 8 && !BLOCKS ? a.k_scale[u.h] : 1.f), by = fmaxf(fabsf(scale), 0x1p-100f);       // (a scale of 0: scores that are)
    Frag q[NK];
    {
        const _Float16* at = a.q + (size_t)(r.first + row) * a.q_stride + (size_t)qh * DIM + 8 * half;
        const uint32_t sign = scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int t = 0; t < NK; ++t) {
            const u4 w = *(const u4*)(at + 16 * t);
#pragma unroll
            for (int e = 0; e < 4; ++e) q[t].u[e] = there ? w[e] ^ sign : 0u;
        }
    }
    f16x O[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) O[d] = f16x{};
    float m = -INFINITY, l = 0.f;

    // where this lane reads: K, row col: piece 2 t + half; V, transposed: rows 4 half + lane % 16 / 4, columns 16 (lane / 16 % 2) + 4 (lane % 4) of 32
    const int k_at = col * ROW, k_turn = half ^ (col & 7);
    const int v_key = 4 * half + (lane & 15) / 4, v_at = KT * ROW + v_key * ROW + 8 * (lane & 3), v_turn = (lane >> 4 & 1) ^ (v_key & VX);

    if (tt < 2) marks[team][tt] = 0;
    look(0);
    if (mine > 0) load(0);
    __syncthreads();
    if (mine > 0) store(0, 0);
    __syncthreads();
    for (int i = 0; i < steps; ++i) {
        const int stage = i & 1;
        const int key0 = i < mine ? key_of(k0 + team + TEAMS * i) : 0;
        unsigned gone = 0;                     // groups of the tile without a page
        if (i < mine) {
#pragma unroll
            for (int g = 0; g < 4; ++g) gone |= (unsigned)(row_at(i, g) < 0) << g;
        }
        if (i + 1 < mine) {
            if (((i + 1) & 15) == 0) look(i + 1);
            load(i + 1);
        }
        // (rows of a wavefront see none of it: behind them, or before their windows)
        const bool some = i < mine && key0 <= whigh && (a.window == 0 || key0 + KT > wlow - a.window + 1 || key0 < a.sinks);
        if (some) {
            const unsigned char* base = smem + (team * 2 + stage) * STAGE;
            f16x S[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                S[b] = f16x{};
#pragma unroll
                for (int t = 0; t < NK; ++t) {
                    Frag k;
                    k.q = *(const u4*)(base + k_at + 32 * b * ROW + 16 * ((2 * t) ^ k_turn));
                    S[b] = mfma32(k.v, q[t].v, S[b]);
                }
            }
            const bool whole = all && gone == 0 && key0 + KT <= wlow + 1 && (a.window == 0 || key0 > whigh - a.window || key0 + KT <= a.sinks);
            if (!whole) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int key = key0 + 32 * b + 8 * (e / 4) + 4 * half + e % 4;
                        const bool seen = key <= pos && (a.window == 0 || key > pos - a.window || key < a.sinks) && !(gone >> (2 * b + e / 8) & 1);
                        S[b][e] = seen ? S[b][e] : -INFINITY;
                    }
            }
            float top = fmaxf(S[0][0], S[1][0]);
#pragma unroll
            for (int e = 1; e < 16; ++e) top = fmaxf(fmaxf(top, S[0][e]), S[1][e]);
            top *= by;
            if (__any(top > m + (RAISE + LOWER))) {
                top = max_of_halves(top);
                const float up = top > m + (RAISE + LOWER) ? top - LOWER : m, f = m == up ? 1.f : exp2_(m - up);      // (a pair's own scores decide, whatever the others of the wavefront have)
                m = up;
                l *= f;
#pragma unroll
                for (int d = 0; d < ND; ++d) O[d] *= f;
            }
            const float ref = m == -INFINITY ? 0.f : m;
            Frag p[4];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float x = exp2_(__builtin_fmaf(S[b][e], by, -ref)), y = exp2_(__builtin_fmaf(S[b][e + 1], by, -ref));
                    l += x;
                    l += y;
                    p[2 * b + e / 8].p[e % 8 / 2] = h2{(_Float16)x, (_Float16)y};
                }
            auto second = [&](bool careful) {
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        Frag v;
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const unsigned char* at = base + v_at + (16 * s + 8 * e) * ROW + 32 * ((2 * d) ^ v_turn);
                            const auto w = __builtin_amdgcn_ds_read_tr16_b64_v4f16((tr4_lds)at);
                            __builtin_memcpy(&v.u[2 * e], &w, 8);
                        }
                        if (careful) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if ((v.u[e] & 0x7c00u) == 0x7c00u) v.u[e] &= 0xffff0000u;
                                if ((v.u[e] & 0x7c000000u) == 0x7c000000u) v.u[e] &= 0xffffu;
                            }
                        }
                        O[d] = mfma32(v.v, p[s].v, O[d]);
                    }
            };
            if (marks[team][stage] != i + 1) {
                second(false);
            } else {
                // values that are not finite, key by key, for the rows that have a weight for them
                second(true);
                for (int key = 0; key < KT; ++key) {
                    // the weight: register 8 (key / 16) + 4 (key / 8 % 2) + key % 4 of the lanes of half key / 4 % 2
                    uint32_t w = 0;
#pragma unroll
                    for (int e = 0; e < 16; ++e) w = e == key / 16 * 4 + key / 8 % 2 * 2 + key % 4 / 2 ? p[e / 4].u[e % 4] : w;
                    w = key % 2 ? w >> 16 : w & 0xffffu;
                    const auto both = __builtin_amdgcn_permlane32_swap(w, w, false, false);
                    const float x = (float)__builtin_bit_cast(_Float16, (unsigned short)(key / 4 % 2 ? both[1] : both[0]));
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int c = 32 * d + 8 * (e / 4) + 4 * half + e % 4;
                            const float v = (float)*(const _Float16*)(base + KT * ROW + key * ROW + 32 * ((c / 16) ^ (key & VX)) + 2 * (c % 16));
                            if (x != 0.f && !(fabsf(v) < INFINITY)) O[d][e] += x * v;
                        }
                }
            }
        }
        if (i + 1 < mine) store(i + 1, stage ^ 1);
        __syncthreads();
    }
    {
        const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(w[0]) + __uint_as_float(w[1]);
    }

    // the teams' results, added up (all have passed the loop's last barrier)
    if constexpr (TEAMS == 2) {
        float* red = (float*)smem + (size_t)rg * (16 * ND + 2) * 64 + lane;
        if (team == 1) {
            red[0] = m;
            red[64] = l;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) red[(2 + 16 * d + e) * 64] = O[d][e];
        }
        __syncthreads();
        if (team == 0) {
            const float mo = red[0], lo2 = red[64], up = fmaxf(m, mo), f = factor(m, up), g = factor(mo, up);
            l = (m == -INFINITY ? l : l * f) + (mo == -INFINITY ? lo2 : lo2 * g);
            m = up;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) O[d][e] = O[d][e] * f + red[(2 + 16 * d + e) * 64] * g;
        }
    }

    const float vs = BITS == 8 && !BLOCKS ? a.v_scale[u.h] : 1.f;
    if (parts > 1) {
        float* part = a.parts + COUNTERS + (size_t)u.place * part_words<DIM>() + (size_t)rg * (DIM / 4 + 1) * 128 + 2 * lane;
        if (team == 0) {
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int e = 0; e < 16; e += 2) put2(part + (8 * d + e / 2) * 128, O[d][e], O[d][e + 1]);
            put2(part + DIM / 4 * 128, m, l);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) {
            unsigned* counter = (unsigned*)a.parts + u.first;
            last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == (unsigned)parts;
            if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!last || team != 0) return;
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) O[d] = f16x{};
        for (int c = 0; c < parts; ++c) {
            const float* src = a.parts + COUNTERS + (size_t)(u.first + c * a.kv) * part_words<DIM>() + (size_t)rg * (DIM / 4 + 1) * 128 + 2 * lane;
            const float2 ml = get2(src + DIM / 4 * 128);
            const float up = fmaxf(m, ml.x), f = factor(m, up), g = factor(ml.x, up);
            l = (m == -INFINITY ? l : l * f) + (ml.x == -INFINITY ? ml.y : ml.y * g);
            m = up;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float2 x = get2(src + (8 * d + e / 2) * 128);
                    O[d][e] = O[d][e] * f + x.x * g;
                    O[d][e + 1] = O[d][e + 1] * f + x.y * g;
                }
        }
    }
    if (team != 0 || !there) return;
    const size_t at = (size_t)(r.first + row) * a.heads + qh;
    const float f = vs / l;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            h4 y;
#pragma unroll
            for (int c = 0; c < 4; ++c) y[c] = (_Float16)(l == 0.f ? 0.f : O[d][e + c] * f);
            *(h4*)(a.out + at * DIM + 32 * d + 2 * e + 4 * half) = y;
        }
    if (half == 0 && a.lse) a.lse[at] = LN2 * (m + __log2f(l));
}

template <int DIM, int BITS, bool BLOCKS>
hipError_t start(const PromptArgs& a, hipStream_t stream)
{
    constexpr int lds = teams<DIM>() * 2 * 2 * KT * 2 * DIM;
    const auto kern = prompt_kernel<DIM, BITS, BLOCKS>;
    const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    kern<<<(unsigned)prompt_units(a.M, a.B, a.heads, a.kv, DIM), 64 * RG * teams<DIM>(), lds, stream>>>(a);
    return hipGetLastError();
}

template <int DIM>
hipError_t start(const PromptArgs& a, hipStream_t stream)
{
    if (a.bits == 16) return start<DIM, 16, false>(a, stream);
    return a.k_scales ? start<DIM, 8, true>(a, stream) : start<DIM, 8, false>(a, stream);
}

}  // namespace

long long prompt_units(int M, int B, int heads, int kv, int dim)
{
    const long long group = heads / kv;
    return (((long long)M * group + TQ - 1) / TQ + B) * kv + MAX_PARTS;
}

size_t prompt_workspace_bytes(int dim)
{
    const size_t words = dim == 64 ? part_words<64>() : (dim == 128 ? part_words<128>() : part_words<256>());
    return (COUNTERS + MAX_PARTS * words) * sizeof(float);
}

hipError_t launch_prompt(const PromptArgs& a, hipStream_t stream)
{
    return a.dim == 64 ? start<64>(a, stream) : (a.dim == 128 ? start<128>(a, stream) : start<256>(a, stream));
}

}  // namespace eora
