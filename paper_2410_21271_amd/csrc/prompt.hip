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

#include <utility>

namespace eora {
namespace {

constexpr int RG = 4, THREADS = 64 * RG, TQ = 32 * RG;           // wavefronts; pairs of a tile
constexpr int KT = 64;                         // keys of a tile
constexpr int CUS = 256;
// Parts that all tiles together are cut into at least, where they have the work; partial results that there are: see unit_of().
constexpr int WANT = 2 * CUS;
constexpr int MAX_PARTS = 2 * WANT;
constexpr int LEAST_PART = 4;                  // tiles of keys of a part
constexpr int COUNTERS = ATTEND_COUNTERS;      // words before the partial results: the first of them one for each tile that is cut
static_assert(MAX_PARTS <= COUNTERS, "a counter for each tile that is cut");
constexpr float RAISE = 4.f, LOWER = 11.f;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

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

// 64 pieces of 16 bytes from memory straight into 1 KiB of LDS, lane after lane: from base + off + OFF to lds + OFF.  The compiler does not know of the request: it counts in vmcnt all
// the same, so the compiler's own waits only get longer, and whoever reads the bytes waits for them (arrived()) before the barrier in front of the reads.
template <int OFF>
__device__ __forceinline__ void memory_to_lds(const char* base, unsigned off, unsigned lds)
{
    static_assert(OFF >= 0 && OFF < 4096, "");
    const unsigned long long at = (unsigned long long)base;
    const unsigned low = __builtin_amdgcn_readfirstlane((unsigned)at), high = __builtin_amdgcn_readfirstlane((unsigned)(at >> 32));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3"
                 : : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"((unsigned long long)high << 32 | low), "i"(OFF) : "memory", "m0");
}
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// A request as the kernel takes it: n tokens, rows [first, first + rows), tiles of its pairs, tiles of keys of its longest one at most
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

// What a workgroup does: part `part` of `parts` of a tile of a request.  place: its partial results' number; first: of its tile's first part.
struct Unit {
    Request r;
    int b, h, tile, part, parts;
    int place, first;
};
// Tiles of a request are cut into ceil(cost / share) parts, share = a WANT-th of all work: with parts > 1 a request has less than 2 cost / share, so all of them have at most 2 WANT parts.
// (The work is added up in floats, in one order: everyone finds the same share.)
__device__ __forceinline__ int share_of(float work, int kv)
{
    const float x = work * (float)kv * (1.f / WANT);
    const int share = x < 1e9f ? (int)x + 1 : 0x7fffffff;
    return share < LEAST_PART ? LEAST_PART : share;
}
__device__ __forceinline__ int parts_of(const Request& r, int share) { return r.cost <= share ? 1 : (int)((unsigned)(r.cost - 1) / (unsigned)share) + 1; }
__device__ __forceinline__ Unit unit_in(const PromptArgs& a, const Request& r, int b, int parts, int local, int cut)
{
    Unit u;
    u.r = r;
    u.b = b;
    u.parts = parts;
    const int rest = (int)((unsigned)local / (unsigned)a.kv), tile = (int)((unsigned)rest / (unsigned)parts);
    u.h = local - rest * a.kv;
    u.part = rest - tile * parts;
    u.tile = r.tiles - 1 - tile;               // (the last rows see most)
    u.first = cut + tile * parts * a.kv + u.h;
    u.place = u.first + u.part * a.kv;
    return u;
}
// the sum over this lane and those before it
template <typename T>
__device__ __forceinline__ T scan(T v)
{
    auto add = [&](auto ctrl, auto rows) {
        const int w = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
        v += __builtin_bit_cast(T, w);
    };
    add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xF>{});         // the lane before, of the row of 16
    add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});         // the last of rows 0 and 2 to rows 1 and 3
    add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});         // the last of row 1 to rows 2 and 3
    return v;
}
// Up to 64 requests: each wavefront for itself, a request a lane, read once.
__device__ __forceinline__ bool unit_of_few(const PromptArgs& a, int id, Unit& u)
{
    const int lane = threadIdx.x & 63;
    Request r = request_of(a, lane < a.B ? lane : a.B - 1);
    if (lane >= a.B) r.tiles = 0;
    const int share = share_of(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scan((float)r.tiles * (float)r.cost)), 63)), a.kv);
    const int parts = parts_of(r, share), units = r.tiles * parts * a.kv, cut = parts > 1 ? units : 0;
    const int v = scan(units), c = scan(cut);
    const unsigned long long mine = __ballot(id >= v - units && id < v);
    if (mine == 0) return false;
    const int b = __builtin_ctzll(mine);
    auto of = [&](int x) { return __builtin_amdgcn_readlane(x, b); };
    Request q;
    q.n = of(r.n);
    q.first = of(r.first);
    q.rows = of(r.rows);
    q.tiles = of(r.tiles);
    q.cost = of(r.cost);
    u = unit_in(a, q, b, of(parts), id - of(v - units), of(c - cut));
    return true;
}
// Any number of them: all threads, a request each at a time.
__device__ __forceinline__ bool unit_of(const PromptArgs& a, int id, Unit& u, int* scratch)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float* sums = (float*)scratch;                                              // RG
    int* found = scratch + RG;                                                  // b, id within the request, parts before
    int* totals = found + 4;                                                    // 2 RG
    float work = 0.f;
    for (int b = threadIdx.x; b < a.B; b += THREADS) {
        const Request r = request_of(a, b);
        work += (float)r.tiles * (float)r.cost;
    }
    work = scan(work);
    if (lane == 63) sums[wave] = work;
    if (threadIdx.x == 0) found[0] = -1;
    __syncthreads();
    work = 0.f;
#pragma unroll
    for (int w = 0; w < RG; ++w) work += sums[w];
    const int share = share_of(work, a.kv);
    int before = 0, cut_before = 0;
    for (int b0 = 0; b0 < a.B; b0 += THREADS) {
        const int b = b0 + (int)threadIdx.x;
        int units = 0, cut = 0;
        if (b < a.B) {
            const Request r = request_of(a, b);
            const int parts = parts_of(r, share);
            units = r.tiles * parts * a.kv;
            cut = parts > 1 ? units : 0;
        }
        int v = scan(units), c = scan(cut);
        if (lane == 63) {
            totals[2 * wave] = v;
            totals[2 * wave + 1] = c;
        }
        __syncthreads();
        int sum = 0, cut_sum = 0;
#pragma unroll
        for (int w = 0; w < RG; ++w) {
            v += w < wave ? totals[2 * w] : 0;
            c += w < wave ? totals[2 * w + 1] : 0;
            sum += totals[2 * w];
            cut_sum += totals[2 * w + 1];
        }
        v += before;
        c += cut_before;
        if (id >= v - units && id < v) {
            found[0] = b;
            found[1] = id - (v - units);
            found[2] = c - cut;
        }
        before += sum;
        cut_before += cut_sum;
        __syncthreads();
        if (id < before) break;
    }
    const int b = __builtin_amdgcn_readfirstlane(found[0]);
    if (b < 0) return false;
    Request r = request_of(a, b);
    r.n = __builtin_amdgcn_readfirstlane(r.n);
    r.first = __builtin_amdgcn_readfirstlane(r.first);
    r.rows = __builtin_amdgcn_readfirstlane(r.rows);
    r.tiles = __builtin_amdgcn_readfirstlane(r.tiles);
    r.cost = __builtin_amdgcn_readfirstlane(r.cost);
    u = unit_in(a, r, b, parts_of(r, share), __builtin_amdgcn_readfirstlane(found[1]), __builtin_amdgcn_readfirstlane(found[2]));
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

// f(0) .. f(N - 1), each number a type
template <int N, typename F, int... I>
__device__ __forceinline__ void each_of(const F& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void each_piece(const F& f) { each_of<N>(f, std::make_integer_sequence<int, N>{}); }

// words of a partial result: (m, sum) and O of each pair
constexpr size_t part_words(int dim) { return (size_t)TQ * (dim + 2); }

// K in LDS: rows in groups of 1 KiB, as they come from memory, with a gap behind each group
constexpr int k_group(int dim) { return 512 / dim; }
constexpr int K_GAP = 64, K_GAP_256 = 32;
constexpr int k_pitch(int dim) { return 1024 + (dim == 256 ? K_GAP_256 : K_GAP); }
constexpr int stage_bytes(int dim) { return KT / k_group(dim) * k_pitch(dim) + KT * 2 * dim; }
template <int DIM, int BITS>
constexpr int lds_bytes()
{
    constexpr int loop = 2 * stage_bytes(DIM) + BLOCK_TOKENS * DIM * BITS / 8, end = TQ * DIM * 4;
    return loop > end ? loop : end;
}

// Workgroups a compute unit has at a time, as registers and LDS allow
constexpr int residents(int dim) { return dim == 256 ? 1 : 2; }

template <int DIM, int BITS, bool BLOCKS>
__global__ __launch_bounds__(THREADS, residents(DIM)) void prompt_kernel(const PromptArgs a)
{
    constexpr int ROW = 2 * DIM;               // bytes of a row in LDS
    constexpr int GROUP = k_group(DIM), PITCH = k_pitch(DIM);
    constexpr int STAGE = stage_bytes(DIM), VALUES = STAGE - KT * ROW;            // keys, then values
    constexpr int NK = DIM / 16, ND = DIM / 32;                   // k-steps of the first product, blocks of O^T
    constexpr int BYTES = DIM * BITS / 8;      // of a row in memory
    constexpr int PIECES = BLOCK_TOKENS * BYTES / 1024;           // KiB of a wavefront's 16 keys (or values) of a tile
    constexpr int AHEAD = 4;                   // matrix instructions between an operand's read and its use
    // How pieces of 16 bytes change places in the row of a key, so that the lanes that read at a time meet different banks: 16 keys' pieces of the same columns; two units of 32 bytes
    // of four keys
    auto k_turn_of = [](int key) { return DIM == 64 ? key >> 1 & 3 : (DIM == 128 ? key & 3 : key & 1); };
    auto v_turn_of = [](int key) { return 4 * (DIM == 64 ? key >> 1 & 1 : key & 3); };

    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ int scratch[RG + 4 + 2 * RG];
    __shared__ int odd_one;                    // some value that not all rows see is not finite
    __shared__ int last;
    __shared__ float row_m[TQ], row_l[TQ];

    Unit u;
    if (!(a.B <= 64 ? unit_of_few(a, (int)blockIdx.x, u) : unit_of(a, (int)blockIdx.x, u, scratch))) return;
    const Request r = u.r;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
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
    const int steps = k1 - k0;

    // this lane's pair, and the positions that this wavefront's pairs have
    const int pair = pair0 + 32 * wave + col;
    const bool there = pair < pair1;
    const int row = there ? pair / group : 0, qh = u.h * group + (there ? pair - row * group : 0);
    const int pos = there ? from + row : -1;
    const int w0 = pair0 + 32 * wave, w1 = w0 + 32 < pair1 ? w0 + 32 : pair1;                    // (w1 <= w0: no pair)
    const int wlow = from + w0 / group, whigh = w1 > w0 ? from + (w1 - 1) / group : -1;
    const bool all = w1 - w0 == 32;

    // Blocks of 16 tokens of the next 64 groups of 16 keys: lane 4 i + g has where that of group g of its tile i begins in the cache, in bytes (0: no page, or no key that a
    // row sees: those are in `lost`), and its scales
    unsigned off_low = 0, off_high = 0;
    unsigned k_byte = 0, v_byte = 0;
    unsigned long long lost = 0;
    const int* table = a.table + (size_t)u.b * a.width;
    const int per_page = a.page / BLOCK_TOKENS;
    auto block_at = [&](int key) {
        const int p = key / a.page, page = table[p];
        return (unsigned)page < (unsigned)a.n_pages ? (page * a.kv + u.h) * per_page + (key - p * a.page) / BLOCK_TOKENS : -1;
    };
    auto gone_at = [&](int key0) {
        unsigned gone = 0;
        for (int g = 0; g < 4; ++g) gone |= (unsigned)(key0 + 16 * g < hi && block_at(key0 + 16 * g) < 0) << g;
        return gone;
    };
    auto tile_at = [&](int i) { return key_of(k0 + i); };
    auto look = [&](int i0) {
        const int i = i0 + (lane >> 2), key = i < steps ? tile_at(i) + 16 * (lane & 3) : hi, block = key < hi ? block_at(key) : -1;
        lost = __ballot(block < 0);
        const size_t off = (size_t)(unsigned)(block < 0 ? 0 : block) * (BLOCK_TOKENS * BYTES);
        off_low = (unsigned)off;
        off_high = (unsigned)(off >> 32);
        if constexpr (BLOCKS) {
            k_byte = block < 0 ? 0 : a.k_scales[block];
            v_byte = block < 0 ? 0 : a.v_scales[block];
        }
    };
    auto gone_of = [&](int i) { return (unsigned)(lost >> (4 * (i & 15))) & 15u; };
    // Whether a tile's values can go to LDS as they are: all rows see all of its tokens
    auto plain = [&](int key0, unsigned gone) { return gone == 0 && key0 + KT <= low + 1 && (a.window == 0 || key0 > high - a.window || key0 + KT <= a.sinks); };

    // A wavefront moves the tile's group of 16 keys that has its number, a KiB at a time: this lane's row of the KiB, and its piece of 16 bytes of it
    constexpr int PR = BYTES / 16, ROWS = 64 / PR;
    const int lrow = lane / PR, lpiece = lane % PR;
    auto block_of = [&](int i) {
        const int from_lane = 4 * (i & 15) + wave;
        return (unsigned long long)__builtin_amdgcn_readlane(off_high, from_lane) << 32 | __builtin_amdgcn_readlane(off_low, from_lane);
    };
    auto power_at = [&](unsigned bytes, int i) { return BLOCKS ? power_of(__builtin_amdgcn_readlane(bytes, 4 * (i & 15) + wave)) : 1.f; };
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem, aside = lds0 + 2 * STAGE;      // (what nobody reads)
    constexpr int K_MINE = BLOCK_TOKENS / GROUP * PITCH, V_MINE = BLOCK_TOKENS * ROW;           // a wavefront's part of a stage
    // fp16: pieces change places on the way, as the addresses say.  8 bits: codes as they are, at the beginning of the wavefront's part; it spreads them out there itself
    const unsigned linear = 16u * lane, k_off = BITS == 16 ? (unsigned)(lrow * ROW + 16 * (lpiece ^ k_turn_of(lrow))) : linear;
    const unsigned v_off = BITS == 16 ? (unsigned)(lrow * ROW + 16 * (lpiece ^ v_turn_of(lrow))) : linear;
    auto send_keys = [&](const char* base, auto piece, int stage) {
        constexpr int e = decltype(piece)::value, far = e / 4 * 4096, off = e % 4 * 1024;
        memory_to_lds<off>(base + far, k_off, lds0 + (unsigned)(stage * STAGE + wave * K_MINE + (BITS == 16 ? e * PITCH - off : far)));
    };
    auto send_values = [&](const char* base, auto piece, unsigned to) {         // (of heads of 256 a KiB has two of the four keys whose pieces change places together)
        constexpr int e = decltype(piece)::value, far = e / 4 * 4096, off = e % 4 * 1024;
        memory_to_lds<off>(base + far, BITS == 16 && DIM == 256 && e % 2 ? v_off ^ 128u : v_off, to + far);
    };
    auto values_to = [&](int stage) { return lds0 + (unsigned)(stage * STAGE + VALUES + wave * V_MINE); };
    auto codes = [](const u4& w, float scale, Frag (&f)[2]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e / 2].p[2 * (e % 2)] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[e], scale, false);
            f[e / 2].p[2 * (e % 2) + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[e], scale, true);
        }
    };
    auto k_place = [&](int key, int piece) { return key / GROUP * PITCH + key % GROUP * ROW + 16 * (piece ^ k_turn_of(key)); };
    auto v_place = [&](int key, int piece) { return VALUES + key * ROW + 16 * (piece ^ v_turn_of(key)); };
    auto spread_keys = [&](int stage, float scale) {
        unsigned char* to = smem + stage * STAGE;
        u4 w[PIECES];
#pragma unroll
        for (int e = 0; e < PIECES; ++e) w[e] = *(const u4*)(to + wave * K_MINE + e * 1024 + linear);
#pragma unroll
        for (int e = 0; e < PIECES; ++e) {
            Frag f[2];
            codes(w[e], scale, f);
#pragma unroll
            for (int h = 0; h < 2; ++h) *(u4*)(to + k_place(BLOCK_TOKENS * wave + e * ROWS + lrow, 2 * lpiece + h)) = f[h].q;
        }
    };
    // Tokens that no row sees become zeros, and so do values that are not finite where some rows see them and others do not: those are added at the end.
    auto clean = [&](Frag& f, int key, int key0, unsigned gone) {
        const int at = key0 + key;
        const bool seen = at < hi && (at >= lo || at < sinks) && !(gone >> wave & 1);
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = seen ? f.u[e] : 0u;
            const uint32_t low_half = (x & 0x7c00u) == 0x7c00u ? 0xffffu : 0u, high_half = (x & 0x7c000000u) == 0x7c000000u ? 0xffff0000u : 0u;
            odd |= (low_half | high_half) != 0;
            f.u[e] = x & ~(low_half | high_half);
        }
        if (odd) odd_one = 1;
    };
    auto spread_values = [&](int stage, float scale, int key0, unsigned gone, bool as_it_is) {
        unsigned char* to = smem + stage * STAGE;
        u4 w[PIECES];
#pragma unroll
        for (int e = 0; e < PIECES; ++e) w[e] = *(const u4*)(to + VALUES + wave * V_MINE + e * 1024 + linear);
#pragma unroll
        for (int e = 0; e < PIECES; ++e) {
            Frag f[2];
            codes(w[e], scale, f);
            const int key = BLOCK_TOKENS * wave + e * ROWS + lrow;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!as_it_is) clean(f[h], key, key0, gone);
                *(u4*)(to + v_place(key, 2 * lpiece + h)) = f[h].q;
            }
        }
    };
    // fp16 values that need it, by way of registers
    auto put_values = [&](const char* base, int stage, int key0, unsigned gone) {
        Frag f[PIECES];
#pragma unroll
        for (int e = 0; e < PIECES; ++e) f[e].q = *(const u4*)(base + (e * 1024 + linear));
#pragma unroll
        for (int e = 0; e < PIECES; ++e) {
            const int key = BLOCK_TOKENS * wave + e * ROWS + lrow;
            clean(f[e], key, key0, gone);
            *(u4*)(smem + stage * STAGE + v_place(key, lpiece)) = f[e].q;
        }
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
    constexpr int BLOCK_OF_KEYS = 32 / GROUP * PITCH;
    const int k_at = col / GROUP * PITCH + col % GROUP * ROW, k_turn = half ^ k_turn_of(col);
    const int v_key = 4 * half + (lane & 15) / 4, v_at = VALUES + v_key * ROW + 8 * (lane & 3), v_turn = (lane >> 4 & 1) ^ (v_turn_of(v_key) / 2);
    auto first_product = [&](const unsigned char* base, f16x (&S)[2]) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f16x z = {};
#pragma unroll
            for (int t = 0; t < NK; ++t) {
                Frag k;
                k.q = *(const u4*)(base + k_at + b * BLOCK_OF_KEYS + 16 * ((2 * t) ^ k_turn));
                z = mfma32(k.v, q[t].v, z);
            }
            S[b] = z;
        }
    };
    auto largest = [&](const f16x (&S)[2]) {
        float top = fmaxf(S[0][0], S[1][0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(fmaxf(top, S[0][e]), S[1][e]);
        return top;
    };

    // Tile i: its scores are there when its step begins, found beside the softmax of the tile before it
    f16x Sa[2], Sb[2];
    float top = -INFINITY;
    unsigned gone = 0, gone_next = 0;          // of tiles i and i + 1
    const bool busy = w1 > w0;                 // (a wavefront without a pair moves its part of the tiles, and no more)
    if (threadIdx.x == 0) odd_one = 0;
    look(0);
    if (steps > 0) {
        gone = gone_of(0);
        const int key0 = tile_at(0), second = steps > 1 ? 1 : 0;
        const bool as_it_is = plain(key0, gone);
        const unsigned long long here = block_of(0), there_on = block_of(second);
        const char *k0_at = (const char*)a.pages_k + here, *v0_at = (const char*)a.pages_v + here, *k1_at = (const char*)a.pages_k + there_on;
        each_piece<PIECES>([&](auto e) { send_keys(k0_at, e, 0); });
        if (BITS == 8 || as_it_is) each_piece<PIECES>([&](auto e) { send_values(v0_at, e, values_to(0)); });
        each_piece<PIECES>([&](auto e) { send_keys(k1_at, e, 1); });
        __syncthreads();                       // (odd_one)
        if (BITS == 16 && !as_it_is) put_values(v0_at, 0, key0, gone);
        arrived();
        if constexpr (BITS == 8) {
            spread_keys(0, power_at(k_byte, 0));
            spread_values(0, power_at(v_byte, 0), key0, gone, as_it_is);
            spread_keys(1, power_at(k_byte, second));
        }
    }
    __syncthreads();
    if (steps > 0 && busy) {
        first_product(smem, Sa);
        top = largest(Sa);
    }
    __syncthreads();
    auto step = [&](int i, f16x (&S)[2], f16x (&N)[2], int stage) {
        // tiles whose values and keys this step moves (behind the last tile: it again, to where nobody reads)
        const bool more = i + 1 < steps;
        const int iv = more ? i + 1 : i, ik = i + 2 < steps ? i + 2 : steps - 1, key_next = tile_at(iv);
        const char* v_base = (const char*)a.pages_v + block_of(iv);
        const float v_by = power_at(v_byte, iv);
        gone_next = gone_of(iv);
        const bool as_it_is = plain(key_next, gone_next);
        if (BITS == 16 && more && !as_it_is) put_values(v_base, stage ^ 1, key_next, gone_next);
        const unsigned v_to = more && (BITS == 8 || as_it_is) ? values_to(stage ^ 1) : aside;
        if (((i + 2) & 15) == 0 && i + 2 < steps) look(i + 2);
        const char* k_base = (const char*)a.pages_k + block_of(ik);
        if (busy) {
            const unsigned char* base = smem + stage * STAGE;
            const int key0 = tile_at(i);
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
                top = largest(S);
            }
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
            // One matrix instruction a slot, kept in this order: beside those of the next tile's scores (behind the last tile: of what lies there, unused) two weights of this one
            // each, beside those of O the next tile's largest score.  Operands are read AHEAD slots before.
            const unsigned char* next = smem + (stage ^ 1) * STAGE;
            Frag kf[AHEAD], vf[AHEAD], p[4];
            auto read_k = [&](int x) { kf[x % AHEAD].q = *(const u4*)(next + k_at + x % 2 * BLOCK_OF_KEYS + 16 * ((2 * (x / 2)) ^ k_turn)); };
            auto read_v = [&](int x) {
                const int s = x / ND, d = x % ND;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const unsigned char* at = base + v_at + (16 * s + 8 * e) * ROW + 32 * ((2 * d) ^ v_turn);
                    const auto w = __builtin_amdgcn_ds_read_tr16_b64_v4f16((tr4_lds)at);
                    __builtin_memcpy(&vf[x % AHEAD].u[2 * e], &w, 8);
                }
            };
            auto weights = [&](int x) {        // elements 2 x and 2 x + 1
                const int b = x / 8, e = 2 * x % 16;
                const float v = exp2_(__builtin_fmaf(S[b][e], by, -ref)), w = exp2_(__builtin_fmaf(S[b][e + 1], by, -ref));
                l += v;                        // (not what the weights are rounded to: lse would be off by 2^-12)
                l += w;
                p[2 * b + e / 8].p[e % 8 / 2] = h2{(_Float16)v, (_Float16)w};
            };
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) read_k(x);
            __builtin_amdgcn_sched_barrier(0);
            each_piece<2 * NK>([&](auto slot) {
                constexpr int x = decltype(slot)::value, b = x % 2, t = x / 2;
                if (t == 0) N[b] = f16x{};
                N[b] = mfma32(kf[x % AHEAD].v, q[t].v, N[b]);
                if (x + AHEAD < 2 * NK) read_k(x + AHEAD);
                else read_v(x + AHEAD - 2 * NK);
                if constexpr (x < PIECES) send_keys(k_base, slot, stage);
                else if constexpr (x < 2 * PIECES) send_values(v_base, std::integral_constant<int, x - PIECES>{}, v_to);
#pragma unroll
                for (int w = 16 * x / (2 * NK); w < 16 * (x + 1) / (2 * NK); ++w) weights(w);
                __builtin_amdgcn_sched_barrier(0);
            });
#pragma unroll
            for (int x = 0; x < 4 * ND; ++x) {
                const int s = x / ND, d = x % ND;
                O[d] = mfma32(vf[x % AHEAD].v, p[s].v, O[d]);
                if (x + AHEAD < 4 * ND) read_v(x + AHEAD);
#pragma unroll
                for (int e = 16 * x / (4 * ND); e < 16 * (x + 1) / (4 * ND); ++e) top = e == 0 ? fmaxf(N[0][0], N[1][0]) : fmaxf(fmaxf(top, N[0][e]), N[1][e]);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            each_piece<PIECES>([&](auto e) { send_keys(k_base, e, stage); });
            each_piece<PIECES>([&](auto e) { send_values(v_base, e, v_to); });
        }
        arrived();
        if constexpr (BITS == 8) {
            spread_keys(stage, power_at(k_byte, ik));
            if (more) spread_values(stage ^ 1, v_by, key_next, gone_next, as_it_is);
        }
        gone = gone_next;
        __syncthreads();
    };
    for (int i = 0; i < steps; i += 2) {
        step(i, Sa, Sb, 0);
        if (i + 1 < steps) step(i + 1, Sb, Sa, 1);
    }
    {
        const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(w[0]) + __uint_as_float(w[1]);
    }

    // The results go to LDS, as rows of fp32 (all have passed the loop's last barrier).  This lane's elements: columns 32 d + 8 q + 4 half of row 32 wave + col; pieces of
    // 16 bytes change places within their row, so that the lanes that write at a time meet different banks.
    float* sum = (float*)smem;
    const int my_row = 32 * wave + col;
    auto piece_at = [&](int r, int c) { return sum + r * DIM + 4 * (c ^ (r & 15)); };
    if (half == 0) {
        row_m[my_row] = m;
        row_l[my_row] = l;
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) *(f4*)piece_at(my_row, 8 * d + 2 * e + half) = f4{O[d][4 * e], O[d][4 * e + 1], O[d][4 * e + 2], O[d][4 * e + 3]};
    __syncthreads();
    if (odd_one) {
        // Values that are not finite, in tiles of which not all rows see all: for the rows that see them, unless their score is -inf
        for (int e = threadIdx.x; e < TQ * (DIM / 4); e += THREADS) {
            const int r2 = e / (DIM / 4), c = e % (DIM / 4), pr = pair0 + r2;
            if (pr >= pair1) continue;
            const int rw = pr / group, at_pos = from + rw, head2 = u.h * group + pr - rw * group;
            f4 add = {0.f, 0.f, 0.f, 0.f};
            for (int i = k0; i < k1; ++i) {
                const int key0 = key_of(i);
                for (int key = key0; key < key0 + KT && key <= at_pos; ++key) {
                    if (!(a.window == 0 || key > at_pos - a.window || key < a.sinks)) continue;
                    const int block = block_at(key & ~(BLOCK_TOKENS - 1));
                    if (block < 0) continue;
                    const size_t at = ((size_t)(unsigned)block * BLOCK_TOKENS + key % BLOCK_TOKENS) * DIM;
                    bool any = false;
                    float v[4];
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        if constexpr (BITS == 16) v[q4] = (float)((const _Float16*)a.pages_v)[at + 4 * c + q4];
                        else v[q4] = (((const uint8_t*)a.pages_v)[at + 4 * c + q4] & 127) == 127 ? __builtin_nanf("") : 0.f;
                        any |= !(fabsf(v[q4]) < INFINITY);
                    }
                    if (!any || plain(key0, gone_at(key0))) continue;
                    if constexpr (BITS == 16) {
                        const _Float16 *x = a.q + (size_t)(r.first + rw) * a.q_stride + (size_t)head2 * DIM, *y = (const _Float16*)a.pages_k + at;
                        float score = 0.f;
                        for (int t = 0; t < DIM; ++t) score += (float)x[t] * (float)y[t];
                        if (score * scale == -INFINITY) continue;
                    }
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) add[q4] += fabsf(v[q4]) < INFINITY ? 0.f : v[q4];
                }
            }
            *(f4*)piece_at(r2, c) += add;
        }
        __syncthreads();
    }

    const float vs = BITS == 8 && !BLOCKS ? a.v_scale[u.h] : 1.f;
    // Pieces of four columns: thread after thread along the rows
    constexpr int MY = TQ * (DIM / 4) / THREADS;
    const int used = pair1 - pair0;
    if (parts > 1) {
        // a partial result: rows of (m, sum), then rows of DIM
        float* part = a.parts + COUNTERS + (size_t)u.place * part_words(DIM);
#pragma unroll 4
        for (int e = 0; e < MY; ++e) {
            const int at = threadIdx.x + e * THREADS, r2 = at / (DIM / 4), c = at % (DIM / 4);
            if (r2 < used) {
                const f4 x = *(const f4*)piece_at(r2, c);
                put2(part + 2 * TQ + 4 * at, x[0], x[1]);
                put2(part + 2 * TQ + 4 * at + 2, x[2], x[3]);
            }
        }
        if (threadIdx.x < used) put2(part + 2 * threadIdx.x, row_m[threadIdx.x], row_l[threadIdx.x]);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) {
            unsigned* counter = (unsigned*)a.parts + u.first;
            last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == (unsigned)parts;
            if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!last) return;
        const float* src = a.parts + COUNTERS + (size_t)u.first * part_words(DIM);
        const size_t step_words = (size_t)a.kv * part_words(DIM);
        for (int e = 0; e < MY; ++e) {
            const int at = threadIdx.x + e * THREADS, r2 = at / (DIM / 4), c = at % (DIM / 4);
            if (r2 >= used) break;
            float mm = -INFINITY, ll = 0.f;
            f4 x = {0.f, 0.f, 0.f, 0.f};
            // (four at a time on their way)
            for (int c0 = 0; c0 < parts; c0 += 4) {
                float2 ml[4], y[4][2];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float* one = src + (size_t)(c0 + k < parts ? c0 + k : parts - 1) * step_words;
                    ml[k] = get2(one + 2 * r2);
                    y[k][0] = get2(one + 2 * TQ + 4 * at);
                    y[k][1] = get2(one + 2 * TQ + 4 * at + 2);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (c0 + k >= parts) break;
                    const float up = fmaxf(mm, ml[k].x), f = factor(mm, up), g = factor(ml[k].x, up);
                    ll = (mm == -INFINITY ? ll : ll * f) + (ml[k].x == -INFINITY ? ml[k].y : ml[k].y * g);
                    mm = up;
                    x = x * f + f4{y[k][0].x, y[k][0].y, y[k][1].x, y[k][1].y} * g;
                }
            }
            *(f4*)piece_at(r2, c) = x;         // (its own thread reads it below)
            if (c == 0) {
                row_m[r2] = mm;
                row_l[r2] = ll;
            }
        }
        __syncthreads();
    }
    for (int e = 0; e < MY; ++e) {
        const int at = threadIdx.x + e * THREADS, r2 = at / (DIM / 4), c = at % (DIM / 4);
        if (r2 >= used) break;
        const int pr = pair0 + r2, rw = pr / group;
        const size_t place = (size_t)(r.first + rw) * a.heads + u.h * group + (pr - rw * group);
        const float ll = row_l[r2], f = vs / ll;
        const f4 x = *(const f4*)piece_at(r2, c);
        h4 y;
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) y[q4] = (_Float16)(ll == 0.f ? 0.f : x[q4] * f);
        *(h4*)(a.out + place * DIM + 4 * c) = y;
        if (c == 0 && a.lse) a.lse[place] = LN2 * (row_m[r2] + __log2f(ll));
    }
}

template <int DIM, int BITS, bool BLOCKS>
hipError_t start(const PromptArgs& a, hipStream_t stream)
{
    constexpr int lds = lds_bytes<DIM, BITS>();
    const auto kern = prompt_kernel<DIM, BITS, BLOCKS>;
    const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    kern<<<(unsigned)prompt_units(a.M, a.B, a.heads, a.kv), THREADS, lds, stream>>>(a);
    return hipGetLastError();
}

template <int DIM>
hipError_t start(const PromptArgs& a, hipStream_t stream)
{
    if (a.bits == 16) return start<DIM, 16, false>(a, stream);
    return a.k_scales ? start<DIM, 8, true>(a, stream) : start<DIM, 8, false>(a, stream);
}

}  // namespace

long long prompt_units(int M, int B, int heads, int kv)
{
    return (((long long)M * (heads / kv) + TQ - 1) / TQ + B) * kv + MAX_PARTS;
}

size_t prompt_workspace_bytes(int dim) { return (COUNTERS + MAX_PARTS * part_words(dim)) * sizeof(float); }

hipError_t launch_prompt(const PromptArgs& a, hipStream_t stream)
{
    return a.dim == 64 ? start<64>(a, stream) : (a.dim == 128 ? start<128>(a, stream) : start<256>(a, stream));
}

}  // namespace eora
