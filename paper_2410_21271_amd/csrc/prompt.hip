// Attention of many new tokens per request (a prompt, a piece of one, some drafted tokens) over a paged key-value cache.
//
//      s_rt = scale q_r . k_t,   out_r = sum_t 2^(s_rt log2 e - m) v_t / sum_t 2^(s_rt log2 e - m)      t <= p_r, and t > p_r - window or t < sinks
//
// Row r of a request's n sits at p_r = length - n + r.  Bound by the matrix instructions where there are many rows (4 dim flops for each pair of a query head's row and a token), by memory
// where there are few.  64 / 8 heads of 128: 8192 rows in fp16 in 1510 us, 728 TF (1090 with the second halves of the weights, on a card where a large matrix product reaches
// 1470); 32 / 8 heads: 2048 rows in 70 us in fp16, 79 in 8 bits; 32 requests of 5 rows and 8192 tokens in 8 bits (537 MB) in 110 to 115 us, 4.8 TB/s; 17 rows of 17 in 9.6 us.  Times of what was not
// kept, here and below, were taken beside a kernel with one fp16 a weight, which took 1120, 56, 67, 107 and 9.2 for these.
//
// Tile: 128 pairs of a row and a query head of one kv head (32 a wavefront) by 64 keys.  A column of the matrix instructions is a pair, all query heads of a kv head share the keys.
// S^T = K Q^T (32 x 32 x 16): a lane holds one pair's scores of 16 keys of 32, so that softmax needs no exchange between lanes but one of the largest score, and the scores are,
// as weights, two fp16 each, the second operand of O^T = V^T P^T, if that takes its keys in the order in which they lie: 8 (e / 4) + 4 half + e % 4 of 16.
// K and V lie in LDS as fp16 rows, in two stages; V's operand is read transposed (ds_read_tr16_b64: four keys of a column a lane).  fp16 tiles go from memory to LDS without registers
// (by way of them a wavefront's 32 words of a tile on its way spilled: 3749 us where 1418 were left without); codes of 8 bits go there as they are, and become fp16, exactly, once,
// by the wavefront that moved them.
//
// A step: the scores of the next tile beside the softmax of this one, then this one's O, one matrix instruction a slot in an order that the compiler keeps, operands read four ahead (left to itself it
// reads one, waits, multiplies: 1418 us -> 1395).  Alone on its compute unit a workgroup takes 3480 cycles a step, 1536 of matrix instructions: 860 before the first (scalar work, masks, the
// first operands), 1420 beside the softmax, 1045 beside V, 155 for tiles and the barrier.  So there are two workgroups a compute unit, which fill each other's gaps (8192 rows: 4600 cycles a step of both, 67 % with a
// matrix instruction, at a clock that the card's power holds at 1.6 GHz).  What did not help: two teams of wavefronts on one tile of pairs (1378 us), eight wavefronts on tiles of 256 (1206, and 71 where 2048 rows take 59), 64 pairs a wavefront
// (twice the work for an operand, one wavefront a SIMD: 1.4 times as long), O one step later (registers), waits of a step and a half for tiles, scalar work between the matrix instructions.
//
// Few rows: tiles of 32 pairs by 32 keys (few_kernel() below).
//
// Softmax: as for single tokens, m is a reference (LOWER below the largest score when it is set, raised when a score has risen by RAISE more), the largest weight 2^11 to 2^15.  A weight meets
// V as two fp16, the second what cutting off the first leaves: 20.7 bits together, beside which the result's own rounding is all that shows.  (One fp16 put out off by up to 2^-11 of sum p |v|, where the
// plain definition in fp32 is off by its last rounding: 8192 rows 2.6e-4 of out's norm in place of 2.0e-4.  It took 1120 us, two take 1510: a product's matrix instructions once more, at the clock that the card's power
// holds; fewer vector instructions or another order of the two products change nothing.)  The second is positive as well: an infinite value gives an infinity (NaN where a weight is below 2^-24 of the largest).  The sum of the weights is of those that were not
// rounded, tile by tile (weight by weight, roundings of equal weights, all of one sign, put lse off by 5e-5 behind 8192 tokens and 6e-4 behind 131072; same times).  Scores, sums and O are fp32.
//
// What rows may not see: a tile that all rows of a wavefront see as a whole takes no test.  Tokens that no row of the tile sees are zeros in LDS; where some rows see a token and others do not, a value
// that is not finite would spoil a product with weights of 0: it is a zero there too, and added at the end, to the rows that see it (add_odd()).
//
// Split: tiles with more than their share of all work are cut along the keys, into equal parts by a rule on the lengths of all requests; the last part to
// arrive adds up the results of all, in the order of the keys.  Units in the order of falling work, kv heads side by side: with eight of them each XCD has the keys of one.
#include "heads.hpp"
#include "serving.hpp"

#include <utility>
#include <vector>

namespace eora {
namespace {

constexpr int RG = 4, THREADS = 64 * RG;       // wavefronts of a workgroup
// Pairs and keys of a tile, and keys of a part of it at least: of many rows (a wavefront a quarter of the pairs), and of few (a wavefront every fourth tile of keys)
struct Wide {
    static constexpr int TQ = 128, KT = 64, LEAST_PART = 8;
};
struct Narrow {
    static constexpr int TQ = 32, KT = 32, LEAST_PART = 16;
};
constexpr int CUS = 256;
// Workgroups a compute unit has at a time, as registers and LDS allow
constexpr int residents(int dim) { return dim == 256 ? 1 : 2; }
// Parts that all tiles that are cut have together, where they have the work: as many as the chip has at a time (32 requests of 5 rows of 4096 tokens, heads of 256 in 8 bits, with twice as many
// 157 us, with these 136); room for an eighth more
constexpr int want_of(int dim) { return CUS * residents(dim); }
constexpr int most_of(int dim) { return want_of(dim) * 9 / 8; }
constexpr int MAX_PARTS = most_of(128);
constexpr int COUNTERS = ATTEND_COUNTERS;      // words before the partial results: the first of them one for each tile that is cut
static_assert(MAX_PARTS <= COUNTERS, "a counter for each tile that is cut");
constexpr int PLAN_BYTES = 32;                 // of a request's plan, behind the partial results
constexpr float RAISE = 4.f, LOWER = 11.f;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

typedef uint32_t u2 __attribute__((ext_vector_type(2)));
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

// Two weights as two fp16 each: cut off, and what that leaves of ABOVE times the weight, which is positive whatever the weight is.  (The results are divided by ABOVE in the end.)
constexpr float ABOVE = 1.f + 0x1p-12f;
__device__ __forceinline__ void halves(float x, float y, h2& high, h2& low)
{
    high = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(x, y));
    low = h2{(_Float16)__builtin_fmaf(x, ABOVE, -(float)high[0]), (_Float16)__builtin_fmaf(y, ABOVE, -(float)high[1])};
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
template <typename SHAPE>
__host__ __device__ __forceinline__ Request request_of(const PromptArgs& a, int b)
{
    constexpr int TQ = SHAPE::TQ, KT = SHAPE::KT;
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
// Tiles of a request are cut into cost / share parts, rounded down, up from an eighth below: share = a want_of(dim)-th of all work, so all of them have hardly more parts than the chip
// holds workgroups.  (Rounded up, parts that do not fit wait for others to end: 1536 rows of 32 / 8 heads 52 us, these 42; always rounded down, 11 requests of 200 rows and 2000 tokens with a window of
// 1000, 1.94 shares each, 15 / 3 heads of 64: 51 us, these 43.  All tiles of a request alike, as if each saw as much as the last: each by what
// it sees, 2048 rows, whose tiles fill the chip once, would take 67 in place of 56.)
// The work is added up in floats, in one order: everyone finds the same parts.  With two or more of them cost / share is 1.875 or more: together they are 1.07 want_of(dim) at most.
__host__ __device__ __forceinline__ float shares_of(const PromptArgs& a, float work) { return (float)want_of(a.dim) / fmaxf(work * (float)a.kv, 1.f); }
template <typename SHAPE>
__host__ __device__ __forceinline__ int parts_of(const Request& r, float shares)
{
    const int most = (r.cost + SHAPE::LEAST_PART - 1) / SHAPE::LEAST_PART, parts = (int)fminf(__builtin_fmaf((float)r.cost, shares, 0.125f), (float)MAX_PARTS);
    return parts < 1 ? 1 : (parts < most ? parts : most);
}
__host__ __device__ __forceinline__ Unit unit_in(const PromptArgs& a, const Request& r, int b, int parts, int local, int cut)
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
template <typename SHAPE>
__device__ __forceinline__ bool unit_of_few(const PromptArgs& a, int id, Unit& u)
{
    const int lane = threadIdx.x & 63;
    Request r = request_of<SHAPE>(a, lane < a.B ? lane : a.B - 1);
    if (lane >= a.B) r.tiles = 0;
    const float shares = shares_of(a, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scan((float)r.tiles * (float)r.cost)), 63)));
    const int parts = parts_of<SHAPE>(r, shares), units = r.tiles * parts * a.kv, cut = parts > 1 ? units : 0;
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
// More of them: a launch before this one has written down for each request where its units end and what they are, each wavefront looks for its own.  (In place of every workgroup adding up
// all requests for itself: 5 rows of each of 128, 512, 2048 requests of 100 tokens,
// 32 / 8 heads of 128 in 8 bits, 26, 105, 593 -> 25, 83, 304 us.)
struct Planned {
    int4 at, what;                             // end of its units, parts before it, n, first; rows, tiles, parts, cost
};
// Units are counted up to here, beyond all that a launch may have (2^23): where row_starts decrease, requests share rows, and all of them together may have more units than 32 bits hold
constexpr int MOST_UNITS = 1 << 24;
__host__ __device__ __forceinline__ int counted(int units) { return units < MOST_UNITS ? units : MOST_UNITS; }
// requests [b0, b1): their units and, of them, those of tiles that are cut; then their plans, behind `end` units and `before` parts
template <typename SHAPE>
__host__ __device__ __forceinline__ void count_units(const PromptArgs& a, int b0, int b1, float shares, int& units, int& cut)
{
    units = cut = 0;
    for (int b = b0; b < b1; ++b) {
        const Request r = request_of<SHAPE>(a, b);
        const int parts = parts_of<SHAPE>(r, shares), mine = r.tiles * parts * a.kv;
        units = counted(units + mine);
        cut = counted(cut + (parts > 1 ? mine : 0));
    }
}
template <typename SHAPE>
__host__ __device__ __forceinline__ void write_plans(const PromptArgs& a, int b0, int b1, float shares, int end, int before, Planned* plan)
{
    for (int b = b0; b < b1; ++b) {
        const Request r = request_of<SHAPE>(a, b);
        const int parts = parts_of<SHAPE>(r, shares), mine = r.tiles * parts * a.kv;
        end += mine;
        plan[b].at = make_int4(end, before, r.n, r.first);
        plan[b].what = make_int4(r.rows, r.tiles, parts, r.cost);
        before += parts > 1 ? mine : 0;
    }
}
static_assert(sizeof(Planned) == PLAN_BYTES, "");
constexpr int PLAN_THREADS = 1024;
template <typename SHAPE>
__global__ __launch_bounds__(PLAN_THREADS) void plan_kernel(const PromptArgs a)
{
    constexpr int WAVES = PLAN_THREADS / 64;
    __shared__ float sums[WAVES];
    __shared__ int totals[WAVES][2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, each = (a.B + PLAN_THREADS - 1) / PLAN_THREADS;
    const int b0 = threadIdx.x * each < a.B ? threadIdx.x * each : a.B, b1 = b0 + each < a.B ? b0 + each : a.B;
    float work = 0.f;
    for (int b = b0; b < b1; ++b) {
        const Request r = request_of<SHAPE>(a, b);
        work += (float)r.tiles * (float)r.cost;
    }
    work = scan(work);
    if (lane == 63) sums[wave] = work;
    __syncthreads();
    work = 0.f;
    for (int w = 0; w < WAVES; ++w) work += sums[w];
    const float shares = shares_of(a, work);
    int units, cut;
    count_units<SHAPE>(a, b0, b1, shares, units, cut);
    const int v = scan(units), c = scan(cut);
    if (lane == 63) {
        totals[wave][0] = counted(v);
        totals[wave][1] = counted(c);
    }
    __syncthreads();
    int end = v - units, before = c - cut;
    for (int w = 0; w < wave; ++w) {
        end += totals[w][0];
        before += totals[w][1];
    }
    write_plans<SHAPE>(a, b0, b1, shares, end, before, (Planned*)a.plan);
}
__device__ __forceinline__ bool unit_planned(const PromptArgs& a, int id, Unit& u)
{
    const Planned* plan = (const Planned*)a.plan;
    const int lane = threadIdx.x & 63, each = (a.B + 63) / 64;
    // the first of 64 stretches of requests that ends behind this unit, then the first request of it
    const int stop = (lane + 1) * each < a.B ? (lane + 1) * each : a.B;
    const unsigned long long stretches = __ballot(id < plan[stop - 1].at.x);
    if (stretches == 0) return false;
    const int begin = __builtin_ctzll(stretches) * each;
    for (int b0 = begin; b0 < begin + each; b0 += 64) {
        const int b = b0 + lane < a.B ? b0 + lane : a.B - 1;
        const int4 at = plan[b].at, what = plan[b].what;
        const unsigned long long mine = __ballot(id < at.x);
        if (mine == 0) continue;               // (a stretch of more than 64 requests)
        const int from = __builtin_ctzll(mine);
        auto of = [&](int x) { return __builtin_amdgcn_readlane(x, from); };
        Request r;
        r.n = of(at.z);
        r.first = of(at.w);
        r.rows = of(what.x);
        r.tiles = of(what.y);
        r.cost = of(what.w);
        const int parts = of(what.z);
        u = unit_in(a, r, b0 + from, parts, id - (of(at.x) - r.tiles * parts * a.kv), of(at.y));
        return true;
    }
    return false;
}

// Stores and loads of partial results go past the caches of an XCD (agent scope: SC1), 16 bytes each, or a pair
constexpr int AGENT = 16;
struct Partial {
    __amdgpu_buffer_rsrc_t at;
    __device__ __forceinline__ Partial(float* p, size_t words) : at(__builtin_amdgcn_make_buffer_rsrc(p, 0, (int)(words * sizeof(float)), 0x00027000)) {}
    __device__ __forceinline__ void put(int word, f4 x) const { __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, x), at, 4 * word, 0, AGENT); }
    __device__ __forceinline__ void put(int word, float2 x) const { __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u2, x), at, 4 * word, 0, AGENT); }
    __device__ __forceinline__ f4 get(int word) const { return __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(at, 4 * word, 0, AGENT)); }
    __device__ __forceinline__ float2 get2(int word) const { return __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(at, 4 * word, 0, AGENT)); }
};
__device__ __forceinline__ float factor(float m, float to) { return m == -INFINITY ? 0.f : exp2_(m - to); }

// f(0) .. f(N - 1), each number a type
template <int N, typename F, int... I>
__device__ __forceinline__ void each_of(const F& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void each_piece(const F& f) { each_of<N>(f, std::make_integer_sequence<int, N>{}); }

// words of a partial result: (m, sum) and O of each pair
template <typename SHAPE>
constexpr size_t part_words(int dim) { return (size_t)SHAPE::TQ * (dim + 2); }

// A tile's part in LDS, fp16: K's rows in groups of 1 KiB, as they come from memory, with a gap behind each group; then V's rows.  Pieces of 16 bytes change places in the row of a key, so that the
// lanes that read at a time meet different banks: 16 keys' pieces of the same columns; two units of 32 bytes of four keys.
template <int DIM, int KT>
struct Stage {
    static constexpr int ROW = 2 * DIM, GROUP = 512 / DIM, PITCH = 1024 + (DIM == 256 ? 32 : 64);
    static constexpr int VALUES = KT / GROUP * PITCH, BYTES = VALUES + KT * ROW;
    static constexpr int BLOCK_OF_KEYS = 32 / GROUP * PITCH;
    __device__ static __forceinline__ int k_turn(int key) { return DIM == 64 ? key >> 1 & 3 : (DIM == 128 ? key & 3 : key & 1); }
    __device__ static __forceinline__ int v_turn(int key) { return 4 * (DIM == 64 ? key >> 1 & 1 : key & 3); }
    __device__ static __forceinline__ int k_place(int key, int piece) { return key / GROUP * PITCH + key % GROUP * ROW + 16 * (piece ^ k_turn(key)); }
    __device__ static __forceinline__ int v_place(int key, int piece) { return VALUES + key * ROW + 16 * (piece ^ v_turn(key)); }
    // where a lane reads: K, row lane % 32: piece 2 t + lane / 32; V, transposed: rows 4 (lane / 32) + lane % 16 / 4, columns 16 (lane / 16 % 2) + 4 (lane % 4) of 32
    int k_at, k_way, v_at, v_way;
    __device__ __forceinline__ explicit Stage(int lane)
    {
        const int col = lane & 31, half = lane >> 5, v_key = 4 * half + (lane & 15) / 4;
        k_at = col / GROUP * PITCH + col % GROUP * ROW;
        k_way = half ^ k_turn(col);
        v_at = VALUES + v_key * ROW + 8 * (lane & 3);
        v_way = (lane >> 4 & 1) ^ (v_turn(v_key) / 2);
    }
    // columns 16 t .. + 15 of keys 32 b .. + 31; keys 16 s .. + 15 of columns 32 d .. + 31
    __device__ __forceinline__ void keys(const unsigned char* base, int b, int t, Frag& f) const { f.q = *(const u4*)(base + k_at + b * BLOCK_OF_KEYS + 16 * ((2 * t) ^ k_way)); }
    __device__ __forceinline__ void values(const unsigned char* base, int s, int d, Frag& f) const
    {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const auto w = __builtin_amdgcn_ds_read_tr16_b64_v4f16((tr4_lds)(base + v_at + (16 * s + 8 * e) * ROW + 32 * ((2 * d) ^ v_way)));
            __builtin_memcpy(&f.u[2 * e], &w, 8);
        }
    }
};
// 16 codes, times a power of two
__device__ __forceinline__ void spread(const u4& w, float scale, Frag (&f)[2])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[e / 2].p[2 * (e % 2)] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[e], scale, false);
        f[e / 2].p[2 * (e % 2) + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[e], scale, true);
    }
}

// A tile of pairs, and which of the keys its rows see
template <typename SHAPE>
struct Tile {
    static constexpr int TQ = SHAPE::TQ, KT = SHAPE::KT;
    Unit u;
    int group, pair0, pair1;                   // its pairs: [pair0, pair1)
    int from, low, high;                       // positions of the request's row 0 (below 0: rows that see nothing), of the tile's first row and of its last
    int lo, hi, sinks, first, head;            // tokens that some row sees: [lo, hi) and those before `sinks`; tiles of keys: those from `first` on, behind `head` of the first
    int parts, k0, k1;                         // tiles [k0, k1) of them are this workgroup's
    const int* table;
    __device__ __forceinline__ bool find(const PromptArgs& a, int id)
    {
        return (a.B <= 64 ? unit_of_few<SHAPE>(a, id, u) : unit_planned(a, id, u)) && set(a);
    }
    __host__ __device__ __forceinline__ bool set(const PromptArgs& a)            // u is known
    {
        group = a.heads / a.kv;
        const int pairs = u.r.rows * group;
        from = u.r.n - u.r.rows;
        pair0 = u.tile * TQ;
        pair1 = pair0 + TQ < pairs ? pair0 + TQ : pairs;
        low = from + pair0 / group;
        high = from + (pair1 - 1) / group;
        hi = high + 1 < 0 ? 0 : high + 1;
        lo = a.window > 0 && low - a.window + 1 > 0 ? low - a.window + 1 : 0;
        if (lo <= a.sinks) lo = 0;
        sinks = lo > 0 ? a.sinks : 0;
        first = lo / KT;
        head = (sinks + KT - 1) / KT;
        head = head < first ? head : first;
        int tiles = (hi + KT - 1) / KT - first + head;
        tiles = tiles > 0 ? tiles : 0;
        parts = (tiles + SHAPE::LEAST_PART - 1) / SHAPE::LEAST_PART;
        parts = parts < 1 ? 1 : (parts < u.parts ? parts : u.parts);
        if (u.part >= parts) return false;
        k0 = (int)((long long)tiles * u.part / parts);
        k1 = (int)((long long)tiles * (u.part + 1) / parts);
        table = a.table + (size_t)u.b * a.width;
        return true;
    }
    __device__ __forceinline__ int key_of(int i) const { return (i < head ? i : i - head + first) * KT; }
    // the block of 16 tokens that a key (a multiple of 16) begins: page, head and place in one number; -1: no page
    __device__ __forceinline__ int block_at(const PromptArgs& a, int key) const
    {
        const int p = key / a.page, page = table[p];
        return (unsigned)page < (unsigned)a.n_pages ? (page * a.kv + u.h) * (a.page / BLOCK_TOKENS) + (key - p * a.page) / BLOCK_TOKENS : -1;
    }
    __device__ __forceinline__ unsigned gone_at(const PromptArgs& a, int key0) const
    {
        unsigned gone = 0;
        for (int g = 0; g < KT / BLOCK_TOKENS; ++g) gone |= (unsigned)(key0 + BLOCK_TOKENS * g < hi && block_at(a, key0 + BLOCK_TOKENS * g) < 0) << g;
        return gone;
    }
    // whether a tile's values can go to LDS as they are: all rows see all of its tokens
    __device__ __forceinline__ bool plain(const PromptArgs& a, int key0, unsigned gone) const
    {
        return gone == 0 && key0 + KT <= low + 1 && (a.window == 0 || key0 > high - a.window || key0 + KT <= a.sinks);
    }
    // Eight values of a token: one that no row sees becomes zeros, and so do values that are not finite where some rows see them and others do not: those are added at the end.
    __device__ __forceinline__ void clean(Frag& f, int at, bool gone, int& odd_one) const
    {
        const bool seen = at < hi && (at >= lo || at < sinks) && !gone;
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = seen ? f.u[e] : 0u;
            const uint32_t low_half = (x & 0x7c00u) == 0x7c00u ? 0xffffu : 0u, high_half = (x & 0x7c000000u) == 0x7c000000u ? 0xffff0000u : 0u;
            odd |= (low_half | high_half) != 0;
            f.u[e] = x & ~(low_half | high_half);
        }
        if (odd) odd_one = 1;
    }
};

// Where pieces of four columns of the results lie in LDS, rows of fp32: they change places within their row, so that the lanes that write at a time meet different banks
template <int DIM>
__device__ __forceinline__ float* piece_at(float* sum, int row, int c) { return sum + row * DIM + 4 * (c ^ (row & 15)); }

// Values that are not finite, in tiles of which not all rows see all: for the rows that see them, unless their score is -inf
template <int DIM, int BITS, typename SHAPE>
__device__ __forceinline__ void add_odd(const PromptArgs& a, const Tile<SHAPE>& t, float scale, float* sum)
{
    for (int e = threadIdx.x; e < SHAPE::TQ * (DIM / 4); e += THREADS) {
        const int r = e / (DIM / 4), c = e % (DIM / 4), pair = t.pair0 + r;
        if (pair >= t.pair1) continue;
        const int row = pair / t.group, pos = t.from + row, head = t.u.h * t.group + pair - row * t.group;
        f4 add = {0.f, 0.f, 0.f, 0.f};
        for (int i = t.k0; i < t.k1; ++i) {
            const int key0 = t.key_of(i);
            if (t.plain(a, key0, t.gone_at(a, key0))) continue;
            for (int key = key0; key < key0 + SHAPE::KT && key <= pos; ++key) {
                if (!(a.window == 0 || key > pos - a.window || key < a.sinks)) continue;
                const int block = t.block_at(a, key & ~(BLOCK_TOKENS - 1));
                if (block < 0) continue;
                const size_t at = ((size_t)(unsigned)block * BLOCK_TOKENS + key % BLOCK_TOKENS) * DIM;
                bool any = false;
                float v[4];
                for (int k = 0; k < 4; ++k) {
                    if constexpr (BITS == 16) v[k] = (float)((const _Float16*)a.pages_v)[at + 4 * c + k];
                    else v[k] = (((const uint8_t*)a.pages_v)[at + 4 * c + k] & 127) == 127 ? __builtin_nanf("") : 0.f;
                    any |= !(fabsf(v[k]) < INFINITY);
                }
                if (!any) continue;
                if constexpr (BITS == 16) {
                    const _Float16 *x = a.q + (size_t)(t.u.r.first + row) * a.q_stride + (size_t)head * DIM, *y = (const _Float16*)a.pages_k + at;
                    float score = 0.f;
                    for (int k = 0; k < DIM; ++k) score += (float)x[k] * (float)y[k];
                    if (score * scale == -INFINITY) continue;
                }
                for (int k = 0; k < 4; ++k) add[k] += fabsf(v[k]) < INFINITY ? 0.f : v[k];
            }
        }
        *(f4*)piece_at<DIM>(sum, r, c) += add;
    }
}

// The results of a tile, or of a part of one, from LDS (O's rows, (m, sum) of each) to where they belong.  All threads, behind a barrier.
template <int DIM, typename SHAPE>
__device__ __forceinline__ void finish(const PromptArgs& a, const Tile<SHAPE>& t, float vs, float* sum, float* row_m, float* row_l, int& last)
{
    constexpr int TQ = SHAPE::TQ, MY = TQ * (DIM / 4) / THREADS;                 // pieces of four columns: thread after thread along the rows
    constexpr size_t WORDS = part_words<SHAPE>(DIM);
    const int used = t.pair1 - t.pair0, parts = t.parts;
    if (parts > 1) {
        // a partial result: rows of (m, sum), then rows of DIM
        const Partial part(a.parts + COUNTERS + (size_t)t.u.place * WORDS, WORDS);
#pragma unroll 4
        for (int e = 0; e < MY; ++e) {
            const int at = threadIdx.x + e * THREADS, r = at / (DIM / 4), c = at % (DIM / 4);
            if (r < used) part.put(2 * TQ + 4 * at, *(const f4*)piece_at<DIM>(sum, r, c));
        }
        if (threadIdx.x < used) part.put(2 * threadIdx.x, make_float2(row_m[threadIdx.x], row_l[threadIdx.x]));
        arrived();
        __syncthreads();
        if (threadIdx.x == 0) {
            unsigned* counter = (unsigned*)a.parts + t.u.first;
            last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == (unsigned)parts;
            if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!last) return;
        float* src = a.parts + COUNTERS + (size_t)t.u.first * WORDS;
        const size_t step_words = (size_t)a.kv * WORDS;
        // (16 pieces of 16 bytes a thread on their way at a time, not eight of 8 bytes twice: 512 rows behind 7680 tokens 96 -> 91 us, 1536 rows 59.5 -> 52)
        constexpr int BATCH = MY < 8 ? MY : 8, AT_ONCE = 2;
        static_assert(MY % BATCH == 0, "");
        for (int e0 = 0; e0 < MY; e0 += BATCH) {
            if ((threadIdx.x + e0 * THREADS) / (DIM / 4) >= used) break;
            int at[BATCH], r[BATCH], c[BATCH];
            float m[BATCH], l[BATCH];
            f4 x[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int e = e0 + i < MY ? e0 + i : MY - 1, there = threadIdx.x + e * THREADS;
                at[i] = there / (DIM / 4) < used ? there : threadIdx.x + e0 * THREADS;          // (behind the last row: the first of the batch again)
                r[i] = at[i] / (DIM / 4);
                c[i] = at[i] % (DIM / 4);
                m[i] = -INFINITY;
                l[i] = 0.f;
                x[i] = f4{0.f, 0.f, 0.f, 0.f};
            }
            for (int p0 = 0; p0 < parts; p0 += AT_ONCE) {
                float2 ml[AT_ONCE][BATCH];
                f4 y[AT_ONCE][BATCH];
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    const Partial one(src + (size_t)(p0 + k < parts ? p0 + k : parts - 1) * step_words, WORDS);
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
                        ml[k][i] = one.get2(2 * r[i]);
                        y[k][i] = one.get(2 * TQ + 4 * at[i]);
                    }
                }
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    if (p0 + k >= parts) break;
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
                        const float mk = ml[k][i].x, up = fmaxf(m[i], mk), f = factor(m[i], up), g = factor(mk, up);
                        l[i] = (m[i] == -INFINITY ? l[i] : l[i] * f) + (mk == -INFINITY ? ml[k][i].y : ml[k][i].y * g);
                        m[i] = up;
                        x[i] = x[i] * f + y[k][i] * g;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                *(f4*)piece_at<DIM>(sum, r[i], c[i]) = x[i];                     // (its own thread reads it below)
                if (c[i] == 0) {
                    row_m[r[i]] = m[i];
                    row_l[r[i]] = l[i];
                }
            }
        }
        __syncthreads();
    }
    for (int e = 0; e < MY; ++e) {
        const int at = threadIdx.x + e * THREADS, r = at / (DIM / 4), c = at % (DIM / 4);
        if (r >= used) break;
        const int pair = t.pair0 + r, row = pair / t.group;
        const size_t place = (size_t)(t.u.r.first + row) * a.heads + t.u.h * t.group + (pair - row * t.group);
        const float l = row_l[r], f = vs / l;
        const f4 x = *(const f4*)piece_at<DIM>(sum, r, c);
        h4 y;
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = (_Float16)(l == 0.f ? 0.f : x[k] * f);
        *(h4*)(a.out + place * DIM + 4 * c) = y;
        if (c == 0 && a.lse) a.lse[place] = LN2 * (row_m[r] + __log2f(l));
    }
}

// A lane's operand of q: pair `pair` of the tile's, its sign that of the scores' scale.  The scale's size is applied to the scores, where no value of a masked one may come of it: a scale that is 0 or not
// finite (a head's, of a cache of 8 bits) goes into q, so that scores are 0 or, of what is not finite on either side, NaN.
template <int DIM>
__device__ __forceinline__ void load_q(const PromptArgs& a, const Unit& u, int group, int pair, bool there, int half, float scale, Frag (&q)[DIM / 16])
{
    const int row = there ? pair / group : 0, head = u.h * group + (there ? pair - row * group : 0);
    const _Float16* at = a.q + (size_t)(u.r.first + row) * a.q_stride + (size_t)head * DIM + 8 * half;
    const uint32_t sign = scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int t = 0; t < DIM / 16; ++t) {
        const u4 w = *(const u4*)(at + 16 * t);
#pragma unroll
        for (int e = 0; e < 4; ++e) q[t].u[e] = there ? w[e] ^ sign : 0u;
    }
    if (scale == 0.f || !(fabsf(scale) < INFINITY)) {
        const _Float16 by = (_Float16)(scale == 0.f ? 0.f : __builtin_nanf(""));
#pragma unroll
        for (int t = 0; t < DIM / 16; ++t) q[t].v *= by;
    }
}
// ... and that size, for scores that are finite or -inf
__device__ __forceinline__ float size_of(float scale) { return fabsf(scale) < INFINITY ? fmaxf(fabsf(scale), 0x1p-100f) : 1.f; }
__device__ __forceinline__ float both_halves(float v)
{
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}

template <int DIM, int BITS, bool BLOCKS>
__global__ __launch_bounds__(THREADS, residents(DIM)) void prompt_kernel(const PromptArgs a)
{
    constexpr int TQ = Wide::TQ, KT = Wide::KT;
    typedef Stage<DIM, KT> St;
    constexpr int ROW = St::ROW, PITCH = St::PITCH, STAGE = St::BYTES, VALUES = St::VALUES;
    constexpr int NK = DIM / 16, ND = DIM / 32;                   // k-steps of the first product, blocks of O^T
    constexpr int BYTES = DIM * BITS / 8;      // of a row in memory
    constexpr int PIECES = BLOCK_TOKENS * BYTES / 1024;           // KiB of a wavefront's 16 keys (or values) of a tile
    constexpr int AHEAD = 4;                   // matrix instructions between an operand's read and its use

    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ int odd_one;                    // some value that not all rows see is not finite
    __shared__ int last;
    __shared__ float row_m[TQ], row_l[TQ];

    Tile<Wide> tile;
    if (!tile.find(a, (int)blockIdx.x)) return;
    const Unit& u = tile.u;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int steps = tile.k1 - tile.k0;

    // this lane's pair, and the positions that this wavefront's pairs have
    const int w0 = tile.pair0 + 32 * wave, w1 = w0 + 32 < tile.pair1 ? w0 + 32 : tile.pair1;         // (w1 <= w0: no pair)
    const int wlow = tile.from + w0 / tile.group, whigh = w1 > w0 ? tile.from + (w1 - 1) / tile.group : -1;
    const bool all = w1 - w0 == 32, there = w0 + col < tile.pair1;
    const int pos = there ? tile.from + (w0 + col) / tile.group : -1;

    // Blocks of 16 tokens of the next 64 groups of 16 keys: lane 4 i + g has where that of group g of its tile i begins in the cache, in bytes (0: no page, or no key that a
    // row sees: those are in `lost`), and its scales
    unsigned off_low = 0, off_high = 0;
    unsigned k_byte = 0, v_byte = 0;
    unsigned long long lost = 0;
    auto tile_at = [&](int i) { return tile.key_of(tile.k0 + i); };
    auto look = [&](int i0) {
        const int i = i0 + (lane >> 2), key = i < steps ? tile_at(i) + 16 * (lane & 3) : tile.hi, block = key < tile.hi ? tile.block_at(a, key) : -1;
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
    // A wavefront moves the tile's group of 16 keys that has its number, a KiB at a time: this lane's row of the KiB, and its piece of 16 bytes of it
    constexpr int PR = BYTES / 16, ROWS = 64 / PR;
    const int lrow = lane / PR, lpiece = lane % PR;
    auto block_of = [&](int i) {
        const int from_lane = 4 * (i & 15) + wave;
        return (unsigned long long)__builtin_amdgcn_readlane(off_high, from_lane) << 32 | __builtin_amdgcn_readlane(off_low, from_lane);
    };
    auto power_at = [&](unsigned bytes, int i) { return BLOCKS ? power_of(__builtin_amdgcn_readlane(bytes, 4 * (i & 15) + wave)) : 1.f; };
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem, aside = lds0 + 2 * STAGE;      // (what nobody reads)
    constexpr int K_MINE = BLOCK_TOKENS / St::GROUP * PITCH, V_MINE = BLOCK_TOKENS * ROW;           // a wavefront's part of a stage
    // fp16: pieces change places on the way, as the addresses say.  8 bits: codes as they are, at the beginning of the wavefront's part; it spreads them out there itself
    const unsigned linear = 16u * lane, k_off = BITS == 16 ? (unsigned)(lrow * ROW + 16 * (lpiece ^ St::k_turn(lrow))) : linear;
    const unsigned v_off = BITS == 16 ? (unsigned)(lrow * ROW + 16 * (lpiece ^ St::v_turn(lrow))) : linear;
    auto send_keys = [&](const char* base, auto piece, int stage) {
        constexpr int e = decltype(piece)::value, far = e / 4 * 4096, off = e % 4 * 1024;
        memory_to_lds<off>(base + far, k_off, lds0 + (unsigned)(stage * STAGE + wave * K_MINE + (BITS == 16 ? e * PITCH - off : far)));
    };
    auto send_values = [&](const char* base, auto piece, unsigned to) {         // (of heads of 256 a KiB has two of the four keys whose pieces change places together)
        constexpr int e = decltype(piece)::value, far = e / 4 * 4096, off = e % 4 * 1024;
        memory_to_lds<off>(base + far, BITS == 16 && DIM == 256 && e % 2 ? v_off ^ 128u : v_off, to + far);
    };
    auto values_to = [&](int stage) { return lds0 + (unsigned)(stage * STAGE + VALUES + wave * V_MINE); };
    auto spread_keys = [&](int stage, float scale) {
        unsigned char* to = smem + stage * STAGE;
        u4 w[PIECES];
#pragma unroll
        for (int e = 0; e < PIECES; ++e) w[e] = *(const u4*)(to + wave * K_MINE + e * 1024 + linear);
#pragma unroll
        for (int e = 0; e < PIECES; ++e) {
            Frag f[2];
            spread(w[e], scale, f);
#pragma unroll
            for (int h = 0; h < 2; ++h) *(u4*)(to + St::k_place(BLOCK_TOKENS * wave + e * ROWS + lrow, 2 * lpiece + h)) = f[h].q;
        }
    };
    auto spread_values = [&](int stage, float scale, int key0, unsigned gone, bool as_it_is) {
        unsigned char* to = smem + stage * STAGE;
        u4 w[PIECES];
#pragma unroll
        for (int e = 0; e < PIECES; ++e) w[e] = *(const u4*)(to + VALUES + wave * V_MINE + e * 1024 + linear);
#pragma unroll
        for (int e = 0; e < PIECES; ++e) {
            Frag f[2];
            spread(w[e], scale, f);
            const int key = BLOCK_TOKENS * wave + e * ROWS + lrow;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!as_it_is) tile.clean(f[h], key0 + key, gone >> wave & 1, odd_one);
                *(u4*)(to + St::v_place(key, 2 * lpiece + h)) = f[h].q;
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
            tile.clean(f[e], key0 + key, gone >> wave & 1, odd_one);
            *(u4*)(smem + stage * STAGE + St::v_place(key, lpiece)) = f[e].q;
        }
    };

    // q, its sign that of the scale
    const float scale = a.scale * LOG2E * (BITS == 8 && !BLOCKS ? a.k_scale[u.h] : 1.f), by = size_of(scale);
    Frag q[NK];
    load_q<DIM>(a, u, tile.group, w0 + col, there, half, scale, q);
    f16x O[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) O[d] = f16x{};
    float m = -INFINITY, l = 0.f;

    const St st(lane);
    auto first_product = [&](const unsigned char* base, f16x (&S)[2]) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f16x z = {};
#pragma unroll
            for (int t = 0; t < NK; ++t) {
                Frag k;
                st.keys(base, b, t, k);
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
        const bool as_it_is = tile.plain(a, key0, gone);
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
        const bool as_it_is = tile.plain(a, key_next, gone_next);
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
            Frag kf[AHEAD], vf[AHEAD], high[4], low[4];
            float sum = 0.f;                   // of this tile's weights
            auto read_k = [&](int x) { st.keys(next, x % 2, x / 2, kf[x % AHEAD]); };
            auto read_v = [&](int x) { st.values(base, x / ND, x % ND, vf[x % AHEAD]); };
            auto weights = [&](int x) {        // elements 2 x and 2 x + 1
                const int b = x / 8, e = 2 * x % 16;
                const float v = exp2_(__builtin_fmaf(S[b][e], by, -ref)), w = exp2_(__builtin_fmaf(S[b][e + 1], by, -ref));
                sum += v;
                sum += w;
                halves(v, w, high[2 * b + e / 8].p[e % 8 / 2], low[2 * b + e / 8].p[e % 8 / 2]);
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
            l += sum;
#pragma unroll
            for (int x = 0; x < 4 * ND; ++x) {
                const int s = x / ND, d = x % ND;
                O[d] = mfma32(vf[x % AHEAD].v, high[s].v, O[d]);
                O[d] = mfma32(vf[x % AHEAD].v, low[s].v, O[d]);
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
    l = both_halves(l);

    // The results go to LDS (all have passed the loop's last barrier).  This lane's elements: columns 32 d + 8 q + 4 half of row 32 wave + col
    float* sum = (float*)smem;
    if (half == 0) {
        row_m[32 * wave + col] = m;
        row_l[32 * wave + col] = l;
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) *(f4*)piece_at<DIM>(sum, 32 * wave + col, 8 * d + 2 * e + half) = f4{O[d][4 * e], O[d][4 * e + 1], O[d][4 * e + 2], O[d][4 * e + 3]};
    __syncthreads();
    if (odd_one) {
        add_odd<DIM, BITS>(a, tile, scale, sum);
        __syncthreads();
    }
    finish<DIM>(a, tile, (BITS == 8 && !BLOCKS ? a.v_scale[u.h] : 1.f) * (1.f / ABOVE), sum, row_m, row_l, last);
}

// Few rows, which leave the matrix instructions idle: bound by memory.  Tiles of 32 pairs (one column block) by 32 keys; each wavefront has every fourth tile of keys for itself, with LDS
// of its own and no barrier, the next one on its way to its registers meanwhile: 64 KiB on their way a compute unit in fp16.  The four add up at the end.  (32 requests of 5 rows and 8192 tokens:
// 110 us; with the tiles of many rows, of which three wavefronts of four have no pair and all wait for each other at every tile, 270.)
template <int DIM, int BITS, bool BLOCKS>
__global__ __launch_bounds__(THREADS, residents(DIM)) void few_kernel(const PromptArgs a)
{
    constexpr int TQ = Narrow::TQ, KT = Narrow::KT;
    typedef Stage<DIM, KT> St;
    constexpr int NK = DIM / 16, ND = DIM / 32;
    constexpr int BYTES = DIM * BITS / 8, PIECES = BLOCK_TOKENS * BYTES / 1024, PR = BYTES / 16, ROWS = 64 / PR;      // of a row in memory; KiB of 16 keys; pieces of a row, rows of a KiB

    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ int odd_one, last;
    __shared__ float red_m[RG][TQ], red_l[RG][TQ], row_m[TQ], row_l[TQ];

    Tile<Narrow> tile;
    if (!tile.find(a, (int)blockIdx.x)) return;
    const Unit& u = tile.u;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int mine = (tile.k1 - tile.k0 - wave + RG - 1) / RG;                   // tiles of keys
    const bool all = tile.pair1 - tile.pair0 == TQ, there = tile.pair0 + col < tile.pair1;
    const int pos = there ? tile.from + (tile.pair0 + col) / tile.group : -1;
    if (threadIdx.x == 0) odd_one = 0;
    __syncthreads();

    // Blocks of 16 tokens of the next 32 tiles: lane 2 i + g has that of group g of tile i (-1: no page, or no key that a row sees)
    int block_of = -1;
    unsigned k_byte = 0, v_byte = 0;
    auto key_at = [&](int i) { return tile.key_of(tile.k0 + wave + RG * i); };
    auto look = [&](int i0) {
        const int i = i0 + (lane >> 1), key = i < mine ? key_at(i) + BLOCK_TOKENS * (lane & 1) : tile.hi;
        block_of = key < tile.hi ? tile.block_at(a, key) : -1;
        if constexpr (BLOCKS) {
            k_byte = block_of < 0 ? 0 : a.k_scales[block_of];
            v_byte = block_of < 0 ? 0 : a.v_scales[block_of];
        }
    };
    u4 mk[2][PIECES], mv[2][PIECES];
    float k_by[2], v_by[2];
    unsigned gone = 0;
    auto load = [&](int i) {
        gone = 0;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int from = 2 * (i & 31) + g, block = __builtin_amdgcn_readlane(block_of, from);
            gone |= (unsigned)(block < 0) << g;
            const size_t at = (size_t)(unsigned)(block < 0 ? 0 : block) * (BLOCK_TOKENS * BYTES);
#pragma unroll
            for (int e = 0; e < PIECES; ++e) {
                mk[g][e] = *(const u4*)((const char*)a.pages_k + at + (e * 1024 + 16u * lane));
                mv[g][e] = *(const u4*)((const char*)a.pages_v + at + (e * 1024 + 16u * lane));
            }
            k_by[g] = BLOCKS ? power_of(__builtin_amdgcn_readlane(k_byte, from)) : 1.f;
            v_by[g] = BLOCKS ? power_of(__builtin_amdgcn_readlane(v_byte, from)) : 1.f;
        }
    };
    unsigned char* base = smem + wave * St::BYTES;
    auto put = [&](int key0) {
        const bool as_it_is = tile.plain(a, key0, gone);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int e = 0; e < PIECES; ++e) {
                constexpr int HALVES = BITS == 16 ? 1 : 2;
                const int key = BLOCK_TOKENS * g + e * ROWS + lane / PR, piece = HALVES * (lane % PR);
                Frag k[2], v[2];
                if constexpr (BITS == 16) {
                    k[0].q = mk[g][e];
                    v[0].q = mv[g][e];
                } else {
                    spread(mk[g][e], k_by[g], k);
                    spread(mv[g][e], v_by[g], v);
                }
#pragma unroll
                for (int h = 0; h < HALVES; ++h) {
                    if (!as_it_is) tile.clean(v[h], key0 + key, gone >> g & 1, odd_one);
                    *(u4*)(base + St::k_place(key, piece + h)) = k[h].q;
                    *(u4*)(base + St::v_place(key, piece + h)) = v[h].q;
                }
            }
    };

    const float scale = a.scale * LOG2E * (BITS == 8 && !BLOCKS ? a.k_scale[u.h] : 1.f), by = size_of(scale);
    Frag q[NK];
    load_q<DIM>(a, u, tile.group, tile.pair0 + col, there, half, scale, q);
    f16x O[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) O[d] = f16x{};
    float m = -INFINITY, l = 0.f;
    const St st(lane);
    if (mine > 0) {
        look(0);
        load(0);
    }
    for (int i = 0; i < mine; ++i) {
        const int key0 = key_at(i);
        const unsigned missing = gone;
        put(key0);
        if (i + 1 < mine) {
            if (((i + 1) & 31) == 0) look(i + 1);
            load(i + 1);
        }
        f16x S = {};
#pragma unroll
        for (int t = 0; t < NK; ++t) {
            Frag k;
            st.keys(base, 0, t, k);
            S = mfma32(k.v, q[t].v, S);
        }
        const bool whole = all && missing == 0 && key0 + KT <= tile.low + 1 && (a.window == 0 || key0 > tile.high - a.window || key0 + KT <= a.sinks);
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int key = key0 + 8 * (e / 4) + 4 * half + e % 4;
                const bool seen = key <= pos && (a.window == 0 || key > pos - a.window || key < a.sinks) && !(missing >> (e / 8) & 1);
                S[e] = seen ? S[e] : -INFINITY;
            }
        }
        float top = S[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(top, S[e]);
        top *= by;
        if (__any(top > m + (RAISE + LOWER))) {
            top = max_of_halves(top);
            const float up = top > m + (RAISE + LOWER) ? top - LOWER : m, f = m == up ? 1.f : exp2_(m - up);
            m = up;
            l *= f;
#pragma unroll
            for (int d = 0; d < ND; ++d) O[d] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        Frag high[2], low[2];
        float sum = 0.f;                       // of this tile's weights
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float x = exp2_(__builtin_fmaf(S[e], by, -ref)), y = exp2_(__builtin_fmaf(S[e + 1], by, -ref));
            sum += x;
            sum += y;
            halves(x, y, high[e / 8].p[e % 8 / 2], low[e / 8].p[e % 8 / 2]);
        }
        l += sum;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                Frag v;
                st.values(base, s, d, v);
                O[d] = mfma32(v.v, high[s].v, O[d]);
                O[d] = mfma32(v.v, low[s].v, O[d]);
            }
    }
    l = both_halves(l);

    // The four wavefronts' results, added up in LDS
    if (half == 0) {
        red_m[wave][col] = m;
        red_l[wave][col] = l;
    }
    __syncthreads();
    float up = red_m[0][col];
#pragma unroll
    for (int w = 1; w < RG; ++w) up = fmaxf(up, red_m[w][col]);
    const float f = factor(m, up);
    float* sum = (float*)smem;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            *(f4*)piece_at<DIM>(sum + wave * TQ * DIM, col, 8 * d + 2 * e + half) = f4{O[d][4 * e] * f, O[d][4 * e + 1] * f, O[d][4 * e + 2] * f, O[d][4 * e + 3] * f};
    if (wave == 0 && half == 0) {
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < RG; ++w) total += red_m[w][col] == -INFINITY ? red_l[w][col] : red_l[w][col] * exp2_(red_m[w][col] - up);
        row_m[col] = up;
        row_l[col] = total;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < TQ * (DIM / 4); e += THREADS) {
        f4 x = *(const f4*)(sum + 4 * e);
#pragma unroll
        for (int w = 1; w < RG; ++w) x += *(const f4*)(sum + w * TQ * DIM + 4 * e);
        *(f4*)(sum + 4 * e) = x;
    }
    __syncthreads();
    if (odd_one) {
        add_odd<DIM, BITS>(a, tile, scale, sum);
        __syncthreads();
    }
    finish<DIM>(a, tile, (BITS == 8 && !BLOCKS ? a.v_scale[u.h] : 1.f) * (1.f / ABOVE), sum, row_m, row_l, last);
}

// Tiles of tq pairs at most, and the parts that some are cut into
long long units_of(int M, int B, int heads, int kv, int tq) { return (((long long)M * (heads / kv) + tq - 1) / tq + B) * kv + MAX_PARTS; }

// Narrow tiles up to so many pairs of a request's rows and a kv head's query heads, on the average (32 requests of 8192 tokens, 32 / 8 heads of 128 in 8 bits, 5, 16, 20 rows each: narrow 110,
// 162, 299 us, wide 270, 179, 281), or so many wide tiles in all, which would leave much of the chip idle: as many as make narrow ones for the chip once where the table has room for short contexts only, fewer where
// it has for long ones, over which wide ones read LDS less often (384, 512, 640 rows of 32 / 8 heads in fp16: narrow 14.2, 15.8, 23.4 us, wide 19.6, 22.5, 25.7; behind 1024 tokens 28, 32, 55 and 37, 39, 42;
// behind 4096 72, 83, 130 and 62, 76, 87; 256 rows 11.7, 24.8, 51.0 and 17.2, 30.4, 57.7; heads of 64 and 8 bits alike).  The lengths are on the device: in a table with more room short contexts get what
// suits long ones (384 and 512 rows in one for 131072 tokens 19.6 and 22.7 us).  Heads of 256 in fp16 have no registers for a narrow tile on its way (32 x 5 rows of
// 4096: narrow 302 us, wide 275, with one fp16 a weight).
constexpr int FEW_PAIRS = 64, FEW_TILES = 64, FEW_TILES_SHORT = 128, SHORT = 2048;

bool takes_narrow(const PromptArgs& a)
{
    const int tiles = a.dim < 256 && (long long)a.width * a.page <= SHORT ? FEW_TILES_SHORT : FEW_TILES;
    return (a.dim < 256 || a.bits == 8) &&
           ((long long)a.M * (a.heads / a.kv) <= (long long)FEW_PAIRS * a.B || (long long)a.M * a.heads <= (long long)tiles * Wide::TQ);
}

template <int DIM, int BITS, bool BLOCKS>
hipError_t start(const PromptArgs& a, hipStream_t stream)
{
    const bool few = takes_narrow(a);
    constexpr int sums = 128 * DIM * 4;        // (128 rows of O, or four times 32)
    constexpr int wide = 2 * Stage<DIM, Wide::KT>::BYTES + BLOCK_TOKENS * DIM * BITS / 8, narrow = RG * Stage<DIM, Narrow::KT>::BYTES;
    const int lds = few ? (narrow > sums ? narrow : sums) : (wide > sums ? wide : sums);
    auto kern = prompt_kernel<DIM, BITS, BLOCKS>;
    if constexpr (DIM < 256 || BITS == 8) kern = few ? few_kernel<DIM, BITS, BLOCKS> : kern;
    const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    if (a.B > 64) {
        if (few) plan_kernel<Narrow><<<1, PLAN_THREADS, 0, stream>>>(a);
        else plan_kernel<Wide><<<1, PLAN_THREADS, 0, stream>>>(a);
        const hipError_t p = hipGetLastError();
        if (p != hipSuccess) return p;
    }
    kern<<<(unsigned)units_of(a.M, a.B, a.heads, a.kv, few ? Narrow::TQ : Wide::TQ), THREADS, lds, stream>>>(a);
    return hipGetLastError();
}

template <int DIM>
hipError_t start(const PromptArgs& a, hipStream_t stream)
{
    if (a.bits == 16) return start<DIM, 16, false>(a, stream);
    return a.k_scales ? start<DIM, 8, true>(a, stream) : start<DIM, 8, false>(a, stream);
}

// What workgroup `id` of a launch does, found on the host as plan_kernel() and unit_planned() find it (their sum in floats may be rounded otherwise)
template <typename SHAPE>
PromptUnit unit_on_host(const PromptArgs& a, int id)
{
    float work = 0.f;
    for (int b = 0; b < a.B; ++b) {
        const Request r = request_of<SHAPE>(a, b);
        work += (float)r.tiles * (float)r.cost;
    }
    const float shares = shares_of(a, work);
    std::vector<Planned> plan(a.B);
    const int each = (a.B + PLAN_THREADS - 1) / PLAN_THREADS;
    int end = 0, before = 0;
    for (int b = 0; b < a.B; b += each) {
        const int stop = b + each < a.B ? b + each : a.B;
        int units, cut;
        count_units<SHAPE>(a, b, stop, shares, units, cut);
        write_plans<SHAPE>(a, b, stop, shares, end, before, plan.data());
        end = counted(end + units);
        before = counted(before + cut);
    }
    PromptUnit to{};
    to.narrow = SHAPE::TQ == Narrow::TQ;
    to.workgroups = units_of(a.M, a.B, a.heads, a.kv, SHAPE::TQ);
    to.request = to.place = -1;
    int b = 0;
    while (b < a.B && id >= plan[b].at.x) ++b;
    if (b == a.B) return to;
    const int4 at = plan[b].at, what = plan[b].what;
    Tile<SHAPE> t;
    t.u = unit_in(a, Request{at.z, at.w, what.x, what.y, what.w}, b, what.z, id - (at.x - what.y * what.z * a.kv), at.y);
    const bool some = t.set(a);
    to.head = t.u.h;
    to.tile = t.u.tile;
    to.tiles = what.y;
    to.part = t.u.part;
    to.parts = t.parts;
    if (!some) return to;
    to.request = b;
    to.steps = t.k1 - t.k0;
    if (t.parts > 1) to.place = t.u.place;
    return to;
}

}  // namespace

PromptUnit prompt_unit(const PromptArgs& a, int id) { return takes_narrow(a) ? unit_on_host<Narrow>(a, id) : unit_on_host<Wide>(a, id); }

long long prompt_units(int M, int B, int heads, int kv) { return units_of(M, B, heads, kv, Narrow::TQ); }

// bytes before the plan: counters, partial results (a workspace for wide heads also serves narrower ones, of which there are more at a time)
static size_t before_plan(int dim)
{
    size_t words = 0;
    for (int d = 64; d <= dim; d *= 2) {
        const size_t one = (size_t)most_of(d) * part_words<Wide>(d);
        words = one > words ? one : words;
    }
    return (COUNTERS + words) * sizeof(float);
}
size_t prompt_workspace_bytes(int B, int dim) { return before_plan(dim) + (size_t)B * PLAN_BYTES; }

hipError_t launch_prompt(PromptArgs a, hipStream_t stream)
{
    a.plan = (char*)a.parts + before_plan(a.dim);
    return a.dim == 64 ? start<64>(a, stream) : (a.dim == 128 ? start<128>(a, stream) : start<256>(a, stream));
}

}  // namespace eora
