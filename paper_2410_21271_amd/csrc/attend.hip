// Attention of one new token per request over a paged key-value cache.
//
//      s_t = scale q . k_t,   out = sum_t 2^(s_t log2 e - m) v_t / sum_t 2^(s_t log2 e - m)       lo <= t < length
//
// Bound by memory: every key and value is read once (the query heads of a kv head, up to 16, share one read as the columns of the
// matrix instructions), against 4 flops per query head and cached value.  32 / 8 heads of 128: 64 requests of 2048 tokens in 83.8 us, 6.4 TB/s, of 1 to 4096 (138 MB) in 38.3; 64 / 8 heads in
// 8 bits: one of 131072 (268 MB) in 56, 160 to 8192 (1089 MB) in 197.5.
//
// Tile: 32 keys a wavefront.  S^T = K Q^T: a lane (n = lane % 16, j = lane / 16) holds row n of K as the first operand, so an fp16 key row is read in
// pieces of 64 bytes, and ends with the scores of head n for keys 4j + i and 16 + 4j + i: exactly its eight k-slots of the second product
// O^T = V^T P^T, if that takes its keys in this order.  So P goes from one product to the next without leaving the lane.  For the first
// operand V^T a lane reads, of each of its eight keys, the dim / 16 columns from dim / 16 * n on (whole rows, contiguous over the lanes); block b of O^T
// has column dim / 16 * n + b as its row n, and a lane's operand is a transposition of 16-bit values in its own registers.  No LDS, no exchange between lanes in the loop.
//
// Softmax: m is a reference, common to the lanes of a head, not the exact maximum: LOWER below it when it is set, raised, and O and the sum rescaled, only when a score
// has risen by RAISE or more since.  So the largest weight is 2^11 to 2^15, and one of 2^-36 of it still 2^-25, the least that fp16 rounds to anything: tokens far
// below the largest, of which there may be many, keep their part (with a largest weight of 1, 4000 of them 16 and 17 nats below it were off by 0.3 and 1.9 %).
// Scores, sums and O are fp32.  A weight meets V as two fp16, the second what the first leaves of it: 20.7 bits together, beside which the rounding of the result is all
// that shows (one fp16 put out off by up to 2^-12 of sum p |v|).  The first is cut off from a little below the weight, so that the second is positive as well: an infinite
// value then gives an infinity, which halves of zero or of two signs would make a NaN (and does where a weight is below 2^-24 of the largest).
//
// Split: all units (a request's kv head, or block of 16 of its query heads) in one row are cut into equal runs, whatever the lengths are: a request of 100 000
// tokens is spread over the whole chip, and one of 10 costs a tile.  A workgroup whose run lies in one unit works on it together and adds up in
// LDS; otherwise each wavefront has its own part of the run.  Results of parts of a unit go to the workspace past the caches; the
// last one to arrive (one counter a unit) joins them, in the order of the tiles, whoever it is: the bits do not depend on the order of arrival.
#include "serving.hpp"
#include "tiles.hpp"

namespace eora {
namespace {

constexpr int NW = 4, THREADS = 64 * NW;
constexpr int TILE = 32;
constexpr int START = 1;                       // what beginning a unit costs, in tiles (see Runs; with 2, 64 requests of 1 to 4096 tokens 38.3 -> 38.8 us)
// Cost of a workgroup's run at least, where a join costs more than a longer run.  Requests of one length (1 of 8192 tokens, 4 of 4096 in 8 bits: 10: 16.8, 18.8 us; 20: 17.1, 15.8;
// 40: 20.5, 17.6), of several (37 of up to 1000 tokens, 13 heads of 64: 4: 18.6; 8: 17.9; 16: 22.7)
constexpr int MIN_RUN = 20, FEW = 8;
constexpr int MAX_WG = 1024;                   // workgroups that there are counters for
constexpr int SLOTS = 2 * NW * MAX_WG;
constexpr int COUNTERS = SLOTS + NW * MAX_WG;  // words before the partial results: a counter for each group of them, and for each unit
constexpr float RAISE = 4.f, LOWER = 11.f;     // (2^15 is below fp16's 65504; raised less often, by 8, 64 requests of 1 to 4096 tokens take the same)
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
static_assert(START < NW, "the run of a workgroup holds a tile of each unit that it touches alone");

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// what the first half of a weight is cut off from
constexpr float BELOW = 1.f - 0x1p-12f;
__device__ __forceinline__ h2 toward_zero(float x, float y) { return __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(x, y)); }

// tokens and tiles of a request of n tokens
struct Span {
    int lo, hi, first, tiles;
};
__device__ __forceinline__ Span span_of(const AttendArgs& a, int n)
{
    Span s;
    s.hi = n;
    s.lo = a.window > 0 && n > a.window ? n - a.window : 0;
    s.first = s.lo / TILE;
    s.tiles = (n + TILE - 1) / TILE - s.first;
    return s;
}

// Requests, in LDS: plan[b].y: tokens; plan[b + 1].x: cost of one kv head in requests 0 .. b; plan[0].x = 0.  All threads of the workgroup.
__device__ __forceinline__ void add_costs(const AttendArgs& a, int2* plan, int* scratch)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, most = a.width * a.page;
    int before = 0;
    if (threadIdx.x == 0) plan[0].x = 0;
    for (int b0 = 0; b0 < a.B; b0 += THREADS) {
        const int b = b0 + (int)threadIdx.x;
        int n = b < a.B ? a.lengths[b] : 0;
        n = n < 0 ? 0 : (n > most ? most : n);
        const int tiles = span_of(a, n).tiles;
        int v = tiles > 0 ? tiles + START : 0;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int w = __shfl_up(v, o, 64);
            v += lane >= o ? w : 0;
        }
        if (lane == 63) scratch[wave] = v;
        __syncthreads();
        int sum = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int x = scratch[w];
            v += w < wave ? x : 0;
            sum += x;
        }
        if (b < a.B) {
            plan[b + 1].x = before + v;
            plan[b].y = n;
        }
        before += sum;
        __syncthreads();
    }
}

// The units in one row, each START + tiles long (the first START places stand for what a unit costs beside its tiles), cut into runs that differ by one at
// most: wavefront w of n workgroups has [cut(w), cut(w + 1)).  With requests of one length, and workgroups for all of them, each unit is cut for itself, into `each` runs.
struct Runs {
    unsigned n, each, length, q, r;            // a stretch of `length` = q each + r places has `each` runs, at most 4 MAX_WG
    __device__ unsigned cut(unsigned w) const
    {
        const unsigned stretch = w / each, i = w - stretch * each;
        return stretch * length + i * q + i * r / each;       // floor(i length / each), without 64 bits
    }
    // the wavefront whose run holds a place
    __device__ unsigned owner(unsigned at) const
    {
        const unsigned stretch = at / length;
        unsigned w = stretch * each + (unsigned)((float)(at - stretch * length) * ((float)each / (float)length));     // one off at most
        w = w < n * NW ? w : n * NW - 1;
        while (cut(w) > at) --w;
        while (cut(w + 1) <= at) ++w;
        return w;
    }
};
__device__ __forceinline__ Runs runs_of(const AttendArgs& a, const int2* plan)
{
    const unsigned pairs = (unsigned)(a.kv * a.hblocks), units = (unsigned)a.B * pairs, total = (unsigned)plan[a.B].x * pairs, cost = (unsigned)plan[1].x;
    Runs r;
    r.n = (unsigned)a.nwg;
    r.each = 0;
    if (units <= r.n && cost * (unsigned)a.B == (unsigned)plan[a.B].x) {
        const unsigned k = (cost + MIN_RUN - 1) / MIN_RUN, most = r.n / units;
        r.each = NW * (k > most ? most : (k < 1 ? 1 : k));
        r.length = cost;
        r.n = units * r.each / NW;
    }
    if (r.each == 0 || r.each > r.length) {    // (runs are not empty: at least NW places a workgroup, unless there are fewer in all)
        if (r.n > total / FEW + 1) r.n = total / FEW + 1;
        if (r.n > total / NW) r.n = total / NW;
        if (r.n == 0 && total) r.n = 1;
        r.each = NW * r.n;
        r.length = total;
    }
    r.each = __builtin_amdgcn_readfirstlane(r.each);
    r.length = __builtin_amdgcn_readfirstlane(r.length);
    r.n = __builtin_amdgcn_readfirstlane(r.n);
    r.q = r.each ? r.length / r.each : 0;
    r.r = r.length - r.q * r.each;
    return r;
}

struct Unit {
    int b, pair;                               // pair = kv head * hblocks + block of query heads
    unsigned begin, end;                       // places
};
__device__ __forceinline__ Unit unit_at(const AttendArgs& a, const int2* plan, unsigned at)
{
    const unsigned pairs = (unsigned)(a.kv * a.hblocks);
    // the last request that begins at or before `at`: 64 places a look
    int lo = 0;
    for (int range = a.B; range > 1;) {
        const int stride = (range + 63) / 64, mine = lo + (int)(threadIdx.x & 63) * stride;
        const bool before = mine < lo + range && (unsigned)plan[mine < a.B ? mine : a.B].x * pairs <= at;
        const int past = lo + range;
        lo += (__popcll(__ballot(before)) - 1) * stride;
        range = past - lo < stride ? past - lo : stride;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    Unit u;
    u.b = lo;
    const unsigned begin = (unsigned)__builtin_amdgcn_readfirstlane(plan[lo].x) * pairs;
    const unsigned cost = (unsigned)__builtin_amdgcn_readfirstlane(plan[lo + 1].x - plan[lo].x);
    u.pair = (int)((at - begin) / cost);
    u.begin = begin + (unsigned)u.pair * cost;
    u.end = u.begin + cost;
    return u;
}
// the one behind it (there is one)
__device__ __forceinline__ Unit unit_after(const AttendArgs& a, const int2* plan, const Unit& u)
{
    Unit v;
    v.b = u.b;
    v.pair = u.pair + 1;
    v.begin = u.end;
    v.end = u.end + (u.end - u.begin);
    if (v.pair == a.kv * a.hblocks) {
        v.pair = 0;
        int cost;
        do {
            ++v.b;
            cost = __builtin_amdgcn_readfirstlane(plan[v.b + 1].x - plan[v.b].x);
        } while (cost == 0);
        v.end = v.begin + (unsigned)cost;
    }
    return v;
}

// Whether the wavefronts of a workgroup go through its run together, tile by tile in turn, with their results added up in LDS at each unit's end: in one unit,
// or where units are long.  Otherwise each has a quarter of the run for itself (short units would leave three of four idle).
// From so many tiles a unit on (64 requests of 1 to 4096 tokens, 37 of up to 1000: 4: 40.7, 22.9 us; 8: 38.3, 17.9; 16: 39.9, 17.9)
constexpr unsigned LONG = 8;
__device__ __forceinline__ bool together_at(const AttendArgs& a, const Runs& r, const int2* plan, unsigned g)
{
    const unsigned pairs = (unsigned)(a.kv * a.hblocks), at = r.cut(NW * g), to = r.cut(NW * g + NW);
    const Unit first = unit_at(a, plan, at);
    if (to <= first.end) return true;
    const Unit last = unit_at(a, plan, to - 1);
    return to - at >= LONG * ((unsigned)(last.b - first.b) * pairs + (unsigned)last.pair - (unsigned)first.pair + 1u);
}

// Who contributes to a unit that is cut: workgroups g0 .. g1, once where their wavefronts go together, else (g0, g1) their wavefronts
// w0 .. w1 that have tiles of it.  Contribution c, in the order of the tiles, has its result in slot(c).
struct Parts {
    unsigned w0, w1, g0, g1, first, count;     // first: contributions of workgroup g0
    bool whole0;
};
__device__ __forceinline__ Parts parts_of(const AttendArgs& a, const Runs& r, const int2* plan, const Unit& u)
{
    Parts p;
    p.w0 = r.owner(u.begin + START);
    p.w1 = r.owner(u.end - 1);
    p.g0 = p.w0 / NW;
    p.g1 = p.w1 / NW;
    p.whole0 = together_at(a, r, plan, p.g0);
    const bool whole1 = p.g1 > p.g0 && together_at(a, r, plan, p.g1);
    const unsigned last = p.g1 > p.g0 ? NW * p.g0 + NW - 1 : p.w1;
    p.first = p.whole0 ? 1 : last - p.w0 + 1;
    p.count = p.first + (p.g1 > p.g0 ? p.g1 - p.g0 - 1 + (whole1 ? 1 : p.w1 - NW * p.g1 + 1) : 0);
    return p;
}
// A wavefront may end one cut unit and begin another: two slots each, the second for the beginning of a unit.  A workgroup's common results have those of its
// first wavefront.
__device__ __forceinline__ unsigned slot_of(const Parts& p, unsigned c)
{
    if (c < p.first) return 2 * (p.whole0 ? NW * p.g0 : p.w0 + c) + (c == 0);
    const unsigned d = c - p.first;
    return d < p.g1 - p.g0 - 1 ? 2 * NW * (p.g0 + 1 + d) : 2 * (NW * p.g1 + (d - (p.g1 - p.g0 - 1)));
}

// A partial result: rows x (m, sum), then rows x dim of O.  Stores and loads go past the caches of an XCD, eight bytes each (relaxed, agent scope).
__device__ __forceinline__ float* part_at(const AttendArgs& a, unsigned slot) { return a.parts + COUNTERS + (size_t)slot * ((size_t)a.rows * (a.dim + 2)); }
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

// One lane, after its wavefront's (workgroup's) stores are through: whether this is the last of `count` to arrive.  The counter is left at zero.
__device__ __forceinline__ bool arrive(const AttendArgs& a, unsigned counter, unsigned count)
{
    unsigned* at = (unsigned*)a.parts + counter;
    const bool last = __hip_atomic_fetch_add(at, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == count;
    if (last) __hip_atomic_store(at, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return last;
}
__device__ __forceinline__ void stores_through() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// exp2(m - to), 0 for no tokens
__device__ __forceinline__ float factor(float m, float to) { return m == -INFINITY ? 0.f : exp2_(m - to); }

// where a query head's results go
__device__ __forceinline__ size_t head_at(const AttendArgs& a, const Unit& u, int row)
{
    const int h = u.pair / a.hblocks;
    return (size_t)u.b * a.heads + h * a.group + 16 * (u.pair - h * a.hblocks) + row;
}
__device__ __forceinline__ float lse_of(float m, float sum) { return LN2 * (m + __log2f(sum)); }

// Contributions c0, c0 + step, .. (`count` of them) of a unit, joined by one wavefront (wave 0 of 1) or by the workgroup (its wavefronts take
// 64 float2 of the rows x dim of O in turn): the unit's result, or, for a group of contributions, a contribution in the place of the first.
// Added up four at a time, in order, whatever CH and BATCH are, with nothing left to the compiler to fuse or not: a unit may have contributions from workgroups and from
// wavefronts, either may be the last to arrive, and the bits are the same.
template <int DIM, int CH, int BATCH>          // CH times 64 float2 and BATCH contributions are requested at a time
__device__ __forceinline__ void join(const AttendArgs& a, const Parts& p, const Unit& u, unsigned c0, unsigned step, unsigned count, int nrows, int wave, int waves, bool final, float vs)
{
    static_assert(BATCH % 4 == 0, "contributions are added up four at a time");
    const int lane = threadIdx.x & 63, words = nrows * (DIM / 2);
    float m0 = -INFINITY, l0 = 0.f;
    for (int e0 = 64 * wave; e0 < words; e0 += 64 * waves * CH) {
        int e[CH], row[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int at = e0 + 64 * waves * i + lane;
            e[i] = at < words ? at : words - 1;
            row[i] = e[i] / (DIM / 2);
        }
        float m = -INFINITY, l = 0.f;          // of row `lane`
        float2 acc[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) acc[i] = make_float2(0.f, 0.f);
#pragma clang loop unroll(disable)
        for (unsigned c = 0; c < count; c += BATCH) {
            float2 ml[BATCH], x[BATCH][CH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {  // (beyond the last: the last again, of no weight)
                const float* src = part_at(a, slot_of(p, c0 + step * (c + k < count ? c + k : count - 1)));
                ml[k] = get2(src + 2 * (lane < nrows ? lane : 0));
#pragma unroll
                for (int i = 0; i < CH; ++i) x[k][i] = get2(src + 2 * a.rows + 2 * e[i]);
            }
#pragma unroll
            for (int four = 0; four < BATCH; four += 4) {
                if (c + four >= count) break;
                float up = m;
#pragma unroll
                for (int k = four; k < four + 4; ++k) up = fmaxf(up, ml[k].x);
                const float f = factor(m, up);
                l = m == -INFINITY ? l : l * f;
                m = up;
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const float g = __shfl(f, row[i], 64);
                    acc[i].x *= g;
                    acc[i].y *= g;
                }
#pragma unroll
                for (int k = four; k < four + 4; ++k) {
                    if (c + k >= count) break;
                    const float fk = factor(ml[k].x, up);
                    l = ml[k].x == -INFINITY ? l + ml[k].y : __builtin_fmaf(ml[k].y, fk, l);
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        const float gk = __shfl(fk, row[i], 64);
                        acc[i].x = __builtin_fmaf(x[k][i].x, gk, acc[i].x);
                        acc[i].y = __builtin_fmaf(x[k][i].y, gk, acc[i].y);
                    }
                }
            }
        }
        if (e0 == 0 && final && lane < nrows && a.lse) a.lse[head_at(a, u, lane)] = lse_of(m, l);
        m0 = m;
        l0 = l;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const bool there = e0 + 64 * waves * i + lane < words;
            if (final) {
                const float sum = __shfl(l, row[i], 64), by = vs / sum;
                const h2 y = {(_Float16)(sum == 0.f ? 0.f : acc[i].x * by), (_Float16)(sum == 0.f ? 0.f : acc[i].y * by)};
                if (there) *(h2*)(a.out + head_at(a, u, 0) * DIM + 2 * e[i]) = y;
            } else if (there) {
                put2(part_at(a, slot_of(p, c0)) + 2 * a.rows + 2 * e[i], acc[i].x, acc[i].y);
            }
        }
    }
    if (!final) {
        if (waves > 1) __syncthreads();        // all have read the first contribution's (m, sum)
        if (wave == 0 && lane < nrows) put2(part_at(a, slot_of(p, c0)) + 2 * lane, m0, l0);
    }
}

// A wavefront (the workgroup) has stored contribution c: the last of a group of contributions to arrive joins the group, the last group's the unit.
// Groups of the square root of their number: one workgroup would take 25 us for the 128 contributions of one of eight heads of a long request.
template <int DIM, int CH, int BATCH>
__device__ __forceinline__ void finish(const AttendArgs& a, const Parts& p, const Unit& u, unsigned c, int nrows, int wave, int waves, int* scratch, float vs)
{
    const unsigned size = p.count <= 16 ? p.count : (unsigned)ceilf(sqrtf((float)p.count)), groups = (p.count + size - 1) / size;
    const unsigned k = c / size, here = (k + 1) * size <= p.count ? size : p.count - k * size;
    auto last_of = [&](unsigned counter, unsigned count) {
        stores_through();
        bool last = false;
        if (waves == 1) {
            if ((threadIdx.x & 63) == 0) last = arrive(a, counter, count);
            return (bool)__builtin_amdgcn_readfirstlane(last);
        }
        __syncthreads();
        if (threadIdx.x == 0) scratch[0] = arrive(a, counter, count);
        __syncthreads();
        return scratch[0] != 0;
    };
    if (!last_of(slot_of(p, k * size), here)) return;
    join<DIM, CH, BATCH>(a, p, u, k * size, 1, here, nrows, wave, waves, groups == 1, vs);
    if (groups == 1 || !last_of(SLOTS + p.w0, groups)) return;         // (a wavefront begins one cut unit at most)
    join<DIM, CH, BATCH>(a, p, u, 0, size, groups, nrows, wave, waves, true, vs);
}

// eight (keys) x two columns of 16-bit values, one word a key -> two operands of eight keys
__device__ __forceinline__ void transpose_keys(const uint32_t (&in)[8], Frag& a, Frag& b)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        a.u[k] = __builtin_amdgcn_perm(in[2 * k + 1], in[2 * k], 0x05040100u);
        b.u[k] = __builtin_amdgcn_perm(in[2 * k + 1], in[2 * k], 0x07060302u);
    }
}

// two e4m3 codes -> two fp16, exactly (scale 1)
template <bool HIGH>
__device__ __forceinline__ uint32_t two_codes(uint32_t w)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HIGH));
}

// Wavefronts a SIMD: what the registers leave room for, which hold one tile and, at D = 256, 64 words of O.  Eight wavefronts a compute unit have 64 to 128 KiB
// in flight; with a second tile in registers, for half the wavefronts, and loads through the caches, 64 requests of 1 to 4096 tokens went from 40.6 us to 44.5, 160 to 8192 in 8 bits from 215 to 229, one of 131072 from
// 59.6 to 58.8.
template <int DIM>
constexpr int residents() { return DIM == 64 ? 3 : (DIM == 128 ? 2 : 1); }
constexpr int CUS = 256;
static_assert(CUS * residents<64>() <= MAX_WG, "a launch of more workgroups than there are counters for");

// Keys and values past the caches (once read, of no more use), or through them
template <bool PAST, typename T>
__device__ __forceinline__ T fetch(const char* p)
{
    if constexpr (PAST) return __builtin_nontemporal_load((const T*)p);
    else return *(const T*)p;
}

// The reductions' room in LDS
struct Shared {
    int scratch[NW];
    float red_m[NW][16], red_l[NW][16];
};

// The run of workgroup g
template <int DIM, int BITS, bool PAST>
__device__ __forceinline__ void go(const AttendArgs& a, const Runs& runs, const int2* plan, unsigned g, float* red_o, Shared& shared)
{
    constexpr int NT = DIM / 32;               // k-steps of the first product
    constexpr int W = DIM / 16;                // columns of V a lane holds, blocks of O^T
    constexpr int BYTES = BITS / 8;
    constexpr int KL = BITS == 16 ? NT : DIM / 64;        // 16-byte loads of a key row a lane makes
    constexpr int VW = W * BYTES / 4;          // words of a value row a lane holds
    typedef uint32_t words __attribute__((ext_vector_type(VW < 4 ? VW : 4)));
    constexpr int VL = VW < 4 ? 1 : VW / 4;    // loads of a value row
    // (where three wavefronts share a SIMD's registers, more float2 at a time spill: 37 requests of up to 1000 tokens 20.2 us with 4 and 4, 17.6)
    constexpr int LONE_CH = DIM == 64 ? 2 : 4, LONE_BATCH = DIM == 64 ? 8 : 4;

    auto& red_m = shared.red_m;
    auto& red_l = shared.red_l;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, j = lane >> 4;
    const bool together = together_at(a, runs, plan, g);
    unsigned at = runs.cut(NW * g + (together ? 0 : wave));
    const unsigned stop_at = runs.cut(NW * g + (together ? NW : wave + 1));

    Unit u = unit_at(a, plan, at), then = u;
    for (; at < stop_at; u = then) {
        const unsigned stop = stop_at < u.end ? stop_at : u.end;
        // tiles of the unit
        const int r0 = at > u.begin + START ? (int)(at - u.begin) - START : 0, r1 = (int)(stop - u.begin) - START;
        at = stop;
        if (at < stop_at) then = unit_after(a, plan, u);
        if (r1 <= r0) continue;
        const bool full = r0 == 0 && stop == u.end;
        const Span span = span_of(a, __builtin_amdgcn_readfirstlane(plan[u.b].y));
        const int h = u.pair / a.hblocks, hb = u.pair - h * a.hblocks;
        const int nrows = a.group - 16 * hb < a.rows ? a.group - 16 * hb : a.rows;
        const int* table = a.table + (size_t)u.b * a.width;
        const int t0 = span.first + r0 + (together ? wave : 0), step = together ? NW : 1;
        const int mine = together ? (r1 - r0 > wave ? (r1 - r0 - wave + NW - 1) / NW : 0) : r1 - r0;

        // Pages of the next 32 tiles: lane i has the row of tile i's first half, lane 32 + i of its second (-1: no page)
        long long rows_of = -1;
        auto look = [&](int i0) {
            const int key = (t0 + step * (i0 + (lane & 31))) * TILE + 16 * (lane >> 5);
            rows_of = -1;
            if (i0 + (lane & 31) < mine && key < span.hi) {
                const int p = key / a.page, page = table[p];
                if ((unsigned)page < (unsigned)a.n_pages) rows_of = ((long long)page * a.kv + h) * a.page + (key - p * a.page);
            }
        };
        auto half_row = [&](int i, int half) {
            const int from = (i & 31) + 32 * half;
            const unsigned lo = __builtin_amdgcn_readlane((unsigned)rows_of, from), hi = __builtin_amdgcn_readlane((unsigned)(rows_of >> 32), from);
            return (long long)(((unsigned long long)hi << 32) | lo);
        };
        // One tile in registers.  Its keys' are requested anew, for the next tile, as soon as the scores are there, its values' behind the second product; behind the
        // last tile the requests go on, all lanes to one place: a request behind a branch would make every wait one for all requests.
        u4 tk[2][KL];
        words tv[8][VL];
        long long rows[2];
        auto find = [&](int i, long long (&row)[2]) {
            row[0] = half_row(i, 0);
            row[1] = half_row(i, 1);
        };
        const unsigned k_at = (unsigned)(n * DIM * BYTES + 16 * j), v_at = (unsigned)(4 * j * DIM * BYTES + n * W * BYTES);
        auto load_k = [&](const long long (&row)[2], unsigned all) {
            const unsigned off = k_at & all;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const char* base = (const char*)a.pages_k + (size_t)(row[s] < 0 ? 0 : row[s]) * (DIM * BYTES);
#pragma unroll
                for (int e = 0; e < KL; ++e) tk[s][e] = fetch<PAST, u4>(base + off + 64 * e);
            }
        };
        auto load_v = [&](const long long (&row)[2], unsigned all) {
            const unsigned off = v_at & all;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const char* base = (const char*)a.pages_v + (size_t)(row[s] < 0 ? 0 : row[s]) * (DIM * BYTES);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int v = 0; v < VL; ++v) tv[4 * s + i][v] = fetch<PAST, words>(base + off + i * DIM * BYTES + 16 * v);
            }
        };
        if (mine > 0) look(0);
        // q: k-slots of lane (n, j) as the key's loads have them; heads that are not there are zero columns
        Frag qf[NT];
        {
            const _Float16* q = a.q + (size_t)u.b * a.q_stride + (size_t)(h * a.group + 16 * hb + (n < nrows ? n : 0)) * DIM;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int col = BITS == 16 ? 32 * t + 8 * j : 64 * (t / 2) + 16 * j + 8 * (t % 2);
                const u4 w = *(const u4*)(q + col);
                qf[t].q = n < nrows ? w : u4{0, 0, 0, 0};
            }
        }
        const float by = a.scale * LOG2E * (BITS == 8 ? a.k_scale[h] : 1.f), vs = BITS == 8 ? a.v_scale[h] : 1.f;
        f4 O[W];
#pragma unroll
        for (int b = 0; b < W; ++b) O[b] = f4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        if (mine > 0) {
            find(0, rows);
            load_k(rows, ~0u);
            load_v(rows, ~0u);
        }
        for (int i = 0; i < mine; ++i) {
            // scores
            f4 S[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                S[s] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < NT; ++e) {
                    Frag k;
                    if constexpr (BITS == 16) {
                        k.q = tk[s][e];
                    } else {
                        const uint32_t w0 = tk[s][e / 2][2 * (e % 2)], w1 = tk[s][e / 2][2 * (e % 2) + 1];
                        k.u[0] = two_codes<false>(w0);
                        k.u[1] = two_codes<true>(w0);
                        k.u[2] = two_codes<false>(w1);
                        k.u[3] = two_codes<true>(w1);
                    }
                    S[s] = mfma16(k.v, qf[e].v, S[s]);
                }
            }
            if (((i + 1) & 31) == 0) look(i + 1);
            const unsigned all = i + 1 < mine ? ~0u : 0u;
            long long next[2];
            find(i + 1, next);
            load_k(next, all);
            const int key0 = (t0 + step * i) * TILE;
            const bool whole = key0 >= span.lo && key0 + TILE <= span.hi && rows[0] >= 0 && rows[1] >= 0;
            float p[8];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[4 * s + e] = S[s][e] * by;
            unsigned out = 0;                  // keys of this lane that do not count
            if (!whole) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + 16 * s + 4 * j + e;
                        if (key < span.lo || key >= span.hi || rows[s] < 0) {
                            out |= 1u << (4 * s + e);
                            p[4 * s + e] = -INFINITY;
                        }
                    }
            }
            float top = p[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, p[e]);
            if (__any(top > m + (RAISE + LOWER))) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float up = fmaxf(m, top - LOWER), f = m == up ? 1.f : exp2_(m - up);
                m = up;
                l *= f;
#pragma unroll
                for (int b = 0; b < W; ++b) O[b] *= f;
            }
            const float ref = m == -INFINITY ? 0.f : m;
            Frag high, low;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = exp2_(p[e] - ref);
                l += p[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) high.p[e] = toward_zero(p[2 * e] * BELOW, p[2 * e + 1] * BELOW);
#pragma unroll
            for (int e = 0; e < 8; ++e) low.v[e] = (_Float16)(p[e] - (float)high.v[e]);
            // values: two columns of eight keys at a time
#pragma unroll
            for (int c = 0; c < W / 2; ++c) {
                uint32_t raw[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at_word = BITS == 16 ? c : c / 2;
                    const uint32_t w = tv[e][at_word / 4][VW < 4 ? at_word : at_word % 4];
                    if constexpr (BITS == 16) raw[e] = w;
                    else raw[e] = c % 2 ? two_codes<true>(w) : two_codes<false>(w);
                    // what lies in places that do not count may be anything, NaN among it, and 0 NaN is NaN
                    if (!whole) raw[e] = out >> e & 1 ? 0u : raw[e];
                }
                Frag v0, v1;
                transpose_keys(raw, v0, v1);
                O[2 * c] = mfma16(v0.v, high.v, O[2 * c]);
                O[2 * c + 1] = mfma16(v1.v, high.v, O[2 * c + 1]);
                O[2 * c] = mfma16(v0.v, low.v, O[2 * c]);
                O[2 * c + 1] = mfma16(v1.v, low.v, O[2 * c + 1]);
            }
            load_v(next, all);
            rows[0] = next[0];
            rows[1] = next[1];
        }
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);

        if (!together) {
            // This wavefront's result: all of the unit, or a part
            const float f = l == 0.f ? 0.f : vs / l;
            if (full) {
                if (n < nrows) {
                    const size_t head = head_at(a, u, n);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        _Float16 y[W];
#pragma unroll
                        for (int b = 0; b < W; ++b) y[b] = (_Float16)(l == 0.f ? 0.f : O[b][i] * f);
                        __builtin_memcpy((_Float16*)__builtin_assume_aligned(a.out + head * DIM + W * (4 * j + i), 2 * W), y, 2 * W);
                    }
                    if (j == 0 && a.lse) a.lse[head] = lse_of(m, l);
                }
                continue;
            }
            const Parts parts = parts_of(a, runs, plan, u);
            float* part = part_at(a, 2 * (NW * g + wave) + (r0 == 0));
            if (n < nrows) {
                if (j == 0) put2(part + 2 * n, m, l);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int b = 0; b < W; b += 2) put2(part + 2 * a.rows + n * DIM + W * (4 * j + i) + b, O[b][i], O[b + 1][i]);
            }
            const unsigned w = NW * g + wave;
            finish<DIM, LONE_CH, LONE_BATCH>(a, parts, u, g == parts.g0 ? w - parts.w0 : parts.first + (parts.g1 - parts.g0 - 1) + (w - NW * parts.g1), nrows, 0, 1, shared.scratch, vs);
            continue;
        }

        // The workgroup's results, added up
        __syncthreads();                       // (the last unit's have been read)
        if (lane < 16) {
            red_m[wave][lane] = m;
            red_l[wave][lane] = l;
        }
        __syncthreads();
        {
            float M = red_m[0][n];
#pragma unroll
            for (int w = 1; w < NW; ++w) M = fmaxf(M, red_m[w][n]);
            const float f = factor(m, M);
            if (n < nrows) {
                float* o = red_o + ((size_t)wave * a.rows + n) * DIM;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int b = 0; b < W; b += 4)
                        *(f4*)(o + W * (4 * j + i) + b) = f4{O[b][i] * f, O[b + 1][i] * f, O[b + 2][i] * f, O[b + 3][i] * f};
            }
        }
        __syncthreads();
        float* part = part_at(a, 2 * NW * g + (r0 == 0));
        for (int e = threadIdx.x; e < nrows * (DIM / 4); e += THREADS) {
            const int r = e / (DIM / 4), c = 4 * (e % (DIM / 4));
            float M = red_m[0][r];
#pragma unroll
            for (int w = 1; w < NW; ++w) M = fmaxf(M, red_m[w][r]);
            float sum = 0.f;
            f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float mw = red_m[w][r];
                sum += mw == -INFINITY ? red_l[w][r] : red_l[w][r] * exp2_(mw - M);
                x += *(const f4*)(red_o + ((size_t)w * a.rows + r) * DIM + c);
            }
            if (full) {
                const size_t head = head_at(a, u, r);
                const float f = vs / sum;
                typedef _Float16 h4 __attribute__((ext_vector_type(4)));
                h4 v;
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = (_Float16)(sum == 0.f ? 0.f : x[q] * f);         // (every token masked: as without tokens)
                *(h4*)(a.out + head * DIM + c) = v;
                if (c == 0 && a.lse) a.lse[head] = lse_of(M, sum);
            } else {
                float* o = part + 2 * a.rows + (size_t)r * DIM + c;
                put2(o, x[0], x[1]);
                put2(o + 2, x[2], x[3]);
                if (c == 0) put2(part + 2 * r, M, sum);
            }
        }
        if (full) continue;
        const Parts parts = parts_of(a, runs, plan, u);
        finish<DIM, 2, 8>(a, parts, u, g == parts.g0 ? 0 : parts.first + (g - parts.g0 - 1), nrows, wave, NW, shared.scratch, vs);
    }
}

// Past the caches where the requests hold so much (in whole tiles, and one a request): of less the last-level cache has some from the call before.  One cache call after call, then three
// in turn, as a model's layers have them, through and past: 32 / 8 heads of 128, 104 MiB 25.5 and 28.3 us, 29.0 and 29.4; 120 MiB 27.9 and 29.0, 31.5 and 30.0; 512 MiB 93.1 and 81.4, 93.6
// and 82.5; 13 heads of 64, 95 MiB 20.9 and 22.8, 23.5 and 23.9; 117 MiB 23.0 and 24.1, 27.6 and 24.9.  What they hold, not what their table has room for: with one of 131072 tokens, 1 request of
// 8192 takes 19.7 past and 17.0 through, 8 of 500 12.2 and 11.0.
constexpr size_t PAST_BYTES = (size_t)112 << 20;

// WIDE: the table has room for so much, and the requests' lengths decide
template <int DIM, int BITS, bool WIDE>
__global__ __launch_bounds__(THREADS, residents<DIM>()) void attend_kernel(const AttendArgs a)
{
    __shared__ Shared shared;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    float* red_o = (float*)smem;               // NW x rows x DIM
    int2* plan = (int2*)(red_o + NW * a.rows * DIM);

    const unsigned g = blockIdx.x;
    add_costs(a, plan, shared.scratch);
    __syncthreads();
    // requests without a token have no unit
    for (int b = (int)g; b < a.B; b += (int)gridDim.x) {
        if (plan[b + 1].x != plan[b].x) continue;
        for (int e = threadIdx.x; e < a.heads * (DIM / 8); e += THREADS) *(u4*)(a.out + (size_t)b * a.heads * DIM + 8 * e) = u4{0, 0, 0, 0};
        if (a.lse)
            for (int e = threadIdx.x; e < a.heads; e += THREADS) a.lse[(size_t)b * a.heads + e] = -INFINITY;
    }
    const Runs runs = runs_of(a, plan);
    if (g >= runs.n) return;
    if constexpr (WIDE) {
        const size_t held = (size_t)(unsigned)__builtin_amdgcn_readfirstlane(plan[a.B].x) * (unsigned)a.kv * (TILE * DIM * (BITS / 8) * 2);
        if (held >= PAST_BYTES) {
            go<DIM, BITS, true>(a, runs, plan, g, red_o, shared);
            return;
        }
    }
    go<DIM, BITS, false>(a, runs, plan, g, red_o, shared);
}

// query heads of a kv head in blocks of up to 16
void set_blocks(AttendArgs& a)
{
    a.group = a.heads / a.kv;
    a.hblocks = (a.group + 15) / 16;
    a.rows = a.group < 16 ? a.group : 16;
}

template <int DIM, int BITS, bool WIDE>
hipError_t start(AttendArgs& a, hipStream_t stream)
{
    const size_t lds = NW * a.rows * DIM * sizeof(float) + ((size_t)a.B + 1) * sizeof(int2);
    const auto kern = attend_kernel<DIM, BITS, WIDE>;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    // as many workgroups as the chip holds at a time (registers, 160 KiB of LDS), and no more than the table's widest requests have work for
    int each = (int)(159 * 1024 / (lds + 1024));
    each = each < residents<DIM>() ? each : residents<DIM>();
    const size_t most = (size_t)a.B * a.kv * a.hblocks * (((size_t)a.width * a.page + TILE - 1) / TILE + START + 1) / NW + 1;
    a.nwg = most < (size_t)CUS * each ? (int)most : CUS * each;
    kern<<<a.nwg, THREADS, lds, stream>>>(a);
    return hipGetLastError();
}

template <int DIM, int BITS>
hipError_t start(AttendArgs& a, hipStream_t stream)
{
    // (tables with no such room: the loop past the caches left out, 0.2 us of 7.5 for one request of 100 tokens)
    const size_t tokens = (size_t)a.width * a.page, seen = a.window > 0 && (size_t)a.window < tokens ? (size_t)a.window : tokens;
    return a.B * (seen + 2 * TILE) * a.kv * DIM * (BITS / 8) * 2 >= PAST_BYTES ? start<DIM, BITS, true>(a, stream) : start<DIM, BITS, false>(a, stream);
}

template <int DIM>
hipError_t start(AttendArgs& a, hipStream_t stream)
{
    return a.bits == 8 ? start<DIM, 8>(a, stream) : start<DIM, 16>(a, stream);
}

}  // namespace

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

hipError_t launch_attend(AttendArgs a, hipStream_t stream)
{
    set_blocks(a);
    return a.dim == 64 ? start<64>(a, stream) : (a.dim == 128 ? start<128>(a, stream) : start<256>(a, stream));
}

}  // namespace eora
