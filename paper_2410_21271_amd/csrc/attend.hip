// Attention of one new token per request over a paged key-value cache.
//
//      s_t = scale q . k_t,   out = sum_t 2^(s_t log2 e - m) v_t / sum_t 2^(s_t log2 e - m)       lo <= t < length
//
// Bound by memory: every key and value is read once (the query heads of a kv head, up to 16, share one read as the columns of the
// matrix instructions), against 4 flops per query head and cached value.
//
// Tile: 32 keys a wavefront.  S^T = K Q^T: a lane (n = lane % 16, j = lane / 16) holds row n of K as the first operand, so an fp16 key row is read in
// pieces of 64 bytes, and ends with the scores of head n for keys 4j + i and 16 + 4j + i: exactly its eight k-slots of the second product
// O^T = V^T P^T, if that takes its keys in this order.  So P goes from one product to the next without leaving the lane.  For the first
// operand V^T a lane reads, of each of its eight keys, the dim / 16 columns from dim / 16 * n on (whole rows, contiguous over the lanes); block b of O^T
// has column dim / 16 * n + b as its row n, and a lane's operand is a transposition of 16-bit values in its own registers.  No LDS, no exchange between lanes in the loop.
//
// Softmax: m is a reference, common to the lanes of a head, not the exact maximum: it is raised, and O and the sum rescaled, only when a score
// exceeds it by 2^8 or more (weights up to 256 are as exact in fp16 as weights up to 1).  Scores, sums and O are fp32; a weight is
// rounded to fp16 (nearest-even) for the product with V, the sum takes it unrounded.
//
// Split: the tiles of all (request, kv head) pairs in one row are cut into equal runs, one a workgroup, whatever the lengths are: a request of 100 000 tokens is spread
// over the whole chip, and one of 10 costs a tile.  A run that ends inside a pair leaves its (m, sum, O) in the workspace and a second
// kernel joins them, in the order of the tiles.
#include "serving.hpp"
#include "tiles.hpp"

namespace eora {
namespace {

constexpr int NW = 4, THREADS = 64 * NW;
constexpr int TILE = 32;
constexpr int MIN_RUN = 4;                     // tiles of a workgroup at least: one a wavefront
constexpr float RAISE = 8.f;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// tokens and tiles of a request
struct Span {
    int lo, hi, first, tiles;
};
__device__ __forceinline__ Span span_of(const AttendArgs& a, int b)
{
    const int most = a.width * a.page;
    int n = a.lengths[b];
    n = n < 0 ? 0 : (n > most ? most : n);
    Span s;
    s.hi = n;
    s.lo = a.window > 0 && n > a.window ? n - a.window : 0;
    s.first = s.lo / TILE;
    s.tiles = (n + TILE - 1) / TILE - s.first;
    return s;
}

// ends[b + 1] = tiles of one kv head in requests 0 .. b; ends[0] = 0.  All threads of the workgroup.
__device__ __forceinline__ void count_tiles(const AttendArgs& a, int* ends, int* scratch)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    if (threadIdx.x == 0) ends[0] = 0;
    for (int b0 = 0; b0 < a.B; b0 += THREADS) {
        const int b = b0 + (int)threadIdx.x;
        int v = b < a.B ? span_of(a, b).tiles : 0;
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
        if (b < a.B) ends[b + 1] = before + v;
        before += sum;
        __syncthreads();
    }
}

// The runs: workgroup g of `n` has tiles [cut(g), cut(g + 1)) of `total`
struct Runs {
    unsigned total, n;
    __device__ unsigned cut(unsigned g) const { return (unsigned)((unsigned long long)g * total / n); }
    // the workgroup whose run holds a tile
    __device__ unsigned owner(unsigned tile) const
    {
        unsigned g = (unsigned)((unsigned long long)tile * n / total);
        while (cut(g + 1) <= tile) ++g;
        while (cut(g) > tile) --g;
        return g;
    }
};
__device__ __forceinline__ Runs runs_of(const AttendArgs& a, int tiles)
{
    Runs r;
    r.total = (unsigned)tiles * (unsigned)(a.kv * a.hblocks);
    const unsigned most = (r.total + MIN_RUN - 1) / MIN_RUN;
    r.n = most < (unsigned)a.nwg ? most : (unsigned)a.nwg;
    return r;
}

// Where a unit (request b, kv head h, block hb of its query heads) begins: units of a request follow each other
struct Unit {
    int b, pair;                               // pair = h * hblocks + hb
    unsigned begin, end;                       // tiles
};
__device__ __forceinline__ Unit unit_at(const AttendArgs& a, const int* ends, unsigned tile)
{
    const unsigned pairs = (unsigned)(a.kv * a.hblocks);
    int lo = 0, hi = a.B;                      // ends[lo] * pairs <= tile < ends[hi] * pairs
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((unsigned)ends[mid] * pairs <= tile) lo = mid;
        else hi = mid;
    }
    Unit u;
    u.b = lo;
    const unsigned begin = (unsigned)ends[lo] * pairs, tiles = (unsigned)(ends[lo + 1] - ends[lo]);
    u.pair = (int)((tile - begin) / tiles);
    u.begin = begin + (unsigned)u.pair * tiles;
    u.end = u.begin + tiles;
    return u;
}

// A partial result: rows x (m, sum), then, from a 16-byte boundary, rows x dim of O
__host__ __device__ constexpr int part_head(int rows) { return (2 * rows + 3) & ~3; }
__device__ __forceinline__ float* part_at(const AttendArgs& a, unsigned g, int second)
{
    return a.parts + ((size_t)2 * g + second) * (size_t)(part_head(a.rows) + a.rows * a.dim);
}

// eight (keys) x W (columns) 16-bit values, one register row a key -> W registers rows of eight keys
template <int W>
__device__ __forceinline__ void transpose_keys(const uint32_t (&in)[8][W / 2], Frag (&out)[W])
{
#pragma unroll
    for (int c = 0; c < W / 2; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            out[2 * c].u[k] = __builtin_amdgcn_perm(in[2 * k + 1][c], in[2 * k][c], 0x05040100u);
            out[2 * c + 1].u[k] = __builtin_amdgcn_perm(in[2 * k + 1][c], in[2 * k][c], 0x07060302u);
        }
}

// two e4m3 codes -> two fp16, exactly (scale 1)
template <bool HIGH>
__device__ __forceinline__ uint32_t two_codes(uint32_t w)
{
    typedef _Float16 half2v __attribute__((ext_vector_type(2)));
    const half2v v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HIGH);
    return __builtin_bit_cast(uint32_t, v);
}

template <int DIM, int BITS>
__global__ __launch_bounds__(THREADS) void attend_kernel(const AttendArgs a)
{
    constexpr int NT = DIM / 32;               // k-steps of the first product
    constexpr int W = DIM / 16;                // columns of V a lane holds, blocks of O^T
    constexpr int BYTES = BITS / 8;
    constexpr int KL = BITS == 16 ? NT : DIM / 64;        // 16-byte loads of a key row a lane makes
    constexpr int VW = W * BYTES / 4;          // words of a value row a lane holds
    static_assert(DIM % 64 == 0, "");
    typedef uint32_t words __attribute__((ext_vector_type(VW < 4 ? VW : 4)));
    constexpr int VL = VW < 4 ? 1 : VW / 4;    // loads of a value row

    __shared__ int scratch[NW];
    __shared__ float red_m[NW][16], red_l[NW][16];
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    float* red_o = (float*)smem;               // NW x rows x DIM
    int* ends = (int*)(red_o + NW * a.rows * DIM);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, j = lane >> 4;
    count_tiles(a, ends, scratch);
    __syncthreads();
    const Runs runs = runs_of(a, ends[a.B]);
    const unsigned g = blockIdx.x;
    if (g >= runs.n) return;
    const unsigned run_end = runs.cut(g + 1);

    for (unsigned at = runs.cut(g); at < run_end;) {
        const Unit u = unit_at(a, ends, at);
        const unsigned stop = run_end < u.end ? run_end : u.end;
        const Span span = span_of(a, u.b);
        const int h = u.pair / a.hblocks, hb = u.pair - h * a.hblocks;
        const int nrows = a.group - 16 * hb < a.rows ? a.group - 16 * hb : a.rows;
        const int t0 = span.first + (int)(at - u.begin), t1 = span.first + (int)(stop - u.begin);
        const int* table = a.table + (size_t)u.b * a.width;

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
        const float by = a.scale * LOG2E * (BITS == 8 ? a.k_scale[h] : 1.f);

        f4 O[W];
#pragma unroll
        for (int b = 0; b < W; ++b) O[b] = f4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;

        // Pages of this wavefront's next 32 tiles: lane i has the row of tile i's first half, lane 32 + i of its second (-1: no page)
        const int mine = t1 - t0 > wave ? (t1 - t0 - wave + NW - 1) / NW : 0;
        long long rows_of = -1;
        auto look = [&](int i0) {
            const int key = (t0 + wave + NW * (i0 + (lane & 31))) * TILE + 16 * (lane >> 5);
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
        u4 kw[2][KL];
        words vw[8][VL];
        auto load_k = [&](const long long (&row)[2]) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const char* base = (const char*)a.pages_k + (size_t)(row[s] < 0 ? 0 : row[s]) * (DIM * BYTES);
#pragma unroll
                for (int t = 0; t < KL; ++t) kw[s][t] = *(const u4*)(base + (unsigned)(n * DIM * BYTES + 64 * t + 16 * j));
            }
        };
        auto load_v = [&](const long long (&row)[2]) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const char* base = (const char*)a.pages_v + (size_t)(row[s] < 0 ? 0 : row[s]) * (DIM * BYTES);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int v = 0; v < VL; ++v) vw[4 * s + i][v] = *(const words*)(base + (unsigned)((4 * j + i) * DIM * BYTES + n * W * BYTES + 16 * v));
            }
        };
        long long row[2], next[2];
        if (mine > 0) {
            look(0);
            row[0] = half_row(0, 0);
            row[1] = half_row(0, 1);
            load_k(row);
            load_v(row);
        }
        for (int i = 0; i < mine; ++i) {
            // scores
            f4 S[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                S[s] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    Frag k;
                    if constexpr (BITS == 16) {
                        k.q = kw[s][t];
                    } else {
                        const uint32_t w0 = kw[s][t / 2][2 * (t % 2)], w1 = kw[s][t / 2][2 * (t % 2) + 1];
                        k.u[0] = two_codes<false>(w0);
                        k.u[1] = two_codes<true>(w0);
                        k.u[2] = two_codes<false>(w1);
                        k.u[3] = two_codes<true>(w1);
                    }
                    S[s] = mfma16(k.v, qf[t].v, S[s]);
                }
            }
            const bool more = i + 1 < mine;
            if (more) {
                if (((i + 1) & 31) == 0) look(i + 1);
                next[0] = half_row(i + 1, 0);
                next[1] = half_row(i + 1, 1);
                load_k(next);
            }
            const int key0 = (t0 + wave + NW * i) * TILE;
            const bool whole = key0 >= span.lo && key0 + TILE <= span.hi && row[0] >= 0 && row[1] >= 0;
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
                        if (key < span.lo || key >= span.hi || row[s] < 0) {
                            out |= 1u << (4 * s + e);
                            p[4 * s + e] = -INFINITY;
                        }
                    }
            }
            float top = p[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, p[e]);
            if (__any(top > m + RAISE)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float up = fmaxf(m, top), f = m == up ? 1.f : exp2_(m - up);
                m = up;
                l *= f;
#pragma unroll
                for (int b = 0; b < W; ++b) O[b] *= f;
            }
            const float ref = m == -INFINITY ? 0.f : m;
            Frag pf;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = exp2_(p[e] - ref);
                l += p[e];
                pf.v[e] = (_Float16)p[e];
            }
            // values: rows of eight keys
            uint32_t raw[8][W / 2];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int c = 0; c < VW; ++c) {
                    const uint32_t w = vw[e][c / 4][VW < 4 ? c : c % 4];
                    if constexpr (BITS == 16) {
                        raw[e][c] = w;
                    } else {
                        raw[e][2 * c] = two_codes<false>(w);
                        raw[e][2 * c + 1] = two_codes<true>(w);
                    }
                }
                // what lies in places that do not count may be anything, NaN among it, and 0 NaN is NaN
                if (!whole) {
#pragma unroll
                    for (int c = 0; c < W / 2; ++c) raw[e][c] = out >> e & 1 ? 0u : raw[e][c];
                }
            }
            if (more) {
                load_v(next);
                row[0] = next[0];
                row[1] = next[1];
            }
            Frag vf[W];
            transpose_keys<W>(raw, vf);
#pragma unroll
            for (int b = 0; b < W; ++b) O[b] = mfma16(vf[b].v, pf.v, O[b]);
        }
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);

        // the four wavefronts' results
        if (lane < 16) {
            red_m[wave][lane] = m;
            red_l[wave][lane] = l;
        }
        __syncthreads();
        float M = red_m[0][n];
#pragma unroll
        for (int w = 1; w < NW; ++w) M = fmaxf(M, red_m[w][n]);
        const float mine_f = m == -INFINITY ? 0.f : exp2_(m - M);
        if (n < nrows) {
            float* o = red_o + ((size_t)wave * a.rows + n) * DIM;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int b = 0; b < W; b += 4)
                    *(f4*)(o + W * (4 * j + i) + b) = f4{O[b][i] * mine_f, O[b + 1][i] * mine_f, O[b + 2][i] * mine_f, O[b + 3][i] * mine_f};
        }
        __syncthreads();
        const bool full = at == u.begin && stop == u.end;
        const float vs = BITS == 8 ? a.v_scale[h] : 1.f;
        float* part = part_at(a, g, at == u.begin);
        for (int e = threadIdx.x; e < nrows * (DIM / 8); e += THREADS) {
            const int r = e / (DIM / 8), c = 8 * (e % (DIM / 8));
            float Mr = red_m[0][r];
#pragma unroll
            for (int w = 1; w < NW; ++w) Mr = fmaxf(Mr, red_m[w][r]);
            float sum = 0.f;
            f4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float mw = red_m[w][r];
                sum += mw == -INFINITY ? red_l[w][r] : red_l[w][r] * exp2_(mw - Mr);
                const float* o = red_o + ((size_t)w * a.rows + r) * DIM + c;
                x += *(const f4*)o;
                y += *(const f4*)(o + 4);
            }
            if (full) {
                const size_t head = (size_t)u.b * a.heads + h * a.group + 16 * hb + r;
                const float f = vs / sum;
                h8 v;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v[q] = (_Float16)(sum == 0.f ? 0.f : x[q] * f);         // (every token masked: as without tokens)
                    v[4 + q] = (_Float16)(sum == 0.f ? 0.f : y[q] * f);
                }
                *(h8*)(a.out + head * DIM + c) = v;
                if (c == 0 && a.lse) a.lse[head] = LN2 * (Mr + __log2f(sum));
            } else {
                float* o = part + part_head(a.rows) + (size_t)r * DIM + c;
                *(f4*)o = x;
                *(f4*)(o + 4) = y;
                if (c == 0) {
                    part[2 * r] = Mr;
                    part[2 * r + 1] = sum;
                }
            }
        }
        __syncthreads();
        at = stop;
    }
}

// Units that several workgroups share, and requests without tokens.  A workgroup takes `per` of a unit's query heads.
template <int DIM, int BITS>
__global__ __launch_bounds__(THREADS) void join_kernel(const AttendArgs a, int per)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ int scratch[NW];
    constexpr int LPR = DIM / 8, SPAN = THREADS / LPR;    // lanes of a row; partial results read side by side
    float* red = (float*)smem;                 // SPAN x (DIM + 2)
    int* ends = (int*)(red + SPAN * (DIM + 2));
    count_tiles(a, ends, scratch);
    __syncthreads();
    const int shares = (a.rows + per - 1) / per;
    const int share = blockIdx.x % shares, unit = blockIdx.x / shares, pairs = a.kv * a.hblocks, b = unit / pairs, pair = unit - b * pairs;
    const int h = pair / a.hblocks, hb = pair - h * a.hblocks;
    const int nrows = a.group - 16 * hb < a.rows ? a.group - 16 * hb : a.rows;
    const unsigned tiles = (unsigned)(ends[b + 1] - ends[b]), begin = (unsigned)ends[b] * pairs + (unsigned)pair * tiles;
    const int r0 = share * per, r1 = r0 + per < nrows ? r0 + per : nrows;
    const size_t head0 = (size_t)b * a.heads + h * a.group + 16 * hb;
    const int c = 8 * (threadIdx.x % LPR), k = threadIdx.x / LPR;
    if (tiles == 0) {
        for (int r = r0 + k; r < r1; r += SPAN) {
            *(u4*)(a.out + (head0 + r) * DIM + c) = u4{0, 0, 0, 0};
            if (c == 0 && a.lse) a.lse[head0 + r] = -INFINITY;
        }
        return;
    }
    const Runs runs = runs_of(a, ends[a.B]);
    const unsigned g0 = runs.owner(begin), g1 = runs.owner(begin + tiles - 1);
    if (g0 == g1) return;
    const float vs = BITS == 8 ? a.v_scale[h] : 1.f;
    for (int r = r0; r < r1; ++r) {
        float m = -INFINITY, l = 0.f;
        f4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
        for (unsigned g = g0 + k; g <= g1; g += SPAN) {
            const float* part = part_at(a, g, g == g0);
            const float pm = part[2 * r], pl = part[2 * r + 1];
            const float* o = part + part_head(a.rows) + (size_t)r * DIM + c;
            const f4 px = *(const f4*)o, py = *(const f4*)(o + 4);
            const float up = fmaxf(m, pm), f0 = m == -INFINITY ? 0.f : exp2_(m - up), f1 = pm == -INFINITY ? 0.f : exp2_(pm - up);
            l = l * f0 + pl * (pm == -INFINITY ? 1.f : f1);
            x = x * f0 + px * f1;
            y = y * f0 + py * f1;
            m = up;
        }
        float* mine = red + k * (DIM + 2);
        if (c == 0) {
            mine[0] = m;
            mine[1] = l;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            mine[2 + c + q] = x[q];
            mine[6 + c + q] = y[q];
        }
        __syncthreads();
        if (k == 0) {
            float M = red[0];
#pragma unroll
            for (int s = 1; s < SPAN; ++s) M = fmaxf(M, red[s * (DIM + 2)]);
            float sum = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < SPAN; ++s) {
                const float* p = red + s * (DIM + 2);
                const float f = p[0] == -INFINITY ? 0.f : exp2_(p[0] - M);
                sum += p[0] == -INFINITY ? p[1] : p[1] * f;
#pragma unroll
                for (int q = 0; q < 8; ++q) o[q] += p[2 + c + q] * f;
            }
            const float f = vs / sum;
            h8 v;
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = (_Float16)(sum == 0.f ? 0.f : o[q] * f);
            *(h8*)(a.out + (head0 + r) * DIM + c) = v;
            if (c == 0 && a.lse) a.lse[head0 + r] = LN2 * (M + __log2f(sum));
        }
        __syncthreads();
    }
}

// query heads of a kv head in blocks of up to 16
void set_blocks(AttendArgs& a)
{
    a.group = a.heads / a.kv;
    a.hblocks = (a.group + 15) / 16;
    a.rows = a.group < 16 ? a.group : 16;
}

constexpr int MAX_WG = 768;

template <int DIM, int BITS>
hipError_t start(const AttendArgs& a, hipStream_t stream)
{
    const size_t ends = ((size_t)a.B + 1) * sizeof(int), lds = NW * a.rows * DIM * sizeof(float) + ends;
    const auto kern = attend_kernel<DIM, BITS>;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    kern<<<a.nwg, THREADS, lds, stream>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int units = a.B * a.kv * a.hblocks, per = units >= 512 ? a.rows : 1;
    join_kernel<DIM, BITS><<<units * ((a.rows + per - 1) / per), THREADS, THREADS / (DIM / 8) * (DIM + 2) * sizeof(float) + ends, stream>>>(a, per);
    return hipGetLastError();
}

template <int DIM>
hipError_t start(const AttendArgs& a, hipStream_t stream)
{
    return a.bits == 8 ? start<DIM, 8>(a, stream) : start<DIM, 16>(a, stream);
}

}  // namespace

size_t attend_workspace_bytes(int B, int heads, int kv, int dim, int max_tokens)
{
    AttendArgs a{};
    a.heads = heads;
    a.kv = kv;
    set_blocks(a);
    return (size_t)2 * MAX_WG * (part_head(a.rows) + a.rows * dim) * sizeof(float);
}

hipError_t launch_attend(AttendArgs a, hipStream_t stream)
{
    set_blocks(a);
    // no more workgroups than the longest requests the table allows have runs
    const size_t most = (size_t)a.B * a.kv * a.hblocks * (((size_t)a.width * a.page + TILE - 1) / TILE + 1);
    a.nwg = most / MIN_RUN + 1 < MAX_WG ? (int)(most / MIN_RUN + 1) : MAX_WG;
    return a.dim == 64 ? start<64>(a, stream) : (a.dim == 128 ? start<128>(a, stream) : start<256>(a, stream));
}

}  // namespace eora
