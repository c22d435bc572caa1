// C-ABI entry points of the operators between a decoder layer's linears: argument validation, nothing else.
#include "serving.hpp"
#include "checks.hpp"
#include "eora.h"
#include "kernels.hpp"

#include <cmath>

namespace {

using namespace eora;

bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// the cache's sizes, as eora_cache_append() and eora_cache_attention() take them; scale_block: tokens that share a scale, 0: all of a head
int check_cache(const void* pages_k, const void* pages_v, const void* k_scale, const void* v_scale, int n_kv_heads, int head_dim, int n_pages,
                int page_size, int cache_bits, int scale_block = 0)
{
    if (!pages_k || !pages_v) return EORA_ERR_NULL;
    if (cache_bits != 16 && cache_bits != 8) return EORA_ERR_UNSUPPORTED;
    if (scale_block != 0 && (scale_block != BLOCK_TOKENS || cache_bits != 8)) return EORA_ERR_UNSUPPORTED;
    if (cache_bits == 8 && (!k_scale || !v_scale)) return EORA_ERR_NULL;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return EORA_ERR_UNSUPPORTED;
    if (n_kv_heads <= 0 || n_pages <= 0 || page_size <= 0 || page_size % 16) return EORA_ERR_SHAPE;
    if ((long long)n_pages * page_size > 0x7fffffffll) return EORA_ERR_SHAPE;
    if (!aligned16(pages_k) || !aligned16(pages_v) || (!scale_block && (!aligned_to(k_scale, 4) || !aligned_to(v_scale, 4)))) return EORA_ERR_ALIGN;
    return EORA_OK;
}

// rows of `heads` heads, `stride` elements apart
int check_rows(int heads, int head_dim, int stride)
{
    if (heads <= 0 || heads > 0x7fffffff / head_dim || stride < heads * head_dim || stride % 8) return EORA_ERR_SHAPE;
    return EORA_OK;
}

// new tokens on their way to the cache, as eora_cache_append() takes them
int check_append(const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight, const void* rotations, const void* positions,
                 const void* slots, const void* q_out, int M, int n_heads, int n_kv_heads, int head_dim, int q_stride, int k_stride, int v_stride,
                 int rot_dim, int n_positions, float eps)
{
    int rc;
    if (M < 0) return EORA_ERR_SHAPE;
    if ((rc = check_rows(n_heads, head_dim, q_stride)) != EORA_OK || (rc = check_rows(n_kv_heads, head_dim, k_stride)) != EORA_OK ||
        (rc = check_rows(n_kv_heads, head_dim, v_stride)) != EORA_OK)
        return rc;
    if (n_heads > 0x3fffffff - 2 * (long long)n_kv_heads) return EORA_ERR_SHAPE;
    if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 16) return EORA_ERR_SHAPE;
    if (rot_dim > 0 && (!rotations || !positions)) return EORA_ERR_NULL;
    if (rot_dim > 0 && n_positions <= 0) return EORA_ERR_SHAPE;
    if ((q_weight || k_weight) && !(eps >= 0.f && std::isfinite(eps))) return EORA_ERR_VALUE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_weight) || !aligned16(k_weight) || !aligned16(q_out)) return EORA_ERR_ALIGN;
    if (!aligned16(rotations) || !aligned_to(positions, 4) || !aligned_to(slots, 8)) return EORA_ERR_ALIGN;
    return EORA_OK;
}

// attention over the cache: what its entry points have in common
int check_attention(const void* q, const void* page_table, const void* lengths, const void* out, const void* lse, int n_heads, int n_kv_heads, int head_dim,
                    int q_stride, int page_size, int max_pages, float scale)
{
    const int rc = check_rows(n_heads, head_dim, q_stride);
    if (rc != EORA_OK) return rc;
    // keys and tiles are counted in 32 bits
    if ((long long)max_pages * page_size > 1ll << 30) return EORA_ERR_SHAPE;
    if (!std::isfinite(scale)) return EORA_ERR_VALUE;
    if (!aligned16(q) || !aligned16(out) || !aligned_to(page_table, 4) || !aligned_to(lengths, 4) || !aligned_to(lse, 4)) return EORA_ERR_ALIGN;
    return EORA_OK;
}
bool too_many_tiles(int B, int n_heads, int n_kv_heads, int page_size, int max_pages)
{
    const int group = n_heads / n_kv_heads;
    return ((double)max_pages * page_size / 32 + 2) * B * n_kv_heads * ((group + 15) / 16) > 2e9;
}

}  // namespace

extern "C" {

size_t eora_adapters_workspace_bytes(int M, int d_in, int d_out, int r)
{
    if (M < 0 || d_in <= 0 || d_in % 128 || d_out <= 0 || d_out % 16 || r <= 0 || r % 32 || r > 512) return 0;
    return round256(adapters_workspace_bytes(M < 1 ? 1 : M, d_in, d_out, r));
}

int eora_linear_adapters(const void* x, const void* A_pool, const void* B_pool, const void* A_scales, const void* B_scales, const void* ranks,
                         const void* scalings, const void* adapter_of_row, const void* base, void* y, int M, int d_in, int d_out, int r,
                         int n_adapters, int ab_bits, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!x || !A_pool || !B_pool || !adapter_of_row || !y) return EORA_ERR_NULL;
    if (ab_bits != 16 && ab_bits != 4 && ab_bits != 3) return EORA_ERR_UNSUPPORTED;
    if (ab_bits != 16 && (!A_scales || !B_scales)) return EORA_ERR_NULL;
    if (M < 0 || d_in <= 0 || d_in % 128 || d_out <= 0 || d_out % 16 || r <= 0 || r > 512 || n_adapters <= 0) return EORA_ERR_SHAPE;
    if (ab_bits == 16 ? r % 32 : (ab_bits == 4 ? r != 64 && r % 128 : r % 128)) return EORA_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(A_pool) || !aligned16(B_pool) || !aligned16(A_scales) || !aligned16(B_scales) || !aligned16(base) || !aligned16(y))
        return EORA_ERR_ALIGN;
    if (!aligned_to(ranks, 4) || !aligned_to(scalings, 4) || !aligned_to(adapter_of_row, 4)) return EORA_ERR_ALIGN;
    if (!workspace) return EORA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return EORA_ERR_ALIGN;
    if (workspace_bytes < eora_adapters_workspace_bytes(M, d_in, d_out, r)) return EORA_ERR_WORKSPACE;
    if (M == 0) return EORA_OK;
    AdapterArgs a{};
    a.x = (const _Float16*)x;
    a.A = A_pool;
    a.B = B_pool;
    a.A_scales = (const _Float16*)A_scales;
    a.B_scales = (const _Float16*)B_scales;
    a.ranks = (const int*)ranks;
    a.scalings = (const float*)scalings;
    a.ids = (const int*)adapter_of_row;
    a.base = (const _Float16*)base;
    a.y = (_Float16*)y;
    a.header = (uint32_t*)workspace;
    a.spin_limit = spin_limit();
    a.M = M;
    a.d_in = d_in;
    a.d_out = d_out;
    a.r = r;
    a.n = n_adapters;
    const int fa = ab_bits == 16 ? S_F16 : (ab_bits == 4 ? S_Q4S128 : S_Q3S128), fe = ab_bits == 4 && r == 64 ? S_Q4S64 : fa;
    if (failed(launch_adapters(a, fa, fe, (hipStream_t)stream), "linear_adapters")) return EORA_ERR_LAUNCH;
    return EORA_OK;
}

int eora_cache_append(const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight, const void* rotations,
                      const void* positions, const void* slots, void* q_out, void* pages_k, void* pages_v, const void* k_scale,
                      const void* v_scale, int M, int n_heads, int n_kv_heads, int head_dim, int q_stride, int k_stride, int v_stride, int rot_dim,
                      int interleaved, int n_positions, float eps, int n_pages, int page_size, int cache_bits, void* stream)
{
    if (!q || !k || !v || !slots || !q_out) return EORA_ERR_NULL;
    int rc = check_cache(pages_k, pages_v, k_scale, v_scale, n_kv_heads, head_dim, n_pages, page_size, cache_bits);
    if (rc != EORA_OK) return rc;
    rc = check_append(q, k, v, q_weight, k_weight, rotations, positions, slots, q_out, M, n_heads, n_kv_heads, head_dim, q_stride, k_stride, v_stride,
                      rot_dim, n_positions, eps);
    if (rc != EORA_OK) return rc;
    if (M == 0) return EORA_OK;
    AppendArgs a{};
    a.q = (const _Float16*)q;
    a.k = (const _Float16*)k;
    a.v = (const _Float16*)v;
    a.q_weight = (const _Float16*)q_weight;
    a.k_weight = (const _Float16*)k_weight;
    a.rotations = (const float*)rotations;
    a.positions = (const int*)positions;
    a.slots = (const long long*)slots;
    a.q_out = (_Float16*)q_out;
    a.pages_k = pages_k;
    a.pages_v = pages_v;
    a.k_scale = (const float*)k_scale;
    a.v_scale = (const float*)v_scale;
    a.M = M;
    a.heads = n_heads;
    a.kv = n_kv_heads;
    a.dim = head_dim;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.rot = rot_dim;
    a.interleaved = interleaved != 0;
    a.n_positions = n_positions;
    a.eps = eps;
    a.page = page_size;
    a.n_slots = (unsigned)n_pages * (unsigned)page_size;
    a.bits = cache_bits;
    if (failed(launch_append(a, (hipStream_t)stream), "cache_append")) return EORA_ERR_LAUNCH;
    return EORA_OK;
}

size_t eora_cache_attention_workspace_bytes(int B, int n_heads, int n_kv_heads, int head_dim, int max_tokens)
{
    if (B < 0 || B > ATTEND_MAX_B || n_kv_heads <= 0 || n_heads <= 0 || n_heads % n_kv_heads || max_tokens < 0) return 0;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return 0;
    return round256(attend_workspace_bytes(n_heads, n_kv_heads, head_dim));
}

int eora_cache_attention(const void* q, const void* pages_k, const void* pages_v, const void* k_scale, const void* v_scale, const void* page_table,
                         const void* lengths, void* out, void* lse, int B, int n_heads, int n_kv_heads, int head_dim, int q_stride, int n_pages,
                         int page_size, int cache_bits, int max_pages, int window, float scale, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!q || !page_table || !lengths || !out) return EORA_ERR_NULL;
    int rc = check_cache(pages_k, pages_v, k_scale, v_scale, n_kv_heads, head_dim, n_pages, page_size, cache_bits);
    if (rc != EORA_OK) return rc;
    if (B < 0 || B > ATTEND_MAX_B || n_heads % n_kv_heads || max_pages <= 0 || window < 0) return EORA_ERR_SHAPE;
    rc = check_attention(q, page_table, lengths, out, lse, n_heads, n_kv_heads, head_dim, q_stride, page_size, max_pages, scale);
    if (rc != EORA_OK) return rc;
    if (too_many_tiles(B, n_heads, n_kv_heads, page_size, max_pages)) return EORA_ERR_SHAPE;
    if (!workspace) return EORA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return EORA_ERR_ALIGN;
    if (workspace_bytes < eora_cache_attention_workspace_bytes(B, n_heads, n_kv_heads, head_dim, max_pages * page_size)) return EORA_ERR_WORKSPACE;
    if (B == 0) return EORA_OK;
    AttendArgs a{};
    a.q = (const _Float16*)q;
    a.pages_k = pages_k;
    a.pages_v = pages_v;
    a.k_scale = (const float*)k_scale;
    a.v_scale = (const float*)v_scale;
    a.table = (const int*)page_table;
    a.lengths = (const int*)lengths;
    a.out = (_Float16*)out;
    a.lse = (float*)lse;
    a.parts = (float*)workspace;
    a.B = B;
    a.heads = n_heads;
    a.kv = n_kv_heads;
    a.dim = head_dim;
    a.q_stride = q_stride;
    a.n_pages = n_pages;
    a.page = page_size;
    a.bits = cache_bits;
    a.width = max_pages;
    a.window = window;
    a.scale = scale;
    if (failed(launch_attend(a, (hipStream_t)stream), "cache_attention")) return EORA_ERR_LAUNCH;
    return EORA_OK;
}

int eora_cache_append_blocks(const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight, const void* rotations,
                             const void* positions, const void* slots, void* q_out, void* pages_k, void* pages_v, void* k_scales, void* v_scales, int M,
                             int n_heads, int n_kv_heads, int head_dim, int q_stride, int k_stride, int v_stride, int rot_dim, int interleaved,
                             int n_positions, float eps, int n_pages, int page_size, void* stream)
{
    if (!q || !k || !v || !slots || !q_out) return EORA_ERR_NULL;
    int rc = check_cache(pages_k, pages_v, k_scales, v_scales, n_kv_heads, head_dim, n_pages, page_size, 8, BLOCK_TOKENS);
    if (rc != EORA_OK) return rc;
    rc = check_append(q, k, v, q_weight, k_weight, rotations, positions, slots, q_out, M, n_heads, n_kv_heads, head_dim, q_stride, k_stride, v_stride,
                      rot_dim, n_positions, eps);
    if (rc != EORA_OK) return rc;
    if (M == 0) return EORA_OK;
    BlocksArgs a{};
    a.q = (const _Float16*)q;
    a.k = (const _Float16*)k;
    a.v = (const _Float16*)v;
    a.q_weight = (const _Float16*)q_weight;
    a.k_weight = (const _Float16*)k_weight;
    a.rotations = (const float*)rotations;
    a.positions = (const int*)positions;
    a.slots = (const long long*)slots;
    a.q_out = (_Float16*)q_out;
    a.pages_k = pages_k;
    a.pages_v = pages_v;
    a.k_scales = (uint8_t*)k_scales;
    a.v_scales = (uint8_t*)v_scales;
    a.M = M;
    a.heads = n_heads;
    a.kv = n_kv_heads;
    a.dim = head_dim;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.rot = rot_dim;
    a.interleaved = interleaved != 0;
    a.n_positions = n_positions;
    a.eps = eps;
    a.page = page_size;
    a.n_slots = (unsigned)n_pages * (unsigned)page_size;
    if (failed(launch_append_blocks(a, (hipStream_t)stream), "cache_append_blocks")) return EORA_ERR_LAUNCH;
    return EORA_OK;
}

int eora_cache_read(const void* pages_k, const void* pages_v, const void* k_scale, const void* v_scale, const void* slots, void* k, void* v, int M,
                    int n_kv_heads, int head_dim, int n_pages, int page_size, int cache_bits, int scale_block, void* stream)
{
    if (!slots || !k || !v) return EORA_ERR_NULL;
    const int rc = check_cache(pages_k, pages_v, k_scale, v_scale, n_kv_heads, head_dim, n_pages, page_size, cache_bits, scale_block);
    if (rc != EORA_OK) return rc;
    if (M < 0 || n_kv_heads > 0x7fffffff / head_dim) return EORA_ERR_SHAPE;
    if (!aligned16(k) || !aligned16(v) || !aligned_to(slots, 8)) return EORA_ERR_ALIGN;
    if (M == 0) return EORA_OK;
    ReadArgs a{};
    a.pages_k = pages_k;
    a.pages_v = pages_v;
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.slots = (const long long*)slots;
    a.k = (_Float16*)k;
    a.v = (_Float16*)v;
    a.M = M;
    a.kv = n_kv_heads;
    a.dim = head_dim;
    a.page = page_size;
    a.bits = cache_bits;
    a.blocks = scale_block != 0;
    a.n_slots = (unsigned)n_pages * (unsigned)page_size;
    if (failed(launch_read(a, (hipStream_t)stream), "cache_read")) return EORA_ERR_LAUNCH;
    return EORA_OK;
}

size_t eora_cache_attention_rows_workspace_bytes(int M, int B, int n_heads, int n_kv_heads, int head_dim, int max_tokens)
{
    const size_t tokens = eora_cache_attention_workspace_bytes(B, n_heads, n_kv_heads, head_dim, max_tokens);       // (single tokens: checks of all but M)
    if (tokens == 0 || M < 0) return 0;
    const size_t rows = round256(prompt_workspace_bytes(B, head_dim));
    return rows > tokens ? rows : tokens;
}

int eora_cache_attention_rows(const void* q, const void* pages_k, const void* pages_v, const void* k_scale, const void* v_scale, const void* page_table,
                              const void* lengths, const void* row_starts, void* out, void* lse, int M, int B, int n_heads, int n_kv_heads, int head_dim,
                              int q_stride, int n_pages, int page_size, int cache_bits, int scale_block, int max_pages, int window, int sinks, float scale,
                              void* workspace, size_t workspace_bytes, void* stream)
{
    if (!q || !page_table || !lengths || !out) return EORA_ERR_NULL;
    int rc = check_cache(pages_k, pages_v, k_scale, v_scale, n_kv_heads, head_dim, n_pages, page_size, cache_bits, scale_block);
    if (rc != EORA_OK) return rc;
    if (M < 0 || B < 0 || B > ATTEND_MAX_B || n_heads % n_kv_heads || max_pages <= 0 || window < 0 || sinks < 0) return EORA_ERR_SHAPE;
    if (!row_starts && M != B) return EORA_ERR_SHAPE;
    rc = check_attention(q, page_table, lengths, out, lse, n_heads, n_kv_heads, head_dim, q_stride, page_size, max_pages, scale);
    if (rc != EORA_OK) return rc;
    if (!row_starts && too_many_tiles(B, n_heads, n_kv_heads, page_size, max_pages)) return EORA_ERR_SHAPE;
    // (blocks of 16 tokens are counted in 32 bits)
    if (row_starts && (double)n_pages * page_size * n_kv_heads >= 16.0 * 0x7fffffff) return EORA_ERR_SHAPE;
    if (row_starts && ((long long)M * (n_heads / n_kv_heads) > 0x7fffffff || prompt_units(M, B, n_heads, n_kv_heads) > 0x7fffff)) return EORA_ERR_SHAPE;
    if (!aligned_to(row_starts, 4)) return EORA_ERR_ALIGN;
    if (!workspace) return EORA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return EORA_ERR_ALIGN;
    if (workspace_bytes < eora_cache_attention_rows_workspace_bytes(M, B, n_heads, n_kv_heads, head_dim, max_pages * page_size)) return EORA_ERR_WORKSPACE;
    if (M == 0 || B == 0) return EORA_OK;
    if (window >= max_pages * page_size) window = 0;
    if (window == 0) sinks = 0;                // (all tokens are visible)
    if (sinks > max_pages * page_size) sinks = max_pages * page_size;
    if (row_starts) {
        PromptArgs a{};
        a.q = (const _Float16*)q;
        a.pages_k = pages_k;
        a.pages_v = pages_v;
        (scale_block ? (const void*&)a.k_scales : (const void*&)a.k_scale) = k_scale;
        (scale_block ? (const void*&)a.v_scales : (const void*&)a.v_scale) = v_scale;
        a.table = (const int*)page_table;
        a.lengths = (const int*)lengths;
        a.starts = (const int*)row_starts;
        a.out = (_Float16*)out;
        a.lse = (float*)lse;
        a.parts = (float*)workspace;
        a.M = M;
        a.B = B;
        a.heads = n_heads;
        a.kv = n_kv_heads;
        a.dim = head_dim;
        a.q_stride = q_stride;
        a.n_pages = n_pages;
        a.page = page_size;
        a.bits = cache_bits;
        a.width = max_pages;
        a.window = window;
        a.sinks = sinks;
        a.scale = scale;
        if (failed(launch_prompt(a, (hipStream_t)stream), "cache_attention_rows")) return EORA_ERR_LAUNCH;
        return EORA_OK;
    }
    AttendArgs a{};
    a.q = (const _Float16*)q;
    a.pages_k = pages_k;
    a.pages_v = pages_v;
    (scale_block ? (const void*&)a.k_scales : (const void*&)a.k_scale) = k_scale;
    (scale_block ? (const void*&)a.v_scales : (const void*&)a.v_scale) = v_scale;
    a.table = (const int*)page_table;
    a.lengths = (const int*)lengths;
    a.out = (_Float16*)out;
    a.lse = (float*)lse;
    a.parts = (float*)workspace;
    a.B = B;
    a.heads = n_heads;
    a.kv = n_kv_heads;
    a.dim = head_dim;
    a.q_stride = q_stride;
    a.n_pages = n_pages;
    a.page = page_size;
    a.bits = cache_bits;
    a.width = max_pages;
    a.window = window;
    a.sinks = sinks;
    a.scale = scale;
    const bool far = sinks > 0 || scale_block;
    if (failed(far ? launch_attend_far(a, (hipStream_t)stream) : launch_attend(a, (hipStream_t)stream), "cache_attention_rows")) return EORA_ERR_LAUNCH;
    return EORA_OK;
}

int eora_debug_attention_rows_unit(const int* lengths, const int* row_starts, int M, int B, int n_heads, int n_kv_heads, int head_dim, int page_size, int cache_bits,
                                   int max_pages, int window, int sinks, int unit, int* plan)
{
    if (!lengths || !row_starts || !plan) return EORA_ERR_NULL;
    if ((cache_bits != 16 && cache_bits != 8) || (head_dim != 64 && head_dim != 128 && head_dim != 256)) return EORA_ERR_UNSUPPORTED;
    if (M <= 0 || B <= 0 || B > ATTEND_MAX_B || n_kv_heads <= 0 || n_heads <= 0 || n_heads % n_kv_heads || page_size <= 0 || page_size % 16 || max_pages <= 0 || window < 0 ||
        sinks < 0 || unit < 0 || (long long)max_pages * page_size > 1ll << 30)
        return EORA_ERR_SHAPE;
    if ((long long)M * (n_heads / n_kv_heads) > 0x7fffffff || prompt_units(M, B, n_heads, n_kv_heads) > 0x7fffff) return EORA_ERR_SHAPE;
    PromptArgs a{};
    a.lengths = lengths;
    a.starts = row_starts;
    a.M = M;
    a.B = B;
    a.heads = n_heads;
    a.kv = n_kv_heads;
    a.dim = head_dim;
    a.page = page_size;
    a.bits = cache_bits;
    a.width = max_pages;
    a.window = window >= max_pages * page_size ? 0 : window;
    a.sinks = a.window == 0 ? 0 : (sinks < max_pages * page_size ? sinks : max_pages * page_size);
    const PromptUnit u = prompt_unit(a, unit);
    const int found[10] = {u.narrow, (int)u.workgroups, u.request, u.head, u.tile, u.tiles, u.part, u.parts, u.steps, u.place};
    for (int i = 0; i < 10; ++i) plan[i] = found[i];
    return EORA_OK;
}

}  // extern "C"
