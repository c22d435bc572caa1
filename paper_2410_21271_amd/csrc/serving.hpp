// Internal launch interface of the operators between a decoder layer's linears: many requests' adapters (adapters.hip),
// head norms and rotations into the cache (append.hip), attention over the cache (attend.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace eora {

struct AppendArgs {
    const _Float16* q;              // M rows of heads x dim
    const _Float16* k;              // M rows of kv x dim
    const _Float16* v;
    const _Float16* q_weight;       // dim, or null: no norm
    const _Float16* k_weight;
    const float* rotations;         // positions x rot/2 (cos, sin) pairs
    const int* positions;           // M
    const long long* slots;         // M
    _Float16* q_out;                // M x heads x dim
    void* pages_k;                  // pages x kv x page x dim
    void* pages_v;
    const float* k_scale;           // kv (8-bit cache)
    const float* v_scale;
    int M, heads, kv, dim;
    int q_stride, k_stride, v_stride;
    int rot, interleaved, n_positions;
    float eps;
    int page;
    unsigned n_slots;               // pages x page
    int bits;
    int slices;                     // workgroups per token (set by the launcher)
};
hipError_t launch_append(const AppendArgs& a, hipStream_t stream);

struct AttendArgs {
    const _Float16* q;              // B rows of heads x dim, q_stride apart
    const void* pages_k;            // pages x kv x page x dim
    const void* pages_v;
    const float* k_scale;           // kv (8-bit cache), else null
    const float* v_scale;
    const int* table;               // B x width
    const int* lengths;             // B
    _Float16* out;                  // B x heads x dim
    float* lse;                     // B x heads, or null
    float* parts;                   // arrival counters, partial results of units that several wavefronts share
    int B, heads, kv, dim, q_stride, n_pages, page, bits, width, window;
    float scale;
    int group, hblocks, rows;       // query heads per kv head; blocks of 16 of them; of them in a block (set by the launcher)
    int nwg;                        // workgroups (set by the launcher)
};
constexpr int ATTEND_MAX_B = 8192;          // requests per call: their tile counts sit in LDS
size_t attend_workspace_bytes(int heads, int kv, int dim);
hipError_t launch_attend(AttendArgs a, hipStream_t stream);

struct AdapterArgs {
    const _Float16* x;              // M x d_in
    const void* A;                  // n pairs' tiles, one after the other: r x d_in
    const void* B;                  // d_out x r
    const _Float16* A_scales;
    const _Float16* B_scales;
    const int* ranks;               // n, or null: all r
    const float* scalings;          // n, or null: all 1
    const int* ids;                 // M
    const _Float16* base;           // M x d_out, or null: zeros
    _Float16* y;                    // M x d_out
    uint32_t* header;               // counts of the one-launch form
    int spin_limit;
    int* order;                     // (behind the header; these set by the launcher) of the two-launch form: rows of each batch in the order of their pairs
    float* t;                       // (behind those) ranges x M x r partial sums of x A^T
    int M, d_in, d_out, r, n;
    int rgroups, down_wgs, up_wgs;          // groups of ranks; workgroups of either part (of a batch in either launch)
};
size_t adapters_workspace_bytes(int M, int d_in, int d_out, int r);
hipError_t launch_adapters(AdapterArgs a, int fa, int fe, hipStream_t stream);

}  // namespace eora
