// Internal launch interface of the operators between a decoder layer's linears: many requests' adapters (adapters.hip),
// head norms and rotations into the cache (append.hip, blocks.hip), attention over the cache (attend.hip, attend_far.hip, prompt.hip).
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

// A cache with a scale for each block: 16 tokens of a page and head share a power of two, a byte e + 127 (n_pages x kv x page / 16)
constexpr int BLOCK_TOKENS = 16;
constexpr int SCALE_LEAST = -15, SCALE_MOST = 8;

struct BlocksArgs {
    const _Float16* q;              // as AppendArgs
    const _Float16* k;
    const _Float16* v;
    const _Float16* q_weight;
    const _Float16* k_weight;
    const float* rotations;
    const int* positions;
    const long long* slots;
    _Float16* q_out;
    void* pages_k;                  // codes
    void* pages_v;
    uint8_t* k_scales;
    uint8_t* v_scales;
    int M, heads, kv, dim;
    int q_stride, k_stride, v_stride;
    int rot, interleaved, n_positions;
    float eps;
    int page;
    unsigned n_slots;
    int m0, tokens;                 // rows of this launch (these set by the launcher)
    int slices;                     // workgroups per token for its queries
    int look;                       // rows that a wavefront looks through for first rows of blocks
};
hipError_t launch_append_blocks(BlocksArgs a, hipStream_t stream);

struct ReadArgs {
    const void* pages_k;
    const void* pages_v;
    const void* k_scale;            // by head (float) or by block (bytes), or null
    const void* v_scale;
    const long long* slots;         // M
    _Float16* k;                    // M x kv x dim
    _Float16* v;
    int M, kv, dim, page, bits;
    bool blocks;
    unsigned n_slots;
};
hipError_t launch_read(const ReadArgs& a, hipStream_t stream);

// Words at the start of a workspace of attention that are zero between calls, of every kind; partial results lie behind them
constexpr int ATTEND_COUNTERS = 12288;

struct AttendArgs {
    const _Float16* q;              // B rows of heads x dim, q_stride apart
    const void* pages_k;            // pages x kv x page x dim
    const void* pages_v;
    const float* k_scale;           // kv (8-bit cache), else null
    const float* v_scale;
    const uint8_t* k_scales;        // by block, or null (launch_attend_far() only, as `sinks`)
    const uint8_t* v_scales;
    const int* table;               // B x width
    const int* lengths;             // B
    _Float16* out;                  // B x heads x dim
    float* lse;                     // B x heads, or null
    float* parts;                   // arrival counters, partial results of units that several wavefronts share
    int B, heads, kv, dim, q_stride, n_pages, page, bits, width, window, sinks;
    float scale;
    int group, hblocks, rows;       // query heads per kv head; blocks of 16 of them; of them in a block (set by the launcher)
    int nwg;                        // workgroups (set by the launcher)
};
constexpr int ATTEND_MAX_B = 8192;          // requests per call: their tile counts sit in LDS
size_t attend_workspace_bytes(int heads, int kv, int dim);
hipError_t launch_attend(AttendArgs a, hipStream_t stream);
hipError_t launch_attend_far(AttendArgs a, hipStream_t stream);        // first tokens that stay visible, scales by block

struct PromptArgs {
    const _Float16* q;              // M rows of heads x dim, q_stride apart
    const void* pages_k;            // pages x kv x page x dim
    const void* pages_v;
    const float* k_scale;           // kv (8-bit cache with a scale a head), else null
    const float* v_scale;
    const uint8_t* k_scales;        // by block, or null
    const uint8_t* v_scales;
    const int* table;               // B x width
    const int* lengths;             // B
    const int* starts;              // B + 1: rows of each request
    _Float16* out;                  // M x heads x dim
    float* lse;                     // M x heads, or null
    float* parts;                   // arrival counters, partial results of tiles that several workgroups share
    void* plan;                     // (set by the launcher) of many requests: their units
    int M, B, heads, kv, dim, q_stride, n_pages, page, bits, width, window, sinks;
    float scale;
};
size_t prompt_workspace_bytes(int B, int dim);
long long prompt_units(int M, int B, int heads, int kv);               // workgroups of a launch at most
hipError_t launch_prompt(PromptArgs a, hipStream_t stream);
// what workgroup `id` of that launch has (a.lengths and a.starts: host memory)
struct PromptUnit {
    int narrow;                     // tiles of few pairs
    long long workgroups;           // of the launch
    int request, head, tile, tiles, part, parts;               // request -1: nothing; tiles of the request
    int steps, place;               // tiles of keys; number of its partial results among all, -1: its tile is not cut
};
PromptUnit prompt_unit(const PromptArgs& a, int id);

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
