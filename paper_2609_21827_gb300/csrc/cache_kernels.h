// cache_kernels.h -- launch arguments of the paged-cache and log-probability
// kernels, shared by their C-ABI layer (cache_api.cu) and the kernels.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "rheo.h"

namespace rheo {

constexpr int kMaxCacheBatch = 4096;
constexpr int kMaxCacheTokens = 4096;
constexpr int kMaxTop = 32;

struct ReserveArgs {
    int B, T, P, max_pages, pages;
    int in_place;
    const int32_t* ctx_len;
    const int32_t* new_len;   // or null: T
    const int32_t* depth;     // or null
    rheo_pages before, after;
    int64_t* slot;
    int32_t* position;
    unsigned* status;
    unsigned* ticket;
};

struct RopeArgs {
    int B, T, Hq, H, rot, max_position, page_shift;
    int64_t slots;            // pages * page_size
    rheo_qkv in;
    const void* q_weight;
    const void* k_weight;
    float eps;
    const float* cos_sin;
    const int64_t* slot;
    const int32_t* position;
    rheo_kv kv;
    void* q_out;
    int64_t o_batch, o_token, o_head;
    unsigned* status;
};

struct CommitArgs {
    int B, T, H, P, pages, max_pages, layers, depth, kv_elem_bytes;
    rheo_kv kv;
    int64_t key_layer, value_layer;
    const int32_t* block_table;
    const int32_t* ctx_len;
    const int32_t* accepted_len;
    const int32_t* accepted_nodes;
    int32_t* next_len;
    unsigned* status;
};

struct AttendArgs {
    int B, T, H, G, D, P, page_shift, pages, max_pages;
    int ctas;                 // CTAs that share the tiles
    int lead;                 // what an item's start and end cost, in tiles
    int least;                // tiles of a chunk at least, where few items are cut by themselves
    int item_rows;            // query rows of an item
    int part_rows;            // rows kept of an item's partial sums
    rheo_attend_io io;
    rheo_kv kv;
    const int32_t* block_table;
    const int32_t* ctx_len;
    const int32_t* new_len;   // or null: T
    const uint8_t* mask;      // or null: j <= t
    float scale_log2;         // scale * log2(e)
    float* part_o;            // [2 * ctas][part_rows][D] unnormalised sums
    float* part_ml;           // [2 * ctas][part_rows][2] running maximum (log2 units) and sum
    int4* join;               // [ctas] the item that a CTA begins and others go on with: request, item, segments
    unsigned* status;
};

struct LogprobArgs {
    int R, V, k, per_t, segments;
    const char* logits;
    int64_t row_stride_bytes, logit_rows;
    const int32_t* row_index;
    const int32_t* token;
    const float* temperature;
    rheo_logprobs out;
    unsigned* status;
    unsigned* ticket;              // [R], where segments > 1
    float* part;                   // [R * segments][4] reference, sum, weighted sum, count (bits); where segments > 1
    unsigned long long* part_key;  // [R * segments][kMaxTop]
};

cudaError_t launch_reserve(const ReserveArgs& a, int sms, cudaStream_t s);
cudaError_t launch_rope(const RopeArgs& a, int dtype, int D, bool interleaved, int sms, cudaStream_t s);
cudaError_t launch_commit(const CommitArgs& a, int line_bytes, cudaStream_t s);
cudaError_t launch_attend(const AttendArgs& a, int dtype, cudaStream_t s);
cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t s);
int attend_item_rows(int dtype, int T, int G);
int attend_part_rows(int dtype, int T, int G);
int attend_lead(int dtype);
int attend_least(int dtype);
constexpr int kAttendCtas = 152;  // one a multiprocessor
// Rows of logits are cut into segments where two CTAs a multiprocessor leave each of them at least two.
constexpr int kLogprobParts = 2 * 152;
constexpr int kLogprobCutRows = kLogprobParts / 2;
cudaError_t launch_logprobs(const LogprobArgs& a, int dtype, bool aligned, cudaStream_t s);
int logprob_segments(int rows, int vocab, int dtype);

}  // namespace rheo
