// Shared declarations of the serving operators: the paged key/value cache, the plan of a step, attention of drafted tokens
// over the pages and the rules on the logits.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace zq {

constexpr int kTypeF32 = 0, kTypeBf16 = 1, kTypeF16 = 2;     // ZOQAT_TYPE_*
inline int type_bytes(int type) { return type == kTypeF32 ? 4 : 2; }

// device status words (see include/zoqat.h)
constexpr int kPlanBadLength = 1, kPlanNoPages = 2, kPlanBadPage = 4, kPlanBadParent = 8;
constexpr int kErrBadSlot = 40;          // append: a slot or a position outside the cache / the rotary tables
constexpr int kErrBadRequest = 41;       // attention: lengths or row ranges that contradict each other
constexpr int kErrBadPage = 42;          // attention: a block table names a page outside the cache
constexpr int kErrTreeWait = 43;         // attention: a bounded wait ran out

constexpr int kMaxPlanBatch = 16384;

// One layer's pages (zoqat_paged_cache_t): element (page, slot, head, i) of K or V at
// page * page_stride + slot * slot_stride + head * head_stride + i, in elements.
struct PagedCache {
    void *k, *v;
    int type, n_pages, page_size, n_kv_heads, d_head;
    int64_t page_stride, slot_stride, head_stride;
};

struct CachePlanArgs {
    const int32_t *cached_len, *new_len;
    int batch, page_size, n_pages, max_pages;
    const int32_t* free_pages;
    int free_capacity;
    const int32_t* n_free;
    int32_t* block_table;
    const int32_t* parents;
    int max_rows, mask_words;
    int32_t *kv_len, *row_start, *row_request, *row_pos, *slot;
    uint32_t* tree_mask;
    int32_t *n_free_out, *status;
};
int launch_cache_plan(const CachePlanArgs& a, cudaStream_t s);       // 0, or -1: set-up failed

void launch_cache_append(const float* qkv, int64_t ld, const int32_t* row_pos, const int32_t* slot, int rows, int n_heads,
                         const float* cos_t, const float* sin_t, int max_pos, const PagedCache& cache, void* q_out, int64_t q_stride,
                         int32_t* err_flag, cudaStream_t s, bool dependent = false);
void launch_embed_rows(const int32_t* tokens, const int32_t* row_pos, const float* embed, const float* pos_embed, int rows, int d, int vocab,
                       int max_pos, float* h, int32_t* err_flag, cudaStream_t s);
void launch_widen(const void* src, int type, int64_t n, float* dst, cudaStream_t s);      // n % 8 == 0, 16-byte aligned

// Rotary append: norms and rotation of query and key heads on their way into the cache.
struct RotaryAppendArgs {
    const void* qkv;                     // [rows, (n_heads + 2 n_kv_heads) * d_head] of src_type, rows ld elements apart
    int src_type;
    int64_t ld;
    const int32_t *row_pos, *slot;
    int rows, n_heads;
    const double* freq;                  // [rot / 2] radians a position
    int rot;                             // elements of a head that are turned (a multiple of 16; 0: none)
    bool interleaved;
    float magnitude;
    const float *q_gain, *k_gain;        // [d_head] or NULL: no norm
    float eps;
    PagedCache cache;
    void* q_out;
    int64_t q_stride;
    int32_t* err_flag;
};
int launch_rotary_append(const RotaryAppendArgs& a, cudaStream_t s);         // 0, or -1: launch failed

// Beams.
constexpr int kMaxBeams = 32, kMaxBeamEos = 7;
struct BeamSelectArgs {
    const void* logits;                  // [batch * beams, vocab] of `type`, rows ld elements apart
    int type;
    int64_t ld;
    const float* score;                  // [batch, beams]
    int batch, beams, vocab;
    const int32_t* eos;                  // [n_eos]
    int n_eos;
    int32_t *beam, *token;               // [batch, beams] each
    float* score_out;
    int32_t *done_beam, *done_token;
    float* done_score;
};
int launch_beam_select(const BeamSelectArgs& a, cudaStream_t s);

struct ReorderArgs {
    const int32_t *parent, *kv_len, *block_table;
    int batch, beams, page_size, n_pages, max_pages;
    const int32_t* shared_len;           // [batch] or NULL
    const int32_t* free_pages;
    int free_capacity;
    const int32_t* n_free;
    const int32_t *history, *history_len, *token;
    int64_t history_stride;
    int32_t *table_out, *kv_len_out, *free_out, *n_free_out, *copy_from, *copy_to, *copy_len, *history_out, *history_len_out, *status;
};
size_t beam_reorder_scratch_bytes(int batch);
int launch_beam_reorder(const ReorderArgs& a, void* scratch, cudaStream_t s);
constexpr int kCopyLayers = 64;          // layers of one launch
int launch_cache_copy(const PagedCache* caches, int n_layers, const int32_t* from, const int32_t* to, const int32_t* len, int rows, int32_t* err_flag,
                      cudaStream_t s);

// Attention of drafted rows over the pages.
struct TreeAttnArgs {
    const void* q;                       // [rows, n_heads, d_head] of the cache's type, rows q_stride elements apart
    int64_t q_stride;
    PagedCache cache;
    const int32_t* block_table;          // [batch, max_pages]
    int max_pages;
    const int32_t *kv_len, *row_start;   // [batch], [batch + 1]
    const uint32_t* tree_mask;           // [rows, mask_words] or NULL (every draft sees the ones before it)
    int mask_words;
    int batch, rows, n_heads;
    float scale;
    void* out;
    int64_t out_stride;
    uint8_t* scratch;
    int32_t* err_flag;
};
size_t tree_attention_scratch_bytes(int type, int d_head);

// The same with a prefix shared by groups of requests.
struct PrefixAttnArgs {
    TreeAttnArgs t;                      // (t.scratch unused)
    const int32_t *group_start, *prefix_len, *request_group;     // [groups + 1], [groups], [batch]
    int groups;
};
struct PrefixScratch { uint8_t* pieces[2]; void* entries; float* partial; int* row_sides; size_t bytes; };
PrefixScratch prefix_scratch(void* base, int type, int d_head, int64_t rows, int n_heads);
int launch_prefix_attention(const PrefixAttnArgs& a, void* scratch, cudaStream_t s, bool dependent);      // 0 or a ZOQAT_ERR_* code
int launch_prefix_f32(const PrefixAttnArgs& a, const PrefixScratch& at, cudaStream_t s, bool dependent);
// tile: queries per tile of the shared and the own parts, 8, 16, 32, 64 or 256
int launch_prefix_tc(const PrefixAttnArgs& a, const PrefixScratch& at, const int (&tile)[2], cudaStream_t s, bool dependent);
int tree_grid();                         // CTAs of the attention kernels on the current device
int launch_tree_attention_simt(const TreeAttnArgs& a, cudaStream_t s, bool dependent);   // fp32; 0 or a ZOQAT_ERR_* code
int launch_tree_attention_tc(const TreeAttnArgs& a, cudaStream_t s, bool dependent);     // bf16 / fp16

// Rules on logits (zoqat_logit_rules_t).
struct LogitRules {
    const int32_t* row_request;
    int batch;
    const float *repetition, *presence, *frequency;
    const int32_t *history, *history_len, *prompt_len;
    int64_t history_stride;
    const int32_t* bias_token;
    const float* bias_value;
    const int32_t* bias_len;
    int bias_stride;
    const uint32_t* allowed;
    int64_t allowed_stride;
    const int32_t *draft_token, *row_start;
    const uint32_t* tree_mask;
    int mask_words;
};
int launch_logit_rules(const void* logits, int type, int64_t ld, int rows, int vocab, const LogitRules& r, void* out, int64_t out_ld,
                       int32_t* token, cudaStream_t s);           // 0, or -1: launch set-up failed

}  // namespace zq
