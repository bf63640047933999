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
