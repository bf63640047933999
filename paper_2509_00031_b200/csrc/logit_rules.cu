// Rules on the logits of a serving step, and the greedy choice under them, in one pass over the logits:
//
//   x  = logits[r, v]
//   x  = x > 0 ? x / repetition : x * repetition      if v stands in the request's prompt or among its generated tokens
//   x  = x - frequency * n                            n = how often v was generated (drafted ancestors of the row included)
//   x  = x - presence                                 if n > 0
//   x  = x + bias                                     the request's entries for v, added up in the order of the list
//   x  = -inf                                         if the row's grammar mask forbids v
//   out[r, v] = x in the logits' type, token[r] = the lowest v with the largest out[r, v] (-1: nothing above -inf)
//
// Every operation is one binary32 rounding in this order (no contraction), so the choice is the one the formula gives.
//
// A row belongs to a cluster of up to 8 CTAs; each takes slices of the vocabulary.  For a slice the CTA counts the history
// tokens that fall into it in shared memory (integer atomics: the order does not matter), adds the biases up in a second
// array (one warp, list order), streams the slice once and keeps its best (value, index).  The cluster's choices are joined
// through distributed shared memory, so the choice needs no second launch and no scratch.  The history is read once per
// slice, from L2; a dense table of counts per request would instead add its own bytes to the logits' on every step.
#include "common.cuh"
#include "serve.cuh"
#include "tc_ptx.cuh"

#include <cuda_fp16.h>

namespace zq {
namespace {

constexpr int kRuleThreads = 512;
constexpr int kMaxSlice = 8192;                 // 8 bytes a token of the slice: three CTAs of 64 KB fit on an SM
constexpr uint32_t kSeenPrompt = 0x80000000u;   // counts share their word with the prompt's mark

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

struct Best { float v; int i; };
__device__ __forceinline__ void take_better(Best& a, float v, int i) {
    if (v > a.v || (v == a.v && (uint32_t)i < (uint32_t)a.i)) { a.v = v; a.i = i; }   // index -1 (none) is the largest
}

__device__ __forceinline__ uint32_t cluster_nctarank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// logits and out may be the same rows: no __restrict__, and every element is read and written by one thread
template <typename T>
__global__ void __launch_bounds__(kRuleThreads)
logit_rules_kernel(const T* logits, int64_t ld, int rows, int vocab, int slice, LogitRules R, T* out, int64_t out_ld, int32_t* token) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float wv[kRuleThreads / 32];
    __shared__ int wi[kRuleThreads / 32];
    __shared__ __align__(8) uint32_t mine[2];
    uint32_t* cnt = reinterpret_cast<uint32_t*>(smem);
    float* add = reinterpret_cast<float*>(smem) + slice;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = cluster_ctarank(), ranks = cluster_nctarank();
    const int64_t row = blockIdx.y;
    grid_dependency_wait();
    const int req = R.row_request ? __ldg(R.row_request + row) : (int)row;
    if (req < 0 || req >= R.batch) return;      // the same answer in every CTA of the cluster: the row is left as it is

    int n_hist = 0, n_prompt = 0, n_bias = 0, n_draft = 0, draft0 = 0;
    if (R.history) {
        n_hist = __ldg(R.history_len + req);
        n_hist = n_hist < 0 ? 0 : (n_hist > R.history_stride ? (int)R.history_stride : n_hist);
        n_prompt = R.prompt_len ? __ldg(R.prompt_len + req) : 0;
    }
    if (R.bias_token) {
        n_bias = __ldg(R.bias_len + req);
        n_bias = n_bias < 0 ? 0 : (n_bias > R.bias_stride ? R.bias_stride : n_bias);
    }
    if (R.draft_token) {
        draft0 = __ldg(R.row_start + req);
        n_draft = __ldg(R.row_start + req + 1) - draft0;
        if (draft0 < 0 || n_draft < 0 || (int64_t)draft0 + n_draft > rows) n_draft = 0;
        if (n_draft > 32 * R.mask_words) n_draft = 32 * R.mask_words;
    }
    const bool counted = n_hist > 0 || n_draft > 0;
    const float rep = R.repetition ? __ldg(R.repetition + req) : 1.0f;
    const float freq = R.frequency ? __ldg(R.frequency + req) : 0.0f;
    const float pres = R.presence ? __ldg(R.presence + req) : 0.0f;
    const int32_t* hist = R.history + (int64_t)req * R.history_stride;
    const uint32_t* allowed = R.allowed ? R.allowed + row * R.allowed_stride : nullptr;

    Best best{-INFINITY, -1};
    for (int lo = (int)rank * slice; lo < vocab; lo += (int)ranks * slice) {
        const int size = min(slice, vocab - lo);
        if (counted || n_bias) {
            __syncthreads();                    // the slice before has been streamed
            for (int u = tid; u < size; u += kRuleThreads) { cnt[u] = 0; add[u] = 0.0f; }
            __syncthreads();
            if (warp == 0) {
                // entries for the same token are added in the order of the list: lane by lane where one warp load has several
                for (int k0 = 0; k0 < n_bias; k0 += 32) {
                    const int k = k0 + lane;
                    const int u = k < n_bias ? __ldg(R.bias_token + (int64_t)req * R.bias_stride + k) - lo : -1;
                    const float v = k < n_bias ? __ldg(R.bias_value + (int64_t)req * R.bias_stride + k) : 0.0f;
                    const bool in = (uint32_t)u < (uint32_t)size;
                    const uint32_t same = __match_any_sync(0xffffffffu, in ? u : -1 - lane);
                    uint32_t left = same & ((1u << lane) - 1);           // lanes before this one with the same token
                    for (int turn = __popc(left), t = 0; __any_sync(0xffffffffu, in && t <= turn); ++t) {
                        if (in && t == turn) add[u] = __fadd_rn(add[u], v);
                        __syncwarp();
                    }
                }
            }
            for (int k = tid; k < n_hist; k += kRuleThreads) {
                const uint32_t u = (uint32_t)(__ldg(hist + k) - lo);
                if (u < (uint32_t)size) {
                    if (k < n_prompt) atomicOr(&cnt[u], kSeenPrompt); else atomicAdd(&cnt[u], 1u);
                }
            }
            for (int j = tid; j < n_draft; j += kRuleThreads) {
                if ((__ldg(R.tree_mask + row * R.mask_words + (j >> 5)) >> (j & 31)) & 1u) {
                    const uint32_t u = (uint32_t)(__ldg(R.draft_token + draft0 + j) - lo);
                    if (u < (uint32_t)size) atomicAdd(&cnt[u], 1u);
                }
            }
            __syncthreads();
        }
        const T* src = logits + row * ld + lo;
        T* dst = out ? out + row * out_ld + lo : nullptr;
        for (int u0 = tid; u0 < size; u0 += 4 * kRuleThreads) {
            T raw[4];
            uint32_t word[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int u = u0 + k * kRuleThreads;
                if (u < size) {
                    raw[k] = src[u];
                    if (allowed) word[k] = __ldg(allowed + ((lo + u) >> 5));
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int u = u0 + k * kRuleThreads;
                if (u < size) {
                    float x = to_f32<T>(raw[k]);
                    if (counted) {
                        const uint32_t c = cnt[u];
                        if (c) {
                            const uint32_t n = c & ~kSeenPrompt;
                            x = x > 0.0f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
                            x = __fsub_rn(x, __fmul_rn(freq, (float)n));
                            if (n) x = __fsub_rn(x, pres);
                        }
                    }
                    if (n_bias) x = __fadd_rn(x, add[u]);
                    if (allowed && !((word[k] >> ((lo + u) & 31)) & 1u)) x = -INFINITY;
                    const T y = from_f32<T>(x);
                    if (dst) dst[u] = y;
                    const float yf = to_f32<T>(y);
                    if (yf > best.v) { best.v = yf; best.i = lo + u; }       // a thread sees its tokens in ascending order
                }
            }
        }
    }
    if (!token) return;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float ov = __shfl_xor_sync(0xffffffffu, best.v, o);
        const int oi = __shfl_xor_sync(0xffffffffu, best.i, o);
        take_better(best, ov, oi);
    }
    if (lane == 0) { wv[warp] = best.v; wi[warp] = best.i; }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kRuleThreads / 32; ++w) take_better(best, wv[w], wi[w]);
        mine[0] = __float_as_uint(best.v);
        mine[1] = (uint32_t)best.i;
    }
    if (ranks > 1) {
        cluster_sync_all();
        if (rank == 0 && tid == 0) {
            for (uint32_t c = 1; c < ranks; ++c) {
                const uint32_t at = mapa_shared(smem_u32(mine), c);
                take_better(best, __uint_as_float(ld_cluster_u32(at)), (int)ld_cluster_u32(at + 4));
            }
        }
        cluster_sync_all();                     // a CTA's word stays until rank 0 has read it
    }
    if (rank == 0 && tid == 0) token[row] = best.i;
}

template <typename T>
int launch_rules(const T* logits, int64_t ld, int rows, int vocab, const LogitRules& r, T* out, int64_t out_ld, int32_t* token,
                 cudaStream_t s, bool dependent) {
    // at least 1024 tokens to a CTA of a cluster, slices of whole mask words that divide the vocabulary evenly
    int ranks = 1;
    while (ranks < 8 && vocab > 1024 * ranks) ranks *= 2;
    const int slices = (vocab + ranks * kMaxSlice - 1) / (ranks * kMaxSlice) * ranks;
    const int slice = ((vocab + slices - 1) / slices + 31) / 32 * 32;
    const size_t smem = (r.history || r.draft_token || r.bias_token) ? (size_t)slice * 8 : 0;
    static DeviceOnce attr;
    if (attr.first() && cudaFuncSetAttribute(logit_rules_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlice * 8) != cudaSuccess) {
        attr.retry();
        return -1;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ranks, rows);
    cfg.blockDim = dim3(kRuleThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ranks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = dependent ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, logit_rules_kernel<T>, logits, ld, rows, vocab, slice, r, out, out_ld, token) != cudaSuccess) return -1;
    count_launch();
    return 0;
}

}  // namespace

int launch_logit_rules(const void* logits, int type, int64_t ld, int rows, int vocab, const LogitRules& r, void* out, int64_t out_ld,
                       int32_t* token, cudaStream_t s, bool dependent) {
    if (type == kTypeF32) return launch_rules(static_cast<const float*>(logits), ld, rows, vocab, r, static_cast<float*>(out), out_ld, token, s, dependent);
    if (type == kTypeBf16) return launch_rules(static_cast<const __nv_bfloat16*>(logits), ld, rows, vocab, r, static_cast<__nv_bfloat16*>(out), out_ld, token, s, dependent);
    return launch_rules(static_cast<const __half*>(logits), ld, rows, vocab, r, static_cast<__half*>(out), out_ld, token, s, dependent);
}

}  // namespace zq
