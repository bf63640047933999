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
// A row belongs to a cluster of up to 8 CTAs; each takes slices of the vocabulary, whose logits it has requested while it worked
// on the slice before.  A slice with penalties or biases passes through shared memory: the history tokens that fall into it are
// counted (integer atomics: the order does not matter), whoever takes a token's count applies the penalties to its logit, one
// warp adds the biases in list order - so the many tokens that nothing concerns cost no arithmetic for it -, then the slice is
// masked, rounded, written and searched.  The cluster's choices are joined through distributed shared memory, so the choice
// needs no second launch and no scratch.  The history (its first 4096 tokens) is read once and kept in registers; a dense table of
// counts per request would instead add its own bytes to the logits' on every step.
#include "common.cuh"
#include "serve.cuh"
#include "tc_ptx.cuh"

#include <cuda_fp16.h>

namespace zq {
namespace {

constexpr int kRuleThreads = 512;
constexpr int kMaxSlice = 8192;                 // 10 bytes of shared memory a token of the slice, 16 tokens a thread: two CTAs per SM
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

// VEC tokens at a time: 16 bytes where the rows allow it (4 or 8 tokens), else single ones
template <typename T, int VEC> struct alignas(VEC * sizeof(T)) Vec { T v[VEC]; };

// logits and out may be the same rows: no __restrict__, and every element is read and written by one thread
template <typename T, int VEC>
__global__ void __launch_bounds__(kRuleThreads, 2)
logit_rules_kernel(const T* logits, int64_t ld, int rows, int vocab, int slice, LogitRules R, T* out, int64_t out_ld, int32_t* token) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float wv[kRuleThreads / 32];
    __shared__ int wi[kRuleThreads / 32];
    __shared__ __align__(8) uint32_t mine[2];
    __shared__ int list_n[kRuleThreads / 32], met_n;
    __shared__ float2 list[kRuleThreads];       // the slice's entries of the bias list, in its order
    float* xs = reinterpret_cast<float*>(smem);                          // the slice's logits ...
    uint32_t* cnt = reinterpret_cast<uint32_t*>(smem) + slice;           // ... how often their tokens occur (then: the sums of their biases) ...
    uint16_t* met = reinterpret_cast<uint16_t*>(cnt + slice);            // ... and which tokens occur, in any order
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = cluster_ctarank(), ranks = cluster_nctarank();
    const int64_t row = blockIdx.y;
    grid_dependency_wait();
    const int req = R.row_request ? __ldg(R.row_request + row) : (int)row;
    if (req < 0 || req >= R.batch) return;      // the same answer in every CTA of the cluster: the row is left as it is

    const uint32_t* allowed = R.allowed ? R.allowed + row * R.allowed_stride : nullptr;
    constexpr int kSteps = kMaxSlice / (kRuleThreads * VEC);
    Vec<T, VEC> raw[kSteps];
    uint32_t ok[VEC == 1 ? 1 : kSteps];         // the mask's words of the thread's tokens
    auto fetch = [&](int k, int lo) {           // step k of the slice at lo
        const int u = lo + (tid + k * kRuleThreads) * VEC, end = min(lo + slice, vocab);
        if (u + VEC <= end) {
            raw[k] = *reinterpret_cast<const Vec<T, VEC>*>(logits + row * ld + u);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (u + e < end) raw[k].v[e] = logits[row * ld + u + e];
        }
    };
    auto fetch_mask = [&](int k, int lo) {
        const int u = lo + (tid + k * kRuleThreads) * VEC;
        ok[VEC == 1 ? 0 : k] = allowed && u < min(lo + slice, vocab) ? __ldg(allowed + (u >> 5)) >> (u & 31) : 0xFFFFFFFFu;
    };
    // (single tokens) a warp's 32 tokens of step k share one word (slices begin at whole words): lane k keeps that of step k
    auto fetch_words = [&](int lo) {
        const int u = lo + warp * 32 + lane * kRuleThreads;
        ok[0] = allowed && lane < kSteps && u < min(lo + slice, vocab) ? __ldg(allowed + (u >> 5)) : 0xFFFFFFFFu;
    };
    const int step = (int)ranks * slice;
    int lo = (int)rank * slice;
    if (lo < vocab) {
        if (VEC == 1) fetch_words(lo);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) { fetch(k, lo); if (VEC > 1) fetch_mask(k, lo); }
    }

    // the request's words, all at once
    int n_hist = R.history ? __ldg(R.history_len + req) : 0;
    const int n_prompt = R.history && R.prompt_len ? __ldg(R.prompt_len + req) : 0;
    int n_bias = R.bias_token ? __ldg(R.bias_len + req) : 0;
    const int draft0 = R.draft_token ? __ldg(R.row_start + req) : 0;
    int n_draft = R.draft_token ? __ldg(R.row_start + req + 1) - draft0 : 0;
    const float rep = R.repetition ? __ldg(R.repetition + req) : 1.0f;
    const float freq = R.frequency ? __ldg(R.frequency + req) : 0.0f;
    const float pres = R.presence ? __ldg(R.presence + req) : 0.0f;
    n_hist = n_hist < 0 ? 0 : (n_hist > R.history_stride ? (int)R.history_stride : n_hist);
    n_bias = n_bias < 0 ? 0 : (n_bias > R.bias_stride ? R.bias_stride : n_bias);
    if (draft0 < 0 || n_draft < 0 || (int64_t)draft0 + n_draft > rows) n_draft = 0;
    if (n_draft > 32 * R.mask_words) n_draft = 32 * R.mask_words;
    const bool counted = n_hist > 0 || n_draft > 0, sparse = counted || n_bias > 0;
    const int32_t* hist = R.history + (int64_t)req * R.history_stride;

    // The first tokens of the history, the drafts and the biases stay in registers through all slices.  Whatever is not there
    // is -1, which falls into no slice.
    constexpr int kHeld = 8;
    int held[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) held[k] = tid + k * kRuleThreads < n_hist ? __ldg(hist + tid + k * kRuleThreads) : -1;
    auto draft_at = [&](int j) {                // draft j's token if this row sees it
        return (__ldg(R.tree_mask + row * R.mask_words + (j >> 5)) >> (j & 31)) & 1u ? __ldg(R.draft_token + draft0 + j) : -1;
    };
    const int draft = tid < n_draft ? draft_at(tid) : -1;
    const int bias_token = tid < n_bias ? __ldg(R.bias_token + (int64_t)req * R.bias_stride + tid) : -1;
    const float bias_value = tid < n_bias ? __ldg(R.bias_value + (int64_t)req * R.bias_stride + tid) : 0.0f;
    if (tid == 0) met_n = 0;
    if (sparse)
        for (int u = tid; u < (slice >> 2); u += kRuleThreads) reinterpret_cast<uint4*>(cnt)[u] = make_uint4(0, 0, 0, 0);

    Best best{-INFINITY, -1};
    for (; lo < vocab; lo += step) {
        const int size = min(slice, vocab - lo);
        const bool more = lo + step < vocab;
        T* dst = out ? out + row * out_ld + lo : nullptr;
        if (sparse) {
            __syncthreads();                    // the counts are clear, the slice before has been read
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                const int u = (tid + k * kRuleThreads) * VEC;
                if (u < size) {
                    Vec<float, VEC> x;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x.v[e] = to_f32<T>(raw[k].v[e]);
                    *reinterpret_cast<Vec<float, VEC>*>(xs + u) = x;
                }
                if (more) fetch(k, lo + step);  // in flight while this slice is worked on
            }
            if (counted) {
                auto count = [&](int t, bool prompt) {
                    const uint32_t u = (uint32_t)(t - lo);
                    if (t < 0 || u >= (uint32_t)size) return;
                    const uint32_t old = prompt ? atomicOr(&cnt[u], kSeenPrompt) : atomicAdd(&cnt[u], 1u);
                    if (!old) met[atomicAdd(&met_n, 1)] = (uint16_t)u;
                };
#pragma unroll
                for (int k = 0; k < kHeld; ++k) count(held[k], tid + k * kRuleThreads < n_prompt);
                for (int k = kHeld * kRuleThreads + tid; k < n_hist; k += kRuleThreads) count(__ldg(hist + k), k < n_prompt);
                for (int j = tid; j < n_draft; j += kRuleThreads) count(j == tid ? draft : draft_at(j), false);
                __syncthreads();
                // the tokens that occur, spread over all threads: their penalties, and their counts cleared for the next slice
                for (int i = tid; i < met_n; i += kRuleThreads) {
                    const int u = met[i];
                    const uint32_t c = cnt[u], n = c & ~kSeenPrompt;
                    cnt[u] = 0;
                    float x = xs[u];
                    x = x > 0.0f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
                    x = __fsub_rn(x, __fmul_rn(freq, (float)n));
                    if (n) x = __fsub_rn(x, pres);
                    xs[u] = x;
                }
                if (n_bias) __syncthreads();
            }
            auto add_sum = [&](int u) {         // whoever takes a token's sum first (and clears it for the next slice) adds it
                const float sum = __uint_as_float(atomicExch(&cnt[u], 0u));
                if (sum != 0.0f) xs[u] = __fadd_rn(xs[u], sum);
            };
            for (int k0 = 0; k0 < n_bias; k0 += kRuleThreads) {
                // the slice's entries, in the order of the list; then one warp sums them per token and adds the sums
                const int k = k0 + tid;
                const int t = k0 == 0 ? bias_token : (k < n_bias ? __ldg(R.bias_token + (int64_t)req * R.bias_stride + k) : -1);
                const float v = k0 == 0 ? bias_value : (k < n_bias ? __ldg(R.bias_value + (int64_t)req * R.bias_stride + k) : 0.0f);
                const uint32_t u = (uint32_t)(t - lo);
                const bool in = t >= 0 && u < (uint32_t)size;
                const uint32_t all = __ballot_sync(0xffffffffu, in);
                if (lane == 0) list_n[warp] = __popc(all);
                __syncthreads();
                int at = __popc(all & ((1u << lane) - 1)), n = 0;
                for (int w = 0; w < kRuleThreads / 32; ++w) { if (w < warp) at += list_n[w]; n += list_n[w]; }
                if (in) list[at] = make_float2(__int_as_float((int)u), v);
                __syncthreads();
                if (warp == 0) {
                    float* sum = reinterpret_cast<float*>(cnt);
                    for (int i0 = 0; i0 < n; i0 += 32) {
                        const bool live = i0 + lane < n;
                        const float2 e = live ? list[i0 + lane] : make_float2(0.0f, 0.0f);
                        const int x = live ? __float_as_int(e.x) : -1 - lane;
                        const int turn = __popc(__match_any_sync(0xffffffffu, x) & ((1u << lane) - 1));      // entries of this token before
                        for (int i = 0; __any_sync(0xffffffffu, live && i <= turn); ++i) {
                            if (live && i == turn) sum[x] = __fadd_rn(sum[x], e.y);
                            __syncwarp();
                        }
                    }
                }
                if (n_bias > kRuleThreads) __syncthreads();      // the list is written again
                else if (warp == 0)
                    for (int i = lane; i < n; i += 32) add_sum(__float_as_int(list[i].x));
            }
            if (n_bias > kRuleThreads)                           // (a long list: its tokens once more)
                for (int k = tid; k < n_bias; k += kRuleThreads) {
                    const int t = __ldg(R.bias_token + (int64_t)req * R.bias_stride + k);
                    if (t >= 0 && (uint32_t)(t - lo) < (uint32_t)size) add_sum(t - lo);
                }
            __syncthreads();
            if (tid == 0) met_n = 0;
        }
        const uint32_t words = ok[0];
        if (VEC == 1 && more) fetch_words(lo + step);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int u = (tid + k * kRuleThreads) * VEC;
            const uint32_t word = VEC == 1 ? __shfl_sync(0xffffffffu, words, k) >> lane : ok[VEC == 1 ? 0 : k];
            float x[VEC];
            if (sparse) {
                const Vec<float, VEC> s = u < size ? *reinterpret_cast<const Vec<float, VEC>*>(xs + u) : Vec<float, VEC>{};
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[e] = s.v[e];
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[e] = to_f32<T>(raw[k].v[e]);
                if (more) fetch(k, lo + step);
            }
            if (VEC > 1 && more) fetch_mask(k, lo + step);
            if (u >= size) continue;
            Vec<T, VEC> y;
            float top = -INFINITY;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (!((word >> e) & 1u)) x[e] = -INFINITY;
                y.v[e] = from_f32<T>(x[e]);
                x[e] = to_f32<T>(y.v[e]);
                if (u + e < size) top = fmaxf(top, x[e]);
            }
            if (dst) {
                if (u + VEC <= size) {
                    *reinterpret_cast<Vec<T, VEC>*>(dst + u) = y;
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (u + e < size) dst[u + e] = y.v[e];
                }
            }
            if (top > best.v) {                                  // a thread sees its tokens in ascending order; NaN is never larger
                best.v = top;
#pragma unroll
                for (int e = VEC - 1; e >= 0; --e)
                    if (u + e < size && x[e] == top) best.i = lo + u + e;
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

template <typename T, int VEC>
int launch_rules_vec(const T* logits, int64_t ld, int rows, int vocab, const LogitRules& r, T* out, int64_t out_ld, int32_t* token,
                 cudaStream_t s, bool dependent) {
    // at least 1024 tokens to a CTA, and no more CTAs of a cluster than it takes to fill the SMs: a CTA with several slices
    // requests each while it works on the one before
    int ranks = 1;
    while (ranks < 8 && vocab > 1024 * ranks && rows * ranks < 148) ranks *= 2;
    const int slices = (vocab + ranks * kMaxSlice - 1) / (ranks * kMaxSlice) * ranks;
    const int slice = ((vocab + slices - 1) / slices + 31) / 32 * 32;
    const size_t smem = (r.history || r.draft_token || r.bias_token) ? (size_t)slice * 10 : 0;
    static DeviceOnce attr;
    if (attr.first() && cudaFuncSetAttribute(logit_rules_kernel<T, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlice * 10) != cudaSuccess) {
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
    if (cudaLaunchKernelEx(&cfg, logit_rules_kernel<T, VEC>, logits, ld, rows, vocab, slice, r, out, out_ld, token) != cudaSuccess) return -1;
    count_launch();
    return 0;
}

template <typename T>
int launch_rules(const T* logits, int64_t ld, int rows, int vocab, const LogitRules& r, T* out, int64_t out_ld, int32_t* token,
                 cudaStream_t s, bool dependent) {
    // every row begins at 16 bytes: vectors (a row of an odd vocabulary packed tightly does not)
    const uintptr_t at = reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(out) | (uintptr_t)(ld * sizeof(T)) | (uintptr_t)(out_ld * sizeof(T));
    if (at % 16 == 0) return launch_rules_vec<T, 16 / sizeof(T)>(logits, ld, rows, vocab, r, out, out_ld, token, s, dependent);
    return launch_rules_vec<T, 1>(logits, ld, rows, vocab, r, out, out_ld, token, s, dependent);
}

}  // namespace

int launch_logit_rules(const void* logits, int type, int64_t ld, int rows, int vocab, const LogitRules& r, void* out, int64_t out_ld,
                       int32_t* token, cudaStream_t s, bool dependent) {
    if (type == kTypeF32) return launch_rules(static_cast<const float*>(logits), ld, rows, vocab, r, static_cast<float*>(out), out_ld, token, s, dependent);
    if (type == kTypeBf16) return launch_rules(static_cast<const __nv_bfloat16*>(logits), ld, rows, vocab, r, static_cast<__nv_bfloat16*>(out), out_ld, token, s, dependent);
    return launch_rules(static_cast<const __half*>(logits), ld, rows, vocab, r, static_cast<__half*>(out), out_ld, token, s, dependent);
}

}  // namespace zq
