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
// A row belongs to a cluster of up to 8 CTAs; each takes a slice of the vocabulary.  The tokens that the history, the drafts or
// the biases name are marked in a bitmap of the slice.  All others stream through registers, masked, written and searched,
// with no arithmetic for rules that do not concern them; the marked ones are left out there and done by themselves: a marked
// token's place in the bitmap is its place in dense arrays of counts and bias sums (integer atomics: the order does not matter;
// one warp adds the biases up in list order), from which its logit is then computed once.  A crew of four warps counts while the
// others stream.  256 rows of 50272 binary32 logits with histories of 3000, 200 biases and a mask take 35 us, without rules 25, a
// copy of the logits 17 (passing every slice through shared memory next to dense counts took 64, counting before streaming 47).
// The cluster's choices are joined through distributed shared memory, so the choice needs no second launch and no scratch.  A
// table of counts per request would instead add its own bytes to the logits' on every step.
#include "common.cuh"
#include "serve.cuh"
#include "tc_ptx.cuh"

#include <cuda_fp16.h>

namespace zq {
namespace {

constexpr int kRuleThreads = 512;
constexpr int kMaxSlice = 65536;                // tokens whose places within a slice fit 16 bits; 1/4 byte each for marks and places
constexpr int kMaxMarked = 4096;                // marked tokens at a time, 10 bytes each: two CTAs per SM
constexpr int kCrew = 128;                      // threads that count while the others stream
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
logit_rules_kernel(const T* logits, int64_t ld, int rows, int vocab, int slice, int cap, LogitRules R, T* out, int64_t out_ld, int32_t* token) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float wv[kRuleThreads / 32];
    __shared__ int wi[kRuleThreads / 32];
    __shared__ __align__(8) uint32_t mine[2];
    __shared__ uint32_t warp_n[kCrew / 32];
    __shared__ int next_tile, marks;
    const int words = slice >> 5;
    uint32_t* allow = reinterpret_cast<uint32_t*>(smem);                 // the mask's words
    uint32_t* cnt = allow + (R.allowed ? words : 0);                     // how often marked tokens occur, in the order of the vocabulary,
    float* sum = reinterpret_cast<float*>(cnt + cap);                    // their biases
    uint32_t* bits = reinterpret_cast<uint32_t*>(sum + cap);             // the slice's marks
    uint32_t* place = bits + words;                                      // marks before each word
    uint16_t* tok = reinterpret_cast<uint16_t*>(place + words);          // and which tokens of the slice they are
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = cluster_ctarank(), ranks = cluster_nctarank();
    const int64_t row = blockIdx.y;
    const int req = R.row_request ? __ldg(R.row_request + row) : (int)row;
    if (req < 0 || req >= R.batch) return;      // the same answer in every CTA of the cluster: the row is left as it is

    const uint32_t* allowed = R.allowed ? R.allowed + row * R.allowed_stride : nullptr;
    // loads a thread has in flight; 8 tokens at a time have registers for two (four spill: 47 against 41 us)
    constexpr int kSteps = VEC == 1 ? 8 : (VEC == 4 ? 4 : 2), kTile = kSteps * 32 * VEC;  // tokens of a warp at a time
    Vec<T, VEC> raw[kSteps];
    auto fetch = [&](int k, int lo, int tile, int size) {                // step k of a tile of the slice at lo
        const int u = tile * kTile + (k * 32 + lane) * VEC;
        if (u >= size) return;
        const T* src = logits + row * ld + lo + u;
        if (u + VEC <= size) {
            raw[k] = *reinterpret_cast<const Vec<T, VEC>*>(src);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (u + e < size) raw[k].v[e] = src[e];
        }
    };
    const int step = (int)ranks * slice;
    int lo = (int)rank * slice;
    if (lo < vocab) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) fetch(k, lo, warp, min(slice, vocab - lo));
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
    const bool sparse = n_hist > 0 || n_draft > 0 || n_bias > 0;
    const int32_t* hist = R.history + (int64_t)req * R.history_stride;
    const int32_t* bias_t = R.bias_token + (int64_t)req * R.bias_stride;
    const float* bias_v = R.bias_value + (int64_t)req * R.bias_stride;

    auto occurrences = [&](int threads, auto&& f) {      // f(token, in the prompt) for the history and the drafts that the row sees
        for (int k0 = tid; k0 < n_hist; k0 += 8 * threads) {
            int t[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] = k0 + k * threads < n_hist ? __ldg(hist + k0 + k * threads) : -1;      // -1 falls into no slice
#pragma unroll
            for (int k = 0; k < 8; ++k) f(t[k], k0 + k * threads < n_prompt);
        }
        for (int j = tid; j < n_draft; j += threads)
            if ((__ldg(R.tree_mask + row * R.mask_words + (j >> 5)) >> (j & 31)) & 1u) f(__ldg(R.draft_token + draft0 + j), false);
    };
    auto crew_sync = [] { asm volatile("bar.sync 1, %0;" ::"n"(kCrew) : "memory"); };

    const T none = from_f32<T>(-INFINITY);
    Best best{-INFINITY, -1};
    for (; lo < vocab; lo += step) {
        const int size = min(slice, vocab - lo);
        auto inside = [&](int t) { return t >= 0 && (uint32_t)(t - lo) < (uint32_t)size; };
        auto place_of = [&](int u) { return (int)(place[u >> 5] + __popc(bits[u >> 5] & ((1u << (u & 31)) - 1u))); };
        __syncthreads();                        // the slice before has been read
        if (tid == 0) { next_tile = kRuleThreads / 32; marks = 0; }
        if (allowed)
            for (int u = tid; u < (size + 31) >> 5; u += kRuleThreads) allow[u] = __ldg(allowed + (lo >> 5) + u);
        if (sparse) {
            for (int u = tid; u < words; u += kRuleThreads) bits[u] = 0;
            for (int u = tid; u < 2 * cap; u += kRuleThreads) cnt[u] = 0;        // and the sums
            __syncthreads();
            auto mark = [&](int t, bool) { if (inside(t)) atomicOr(&bits[(t - lo) >> 5], 1u << ((t - lo) & 31)); };
            occurrences(kRuleThreads, mark);
            for (int k = tid; k < n_bias; k += kRuleThreads) mark(__ldg(bias_t + k), false);
        }
        __syncthreads();
        auto count = [&](int first) {           // counts and bias sums of the marked tokens [first, first + cap); by the crew
            occurrences(kCrew, [&](int t, bool prompt) {
                if (!inside(t)) return;
                const int i = place_of(t - lo) - first;
                if (i < 0 || i >= cap) return;
                if (prompt) atomicOr(&cnt[i], kSeenPrompt); else atomicAdd(&cnt[i], 1u);
                tok[i] = (uint16_t)(t - lo);
            });
            if (warp == kCrew / 32 - 1) {
                int t = lane < n_bias ? __ldg(bias_t + lane) : -1;
                float v = lane < n_bias ? __ldg(bias_v + lane) : 0.0f;
                for (int k = lane; k - lane < n_bias; k += 32) {
                    const int t_next = k + 32 < n_bias ? __ldg(bias_t + k + 32) : -1;
                    const float v_next = k + 32 < n_bias ? __ldg(bias_v + k + 32) : 0.0f;
                    int i = inside(t) ? place_of(t - lo) - first : -1;
                    const bool live = i >= 0 && i < cap;
                    if (live) tok[i] = (uint16_t)(t - lo); else i = -1 - lane;
                    const int turn = __popc(__match_any_sync(0xffffffffu, i) & ((1u << lane) - 1));      // entries of this token before
                    for (int r = 0; __any_sync(0xffffffffu, live && r <= turn); ++r) {
                        if (live && r == turn) sum[i] = __fadd_rn(sum[i], v);
                        __syncwarp();
                    }
                    t = t_next; v = v_next;
                }
            }
        };
        if (sparse && tid < kCrew) {            // the marks' places, and the first counts
            const int per = (words + kCrew - 1) / kCrew, u0 = min(tid * per, words), u1 = min(u0 + per, words);
            uint32_t n = 0;
            for (int u = u0; u < u1; ++u) n += __popc(bits[u]);
            uint32_t up = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t x = __shfl_up_sync(0xffffffffu, up, o); if (lane >= o) up += x; }
            if (lane == 31) warp_n[warp] = up;
            crew_sync();
            up -= n;
            for (int w = 0; w < warp; ++w) up += warp_n[w];
            for (int u = u0; u < u1; ++u) { place[u] = up; up += __popc(bits[u]); }
            if (tid == kCrew - 1) marks = (int)up;
            crew_sync();
            count(0);
        }
        // the tokens that nothing concerns, and their mask; the warps take the tiles in turn, the crew's when they get there
        for (int tile = warp; tile * kTile < size;) {
            int next = 0;
            if (lane == 0) next = atomicAdd(&next_tile, 1);
            next = __shfl_sync(0xffffffffu, next, 0);
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                const int u = tile * kTile + (k * 32 + lane) * VEC;
                uint32_t word = 0xFFFFFFFFu, left = u + VEC <= size ? 0xFFFFFFFFu : (1u << max(size - u, 0)) - 1u;
                if (u < size) {
                    if (allowed) word = allow[u >> 5] >> (u & 31);
                    if (sparse) left &= ~(bits[u >> 5] >> (u & 31));
                }
                Vec<T, VEC> y;
                float top = -INFINITY, x[VEC];
                const uint32_t both = word & left;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    y.v[e] = (word >> e) & 1u ? raw[k].v[e] : none;
                    x[e] = (both >> e) & 1u ? to_f32<T>(raw[k].v[e]) : -INFINITY;
                    top = fmaxf(top, x[e]);
                }
                fetch(k, lo, next, size);
                if (out) {
                    T* dst = out + row * out_ld + lo + u;
                    if ((left & ((1u << VEC) - 1u)) == (1u << VEC) - 1u) {
                        *reinterpret_cast<Vec<T, VEC>*>(dst) = y;
                    } else {
#pragma unroll
                        for (int e = 0; e < VEC; ++e)
                            if ((left >> e) & 1u) dst[e] = y.v[e];
                    }
                }
                if (top > best.v) {                              // a thread sees its tokens in ascending order; NaN is never larger
                    best.v = top;
#pragma unroll
                    for (int e = VEC - 1; e >= 0; --e)
                        if (x[e] == top) best.i = lo + u + e;
                }
            }
            tile = next;
        }
        if (lo + step < vocab) {
#pragma unroll
            for (int k = 0; k < kSteps; ++k) fetch(k, lo + step, warp, min(slice, vocab - lo - step));
        }
        if (!sparse) continue;
        // the marked ones, `cap` at a time
        __syncthreads();                        // places, counts and sums are complete
        const int marked = marks;
        for (int first = 0; first < marked; first += cap) {
            if (first > 0) {
                __syncthreads();
                for (int u = tid; u < 2 * cap; u += kRuleThreads) cnt[u] = 0;
                __syncthreads();
                if (tid < kCrew) count(first);
                __syncthreads();
            }
            for (int i = tid; i < min(cap, marked - first); i += kRuleThreads) {
                const int u = tok[i], v = lo + u;
                const uint32_t c = cnt[i], n = c & ~kSeenPrompt;
                float x = to_f32<T>(logits[row * ld + v]);
                if (c) {
                    x = x > 0.0f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
                    x = __fsub_rn(x, __fmul_rn(freq, (float)n));
                    if (n) x = __fsub_rn(x, pres);
                }
                if (sum[i] != 0.0f) x = __fadd_rn(x, sum[i]);
                if (allowed && !((allow[u >> 5] >> (u & 31)) & 1u)) x = -INFINITY;
                const T y = from_f32<T>(x);
                x = to_f32<T>(y);
                if (out) out[row * out_ld + v] = y;
                if (x > -INFINITY) take_better(best, x, v);
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
                 cudaStream_t s) {
    // at least 1024 tokens to a CTA, and no more CTAs of a cluster than it takes to fill the SMs (1 / 2 / 4 / 8 CTAs a row, histories
    // of 700, us: 8 rows of 32000 16 / 14 / 14 / 13; 64 of 50272 21 / 16 / 16 / 25; 256 of 50272 29 / 35 / 47 / 74)
    int ranks = 1;
    while (ranks < 8 && vocab > 1024 * ranks && rows * ranks < 148) ranks *= 2;
    const int slices = (vocab + ranks * kMaxSlice - 1) / (ranks * kMaxSlice) * ranks;
    const int slice = ((vocab + slices - 1) / slices + 31) / 32 * 32, cap = slice < kMaxMarked ? slice : kMaxMarked;
    const size_t smem = ((r.history || r.draft_token || r.bias_token) ? (size_t)cap * 10 + slice / 4 : 0) + (r.allowed ? slice / 8 : 0);
    static DeviceOnce attr;
    if (!attr.done([] { return allow_smem(logit_rules_kernel<T, VEC>, kMaxMarked * 10 + kMaxSlice / 8 * 3); })) return -1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ranks, rows);
    cfg.blockDim = dim3(kRuleThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ranks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, logit_rules_kernel<T, VEC>, logits, ld, rows, vocab, slice, cap, r, out, out_ld, token) != cudaSuccess) return -1;
    count_launch();
    return 0;
}

template <typename T>
int launch_rules(const T* logits, int64_t ld, int rows, int vocab, const LogitRules& r, T* out, int64_t out_ld, int32_t* token,
                 cudaStream_t s) {
    // every row begins at 16 bytes: vectors (a row of an odd vocabulary packed tightly does not)
    const uintptr_t at = reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(out) | (uintptr_t)(ld * sizeof(T)) | (uintptr_t)(out_ld * sizeof(T));
    if (at % 16 == 0) return launch_rules_vec<T, 16 / sizeof(T)>(logits, ld, rows, vocab, r, out, out_ld, token, s);
    return launch_rules_vec<T, 1>(logits, ld, rows, vocab, r, out, out_ld, token, s);
}

}  // namespace

int launch_logit_rules(const void* logits, int type, int64_t ld, int rows, int vocab, const LogitRules& r, void* out, int64_t out_ld,
                       int32_t* token, cudaStream_t s) {
    if (type == kTypeF32) return launch_rules(static_cast<const float*>(logits), ld, rows, vocab, r, static_cast<float*>(out), out_ld, token, s);
    if (type == kTypeBf16) return launch_rules(static_cast<const __nv_bfloat16*>(logits), ld, rows, vocab, r, static_cast<__nv_bfloat16*>(out), out_ld, token, s);
    return launch_rules(static_cast<const __half*>(logits), ld, rows, vocab, r, static_cast<__half*>(out), out_ld, token, s);
}

}  // namespace zq
