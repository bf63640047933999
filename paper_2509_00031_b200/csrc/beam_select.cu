// The best continuations of a request's beams over the vocabulary, in one pass over the logits.
//
//   score(b, v) = s[b] + x[b, v] - log sum_u exp x[b, u]          beams b of a request, tokens v; ordered by score, then beam, then logit, then token
//
// Of the beams * (1 + n_eos) best, the first `beams` whose token does not end the text go on; those among the first `beams` whose token
// does are finished.  No row needs more than its own beams + n_eos best logits for that, and within a row the order of scores is that of
// logits, so a row's sum of exponentials and its best logits are found side by side while it streams through registers once.
//
// A cluster of up to 8 CTAs serves a request: a CTA takes whole rows, or a slice of one where there are few.  Of a row's first few thousand
// logits every warp knows its largest few: the least of those is a bound that at least as many logits pass as are wanted.  What passes it
// goes to a buffer, whose sorted best (each key counts the larger ones) set the exact bound for the rest of the row; a logit that
// passes that is rare, so the stream costs a maximum, an exponential and two additions each, sixteen bytes at a time, the next on their way while some are
// worked on.  Keys are (logit, token) in 64 bits: no two are equal, and of equal logits the lower token wins.
// Should the buffer run over, the row's bound is found digit by digit from histograms instead, ten more passes over the row: right, and slow.  That takes long runs of rising or
// equal logits; more than 32 best wanted of a row by a CTA of 256 threads, whose eight warps offer four each (64 x 32 beams of 50272 with one ending token 3420 us, without 313);
// or a first round with fewer live logits than are wanted and thousands behind it (64 x 8 of 50272 whose first 8192 are ruled out 918 us, against 32; one live logit in a thousand 74 us
// where -inf rules the others out, 865 where -1e9 does).
// 64 x 8 beams of 50272 logits: fp32 30 us, 16 of them the 103 MB at the rate of a copy, bf16 27; 96 x 3 of 128256 bf16 with nine tenths masked 33 (11); 4 of 32000 fp32 12.5.  The stream
// itself runs at 7 TB/s (16-bit logits: bound by the exponentials; rows that do not begin on 16 bytes, 50257 of them, 34 and 31 us); 5.5 us go before it (start, first bound, sorting) and 7 behind it (sorting, sums, the cluster, logarithms in 64
// bits, ranking), in short dependent steps that all CTAs go through at the same time.
// Sums: every thread has its own reference (the largest logit it met when it last moved).  Partial sums are fp32, a round's vectors by themselves and then the rounds: among
// few different logits the roundings of equal terms all go one way, and 131072 of them one by one put a score off by 9 half units of its last place, in two steps by one.  The
// row's logarithm and all scores are formed in 64 bits, so that scores of different beams are compared before anything is rounded.  Scores are rounded to fp32 once.
#include "common.cuh"
#include "serve.cuh"
#include "tc_ptx.cuh"
#include <cuda_fp16.h>
#include <float.h>
#include <type_traits>

namespace zq {
namespace {

constexpr int kMaxThreads = 512, kCluster = 8;       // threads of a CTA, CTAs of a cluster at most
constexpr int kMaxEos = kMaxBeamEos, kMaxBest = kMaxBeams + kMaxEos;       // best logits of a row
constexpr int kBuffer = 2048, kMaxCandidates = kMaxBeams * kMaxBest;       // (a row in several slices: at most 8 rows' worth)
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.69314718055994530942;
static_assert(kMaxBeams * (1 + kMaxEos) <= 256, "the best of a request");

typedef unsigned long long u64;

__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
__device__ __forceinline__ u64 ordered64(double x) {
    const u64 b = (u64)__double_as_longlong(x);
    return b >> 63 ? ~b : b | (1ull << 63);
}
// Never 0 for a logit that may be chosen: NaN and -inf have no key, +inf counts as the largest finite value; both zeros are the same.
__device__ __forceinline__ u64 key_of(float x, int token) {
    return x > -INFINITY ? (u64)ordered(fminf(x, FLT_MAX) + 0.0f) << 32 | (uint32_t)~token : 0ull;
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ u64 ld_cluster_u64(uint32_t addr) {
    u64 v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
    return v;
}

template <typename T> __device__ __forceinline__ float value(T v) { return static_cast<float>(v); }
// VEC logits at a time: 16 bytes where the rows allow it, else single ones
template <typename T, int VEC> struct alignas(VEC * sizeof(T)) Vec { T v[VEC]; };
// CTAs of an SM (64 x 8 rows of 50272 bf16: with three CTAs, which spares the compiler a few words of stack, half of the rows wait for the others, 31.0 us against 26.9)
template <int THREADS> constexpr int kResident = THREADS == 512 ? 2 : 4;
// the largest; NaN does not count
template <typename T, int VEC> __device__ __forceinline__ float largest(const Vec<T, VEC>& x) {
    if constexpr (VEC == 1) return value(x.v[0]);
    else if constexpr (sizeof(T) == 4) return fmaxf(fmaxf(x.v[0], x.v[1]), fmaxf(x.v[2], x.v[3]));
    else {
        typedef typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type T2;
        const T2* y = reinterpret_cast<const T2*>(x.v);
        const T2 m = __hmax2(__hmax2(y[0], y[1]), __hmax2(y[2], y[3]));
        return fmaxf(value(m.x), value(m.y));
    }
}
// sum += 2^(x log2 e - ref2), over pairs
template <typename T, int VEC> __device__ __forceinline__ void add_powers(const Vec<T, VEC>& x, float ref2, float2& sum) {
    if constexpr (VEC == 1) {
        sum.x += ex2(fmaf(value(x.v[0]), kLog2e, -ref2));
    } else {
        const float2 scale = make_float2(kLog2e, kLog2e), minus = make_float2(-ref2, -ref2);
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
            float2 y = tree_fma2(make_float2(value(x.v[e]), value(x.v[e + 1])), scale, minus);
            y.x = ex2(y.x);
            y.y = ex2(y.y);
            sum = tree_add2(sum, y);
        }
    }
}

struct Params {
    BeamSelectArgs a;
    int in_parallel, slices, slice;          // rows of a request at a time, CTAs of a row, tokens of a slice (a multiple of a vector)
    int best;                                // best logits wanted of a row
};

struct Shared {
    u64 buf[kBuffer];
    u64 best[kMaxCandidates];                // a row's best keys in order, row after row of this CTA; 0: none
    u64 stat[kMaxBeams];                     // (reference, sum) of a row's slice as two floats
    double lse[kMaxBeams];
    float ref[kMaxThreads / 32], sum[kMaxThreads / 32], score[kMaxBeams];
    uint32_t bound[kMaxThreads / 32];
    int top[kMaxBeams * (1 + kMaxEos)];
    int hist[256];
    int count, eos[kMaxEos];
    u64 prefix;
    int want;
};

// Sorts the n best of m keys (m <= kBuffer) into `to`; 0 behind them.  Four lanes to a key: each counts a quarter of the larger ones.  Starts behind a barrier,
// ends with one.
template <int kThreads>
__device__ __forceinline__ void sort_best(const u64* buf, int m, u64* to, int n) {
    for (int i = threadIdx.x; i < n; i += kThreads)
        if (i >= m) to[i] = 0;
    for (int i0 = 0; i0 < m; i0 += kThreads / 4) {
        const int i = i0 + threadIdx.x / 4;
        const u64 key = i < m ? buf[i] : 0ull;
        int rank = 0;
        if (i < m)
            for (int j = threadIdx.x & 3; j < m; j += 4) rank += buf[j] > key;
        rank += __shfl_xor_sync(0xffffffffu, rank, 1);
        rank += __shfl_xor_sync(0xffffffffu, rank, 2);
        if (i < m && rank < n && (threadIdx.x & 3) == 0) to[rank] = key;
    }
    __syncthreads();
}

// The logits of a thread's vectors that are above the limit (EQUAL: or at it) go to the buffer; x[0] begins with `token`, x[1] stride further on.  Rare, so it is short: the vector
// is picked out first, whichever it is (comparisons and pushes of every element of every vector: the same logits 45.7 us in place of 31.0, most of it the code's own way
// through the instruction caches).
template <bool EQUAL, typename T, int VEC, int N>
__device__ __forceinline__ void push(Shared& sh, const Vec<T, VEC> (&x)[N], float limit, int token, int stride) {
    unsigned hit = 0;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const float v = largest(x[u]);
        hit |= (EQUAL ? v >= limit : v > limit) ? 1u << u : 0u;
    }
#pragma unroll 1
    for (; hit; hit &= hit - 1) {
        const int u = __ffs(hit) - 1;
        Vec<T, VEC> y = x[0];
#pragma unroll
        for (int k = 1; k < N; ++k)
            if (u == k) y = x[k];
        unsigned which = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float v = value(y.v[e]);
            which |= (EQUAL ? v >= limit : v > limit) ? 1u << e : 0u;
        }
        int at = atomicAdd(&sh.count, __popc(which));
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if (!((which >> e) & 1u)) continue;
            if (at < kBuffer) sh.buf[at] = key_of(value(y.v[e]), token + u * stride + e);
            ++at;
        }
    }
}

// Asks for the 64 KB behind a row's first two rounds, so that the memory is busy while the bound is found.
template <typename T, int VEC>
__device__ __forceinline__ void prefetch_row(const T* src, int size, int from) {
    constexpr int kBytes = 4096;
    const int64_t at = (int64_t)from * sizeof(T) + (int64_t)threadIdx.x * kBytes, end = (int64_t)size * sizeof(T) / 16 * 16;
    if (VEC > 1 && threadIdx.x < 65536 / kBytes && at < end)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(reinterpret_cast<const char*>(src) + at), "r"((int)(end - at < kBytes ? end - at : kBytes)) : "memory");
}

template <typename T, int VEC, int kThreads>
__global__ void __launch_bounds__(kThreads, kResident<kThreads>)
beam_select_kernel(const __grid_constant__ Params p) {
    constexpr int kWarps = kThreads / 32, kFly = VEC == 1 ? 8 : 4, kRound = kFly * kThreads;       // vectors of a thread in flight, vectors of a round
    __shared__ Shared sh;
    const BeamSelectArgs& a = p.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_ctarank(), request = blockIdx.x / (p.in_parallel * p.slices);
    const int n = p.best, lo = (rank % p.slices) * p.slice, size = max(0, min(a.vocab, lo + p.slice) - lo);
    const int n_vec = (size + VEC - 1) / VEC, n_whole = size / VEC;
    if (tid < a.n_eos) sh.eos[tid] = __ldg(a.eos + tid);
    if (rank == 0 && tid < a.beams) sh.score[tid] = __ldg(a.score + (int64_t)request * a.beams + tid);

    auto row_of = [&](int row) { return static_cast<const T*>(a.logits) + ((int64_t)request * a.beams + row) * a.ld + lo; };
    typedef Vec<T, VEC> V;
    auto fetch = [&](V (&x)[kFly], const T* src, int base) {     // vectors base + u * kThreads + tid; -inf behind the slice
        const V* at = reinterpret_cast<const V*>(src) + base + tid;
        if (base + kRound <= n_whole) {
#pragma unroll
            for (int u = 0; u < kFly; ++u) x[u] = at[u * kThreads];
            return;
        }
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const int i = base + u * kThreads + tid;
            if (i < n_whole) { x[u] = at[u * kThreads]; continue; }
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[u].v[e] = i * VEC + e < size ? src[i * VEC + e] : T(-INFINITY);
        }
    };
    V now[kFly], ahead[kFly];
    int mine = 0;                                                // rows of this CTA so far
    if (rank / p.slices < a.beams) {
        fetch(now, row_of(rank / p.slices), 0);
        prefetch_row<T, VEC>(row_of(rank / p.slices), size, 2 * kRound * VEC);
    }
    for (int row = rank / p.slices; row < a.beams; row += p.in_parallel, ++mine) {
        const T* src = row_of(row);
        u64* const best = sh.best + mine * n;
        __syncthreads();                                         // the row before is through with the shared words
        if (tid == 0) sh.count = 0;

        // the first round: bound and reference.  Full warps take part; each offers its `each`-th largest thread
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < kFly; ++u) top = fmaxf(top, largest(now[u]));
        if (kRound < n_vec) fetch(ahead, src, kRound);
        const int full = min(kWarps, n_vec >> 5), each = full ? (n + full - 1) / full : 33;
        uint32_t k = ordered(top), offer = 0, high = 0;
        for (int i = 0; i < each && i < 4; ++i) {
            offer = __reduce_max_sync(0xffffffffu, k);
            if (i == 0) high = offer;
            const uint32_t who = __ballot_sync(0xffffffffu, k == offer);
            if (lane == __ffs(who) - 1) k = 0;
        }
        if (lane == 0) { sh.bound[warp] = offer; sh.ref[warp] = unordered(high); }
        __syncthreads();
        uint32_t bound = 0xFFFFFFFFu;
        float ref = -1e30f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < full) bound = min(bound, sh.bound[w]);
            ref = fmaxf(ref, sh.ref[w]);
        }
        ref = fminf(ref, FLT_MAX);
        float limit = each > 4 ? -INFINITY : unordered(bound);
        if (!(limit > -INFINITY)) limit = -FLT_MAX;              // everything but -inf
        float ref2 = __fmul_rn(ref, kLog2e);
        float2 sum = make_float2(0.0f, 0.0f);
        push<true>(sh, now, limit, lo + tid * VEC, kThreads * VEC);
#pragma unroll
        for (int u = 0; u < kFly; ++u) add_powers(now[u], ref2, sum);
        __syncthreads();
        // the rest: what passes the n-th best so far (a later token loses against an equal logit)
        if (n_vec > kRound && sh.count <= kBuffer) {
            auto tighten = [&]() {
                const int m = sh.count;
                sort_best<kThreads>(sh.buf, m, best, n);
                const u64 nth = best[n - 1];
                limit = nth ? unordered((uint32_t)(nth >> 32)) : -INFINITY;
                for (int i = tid; i < n; i += kThreads) sh.buf[i] = best[i];
                if (tid == 0) sh.count = min(m, n);
                __syncthreads();
            };
            tighten();
            auto work = [&](const V (&x)[kFly], int base) {
                float m4 = largest(x[0]);
#pragma unroll
                for (int u = 1; u < kFly; ++u) m4 = fmaxf(m4, largest(x[u]));
                if (m4 > limit) {
                    push<false>(sh, x, limit, lo + (base + tid) * VEC, kThreads * VEC);
                    if (m4 > ref) {                              // the reference moves.  (Logits below the limit may pass it too, once other threads' logits have raised
                                                                 // the limit: should the sum run over then, the careful pass behind the stream mends it)
                        ref = fminf(m4, FLT_MAX);
                        const float to = __fmul_rn(ref, kLog2e), f = ex2(ref2 - to);
                        sum.x *= f;
                        sum.y *= f;
                        ref2 = to;
                    }
                }
                float2 part = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int u = 0; u < kFly; ++u) add_powers(x[u], ref2, part);
                sum = tree_add2(sum, part);
            };
            for (int base = kRound; base < n_vec; base += 2 * kRound) {
                if (base + kRound < n_vec) fetch(now, src, base + kRound);
                work(ahead, base);
                if (base + kRound >= n_vec) break;
                if (base + 2 * kRound < n_vec) fetch(ahead, src, base + 2 * kRound);
                work(now, base + kRound);
                // once more where most of the row is still to come (a bound from a k-th of it lets n (k - 1) of the rest pass)
                if (base == kRound && n_vec > 8 * kRound) {
                    __syncthreads();
                    if (sh.count <= kBuffer) tighten();
                }
            }
            __syncthreads();
        }
        if (row + p.in_parallel < a.beams) {
            fetch(now, row_of(row + p.in_parallel), 0);
            prefetch_row<T, VEC>(row_of(row + p.in_parallel), size, kRound * VEC);
        }
        auto each_key = [&](auto f) {                            // every key of the slice again
            for (int i = tid; i < size; i += kThreads) {
                const u64 key = key_of(value(src[i]), lo + i);
                if (key) f(key);
            }
        };
        const bool again = sh.count > kBuffer;
        if (again) {
            // too many passed: the n-th largest key, digit by digit
            u64 prefix = 0;
            int want = n;
            for (int shift = 56; shift >= 0; shift -= 8) {
                __syncthreads();
                for (int i = tid; i < 256; i += kThreads) sh.hist[i] = 0;
                __syncthreads();
                each_key([&](u64 key) {
                    if (shift == 56 || key >> (shift + 8) == prefix) atomicAdd(&sh.hist[(int)(key >> shift) & 255], 1);
                });
                __syncthreads();
                if (tid == 0) {
                    int d = 255, left = want;
                    for (; d > 0 && sh.hist[d] < left; --d) left -= sh.hist[d];
                    sh.prefix = prefix << 8 | (u64)d;
                    sh.want = left;
                }
                __syncthreads();
                prefix = sh.prefix;
                want = sh.want;
            }
            if (tid == 0) sh.count = 0;
            __syncthreads();
            each_key([&](u64 key) { if (key >= prefix) sh.buf[atomicAdd(&sh.count, 1)] = key; });      // (n of them)
            __syncthreads();
        }
        // the row's sum, relative to 2^(fl(reference * log2 e))
        float x[2] = {ref, sum.x + sum.y};
        auto join = [&](float om, float os) {
            const float t = fmaxf(x[0], om), t2 = __fmul_rn(t, kLog2e);
            x[1] = x[1] * ex2(__fmul_rn(x[0], kLog2e) - t2) + os * ex2(__fmul_rn(om, kLog2e) - t2);
            x[0] = t;
        };
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) join(__shfl_xor_sync(0xffffffffu, x[0], o), __shfl_xor_sync(0xffffffffu, x[1], o));
        if (lane == 0) { sh.ref[warp] = x[0]; sh.sum[warp] = x[1]; }
        sort_best<kThreads>(sh.buf, sh.count, best, n);
        x[0] = sh.ref[0]; x[1] = sh.sum[0];
        for (int w = 1; w < kWarps; ++w) join(sh.ref[w], sh.sum[w]);
        // Once more, with care: where the stream was left out above, NaN and +inf, logits near either end of the range.  Relative to
        // the largest logit itself, which a negative sign says.
        if (again || !(x[1] > 0.0f && x[1] < INFINITY && x[0] < 1e37f)) {
            __syncthreads();
            const u64 first = best[0];
            x[0] = first ? unordered((uint32_t)(first >> 32)) : 0.0f;
            x[1] = 0.0f;
            for (int i0 = tid; first && i0 < size; i0 += 32 * kThreads) {
                float part = 0.0f;
                for (int i = i0; i < size && i < i0 + 32 * kThreads; i += kThreads) {
                    const float v = value(src[i]);
                    if (v > -INFINITY) part += ex2((fminf(v, FLT_MAX) - x[0]) * kLog2e);
                }
                x[1] += part;
            }
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) x[1] += __shfl_xor_sync(0xffffffffu, x[1], o);
            if (lane == 0) sh.sum[warp] = x[1];
            __syncthreads();
            x[1] = 0.0f;
            for (int w = 0; w < kWarps; ++w) x[1] -= sh.sum[w];
        }
        if (tid == 0) sh.stat[mine] = (u64)__float_as_uint(x[1]) << 32 | __float_as_uint(x[0]);
    }

    // the request: rank 0 gathers keys and sums, the other CTAs stay until they have been read
    __syncthreads();
    cluster_sync_all();
    const int per_row = p.slices * n, total = a.beams * per_row;
    u64* const keys = sh.buf;
    static_assert(kMaxCandidates <= kBuffer && kCluster * (kCluster + kMaxEos) <= kMaxCandidates, "the candidates of a request fit");
    if (rank == 0) {
        for (int i = tid; i < total; i += kThreads) {
            const int row = i / per_row, rest = i - row * per_row, s = rest / n;
            keys[i] = ld_cluster_u64(mapa_shared(smem_u32(sh.best + row / p.in_parallel * n + rest - s * n), (row % p.in_parallel) * p.slices + s));
        }
        if (tid < a.beams) {
            double top = -INFINITY, sum = 0.0;
            u64 w[kCluster];
            for (int s = 0; s < p.slices; ++s) w[s] = ld_cluster_u64(mapa_shared(smem_u32(sh.stat + tid / p.in_parallel), (tid % p.in_parallel) * p.slices + s));
            for (int pass = 0; pass < 2; ++pass)
                for (int s = 0; s < p.slices; ++s) {
                    const float r = __uint_as_float((uint32_t)w[s]), v = __uint_as_float((uint32_t)(w[s] >> 32));
                    if (v == 0.0f) continue;
                    // what the rounding of reference * log2 e moved is put back here
                    const double at = v < 0.0f ? (double)r : (double)r + kLn2 * ((double)__fmul_rn(r, kLog2e) - (double)r * (double)kLog2e);
                    if (pass == 0) top = fmax(top, at);
                    else sum += fabs((double)v) * (p.slices > 1 ? exp(at - top) : 1.0);
                }
            sh.lse[tid] = sum > 0.0 ? top + log(sum) : INFINITY;
        }
    }
    cluster_sync_all();
    if (rank != 0) return;
    auto score_of = [&](int i) {
        const int row = i / per_row;
        return (double)sh.score[row] + ((double)unordered((uint32_t)(keys[i] >> 32)) - sh.lse[row]);
    };
    u64* const order = sh.best;                                  // (all have read their keys)
    for (int i = tid; i < total; i += kThreads) {
        const double sc = keys[i] ? score_of(i) : -INFINITY;
        order[i] = sc > -INFINITY ? ordered64(sc) : 0ull;
    }
    const int most = a.beams * (1 + a.n_eos);
    for (int i = tid; i < most; i += kThreads) sh.top[i] = -1;
    __syncthreads();
    for (int i = tid; i < total; i += kThreads) {
        const u64 key = order[i];
        if (!key) continue;
        int r = 0;
        if (p.slices == 1) {
            for (int j = 0; j < total; ++j) r += order[j] > key || (order[j] == key && j < i);
        } else {
            // a row's slices stand one after the other, each in its own order: of equal scores of a row the larger key comes first.  Without branches (with them, and for all
            // rows: 4 us more for 4 x 32000 and for 64 x 8 x 50272 alike)
            const int row0 = i / per_row * per_row;
            const u64 mine = keys[i];
            for (int j = 0; j < total; ++j) {
                const u64 other = order[j], its = keys[j];
                const bool before = (unsigned)(j - row0) < (unsigned)per_row ? its > mine : j < i;
                r += (int)(other > key) | ((int)(other == key) & (int)before);
            }
        }
        if (r < most) sh.top[r] = i;
    }
    __syncthreads();
    // those that go on, those that are finished: each counts the ones of its kind before it
    int* kind = sh.hist;                                         // 0 none, 1 goes on, 2 finished
    for (int r = tid; r < most; r += kThreads) {
        int is = 0;
        if (sh.top[r] >= 0) {
            const int token = (int)~(uint32_t)keys[sh.top[r]];
            is = 1;
            for (int e = 0; e < a.n_eos; ++e)
                if (sh.eos[e] == token) is = 2;
            if (is == 2 && r >= a.beams) is = 0;
        }
        kind[r] = is;
    }
    __syncthreads();
    const int64_t out = (int64_t)request * a.beams;
    for (int r = tid; r < most; r += kThreads) {
        const int is = kind[r];
        int at = 0, on = 0, done = 0;
        for (int j = 0; j < most; ++j) {
            at += j < r && kind[j] == is;
            on += kind[j] == 1;
            done += kind[j] == 2;
        }
        if (r < a.beams) {                                       // slots that stay empty
            if (r >= on) { a.beam[out + r] = -1; a.token[out + r] = -1; a.score_out[out + r] = -INFINITY; }
            if (r >= done) { a.done_beam[out + r] = -1; a.done_token[out + r] = -1; a.done_score[out + r] = -INFINITY; }
        }
        if (is == 0 || at >= a.beams) continue;
        const int i = sh.top[r];
        (is == 1 ? a.beam : a.done_beam)[out + at] = i / per_row;
        (is == 1 ? a.token : a.done_token)[out + at] = (int)~(uint32_t)keys[i];
        (is == 1 ? a.score_out : a.done_score)[out + at] = (float)score_of(i);
    }
}

template <typename T, int VEC, int THREADS>
int launch_threads(const Params& p, cudaStream_t s) {
    const int ranks = p.in_parallel * p.slices;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.a.batch * ranks);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ranks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, beam_select_kernel<T, VEC, THREADS>, p) != cudaSuccess) return -1;
    count_launch();
    return 0;
}

template <typename T, int VEC>
int launch_vec(const BeamSelectArgs& a, cudaStream_t s) {
    Params p{a, 0, 0, 0, 0};
    // Whole rows in parallel, as many as keep all CTAs resident (with more, clusters wait for one another); slices only while the SMs have
    // less than two CTAs, and of two thousand tokens at least.
    int rounds = (a.beams + kCluster - 1) / kCluster;
    for (p.in_parallel = (a.beams + rounds - 1) / rounds; p.in_parallel > 1 && (int64_t)a.batch * p.in_parallel > 148 * kResident<256>; p.in_parallel = (a.beams + rounds - 1) / rounds) ++rounds;
    p.slices = 1;
    while ((p.slices + 1) * p.in_parallel <= kCluster && (int64_t)a.batch * p.in_parallel * (p.slices + 1) <= 148 * 2 && a.vocab >= 2048 * (p.slices + 1)) ++p.slices;
    p.slice = ((a.vocab + p.slices - 1) / p.slices + VEC - 1) / VEC * VEC;
    p.best = a.beams + a.n_eos < a.vocab ? a.beams + a.n_eos : a.vocab;
    // few CTAs: wide ones (two to an SM leave no room for clusters to be placed)
    return (int64_t)a.batch * p.in_parallel * p.slices <= 148 ? launch_threads<T, VEC, 512>(p, s) : launch_threads<T, VEC, 256>(p, s);
}

template <typename T>
int launch_type(const BeamSelectArgs& a, cudaStream_t s) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(a.logits) | (uintptr_t)(a.ld * sizeof(T));
    return at % 16 == 0 ? launch_vec<T, 16 / sizeof(T)>(a, s) : launch_vec<T, 1>(a, s);
}

}  // namespace

int launch_beam_select(const BeamSelectArgs& a, cudaStream_t s) {
    if (a.type == kTypeF32) return launch_type<float>(a, s);
    if (a.type == kTypeBf16) return launch_type<__nv_bfloat16>(a, s);
    return launch_type<__half>(a, s);
}

}  // namespace zq
