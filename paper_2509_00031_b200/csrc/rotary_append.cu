// Query and key heads on their way into the cache: norm of each head, rotation by the row's position, one rounding, in one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * gain                                  q and k heads (without gains: y = x)
//   (a, b) -> m (a cos t - b sin t, b cos t + a sin t),  t = pos * freq[i]    pair i of the first `rot` elements of a head: elements
//                                                                         (i, i + rot / 2), or (2 i, 2 i + 1) where they are interleaved
//   q -> q_out, k and v -> slot                                           of the cache's type
//
// Angles are formed from frequencies, not read from a table: a table for a million positions is half a gigabyte, and fp32 angles of
// such positions are off by 0.03.  t is reduced in 64 bits - the position times the frequency in turns, minus the nearest whole
// number - and only the rest, within half a turn, is rounded to fp32 for the sine and cosine; a row's are formed once and shared by its
// heads through shared memory.
// A thread owns 8 + 8 elements of a head, so that a pair never spans threads: chunks l and l + rot / 16 of the rotated part where the
// halves are paired, and else two that leave neighbouring lanes with neighbouring chunks.  A head is 4 or 8 lanes, its mean square two or three shuffles.  A thread keeps its row and its
// place within the head and walks over the heads, so sines, cosines and gains are read once and stay in registers (read again for every head, they were two thirds of
// what passed through L1: 8191 rows of 40 + 2 * 8 heads of 128, bf16 to binary16, 75 us against 53, where 36 are the bytes at the rate of a copy).  What is left is bound by instructions
// (half of the issue slots) and by waiting for the one head ahead: two ahead cost an SM a third of its CTAs (59 us).  At three CTAs an SM, 80 registers, the compiler spills 24 to 44 bytes a
// thread (28 to 72 loaded again); at four, 64 registers, 164 to 240 (70 us).
// Rounding: sums of squares are fp32, and rsqrtf is off by two units of its last place; fp32 results are off by 6e-8 relative to 64 bits (elementary operations one after the other: 4e-8).
#include "common.cuh"
#include "serve.cuh"
#include "tc_ptx.cuh"
#include "vec8.cuh"

namespace zq {
namespace {

constexpr int kThreads = 256, kMaxRows = 32;
constexpr double kInvTwoPi = 0.15915494309189533577;

struct Params {
    const void* qkv;
    int64_t ld;
    const int32_t *row_pos, *slot;
    int rows, n_heads;
    const double* freq;
    int rot;
    float magnitude;
    const float *q_gain, *k_gain;
    float eps;
    PagedCache cache;
    void* q_out;
    int64_t q_stride;
    int32_t* err_flag;
    int row_threads;                         // of a CTA for each of its rows: whole heads' lanes, a power of two
};

template <typename S, typename T, int DH, bool INTER>
__global__ void __launch_bounds__(kThreads, 3)
rotary_append_kernel(const Params p) {
    constexpr int kLanes = DH / 16, kFly = sizeof(S) == 4 ? 1 : 2;
    extern __shared__ __align__(16) float2 turn[];               // [rows of the CTA][rot / 2] (cos, sin)
    __shared__ int slot_s[kMaxRows], pos_s[kMaxRows];
    const int tid = threadIdx.x, cta_rows = kThreads / p.row_threads, row0 = blockIdx.x * cta_rows, n_rows = min(cta_rows, p.rows - row0);
    const int row = tid / p.row_threads, me = tid - row * p.row_threads, l = me % kLanes, step = p.row_threads / kLanes * gridDim.y;
    const int n_kv = p.cache.n_kv_heads, heads = p.n_heads + 2 * n_kv, half = p.rot >> 1, chunks = INTER ? 0 : p.rot >> 4;
    // this thread's chunks of every head
    const int ca = INTER || l < chunks ? l : chunks + l, cb = INTER ? l + kLanes : (l < chunks ? l + chunks : kLanes + l);
    const bool turn_a = 8 * ca < p.rot, turn_b = 8 * cb < p.rot; // (halves paired: both or none)
    const bool mine = row < n_rows;
    if (tid < n_rows) {
        slot_s[tid] = __ldg(p.slot + row0 + tid);
        pos_s[tid] = p.rot ? __ldg(p.row_pos + row0 + tid) : 0;
    }
    const S* src = static_cast<const S*>(p.qkv) + (int64_t)(row0 + (mine ? row : 0)) * p.ld;
    Raw8<S> ra[kFly], rb[kFly];
    int h0 = me / kLanes + blockIdx.y * (p.row_threads / kLanes);
    auto fetch = [&]() {
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const int h = h0 + u * step;
            if (!mine || h >= heads) continue;
            ra[u].load(src + h * DH + 8 * ca);
            rb[u].load(src + h * DH + 8 * cb);
        }
    };
    fetch();                                                     // on their way while the angles are formed
    __syncthreads();
    for (int i = tid; i < n_rows * half; i += kThreads) {
        const int r = i / half;
        const double turns = (double)pos_s[r] * (__ldg(p.freq + i - r * half) * kInvTwoPi);
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        turn[i] = make_float2(p.magnitude * c, p.magnitude * s);
    }
    __syncthreads();
    const int sl = mine ? slot_s[row] : -1;
    const bool outside = mine && sl >= 0 && (sl >= p.cache.n_pages * p.cache.page_size || pos_s[row] < 0);
    if (outside && me == 0 && blockIdx.y == 0) atomicExch(p.err_flag, kErrBadSlot);
    const bool live = mine && sl >= 0 && !outside;               // (else the row is skipped whole; its lanes go along)
    const int page = live ? sl / p.cache.page_size : 0, off = live ? sl - page * p.cache.page_size : 0;
    const int64_t place = page * p.cache.page_stride + off * p.cache.slot_stride;
    T* const q_row = static_cast<T*>(p.q_out) + (int64_t)(row0 + row) * p.q_stride;
    float cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {                                // pairs 8 l .. 8 l + 7 of the row; interleaved: four of chunk ca, four of cb
        const bool there = mine && (INTER && e >= 2 ? turn_b : turn_a);
        const float2* at = turn + row * half + (INTER ? 4 * (e < 2 ? ca : cb) + 2 * (e & 1) : 8 * l + 2 * e);
        const float4 t = there ? *reinterpret_cast<const float4*>(at) : make_float4(1.0f, 0.0f, 1.0f, 0.0f);
        cs[2 * e] = t.x; sn[2 * e] = t.y; cs[2 * e + 1] = t.z; sn[2 * e + 1] = t.w;
    }
    const bool norms = p.q_gain || p.k_gain;
    float2 gain[8];
    int gains = -1;                                              // whose gains these are: 0 q, 1 k
    for (; h0 - me / kLanes < heads; h0 += kFly * step) {        // (the same number of rounds for all lanes)
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const int h = h0 + u * step;
            float2 x[8] = {};                                    // a, then b
            if (mine && h < heads) { ra[u].widen(reinterpret_cast<float (&)[8]>(x[0])); rb[u].widen(reinterpret_cast<float (&)[8]>(x[4])); }
            if (norms) {
                float2 sum2 = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum2 = tree_fma2(x[e], x[e], sum2);
                float sum = sum2.x + sum2.y;
#pragma unroll
                for (int o = 1; o < kLanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const float* from = h < p.n_heads ? p.q_gain : (h < p.n_heads + n_kv ? p.k_gain : nullptr);
                if (from) {
                    if (gains != (h >= p.n_heads)) {
                        gains = h >= p.n_heads;
                        Raw8<float> g;
                        g.load(from + 8 * ca); g.widen(reinterpret_cast<float (&)[8]>(gain[0]));
                        g.load(from + 8 * cb); g.widen(reinterpret_cast<float (&)[8]>(gain[4]));
                    }
                    const float r = rsqrtf(sum * (1.0f / DH) + p.eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = tree_mul2(tree_mul2(x[e], make_float2(r, r)), gain[e]);
                }
            }
            if (!live || h >= heads) continue;
            if (turn_a && h < p.n_heads + n_kv) {                // (interleaved: the second chunk may lie behind the rotated part)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (INTER && e >= 4 && !turn_b) break;
                    float &v = INTER ? x[e].x : (e & 1 ? x[e >> 1].y : x[e >> 1].x), &w = INTER ? x[e].y : (e & 1 ? x[4 + (e >> 1)].y : x[4 + (e >> 1)].x);
                    const float v0 = v, w0 = w;
                    v = v0 * cs[e] - w0 * sn[e];
                    w = w0 * cs[e] + v0 * sn[e];
                }
            }
            T* dst;
            if (h < p.n_heads) dst = q_row + h * DH;
            else if (h < p.n_heads + n_kv) dst = static_cast<T*>(p.cache.k) + place + (h - p.n_heads) * p.cache.head_stride;
            else dst = static_cast<T*>(p.cache.v) + place + (h - p.n_heads - n_kv) * p.cache.head_stride;
            Pack8<T>::store(dst + 8 * ca, reinterpret_cast<const float (&)[8]>(x[0]));
            Pack8<T>::store(dst + 8 * cb, reinterpret_cast<const float (&)[8]>(x[4]));
        }
        if (h0 - me / kLanes + kFly * step < heads) {
            h0 += kFly * step;
            fetch();
            h0 -= kFly * step;
        }
    }
}

template <typename S, typename T>
cudaError_t launch(const Params& p, int dh, bool inter, dim3 grid, cudaStream_t s) {
    const size_t smem = (size_t)(kThreads / p.row_threads) * (p.rot / 2) * sizeof(float2);
    auto go = [&](void (*kernel)(Params)) { return launch_kernel(kernel, grid, dim3(kThreads), smem, s, false, p); };
    if (dh == 64) return inter ? go(rotary_append_kernel<S, T, 64, true>) : go(rotary_append_kernel<S, T, 64, false>);
    return inter ? go(rotary_append_kernel<S, T, 128, true>) : go(rotary_append_kernel<S, T, 128, false>);
}

template <typename S>
cudaError_t launch_to(const Params& p, int dh, bool inter, dim3 grid, cudaStream_t s) {
    if (p.cache.type == kTypeF32) return launch<S, float>(p, dh, inter, grid, s);
    if (p.cache.type == kTypeBf16) return launch<S, __nv_bfloat16>(p, dh, inter, grid, s);
    return launch<S, __half>(p, dh, inter, grid, s);
}

}  // namespace

int launch_rotary_append(const RotaryAppendArgs& a, cudaStream_t s) {
    Params p{a.qkv, a.ld, a.row_pos, a.slot, a.rows, a.n_heads, a.freq, a.rot, a.magnitude, a.q_gain, a.k_gain, a.eps, a.cache, a.q_out, a.q_stride, a.err_flag, kThreads};
    const int dh = a.cache.d_head, lanes = dh / 16, items = (a.n_heads + 2 * a.cache.n_kv_heads) * lanes, fly = a.src_type == kTypeF32 ? 1 : 2;
    dim3 grid(a.rows, 1);
    // Threads of a row: as few as get through its heads in four rounds, if that still fills the SMs (8191 rows of 56 heads of 128, rounds of 1 / 2 / 4 / 8 / 16: 65 / 57 /
    // 53 / 53 / 64 us: a CTA's angles are formed before its first round); a row over several CTAs where there are few rows.
    while (p.row_threads > lanes && p.row_threads > kThreads / kMaxRows && p.row_threads / 2 * fly * 4 >= items &&
           (int64_t)a.rows * (p.row_threads / 2) >= (int64_t)148 * kThreads)
        p.row_threads /= 2;
    grid.x = (a.rows + kThreads / p.row_threads - 1) / (kThreads / p.row_threads);
    if (p.row_threads == kThreads)
        while (grid.x * grid.y < 148 && (int)grid.y * kThreads < items) ++grid.y;
    cudaError_t rc;
    if (a.src_type == kTypeF32) rc = launch_to<float>(p, dh, a.interleaved, grid, s);
    else if (a.src_type == kTypeBf16) rc = launch_to<__nv_bfloat16>(p, dh, a.interleaved, grid, s);
    else rc = launch_to<__half>(p, dh, a.interleaved, grid, s);
    if (rc != cudaSuccess) return -1;
    count_launch();
    return 0;
}

}  // namespace zq
