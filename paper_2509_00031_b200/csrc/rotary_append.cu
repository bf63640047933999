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
// halves are paired, two neighbouring chunks elsewhere.  A head is 4 or 8 lanes, its mean square two or three shuffles.  A CTA takes so many rows that every
// thread has its loads of two (fp32) or four items on their way before it waits for anything.
#include "common.cuh"
#include "serve.cuh"
#include "vec8.cuh"

namespace zq {
namespace {

constexpr int kThreads = 256, kMaxRows = 16;
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
    int block_rows, row_items, span;         // rows of a CTA, items of a row, items of a CTA
};

template <typename S, typename T, int DH, bool INTER>
__global__ void __launch_bounds__(kThreads)
rotary_append_kernel(const Params p) {
    constexpr int kLanes = DH / 16, kFly = sizeof(S) == 4 ? 2 : 4;
    extern __shared__ __align__(16) float2 turn[];               // [block_rows][rot / 2] (cos, sin)
    __shared__ int slot_s[kMaxRows], pos_s[kMaxRows];
    const int tid = threadIdx.x, row0 = blockIdx.x * p.block_rows, n_rows = min(p.block_rows, p.rows - row0);
    const int first = blockIdx.y * p.span, end = min(n_rows * p.row_items, first + p.span);
    const int n_kv = p.cache.n_kv_heads, half = p.rot >> 1, chunks = INTER ? 0 : p.rot >> 4;
    struct Item { int row, head, a, b; bool live, turned; };
    auto place = [&](int it) {
        Item x;
        x.live = it < end;
        const int row = p.block_rows == 1 ? 0 : it / p.row_items, rest = it - row * p.row_items, l = rest % kLanes;
        x.row = row;
        x.head = rest / kLanes;
        if (INTER) { x.a = 2 * l; x.b = x.a + 1; x.turned = 16 * l < p.rot; }
        else if (l < chunks) { x.a = l; x.b = l + chunks; x.turned = true; }
        else { x.a = 2 * l; x.b = x.a + 1; x.turned = false; }   // (2 chunks + 2 (l - chunks))
        x.turned = x.turned && x.head < p.n_heads + n_kv;
        return x;
    };
    if (tid < n_rows) {
        slot_s[tid] = __ldg(p.slot + row0 + tid);
        pos_s[tid] = p.rot ? __ldg(p.row_pos + row0 + tid) : 0;
    }
    bool ready = false;
    for (int base = first; base < end; base += kFly * kThreads) {
        Raw8<S> ra[kFly], rb[kFly];
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const Item x = place(base + u * kThreads + tid);
            if (!x.live) continue;
            const S* src = static_cast<const S*>(p.qkv) + (int64_t)(row0 + x.row) * p.ld + (int64_t)x.head * DH;
            ra[u].load(src + 8 * x.a);
            rb[u].load(src + 8 * x.b);
        }
        if (!ready) {
            ready = true;
            __syncthreads();
            for (int i = tid; i < n_rows * half; i += kThreads) {
                const int row = i / half;
                const double turns = (double)pos_s[row] * (__ldg(p.freq + i - row * half) * kInvTwoPi);
                float s, c;
                sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
                turn[i] = make_float2(p.magnitude * c, p.magnitude * s);
            }
            if (tid < n_rows && blockIdx.y == 0 && slot_s[tid] >= 0 && (slot_s[tid] >= p.cache.n_pages * p.cache.page_size || pos_s[tid] < 0))
                atomicExch(p.err_flag, kErrBadSlot);
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const Item x = place(base + u * kThreads + tid);
            float a[8] = {}, b[8] = {};
            if (x.live) { ra[u].widen(a); rb[u].widen(b); }
            const float* gain = x.head < p.n_heads ? p.q_gain : (x.head < p.n_heads + n_kv ? p.k_gain : nullptr);
            if (p.q_gain || p.k_gain) {                          // the same for all threads: lanes meet below
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(a[e], a[e], fmaf(b[e], b[e], sum));
#pragma unroll
                for (int o = 1; o < kLanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (gain) {
                    const float r = 1.0f / sqrtf(sum * (1.0f / DH) + p.eps);
                    float ga[8], gb[8];
                    Raw8<float> g;
                    g.load(gain + 8 * x.a); g.widen(ga);
                    g.load(gain + 8 * x.b); g.widen(gb);
#pragma unroll
                    for (int e = 0; e < 8; ++e) { a[e] = a[e] * r * ga[e]; b[e] = b[e] * r * gb[e]; }
                }
            }
            if (!x.live) continue;
            const int sl = slot_s[x.row];
            if (sl < 0 || sl >= p.cache.n_pages * p.cache.page_size || pos_s[x.row] < 0) continue;      // skipped whole
            if (x.turned) {
                // pairs 8 l .. 8 l + 7 of the row
                const float4* cs = reinterpret_cast<const float4*>(turn + x.row * half + 8 * (INTER ? x.a >> 1 : x.a));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float4 t = cs[e];                      // cos, sin of two pairs
                    if (INTER) {
                        float (&v)[8] = e < 2 ? a : b;
                        const int i = 4 * (e & 1);
                        const float w0 = v[i], w1 = v[i + 1], w2 = v[i + 2], w3 = v[i + 3];
                        v[i] = w0 * t.x - w1 * t.y; v[i + 1] = w1 * t.x + w0 * t.y;
                        v[i + 2] = w2 * t.z - w3 * t.w; v[i + 3] = w3 * t.z + w2 * t.w;
                    } else {
                        const float a0 = a[2 * e], b0 = b[2 * e], a1 = a[2 * e + 1], b1 = b[2 * e + 1];
                        a[2 * e] = a0 * t.x - b0 * t.y; b[2 * e] = b0 * t.x + a0 * t.y;
                        a[2 * e + 1] = a1 * t.z - b1 * t.w; b[2 * e + 1] = b1 * t.z + a1 * t.w;
                    }
                }
            }
            T* dst;
            if (x.head < p.n_heads) {
                dst = static_cast<T*>(p.q_out) + (int64_t)(row0 + x.row) * p.q_stride + (int64_t)x.head * DH;
            } else {
                const bool is_k = x.head < p.n_heads + n_kv;
                const int kvh = x.head - p.n_heads - (is_k ? 0 : n_kv), page = sl / p.cache.page_size, off = sl - page * p.cache.page_size;
                dst = static_cast<T*>(is_k ? p.cache.k : p.cache.v) + page * p.cache.page_stride + off * p.cache.slot_stride + kvh * p.cache.head_stride;
            }
            Pack8<T>::store(dst + 8 * x.a, a);
            Pack8<T>::store(dst + 8 * x.b, b);
        }
    }
}

template <typename S, typename T>
cudaError_t launch(const Params& p, int dh, bool inter, dim3 grid, cudaStream_t s) {
    const size_t smem = (size_t)p.block_rows * (p.rot / 2) * sizeof(float2);
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
    Params p{a.qkv, a.ld, a.row_pos, a.slot, a.rows, a.n_heads, a.freq, a.rot, a.magnitude, a.q_gain, a.k_gain, a.eps, a.cache, a.q_out, a.q_stride, a.err_flag, 1, 0, 0};
    const int dh = a.cache.d_head, fly = (a.src_type == kTypeF32 ? 2 : 4) * kThreads;
    p.row_items = (a.n_heads + 2 * a.cache.n_kv_heads) * (dh / 16);
    dim3 grid(a.rows, 1);
    if ((int64_t)a.rows * p.row_items > (int64_t)148 * fly) {
        // enough for all SMs: a thread's loads of one go
        p.block_rows = fly / p.row_items < 1 ? 1 : (fly / p.row_items > kMaxRows ? kMaxRows : fly / p.row_items);
        grid.x = (a.rows + p.block_rows - 1) / p.block_rows;
        p.span = p.block_rows * p.row_items;
    } else {
        p.span = kThreads;                                       // few rows: a row over several CTAs
        grid.y = (p.row_items + p.span - 1) / p.span;
    }
    cudaError_t rc;
    if (a.src_type == kTypeF32) rc = launch_to<float>(p, dh, a.interleaved, grid, s);
    else if (a.src_type == kTypeBf16) rc = launch_to<__nv_bfloat16>(p, dh, a.interleaved, grid, s);
    else rc = launch_to<__half>(p, dh, a.interleaved, grid, s);
    if (rc != cudaSuccess) return -1;
    count_launch();
    return 0;
}

}  // namespace zq
