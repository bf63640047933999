// Work distribution of the attention kernels over a paged cache, shared by the CUDA-core and the tensor-core kernel.
//
// For request b with n new rows and L keys (C = L - n of them cached before this step, the drafts last) and g = n_heads /
// n_kv_heads query heads per key head, the queries that read one key head are the n * g vectors (draft i, head in group) in
// this order, cut into row tiles.  An item is (request, key head, row tile), its work is the number of key
// tiles.  All items' key tiles, laid out one after the other, are cut into gridDim.x equal runs, one per CTA: long contexts
// are split over as many CTAs as it takes, short ones are packed, and no length is needed on the host.  Every CTA finds its
// run by scanning the requests' lengths.  A piece of an item that is not the whole item leaves (reference, sum, output) per
// query in the scratch, at most two pieces per CTA, and tree_combine_kernel joins them in the order of the keys, so results
// do not depend on timing.
#pragma once
#include "common.cuh"
#include "serve.cuh"
#include <cuda_fp16.h>

namespace zq {

struct TreeWork {
    const int32_t *kv_len, *row_start, *block_table;
    int batch, rows, n_heads, n_kv, max_pages, page_size;
    int group;               // query heads per key head
    int tile_rows;           // queries per row tile
    int key_tile;            // keys per key tile
    int32_t* err_flag;
};

struct TreeRequest { int n, L, row0, n_rt, n_kt; };      // n_rt * n_kt = 0: nothing to do

__device__ __forceinline__ TreeRequest tree_request(const TreeWork& w, int b) {
    TreeRequest r;
    r.row0 = __ldg(w.row_start + b);
    r.n = __ldg(w.row_start + b + 1) - r.row0;
    r.L = __ldg(w.kv_len + b);
    if (r.n <= 0 || r.row0 < 0 || r.n > r.L || r.row0 > w.rows - r.n || r.L > (long long)w.max_pages * w.page_size) {
        if (r.n != 0) atomicExch(w.err_flag, kErrBadRequest);
        r.n = r.n_rt = r.n_kt = 0;
        return r;
    }
    r.n_rt = (int)(((long long)r.n * w.group + w.tile_rows - 1) / w.tile_rows);
    r.n_kt = (r.L + w.key_tile - 1) / w.key_tile;
    return r;
}
__device__ __forceinline__ long long tree_tiles(const TreeWork& w, int b) {
    const TreeRequest r = tree_request(w, b);
    return (long long)w.n_kv * r.n_rt * r.n_kt;
}

// Position in the sequence of key tiles.  next() moves on by one tile; tiles of requests without work do not exist.
struct TreeCursor {
    TreeRequest r;
    int b, h, rt, kt;
    __device__ __forceinline__ void load(const TreeWork& w) { r = tree_request(w, b); }
    // first query of the row tile and how many it has
    __device__ __forceinline__ int first_query(const TreeWork& w) const { return rt * w.tile_rows; }
    __device__ __forceinline__ int queries(const TreeWork& w) const { return min(w.tile_rows, r.n * w.group - rt * w.tile_rows); }
    __device__ __forceinline__ bool item_begins() const { return kt == 0; }
    __device__ __forceinline__ bool item_ends() const { return kt == r.n_kt - 1; }
    __device__ __forceinline__ void next(const TreeWork& w) {
        if (++kt < r.n_kt) return;
        kt = 0;
        if (++rt < r.n_rt) return;
        rt = 0;
        if (++h < w.n_kv) return;
        h = 0;
        do { if (++b >= w.batch) return; load(w); } while (r.n_kt == 0);
    }
};

// a / b for a >= 0, b > 0; almost always in 32 bits, which is several times faster
__device__ __forceinline__ long long tree_div(long long a, long long b) {
    return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}

struct TreeRun { long long begin, end, total; int ctas; TreeCursor at; };   // ctas: CTAs that have a run

// Run c of `total` tiles in `ctas` runs begins here: the first total % ctas runs have one tile more than the others.
__device__ __forceinline__ long long tree_run_begin(long long total, int ctas, int c) {
    const long long q = tree_div(total, ctas), r = total - q * ctas;
    return q * c + (c < r ? c : r);
}
// The CTA whose run holds tile `x`.
__device__ __forceinline__ int tree_cta_of(long long x, long long total, int ctas) {
    const long long q = tree_div(total, ctas), r = total - q * ctas, wide = r * (q + 1);
    return (int)(x < wide ? tree_div(x, q + 1) : r + tree_div(x - wide, q));
}

// The run of this CTA; called by all threads of the block (part: one word per warp, out: shared).  Ends with a barrier.
__device__ __forceinline__ void tree_find_run(const TreeWork& w, long long* part, TreeRun* out) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const int per = (w.batch + blockDim.x - 1) / blockDim.x;
    const int b0 = min(tid * per, w.batch), b1 = min(b0 + per, w.batch);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) mine += tree_tiles(w, b);
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += u;
    }
    if (lane == 31) part[warp] = upto;
    __syncthreads();
    long long total = 0;
    for (int k = 0; k < warps; ++k) {
        if (k == warp) upto += total;
        total += part[k];
    }
    // the runs are those of the CTAs or, where there are fewer tiles, of as many CTAs as there are tiles: none is empty
    const int ctas = total < (long long)gridDim.x ? (int)total : (int)gridDim.x;
    const bool idle = (int)blockIdx.x >= ctas;
    const long long begin = idle ? 0 : tree_run_begin(total, ctas, blockIdx.x), end = idle ? 0 : tree_run_begin(total, ctas, blockIdx.x + 1);
    if (tid == 0) { out->begin = begin; out->end = end; out->total = total; out->ctas = ctas; }
    if (begin < end && begin >= upto - mine && begin < upto) {       // exactly one thread
        long long rest = begin - (upto - mine);
        TreeCursor c;
        for (c.b = b0; c.b < b1; ++c.b) {
            c.load(w);
            const long long t = (long long)w.n_kv * c.r.n_rt * c.r.n_kt;
            if (rest < t) break;
            rest -= t;
        }
        const long long item = tree_div(rest, c.r.n_kt), head = tree_div(item, c.r.n_rt);
        c.kt = (int)(rest - item * c.r.n_kt);
        c.rt = (int)(item - head * c.r.n_rt);
        c.h = (int)head;
        out->at = c;
    }
    __syncthreads();
}

// ---- partial results ------------------------------------------------------------------------------------------------
// One descriptor per CTA, then 2 * G slots of [tile_rows] references, [tile_rows] sums and [tile_rows][d_head] outputs (fp32).
struct TreeTail { int last_cta, queries, row0, q0, h, pad[3]; };   // an item that begins in this CTA and ends in last_cta; -1: none
constexpr size_t kTailBytes = 8192;                      // room for the descriptors
constexpr int kMaxTreeGrid = 148;                        // one CTA per SM

__host__ __device__ inline size_t tree_slot_floats(int tile_rows, int dh) { return (size_t)tile_rows * (dh + 2); }

__device__ __forceinline__ float* tree_slot(uint8_t* scratch, int index, int tile_rows, int dh) {
    return reinterpret_cast<float*>(scratch + kTailBytes) + (size_t)index * tree_slot_floats(tile_rows, dh);
}

__device__ __forceinline__ float tree_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <typename T> __device__ __forceinline__ T tree_round(float v);
template <> __device__ __forceinline__ float tree_round<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 tree_round<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half tree_round<__half>(float v) { return __float2half_rn(v); }

// Joins the pieces of split items: block (c, y) takes the item that begins in CTA c, queries y, y + gridDim.y, ...
// out = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p over its pieces p in key order per warp, the 8 warps' shares then in
// warp order; a query that saw no key gives zeros.  All of it in binary32, one rounding at the end.
template <typename T, int DH>
__global__ void __launch_bounds__(256)
tree_combine_kernel(uint8_t* scratch, int tile_rows, int group, int n_heads, T* out, int64_t out_stride) {
    constexpr int VPL = DH / 32;
    __shared__ float acc_s[8][DH], m_s[8], l_s[8];
    grid_dependency_wait();
    const TreeTail tail = reinterpret_cast<const TreeTail*>(scratch)[blockIdx.x];
    if (tail.last_cta < 0) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = blockIdx.x, pieces = tail.last_cta - c0 + 1;
    for (int q = blockIdx.y; q < tail.queries; q += gridDim.y) {
        float m = -INFINITY, l = 0.0f, acc[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j) acc[j] = 0.0f;
        for (int p0 = warp; p0 < pieces; p0 += 32) {          // four pieces of this warp in flight
            float pm[4], pl[4], po[4][VPL];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int p = p0 + 8 * u;
                pm[u] = -INFINITY; pl[u] = 0.0f;
#pragma unroll
                for (int j = 0; j < VPL; ++j) po[u][j] = 0.0f;
                if (p < pieces) {
                    const float* slot = tree_slot(scratch, p == 0 ? 2 * c0 + 1 : 2 * (c0 + p), tile_rows, DH);
                    pm[u] = slot[q];
                    pl[u] = slot[tile_rows + q];
                    const float* o = slot + 2 * tile_rows + (size_t)q * DH + lane * VPL;
#pragma unroll
                    for (int j = 0; j < VPL; ++j) po[u][j] = o[j];
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (pl[u] == 0.0f) continue;                   // nothing seen in this piece (NaN sums go on)
                const float top = fmaxf(m, pm[u]);
                const float fa = m == -INFINITY ? 0.0f : tree_ex2(m - top), fb = tree_ex2(pm[u] - top);
                l = l * fa + pl[u] * fb;
#pragma unroll
                for (int j = 0; j < VPL; ++j) acc[j] = acc[j] * fa + po[u][j] * fb;
                m = top;
            }
        }
        if (lane == 0) { m_s[warp] = m; l_s[warp] = l; }
#pragma unroll
        for (int j = 0; j < VPL; ++j) acc_s[warp][lane * VPL + j] = acc[j];
        __syncthreads();
        if (threadIdx.x < DH) {
            float top = -INFINITY, sum = 0.0f, o = 0.0f;
#pragma unroll
            for (int w = 0; w < 8; ++w) if (l_s[w] != 0.0f) top = fmaxf(top, m_s[w]);
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                if (l_s[w] == 0.0f) continue;
                const float f = tree_ex2(m_s[w] - top);
                sum += l_s[w] * f;
                o += acc_s[w][threadIdx.x] * f;
            }
            const int token = (tail.q0 + q) / group, head = tail.h * group + (tail.q0 + q - token * group);
            out[(int64_t)(tail.row0 + token) * out_stride + (int64_t)head * DH + threadIdx.x] = tree_round<T>(sum == 0.0f ? 0.0f : o / sum);
        }
        __syncthreads();
    }
}

}  // namespace zq
