// Work distribution of the attention kernels over a paged cache, shared by the CUDA-core and the tensor-core kernel.
//
// For request b with n new rows and L keys (C = L - n of them cached before this step, the drafts last) and g = n_heads /
// n_kv_heads query heads per key head, the queries that read one key head are the n * g vectors (draft i, head in group) in
// this order, cut into row tiles.  An item is (request, key head, row tile), its work the number of key tiles and a constant
// for opening and closing it (in tiles' time: without it the CTAs that get short contexts finish last; 16 x 32 heads of 100 to 2047
// keys at d_head 64, constants of 0 / 2 / 4 / 6: 98 / 70 / 62 / 61 us, 32 x 8 of 4096 at 128: 107 / 108 / 109 / 112).  All items' work, laid out one after the other, is cut into gridDim.x equal runs, one per CTA: long
// contexts are split over as many CTAs as it takes, short ones are packed, and no length is needed on the host.  Every CTA
// finds its run by scanning the requests' lengths.  A piece of an item that is not the whole item leaves (reference, sum, output) per
// query in the scratch, at most two pieces per CTA, and tree_combine_kernel joins them in the order of the keys, so results
// do not depend on timing.
#pragma once
#include "common.cuh"
#include "serve.cuh"
#include <cuda_fp16.h>

namespace zq {

struct TreeWork {
    const int32_t *kv_len, *row_start, *block_table;
    int batch, rows, n_kv, max_pages, page_size;
    int group;               // query heads per key head
    int tile_rows;           // queries per row tile
    int key_tile;            // keys per key tile
    int item_cost;           // work of an item besides its key tiles, in tiles
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

// The run of a CTA: the tiles [begin, end) of all tiles in order.  tail_cta: where the item ends that the run's end cuts in two.
struct TreeRun { long long begin, end; int tail_cta; TreeCursor at; };

// Run c of `total` work in `ctas` runs begins here: the first total % ctas runs have one unit more than the others.
__device__ __forceinline__ long long tree_run_begin(long long total, int ctas, int c) {
    const long long q = tree_div(total, ctas), r = total - q * ctas;
    return q * c + (c < r ? c : r);
}
// The CTA whose run holds unit `x`.
__device__ __forceinline__ int tree_cta_of(long long x, long long total, int ctas) {
    const long long q = tree_div(total, ctas), r = total - q * ctas, wide = r * (q + 1);
    return (int)(x < wide ? tree_div(x, q + 1) : r + tree_div(x - wide, q));
}

// The run of this CTA; called by all threads of the block (part: two words per warp, out: shared).  Ends with a barrier.
// An item's units are its constant, then its tiles: a tile belongs to the CTA whose run holds its unit.
__device__ __forceinline__ void tree_find_run(const TreeWork& w, long long* part, TreeRun* out) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const int per = (w.batch + blockDim.x - 1) / blockDim.x;
    const int b0 = min(tid * per, w.batch), b1 = min(b0 + per, w.batch);
    long long tiles = 0, items = 0;
    for (int b = b0; b < b1; ++b) {
        const TreeRequest r = tree_request(w, b);
        const long long n = r.n_kt ? (long long)w.n_kv * r.n_rt : 0;
        items += n;
        tiles += n * r.n_kt;
    }
    long long up_tiles = tiles, up_items = items;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, up_tiles, o), v = __shfl_up_sync(0xffffffffu, up_items, o);
        if (lane >= o) { up_tiles += u; up_items += v; }
    }
    if (lane == 31) { part[2 * warp] = up_tiles; part[2 * warp + 1] = up_items; }
    __syncthreads();
    long long all_tiles = 0, all_items = 0;
    for (int k = 0; k < warps; ++k) {
        if (k == warp) { up_tiles += all_tiles; up_items += all_items; }
        all_tiles += part[2 * k];
        all_items += part[2 * k + 1];
    }
    const long long total = all_tiles + w.item_cost * all_items;
    const int ctas = total < (long long)gridDim.x ? (int)total : (int)gridDim.x;
    const bool idle = (int)blockIdx.x >= ctas;
    if (tid == 0 && idle) { out->begin = out->end = 0; }
    if (!idle) {
        const long long lo = (up_tiles - tiles) + w.item_cost * (up_items - items), hi = up_tiles + w.item_cost * up_items;   // this thread's units
        const long long edge[2] = {tree_run_begin(total, ctas, blockIdx.x), tree_run_begin(total, ctas, blockIdx.x + 1)};
        if (tid == 0 && edge[1] == total) { out->end = all_tiles; out->tail_cta = -1; }
#pragma unroll 1
        for (int e = 0; e < 2; ++e) {
            if (edge[e] < lo || edge[e] >= hi) continue;           // exactly one thread goes on (none for the end of the last run)
            long long rest = edge[e] - lo, at_tile = up_tiles - tiles, unit = lo;
            TreeCursor c;
            int cost = 1;
            for (c.b = b0; c.b < b1; ++c.b) {
                c.load(w);
                if (c.r.n_kt == 0) continue;
                cost = c.r.n_kt + w.item_cost;
                const long long n = (long long)w.n_kv * c.r.n_rt;
                if (rest < n * cost) break;
                rest -= n * cost;
                unit += n * cost;
                at_tile += n * c.r.n_kt;
            }
            const long long item = tree_div(rest, cost), head = tree_div(item, c.r.n_rt);
            const int off = (int)(rest - item * cost);
            c.kt = max(0, off - w.item_cost);
            c.rt = (int)(item - head * c.r.n_rt);
            c.h = (int)head;
            at_tile += item * c.r.n_kt + c.kt;
            if (e == 0) { out->begin = at_tile; out->at = c; }
            else { out->end = at_tile; out->tail_cta = c.kt > 0 ? tree_cta_of(unit + (item + 1) * cost - 1, total, ctas) : -1; }
        }
    }
    __syncthreads();
}

// ---- partial results ------------------------------------------------------------------------------------------------
// One descriptor per CTA, a word that says whether its front slot is in use, then 2 * G slots of [tile_rows] references, [tile_rows] sums and [tile_rows][d_head] outputs (fp32).
struct TreeTail { int last_cta, queries, row0, q0, h, pad[3]; };   // an item that begins in this CTA and ends in last_cta; -1: none
constexpr int kMaxTreeGrid = 2 * 148;                    // one or two CTAs per SM
constexpr size_t kTailBytes = 12288, kFrontOffset = kMaxTreeGrid * sizeof(TreeTail);
static_assert(kFrontOffset + kMaxTreeGrid * sizeof(int) <= kTailBytes, "descriptors");

__host__ __device__ inline size_t tree_slot_floats(int tile_rows, int dh) { return (size_t)tile_rows * (dh + 2); }

// which CTAs have a front piece: one that continues an item of an earlier CTA (slot 2 c; slot 2 c + 1: one that goes on in the next)
__device__ __forceinline__ int* tree_front(uint8_t* scratch) { return reinterpret_cast<int*>(scratch + kFrontOffset); }

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
tree_combine_kernel(uint8_t* scratch, int tile_rows, int group, T* out, int64_t out_stride) {
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
                if (p < pieces && (p == 0 || tree_front(scratch)[c0 + p])) {
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
