// Attention of a batch whose requests share a long prefix: the prefix's keys are read once for all requests of a group.
//
//   out[r, h] = softmax(scale q[r, h] . K) V over [the shared keys | the request's own]
//
// The attention kernels over the pages (tree_attention*.cu) run over a list of parts - the shared keys with the queries of all the group's
// requests as rows, each request's own keys with its queries (tree_attention.cuh) - and leave a reference m, a sum l and an unscaled output o for each
// query and part, in one piece or, where a part was split over CTAs, in several:
//
//   M = max_p m_p      out = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p
//
// over the pieces of the shared part, then of the own, in the order of the keys; in fp32, one rounding at the end.  prefix_join_kernel does that:
// a warp per query and head, or, where there are few queries (whose parts are then split over many CTAs), eight warps.
#include "tree_attention.cuh"
#include "../../include/zoqat.h"

namespace zq {
namespace {

struct JoinParams {
    PrefixWork w;                            // tile_rows: unused
    uint8_t* pieces[2];                      // of the shared and the own parts
    int tile_rows[2];
    int grid;                                // CTAs that wrote them
    void* out;
    int64_t out_stride;
};

struct Sum { float m, l; };

template <typename T, int DH, bool WIDE>
__global__ void __launch_bounds__(256)
prefix_join_kernel(const JoinParams p) {
    constexpr int VPL = DH / 32;
    __shared__ int request_s;
    __shared__ float acc_s[WIDE ? 8 : 1][DH], m_s[8], l_s[8];
    const PrefixWork& w = p.w;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.x, heads = w.n_kv * w.group;
    if (tid == 0) request_s = -1;
    grid_dependency_wait();
    __syncthreads();
    for (int b = tid; b < w.requests; b += 256)
        if (__ldg(w.row_start + b) <= row && row < __ldg(w.row_start + b + 1)) request_s = b;
    __syncthreads();
    const int b = request_s;
    if (b < 0) return;                                           // no request's row: left as it is
    bool ok;
    const PrefixRequest own = prefix_own(w, b, ok);
    if (!ok || own.n_kt == 0 || row < own.row0 || row >= own.row0 + own.n) return;
    const PrefixRequest shared = prefix_shared(w, __ldg(w.request_group + b), ok);
    if (!ok) return;
    const int h = WIDE ? blockIdx.y : blockIdx.y * 8 + warp;
    if (!WIDE && h >= heads) return;
    const int first = WIDE ? warp : 0, step = WIDE ? 8 : 1;      // pieces of this warp
    float m = -INFINITY, l = 0.0f, acc[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) acc[j] = 0.0f;
    for (int side = shared.n_kt > 0 ? 0 : 1; side < 2; ++side) {
        const int64_t at = ((int64_t)side * w.rows + row) * heads + h;
        const int2 e = w.entries[at];
        const bool whole = e.y < 0;
        const int c0 = whole ? 0 : e.x & 0xFFFF, pieces = whole ? 1 : (e.x >> 16) - c0 + 1;
        if (!whole && (c0 + pieces > p.grid || e.y >= p.tile_rows[side])) continue;      // (a wait ran out: nothing was written)
        for (int p0 = first; p0 < pieces; p0 += 4 * step) {      // four pieces in flight
            float pm[4], pl[4], po[4][VPL];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int k = p0 + u * step;
                pm[u] = -INFINITY; pl[u] = 0.0f;
#pragma unroll
                for (int j = 0; j < VPL; ++j) po[u][j] = 0.0f;
                if (k >= pieces || (k > 0 && !tree_front(p.pieces[side])[c0 + k])) continue;
                const float* slot = whole ? nullptr : tree_slot(p.pieces[side], k == 0 ? 2 * c0 + 1 : 2 * (c0 + k), p.tile_rows[side], DH);
                const float* o = whole ? w.partial + at * (DH + 4) : slot + 2 * p.tile_rows[side] + (size_t)e.y * DH;
                pm[u] = whole ? o[DH] : slot[e.y];
                pl[u] = whole ? o[DH + 1] : slot[p.tile_rows[side] + e.y];
#pragma unroll
                for (int j = 0; j < VPL; ++j) po[u][j] = o[lane * VPL + j];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (pl[u] == 0.0f) continue;                     // nothing seen in this piece (NaN sums go on)
                const float top = fmaxf(m, pm[u]);
                const float fa = m == -INFINITY ? 0.0f : tree_ex2(m - top), fb = tree_ex2(pm[u] - top);
                l = l * fa + pl[u] * fb;
#pragma unroll
                for (int j = 0; j < VPL; ++j) acc[j] = acc[j] * fa + po[u][j] * fb;
                m = top;
            }
        }
    }
    T* dst = static_cast<T*>(p.out) + (int64_t)row * p.out_stride + (int64_t)h * DH;
    if (!WIDE) {
#pragma unroll
        for (int j = 0; j < VPL; ++j) dst[lane * VPL + j] = tree_round<T>(l == 0.0f ? 0.0f : acc[j] / l);
        return;
    }
    if (lane == 0) { m_s[warp] = m; l_s[warp] = l; }
#pragma unroll
    for (int j = 0; j < VPL; ++j) acc_s[WIDE ? warp : 0][lane * VPL + j] = acc[j];
    __syncthreads();
    if (tid >= DH) return;
    float top = -INFINITY, sum = 0.0f, o = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) if (l_s[k] != 0.0f) top = fmaxf(top, m_s[k]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (l_s[k] == 0.0f) continue;
        const float f = tree_ex2(m_s[k] - top);
        sum += l_s[k] * f;
        o += acc_s[WIDE ? k : 0][tid] * f;
    }
    dst[tid] = tree_round<T>(sum == 0.0f ? 0.0f : o / sum);
}

template <typename T, int DH>
int join(const JoinParams& p, cudaStream_t s) {
    const int heads = p.w.n_kv * p.w.group;
    const bool wide = (int64_t)p.w.rows * heads <= 148 * 8;
    const cudaError_t rc = wide ? launch_kernel(prefix_join_kernel<T, DH, true>, dim3(p.w.rows, heads), dim3(256), 0, s, true, p)
                                : launch_kernel(prefix_join_kernel<T, DH, false>, dim3(p.w.rows, (heads + 7) / 8), dim3(256), 0, s, true, p);
    if (rc != cudaSuccess) return ZOQAT_ERR_CUDA;
    count_launch();
    return ZOQAT_OK;
}

}  // namespace

PrefixScratch prefix_scratch(void* base, int type, int d_head, int64_t rows, int n_heads) {
    PrefixScratch at{};
    uint8_t* p = static_cast<uint8_t*>(base);
    size_t used = 0;
    auto take = [&](size_t bytes) { const size_t o = used; used += (bytes + 255) / 256 * 256; return p ? p + o : nullptr; };
    at.pieces[0] = take(tree_attention_scratch_bytes(type, d_head));
    at.pieces[1] = type == kTypeF32 ? at.pieces[0] : take(tree_attention_scratch_bytes(type, d_head));
    at.entries = take((size_t)rows * n_heads * 2 * sizeof(int2));
    at.partial = reinterpret_cast<float*>(take((size_t)rows * n_heads * 2 * (d_head + 4) * sizeof(float)));
    at.bytes = used;
    return at;
}

int launch_prefix_attention(const PrefixAttnArgs& a, void* scratch, cudaStream_t s, bool dependent) {
    const TreeAttnArgs& t = a.t;
    const PrefixScratch at = prefix_scratch(scratch, t.cache.type, t.cache.d_head, t.rows, t.n_heads);
    JoinParams p{};
    const int group = t.n_heads / t.cache.n_kv_heads;
    static_cast<TreeWork&>(p.w) = TreeWork{t.kv_len, t.row_start, t.block_table, t.batch, t.rows, t.cache.n_kv_heads, t.max_pages, t.cache.page_size, group, 1, kSimtKeys, 0, t.err_flag};
    prefix_work(a, at, 0, 0, p.w);
    p.pieces[0] = p.pieces[1] = at.pieces[0];
    p.grid = tree_grid();
    p.out = t.out; p.out_stride = t.out_stride;
    if (t.cache.type == kTypeF32) {
        p.tile_rows[0] = p.tile_rows[1] = kSimtRows;
        p.grid *= 2;
        if (int rc = launch_prefix_simt(a, at, s, dependent)) return rc;
        return t.cache.d_head == 64 ? join<float, 64>(p, s) : join<float, 128>(p, s);
    }
    // Queries per tile from averages (the host does not know the lengths).
    const long long queries = (long long)t.rows * group;
    const long long own = t.rows <= t.batch ? group : (3 * queries + 2 * t.batch - 1) / (2 * t.batch);       // 1.5 x the average
    const long long shared = (queries + a.groups - 1) / a.groups;
    int tile_shared = shared <= 64 ? (int)shared : 256, tile_own = own <= 64 ? (int)own : 256;
    if (tile_shared <= 64 && tile_own <= 64) tile_shared = tile_own = tile_shared > tile_own ? tile_shared : tile_own;
    p.w.key_tile = kKeys;
    auto rows_of = [](int n) { return n <= 16 ? 16 : (n <= 32 ? 32 : (n <= 64 ? 64 : 256)); };
    p.tile_rows[0] = rows_of(tile_shared); p.tile_rows[1] = rows_of(tile_own);
    if (p.tile_rows[0] != p.tile_rows[1]) p.pieces[1] = at.pieces[1];
    if (int rc = launch_prefix_tc(a, at, tile_shared, tile_own, s, dependent)) return rc;
    if (t.cache.type == kTypeBf16) return t.cache.d_head == 64 ? join<__nv_bfloat16, 64>(p, s) : join<__nv_bfloat16, 128>(p, s);
    return t.cache.d_head == 64 ? join<__half, 64>(p, s) : join<__half, 128>(p, s);
}

}  // namespace zq
