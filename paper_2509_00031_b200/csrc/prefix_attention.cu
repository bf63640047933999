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
#include <type_traits>
#include "../../include/zoqat.h"

namespace zq {
namespace {

struct JoinParams {
    PrefixWork w;                            // tile_rows: unused
    uint8_t* pieces[2];                      // of the shared and the own parts
    int tile_rows[2];
    int workers[2];                          // that wrote them
    void* out;
    int64_t out_stride;
};

template <typename T, int DH, bool WIDE>
__global__ void __launch_bounds__(256)
prefix_join_kernel(const __grid_constant__ JoinParams p) {
    constexpr int VPL = DH / 32, kFly = WIDE ? 4 : 8;            // columns of a lane; pieces of a warp in flight
    typedef typename std::conditional<VPL == 4, float4, float2>::type Vec;
    __shared__ float acc_s[WIDE ? 8 : 1][DH], m_s[8], l_s[8];
    const PrefixWork& w = p.w;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.x, heads = w.n_kv * w.group;
    const int h = WIDE ? blockIdx.y : blockIdx.y * 8 + warp;
    if (!WIDE && h >= heads) return;
    const int64_t query = (int64_t)row * heads + h, side_queries = (int64_t)w.rows * heads;
    grid_dependency_wait();
    const int sides = w.row_sides[row];
    const int2 e0 = w.entries[query], e1 = w.entries[side_queries + query];      // (anything where there is no part)
    if (sides == 0) return;                                      // no request's row: left as it is
    // pieces of the shared part, then of the own one.  (Places that no worker can have: a wait ran out and nothing was written)
    int n[2], c0[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const int2 e = side ? e1 : e0;
        c0[side] = e.x & 0xFFFF;
        n[side] = e.y < 0 ? 1 : (e.x >> 16) - c0[side] + 1;
        if (e.y >= 0 && (n[side] < 0 || c0[side] + n[side] > p.workers[side] || e.y >= p.tile_rows[side])) n[side] = 0;
    }
    if (sides != 3) n[0] = 0;
    const int pieces = n[0] + n[1], first = WIDE ? warp : 0, step = WIDE ? 8 : 1;
    float m = -INFINITY, l = 0.0f, acc[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) acc[j] = 0.0f;
    for (int p0 = first; p0 < pieces; p0 += kFly * step) {
        float pm[kFly], pl[kFly];
        Vec po[kFly];
        bool there[kFly];
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const int i = p0 + u * step, side = i >= n[0], k = i - (side ? n[0] : 0), y = side ? e1.y : e0.y, c = side ? c0[1] : c0[0];
            pl[u] = 0.0f;
            there[u] = i < pieces;
            if (!there[u]) continue;
            const int rows = p.tile_rows[side];
            const float *o = w.partial + (side * side_queries + query) * (DH + 4), *ref = o + DH, *sum = o + DH + 1;
            if (y >= 0) {
                const float* slot = tree_slot(p.pieces[side], k == 0 ? 2 * c + 1 : 2 * (c + k), rows, DH);
                ref = slot + y; sum = slot + rows + y; o = slot + 2 * rows + (size_t)y * DH;
                if (k > 0) there[u] = prefix_front(p.pieces[side])[c + k];       // (else: its worker had no tile of the part)
            }
            pm[u] = *ref;
            pl[u] = *sum;
            po[u] = *reinterpret_cast<const Vec*>(o + lane * VPL);
        }
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            if (!there[u] || pl[u] == 0.0f) continue;            // nothing seen in this piece (NaN sums go on)
            const float top = fmaxf(m, pm[u]);
            const float fa = m == -INFINITY ? 0.0f : tree_ex2(m - top), fb = tree_ex2(pm[u] - top);
            const float* o = reinterpret_cast<const float*>(&po[u]);
            l = l * fa + pl[u] * fb;
#pragma unroll
            for (int j = 0; j < VPL; ++j) acc[j] = acc[j] * fa + o[j] * fb;
            m = top;
        }
    }
    T* dst = static_cast<T*>(p.out) + (int64_t)row * p.out_stride + (int64_t)h * DH;
    if (!WIDE) {
        T x[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j) x[j] = tree_round<T>(l == 0.0f ? 0.0f : acc[j] / l);
        struct alignas(VPL * sizeof(T)) Out { T x[VPL]; };
        *reinterpret_cast<Out*>(dst + lane * VPL) = *reinterpret_cast<const Out*>(x);
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
    // Eight warps a query while the queries are fewer than the warps that fit on the SMs: 512 / 1024 / 1536 / 2048 / 4096 queries and heads of one group behind
    // 16000 keys 46 / 47 / 53 / 56 / 78 us against 52 / 50 / 56 / 56 / 75 with one, behind 2000 25 / 28 / 32 / 37 / 49 against 29 / 29 / 31 / 35 / 44.
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
    // two slots to a worker: 148 of 256 queries, or their warps of up to 8
    const size_t f32 = kTailBytes + 2 * (size_t)(kMaxTreeGrid / 2 * kF32Warps) * tree_slot_floats(kF32Rows, d_head) * 4;
    const size_t narrow = kTailBytes + 2 * (size_t)kMaxWorkers * tree_slot_floats(kNarrowRows, d_head) * 4, wide = tree_attention_scratch_bytes(type, d_head);
    const size_t pieces = type == kTypeF32 ? f32 : (narrow > wide ? narrow : wide);
    at.pieces[0] = take(pieces);
    at.pieces[1] = type == kTypeF32 ? at.pieces[0] : take(pieces);
    at.entries = take((size_t)rows * n_heads * 2 * sizeof(int2));
    at.partial = reinterpret_cast<float*>(take((size_t)rows * n_heads * 2 * (d_head + 4) * sizeof(float)));
    at.row_sides = reinterpret_cast<int*>(take((size_t)rows * sizeof(int)));
    at.bytes = used;
    return at;
}

int launch_prefix_attention(const PrefixAttnArgs& a, void* scratch, cudaStream_t s, bool dependent) {
    const TreeAttnArgs& t = a.t;
    const PrefixScratch at = prefix_scratch(scratch, t.cache.type, t.cache.d_head, t.rows, t.n_heads);
    JoinParams p{};
    const int group = t.n_heads / t.cache.n_kv_heads;
    static_cast<TreeWork&>(p.w) = TreeWork{t.kv_len, t.row_start, t.block_table, t.batch, t.rows, t.cache.n_kv_heads, t.max_pages, t.cache.page_size, group, 1, 1, 0, t.err_flag};
    prefix_work(a, at, 0, 0, p.w);
    p.pieces[0] = p.pieces[1] = at.pieces[0];
    p.workers[0] = p.workers[1] = tree_grid();
    p.out = t.out; p.out_stride = t.out_stride;
    if (t.cache.type == kTypeF32) {
        p.tile_rows[0] = p.tile_rows[1] = kF32Rows;
        p.workers[0] = p.workers[1] = kF32Warps * tree_grid();
        if (int rc = launch_prefix_f32(a, at, s, dependent)) return rc;
        return t.cache.d_head == 64 ? join<float, 64>(p, s) : join<float, 128>(p, s);
    }
    // Queries per tile from averages (the host does not know the lengths; rows behind the last request count too, hence borders a little above the tiles).  us at tiles of
    // 8 / 32 / 64 / 256, 8 key heads of 128, bf16.  8 groups behind 8000 keys, own keys few: 4 queries 55 / 79 / 78 / 108; 8: 58 / 77 / 77 / 98; 16: 68 / 78 / 79 / 100; 32: 173 / 75 /
    // 76 / 100; 64: 245 / 106 / 83 / 98; 128: 441 / 176 / 125 / 108.  64 requests with 700 own keys: 8 queries 80 / 109 / 100 / 169; 16: 84 / 102 / 104 / 121; 24: 125 / 123 / 126 / 137;
    // 32: 141 / 129 / 132 / 148; 64: 219 / 261 / 242 / 181 (short parts: what it costs to open a tile counts, hence the margin of a half).
    const long long queries = (long long)t.rows * group;
    const long long shared = (queries + a.groups - 1) / a.groups, own = (queries + t.batch - 1) / t.batch;
    auto tile = [](long long want) { return want <= 32 ? 32 : (want <= 64 ? 64 : 256); };
    p.tile_rows[0] = shared <= 18 ? kNarrowRows : tile(shared - shared / 8);
    p.tile_rows[1] = own <= 18 ? kNarrowRows : tile(own + own / 2);
    if (p.tile_rows[0] != p.tile_rows[1]) p.pieces[1] = at.pieces[1];
    for (int side = 0; side < 2; ++side) p.workers[side] = p.tile_rows[side] <= kNarrowRows ? p.workers[side] * kNarrowWarps : p.workers[side];
    if (int rc = launch_prefix_tc(a, at, p.tile_rows, s, dependent)) return rc;
    if (t.cache.type == kTypeBf16) return t.cache.d_head == 64 ? join<__nv_bfloat16, 64>(p, s) : join<__nv_bfloat16, 128>(p, s);
    return t.cache.d_head == 64 ? join<__half, 64>(p, s) : join<__half, 128>(p, s);
}

}  // namespace zq
