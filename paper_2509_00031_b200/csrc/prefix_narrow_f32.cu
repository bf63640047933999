// Parts of an attention over a paged fp32 cache, on the CUDA cores (parts of a shared prefix and requests' own keys: tree_attention.cuh).
//
// As in prefix_narrow.cu a warp is a worker of its own: the 10 warps of every SM cut the tiles of all parts into equal runs and never wait for one
// another.  A tile is 32 keys at d_head 64 and 16 at 128, its K and V 16 KB; they pass through shared memory as a queue of each thread's own 16-byte
// chunks (cp.async): a thread reads back exactly what it asked for, so there are neither barriers nor bank conflicts, and pages of any size
// will do.  With g = lane / 4, j = lane % 4
//   scores  a thread has chunks j + 4 i of the keys g + 8 u and adds up their products with 8 queries (from shared memory, the same for all keys);
//           the four lanes of a key swap halves twice, which leaves queries 2 j, 2 j + 1 of its keys with each
//   output  a thread has one chunk (4 columns) of every key (d_head 64: of every other key), and 8 queries' weights from shared memory
// both as pairs of products in one instruction (fma.rn.f32x2).  Eight queries cost 2 x 8 x d_head fused operations a key against 8 x d_head bytes from memory: 128
// instructions of a warp for 16 keys at d_head 64, where the memory's share is some 190 cycles of the SM.  3 prompts of 500 to 4000 keys, 2 to 6 requests each with 1 to 3
// drafts, 32 heads of 64: 51.3 us, 20 of them the cache's 131 MB at the rate of a copy (the way of tree_attention.cu, which reads every query from shared memory for every key
// and meets at a barrier for every tile: 110).  Bound by a warp's own chain of some 1000 instructions for a tile, a third of them products, with
// ten warps an SM (28 % of the issue slots, 32 % of the memory's rate); at d_head 64 the compiler spills 64 bytes a thread and loads 24 again, 168 registers (with 138 and 184: 55.5 us).
// The running maximum is exact for every tile; everything is binary32.
#include "tree_attention.cuh"
#include "tc_ptx.cuh"
#include "../../include/zoqat.h"

namespace zq {
namespace {

constexpr int kWarps = kF32Warps, kThreads = 32 * kWarps, kQ = kF32Rows;

template <int DH> struct F32Cfg {
    static constexpr int kTile = DH == 64 ? 32 : 16;
    static constexpr int kFifo = 2 * kTile * DH * 4;                        // K, then V of a tile
    static constexpr int kOffQ = kFifo, kOffP = kOffQ + kQ * DH * 4, kOffPlace = kOffP + kTile * kQ * 4;
    static constexpr int kWarpBytes = kOffPlace + 2 * kTile * 8;            // queries, weights, places of two tiles' keys
    static constexpr int kSmem = kWarps * kWarpBytes;
    static_assert(kTile <= kF32Border, "the border between the parts");
};

struct F32Params {
    PrefixWork w;
    const float* q;
    int64_t q_stride;
    PagedCache cache;
    const uint32_t* tree_mask;
    int mask_words;
    float scale_log2;
    uint8_t* scratch;
};

__device__ __forceinline__ void async16(uint32_t dst, const float* src, bool live) {
    const int n = live ? 16 : 0;             // 0: zeros, nothing is read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ float4 lds4(uint32_t at) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}

template <int DH>
__global__ void __launch_bounds__(kThreads, 1)
prefix_f32_kernel(const __grid_constant__ F32Params p) {
    using Cfg = F32Cfg<DH>;
    constexpr int kTile = Cfg::kTile, kU = kTile / 8, kI = DH / 16, kV = 16, kRows = kTile / kV;      // keys and chunks of K a thread has; keys of V; rows of V a warp reads at once
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ TreeRunT<PrefixWork> runs[kWarps];
    __shared__ PrefixScan scan;
    const PrefixWork& w = p.w;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, j = lane & 3;
    const int worker = blockIdx.x * kWarps + warp;
    grid_dependency_wait();
    grid_dependency_release();
    prefix_find_runs<kWarps>(w, scan, runs);
    if (blockIdx.x == gridDim.x - 1) prefix_map_rows(w, scan);
    const TreeRunT<PrefixWork>& run = runs[warp];
    const int n_tiles = (int)(run.end - run.begin);
    if (lane == 0) prefix_front(p.scratch)[worker] = n_tiles > 0 && !run.at.item_begins();
    if (n_tiles <= 0) return;

    uint8_t* const mine = smem + warp * Cfg::kWarpBytes;
    const uint32_t fifo = smem_u32(mine) + lane * 16, values = fifo + kU * kI * 512;
    float* const q_s = reinterpret_cast<float*>(mine + Cfg::kOffQ);
    float* const p_s = reinterpret_cast<float*>(mine + Cfg::kOffP);
    int64_t* const place_s = reinterpret_cast<int64_t*>(mine + Cfg::kOffPlace);
    const int col = 4 * (DH == 64 ? lane & 15 : lane), hi = DH == 64 ? lane >> 4 : 0;
    PrefixCursor c, ahead;
    c.r = run.at.r; c.b = run.at.b; c.h = run.at.h; c.rt = run.at.rt; c.kt = run.at.kt;
    ahead = c;
    int page = 0, off = 0;                                       // of key `lane` of the tile ahead
    auto look_up = [&]() {
        const int key = ahead.kt * kTile + (lane & (kTile - 1)), i = key / w.page_size;
        off = key < ahead.r.L ? key - i * w.page_size : -1;
        page = off >= 0 ? __ldg(w.block_table + (size_t)ahead.r.row * w.max_pages + i) : 0;
    };
    auto note = [&](int t) {                                     // where the keys of tile t stand; -1: behind the end, or on a bad page
        int64_t at = -1;
        if (off >= 0) {
            if (page < 0 || page >= p.cache.n_pages) atomicExch(w.err_flag, kErrBadPage);
            else at = page * p.cache.page_stride + off * p.cache.slot_stride + ahead.h * p.cache.head_stride;
        }
        __syncwarp();
        if (lane < kTile) place_s[(t & 1) * kTile + lane] = at;
        __syncwarp();
    };
    auto request_keys = [&](int t) {
        const float* k = static_cast<const float*>(p.cache.k) + 4 * j;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int64_t at = place_s[(t & 1) * kTile + 8 * u + g];
#pragma unroll
            for (int i = 0; i < kI; ++i) async16(fifo + (u * kI + i) * 512, k + (at < 0 ? 0 : at + 16 * i), at >= 0);
        }
    };
    auto request_values = [&](int t) {
        const float* v = static_cast<const float*>(p.cache.v) + col;
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            const int64_t at = place_s[(t & 1) * kTile + kRows * e + hi];
            async16(values + e * 512, v + (at < 0 ? 0 : at), at >= 0);
        }
    };
    look_up();
    note(0);
    request_keys(0);
    async_commit();
    request_values(0);
    async_commit();
    if (n_tiles > 1) { ahead.next(w, scan); look_up(); }

    bool split_front = !run.at.item_begins(), opens = true;
    int nq = 0, q0 = 0;
    float2 o[kQ / 2][4];                                         // queries 2 n, 2 n + 1; columns
    float m[2], l[2];                                            // queries 2 j, 2 j + 1
#pragma unroll 1
    for (int t = 0; t < n_tiles; ++t) {
        if (t + 1 < n_tiles) note(t + 1);
        if (opens) {
            opens = false;
            q0 = c.rt * kQ;
            nq = min(kQ, c.r.n * w.group - q0);
            __syncwarp();
#pragma unroll
            for (int i = lane; i < kQ * DH / 4; i += 32) {
                const int row = i / (DH / 4), tok = (q0 + row) / w.group;
                float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (row < nq)
                    x = __ldg(reinterpret_cast<const float4*>(p.q + (int64_t)(c.r.row0 + tok) * p.q_stride + (int64_t)(c.h * w.group + q0 + row - tok * w.group) * DH) + i % (DH / 4));
                reinterpret_cast<float4*>(q_s)[i] = x;
            }
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 2; ++e) { m[e] = -INFINITY; l[e] = 0.0f; }
#pragma unroll
            for (int n = 0; n < kQ / 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = make_float2(0.0f, 0.0f);
        }
        async_wait<1>();                                         // the keys
        float2 s2[kU][kQ] = {};
        const uint32_t q_at = smem_u32(q_s) + 16 * j;
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            float4 k[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) k[u] = lds4(fifo + (u * kI + i) * 512);
#pragma unroll
            for (int n = 0; n < kQ; ++n) {
                const float4 x = lds4(q_at + n * (DH * 4) + 64 * i);
#pragma unroll
                for (int u = 0; u < kU; ++u)
                    s2[u][n] = tree_fma2(make_float2(x.z, x.w), make_float2(k[u].z, k[u].w), tree_fma2(make_float2(x.x, x.y), make_float2(k[u].x, k[u].y), s2[u][n]));
            }
        }
        if (t + 1 < n_tiles) request_keys(t + 1);                // (a thread's own chunks have been read)
        async_commit();
        // over the four lanes of a key: queries 2 j, 2 j + 1 stay
        float s[kU][2];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            float v[kQ];
#pragma unroll
            for (int n = 0; n < kQ; ++n) v[n] = s2[u][n].x + s2[u][n].y;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float keep = j & 2 ? v[n + 4] : v[n], give = j & 2 ? v[n] : v[n + 4];
                v[n] = keep + __shfl_xor_sync(0xffffffffu, give, 2);
            }
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float keep = j & 1 ? v[n + 2] : v[n], give = j & 1 ? v[n] : v[n + 2];
                s[u][n] = __fmul_rn(keep + __shfl_xor_sync(0xffffffffu, give, 1), p.scale_log2);      // rounded by itself: references are such products
            }
        }
        const int key0 = c.kt * kTile, C = c.r.L - c.r.drafts();
        const bool tail = key0 + kTile > C;
        uint32_t seen[2] = {0xFFFFFFFFu, 0xFFFFFFFFu};           // bits of the tile's keys
        if (tail) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int tok = (q0 + 2 * j + e) / w.group;
                uint32_t vis = 0;
                if (2 * j + e < nq) {
                    const uint32_t* mask = p.tree_mask ? p.tree_mask + (size_t)(c.r.row0 + tok) * p.mask_words : nullptr;
                    for (int k = 0; k < kTile && key0 + k < c.r.L; ++k) {
                        const int d = key0 + k - C;
                        const bool sees = d < 0 || (mask ? d < 32 * p.mask_words && (__ldg(mask + (d >> 5)) >> (d & 31)) & 1u : d <= tok);
                        vis |= (uint32_t)sees << k;
                    }
                }
                seen[e] = vis;
#pragma unroll
                for (int u = 0; u < kU; ++u)
                    if (!((vis >> (8 * u + g)) & 1u)) s[u][e] = -INFINITY;
            }
        }
        float f[2];
        bool moved = false;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float top = s[0][e];
#pragma unroll
            for (int u = 1; u < kU; ++u) top = fmaxf(top, s[u][e]);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            top = fmaxf(top, m[e]);
            const float ref = top == -INFINITY ? 0.0f : top;     // nothing seen yet: every weight is 0
            f[e] = tree_ex2(m[e] - ref);
            moved = moved || top != m[e];
            m[e] = top;
            l[e] *= f[e];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                s[u][e] = tree_ex2(s[u][e] - ref);
                l[e] += s[u][e];
                // (a weight below zero: not seen, whatever the value holds)
                if (tail && !((seen[e] >> (8 * u + g)) & 1u)) s[u][e] = -1.0f;
            }
        }
        __syncwarp();                                            // the weights before have been read
#pragma unroll
        for (int u = 0; u < kU; ++u) *reinterpret_cast<float2*>(p_s + (8 * u + g) * kQ + 2 * j) = make_float2(s[u][0], s[u][1]);
        __syncwarp();
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int n = 0; n < kQ / 2; ++n) {                   // (queries 2 n, 2 n + 1 are lane n's)
                const float2 ff = make_float2(__shfl_sync(0xffffffffu, f[0], n), __shfl_sync(0xffffffffu, f[1], n));
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = tree_mul2(o[n][e], ff);
            }
        }
        async_wait<1>();                                         // the values
        const uint32_t p_at = smem_u32(p_s) + hi * (kQ * 4);
        auto add = [&](auto all) {
#pragma unroll
            for (int e = 0; e < kV; ++e) {
                const float4 v = lds4(values + e * 512), a = lds4(p_at + e * (kRows * kQ * 4)), b = lds4(p_at + e * (kRows * kQ * 4) + 16);
                const float2 x[4] = {make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)};
                const float y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int n = 0; n < kQ / 2; ++n)
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        if constexpr (all.value) {
                            o[n][d] = tree_fma2(x[n], make_float2(y[d], y[d]), o[n][d]);
                        } else {
                            if (!(x[n].x < 0.0f)) o[n][d].x = fmaf(x[n].x, y[d], o[n][d].x);
                            if (!(x[n].y < 0.0f)) o[n][d].y = fmaf(x[n].y, y[d], o[n][d].y);
                        }
                    }
            }
        };
        if (tail) add(std::false_type{});
        else add(std::true_type{});
        if (t + 1 < n_tiles) request_values(t + 1);
        async_commit();
        if (t + 2 < n_tiles) { ahead.next(w, scan); look_up(); }
        const bool ends = c.kt == c.r.n_kt - 1;
        if (ends || t == n_tiles - 1) {
            const bool whole = ends && !split_front;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[e] += __shfl_xor_sync(0xffffffffu, l[e], 4);
                l[e] += __shfl_xor_sync(0xffffffffu, l[e], 8);
                l[e] += __shfl_xor_sync(0xffffffffu, l[e], 16);
            }
            float* slot = tree_slot(p.scratch, split_front ? 2 * worker : 2 * worker + 1, kQ, DH);
#pragma unroll
            for (int n = 0; n < kQ; ++n) {
                float4 x;
                float* const y = &x.x;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    y[d] = n & 1 ? o[n >> 1][d].y : o[n >> 1][d].x;
                    if (DH == 64) y[d] += __shfl_xor_sync(0xffffffffu, y[d], 16);
                }
                const float ref = __shfl_sync(0xffffffffu, n & 1 ? m[1] : m[0], n >> 1), sum = __shfl_sync(0xffffffffu, n & 1 ? l[1] : l[0], n >> 1);
                if (n >= nq) continue;
                const int64_t query = prefix_query(w, c.r, q0 + n, c.h);
                float* to = whole ? w.partial + query * (DH + 4) : slot + 2 * kQ + n * DH;
                if (hi == 0) *reinterpret_cast<float4*>(to + col) = x;
                if (lane == 0) {
                    if (whole) { to[DH] = ref; to[DH + 1] = sum; }
                    else { slot[n] = ref; slot[kQ + n] = sum; }
                    if (!split_front) w.entries[query] = ends ? make_int2(0, -1) : make_int2(worker | run.tail_cta << 16, n);
                }
            }
            split_front = false;
            opens = true;
        }
        c.next(w, scan);
    }
    async_wait<0>();
}

template <int DH>
int f32_launch(const F32Params& p, int grid, cudaStream_t s, bool dependent) {
    static DeviceOnce attr;
    if (!attr.done([] { return allow_smem(prefix_f32_kernel<DH>, F32Cfg<DH>::kSmem); })) return ZOQAT_ERR_CUDA;
    if (launch_kernel(prefix_f32_kernel<DH>, dim3(grid), dim3(kThreads), F32Cfg<DH>::kSmem, s, dependent, p) != cudaSuccess) return ZOQAT_ERR_CUDA;
    count_launch();
    return ZOQAT_OK;
}

}  // namespace

int launch_prefix_f32(const PrefixAttnArgs& a, const PrefixScratch& at, cudaStream_t s, bool dependent) {
    const TreeAttnArgs& t = a.t;
    F32Params p{};
    static_cast<TreeWork&>(p.w) = TreeWork{t.kv_len, t.row_start, t.block_table, t.batch, t.rows, t.cache.n_kv_heads, t.max_pages, t.cache.page_size,
                                           t.n_heads / t.cache.n_kv_heads, kQ, t.cache.d_head == 64 ? F32Cfg<64>::kTile : F32Cfg<128>::kTile, 2, t.err_flag};
    prefix_work(a, at, 0, a.groups + t.batch, p.w);
    p.q = static_cast<const float*>(t.q); p.q_stride = t.q_stride; p.cache = t.cache;
    p.tree_mask = t.tree_mask; p.mask_words = t.mask_words;
    p.scale_log2 = (float)(1.4426950408889634 * (double)t.scale);
    p.scratch = at.pieces[0];
    return t.cache.d_head == 64 ? f32_launch<64>(p, tree_grid(), s, dependent) : f32_launch<128>(p, tree_grid(), s, dependent);
}

}  // namespace zq
