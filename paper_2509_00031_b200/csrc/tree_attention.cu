// Attention of drafted rows over a paged fp32 cache on the CUDA cores (the type of the decode path's own cache; bf16 and
// fp16 caches run on the tensor cores, tree_attention_tc.cu).
//
//   out[i, h] = sum_t softmax_t(scale q[i, h] . k[t, h / g]) v[t, h / g]      over the keys t < C cached before the step and
//                                                                            the drafts j (t = C + j) whose mask bit is set
//
// With up to 8 queries per key head a key costs 2 * 8 * d_head fused multiply-adds against 8 * d_head bytes from memory: the
// kernel is bound by reading the cache: 5.7 TB/s for 8 x 32 heads of 4096 keys at d_head 128.  A CTA of 8 warps takes key tiles of
// 32 keys through two stages filled by cp.async, two CTAs per SM (8 x 32 heads of 1 to 1020 keys: 59.8 us; one CTA with a ring of
// five stages, 128 KB in flight, 65: two hide one another's joins); each warp owns 4 keys of every tile and keeps its own running maximum, sum and output
// for all 8 queries in registers, so the warps meet once per tile, where a stage is handed over, and once per item, when
// their results are joined in shared memory.  Two CTAs per SM leave 128 registers a thread: at d_head 128 ptxas spills 108 bytes.
//   scores  8 lanes per key, each an eighth of its elements (every K element is read from shared memory once), joined by three
//           shuffles per query
//   output  a lane owns 4 (2) columns of all queries; every V element is read once
#include "tree_attention.cuh"
#include "../../include/zoqat.h"

namespace zq {
namespace {

constexpr int kSimtThreads = 256, kSimtKeys = 32, kSimtRows = 8, kSimtStages = 2;
constexpr int kWarpKeys = kSimtKeys / 8, kKeyLanes = 32 / kWarpKeys;      // keys of a tile per warp, lanes per key

template <int DH> struct SimtCfg {
    static constexpr int kStageFloats = 2 * kSimtKeys * DH;                 // K, then V
    static constexpr int kOffQ = kSimtStages * kStageFloats;
    static constexpr int kOffP = kOffQ + kSimtRows * DH;                    // [8 warps][8 queries][4 keys]
    static constexpr int kOffAcc = kOffP + 8 * kSimtRows * kWarpKeys;               // [8 warps][8 queries][DH]
    static constexpr int kOffML = kOffAcc + 8 * kSimtRows * DH;             // [8 warps][8 queries] references, then sums
    static constexpr int kOffKeys = kOffML + 2 * 8 * kSimtRows;             // [2][32] places of keys (64-bit)
    static constexpr int kSmemBytes = (kOffKeys + 4 * kSimtKeys) * 4;
};

struct SimtParams {
    TreeWork w;
    const float* q;
    int64_t q_stride;
    PagedCache cache;
    const uint32_t* tree_mask;
    int mask_words;
    float scale_log2;
    float* out;
    int64_t out_stride;
    uint8_t* scratch;
};

__device__ __forceinline__ void cp_async16(float* dst, const float* src, bool live) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    const int n = live ? 16 : 0;                           // 0: the 16 bytes are filled with zeros, nothing is read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Where the keys of the cursor's tile stand in the cache, in elements; -1: behind the request's end, or on a bad page.
__device__ __forceinline__ void find_keys(const SimtParams& p, const TreeCursor& c, int64_t* offs) {
    const int key = threadIdx.x;
    if (key >= kSimtKeys) return;
    const int t = c.kt * kSimtKeys + key;
    int64_t off = -1;
    if (t < c.r.L) {
        const int pg = t / p.w.page_size;
        const int page = __ldg(p.w.block_table + (size_t)c.b * p.w.max_pages + pg);
        if (page < 0 || page >= p.cache.n_pages) atomicExch(p.w.err_flag, kErrBadPage);
        else off = page * p.cache.page_stride + (t - pg * p.w.page_size) * p.cache.slot_stride + c.h * p.cache.head_stride;
    }
    offs[key] = off;
}

// Requests the keys and values of a tile; keys without a place become zeros.
template <int DH>
__device__ __forceinline__ void load_tile(const SimtParams& p, const int64_t* offs, float* stage) {
    constexpr int kPer = DH / 4;                           // 16-byte chunks of a key
    constexpr int kStep = kSimtThreads / kPer;
    const int ch = threadIdx.x % kPer;
    const float* kb = static_cast<const float*>(p.cache.k) + 4 * ch;
    const float* vb = static_cast<const float*>(p.cache.v) + 4 * ch;
#pragma unroll
    for (int key = threadIdx.x / kPer; key < kSimtKeys; key += kStep) {
        const int64_t off = offs[key];
        const bool live = off >= 0;
        cp_async16(stage + key * DH + 4 * ch, kb + (live ? off : 0), live);
        cp_async16(stage + (kSimtKeys + key) * DH + 4 * ch, vb + (live ? off : 0), live);
    }
}

// One tile for MR queries of the row tile (q0: the first).  m, l, acc: the warp's running state (l: per lane).
template <int DH, int MR>
__device__ __forceinline__ void tile_step(const SimtParams& p, const TreeCursor& c, int q0, int nq, const float* stage, const float* qs, float* ps,
                                          float (&m)[kSimtRows], float (&l)[kSimtRows], float (&acc)[kSimtRows][DH / 32]) {
    constexpr int VPL = DH / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int key = kWarpKeys * warp + lane / kKeyLanes, share = lane % kKeyLanes;
    const float4* kr = reinterpret_cast<const float4*>(stage + key * DH);
    const float* vs = stage + (kSimtKeys + kWarpKeys * warp) * DH + lane * VPL;
    float s[MR];
#pragma unroll
    for (int r = 0; r < MR; ++r) s[r] = 0.0f;
#pragma unroll
    for (int i = 0; i < DH / (4 * kKeyLanes); ++i) {
        const float4 kv = kr[share + kKeyLanes * i];
#pragma unroll
        for (int r = 0; r < MR; ++r) {
            const float4 qv = reinterpret_cast<const float4*>(qs + r * DH)[share + kKeyLanes * i];
            s[r] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, s[r]))));
        }
    }
    const int C = c.r.L - c.r.n, t = c.kt * kSimtKeys + key;
    const bool tail = (c.kt + 1) * kSimtKeys > C;          // some of the tile's keys are drafts, or lie behind the end
    uint32_t seen[MR];                                     // bit kKeyLanes * j: key j of this warp counts for query r
#pragma unroll
    for (int r = 0; r < MR; ++r) {
        s[r] += __shfl_xor_sync(0xffffffffu, s[r], 1);
        s[r] += __shfl_xor_sync(0xffffffffu, s[r], 2);
        s[r] += __shfl_xor_sync(0xffffffffu, s[r], 4);
        s[r] = __fmul_rn(s[r], p.scale_log2);              // rounded by itself: the reference is such a product
        if (tail) {
            bool vis = t < C;
            if (!vis && t < c.r.L && r < nq) {
                const int i = (q0 + r) / p.w.group, j = t - C;
                vis = p.tree_mask ? (j < 32 * p.mask_words && ((__ldg(p.tree_mask + (size_t)(c.r.row0 + i) * p.mask_words + (j >> 5)) >> (j & 31)) & 1u))
                                  : j <= i;
            }
            if (!vis) s[r] = -INFINITY;
            seen[r] = __ballot_sync(0xffffffffu, vis);
        }
        float mx = s[r];
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        const float top = fmaxf(m[r], mx);
        const float ref = top == -INFINITY ? 0.0f : top;   // nothing seen yet: every weight is 0
        const float f = tree_ex2(m[r] - ref);
        const float pr = tree_ex2(s[r] - ref);
        l[r] = l[r] * f + pr;
#pragma unroll
        for (int j = 0; j < VPL; ++j) acc[r][j] *= f;
        m[r] = top;
        if (share == r) ps[r * kWarpKeys + lane / kKeyLanes] = pr;
    }
    __syncwarp();
    float v[kWarpKeys][VPL];
#pragma unroll
    for (int j = 0; j < kWarpKeys; ++j)
#pragma unroll
        for (int e = 0; e < VPL; ++e) v[j][e] = vs[j * DH + e];
#pragma unroll
    for (int r = 0; r < MR; ++r) {
        const float4 w4 = *reinterpret_cast<const float4*>(ps + r * kWarpKeys);
        const float wj[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
        for (int j = 0; j < kWarpKeys; ++j) {
            // a key that the query does not see contributes nothing whatever its value holds (0 * inf would be NaN)
            if (tail && !((seen[r] >> (kKeyLanes * j)) & 1u)) continue;
#pragma unroll
            for (int e = 0; e < VPL; ++e) acc[r][e] = fmaf(wj[j], v[j][e], acc[r][e]);
        }
    }
    __syncwarp();                                          // ps is written again by the next tile
}

template <int DH>
__global__ void __launch_bounds__(kSimtThreads, 2)
tree_attention_simt_kernel(SimtParams p) {
    using Cfg = SimtCfg<DH>;
    constexpr int VPL = DH / 32;
    extern __shared__ __align__(16) float sm[];
    __shared__ long long part[16];
    __shared__ TreeRun run;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    float* qs = sm + Cfg::kOffQ;
    float* ps = sm + Cfg::kOffP + warp * kSimtRows * kWarpKeys;
    float* acc_s = sm + Cfg::kOffAcc;
    float* m_s = sm + Cfg::kOffML;
    float* l_s = m_s + 8 * kSimtRows;
    int64_t* offs = reinterpret_cast<int64_t*>(sm + Cfg::kOffKeys);
    TreeTail* tails = reinterpret_cast<TreeTail*>(p.scratch);
    grid_dependency_wait();
    tree_find_run(p.w, part, &run);
    if (tid == 0) {
        tails[blockIdx.x].last_cta = -1;
        tree_front(p.scratch)[blockIdx.x] = run.begin < run.end && !run.at.item_begins();
    }
    if (run.begin >= run.end) return;

    TreeCursor c = run.at, ahead = run.at;
    bool split_front = !c.item_begins();                   // the first piece continues an item of an earlier CTA
    float m[kSimtRows], l[kSimtRows], acc[kSimtRows][VPL];
    const long long n_tiles = run.end - run.begin;
    // the places of a tile's keys are looked up a tile before it is requested
    long long asked = 0;                                   // tiles requested
    find_keys(p, ahead, offs);
    for (int k = 0; k < kSimtStages - 1; ++k) {
        __syncthreads();
        if (asked < n_tiles) {
            load_tile<DH>(p, offs + (k & 1) * kSimtKeys, sm + k * Cfg::kStageFloats);
            if (++asked < n_tiles) { ahead.next(p.w); find_keys(p, ahead, offs + ((k + 1) & 1) * kSimtKeys); }
        }
        cp_async_commit();
    }
    bool fresh = true;                                     // the next tile opens a piece
    int q0 = 0, nq = 0;
    int at = 0, fill = kSimtStages - 1;                    // stage of tile k, stage of the tile requested next
    for (long long k = 0; k < n_tiles; ++k) {
        if (fresh) {
            fresh = false;
            q0 = c.first_query(p.w);
            nq = c.queries(p.w);
            for (int i = tid; i < kSimtRows * DH; i += kSimtThreads) {
                const int r = i / DH, e = i - r * DH;
                float x = 0.0f;
                if (r < nq) {
                    const int tok = (q0 + r) / p.w.group, hg = q0 + r - tok * p.w.group;
                    x = __ldg(p.q + (int64_t)(c.r.row0 + tok) * p.q_stride + (int64_t)(c.h * p.w.group + hg) * DH + e);
                }
                qs[i] = x;
            }
#pragma unroll
            for (int r = 0; r < kSimtRows; ++r) {
                m[r] = -INFINITY; l[r] = 0.0f;
#pragma unroll
                for (int e = 0; e < VPL; ++e) acc[r][e] = 0.0f;
            }
        }
        cp_async_wait<kSimtStages - 2>();
        __syncthreads();                                   // tile k is there, and the tile before has been read by all
        if (asked < n_tiles) {
            load_tile<DH>(p, offs + (asked & 1) * kSimtKeys, sm + fill * Cfg::kStageFloats);
            if (++asked < n_tiles) { ahead.next(p.w); find_keys(p, ahead, offs + (asked & 1) * kSimtKeys); }
        }
        cp_async_commit();
        const float* stage = sm + at * Cfg::kStageFloats;
        if (++at == kSimtStages) at = 0;
        if (++fill == kSimtStages) fill = 0;
        if (nq == 1) tile_step<DH, 1>(p, c, q0, nq, stage, qs, ps, m, l, acc);
        else if (nq == 2) tile_step<DH, 2>(p, c, q0, nq, stage, qs, ps, m, l, acc);
        else if (nq <= 4) tile_step<DH, 4>(p, c, q0, nq, stage, qs, ps, m, l, acc);
        else tile_step<DH, 8>(p, c, q0, nq, stage, qs, ps, m, l, acc);
        const bool ends = c.item_ends();
        if (ends || k + 1 == n_tiles) {
            // join the warps
#pragma unroll
            for (int r = 0; r < kSimtRows; ++r) {
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], 8);
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], 16);
                if (lane == 0) { m_s[warp * kSimtRows + r] = m[r]; l_s[warp * kSimtRows + r] = l[r]; }
#pragma unroll
                for (int e = 0; e < VPL; ++e) acc_s[(warp * kSimtRows + r) * DH + lane * VPL + e] = acc[r][e];
            }
            __syncthreads();
            const bool whole = ends && !split_front;
            float* slot = tree_slot(p.scratch, split_front ? 2 * blockIdx.x : 2 * blockIdx.x + 1, kSimtRows, DH);
            if (warp < nq) {                               // warp r joins query r
                const int r = warp;
                float top = -INFINITY, sum = 0.0f, o[VPL];
#pragma unroll
                for (int e = 0; e < VPL; ++e) o[e] = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) if (l_s[w * kSimtRows + r] != 0.0f) top = fmaxf(top, m_s[w * kSimtRows + r]);
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    const float lw = l_s[w * kSimtRows + r];
                    if (lw == 0.0f) continue;
                    const float f = tree_ex2(m_s[w * kSimtRows + r] - top);
                    sum += lw * f;
#pragma unroll
                    for (int e = 0; e < VPL; ++e) o[e] = fmaf(acc_s[(w * kSimtRows + r) * DH + lane * VPL + e], f, o[e]);
                }
                if (whole) {
                    const int tok = (q0 + r) / p.w.group, hg = q0 + r - tok * p.w.group;
                    float* dst = p.out + (int64_t)(c.r.row0 + tok) * p.out_stride + (int64_t)(c.h * p.w.group + hg) * DH + lane * VPL;
#pragma unroll
                    for (int e = 0; e < VPL; ++e) dst[e] = sum == 0.0f ? 0.0f : o[e] / sum;
                } else {
                    if (lane == 0) { slot[r] = top; slot[kSimtRows + r] = sum; }
#pragma unroll
                    for (int e = 0; e < VPL; ++e) slot[2 * kSimtRows + r * DH + lane * VPL + e] = o[e];
                }
            }
            if (!ends && !split_front && tid == 0) {       // begins here, goes on in the next CTAs
                TreeTail t{};
                t.last_cta = run.tail_cta;
                t.queries = nq; t.row0 = c.r.row0; t.q0 = q0; t.h = c.h;
                tails[blockIdx.x] = t;
            }
            __syncthreads();
            split_front = false;
            fresh = true;
        }
        c.next(p.w);
    }
    cp_async_wait<0>();
}

template <int DH>
int simt_launch(const SimtParams& p, int grid, int combine_y, cudaStream_t s, bool dependent) {
    static DeviceOnce attr;
    if (!attr.done([] { return allow_smem(tree_attention_simt_kernel<DH>, SimtCfg<DH>::kSmemBytes); })) return ZOQAT_ERR_CUDA;
    if (launch_kernel(tree_attention_simt_kernel<DH>, dim3(grid), dim3(kSimtThreads), SimtCfg<DH>::kSmemBytes, s, dependent, p) != cudaSuccess)
        return ZOQAT_ERR_CUDA;
    count_launch();
    if (launch_kernel(tree_combine_kernel<float, DH>, dim3(grid, combine_y), dim3(256), 0, s, true, p.scratch, kSimtRows, p.w.group, p.out,
                      p.out_stride) != cudaSuccess)
        return ZOQAT_ERR_CUDA;
    count_launch();
    return ZOQAT_OK;
}

}  // namespace

int tree_grid() {
    int sms = 0, dev = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    return sms <= 0 || sms > kMaxTreeGrid / 2 ? kMaxTreeGrid / 2 : sms;
}

size_t tree_attention_scratch_bytes(int type, int d_head) {
    const int tile_rows = type == kTypeF32 ? kSimtRows : 256;
    return kTailBytes + 2 * (size_t)(type == kTypeF32 ? kMaxTreeGrid : kMaxTreeGrid / 2) * tree_slot_floats(tile_rows, d_head) * 4;
}

int launch_tree_attention_simt(const TreeAttnArgs& a, cudaStream_t s, bool dependent) {
    SimtParams p{};
    p.w = TreeWork{a.kv_len, a.row_start, a.block_table, a.batch, a.rows, a.cache.n_kv_heads, a.max_pages, a.cache.page_size,
                   a.n_heads / a.cache.n_kv_heads, kSimtRows, kSimtKeys, 4, a.err_flag};
    p.q = static_cast<const float*>(a.q); p.q_stride = a.q_stride; p.cache = a.cache;
    p.tree_mask = a.tree_mask; p.mask_words = a.mask_words;
    p.scale_log2 = (float)(1.4426950408889634 * (double)a.scale);
    p.out = static_cast<float*>(a.out); p.out_stride = a.out_stride; p.scratch = a.scratch;
    const int grid = 2 * tree_grid();                      // two CTAs per SM
    return a.cache.d_head == 64 ? simt_launch<64>(p, grid, kSimtRows, s, dependent) : simt_launch<128>(p, grid, kSimtRows, s, dependent);
}

}  // namespace zq
