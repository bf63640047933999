// What the two tensor-core attention kernels over a paged cache share: parameters, the 16-bit types, the warps that fill shared
// memory (K and V tiles by TMA, query tiles by plain loads), and the visibility of drafts.
#pragma once
#include "tree_attention.cuh"
#include "tc_ptx.cuh"

namespace zq {

constexpr int kKeys = 128;           // keys per tile
constexpr int kMaskWords = 4;        // words of a draft's mask that travel with its query tile (trees of up to 128 drafts)
constexpr float kTreeSlack = 8.0f;   // a reference may lag the maximum by up to 2^8
constexpr float kNoRef = -3.0e38f;   // reference of a query that has seen nothing: any score passes it

struct TcParams {
    TreeWork w;
    const void* q;
    int64_t q_stride;
    int box_keys;                // keys of one K / V box: a page, or 128 of a larger one
    int page_shift;              // log2 of the page size, or -1
    int page_units, units;       // a page's step and the end of the maps' outermost dimension, which counts heads through all pages
    int n_pages, mask_words;
    const uint32_t* tree_mask;
    float scale_log2;
    void* out;
    int64_t out_stride;
    uint8_t* scratch;
    const void* v;               // (for the rare repair of non-finite values)
    int64_t page_stride, slot_stride, head_stride;
    uint32_t smem_bytes;
};

template <typename T> struct HalfOps;
template <> struct HalfOps<__nv_bfloat16> {
    static constexpr uint32_t kFormat = 1;                       // operand format of the instruction descriptor
    static constexpr float kBias = 0.0f;                         // weights are scaled by 2^kBias
    static constexpr uint32_t kExpMask = 0x7F80u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi); return *reinterpret_cast<const uint32_t*>(&h); }
    static __device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }
};
template <> struct HalfOps<__half> {
    static constexpr uint32_t kFormat = 0;
    static constexpr float kBias = 7.0f;
    static constexpr uint32_t kExpMask = 0x7C00u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { const __half2 h = __floats2half2_rn(lo, hi); return *reinterpret_cast<const uint32_t*>(&h); }
    static __device__ __forceinline__ float value(__half x) { return __half2float(x); }
};

__device__ __forceinline__ void tmem_store32(uint32_t taddr, const uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
          "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
          "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}
__device__ __forceinline__ void load16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr) : "memory");
}
// The loads issued so far have arrived; v's values are not to be used above this point.
__device__ __forceinline__ void load16_wait(uint32_t (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :: "memory");
}
__device__ __forceinline__ void load32_wait(uint32_t (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]),
                   "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]),
                   "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
                 :: "memory");
}
// two products and sums in binary32 at once
__device__ __forceinline__ float2 tree_fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{ .reg .b64 x, y, z, w; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; fma.rn.f32x2 w, x, y, z; mov.b64 {%0, %1}, w; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 tree_add2(float2 a, float2 b) {
    float2 d;
    asm("{ .reg .b64 x, y, w; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 w, x, y; mov.b64 {%0, %1}, w; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ void store16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A score in base 2 against its reference, in two roundings: references are made from rounded products, so equal ones cancel
// exactly.  Fused, the product's rounding error stays in the exponent: 1 at scores of 2^24, 64 at 2^30, out of a weight's range, but at
// most 1/16 up to 2^20, where the kernels use the fused form.  tree_far: beyond that.
__device__ __forceinline__ float tree_shift(float s, float scale, float ref) { return __fsub_rn(__fmul_rn(s, scale), ref); }
__device__ __forceinline__ bool tree_far(float ref) { return fabsf(ref) > 1048576.0f && ref != kNoRef; }

// Bits of the 32 keys from k0 on that draft i sees.
__device__ __forceinline__ uint32_t visible_word(int k0, int C, int n, int i, const uint32_t* mask, int words) {
    const int rel = k0 - C;                                      // draft index of bit 0
    if (rel <= -32) return 0xFFFFFFFFu;
    const int shift = rel < 0 ? -rel : 0, j0 = rel < 0 ? 0 : rel;
    const uint32_t below = (1u << shift) - 1u;                   // cached keys (shift < 32)
    if (j0 >= n) return below;
    uint32_t d;
    if (mask) {
        const int wi = j0 >> 5;
        const uint32_t lo = wi < words ? __ldg(mask + wi) : 0u, hi = wi + 1 < words ? __ldg(mask + wi + 1) : 0u;
        d = __funnelshift_r(lo, hi, j0 & 31);
    } else {
        const int upto = i - j0 + 1;
        d = upto <= 0 ? 0u : (upto >= 32 ? 0xFFFFFFFFu : (1u << upto) - 1u);
    }
    if (n - j0 < 32) d &= (1u << (n - j0)) - 1u;
    return below | (d << shift);
}


// A K or V tile in shared memory: groups of 8 keys, [16 groups][DH / 64 halves][8 keys][128 bytes], 128-byte swizzle, so that one
// TMA box fetches all of a page's keys of a head.
template <int DH> __host__ __device__ constexpr int tree_group_bytes() { return DH / 64 * 1024; }

// K and V tiles, by a whole warp, in the order in which the products consume them: K(0), V(0), K(1), V(1), ..., or with K LEAD = 1
// tile ahead: K(0), K(1), V(0), K(2), V(1), ...
// Every lane fetches one page (or 128 keys of a larger one), and
// reads its entry of the block table two tiles ahead.
template <int DH, int NS, int LEAD>
__device__ __forceinline__ void tree_load_keys(const TcParams& p, const CUtensorMap* map_k, const CUtensorMap* map_v, const TreeRun* run,
                                               uint32_t ring, uint32_t full, uint32_t empty) {
    constexpr int kTileBytes = kKeys * DH * 2, kGroup = tree_group_bytes<DH>();
    const int lane = threadIdx.x & 31;
    const int n_box = kKeys / p.box_keys, n_tiles = (int)(run->end - run->begin);
    const uint32_t box_bytes = (uint32_t)(p.box_keys >> 3) * kGroup;
    TreeCursor c = run->at;
    uint32_t seq = 0;
    bool ok = true;
    struct Box { int page, group, h, live; bool mine; };         // page: as the table has it, looked at when the box is fetched
    auto look_up = [&](Box& x) {                                 // this lane's box of the cursor's tile
        const int key0 = c.kt * kKeys + lane * p.box_keys, left = c.r.L - c.kt * kKeys;
        x.h = c.h;
        x.live = left >= kKeys ? n_box : (left + p.box_keys - 1) / p.box_keys;
        x.mine = lane < x.live;
        if (!x.mine) return;
        const int idx = p.page_shift >= 0 ? key0 >> p.page_shift : key0 / p.w.page_size;
        x.group = (key0 - idx * p.w.page_size) >> 3;
        x.page = __ldg(p.w.block_table + (size_t)c.b * p.w.max_pages + idx);
    };
    auto fetch = [&](const CUtensorMap* map, const Box& x) -> bool {
        const int slot = seq % NS;
        if (!__all_sync(0xffffffffu, mbar_wait(empty + 8u * slot, ((seq / NS) & 1u) ^ 1u))) return false;
        if (lane == 0) mbar_arrive_expect_tx(full + 8u * slot, (uint32_t)x.live * box_bytes);
        __syncwarp();
        if (x.mine) {
            int unit = p.units;                                  // behind the map's end: zeros
            if (x.page >= 0 && x.page < p.n_pages) unit = x.page * p.page_units + x.h;
            else atomicExch(p.w.err_flag, kErrBadPage);
            tma_load_5d(ring + slot * kTileBytes + lane * box_bytes, map, full + 8u * slot, 0, 0, 0, x.group, unit);
        }
        ++seq;
        return true;
    };
    Box last{}, cur{}, next{}, after{};                          // last: the tile whose V is still to come
    look_up(cur);
    if (n_tiles > 1) { c.next(p.w); look_up(next); }
    for (int t = 0; t < n_tiles + LEAD && ok; ++t) {
        if (t < n_tiles && !fetch(map_k, cur)) { ok = false; break; }
        if (t + 2 < n_tiles) { c.next(p.w); look_up(after); }
        if (LEAD == 0) last = cur;
        if (t >= LEAD && !fetch(map_v, last)) { ok = false; break; }
        last = cur;
        cur = next;
        next = after;
    }
    if (!ok && lane == 0) atomicExch(p.w.err_flag, kErrTreeWait);
    // every load issued above has to land before the CTA may leave
    for (uint32_t k = seq > NS ? seq - NS : 0; k < seq; ++k)
        if (!mbar_wait(full + 8u * (k % NS), (k / NS) & 1u)) break;
}

// Query tiles, by THREADS threads (whole warps; `lane`: which of them), a piece ahead of the products: rows of 128 bytes, 128-byte
// swizzle, [half][NQ rows], BUFFERS buffers in turn.  Rows behind the tile's last query keep what they hold; their results are
// not used.  full counts one arrival per warp.  masks (may be NULL): [2][NQ][kMaskWords], the first words of the drafts' masks, draft by draft; done: four
// barriers, by piece modulo 4, after which a piece's masks are no longer read.
template <int DH, int NQ, int THREADS, int BUFFERS, typename T>
__device__ __forceinline__ void tree_load_queries(const TcParams& p, const TreeRun* run, uint8_t* q_tiles, uint32_t* masks, uint32_t done, uint32_t full,
                                                  uint32_t empty, int lane) {
    constexpr int kChunks = DH / 8, kTileBytes = NQ * DH * 2, kRowsPer = THREADS / kChunks, kMost = NQ >= 256 ? 16 : 8,
                  kFly = NQ / kRowsPer < kMost ? NQ / kRowsPer : kMost;
    const int ch = lane % kChunks;               // a thread copies its 16 bytes of every kRowsPer-th row, kFly rows in flight
    const int n_tiles = (int)(run->end - run->begin);
    TreeCursor c = run->at;
    uint32_t piece = 0;
    for (int t = 0; t < n_tiles; ++t, c.next(p.w)) {
        if (t != 0 && !c.item_begins()) continue;
        const uint32_t b = piece % BUFFERS;
        if (!__all_sync(0xffffffffu, mbar_wait(empty + 8u * b, ((piece / BUFFERS) & 1u) ^ 1u))) { atomicExch(p.w.err_flag, kErrTreeWait); return; }
        const int q0 = c.first_query(p.w), nq = c.queries(p.w);
        const T* base = static_cast<const T*>(p.q) + (int64_t)c.r.row0 * p.q_stride + (int64_t)c.h * p.w.group * DH + 8 * ch;
        uint8_t* dst = q_tiles + b * kTileBytes + (ch >> 3) * (NQ * 128);
        for (int r0 = lane / kChunks; r0 < nq; r0 += kFly * kRowsPer) {
            uint4 w[kFly];
#pragma unroll
            for (int u = 0; u < kFly; ++u) {
                const int r = r0 + u * kRowsPer;
                if (r < nq) {
                    const int tok = (q0 + r) / p.w.group, hg = q0 + r - tok * p.w.group;
                    w[u] = __ldg(reinterpret_cast<const uint4*>(base + (int64_t)tok * p.q_stride + (int64_t)hg * DH));
                }
            }
#pragma unroll
            for (int u = 0; u < kFly; ++u) {
                const int r = r0 + u * kRowsPer;
                if (r < nq) *reinterpret_cast<uint4*>(dst + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = w[u];
            }
        }
        if (masks && p.tree_mask) {
            const int tok0 = q0 / p.w.group, n_tok = (q0 + nq - 1) / p.w.group - tok0 + 1;
            uint32_t* to = masks + b * NQ * kMaskWords;
            const uint32_t old = piece - 2u;                     // the piece whose masks lie there
            if (piece >= 2 && !__all_sync(0xffffffffu, mbar_wait(done + 8u * (old & 3u), (old >> 2) & 1u))) { atomicExch(p.w.err_flag, kErrTreeWait); return; }
            for (int x = lane; x < n_tok * kMaskWords; x += THREADS) {
                const int i = x / kMaskWords, k = x % kMaskWords;
                to[x] = k < p.mask_words ? __ldg(p.tree_mask + (size_t)(c.r.row0 + tok0 + i) * p.mask_words + k) : 0u;
            }
        }
        fence_async_smem();
        __syncwarp();
        if ((lane & 31) == 0) mbar_arrive(full + 8u * b);
        ++piece;
    }
}

// The V tile's keys behind the request's end become zeros (what lies there is not the request's), and a draft's element that is
// not finite becomes zero as well: 0 * inf of a place some row does not see must not reach that row.  Such elements are added
// back at the end to the rows that do see them.  128 threads; true if this thread met one.
template <int DH, uint32_t kExpMask>
__device__ __forceinline__ bool tree_clean_values(uint8_t* v, int first_draft, int end, int thread) {
    bool met = false;
    for (int x = thread; x < (kKeys - first_draft) * (DH / 8); x += 128) {
        const int key = first_draft + x / (DH / 8), ch = x % (DH / 8);
        uint4* at = reinterpret_cast<uint4*>(v + (key >> 3) * tree_group_bytes<DH>() + (ch >> 3) * 1024 + (key & 7) * 128 + (((ch & 7) ^ (key & 7)) << 4));
        if (key >= end) { *at = make_uint4(0, 0, 0, 0); continue; }
        uint4 w = *at;
        uint32_t ww[4] = {w.x, w.y, w.z, w.w};
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if ((ww[e] & kExpMask) == kExpMask) { ww[e] &= 0xFFFF0000u; odd = true; }
            if (((ww[e] >> 16) & kExpMask) == kExpMask) { ww[e] &= 0x0000FFFFu; odd = true; }
        }
        if (odd) { *at = make_uint4(ww[0], ww[1], ww[2], ww[3]); met = true; }
    }
    fence_async_smem();
    return met;
}

// Where the key stands in the cache, or -1 (bad page).
__device__ __forceinline__ int64_t tree_value_offset(const TcParams& p, const TreeCursor& c, int key) {
    const int idx = key / p.w.page_size;
    const int pg = __ldg(p.w.block_table + (size_t)c.b * p.w.max_pages + idx);
    if (pg < 0 || pg >= p.n_pages) return -1;
    return pg * p.page_stride + (key - idx * p.w.page_size) * p.slot_stride + c.h * p.head_stride;
}

// few queries per key head: keys are the rows of the products (tree_attention_keys.cu); nq: queries per tile (16, 32, 64)
int launch_tree_keys(const TcParams& p, const CUtensorMap& map_k, const CUtensorMap& map_v, int dh, int type, int nq, int grid, cudaStream_t s, bool dependent);

}  // namespace zq
