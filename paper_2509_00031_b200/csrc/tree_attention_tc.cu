// Attention of drafted rows over a paged bf16 / fp16 cache on the tensor cores (tcgen05 / TMEM / TMA).
//
//   out[i, h] = sum_t softmax_t(scale q[i, h] . k[t, h / g]) v[t, h / g]      over the keys t < C cached before the step and
//                                                                            the drafts j (t = C + j) whose mask bit is set
//
// The queries that read one key head - every draft times the g heads of the group - share one 128-row tile, so each cached
// byte is fetched once per request, key head and 128 queries.  Up to about 100 queries per key head that fetch bounds the
// kernel (a tile of 128 keys is 64 KB, some 2800 cycles of an SM's share of the memory; its two products are 1024 cycles of
// the tensor pipe whatever the number of live rows); above, the tensor pipe and the exponentials do.
//
// One persistent CTA per SM, 12 warps; the key tiles of all requests are dealt out in equal runs (tree_attention.cuh):
//   warp 0      TMA: every lane fetches one page (a 64-column half of it) of a K or V tile into a ring of tiles; the lanes
//               read the block table themselves, one tile ahead.  Q tiles go into two buffers, a piece ahead.
//   warp 1      one thread issues the products: S = Q K^T into one of two TMEM score buffers, O += P V with P read from TMEM
//               and V as it lies in the page (keys along k, so no transposition).
//   warps 4-7, 8-11  two softmax groups take alternate tiles.  A thread owns a query row: it reads the tile's 128 scores, and
//               writes the weights, rounded to the cache's type, over them.  Each group has a reference, a sum and an output
//               accumulator of its own, so the groups need not agree on anything until the piece ends, when the two
//               results are joined.  The reference moves only when a row's maximum has grown by more than 2^8 since.
// Rounding: the products are exact in binary32 up to accumulation; the weights are rounded to 11 (fp16) or 8 (bf16) bits for
// the second product, the sums are formed from the unrounded weights, the output is rounded once.  fp16 weights are scaled by
// 2^7, which keeps small ones out of the subnormals; the largest is then 2^15.
// Masked values: a key behind the request's end is set to zero in the V tile before the product; a draft's V element that is
// not finite is set to zero as well and added again, at the end, to the rows that see the draft - so that 0 * inf of a
// masked place never reaches a row.
// Every wait is bounded and reports through *err_flag.
#include "tree_attention.cuh"
#include "tc_ptx.cuh"
#include "../../include/zoqat.h"

namespace zq {
namespace {

constexpr int kTcThreads = 384, kKeys = 128, kRows = 128;
constexpr float kRefSlack = 8.0f;

template <int DH> struct TcCfg {
    static constexpr int kTileBytes = kKeys * DH * 2;                       // one K, V or Q tile
    static constexpr int kStages = DH == 128 ? 5 : 10;
    static constexpr int kOffRing = 2 * kTileBytes;
    static constexpr int kOffX = kOffRing + kStages * kTileBytes;           // (reference, sum) of every row: [2 groups][128][2]
    static constexpr int kOffBar = kOffX + 2048;
    static constexpr int kOffMisc = kOffBar + (2 * kStages + 13) * 8;       // TMEM base, non-finite marks, run
    static constexpr int kUsedBytes = kOffMisc + 32 + 96 + (int)sizeof(TreeRun);
    static constexpr int kSmemBytes = kUsedBytes + 1024 > 232448 ? 232448 : kUsedBytes + 1024;
    static_assert(kUsedBytes <= 232448, "shared memory");
};

struct TcParams {
    TreeWork w;
    int q_unit, q_tokens;        // rows and drafts of one Q box
    int box_keys;                // keys of one K / V box: a page, or 128 of a larger one
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
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive_n(uint32_t bar, uint32_t n) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}

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

template <int DH, typename T>
__global__ void __launch_bounds__(kTcThreads, 1)
tree_attention_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                         const __grid_constant__ CUtensorMap map_v, const TcParams p) {
    using Cfg = TcCfg<DH>;
    using Ops = HalfOps<T>;
    constexpr int HALVES = DH / 64, NS = Cfg::kStages;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* const sp = smem_raw + (base - raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if ((base - raw) + (uint32_t)Cfg::kUsedBytes > p.smem_bytes) {           // uniform: nothing has been set up yet
        if (tid == 0) atomicExch(p.w.err_flag, kErrTreeWait);
        if (tid == 0) reinterpret_cast<TreeTail*>(p.scratch)[blockIdx.x].last_cta = -1;
        return;
    }
    const uint32_t bars = base + Cfg::kOffBar;
    auto ring_full = [&](int s) { return bars + 8u * s; };
    auto ring_empty = [&](int s) { return bars + 8u * (NS + s); };
    auto q_full = [&](int s) { return bars + 8u * (2 * NS + s); };
    auto q_empty = [&](int s) { return bars + 8u * (2 * NS + 2 + s); };
    auto s_full = [&](int g) { return bars + 8u * (2 * NS + 4 + g); };
    auto p_full = [&](int g) { return bars + 8u * (2 * NS + 6 + g); };
    auto o_full = [&](int g) { return bars + 8u * (2 * NS + 8 + g); };
    auto o_empty = [&](int g) { return bars + 8u * (2 * NS + 10 + g); };
    const uint32_t x_full = bars + 8u * (2 * NS + 12);
    volatile uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sp + Cfg::kOffMisc);
    volatile uint32_t* odd_piece = reinterpret_cast<uint32_t*>(sp + Cfg::kOffMisc + 8);   // [2]: piece + 1 with a non-finite draft value
    long long* part = reinterpret_cast<long long*>(sp + Cfg::kOffMisc + 32);
    TreeRun* run = reinterpret_cast<TreeRun*>(sp + Cfg::kOffMisc + 32 + 96);

    if (tid == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(ring_full(s), 1); mbar_init(ring_empty(s), 1); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(q_full(s), 1); mbar_init(q_empty(s), 1); mbar_init(s_full(s), 1); mbar_init(p_full(s), 4);
            mbar_init(o_full(s), 1); mbar_init(o_empty(s), 8);
            odd_piece[s] = 0;
        }
        mbar_init(x_full, 8);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_tmap(&map_q); prefetch_tmap(&map_k); prefetch_tmap(&map_v);
    }
    if (warp == 1) {
        tmem_alloc(base + Cfg::kOffMisc, 512);
        tmem_relinquish();
    }
    grid_dependency_wait();                    // lengths, queries and the drafts' keys come from the kernels before
    tree_find_run(p.w, part, run);
    if (tid == 0) reinterpret_cast<TreeTail*>(p.scratch)[blockIdx.x].last_cta = -1;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t tmem_s = tmem, tmem_o = tmem + 256u;          // S (then P) of group g at + 128 g, O of group g at + 128 g
    const int n_tiles = (int)(run->end - run->begin);

    if (warp == 0 && n_tiles > 0) {
        // ---------------- TMA producer: K(0), K(1), V(0), K(2), V(1), ..., the order in which the products consume them
        const int half = lane % HALVES, box = lane / HALVES;
        const int n_box = kKeys / p.box_keys;
        TreeCursor c = run->at;
        uint32_t seq = 0, piece = 0;
        bool ok = true;
        int page = 0, off = 0, prev_page = 0, prev_off = 0, prev_h = 0, prev_live = 0;
        bool prev_mine = false;
        auto look_up = [&](int& pg, int& of) -> bool {           // page and slot of this lane's box of the cursor's tile
            const int key0 = c.kt * kKeys + box * p.box_keys;
            if (box >= n_box || key0 >= c.r.L) return false;
            const int idx = key0 / p.w.page_size;
            of = key0 - idx * p.w.page_size;
            pg = __ldg(p.w.block_table + (size_t)c.b * p.w.max_pages + idx);
            if (pg < 0 || pg >= p.n_pages) { atomicExch(p.w.err_flag, kErrBadPage); pg = p.n_pages; }   // behind the map's end: zeros
            return true;
        };
        auto fetch = [&](const CUtensorMap* map, int h, int live, bool mine, int pg, int of) {
            const int slot = seq % NS;
            if (!__all_sync(0xffffffffu, mbar_wait(ring_empty(slot), ((seq / NS) & 1u) ^ 1u))) return false;
            if (lane == 0) mbar_arrive_expect_tx(ring_full(slot), (uint32_t)(live * HALVES * p.box_keys * 128));
            __syncwarp();
            if (mine) tma_load_4d(base + Cfg::kOffRing + slot * Cfg::kTileBytes + half * (kKeys * 128) + box * p.box_keys * 128, map,
                                  ring_full(slot), half * 64, of, h, pg);
            ++seq;
            return true;
        };
        bool mine = look_up(page, off);
        for (int t = 0; t <= n_tiles && ok; ++t) {
            int live = 0;
            if (t < n_tiles) {
                if (t == 0 || c.item_begins()) {                 // a piece begins: its queries
                    const int b = piece & 1u;
                    const int boxes = (c.queries(p.w) + p.q_unit - 1) / p.q_unit;
                    if (!__all_sync(0xffffffffu, mbar_wait(q_empty(b), ((piece >> 1) & 1u) ^ 1u))) { ok = false; break; }
                    if (lane == 0) mbar_arrive_expect_tx(q_full(b), (uint32_t)(boxes * HALVES * p.q_unit * 128));
                    __syncwarp();
                    if (box < boxes)
                        tma_load_3d(base + b * Cfg::kTileBytes + half * (kRows * 128) + box * p.q_unit * 128, &map_q, q_full(b), half * 64,
                                    c.h * p.w.group, c.r.row0 + c.first_query(p.w) / p.w.group + box * p.q_tokens);
                    ++piece;
                }
                live = min(n_box, (c.r.L - c.kt * kKeys + p.box_keys - 1) / p.box_keys);
                if (!fetch(&map_k, c.h, live, mine, page, off)) { ok = false; break; }
            }
            int next_page = 0, next_off = 0;
            bool next_mine = false;
            const int h = c.h;
            if (t + 1 < n_tiles) { c.next(p.w); next_mine = look_up(next_page, next_off); }   // the next tile's pages, before the wait below
            if (t > 0 && !fetch(&map_v, prev_h, prev_live, prev_mine, prev_page, prev_off)) { ok = false; break; }
            prev_page = page; prev_off = off; prev_h = h; prev_live = live; prev_mine = mine;
            page = next_page; off = next_off; mine = next_mine;
        }
        if (!ok && lane == 0) atomicExch(p.w.err_flag, kErrTreeWait);
        // every load issued above has to land before the CTA may leave: each slot's last tile has been consumed
        for (uint32_t k = seq > NS ? seq - NS : 0; k < seq; ++k)
            if (!mbar_wait(ring_full(k % NS), (k / NS) & 1u)) break;
    } else if (warp == 1 && n_tiles > 0) {
        // ---------------- MMA issuer
        if (lane == 0) {
            constexpr uint32_t kIdesc = (1u << 4) | (Ops::kFormat << 7) | (Ops::kFormat << 10) | ((uint32_t)(kRows >> 4) << 24);
            constexpr uint32_t kIdescS = kIdesc | ((uint32_t)(kKeys >> 3) << 17);
            constexpr uint32_t kIdescO = kIdesc | (1u << 16) | ((uint32_t)(DH >> 3) << 17);      // bit 16: B is MN-major
            TreeCursor c = run->at;                    // of the next S
            uint32_t seq = 0, piece = 0;
            bool ok = true, ends = false;              // ends: the piece of the last S issued ends with it
            auto issue_s = [&](int t) -> bool {
                const int slot = seq % NS, g = t & 1;
                if (t == 0 || c.item_begins()) {
                    if (!mbar_wait(q_full(piece & 1u), (piece >> 1) & 1u)) return false;
                    ++piece;
                }
                const uint32_t b = (piece - 1) & 1u;
                if (!mbar_wait(ring_full(slot), (seq / NS) & 1u)) return false;
                tc_fence_after();
                const uint32_t qa = base + b * Cfg::kTileBytes, ka = base + Cfg::kOffRing + slot * Cfg::kTileBytes;
#pragma unroll
                for (int k = 0; k < DH / 16; ++k) {
                    const uint64_t da = smem_desc_sw128(qa + (k >> 2) * (kRows * 128)) + (uint64_t)(2 * (k & 3));
                    const uint64_t db = smem_desc_sw128(ka + (k >> 2) * (kKeys * 128)) + (uint64_t)(2 * (k & 3));
                    umma_bf16(tmem_s + 128u * g, da, db, kIdescS, k > 0 ? 1u : 0u);
                }
                umma_commit(s_full(g));
                umma_commit(ring_empty(slot));
                ends = c.item_ends();
                if (ends || t == n_tiles - 1) umma_commit(q_empty(b));
                ++seq;
                c.next(p.w);
                return true;
            };
            uint32_t uses0 = 0, uses1 = 0;             // pieces that have used each output accumulator
            int rel = 0;                               // tile within its piece
            if (!issue_s(0)) ok = false;
            for (int t = 0; t < n_tiles && ok; ++t) {
                const int g = t & 1;
                const bool last = ends;
                if (t + 1 < n_tiles && !issue_s(t + 1)) { ok = false; break; }
                if (rel < 2) {                         // the accumulator's last piece has been read out
                    uint32_t& uses = g ? uses1 : uses0;
                    if (uses > 0 && !mbar_wait(o_empty(g), (uses - 1) & 1u)) { ok = false; break; }
                    ++uses;
                }
                const int slot = seq % NS;
                if (!mbar_wait(p_full(g), (t >> 1) & 1u) || !mbar_wait(ring_full(slot), (seq / NS) & 1u)) { ok = false; break; }
                tc_fence_after();
                const uint32_t va = base + Cfg::kOffRing + slot * Cfg::kTileBytes;
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k)
                    umma_f16_ta(tmem_o + 128u * g, tmem_s + 128u * g + 8u * k, smem_desc_sw128_mn(va + k * 2048, kKeys * 128), kIdescO,
                                (rel >= 2 || k > 0) ? 1u : 0u);
                umma_commit(o_full(g));
                umma_commit(ring_empty(slot));
                ++seq;
                rel = last ? 0 : rel + 1;
            }
            if (!ok) atomicExch(p.w.err_flag, kErrTreeWait);
        }
    } else if (warp >= 4 && n_tiles > 0) {
        // ---------------- softmax groups
        const int g = (warp >> 2) - 1;                 // 0: even tiles, 1: odd tiles
        const int quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t t_lane = (uint32_t)(quarter * 32) << 16;
        const uint32_t ts = tmem_s + 128u * g + t_lane;
        float2* const xch = reinterpret_cast<float2*>(sp + Cfg::kOffX);      // [2][128]
        TreeCursor c = run->at;
        bool split_front = !c.item_begins();
        float m_ref = -INFINITY, l_run = 0.0f;
        int first = 0, kt_first = 0;                   // first tile of the piece, its key tile
        uint32_t piece = 0, merges = 0;
        int q0 = 0, nq = 0, tok = 0, hg = 0;
        const uint32_t* mask = nullptr;
        bool ok = true;
        auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)) != 0; };
        for (int t = 0; t < n_tiles && ok; ++t) {
            if (t == first) {
                q0 = c.first_query(p.w); nq = c.queries(p.w); kt_first = c.kt;
                tok = (q0 + row) / p.w.group;
                hg = q0 + row - tok * p.w.group;
                if (p.tree_mask && row < nq) mask = p.tree_mask + (size_t)(c.r.row0 + tok) * p.mask_words;
                m_ref = -INFINITY; l_run = 0.0f;
            }
            const int C = c.r.L - c.r.n;
            const bool warp_live = quarter * 32 < nq;
            if ((t & 1) == g) {
                if (!wait_all(s_full(g), (t >> 1) & 1u)) { ok = false; break; }
                tc_fence_after();
                const bool tail = (c.kt + 1) * kKeys > C;
                if (tail) {
                    // the V tile's rows behind the end become zeros; a draft's non-finite element becomes zero and is marked
                    const uint32_t vseq = t == n_tiles - 1 ? 2u * n_tiles - 1u : 2u * t + 2u;
                    if (!wait_all(ring_full(vseq % NS), (vseq / NS) & 1u)) { ok = false; break; }
                    uint8_t* v = sp + Cfg::kOffRing + (vseq % NS) * Cfg::kTileBytes;
                    const int k_lo = max(C - c.kt * kKeys, 0), k_end = c.r.L - c.kt * kKeys;   // first draft, first key behind the end
                    for (int x = tid & 127; x < (kKeys - k_lo) * (DH / 8); x += 128) {
                        const int key = k_lo + x / (DH / 8), ch = x % (DH / 8);
                        uint4* at = reinterpret_cast<uint4*>(v + (ch >> 3) * (kKeys * 128) + key * 128 + (((ch & 7) ^ (key & 7)) << 4));
                        if (key >= k_end) { *at = make_uint4(0, 0, 0, 0); continue; }
                        uint4 w = *at;
                        uint32_t ww[4] = {w.x, w.y, w.z, w.w};
                        bool odd = false;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if ((ww[e] & Ops::kExpMask) == Ops::kExpMask) { ww[e] &= 0xFFFF0000u; odd = true; }
                            if (((ww[e] >> 16) & Ops::kExpMask) == Ops::kExpMask) { ww[e] &= 0x0000FFFFu; odd = true; }
                        }
                        if (odd) { *at = make_uint4(ww[0], ww[1], ww[2], ww[3]); odd_piece[piece & 1u] = piece + 1; }
                    }
                    fence_async_smem();
                }
                if (warp_live) {
                    uint32_t s[4][32];
#pragma unroll
                    for (int q = 0; q < 4; ++q) tmem_ld32(ts + 32u * q, s[q]);
                    tmem_ld_wait();
                    if (tail) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t vis = row < nq ? visible_word(c.kt * kKeys + 32 * q, C, c.r.n, tok, mask, p.mask_words) : 0u;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((vis >> e) & 1u)) s[q][e] = __float_as_uint(-INFINITY);
                        }
                    }
                    float mx;
                    {
                        float t8[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) t8[e] = __uint_as_float(s[0][e]);
#pragma unroll
                        for (int q = 0; q < 4; ++q)
#pragma unroll
                            for (int e = q == 0 ? 8 : 0; e < 32; ++e) t8[e & 7] = fmaxf(t8[e & 7], __uint_as_float(s[q][e]));
                        mx = fmaxf(fmaxf(fmaxf(t8[0], t8[1]), fmaxf(t8[2], t8[3])), fmaxf(fmaxf(t8[4], t8[5]), fmaxf(t8[6], t8[7])));
                    }
                    mx = mx * p.scale_log2 - Ops::kBias;         // weights 2^(score - reference): the largest is 2^kBias .. 2^(kBias + 8)
                    if (t - first < 2) {
                        m_ref = mx;                              // the group's first tile of the piece
                    } else {
                        const bool grow = row < nq && mx > m_ref + kRefSlack;
                        if (__any_sync(0xffffffffu, grow)) {
                            // rare: rescale the rows' outputs, after the group's previous product has completed
                            if (!wait_all(o_full(g), ((t >> 1) & 1u) ^ 1u)) { ok = false; break; }
                            tc_fence_after();
                            const float f = grow ? tree_ex2(m_ref - mx) : 1.0f;
#pragma unroll 1
                            for (int c0 = 0; c0 < DH; c0 += 32) {
                                uint32_t o[32];
                                const uint32_t at = tmem_o + 128u * g + t_lane + (uint32_t)c0;
                                tmem_ld32(at, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_store32(at, o);
                            }
                            tmem_store_wait();
                            l_run *= f;
                            if (grow) m_ref = mx;
                        }
                    }
                    const float ref = m_ref == -INFINITY ? 0.0f : m_ref;     // nothing seen yet: every weight is 0
                    float sum4[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        uint32_t w[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const float a = tree_ex2(fmaf(__uint_as_float(s[2 * hf + (e >> 4)][2 * (e & 15)]), p.scale_log2, -ref));
                            const float b = tree_ex2(fmaf(__uint_as_float(s[2 * hf + (e >> 4)][2 * (e & 15) + 1]), p.scale_log2, -ref));
                            sum4[(2 * e) & 3] += a;
                            sum4[(2 * e + 1) & 3] += b;
                            w[e] = Ops::pack(a, b);
                        }
                        tmem_store32(ts + 32u * hf, w);
                    }
                    tmem_store_wait();
                    l_run += (sum4[0] + sum4[1]) + (sum4[2] + sum4[3]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(g));
            }
            const bool item_ends = c.item_ends();
            if (item_ends || t == n_tiles - 1) {
                const bool both = t > first;                     // the piece used both groups
                const bool whole = item_ends && !split_front;
                if (both || (t & 1) == g) {
                    const int mine = (t & 1) == g ? t : t - 1;   // this group's last tile
                    if (!wait_all(o_full(g), (mine >> 1) & 1u)) { ok = false; break; }
                    float m = m_ref, l = l_run, fa = 1.0f, fb = 0.0f;        // factors of O of group 0 and 1 (both) or of the own O
                    if (both) {
                        xch[g * kRows + row] = make_float2(m_ref, l_run);
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(x_full);
                        if (!wait_all(x_full, merges & 1u)) { ok = false; break; }
                        ++merges;
                        const float2 a = xch[row], b = xch[kRows + row];
                        m = fmaxf(a.x, b.x);
                        const float ref = m == -INFINITY ? 0.0f : m;
                        fa = tree_ex2(a.x - ref);
                        fb = tree_ex2(b.x - ref);
                        l = a.y * fa + b.y * fb;
                    }
                    tc_fence_after();
                    const bool repair = odd_piece[piece & 1u] == piece + 1;
                    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                    const int head = c.h * p.w.group + hg;
                    T* dst = static_cast<T*>(p.out) + (int64_t)(c.r.row0 + tok) * p.out_stride + (int64_t)head * DH;
                    float* slot = tree_slot(p.scratch, split_front ? 2 * blockIdx.x : 2 * blockIdx.x + 1, p.w.tile_rows, DH);
                    const int col0 = both ? g * (DH / 2) : 0, cols = both ? DH / 2 : DH;
                    if (warp_live) {
#pragma unroll 1
                        for (int c0 = col0; c0 < col0 + cols; c0 += 32) {
                            float o[32];
                            {
                                uint32_t oa[32], ob[32];
                                if (both) {
                                    tmem_ld32(tmem_o + t_lane + (uint32_t)c0, oa);
                                    tmem_ld32(tmem_o + 128u + t_lane + (uint32_t)c0, ob);
                                    tmem_ld_wait();
#pragma unroll
                                    for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(oa[e]) * fa + __uint_as_float(ob[e]) * fb;
                                } else {
                                    tmem_ld32(tmem_o + 128u * g + t_lane + (uint32_t)c0, oa);
                                    tmem_ld_wait();
#pragma unroll
                                    for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(oa[e]);
                                }
                            }
                            if (row < nq) {
                                if (repair) {                    // non-finite values of drafts this row sees, within the piece's tiles
                                    for (int j = 0; j < c.r.n; ++j) {
                                        const int key = C + j, kt = key / kKeys;
                                        if (kt < kt_first || kt > c.kt) continue;
                                        if (!(visible_word(key, C, c.r.n, tok, mask, p.mask_words) & 1u)) continue;
                                        const int idx = key / p.w.page_size;
                                        const int pg = __ldg(p.w.block_table + (size_t)c.b * p.w.max_pages + idx);
                                        if (pg < 0 || pg >= p.n_pages) continue;
                                        const T* v = static_cast<const T*>(p.v) + pg * p.page_stride + (key - idx * p.w.page_size) * p.slot_stride +
                                                     c.h * p.head_stride + c0;
#pragma unroll
                                        for (int e = 0; e < 32; ++e) {
                                            const float x = Ops::value(v[e]);
                                            if (!isfinite(x)) o[e] += x;
                                        }
                                    }
                                }
                                if (whole) {
#pragma unroll
                                    for (int e = 0; e < 32; e += 8) {
                                        uint4 w;
                                        w.x = Ops::pack(o[e] * inv, o[e + 1] * inv); w.y = Ops::pack(o[e + 2] * inv, o[e + 3] * inv);
                                        w.z = Ops::pack(o[e + 4] * inv, o[e + 5] * inv); w.w = Ops::pack(o[e + 6] * inv, o[e + 7] * inv);
                                        *reinterpret_cast<uint4*>(dst + c0 + e) = w;
                                    }
                                } else {
                                    float* po = slot + 2 * p.w.tile_rows + (size_t)row * DH + c0;
#pragma unroll
                                    for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(po + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                                }
                            }
                        }
                        if (!whole && row < nq && col0 == 0) { slot[row] = m; slot[p.w.tile_rows + row] = l; }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if (both) { mbar_arrive(o_empty(0)); mbar_arrive(o_empty(1)); }
                        else mbar_arrive_n(o_empty(g), 2);
                    }
                }
                if (!item_ends && !split_front && tid == 128) {  // begins here, goes on in the next CTAs
                    TreeTail tl{};
                    tl.last_cta = tree_cta_of(run->end + (c.r.n_kt - 1 - c.kt) - 1, run->total, run->ctas);
                    tl.queries = nq; tl.row0 = c.r.row0; tl.q0 = q0; tl.h = c.h;
                    reinterpret_cast<TreeTail*>(p.scratch)[blockIdx.x] = tl;
                }
                split_front = false;
                first = t + 1;
                ++piece;
            }
            c.next(p.w);
        }
        if (!ok && lane == 0) atomicExch(p.w.err_flag, kErrTreeWait);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn tree_encode_fn() {
    static const EncodeTiledFn fn = [] {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess)
            ptr = nullptr;
        return reinterpret_cast<EncodeTiledFn>(ptr);
    }();
    return fn;
}

bool encode(CUtensorMap* map, int type, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    EncodeTiledFn fn = tree_encode_fn();
    if (!fn) return false;
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, type == kTypeBf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank, const_cast<void*>(base),
              dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DH, typename T>
int tc_launch(const TreeAttnArgs& a, cudaStream_t s, bool dependent) {
    using Cfg = TcCfg<DH>;
    TcParams p{};
    const int group = a.n_heads / a.cache.n_kv_heads;
    int gcd8 = group % 8 == 0 ? 8 : (group % 4 == 0 ? 4 : (group % 2 == 0 ? 2 : 1));
    p.q_tokens = 8 / gcd8;
    p.q_unit = group * p.q_tokens;                     // a multiple of 8: the boxes of a Q tile keep the swizzle's rows aligned
    if (p.q_unit > kRows) return ZOQAT_ERR_UNSUPPORTED;
    p.w = TreeWork{a.kv_len, a.row_start, a.block_table, a.batch, a.rows, a.n_heads, a.cache.n_kv_heads, a.max_pages, a.cache.page_size,
                   group, kRows / p.q_unit * p.q_unit, kKeys, a.err_flag};
    p.box_keys = a.cache.page_size < kKeys ? a.cache.page_size : kKeys;
    p.n_pages = a.cache.n_pages; p.mask_words = a.mask_words; p.tree_mask = a.tree_mask;
    p.scale_log2 = (float)(1.4426950408889634 * (double)a.scale);
    p.out = a.out; p.out_stride = a.out_stride; p.scratch = a.scratch;
    p.v = a.cache.v; p.page_stride = a.cache.page_stride; p.slot_stride = a.cache.slot_stride; p.head_stride = a.cache.head_stride;
    p.smem_bytes = Cfg::kSmemBytes;
    alignas(64) CUtensorMap map_q, map_k, map_v;
    const cuuint64_t qd[3] = {(cuuint64_t)DH, (cuuint64_t)a.n_heads, (cuuint64_t)a.rows};
    const cuuint64_t qst[2] = {(cuuint64_t)DH * 2, (cuuint64_t)a.q_stride * 2};
    const cuuint32_t qb[3] = {64, (cuuint32_t)group, (cuuint32_t)p.q_tokens};
    const cuuint64_t kd[4] = {(cuuint64_t)DH, (cuuint64_t)a.cache.page_size, (cuuint64_t)a.cache.n_kv_heads, (cuuint64_t)a.cache.n_pages};
    const cuuint64_t kst[3] = {(cuuint64_t)a.cache.slot_stride * 2, (cuuint64_t)a.cache.head_stride * 2, (cuuint64_t)a.cache.page_stride * 2};
    const cuuint32_t kb[4] = {64, (cuuint32_t)p.box_keys, 1, 1};
    if (!encode(&map_q, a.cache.type, a.q, 3, qd, qst, qb) || !encode(&map_k, a.cache.type, a.cache.k, 4, kd, kst, kb) ||
        !encode(&map_v, a.cache.type, a.cache.v, 4, kd, kst, kb))
        return ZOQAT_ERR_CUDA;
    static DeviceOnce attr;
    if (attr.first() &&
        cudaFuncSetAttribute(tree_attention_tc_kernel<DH, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes) != cudaSuccess) {
        attr.retry();
        return ZOQAT_ERR_CUDA;
    }
    const int grid = tree_grid();
    if (launch_kernel(tree_attention_tc_kernel<DH, T>, dim3(grid), dim3(kTcThreads), Cfg::kSmemBytes, s, dependent, map_q, map_k, map_v, p) != cudaSuccess)
        return ZOQAT_ERR_CUDA;
    count_launch();
    if (launch_kernel(tree_combine_kernel<T, DH>, dim3(grid, 16), dim3(256), 0, s, true, p.scratch, p.w.tile_rows, group, a.n_heads,
                      static_cast<T*>(a.out), a.out_stride) != cudaSuccess)
        return ZOQAT_ERR_CUDA;
    count_launch();
    return ZOQAT_OK;
}

}  // namespace

int launch_tree_attention_tc(const TreeAttnArgs& a, cudaStream_t s, bool dependent) {
    if (a.cache.type == kTypeBf16)
        return a.cache.d_head == 64 ? tc_launch<64, __nv_bfloat16>(a, s, dependent) : tc_launch<128, __nv_bfloat16>(a, s, dependent);
    return a.cache.d_head == 64 ? tc_launch<64, __half>(a, s, dependent) : tc_launch<128, __half>(a, s, dependent);
}

}  // namespace zq
