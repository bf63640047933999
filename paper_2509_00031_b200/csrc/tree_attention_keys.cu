// Attention of drafted rows over a paged bf16 / fp16 cache on the tensor cores, for few queries per key head (up to 64 in a tile:
// single tokens, small trees).  The keys are the rows of both products:
//
//   S^T[key, query] = K Q^T            one thread per key reads its N scores from TMEM
//   P^T[key, query] = 2^(S^T - ref)    rounded to the cache's type, to shared memory
//   O^T[column, query] += V^T P^T      V as it lies in the page
//   l[query] += sum_key P^T            N = 16: every thread adds up its keys' weights, the threads' sums are joined when a piece
//                                      ends; else by a third product with a matrix of ones, which leaves the sums in every TMEM
//                                      lane.  The tensor pipe spends some 45 cycles on a product of 128 x N x 16 however small N
//                                      is, and at d_head 64 the third product is 8 of a tile's 20 (16 x 32 heads of 8192 keys in
//                                      pages laid out head by head: 225 us with it, 187 without); joining 32 sums costs short pieces more than that
//                                      (64 requests of 300 keys, 4 drafts of 4 heads: 51 us with it, 64 without).
//
// so the softmax costs 128 * N exponentials per tile of 128 keys, spread over all four schedulers, whatever the tile's number of
// live queries N = 16, 32 or 64 is; with queries as rows (tree_attention_tc.cu) a single query would cost a whole warp's 128
// exponentials on one scheduler, and the kernel would be bound by them instead of by reading the cache.  What bounds it is
// the cache: 64 KB a tile at d_head 128, some 2800 cycles of an SM's share of the memory, against 700 to 1100 of the tensor pipe
// and 8 N of the exponential units.  Measured, bf16, one token for each of 16 x 32 heads, replayed from a graph: 6.5 TB/s at 8192 keys
// and d_head 128, 5.7 at 2048; at d_head 64 5.6 and 3.7 with pages laid out head by head, 4.0 and 3.6 slot by slot (a head's keys are then
// rows of 128 bytes 4 KB apart).  What short contexts lose is fixed: 4 us until the first scores, 3 for the last piece's
// output, 4 for the launch that joins split pieces, and up to 8 between the first and the last CTA to finish.
//
// One persistent CTA per SM, 12 warps; the key tiles of all requests are dealt out in equal runs (tree_attention.cuh):
//   warp 0      K and V tiles by TMA into a ring; warp 3: query tiles into two buffers, a piece ahead
//   warps 1, 2  one thread issues the scores, one tile ahead, another the products with the weights
//   warps 4-7   softmax.  All keys of a query share one reference; it moves only when a score passes it by more than 2^8, which
//               the warps tell one another once per tile, after computing the weights as if it did not.
//               Maxima over the keys are formed only when a piece begins or a reference moves (or lies beyond 2^20).
//   warps 8-11  outputs of a finished piece, from the other one of two TMEM accumulators, while the next piece runs
// Rounding, masked values and bounded waits as in tree_attention_tc.cu, but for the sums, which are those of the rounded weights.
// Accesses to tensor memory are by whole warps: where lanes may have gone apart before (masks, tails, repairs) they meet first.
#include "tree_attention_tc.cuh"
#include "../../include/zoqat.h"

namespace zq {
namespace {

constexpr int kKeyThreads = 384;

template <int DH, int N, class W> struct KeyCfg {
    static constexpr int kTileBytes = kKeys * DH * 2;
    static constexpr int kQBytes = N * DH * 2, kPBytes = N * kKeys * 2;
    static constexpr bool kAdd = N == 16;                                   // the threads add up the weights
    static constexpr int kSumBytes = kAdd ? 4 * N * 16 : 0;                 // [4 pieces][N][4 warps] floats
    static constexpr int kFixed = 2 * kQBytes + 3 * kPBytes + N * 16 + 8 * N * 4 + 2 * N * kMaskWords * 4 + kSumBytes + 1024;
    static constexpr int kFit = (232448 - kFixed) / kTileBytes;
    // an even number: K tiles (odd places of the sequence) and V tiles (even places) then have slots of their own, so that each
    // slot is consumed by one thread in order and no one can wait for a phase before the one ahead of it has completed
    static constexpr int kStages = kFit > 10 ? 10 : kFit / 2 * 2;
    static constexpr int kOffQ = kStages * kTileBytes;
    static constexpr int kOffP = kOffQ + 2 * kQBytes;
    static constexpr int kOffRed = kOffP + 3 * kPBytes;                     // [N][4 warps] floats
    static constexpr int kOffRef = kOffRed + N * 16;                        // [2][N] floats, then [4][N]: those of the last pieces, then [2][N] stand-ins
    static constexpr int kOffMask = kOffRef + 8 * N * 4;                    // [2][N drafts][kMaskWords]
    static constexpr int kOffSum = kOffMask + 2 * N * kMaskWords * 4;
    static constexpr int kOffBar = kOffSum + kSumBytes;
    // ring full, ring empty; q full, q empty, s full, s empty (2 each), p full, o full (3 each), o empty, out full (2), piece done (4)
    static constexpr int kBars = 2 * kStages + 18 + 4;
    static constexpr int kOffMisc = kOffBar + kBars * 8;
    static constexpr int kUsedBytes = kOffMisc + 32 + 192 + (int)sizeof(TreeRunT<W>);
    static constexpr int kSmemBytes = kUsedBytes + 1024 > 232448 ? 232448 : kUsedBytes + 1024;
    static_assert(kUsedBytes <= 232448 && kStages >= 4 && sizeof(PrefixScan) <= kStages * kTileBytes, "shared memory");
};

// f over the warp's 32 lanes of v[i], for 16 values at once: lanes 2 i and 2 i + 1 return that of v[i].
template <typename F>
__device__ __forceinline__ float join16(float (&v)[16], F f) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 8; h >= 1; h >>= 1) {
        const bool up = lane & (2 * h);
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const float keep = up ? v[i + h] : v[i], give = up ? v[i] : v[i + h];
            v[i] = f(keep, __shfl_xor_sync(0xffffffffu, give, 2 * h));
        }
    }
    return f(v[0], __shfl_xor_sync(0xffffffffu, v[0], 1));
}

// Shared-memory descriptor of the weights: query-major cores of 8 queries x 8 keys (128 bytes), no swizzle; the next 8 keys
// 128 bytes further, the next 8 queries 128 keys * 16 bytes.
__device__ __forceinline__ uint64_t smem_desc_weights(uint32_t saddr) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(128 >> 4) << 16;
    d |= (uint64_t)((kKeys * 16) >> 4) << 32;
    d |= (uint64_t)1 << 46;
    return d;
}

// eight columns of all 32 lanes
__device__ __forceinline__ void store8(uint32_t taddr, uint32_t v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %1, %1, %1, %1, %1, %1, %1};" ::"r"(taddr), "r"(v) : "memory");
}

template <int DH, int N, typename T, class W>
__global__ void __launch_bounds__(kKeyThreads, 1)
tree_attention_keys_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const TcParamsT<W> p) {
    using Cfg = KeyCfg<DH, N, W>;
    using Ops = HalfOps<T>;
    constexpr int NS = Cfg::kStages;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* const sp = smem_raw + (base - raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if ((base - raw) + (uint32_t)Cfg::kUsedBytes > p.smem_bytes) {           // uniform: nothing has been set up yet
        if (tid == 0) atomicExch(p.w.err_flag, kErrTreeWait);
        if (tid == 0) tree_announce<W>(p.scratch, false);
        return;
    }
    const uint32_t bars = base + Cfg::kOffBar;
    auto ring_full = [&](int s) { return bars + 8u * s; };
    auto ring_empty = [&](int s) { return bars + 8u * (NS + s); };
    auto q_full = [&](int s) { return bars + 8u * (2 * NS + s); };
    auto q_empty = [&](int s) { return bars + 8u * (2 * NS + 2 + s); };
    auto s_full = [&](int b) { return bars + 8u * (2 * NS + 4 + b); };
    auto s_empty = [&](int b) { return bars + 8u * (2 * NS + 6 + b); };
    auto p_full = [&](int b) { return bars + 8u * (2 * NS + 8 + b); };
    auto o_full = [&](int b) { return bars + 8u * (2 * NS + 11 + b); };      // the products of a tile (mod 3, as the weights' buffers) have completed
    auto o_empty = [&](int b) { return bars + 8u * (2 * NS + 14 + b); };     // the output of a piece (by its parity) has been read
    auto out_full = [&](int b) { return bars + 8u * (2 * NS + 16 + b); };    // every product of a piece (by its parity) has completed
    auto piece_done = [&](int i) { return bars + 8u * (2 * NS + 18 + i); };  // the softmax warps are through with a piece (mod 4)
    volatile uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sp + Cfg::kOffMisc);
    volatile uint32_t* odd_piece = reinterpret_cast<uint32_t*>(sp + Cfg::kOffMisc + 16);    // [4]: piece + 1 with a non-finite draft value
    float* const refs = reinterpret_cast<float*>(sp + Cfg::kOffRef);
    long long* part = reinterpret_cast<long long*>(sp + Cfg::kOffMisc + 32);
    TreeRunT<W>* run = reinterpret_cast<TreeRunT<W>*>(sp + Cfg::kOffMisc + 32 + 192);

    if (tid < Cfg::kBars) {
        const int i = tid - 2 * NS;              // one barrier a thread
        const bool four = (i >= 6 && i < 11) || i == 14 || i == 15 || i >= 18;       // s empty, p full, o empty, piece done
        mbar_init(bars + 8u * tid, four ? 4 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < 4) odd_piece[tid] = 0;
    if (tid == 64) { prefetch_tmap(&map_k); prefetch_tmap(&map_v); }
    if (warp == 1) {
        __syncwarp();
        tmem_alloc(base + Cfg::kOffMisc, 512);
        tmem_relinquish();
    }
    tree_start(p.w, part, run, sp);            // lengths, queries and the drafts' keys come from the kernels before
    if (tid == 0) tree_announce<W>(p.scratch, run->begin < run->end && !run->at.item_begins());
    if (W::kPrefix) fence_async_smem();        // the scan lay where tiles will
    const uint32_t tmem = *tmem_slot;          // (allocated before the barriers in tree_find_run)
    if (!Cfg::kAdd && warp >= 4 && warp < 8) { // the matrix of ones: 16 keys' worth, the same for every step
        tc_fence_after();
        __syncwarp();
        store8(tmem + 6u * N + ((uint32_t)((warp & 3) * 32) << 16), Ops::pack(1.0f, 1.0f));
        tmem_store_wait();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_s = tmem, tmem_o = tmem + 2u * N, tmem_l = tmem + 4u * N, tmem_1 = tmem + 6u * N;   // scores of a tile by parity, outputs and sums of a piece by parity, ones
    const int n_tiles = (int)(run->end - run->begin);
    constexpr uint32_t kIdesc = (1u << 4) | (Ops::kFormat << 7) | (Ops::kFormat << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);

    if (warp == 0 && n_tiles > 0) {
        tree_load_keys<DH, NS, 1>(p, &map_k, &map_v, run, base, ring_full(0), ring_empty(0));
    } else if (warp == 3 && n_tiles > 0) {
        tree_load_queries<DH, N, 32, 2, T>(p, run, sp + Cfg::kOffQ, reinterpret_cast<uint32_t*>(sp + Cfg::kOffMask), piece_done(0), q_full(0), q_empty(0), lane);
    } else if (warp == 1 && n_tiles > 0) {
        // ---------------- the scores: S^T of the next tile as soon as its buffer has been read
        if (lane == 0) {
            TreeCursorT<W> c = run->at;
            uint32_t piece = 0, b = 0;
            bool ok = true;
            for (int t = 0; t < n_tiles; ++t, c.next(p.w)) {
                const uint32_t seq = t == 0 ? 0u : 2u * t - 1u;
                const int slot = seq % NS, g = t & 1;
                if (t == 0 || c.item_begins()) {
                    b = piece & 1u;
                    if (!mbar_poll(q_full(b), (piece >> 1) & 1u)) { ok = false; break; }
                    ++piece;
                }
                if (!mbar_poll(s_empty(g), ((t >> 1) & 1u) ^ 1u) || !mbar_poll(ring_full(slot), (seq / NS) & 1u)) { ok = false; break; }
                tc_fence_after();
                const uint32_t qa = base + Cfg::kOffQ + b * Cfg::kQBytes, ka = base + slot * Cfg::kTileBytes;
#pragma unroll
                for (int k = 0; k < DH / 16; ++k) {
                    const uint64_t da = smem_desc_sw128(ka + (k >> 2) * 1024, tree_group_bytes<DH>()) + (uint64_t)(2 * (k & 3));
                    const uint64_t db = smem_desc_sw128(qa + (k >> 2) * (N * 128)) + (uint64_t)(2 * (k & 3));
                    umma_bf16(tmem_s + (uint32_t)(g * N), da, db, kIdesc, k > 0 ? 1u : 0u);
                }
                umma_commit(s_full(g));
                umma_commit(ring_empty(slot));
                if (c.item_ends() || t == n_tiles - 1) umma_commit(q_empty(b));
            }
            if (!ok) atomicExch(p.w.err_flag, kErrTreeWait);
        }
    } else if (warp == 2 && n_tiles > 0) {
        // ---------------- the outputs and sums: a thread of its own, so that waiting for weights holds no scores back
        if (lane == 0) {
            constexpr uint32_t kIdescL = kIdesc | (1u << 16), kIdescO = kIdescL | (1u << 15);   // V^T (15) and P^T (16) run along their rows, not along the keys
            TreeCursorT<W> c = run->at;
            uint32_t piece = 0;
            bool ok = true, first = true;              // first: the tile opens its piece
            uint32_t g = 0, round = 0;                 // buffer of the weights: t % 3, t / 3
            for (int t = 0; t < n_tiles; ++t, c.next(p.w)) {
                const uint32_t seq = t == n_tiles - 1 ? 2u * n_tiles - 1u : 2u * t + 2u, b = piece & 1u;
                const int slot = seq % NS;
                if (first && piece >= 2 && !mbar_poll(o_empty(b), ((piece >> 1) & 1u) ^ 1u)) { ok = false; break; }
                if (!mbar_poll(p_full(g), round & 1u) || !mbar_poll(ring_full(slot), (seq / NS) & 1u)) { ok = false; break; }
                tc_fence_after();
                const uint32_t va = base + slot * Cfg::kTileBytes, pa = base + Cfg::kOffP + g * Cfg::kPBytes;
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k)
                    // (at d_head 64 the rows behind 64 repeat the tile: their results are not read)
                    umma_bf16(tmem_o + b * N, smem_desc_sw128_mn(va + k * 2 * tree_group_bytes<DH>(), DH == 128 ? 1024 : 0, tree_group_bytes<DH>()), smem_desc_weights(pa + k * 256), kIdescO,
                              (!first || k > 0) ? 1u : 0u);
                umma_commit(ring_empty(slot));
#pragma unroll
                for (int k = 0; k < kKeys / 16 && !Cfg::kAdd; ++k)
                    umma_f16_ta(tmem_l + b * N, tmem_1, smem_desc_weights(pa + k * 256), kIdescL, (!first || k > 0) ? 1u : 0u);
                umma_commit(o_full(g));
                if (++g == 3) { g = 0; ++round; }
                first = c.item_ends();
                if (first || t == n_tiles - 1) { umma_commit(out_full(b)); ++piece; }
            }
            if (!ok) atomicExch(p.w.err_flag, kErrTreeWait);
        }
    } else if (warp >= 4 && warp < 8 && n_tiles > 0) {
        // ---------------- softmax: thread = key of the tile
        const int quarter = warp & 3, me = quarter * 32 + lane;
        const uint32_t t_lane = (uint32_t)(quarter * 32) << 16;
        float* const red = reinterpret_cast<float*>(sp + Cfg::kOffRed);
        TreeCursorT<W> c = run->at;
        bool ok = true, opens = true;
        int q0 = 0, nq = 0;
        float sums[Cfg::kAdd ? N : 1] = {};                      // of this thread's weights
        auto add = [&](int n, uint32_t w) {                      // queries n, n + 1
            const T* x = reinterpret_cast<const T*>(&w);
            sums[Cfg::kAdd ? n : 0] += Ops::value(x[0]);
            sums[Cfg::kAdd ? n + 1 : 0] += Ops::value(x[1]);
        };
        uint32_t piece = 0, cur = 0;                             // cur: which copy of the references is in use
        uint32_t pb = 0, round = 0;                              // buffer of the weights: t % 3, t / 3
        // A wait that ran out ends nothing here: the four warps go on to meet at the same places, without waiting for or signalling
        // anyone else.
        auto await = [&](uint32_t bar, uint32_t parity) { if (ok) ok = __all_sync(0xffffffffu, mbar_poll(bar, parity)) != 0; };
        auto meet = [] {
            __syncwarp();
            asm volatile("barrier.cta.sync 1, 128;" ::: "memory");
        };
        auto any_of = [](bool mine) -> bool {                    // of the four warps
            uint32_t any;
            __syncwarp();
            asm volatile("{ .reg .pred p, q; setp.ne.u32 p, %1, 0; barrier.cta.red.or.pred q, 1, 128, p; selp.u32 %0, 1, 0, q; }"
                         : "=r"(any) : "r"((uint32_t)mine) : "memory");
            return any != 0;
        };
        for (int t = 0; t < n_tiles; ++t) {
            const int buf = t & 1;
            if (opens) { q0 = c.first_query(p.w); nq = c.queries(p.w); }
            const int C = c.r.L - c.r.drafts();
            const uint32_t s_at = tmem_s + (uint32_t)(buf * N) + t_lane;
            await(s_full(buf), (t >> 1) & 1u);
            uint64_t vis = ~0ull;                                // queries that see this key
            const bool tail = (c.kt + 1) * kKeys > C;            // drafts in the tile, or its end
            if (tail) {
                const int key = c.kt * kKeys + me, j = key - C;
                if (key >= C) {
                    vis = 0;
                    if (key < c.r.L) {
                        const int tok0 = q0 / p.w.group, n_tok = (q0 + nq - 1) / p.w.group - tok0 + 1;
                        // (the masks came with the queries of this piece, whose scores have been seen: they are there)
                        const uint32_t* near = reinterpret_cast<const uint32_t*>(sp + Cfg::kOffMask) + (piece & 1u) * N * kMaskWords + (j >> 5);
                        for (int i = 0; i < n_tok; ++i) {
                            const int tok = tok0 + i, at = tok * p.w.group - q0;               // the draft's first query, from the tile's start
                            uint32_t sees = j <= tok;
                            if (p.tree_mask) {
                                sees = 0;
                                if (j < 32 * kMaskWords) sees = near[i * kMaskWords] >> (j & 31);
                                else if (j < 32 * p.mask_words) sees = __ldg(p.tree_mask + (size_t)(c.r.row0 + tok) * p.mask_words + (j >> 5)) >> (j & 31);
                            }
                            if (!(sees & 1u)) continue;
                            const int lo = max(at, 0), hi = min(at + p.w.group, N);
                            vis |= (hi - lo >= 64 ? ~0ull : ((1ull << (hi - lo)) - 1ull)) << lo;
                        }
                    }
                }
            }
            // Where the tile ends its piece, or holds drafts, the products of two tiles ago have run.  They belong to piece P - 2 or
            // a later one, whose first product waited for the outputs of piece P - 4: what is kept by piece modulo 4 (references, sums,
            // marks, the phase of piece_done) may be written.  A piece ends with its item, in a tile with drafts (a shared prefix: in any),
            // or with the run.
            if (t >= 2 && (tail || (W::kPrefix && c.item_ends()) || t == n_tiles - 1)) await(o_full(pb == 2 ? 0 : pb + 1), (pb == 2 ? round : round - 1u) & 1u);
            if (tail) {
                // (the V tile's slot was last used at least two tiles ago: only this tile's phase is open)
                const uint32_t vseq = t == n_tiles - 1 ? 2u * n_tiles - 1u : 2u * t + 2u;
                await(ring_full(vseq % NS), (vseq / NS) & 1u);
                if (tree_clean_values<DH, Ops::kExpMask>(sp + (vseq % NS) * Cfg::kTileBytes, max(C - c.kt * kKeys, 0), c.r.L - c.kt * kKeys, me))
                    odd_piece[piece & 3u] = piece + 1;
            }
            tc_fence_after();
            // Queries in chunks; those without a live query are left out (their columns of P and O hold anything, a column of the
            // products depends on its own column only).  The chunks are a loop on purpose: unrolled for 64 queries the steady
            // state no longer fits the schedulers' instruction caches (measured: 20 cycles per query and tile instead of 8).
            // P^T goes into the buffer that the products three tiles ago have read
            if (round > 0) await(o_full(pb), (round & 1u) ^ 1u);
            uint8_t* const pt = sp + Cfg::kOffP + pb * Cfg::kPBytes + me * 16;
            bool move = opens;
            if (!opens) {
                // the weights as if no reference moved; whether one does, the warps then tell one another
                constexpr int CH = N == 16 ? 1 : 2;              // chunks of 16 or 32
                const float4* ref4 = reinterpret_cast<const float4*>(refs + (6 + cur) * N);
                float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                uint32_t w[2 * CH][4];
#pragma unroll 1
                for (int n0 = 0; n0 < nq; n0 += 16 * CH) {       // (once where the threads add up)
                    uint32_t s[CH][16];
                    __syncwarp();
#pragma unroll
                    for (int k = 0; k < CH; ++k) load16(s_at + (uint32_t)(n0 + 16 * k), s[k]);
                    float4 r[4 * CH];
#pragma unroll
                    for (int i = 0; i < 4 * CH; ++i) r[i] = ref4[(n0 >> 2) + i];
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 4 * CH; ++i) {
                        const float ref[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t& x = s[i >> 2][4 * (i & 3) + e];
                            x = __float_as_uint(fmaf(__uint_as_float(x), p.scale_log2, -ref[e]));
                        }
                    }
                    if (vis != ~0ull) {
                        const uint32_t seen = (uint32_t)(vis >> n0);
#pragma unroll
                        for (int e = 0; e < 16 * CH; ++e)
                            if (!((seen >> e) & 1u)) s[e >> 4][e & 15] = __float_as_uint(-INFINITY);
                    }
                    uint8_t* at = pt + (n0 >> 3) * (kKeys * 16);
#pragma unroll
                    for (int k = 0; k < 2 * CH; ++k) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float a = __uint_as_float(s[k >> 1][8 * (k & 1) + 2 * e]), b = __uint_as_float(s[k >> 1][8 * (k & 1) + 2 * e + 1]);
                            top4[e] = fmaxf(top4[e], fmaxf(a, b));
                            w[k][e] = Ops::pack(tree_ex2(a), tree_ex2(b));
                        }
                        *reinterpret_cast<uint4*>(at + k * (kKeys * 16)) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
                    }
                }
                const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
                move = any_of(top > Ops::kBias + kTreeSlack);
                if (Cfg::kAdd && !move) {
#pragma unroll
                    for (int k = 0; k < 2 * CH; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) add(8 * k + 2 * e, w[k][e]);
                }
            }
            if (move) {
                // maxima over the keys, new references, outputs and sums brought to them (rare: chunk by chunk, few registers)
#pragma unroll 1
                for (int k = 0; 16 * k < nq; ++k) {
                    const uint32_t seen = (uint32_t)(vis >> (16 * k));
                    uint32_t s[16];
                    __syncwarp();
                    load16(s_at + 16u * k, s);
                    tmem_ld_wait();
                    float v[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = (seen >> e) & 1u ? __uint_as_float(s[e]) * p.scale_log2 : -INFINITY;
                    const float r = join16(v, [](float a, float b) { return fmaxf(a, b); });
                    if (!(lane & 1)) red[(16 * k + (lane >> 1)) * 4 + quarter] = r;
                }
                meet();
                const float* old_ref = refs + cur * N;
                float* new_ref = refs + (cur ^ 1u) * N;
                if (me < N) {
                    const float4 r = *reinterpret_cast<const float4*>(red + me * 4);
                    const float top = fmaxf(fmaxf(r.x, r.y), fmaxf(r.z, r.w)) - Ops::kBias;
                    const float ref = me < nq ? fmaxf(top, opens ? kNoRef : old_ref[me]) : INFINITY; // columns without a query: weight 0
                    new_ref[me] = ref;
                    // a far reference needs rounded products (tree_shift): its stand-in has every tile with a key for the query come here
                    refs[(6 + (cur ^ 1u)) * N + me] = me < nq && tree_far(ref) ? kNoRef : ref;
                }
                meet();
                if (!opens) {
                    // the products before (buffer pb - 1, a round earlier where that is 2)
                    await(o_full(pb ? pb - 1 : 2), (pb ? round : round - 1u) & 1u);
                    tc_fence_after();
#pragma unroll 1
                    for (int n0 = 0; n0 < nq; n0 += 16) {
                        uint32_t o[16], l[16];
                        const uint32_t at = (uint32_t)((piece & 1u) * N + n0) + t_lane;
                        __syncwarp();
                        load16(tmem_o + at, o);
                        if (!Cfg::kAdd) load16(tmem_l + at, l);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float f = tree_ex2(old_ref[n0 + e] - new_ref[n0 + e]);
                            o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            if (!Cfg::kAdd) l[e] = __float_as_uint(__uint_as_float(l[e]) * f);
                        }
                        store16(tmem_o + at, o);
                        if (!Cfg::kAdd) store16(tmem_l + at, l);
                    }
                    tmem_store_wait();
                }
                const float4* moved = reinterpret_cast<const float4*>(new_ref);
                if (Cfg::kAdd && opens) {
#pragma unroll
                    for (int n = 0; n < N; ++n) sums[n] = 0.0f;
                } else if (Cfg::kAdd) {
#pragma unroll
                    for (int n = 0; n < N; ++n) sums[n] *= tree_ex2(old_ref[n] - new_ref[n]);       // (anything in columns without a query)
                }
#pragma unroll 1
                for (int k = 0; 16 * k < nq; ++k) {
                    const uint32_t seen = (uint32_t)(vis >> (16 * k));
                    uint32_t s[16], w[8];
                    __syncwarp();
                    load16(s_at + 16u * k, s);
                    tmem_ld_wait();
#pragma unroll
                    for (int e4 = 0; e4 < 4; ++e4) {
                        const float4 r = moved[4 * k + e4];
                        const float ref[4] = {r.x, r.y, r.z, r.w};
                        float v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            v[e] = tree_ex2((seen >> (4 * e4 + e)) & 1u ? tree_shift(__uint_as_float(s[4 * e4 + e]), p.scale_log2, ref[e]) : -INFINITY);
                        w[2 * e4] = Ops::pack(v[0], v[1]);
                        w[2 * e4 + 1] = Ops::pack(v[2], v[3]);
                    }
                    *reinterpret_cast<uint4*>(pt + (2 * k) * (kKeys * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
                    *reinterpret_cast<uint4*>(pt + (2 * k + 1) * (kKeys * 16)) = make_uint4(w[4], w[5], w[6], w[7]);
                    if (Cfg::kAdd) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) add(2 * i, w[i]);
                    }
                }
                cur ^= 1u;
            }
            fence_async_smem();
            tc_fence_before();
            __syncwarp();
            if (ok && lane == 0) { mbar_arrive(s_empty(buf)); mbar_arrive(p_full(pb)); }
            if (++pb == 3) { pb = 0; ++round; }
            opens = c.item_ends();
            if (opens || t == n_tiles - 1) {
                if (me < N) refs[(2 + (piece & 3u)) * N + me] = refs[cur * N + me];        // (a warp behind may still read the copy in use)
                if (Cfg::kAdd) {
                    float* const to = reinterpret_cast<float*>(sp + Cfg::kOffSum) + (piece & 3u) * (4 * N);
#pragma unroll
                    for (int k = 0; k < N / 16; ++k) {
                        float v[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = sums[Cfg::kAdd ? 16 * k + e : 0];
                        const float r = join16(v, [](float a, float b) { return a + b; });
                        if (!(lane & 1)) to[(16 * k + (lane >> 1)) * 4 + quarter] = r;
                    }
                }
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(piece_done(piece & 3u));
                ++piece;
            }
            c.next(p.w);
        }
        if (!ok && lane == 0) atomicExch(p.w.err_flag, kErrTreeWait);
    } else if (warp >= 8 && n_tiles > 0) {
        // ---------------- outputs of a piece: thread = column of d_head
        const int quarter = warp & 3, me = quarter * 32 + lane;
        const uint32_t t_lane = (uint32_t)(quarter * 32) << 16;
        TreeCursorT<W> c = run->at;
        bool split_front = !c.item_begins(), ok = true;
        uint32_t piece = 0;
        int kt_first = c.kt;
        auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)) != 0; };
        for (int t = 0; t < n_tiles && ok; ++t) {
            const bool item_ends = c.item_ends();
            if (item_ends || t == n_tiles - 1) {
                const int q0 = c.first_query(p.w), nq = c.queries(p.w), C = c.r.L - c.r.drafts();
                const bool whole = item_ends && !split_front;
                if (!wait_all(piece_done(piece & 3u), (piece >> 2) & 1u) || !wait_all(out_full(piece & 1u), (piece >> 1) & 1u)) { ok = false; break; }
                tc_fence_after();
                const bool repair = odd_piece[piece & 3u] == piece + 1;
                float* slot = tree_slot(p.scratch, split_front ? 2 * blockIdx.x : 2 * blockIdx.x + 1, N, DH);
                const float* ref = refs + (2 + (piece & 3u)) * N;
                int tok = q0 / p.w.group, hg = q0 - tok * p.w.group;
                T* dst = static_cast<T*>(p.out) + (int64_t)(c.r.row0 + tok) * p.out_stride + (int64_t)(c.h * p.w.group + hg) * DH + me;
#pragma unroll 1
                for (int n0 = 0; n0 < nq; n0 += 16) {
                    uint32_t o[16], l[16];
                    const uint32_t at = (uint32_t)((piece & 1u) * N + n0) + t_lane;
                    __syncwarp();
                    load16(tmem_o + at, o);
                    if (Cfg::kAdd) {
                        const float4* of = reinterpret_cast<const float4*>(sp + Cfg::kOffSum) + (piece & 3u) * N + n0;
#pragma unroll
                        for (int e = 0; e < 16; ++e) { const float4 x = of[e]; l[e] = __float_as_uint((x.x + x.y) + (x.z + x.w)); }
                    } else {
                        load16(tmem_l + at, l);
                    }
                    tmem_ld_wait();
                    if (repair) {                                // what the non-finite values of drafts add to this column
                        uint32_t last = 0xFFFFFFFFu;
                        float odd = 0.0f;
#pragma unroll 1
                        for (int e = 0; e < 16 && n0 + e < nq; ++e) {
                            const uint32_t tk = (uint32_t)((q0 + n0 + e) / p.w.group);
                            if (tk != last) {
                                last = tk;
                                odd = 0.0f;
                                const uint32_t* mask = p.tree_mask ? p.tree_mask + (size_t)(c.r.row0 + tk) * p.mask_words : nullptr;
                                for (int j = 0; j < c.r.n && me < DH; ++j) {
                                    const int key = C + j, kt = key / kKeys;
                                    if (kt < kt_first || kt > c.kt || !(visible_word(key, C, c.r.n, (int)tk, mask, p.mask_words) & 1u)) continue;
                                    const int64_t off = tree_value_offset(p, c, key);
                                    if (off < 0) continue;
                                    const float v = Ops::value(static_cast<const T*>(p.v)[off + me]);
                                    if (!isfinite(v)) odd += v;
                                }
                            }
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (i == e) o[i] = __float_as_uint(__uint_as_float(o[i]) + odd);
                        }
                    }
                    if (W::kPrefix && whole && me < DH) {
                        if constexpr (W::kPrefix) {
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if (n0 + e < nq) {
                                    float* to = p.w.partial + prefix_query(p.w, c.r, q0 + n0 + e, c.h) * (DH + 4);
                                    to[me] = __uint_as_float(o[e]);
                                    if (me == 0) { to[DH] = ref[n0 + e]; to[DH + 1] = __uint_as_float(l[e]); }
                                }
                        }
                    } else if (!W::kPrefix && whole) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float sum = __uint_as_float(l[e]), x = __uint_as_float(o[e]) * (1.0f / sum);
                            if (n0 + e < nq && me < DH) *dst = tree_round<T>(sum == 0.0f ? 0.0f : x);
                            dst += DH;
                            if (++hg == p.w.group) { hg = 0; dst += p.out_stride - (int64_t)p.w.group * DH; }
                        }
                    } else if (me < DH) {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (n0 + e < nq) {
                                slot[2 * N + (size_t)(n0 + e) * DH + me] = __uint_as_float(o[e]);
                                if (me == 0) { slot[n0 + e] = ref[n0 + e]; slot[N + n0 + e] = __uint_as_float(l[e]); }
                            }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(o_empty(piece & 1u));
                if constexpr (W::kPrefix) {
                    if (!split_front && me < nq)
                        p.w.entries[prefix_query(p.w, c.r, q0 + me, c.h)] = item_ends ? make_int2(0, -1) : make_int2((int)blockIdx.x | run->tail_cta << 16, me);
                } else if (!item_ends && !split_front && me == 0) {     // begins here, goes on in the next CTAs
                    TreeTail tl{};
                    tl.last_cta = run->tail_cta;
                    tl.queries = nq; tl.row0 = c.r.row0; tl.q0 = q0; tl.h = c.h;
                    reinterpret_cast<TreeTail*>(p.scratch)[blockIdx.x] = tl;
                }
                split_front = false;
                ++piece;
            }
            c.next(p.w);
            kt_first = item_ends ? c.kt : kt_first;
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
    tree_finish(p.w);
}

template <int DH, int N, typename T, class W>
int keys_launch(const TcParamsT<W>& p, const CUtensorMap& map_k, const CUtensorMap& map_v, int grid, cudaStream_t s, bool dependent) {
    using Cfg = KeyCfg<DH, N, W>;
    static DeviceOnce attr;
    if (!attr.done([] { return allow_smem(tree_attention_keys_kernel<DH, N, T, W>, Cfg::kSmemBytes); })) return ZOQAT_ERR_CUDA;
    TcParamsT<W> q = p;
    q.smem_bytes = Cfg::kSmemBytes;
    return launch_kernel(tree_attention_keys_kernel<DH, N, T, W>, dim3(grid), dim3(kKeyThreads), Cfg::kSmemBytes, s, dependent, map_k, map_v, q) == cudaSuccess
               ? ZOQAT_OK : ZOQAT_ERR_CUDA;
}

}  // namespace

template <class W>
int launch_tree_keys(const TcParamsT<W>& p, const CUtensorMap& map_k, const CUtensorMap& map_v, int dh, int type, int nq, int grid, cudaStream_t s, bool dependent) {
#define ZQ_KEYS(DH, T) \
    return nq == 16 ? keys_launch<DH, 16, T>(p, map_k, map_v, grid, s, dependent) \
                    : (nq == 32 ? keys_launch<DH, 32, T>(p, map_k, map_v, grid, s, dependent) : keys_launch<DH, 64, T>(p, map_k, map_v, grid, s, dependent))
    if (type == kTypeBf16) { if (dh == 64) { ZQ_KEYS(64, __nv_bfloat16); } ZQ_KEYS(128, __nv_bfloat16); }
    if (dh == 64) { ZQ_KEYS(64, __half); }
    ZQ_KEYS(128, __half);
#undef ZQ_KEYS
}
template int launch_tree_keys(const TcParamsT<TreeWork>&, const CUtensorMap&, const CUtensorMap&, int, int, int, int, cudaStream_t, bool);
template int launch_tree_keys(const TcParamsT<PrefixWork>&, const CUtensorMap&, const CUtensorMap&, int, int, int, int, cudaStream_t, bool);

}  // namespace zq
