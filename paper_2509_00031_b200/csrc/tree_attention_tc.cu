// Attention of drafted rows over a paged bf16 / fp16 cache on the tensor cores (tcgen05 / TMEM / TMA).
//
//   out[i, h] = sum_t softmax_t(scale q[i, h] . k[t, h / g]) v[t, h / g]      over the keys t < C cached before the step and
//                                                                            the drafts j (t = C + j) whose mask bit is set
//
// This file: many queries per key head (wide trees, grouped heads); the host sends fewer to tree_attention_keys.cu.  The queries
// that read one key head - every draft times the g heads of the group - share row tiles of 256, so each cached byte is fetched once
// per request, key head and 256 queries.  For 256 queries a tile of 128 keys at d_head 128 costs 2048 cycles of the tensor pipe
// and 2048 of the exponential unit against some 2800 of an SM's share of the memory; measured 5040 over a whole call (4 contexts of
// 65536 keys), 4350 of them in a traced copy's steady state: a group's weights, then its two products of some 700 cycles each, half
// hidden behind the other group's.  4 contexts of 60-120 thousand keys, 64 drafts of 4 heads: 434 us a call as long as the clock stays near
// 1.9 GHz (up to a hundred calls), 500 in longer loops, which the 1 kW power limit holds at 1.6 GHz.  The other forms below were timed in
// the short way.  (Two tiles of 128 queries apart: 540, the second reads the keys again long after they have left L2.)
//
// One persistent CTA per SM, 12 warps; the key tiles of all requests are dealt out in equal runs (tree_attention.cuh):
//   warp 0      K and V tiles by TMA into a ring; warp 3: the query tile of the next piece
//   warps 4-7, 8-11  two softmax groups, each for 128 of the queries.  A thread owns a query row: it reads the tile's 128 scores
//               from TMEM twice, for the maximum and for the weights, and writes the weights, rounded to the cache's type, over
//               the scores.  Where a row's maximum has grown by more than 2^8 its reference moves, and its outputs with it.
//   warp 1      one thread issues the products of both groups by turns: O += P V with P from TMEM and V as it lies in the page
//               (keys along k, so no transposition), then S = Q K^T of the group's next tile, while the other group forms its
//               weights.  (A thread per group: the tensor pipe then serves both at once, the groups fall into step and nothing
//               is hidden, 503 us; a thread for S, one for PV, P in shared memory: 447.)
// A tile of up to 128 queries leaves the second group idle.  P from TMEM because shared memory feeds 128 bytes a cycle: the
// products alone take 192 KB per tile of 256 queries (P from shared memory: 256, and 64 more to write it), the tiles' arrival
// 64, and its place holds two more stages of the ring.
// Rounding: the products are exact in binary32 up to accumulation; the weights are rounded to 11 (fp16) or 8 (bf16) bits for
// the second product, the sums are formed from the unrounded weights, the output is rounded once.  fp16 weights are scaled by
// 2^7, which keeps small ones out of the subnormals; the largest is then 2^15.
// Masked values: a key behind the request's end is set to zero in the V tile before the product; a draft's V element that is
// not finite is set to zero as well and added again, at the end, to the rows that see the draft - so that 0 * inf of a
// masked place never reaches a row.
// Every wait is bounded and reports through *err_flag.
#include "tree_attention_tc.cuh"
#include "../../include/zoqat.h"

namespace zq {
namespace {

constexpr int kTcThreads = 384, kRows = 128, kTileRows = 2 * kRows;     // rows per group, rows per tile

template <bool V> struct FarScores { static constexpr bool value = V; };

template <int DH> struct TcCfg {
    static constexpr int kTileBytes = kKeys * DH * 2;                       // one K or V tile
    static constexpr int kStages = DH == 128 ? 5 : 8;
    static constexpr int kOffRing = kTileRows * DH * 2;                     // the query tile comes first
    static constexpr int kOffBar = kOffRing + kStages * kTileBytes;
    static constexpr int kBars = 2 * kStages + 10;
    static constexpr int kOffMisc = kOffBar + kBars * 8;                    // TMEM base, non-finite marks, run
    static constexpr int kUsedBytes = kOffMisc + 32 + 192 + (int)sizeof(TreeRun);
    static constexpr int kSmemBytes = kUsedBytes + 1024 > 232448 ? 232448 : kUsedBytes + 1024;
    static_assert(kUsedBytes <= 232448, "shared memory");
};

template <int DH, typename T>
__global__ void __launch_bounds__(kTcThreads, 1)
tree_attention_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const TcParams p) {
    using Cfg = TcCfg<DH>;
    using Ops = HalfOps<T>;
    constexpr int NS = Cfg::kStages;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* const sp = smem_raw + (base - raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if ((base - raw) + (uint32_t)Cfg::kUsedBytes > p.smem_bytes) {           // uniform: nothing has been set up yet
        if (tid == 0) atomicExch(p.w.err_flag, kErrTreeWait);
        if (tid == 0) {
            reinterpret_cast<TreeTail*>(p.scratch)[blockIdx.x].last_cta = -1;
            tree_front(p.scratch)[blockIdx.x] = 0;
        }
        return;
    }
    const uint32_t bars = base + Cfg::kOffBar;
    auto ring_full = [&](int s) { return bars + 8u * s; };
    auto ring_empty = [&](int s) { return bars + 8u * (NS + s); };
    const uint32_t q_full = bars + 8u * (2 * NS), q_empty = q_full + 8u;
    auto s_full = [&](int g) { return bars + 8u * (2 * NS + 2 + g); };
    auto p_full = [&](int g) { return bars + 8u * (2 * NS + 4 + g); };
    auto o_full = [&](int g) { return bars + 8u * (2 * NS + 6 + g); };
    auto o_empty = [&](int g) { return bars + 8u * (2 * NS + 8 + g); };
    volatile uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sp + Cfg::kOffMisc);
    // [4], by piece: piece + 1 with a non-finite draft value.  No product of piece P before both groups have read the outputs of
    // piece P - 2, and scores of piece P follow the first product of piece P - 1: whoever marks piece P, piece P - 4 has been read.
    volatile uint32_t* odd_piece = reinterpret_cast<uint32_t*>(sp + Cfg::kOffMisc + 8);
    long long* part = reinterpret_cast<long long*>(sp + Cfg::kOffMisc + 32);
    TreeRun* run = reinterpret_cast<TreeRun*>(sp + Cfg::kOffMisc + 32 + 192);

    if (tid < Cfg::kBars) {
        const int i = tid - 2 * NS;              // one barrier a thread; a group's four warps arrive for p_full and o_empty
        mbar_init(bars + 8u * tid, i == 4 || i == 5 || i >= 8 ? 4 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < 4) odd_piece[tid] = 0;
    if (tid == 32) { prefetch_tmap(&map_k); prefetch_tmap(&map_v); }
    if (warp == 1) {
        __syncwarp();
        tmem_alloc(base + Cfg::kOffMisc, 512);
        tmem_relinquish();
    }
    grid_dependency_wait();                    // lengths, queries and the drafts' keys come from the kernels before
    tree_find_run(p.w, part, run);
    if (tid == 0) {
        reinterpret_cast<TreeTail*>(p.scratch)[blockIdx.x].last_cta = -1;
        tree_front(p.scratch)[blockIdx.x] = run->begin < run->end && !run->at.item_begins();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t tmem_s = tmem, tmem_o = tmem + 256u;          // S and O of group g at + 128 g
    const int n_tiles = (int)(run->end - run->begin);

    constexpr uint32_t kIdesc = (1u << 4) | (Ops::kFormat << 7) | (Ops::kFormat << 10) | ((uint32_t)(kRows >> 4) << 24);

    if (warp == 0 && n_tiles > 0) {
        tree_load_keys<DH, NS, 0>(p, &map_k, &map_v, run, base + Cfg::kOffRing, ring_full(0), ring_empty(0));
    } else if (warp == 3 && n_tiles > 0) {
        tree_load_queries<DH, kTileRows, 32, 1, T>(p, run, sp, nullptr, 0u, q_full, q_empty, lane);
    } else if (warp == 1 && n_tiles > 0) {
        // ---------------- the products, of the groups by turns
        if (lane == 0) {
            TreeCursor c = run->at;
            uint32_t piece = 0, seq = 0, done[2] = {0, 0}, uses[2] = {0, 0};     // pieces, tiles of the ring; tiles and pieces of each group
            int groups = 0;
            bool ok = true, first = true, last = n_tiles == 1 || c.item_ends();  // the tile opens, closes its piece
            auto scores = [&](int g, uint32_t at) {
                tc_fence_after();
                const uint32_t ka = base + Cfg::kOffRing + (at % NS) * Cfg::kTileBytes;
#pragma unroll
                for (int k = 0; k < DH / 16; ++k) {
                    const uint64_t da = smem_desc_sw128(base + g * (kRows * 128) + (k >> 2) * (kTileRows * 128)) + (uint64_t)(2 * (k & 3));
                    const uint64_t db = smem_desc_sw128(ka + (k >> 2) * 1024, tree_group_bytes<DH>()) + (uint64_t)(2 * (k & 3));
                    umma_bf16(tmem_s + 128u * g, da, db, kIdesc | ((uint32_t)(kKeys >> 3) << 17), k > 0 ? 1u : 0u);
                }
                umma_commit(s_full(g));
            };
            auto filled = [&](uint32_t at) { return mbar_poll(ring_full(at % NS), (at / NS) & 1u); };
            ok = mbar_poll(q_full, 0u) && filled(0u);
            if (ok) {
                groups = c.queries(p.w) > kRows ? 2 : 1;
                for (int g = 0; g < groups; ++g) scores(g, 0u);
                umma_commit(ring_empty(0));
                if (last) umma_commit(q_empty);
                piece = seq = 1;
            }
            // O += P V of this tile, then S of the next - over the weights: the products of one thread run in order - for one group,
            // then for the other, which forms its weights meanwhile
            for (int t = 0; t < n_tiles && ok; ++t) {
                const bool more = t + 1 < n_tiles, next_opens = last;
                const uint32_t v_at = seq, k_at = seq + 1;
                int next_groups = groups;
                bool next_last = false;
                if (more) {
                    c.next(p.w);
                    if (next_opens) next_groups = c.queries(p.w) > kRows ? 2 : 1;
                    next_last = t + 2 == n_tiles || c.item_ends();
                }
                if (!filled(v_at)) { ok = false; break; }
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    if (g < groups) {
                        // A new piece's first product overwrites outputs that have been read.  Where the second group sits the piece
                        // out, its last outputs are waited for as well: through pieces of up to 128 queries the first would otherwise
                        // run ahead of it and reuse its marks.
                        if (first && groups == 1 && uses[1] > 0 && !mbar_poll(o_empty(1), (uses[1] - 1) & 1u)) { ok = false; break; }
                        if ((first && uses[g] > 0 && !mbar_poll(o_empty(g), (uses[g] - 1) & 1u)) || !mbar_poll(p_full(g), done[g] & 1u)) { ok = false; break; }
                        ++done[g];
                        tc_fence_after();
                        const uint32_t va = base + Cfg::kOffRing + (v_at % NS) * Cfg::kTileBytes;
#pragma unroll
                        for (int k = 0; k < kKeys / 16; ++k)
                            umma_f16_ta(tmem_o + 128u * g, tmem_s + 128u * g + 8u * k,
                                        smem_desc_sw128_mn(va + k * 2 * tree_group_bytes<DH>(), 1024, tree_group_bytes<DH>()),
                                        kIdesc | (1u << 16) | ((uint32_t)(DH >> 3) << 17), (!first || k > 0) ? 1u : 0u);      // bit 16: B is MN-major
                        if (g == groups - 1) umma_commit(ring_empty(v_at % NS));
                        if (last) { umma_commit(o_full(g)); ++uses[g]; }
                    }
                    if (more && !next_opens && g < groups) {
                        if (g == 0 && !filled(k_at)) { ok = false; break; }
                        scores(g, k_at);
                    }
                }
                if (!ok) break;
                if (more && next_opens) {                        // other queries: behind the last products with the ones before
                    if (!mbar_poll(q_full, piece & 1u) || !filled(k_at)) { ok = false; break; }
                    ++piece;
                    for (int g = 0; g < next_groups; ++g) scores(g, k_at);
                }
                if (more) {
                    umma_commit(ring_empty(k_at % NS));
                    if (next_last) umma_commit(q_empty);
                }
                seq += 2;
                groups = next_groups;
                first = next_opens;
                last = next_last;
            }
            if (!ok) atomicExch(p.w.err_flag, kErrTreeWait);
        }
    } else if (warp >= 4 && n_tiles > 0) {
        // ---------------- softmax groups
        const int g = (warp >> 2) - 1, quarter = warp & 3, row = quarter * 32 + lane;        // row of the group
        const uint32_t t_lane = (uint32_t)(quarter * 32) << 16;
        const uint32_t ts = tmem_s + 128u * g + t_lane, to = tmem_o + 128u * g + t_lane;
        TreeCursor c = run->at;
        bool split_front = !c.item_begins(), ok = true, opens = true;
        float m_ref = kNoRef, l_run = 0.0f;
        int kt_first = 0, q0 = 0, nq = 0, tok = 0, hg = 0;       // of the group: first query, queries
        uint32_t piece = 0, done = 0, uses = 0;                  // pieces; tiles and pieces of this group
        const uint32_t* mask = nullptr;
        auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_poll(bar, parity)) != 0; };
        for (int t = 0; t < n_tiles && ok; ++t) {
            if (opens) {
                q0 = c.first_query(p.w) + g * kRows;
                nq = min(kRows, c.queries(p.w) - g * kRows);
                kt_first = c.kt;
                tok = (q0 + row) / p.w.group;
                hg = q0 + row - tok * p.w.group;
                if (p.tree_mask && row < nq) mask = p.tree_mask + (size_t)(c.r.row0 + tok) * p.mask_words;
                m_ref = kNoRef; l_run = 0.0f;
            }
            const int C = c.r.L - c.r.n;
            const bool warp_live = quarter * 32 < nq, item_ends = c.item_ends(), piece_ends = item_ends || t == n_tiles - 1;
            if (nq > 0) {
                const bool tail = (c.kt + 1) * kKeys > C;
                if (!wait_all(s_full(g), done & 1u)) { ok = false; break; }      // the product with V before has run as well
                ++done;
                tc_fence_after();
                if (tail && g == 0) {
                    const int slot = (2 * t + 1) % NS;
                    if (!wait_all(ring_full(slot), (uint32_t)((2 * t + 1) / NS) & 1u)) { ok = false; break; }
                    if (tree_clean_values<DH, Ops::kExpMask>(sp + Cfg::kOffRing + slot * Cfg::kTileBytes, max(C - c.kt * kKeys, 0),
                                                             c.r.L - c.kt * kKeys, row))
                        odd_piece[piece & 3u] = piece + 1;
                }
                if (warp_live) {
                    // Loops over chunks of 32 columns, the next on its way while one is worked on.
                    if (tail) {                                  // take out what the row does not see
#pragma unroll 1
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t vis = row < nq ? visible_word(c.kt * kKeys + 32 * q, C, c.r.n, tok, mask, p.mask_words) : 0u;
                            uint32_t s[32];
                            __syncwarp();                        // tensor memory is accessed by whole warps
                            tmem_ld32(ts + 32u * q, s);
                            load32_wait(s);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((vis >> e) & 1u)) s[e] = __float_as_uint(-INFINITY);
                            tmem_store32(ts + 32u * q, s);
                        }
                        tmem_store_wait();
                    }
                    uint32_t sa[32], sb[32];
                    float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    auto highest = [&](const uint32_t (&s)[32]) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) t4[(e >> 1) & 3] = fmaxf(t4[(e >> 1) & 3], fmaxf(__uint_as_float(s[e]), __uint_as_float(s[e + 1])));
                    };
                    __syncwarp();
                    tmem_ld32(ts, sa);
#pragma unroll
                    for (int q = 0; q < 4; q += 2) {
                        load32_wait(sa);
                        tmem_ld32(ts + 32u * q + 32u, sb);
                        highest(sa);
                        load32_wait(sb);
                        tmem_ld32(ts + (q < 2 ? 64u : 0u), sa);  // at last the first chunk again, for the weights
                        highest(sb);
                    }
                    // weights 2^(score - reference): the largest is 2^kBias .. 2^(kBias + 8)
                    // (the scaled maximum is rounded by itself, as the scores are below: see tree_shift)
                    const float high = __fmul_rn(fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])), p.scale_log2), top = high - Ops::kBias;
                    if (opens) {
                        m_ref = fmaxf(top, kNoRef);
                    } else {
                        const bool grow = row < nq && high - m_ref > Ops::kBias + kTreeSlack;
                        if (__any_sync(0xffffffffu, grow)) {     // rare: move the reference, bring the row's outputs and sum to it
                            const float f = grow ? tree_ex2(m_ref - top) : 1.0f;
#pragma unroll 1
                            for (int c0 = 0; c0 < DH; c0 += 16) {
                                uint32_t o[16];
                                load16(to + (uint32_t)c0, o);
                                load16_wait(o);
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                store16(to + (uint32_t)c0, o);
                            }
                            tmem_store_wait();
                            l_run *= f;
                            if (grow) m_ref = top;
                        }
                    }
                    const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), minus = make_float2(-m_ref, -m_ref);
                    float2 sum2[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
                    auto weigh = [&](const uint32_t (&s)[32], int q, auto far) {
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float2 y = make_float2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1]));
                            if constexpr (far.value) y = make_float2(tree_shift(y.x, p.scale_log2, m_ref), tree_shift(y.y, p.scale_log2, m_ref));
                            else y = tree_fma2(y, scale2, minus);
                            y.x = tree_ex2(y.x);
                            y.y = tree_ex2(y.y);
                            sum2[e & 1] = tree_add2(sum2[e & 1], y);
                            w[e] = Ops::pack(y.x, y.y);
                        }
                        store16(ts + 16u * q, w);                // over scores that have been read
                    };
                    auto weigh_all = [&](auto far) {
#pragma unroll 1
                        for (int q = 0; q < 4; q += 2) {         // (no load is under way where the branches and the loop turn)
                            tmem_ld32(ts + 32u * q + 32u, sb);
                            weigh(sa, q, far);
                            load32_wait(sb);
                            if (q < 2) tmem_ld32(ts + 64u, sa);
                            weigh(sb, q + 1, far);
                            load32_wait(sa);
                        }
                    };
                    load32_wait(sa);
                    if (__any_sync(0xffffffffu, row < nq && tree_far(m_ref))) weigh_all(FarScores<true>{});
                    else weigh_all(FarScores<false>{});
                    tmem_store_wait();
                    l_run += (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(g));
                if (piece_ends) {
                    if (!wait_all(o_full(g), uses & 1u)) { ok = false; break; }
                    ++uses;
                    tc_fence_after();
                    const bool whole = item_ends && !split_front;
                    const bool repair = odd_piece[piece & 3u] == piece + 1;
                    const float inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;
                    const int head = c.h * p.w.group + hg, trow = g * kRows + row;
                    T* dst = static_cast<T*>(p.out) + (int64_t)(c.r.row0 + tok) * p.out_stride + (int64_t)head * DH;
                    float* slot = tree_slot(p.scratch, split_front ? 2 * blockIdx.x : 2 * blockIdx.x + 1, kTileRows, DH);
                    if (warp_live) {
#pragma unroll 1
                        for (int c0 = 0; c0 < DH; c0 += 32) {
                            uint32_t oa[32];
                            float o[32];
                            __syncwarp();                        // lanes part below: rows without a query, repairs
                            tmem_ld32(to + (uint32_t)c0, oa);
                            load32_wait(oa);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(oa[e]);
                            if (repair && row < nq) {            // non-finite values of drafts this row sees, within the piece's tiles
                                for (int j = 0; j < c.r.n; ++j) {
                                    const int key = C + j, kt = key / kKeys;
                                    if (kt < kt_first || kt > c.kt || !(visible_word(key, C, c.r.n, tok, mask, p.mask_words) & 1u)) continue;
                                    const int64_t off = tree_value_offset(p, c, key);
                                    if (off < 0) continue;
#pragma unroll
                                    for (int e = 0; e < 32; ++e) {
                                        const float x = Ops::value(static_cast<const T*>(p.v)[off + c0 + e]);
                                        if (!isfinite(x)) o[e] += x;
                                    }
                                }
                            }
                            if (whole && row < nq) {
#pragma unroll
                                for (int e = 0; e < 32; e += 8) {
                                    uint4 w;
                                    w.x = Ops::pack(o[e] * inv, o[e + 1] * inv); w.y = Ops::pack(o[e + 2] * inv, o[e + 3] * inv);
                                    w.z = Ops::pack(o[e + 4] * inv, o[e + 5] * inv); w.w = Ops::pack(o[e + 6] * inv, o[e + 7] * inv);
                                    *reinterpret_cast<uint4*>(dst + c0 + e) = w;
                                }
                            } else if (row < nq) {
                                float* po = slot + 2 * kTileRows + (size_t)trow * DH + c0;
#pragma unroll
                                for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(po + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                            }
                        }
                        if (!whole && row < nq) { slot[trow] = m_ref; slot[kTileRows + trow] = l_run; }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(o_empty(g));
                }
            }
            if (piece_ends) {
                if (!item_ends && !split_front && tid == 128) {  // begins here, goes on in the next CTAs
                    TreeTail tl{};
                    tl.last_cta = run->tail_cta;
                    tl.queries = c.queries(p.w); tl.row0 = c.r.row0; tl.q0 = c.first_query(p.w); tl.h = c.h;
                    reinterpret_cast<TreeTail*>(p.scratch)[blockIdx.x] = tl;
                }
                split_front = false;
                ++piece;
            }
            opens = piece_ends;
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
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    return fn(map, type == kTypeBf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank, const_cast<void*>(base),
              dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DH, typename T>
int tc_launch(const TcParams& p, const CUtensorMap& map_k, const CUtensorMap& map_v, int grid, cudaStream_t s, bool dependent) {
    static DeviceOnce attr;
    if (!attr.done([] { return allow_smem(tree_attention_tc_kernel<DH, T>, TcCfg<DH>::kSmemBytes); })) return ZOQAT_ERR_CUDA;
    TcParams q = p;
    q.smem_bytes = TcCfg<DH>::kSmemBytes;
    return launch_kernel(tree_attention_tc_kernel<DH, T>, dim3(grid), dim3(kTcThreads), TcCfg<DH>::kSmemBytes, s, dependent, map_k, map_v, q) == cudaSuccess
               ? ZOQAT_OK : ZOQAT_ERR_CUDA;
}

template <int DH, typename T>
int combine_launch(const TcParams& p, int grid, int y, cudaStream_t s) {
    return launch_kernel(tree_combine_kernel<T, DH>, dim3(grid, y), dim3(256), 0, s, true, p.scratch, p.w.tile_rows, p.w.group,
                         static_cast<T*>(p.out), p.out_stride) == cudaSuccess ? ZOQAT_OK : ZOQAT_ERR_CUDA;
}

}  // namespace

int launch_tree_attention_tc(const TreeAttnArgs& a, cudaStream_t s, bool dependent) {
    const int dh = a.cache.d_head, type = a.cache.type;
    TcParams p{};
    const int group = a.n_heads / a.cache.n_kv_heads;
    // Queries per tile, from the average number of drafts (the host does not know the lengths).  Up to 64 queries the keys are
    // the rows of the products, which costs exponentials only for queries that exist; a tile that is too small reads the keys
    // again for the next one, a tile that is too large costs products and exponentials of empty columns.  16 requests of 4096
    // keys, 8 key heads of 128, tiles of 16 / 32 / 64 / 256, us: 4 queries 67 / 68 / 71 / 83; 16: 71 / 71 / 73 / 87; 32: 109 / 79 /
    // 81 / 91; 48: 149 / 112 / 89 / 99; 64: 185 / 116 / 97 / 106; 96: 237 / 155 / 126 / 118.  Too small costs far more than too
    // large, hence the margin of a half for batches whose trees differ.
    const long long drafts = (long long)a.rows * group;
    const long long want = a.rows <= a.batch ? group : (3 * drafts + 2 * a.batch - 1) / (2 * a.batch);     // 1.5 x the average
    const int nq = want <= 16 ? 16 : (want <= 32 ? 32 : (want <= 64 ? 64 : kRows));
    p.w = TreeWork{a.kv_len, a.row_start, a.block_table, a.batch, a.rows, a.cache.n_kv_heads, a.max_pages, a.cache.page_size,
                   group, nq < kRows ? nq : kTileRows, kKeys, 4, a.err_flag};
    p.q = a.q; p.q_stride = a.q_stride;
    p.box_keys = a.cache.page_size < kKeys ? a.cache.page_size : kKeys;
    p.n_pages = a.cache.n_pages; p.mask_words = a.mask_words; p.tree_mask = a.tree_mask;
    p.scale_log2 = (float)(1.4426950408889634 * (double)a.scale);
    p.out = a.out; p.out_stride = a.out_stride; p.scratch = a.scratch;
    p.v = a.cache.v; p.page_stride = a.cache.page_stride; p.slot_stride = a.cache.slot_stride; p.head_stride = a.cache.head_stride;
    alignas(64) CUtensorMap map_k, map_v;
    // {64 columns, 8 keys, halves, groups of 8 keys, heads of all pages}
    const int64_t ss = a.cache.slot_stride, unit = a.cache.n_kv_heads > 1 ? a.cache.head_stride : a.cache.page_stride;
    p.page_units = a.cache.n_pages > 1 ? (int)(a.cache.page_stride / unit) : 1;
    const int64_t units = (int64_t)(a.cache.n_pages - 1) * p.page_units + a.cache.n_kv_heads;      // (the caller has checked that they fit)
    p.units = (int)units;
    p.page_shift = -1;
    for (int b = 3; b < 31; ++b)
        if (a.cache.page_size == 1 << b) p.page_shift = b;
    const cuuint64_t kd[5] = {64, 8, (cuuint64_t)dh / 64, (cuuint64_t)a.cache.page_size / 8, (cuuint64_t)units};
    const cuuint64_t kst[4] = {(cuuint64_t)ss * 2, 128, (cuuint64_t)ss * 16, (cuuint64_t)unit * 2};
    const cuuint32_t kb[5] = {64, 8, (cuuint32_t)dh / 64, (cuuint32_t)p.box_keys / 8, 1};
    if (!encode(&map_k, type, a.cache.k, 5, kd, kst, kb) || !encode(&map_v, type, a.cache.v, 5, kd, kst, kb)) return ZOQAT_ERR_CUDA;
    const int grid = tree_grid();
    const int y = want < 2 ? 1 : (want < 32 ? (int)(want + 1) / 2 : 16);      // CTAs that share the queries of a split item
    int rc;
    if (nq < kRows) rc = launch_tree_keys(p, map_k, map_v, dh, type, nq, grid, s, dependent);
    else if (type == kTypeBf16) rc = dh == 64 ? tc_launch<64, __nv_bfloat16>(p, map_k, map_v, grid, s, dependent) : tc_launch<128, __nv_bfloat16>(p, map_k, map_v, grid, s, dependent);
    else rc = dh == 64 ? tc_launch<64, __half>(p, map_k, map_v, grid, s, dependent) : tc_launch<128, __half>(p, map_k, map_v, grid, s, dependent);
    if (rc != ZOQAT_OK) return rc;
    count_launch();
    if (type == kTypeBf16) rc = dh == 64 ? combine_launch<64, __nv_bfloat16>(p, grid, y, s) : combine_launch<128, __nv_bfloat16>(p, grid, y, s);
    else rc = dh == 64 ? combine_launch<64, __half>(p, grid, y, s) : combine_launch<128, __half>(p, grid, y, s);
    if (rc == ZOQAT_OK) count_launch();
    return rc;
}

}  // namespace zq
