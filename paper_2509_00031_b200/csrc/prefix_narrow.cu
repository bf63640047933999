// Parts of an attention over the pages with few queries per key head (8 a tile), bf16 / fp16: the keys that a request has for itself behind
// a shared prefix, and the prefix itself where few beams share it.  Such parts are short or have next to no arithmetic: what
// counts is that every key is on its way early and that opening and closing a part costs little.
//
// A warp is a worker of its own: the 12 warps of every SM cut the tiles of 32 keys of all parts into equal runs (tree_attention.cuh), and no warp waits for another
// within a run.  K and V tiles come by TMA into 16 KB of the warp's own (one tile, two at d_head 64) and are read once into registers; the next keys are asked for
// when these have been read, and so the next values: one of the two is always on its way.
// A product over d_head may take its elements in any order, and so may the keys and the columns of the output; the orders below are those in which every
// thread reads 16 bytes at a time and no two of a quarter warp meet in a bank under the 128-byte swizzle.  The keys and the columns are the rows of the
// products, so that eight queries cost no more than they need; with g = lane / 4, j = lane % 4 and p(g) = g / 2 + 4 (g % 2), for 16 keys of a tile
//   S^T = K Q^T      m16n8k16, row g is key p(g), row g + 8 key 8 + p(g): a thread's chunk j + 4 i holds elements 8 (j + 4 i) .. + 7, which serve as the k pairs
//                    (2 j, 2 j + 8) of steps 2 i and 2 i + 1; the queries are read the same way
//   O^T += V^T P^T   P^T is transposed in registers (movmatrix); a thread has columns 8 p(g) .. + 7 of both halves of the keys j, 4 + j, 8 + j, 12 + j, pairs of
//                    keys are put together by byte permutations, and the rows g, g + 8 of m-tile t are the columns 8 p(g) + t of the halves
// The running maximum is exact for every tile; outputs are brought to a new one only when it moved.  Weights are rounded to the cache's type for the second product, since its
// operands have to be of one type (half a unit of a weight's last place: bf16 outputs are off by 0.0023 relative, 0.0017 with their own rounding alone); sums are of the
// unrounded ones, in fp32.  Waits are bounded and report through *err_flag.
// 64 requests of 4 queries a head, 8 key heads of 128, 700 own keys behind 2000 shared by eight: 67 us, 38 of them the caches' 249 MB at the rate of a copy.  Bound by memory on all
// SMs (6.8 TB/s); an SM alone takes in 76 GB/s.  Tiles of 16 keys in the same memory issue a third more instructions a key and go through two maxima and sets of shuffles one
// after the other (that call 69 us, 128 requests behind 16001 keys with 1 to 1500 own 111 against 105).  Tiles of 16
// queries for parts with more than eight were never the fastest: 8 groups of 16 queries behind 8000 keys 90 us; two tiles of eight, the second from L2, 68; keys as rows 78.
#include "tree_attention_tc.cuh"
#include "../../include/zoqat.h"

namespace zq {
namespace {

constexpr int kWarps = kNarrowWarps, kThreads = 32 * kWarps, kTile = kNarrowKeys;
static_assert(kThreads <= PrefixScan::kMost, "the scan");

template <int DH> struct NarrowCfg {
    static constexpr int kStage = 2 * kTile * DH * 2;                       // K and V of a tile
    static constexpr int kStages = (DH == 128 ? 32 : 64) / kTile;
    static constexpr int kSmem = kWarps * kStages * kStage + 1024;
};

__device__ __forceinline__ uint4 lds16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
template <typename T> __device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b)[2]);
template <> __device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b)[2]) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
template <> __device__ __forceinline__ void mma16816<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b)[2]) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

template <int DH, typename T>
__global__ void __launch_bounds__(kThreads, 1)
prefix_narrow_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ TcParamsT<PrefixWork> p) {
    using Cfg = NarrowCfg<DH>;
    using Ops = HalfOps<T>;
    constexpr int NS = Cfg::kStages, kI = DH / 32, kHalves = DH / 64, kM = DH / 16, kTileBytes = Cfg::kStage / 2, kSub = kTile / 16, kBoxes = kTile / 8, NQ = kNarrowRows;
    constexpr uint32_t kGroup = tree_group_bytes<DH>();          // eight keys
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[kWarps][2 * NS];       // K and V of a stage have arrived
    __shared__ TreeRunT<PrefixWork> runs[kWarps];
    __shared__ PrefixScan scan;
    const PrefixWork& w = p.w;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, j = lane & 3;
    const int worker = blockIdx.x * kWarps + warp, pg = (g >> 1) | (g & 1) << 2;
    if (tid < kWarps * 2 * NS) {
        mbar_init(smem_u32(&bars[0][0]) + 8u * tid, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 0) { prefetch_tmap(&map_k); prefetch_tmap(&map_v); }
    if (!w.late_wait) grid_dependency_wait();
    grid_dependency_release();
    const int ctas = prefix_find_runs<kWarps>(w, scan, runs);
    if ((int)blockIdx.x == max(ctas, 1) - 1 && w.first + w.batch > w.groups) prefix_map_rows(w, scan);
    const TreeRunT<PrefixWork>& run = runs[warp];
    const int n_tiles = (int)(run.end - run.begin);
    if (lane == 0) prefix_front(p.scratch)[worker] = n_tiles > 0 && !run.at.item_begins();

    if (n_tiles > 0) {
    const uint32_t ring = ((smem_u32(smem) + 1023u) & ~1023u) + warp * (NS * Cfg::kStage), bar = smem_u32(&bars[warp][0]);
    PrefixCursor c, ahead;
    c.r = run.at.r; c.b = run.at.b; c.h = run.at.h; c.rt = run.at.rt; c.kt = run.at.kt;
    ahead = c;
    // the boxes of a tile (up to four where pages have 8 slots), looked up a tile before they are requested
    const int box_shift = 31 - __clz(p.box_keys), n_box = kTile >> box_shift;            // (8, 16 or 32 keys)
    const uint32_t box_bytes = (uint32_t)(p.box_keys >> 3) * kGroup;
    int page = 0, group = 0;                                     // of box `lane`
    auto look_up = [&]() {
        const int key = ahead.kt * kTile + (lane & (kBoxes - 1)) * p.box_keys;
        const int i = p.page_shift >= 0 ? key >> p.page_shift : key / w.page_size;
        group = (key - i * w.page_size) >> 3;
        page = key < ahead.r.L ? __ldg(w.block_table + (size_t)ahead.r.row * w.max_pages + i) : -1;
    };
    // box u by lane u; those behind the last key are left out
    auto request = [&](const CUtensorMap* map, uint32_t to, uint32_t full) {
        const int boxes = min(n_box, (ahead.r.L - ahead.kt * kTile + p.box_keys - 1) >> box_shift);
        if (lane == 0) mbar_arrive_expect_tx(full, boxes * box_bytes);
        __syncwarp();
        if (lane < boxes) {
            int unit = p.units;                                  // behind the map's end: zeros
            if (page >= 0 && page < p.n_pages) unit = page * p.page_units + ahead.h;
            else atomicExch(w.err_flag, kErrBadPage);
            tma_load_5d(to + lane * box_bytes, map, full, 0, 0, 0, group, unit);
        }
    };
    look_up();
#pragma unroll 1
    for (int k = 0; k < NS && k < n_tiles; ++k) {
        request(&map_k, ring + k * Cfg::kStage, bar + 16u * k);
        request(&map_v, ring + k * Cfg::kStage + kTileBytes, bar + 16u * k + 8u);
        if (k + 1 < n_tiles) { ahead.next(w, scan); look_up(); }
    }

    bool split_front = !run.at.item_begins(), opens = true, odd = false;
    bool ok = true, values = false;                              // values: they were waited for last
    int t = 0, kt_first = 0, stage = 0, nq = 0, q0 = 0;
    uint32_t phase = 0;
    uint32_t q[2 * kI][2];
    float o[kM][4], m[2], l[2];
    auto seen = [&](int e, int key, int C) {                     // bits of the 32 keys from `key` on
        const int tok = (q0 + 2 * j + e) / w.group;
        if (2 * j + e >= nq) return 0u;
        return visible_word(key, C, c.r.n, tok, p.tree_mask ? p.tree_mask + (size_t)(c.r.row0 + tok) * p.mask_words : nullptr, p.mask_words);
    };
#pragma unroll 1
    for (; t < n_tiles; ++t) {
        if (opens) {
            opens = false;
            odd = false;
            kt_first = c.kt;
            q0 = c.rt * NQ;
            nq = min(NQ, c.r.n * w.group - q0);
            const int tok = (q0 + g) / w.group;
            const bool live = g < nq;
            const T* src = static_cast<const T*>(p.q) + (int64_t)(c.r.row0 + tok) * p.q_stride + (int64_t)(c.h * w.group + q0 + g - tok * w.group) * DH + 8 * j;
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                const uint4 x = live ? __ldg(reinterpret_cast<const uint4*>(src + 32 * i)) : make_uint4(0, 0, 0, 0);
                q[2 * i][0] = x.x; q[2 * i][1] = x.y; q[2 * i + 1][0] = x.z; q[2 * i + 1][1] = x.w;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) { m[e] = kNoRef; l[e] = 0.0f; }
#pragma unroll
            for (int i = 0; i < kM; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
        }
        const uint32_t at = ring + stage * Cfg::kStage, full = bar + 16u * stage, parity = phase;
        if (++stage == NS) { stage = 0; phase ^= 1u; }
        values = false;
        if (!__all_sync(0xffffffffu, mbar_poll(full, parity))) { ok = false; break; }
        float s[kSub][4] = {};
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
            for (int a = 0; a < kSub; ++a) {
                const uint32_t from = at + 2 * a * kGroup + (i >> 1) * 1024 + pg * 128 + (((j + 4 * (i & 1)) ^ pg) << 4);
                const uint4 x = lds16(from), y = lds16(from + kGroup);
                mma16816<T>(s[a], x.x, y.x, x.y, y.y, q[2 * i]);
                mma16816<T>(s[a], x.z, y.z, x.w, y.w, q[2 * i + 1]);
            }
        __syncwarp();
        if (t + NS < n_tiles) request(&map_k, at, full);         // (the keys have been read)
        const int key0 = c.kt * kTile, C = c.r.L - c.r.drafts();
        const bool tail = key0 + kTile > C;
        uint32_t b[kSub][2];
        bool moved = false;
        float f[2];
#pragma unroll
        for (int a = 0; a < kSub; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[a][e] = __fmul_rn(s[a][e], p.scale_log2);      // rounded by itself: references are such products
        if (tail) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t vis = seen(e, key0, C);
#pragma unroll
                for (int a = 0; a < kSub; ++a) {
                    if (!((vis >> (16 * a + pg)) & 1u)) s[a][e] = -INFINITY;
                    if (!((vis >> (16 * a + pg + 8)) & 1u)) s[a][2 + e] = -INFINITY;
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float top = fmaxf(s[0][e], s[0][2 + e]);
#pragma unroll
            for (int a = 1; a < kSub; ++a) top = fmaxf(top, fmaxf(s[a][e], s[a][2 + e]));
            top -= Ops::kBias;
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            top = fmaxf(top, m[e]);
            f[e] = tree_ex2(m[e] - top);
            moved = moved || top != m[e];
            m[e] = top;
            float sum = 0.0f;
#pragma unroll
            for (int a = 0; a < kSub; ++a) {
                s[a][e] = tree_ex2(s[a][e] - top);
                s[a][2 + e] = tree_ex2(s[a][2 + e] - top);
                sum += s[a][e] + s[a][2 + e];
            }
            l[e] = l[e] * f[e] + sum;
        }
#pragma unroll
        for (int a = 0; a < kSub; ++a) {
            b[a][0] = transpose8(Ops::pack(s[a][0], s[a][1]));
            b[a][1] = transpose8(Ops::pack(s[a][2], s[a][3]));
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int i = 0; i < kM; ++i) { o[i][0] *= f[0]; o[i][1] *= f[1]; o[i][2] *= f[0]; o[i][3] *= f[1]; }
        }
        values = true;
        if (!__all_sync(0xffffffffu, mbar_poll(full + 8u, parity))) { ok = false; break; }
#pragma unroll
        for (int a = 0; a < kSub; ++a) {
            uint32_t v[4][4 * kHalves];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    const int key = 4 * (e & 1) + j;
                    const uint4 x = lds16(at + kTileBytes + (2 * a + (e >> 1)) * kGroup + hf * 1024 + key * 128 + ((pg ^ key) << 4));
                    v[e][4 * hf] = x.x; v[e][4 * hf + 1] = x.y; v[e][4 * hf + 2] = x.z; v[e][4 * hf + 3] = x.w;
                }
            if (tail) {                                          // a draft's element that is not finite: put back at the end for those who see it
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = key0 + 16 * a + 8 * (e >> 1) + 4 * (e & 1) + j;
                    if (key < C) continue;
#pragma unroll
                    for (int i = 0; i < 4 * kHalves; ++i) {
                        if (key >= c.r.L) { v[e][i] = 0; continue; }                     // what lies there is not the request's
                        if ((v[e][i] & Ops::kExpMask) == Ops::kExpMask) { v[e][i] &= 0xFFFF0000u; odd = true; }
                        if (((v[e][i] >> 16) & Ops::kExpMask) == Ops::kExpMask) { v[e][i] &= 0x0000FFFFu; odd = true; }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kM; ++i) {
                // element i of both halves (d_head 64: of the eight columns, i and i + 4)
                const int lo = i >> 1, hi = kHalves == 2 ? 4 + lo : 2 + lo;
                const uint32_t pick = i & 1 ? 0x7632u : 0x5410u;
                const uint32_t a0 = __byte_perm(v[0][lo], v[1][lo], pick), a1 = __byte_perm(v[0][hi], v[1][hi], pick);
                const uint32_t a2 = __byte_perm(v[2][lo], v[3][lo], pick), a3 = __byte_perm(v[2][hi], v[3][hi], pick);
                mma16816<T>(o[i], a0, a1, a2, a3, b[a]);
            }
        }
        __syncwarp();
        if (t + NS < n_tiles) {
            request(&map_v, at + kTileBytes, full + 8u);
            if (t + NS + 1 < n_tiles) { ahead.next(w, scan); look_up(); }
        }
        const bool ends = c.kt == c.r.n_kt - 1;
        if (ends || t == n_tiles - 1) {
            const bool whole = ends && !split_front;
            const bool repair = __any_sync(0xffffffffu, odd);
            float* slot = tree_slot(p.scratch, split_front ? 2 * worker : 2 * worker + 1, NQ, DH);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[e];
                sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                const int row = 2 * j + e;
                if (row >= nq) continue;
                const int64_t query = prefix_query(w, c.r, q0 + row, c.h);
                float* to = whole ? w.partial + query * (DH + 4) : slot + 2 * NQ + row * DH;
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {           // columns 64 hf + 8 p(g) .. + 7
                    float x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = kHalves == 2 ? o[i % kM][2 * hf + e] : o[i % 4][2 * (i >> 2) + e];
                    const int col = 64 * hf + 8 * pg;
                    for (int d = 0; repair && d < c.r.n; ++d) {
                        const int key = C + d, kt = key / kTile;
                        if (kt < kt_first || kt > c.kt || !(seen(e, key, C) & 1u)) continue;
                        const int of = __ldg(w.block_table + (size_t)c.r.row * w.max_pages + key / w.page_size);
                        if (of < 0 || of >= p.n_pages) continue;
                        const T* y = static_cast<const T*>(p.v) + of * p.page_stride + key % w.page_size * p.slot_stride + c.h * p.head_stride + col;
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (!isfinite(Ops::value(y[i]))) x[i] += Ops::value(y[i]);
                    }
                    *reinterpret_cast<float4*>(to + col) = make_float4(x[0], x[1], x[2], x[3]);
                    *reinterpret_cast<float4*>(to + col + 4) = make_float4(x[4], x[5], x[6], x[7]);
                }
                if (g == 0) {
                    if (whole) { to[DH] = m[e]; to[DH + 1] = sum; }
                    else { slot[row] = m[e]; slot[NQ + row] = sum; }
                    if (!split_front) w.entries[query] = ends ? make_int2(0, -1) : make_int2(worker | run.tail_cta << 16, row);
                }
            }
            split_front = false;
            opens = true;
        }
        c.next(w, scan);
    }
    if (!ok) {
        if (lane == 0) atomicExch(w.err_flag, kErrTreeWait);
        // what has been asked for has to land before the CTA may leave: of every stage, the next keys and values not seen yet
        for (int k = 0; k < NS; ++k) {
            const int next = t + (k + NS - t % NS) % NS, keys = values && next == t ? next + NS : next;
            if (keys < n_tiles) mbar_wait(bar + 16u * k, (uint32_t)(keys / NS) & 1u);
            if (next < n_tiles) mbar_wait(bar + 16u * k + 8u, (uint32_t)(next / NS) & 1u);
        }
    }
    }
    if (w.late_wait) grid_dependency_wait();
}

template <int DH, typename T>
int narrow_launch(const TcParamsT<PrefixWork>& p, const CUtensorMap& map_k, const CUtensorMap& map_v, int grid, cudaStream_t s, bool dependent) {
    static DeviceOnce attr;
    if (!attr.done([] { return allow_smem(prefix_narrow_kernel<DH, T>, NarrowCfg<DH>::kSmem); })) return ZOQAT_ERR_CUDA;
    if (launch_kernel(prefix_narrow_kernel<DH, T>, dim3(grid), dim3(kThreads), NarrowCfg<DH>::kSmem, s, dependent, map_k, map_v, p) != cudaSuccess) return ZOQAT_ERR_CUDA;
    count_launch();
    return ZOQAT_OK;
}

template <typename T>
int narrow_launch(const TcParamsT<PrefixWork>& p, const CUtensorMap& map_k, const CUtensorMap& map_v, int dh, int grid, cudaStream_t s, bool dependent) {
    return dh == 64 ? narrow_launch<64, T>(p, map_k, map_v, grid, s, dependent) : narrow_launch<128, T>(p, map_k, map_v, grid, s, dependent);
}

}  // namespace

int launch_prefix_narrow(const TcParamsT<PrefixWork>& p, const CUtensorMap& map_k, const CUtensorMap& map_v, int dh, int type, int grid, cudaStream_t s, bool dependent) {
    return type == kTypeBf16 ? narrow_launch<__nv_bfloat16>(p, map_k, map_v, dh, grid, s, dependent) : narrow_launch<__half>(p, map_k, map_v, dh, grid, s, dependent);
}

}  // namespace zq
