// What a serving step needs before its attention: the plan of a batch of requests over a paged key/value cache
// (block tables, slots, positions, tree masks) and the append of the new rows' keys and values into the pages.
//
//   cache_plan_kernel     lengths -> where every new row goes.  With c_b cached and n_b new rows of request b and pages of P
//                         slots: held_b = ceil(c_b / P), need_b = ceil((c_b + n_b) / P) - held_b, both prefix-summed over
//                         the requests; the k-th new page of request b is free[n_free - 1 - (first_b + k)].  One launch:
//                         every CTA scans all requests itself (a few kB from L2) and then writes its share of the rows and
//                         of the tables, so no CTA waits for another and no scratch is needed.
//                         Bound by latency: a launch, two chained loads and two block scans; 12 to 13 us a call from
//                         Python; replayed from a graph 3.3 us for 8 requests of one token, 4.7 for 64 prompts, 8.6 for 1024 trees.
//   cache_append_kernel   (a, b) -> (a cos - b sin, b cos + a sin) for q and k, then one rounding into the cache's type.
//                         Bound by memory: 8191 rows of 40 + 2 * 8 heads of 128 into binary16, 356 MB in 63.5 us, 87 % of the
//                         rate of a plain copy.
//   embed_rows_kernel     the residual rows of drafted tokens (each row has a position of its own).
//   widen_kernel          attention outputs of a 16-bit cache for the fp32 activation quantisers of a model's step.
#include "common.cuh"
#include "serve.cuh"
#include "vec8.cuh"

namespace zq {
namespace {

constexpr int kPlanThreads = 1024;

struct PlanParams {
    const int32_t *cached_len, *new_len;
    int batch, page_size, n_pages, max_pages;
    const int32_t* free_pages;
    int free_capacity;
    const int32_t* n_free;
    int32_t* table;
    const int32_t* parents;
    int max_rows, mask_words;
    int32_t *kv_len, *row_start, *row_request, *row_pos, *slot;
    uint32_t* tree_mask;
    int32_t *n_free_out, *status;
};

// Inclusive sum over the CTA's threads of two values at once (rows and pages share the two barriers).
__device__ __forceinline__ void block_scan2(long long& a, long long& b, long long (*part)[2]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long ua = __shfl_up_sync(0xffffffffu, a, o), ub = __shfl_up_sync(0xffffffffu, b, o);
        if (lane >= o) { a += ua; b += ub; }
    }
    if (lane == 31) { part[warp][0] = a; part[warp][1] = b; }
    __syncthreads();
    if (warp == 0) {
        long long pa = part[lane][0], pb = part[lane][1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long ua = __shfl_up_sync(0xffffffffu, pa, o), ub = __shfl_up_sync(0xffffffffu, pb, o);
            if (lane >= o) { pa += ua; pb += ub; }
        }
        part[lane][0] = pa; part[lane][1] = pb;
    }
    __syncthreads();
    if (warp > 0) { a += part[warp - 1][0]; b += part[warp - 1][1]; }
}

// the last b with first[b] <= x (first ascending, first[0] = 0 <= x)
__device__ __forceinline__ int owner_of(const int32_t* first, int batch, int x) {
    int lo = 0, hi = batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kPlanThreads)
cache_plan_kernel(PlanParams p) {
    extern __shared__ int32_t first[];          // [2][batch + 1]: rows, then new pages, before each request
    __shared__ long long part[32][2];
    __shared__ int bad;
    int32_t* row_first = first;
    int32_t* page_first = first + p.batch + 1;
    const int tid = threadIdx.x;
    const long long room = (long long)p.max_pages * p.page_size;
    if (tid == 0) bad = 0;
    __syncthreads();
    long long rows = 0, pages = 0;              // before this tile of requests
    for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
        const int b = b0 + tid;
        long long n = 0, need = 0;
        if (b < p.batch) {
            const long long c = __ldg(p.cached_len + b);
            n = __ldg(p.new_len + b);
            if (c < 0 || n < 0 || c + n > room || (p.mask_words && n > 32ll * p.mask_words)) {
                n = 0;
                bad = 1;                        // every writer stores the same value
            } else {
                need = (c + n + p.page_size - 1) / p.page_size - (c + p.page_size - 1) / p.page_size;
            }
        }
        long long n_in = n, need_in = need;
        block_scan2(n_in, need_in, part);
        // sums of refused plans may pass 32 bits; nothing reads them
        if (b < p.batch) { row_first[b] = (int32_t)(rows + n_in - n); page_first[b] = (int32_t)(pages + need_in - need); }
        rows += part[31][0];
        pages += part[31][1];
        __syncthreads();                        // part[] is written again by the next tile
    }
    const int free_now = __ldg(p.n_free);
    // nothing is planned when a length cannot be served, or when the pages do not suffice: every CTA comes to the same answer
    const bool refused = bad || rows > p.max_rows || free_now < 0 || free_now > p.free_capacity;
    const bool dry = !refused && pages > free_now;
    const bool idle = refused || dry;
    const int total = idle ? 0 : (int)rows, fresh = idle ? 0 : (int)pages;
    if (tid == 0) { row_first[p.batch] = total; page_first[p.batch] = fresh; }
    __syncthreads();
    const int step = gridDim.x * kPlanThreads, at = blockIdx.x * kPlanThreads + tid;
    if (at == 0) {
        *p.n_free_out = free_now - fresh;
        if (idle) atomicOr(p.status, refused ? kPlanBadLength : kPlanNoPages);
    }
    for (int b = at; b <= p.batch; b += step) {
        p.row_start[b] = idle ? 0 : row_first[b];
        if (b < p.batch) p.kv_len[b] = idle ? 0 : __ldg(p.cached_len + b) + __ldg(p.new_len + b);
    }
    // new entries of the tables; the entries a request holds already are only read
    for (int j = at; j < fresh; j += step) {
        const int b = owner_of(page_first, p.batch, j);
        const int held = (__ldg(p.cached_len + b) + p.page_size - 1) / p.page_size;
        p.table[(size_t)b * p.max_pages + held + (j - page_first[b])] = __ldg(p.free_pages + (free_now - 1 - j));
    }
    for (int r = at; r < p.max_rows; r += step) {
        if (r >= total) {                       // padding: consumers skip rows without a slot
            p.row_request[r] = -1; p.row_pos[r] = -1; p.slot[r] = -1;
            for (int w = 0; w < p.mask_words; ++w) p.tree_mask[(size_t)r * p.mask_words + w] = 0;
            continue;
        }
        const int b = owner_of(row_first, p.batch, r);
        const int start = row_first[b], i = r - start, c = __ldg(p.cached_len + b);
        const int t = c + i, pg = t / p.page_size;
        const int held = (c + p.page_size - 1) / p.page_size;
        const int page = pg < held ? p.table[(size_t)b * p.max_pages + pg]
                                   : __ldg(p.free_pages + (free_now - 1 - (page_first[b] + pg - held)));
        int slot = -1;
        if (page >= 0 && page < p.n_pages) slot = page * p.page_size + (t - pg * p.page_size);
        else atomicOr(p.status, kPlanBadPage);
        p.row_request[r] = b;
        p.slot[r] = slot;
        uint32_t* mask = p.tree_mask + (size_t)r * p.mask_words;
        if (!p.parents) {                       // a chain: everything up to the row itself
            for (int w = 0; w < p.mask_words; ++w) {
                const int upto = i + 1 - 32 * w;
                mask[w] = upto <= 0 ? 0u : (upto >= 32 ? 0xFFFFFFFFu : (1u << upto) - 1u);
            }
            p.row_pos[r] = t;
            continue;
        }
        // the draft and its ancestors, from itself down: parents come before their children, so the words of the mask are
        // finished one after the other
        int depth = 0, j = i, word = p.mask_words - 1;
        uint32_t bits = 0;
        while (true) {
            while (word >= 0 && word > (j >> 5)) { mask[word--] = bits; bits = 0; }
            bits |= 1u << (j & 31);
            const int up = __ldg(p.parents + start + j);
            if (up < -1 || up >= j) { atomicOr(p.status, kPlanBadParent); break; }
            if (up < 0) break;
            ++depth;
            j = up;
        }
        while (word >= 0) { mask[word--] = bits; bits = 0; }
        p.row_pos[r] = c + depth;
    }
}

// ---- append -------------------------------------------------------------------------------------------------------
// One thread per 8 + 8 elements (i .. i+7 and their partners d_head / 2 further) of a head of a row: q heads, then k heads,
// then v heads, as they stand in the row.  max_pos > 0: positions lie in [0, max_pos), with or without tables (a model may add
// its position embeddings before).
template <typename T>
__global__ void __launch_bounds__(256)
cache_append_kernel(const float* __restrict__ qkv, int64_t ld, const int32_t* __restrict__ row_pos, const int32_t* __restrict__ slot,
                    int n_heads, const float* __restrict__ cos_t, const float* __restrict__ sin_t, int max_pos, PagedCache cache,
                    T* __restrict__ q_out, int64_t q_stride, int32_t* __restrict__ err_flag) {
    const int half = cache.d_head >> 1, chunks = half >> 3;         // 4 (d_head 64) or 8 (d_head 128) chunks a head
    const int item = blockIdx.y * 256 + threadIdx.x;
    const int head = item / chunks, ch = item - head * chunks;
    const int n_kv = cache.n_kv_heads;
    grid_dependency_wait();                                         // (in a step of the model the projections come before)
    const int64_t row = blockIdx.x;
    const int sl = __ldg(slot + row), pos = max_pos > 0 ? __ldg(row_pos + row) : 0;      // both on their way at once
    if (head >= n_heads + 2 * n_kv || sl < 0) return;
    // a row with a slot or position outside is skipped whole, its v as well
    if (sl >= cache.n_pages * cache.page_size || pos < 0 || (max_pos > 0 && pos >= max_pos)) {
        if (item == 0) atomicExch(err_flag, kErrBadSlot);
        return;
    }
    const float* src = qkv + row * ld + (int64_t)head * cache.d_head + 8 * ch;
    float a[8], b[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        *reinterpret_cast<float4*>(a + 4 * i) = __ldg(reinterpret_cast<const float4*>(src) + i);
        *reinterpret_cast<float4*>(b + 4 * i) = __ldg(reinterpret_cast<const float4*>(src + half) + i);
    }
    if (cos_t && head < n_heads + n_kv) {
        const float* cp = cos_t + (int64_t)pos * half + 8 * ch;
        const float* sp = sin_t + (int64_t)pos * half + 8 * ch;
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            *reinterpret_cast<float4*>(c + 4 * i) = __ldg(reinterpret_cast<const float4*>(cp) + i);
            *reinterpret_cast<float4*>(s + 4 * i) = __ldg(reinterpret_cast<const float4*>(sp) + i);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = a[i], y = b[i];
            a[i] = x * c[i] - y * s[i];
            b[i] = y * c[i] + x * s[i];
        }
    }
    T* dst;
    if (head < n_heads) {
        dst = q_out + row * q_stride + (int64_t)head * cache.d_head;
    } else {
        const int kvh = head - n_heads < n_kv ? head - n_heads : head - n_heads - n_kv;
        const int page = sl / cache.page_size, off = sl - page * cache.page_size;
        T* base = static_cast<T*>(head - n_heads < n_kv ? cache.k : cache.v);
        dst = base + page * cache.page_stride + off * cache.slot_stride + kvh * cache.head_stride;
    }
    Pack8<T>::store(dst + 8 * ch, a);
    Pack8<T>::store(dst + half + 8 * ch, b);
}

// h[r] = embed[token] (+ pos_embed[position of r]); a token outside the vocabulary and a padded row give zeros
__global__ void __launch_bounds__(256)
embed_rows_kernel(const int32_t* __restrict__ tokens, const int32_t* __restrict__ row_pos, const float* __restrict__ embed,
                  const float* __restrict__ pos_embed, int d, int vocab, int max_pos, float* __restrict__ h, int32_t* __restrict__ err_flag) {
    const int r = blockIdx.x;
    const int tok = tokens[r], pos = row_pos[r];
    const bool live = pos >= 0 && pos < max_pos && tok >= 0 && tok < vocab;
    if (threadIdx.x == 0 && pos >= max_pos) atomicExch(err_flag, kErrBadSlot);
    for (int i = threadIdx.x; i < d; i += 256) {
        float x = 0.0f;
        if (live) {
            x = embed[(size_t)tok * d + i];
            if (pos_embed) x += pos_embed[(size_t)pos * d + i];
        }
        h[(size_t)r * d + i] = x;
    }
}

template <typename T>
__global__ void __launch_bounds__(256)
widen_kernel(const T* __restrict__ src, float* __restrict__ dst, int n8) {
    grid_dependency_wait();
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n8) return;
    const uint4 w = reinterpret_cast<const uint4*>(src)[i];
    const T* v = reinterpret_cast<const T*>(&w);
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = static_cast<float>(v[e]);
    Pack8<float>::store(dst + 8 * (size_t)i, f);
}

}  // namespace

int launch_cache_plan(const CachePlanArgs& a, cudaStream_t s) {
    PlanParams p{a.cached_len, a.new_len, a.batch, a.page_size, a.n_pages, a.max_pages, a.free_pages, a.free_capacity, a.n_free,
                 a.block_table, a.parents, a.max_rows, a.mask_words, a.kv_len, a.row_start, a.row_request, a.row_pos, a.slot,
                 a.tree_mask, a.n_free_out, a.status};
    const size_t smem = (size_t)2 * (a.batch + 1) * sizeof(int32_t);
    if (a.batch > kMaxPlanBatch) return -1;
    static DeviceOnce attr;
    if (!attr.done([] { return allow_smem(cache_plan_kernel, (int)(2 * (kMaxPlanBatch + 1) * sizeof(int32_t))); })) return -1;
    // one row (and its tables' share) a thread up to a wave of the 148 SMs
    int grid = (a.max_rows + kPlanThreads - 1) / kPlanThreads;
    grid = grid < 1 ? 1 : (grid > 148 ? 148 : grid);
    cache_plan_kernel<<<grid, kPlanThreads, smem, s>>>(p);
    count_launch();
    return 0;
}

void launch_cache_append(const float* qkv, int64_t ld, const int32_t* row_pos, const int32_t* slot, int rows, int n_heads,
                         const float* cos_t, const float* sin_t, int max_pos, const PagedCache& cache, void* q_out, int64_t q_stride,
                         int32_t* err_flag, cudaStream_t s, bool dependent) {
    const int items = (n_heads + 2 * cache.n_kv_heads) * (cache.d_head / 16);
    const dim3 grid(rows, (items + 255) / 256);
#define ZQ_APPEND(T) launch_kernel(cache_append_kernel<T>, grid, dim3(256), 0, s, dependent, qkv, ld, row_pos, slot, n_heads, cos_t, \
                                   sin_t, max_pos, cache, static_cast<T*>(q_out), q_stride, err_flag)
    if (cache.type == kTypeF32) ZQ_APPEND(float);
    else if (cache.type == kTypeBf16) ZQ_APPEND(__nv_bfloat16);
    else ZQ_APPEND(__half);
#undef ZQ_APPEND
    count_launch();
}

void launch_embed_rows(const int32_t* tokens, const int32_t* row_pos, const float* embed, const float* pos_embed, int rows, int d, int vocab,
                       int max_pos, float* h, int32_t* err_flag, cudaStream_t s) {
    embed_rows_kernel<<<rows, 256, 0, s>>>(tokens, row_pos, embed, pos_embed, d, vocab, max_pos, h, err_flag);
    count_launch();
}

void launch_widen(const void* src, int type, int64_t n, float* dst, cudaStream_t s) {
    const int n8 = (int)(n / 8);
    if (type == kTypeBf16) launch_kernel(widen_kernel<__nv_bfloat16>, dim3((n8 + 255) / 256), dim3(256), 0, s, true, static_cast<const __nv_bfloat16*>(src), dst, n8);
    else launch_kernel(widen_kernel<__half>, dim3((n8 + 255) / 256), dim3(256), 0, s, true, static_cast<const __half*>(src), dst, n8);
    count_launch();
}

}  // namespace zq
