// The states of beams follow the ones that go on: block tables, pages given back and taken, token histories, and the copies of
// half-filled pages in every layer's cache.
//
// Row j of a request continues its row parent[j].  Whole pages are shared by all rows that descend from them and are never copied.
// The page that a row is still filling can have one owner: the first child in row order keeps it, every further child gets a page of its
// own with a copy of the slots filled so far, and so does the first where a longer row goes on that holds the page whole.  A page that no row
// holds any more goes back.  Nothing is counted over steps: all holders of a page are rows of one request and hold it in the same column of their
// tables (pages shared with other requests lie below shared_len and are left alone), so comparing a column before and after says which pages are gone.
//
//   beam_count_kernel   a CTA per request counts pages given back and wanted; further CTAs copy tables and histories meanwhile
//   beam_place_kernel   (dependent launch) every CTA sums the counts of the requests before its own, lists its pages in the order column,
//                       row, hands them to its new rows and writes what is left behind the free pages
// The order of all lists is fixed by rows and columns, so the same call gives the same pages.
//   beam_reorder_kernel both in one, for few requests
//   cache_copy_kernel   slots of pages, for all layers in one launch; bound by memory
// 64 requests of eight beams, 100 to 2000 tokens, and the copies of 16 layers (two rows in five get one, 452 MB read and written): 78 us replayed, 69 those bytes at the
// rate of a copy.
#include "common.cuh"
#include "serve.cuh"

namespace zq {
namespace {

constexpr int kThreads = 256, kFew = 4;      // requests that one launch serves

struct ReorderParams {
    ReorderArgs a;
    int32_t* counts;                         // [batch][2]: pages given back, pages wanted
};

// What a CTA knows of its request, in shared memory.
struct Request {
    int len[kMaxBeams], held[kMaxBeams];     // of the old rows
    int parent[kMaxBeams];                   // of the new rows, -1: none
    unsigned full, kept;                     // old rows with a child; old rows whose unfinished page a child keeps
    unsigned copies;                         // new rows that get a copy of their parent's unfinished page
    int shared, status;
};

// By one warp.
__device__ __forceinline__ void read_request_warp(const ReorderArgs& a, int b, Request& r) {
    const int lane = threadIdx.x & 31, K = a.beams, P = a.page_size;
    const bool mine = lane < K;
    int bad = 0;
    int len = mine ? __ldg(a.kv_len + (int64_t)b * K + lane) : 0, parent = mine ? __ldg(a.parent + (int64_t)b * K + lane) : -1;
    if (len < 0 || len > (int64_t)a.max_pages * P) { len = 0; bad |= kPlanBadLength; }
    if (parent < -1 || parent >= K) { parent = -1; bad |= kPlanBadParent; }
    int shared = a.shared_len ? __ldg(a.shared_len + b) : 0;
    if (shared < 0) { shared = 0; bad |= kPlanBadLength; }
    const int new_len = __shfl_sync(0xffffffffu, len, parent < 0 ? 0 : parent);
    const bool part = parent >= 0 && new_len % P != 0;
    const int last = new_len / P;                                // < max_pages: the page exists
    const int page = part ? __ldg(a.block_table + ((int64_t)b * K + parent) * a.max_pages + last) : -1;
    bool keep = part && (int64_t)last * P >= shared;
    for (int j = 0; j < K; ++j) {
        const int pg = __shfl_sync(0xffffffffu, page, j), lt = __shfl_sync(0xffffffffu, last, j), of = __shfl_sync(0xffffffffu, parent, j);
        const bool pt = __shfl_sync(0xffffffffu, (int)part, j);
        if (j < lane && pt && pg == page && lt == last) keep = false;
        // a longer row may hold the page whole, and what a shorter one adds would fall among its keys
        if (keep && of >= 0 && lt > last && __ldg(a.block_table + ((int64_t)b * K + of) * a.max_pages + last) == page) keep = false;
    }
    if (part && (page < 0 || page >= a.n_pages)) { bad |= kPlanBadPage; keep = true; }      // nothing to copy from
    if (mine) { r.len[lane] = len; r.held[lane] = len / P + (len % P != 0); r.parent[lane] = parent; }
    const unsigned copies = __ballot_sync(0xffffffffu, part && !keep);
    const unsigned full = __reduce_or_sync(0xffffffffu, parent >= 0 ? 1u << parent : 0u);
    const unsigned kept = __reduce_or_sync(0xffffffffu, keep ? 1u << parent : 0u);
    bad = __reduce_or_sync(0xffffffffu, (unsigned)bad);
    if (lane == 0) { r.full = full; r.kept = kept; r.copies = copies; r.shared = shared; r.status = bad; }
}
// Called by all threads; the first warp fills `r`.  Ends with a barrier.
__device__ __forceinline__ void read_request(const ReorderArgs& a, int b, Request& r) {
    if (threadIdx.x < 32) read_request_warp(a, b, r);
    __syncthreads();
}

// Old rows whose page in column c is given back with this call, as bits.
__device__ __forceinline__ unsigned pages_gone(const ReorderArgs& a, const Request& r, int64_t row0, int c) {
    if ((int64_t)c * a.page_size < r.shared) return 0;
    const int32_t* at = a.block_table + row0 * a.max_pages + c;
    unsigned has = 0, stays = 0;                                 // rows with a page there; whose page goes on
    for (int p = 0; p < a.beams; ++p) {
        if (c >= r.held[p]) continue;
        has |= 1u << p;
        const bool filling = r.len[p] % a.page_size != 0 && c == r.held[p] - 1;
        if (((filling ? r.kept : r.full) >> p) & 1u) stays |= 1u << p;
    }
    unsigned gone = has & ~stays;
    for (unsigned m = gone; m; m &= m - 1) {
        const int p = __ffs(m) - 1, page = __ldg(at + (int64_t)p * a.max_pages);
        bool other = page < 0 || page >= a.n_pages;              // (not a page: nothing to give back)
        for (unsigned o = stays | (has & ((1u << p) - 1u)); o && !other; o &= o - 1)
            other = __ldg(at + (int64_t)(__ffs(o) - 1) * a.max_pages) == page;
        if (other) gone &= ~(1u << p);
    }
    return gone;
}

// Sums over the block (called by all threads; part: N words a warp; ends with a barrier).
template <int N>
__device__ __forceinline__ void block_sums(int (&x)[N], int* part) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = __reduce_add_sync(0xffffffffu, x[i]);
        if ((threadIdx.x & 31) == 0) part[(threadIdx.x >> 5) * N + i] = x[i];
        x[i] = 0;
    }
    __syncthreads();
    for (int w = 0; w < kThreads / 32; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += part[w * N + i];
    __syncthreads();
}

// Tables and histories, row by row: rows first, first + step, ... of a request.
__device__ __forceinline__ void move_rows(const ReorderArgs& a, const Request& r, int64_t row0, int first, int step) {
    const int tid = threadIdx.x;
    for (int j = first; j < a.beams; j += step) {
        const int from = r.parent[j];
        const int64_t src = row0 + (from < 0 ? 0 : from), dst = row0 + j;
        const int n = from < 0 ? 0 : r.held[from], skip = (r.copies >> j) & 1u ? n - 1 : -1;      // (a copied page's entry is another's to write)
        int bad = 0;
        for (int c = tid; c < n; c += kThreads) {
            const int page = __ldg(a.block_table + src * a.max_pages + c);
            if (page < 0 || page >= a.n_pages) bad = kPlanBadPage;
            if (c != skip) a.table_out[dst * a.max_pages + c] = page;
        }
        if (a.history) {
            int64_t h = from < 0 ? 0 : __ldg(a.history_len + src);
            const int64_t room = a.history_stride - (a.token ? 1 : 0);
            if (h < 0 || h > room) { bad |= kPlanBadLength; h = 0; }
            for (int64_t i = tid; i < h; i += kThreads) a.history_out[dst * a.history_stride + i] = __ldg(a.history + src * a.history_stride + i);
            if (tid == 0) {
                const bool more = a.token && from >= 0 && h <= room;
                if (more) a.history_out[dst * a.history_stride + h] = __ldg(a.token + dst);
                a.history_len_out[dst] = (int)h + (more ? 1 : 0);
            }
        }
        if (bad) atomicOr(a.status, bad);
    }
}

__global__ void __launch_bounds__(kThreads)
beam_count_kernel(const ReorderParams p) {
    __shared__ Request r;
    __shared__ int part[kThreads / 32];
    const ReorderArgs& a = p.a;
    const int b = blockIdx.x, K = a.beams, tid = threadIdx.x;
    const int64_t row0 = (int64_t)b * K;
    grid_dependency_release();                                   // the second launch may get ready
    read_request(a, b, r);
    if (blockIdx.y == 0) {
        int most = 0, n[1] = {0};
        for (int k = 0; k < K; ++k) most = max(most, r.held[k]);
        for (int c = tid; c < most; c += kThreads) n[0] += __popc(pages_gone(a, r, row0, c));
        block_sums(n, part);
        if (tid == 0) {
            p.counts[2 * b] = n[0];
            p.counts[2 * b + 1] = __popc(r.copies);
            if (r.status) atomicOr(a.status, r.status);
        }
        return;
    }
    move_rows(a, r, row0, blockIdx.y - 1, gridDim.y - 1);
}

// Gives the request's new rows their pages and lists those it gives back; counts: [batch][2], first: rows that give back a page in column threadIdx.x, part: 4 words a warp.
__device__ __forceinline__ void place_pages(const ReorderArgs& a, const Request& r, int b, const int32_t* counts, int n_free, unsigned first, int* part, int* mine) {
    const int K = a.beams, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row0 = (int64_t)b * K;
    int sums[4] = {0, 0, 0, 0}, most = 0;                        // pages taken from the free ones and given to them, by all requests and by those before this one
    for (int i = tid; i < a.batch; i += kThreads) {
        const int gone = counts[2 * i], want = counts[2 * i + 1], inside = min(gone, want);
        sums[0] += want - inside;
        sums[1] += gone - inside;
        if (i < b) { sums[2] += want - inside; sums[3] += gone - inside; }
    }
    block_sums(sums, part);
    const int taken = sums[0], given = sums[1], taken_before = sums[2], given_before = sums[3];
    const int own_gone = counts[2 * b], own_want = counts[2 * b + 1], inside = min(own_gone, own_want);
    // nothing is reordered where lengths are impossible or pages are short
    int bad = n_free < 0 || n_free > a.free_capacity ? kPlanBadLength : 0;
    if (bad) n_free = 0;
    else if (taken > n_free) bad = kPlanNoPages;
    else if (n_free - taken + given > a.free_capacity) bad = kPlanBadLength;
    const int left = bad ? n_free : n_free - taken;
    if (b == 0 && tid == 0) {
        *a.n_free_out = bad ? n_free : left + given;
        if (bad) atomicOr(a.status, bad);
    }
    for (int i = b * kThreads + tid; i < left; i += gridDim.x * kThreads) a.free_out[i] = __ldg(a.free_pages + i);
    for (int k = 0; k < K; ++k) most = max(most, r.held[k]);
    // pages given back, in the order column, row: the first `inside` go to the request's own new rows
    int done = 0;
    for (int c0 = 0; c0 < most && own_gone > 0 && !bad; c0 += kThreads) {
        const int c = c0 + tid;
        const unsigned gone = c0 == 0 ? first : (c < most ? pages_gone(a, r, row0, c) : 0u);
        int n = __popc(gone), up = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, up, o);
            if (lane >= o) up += v;
        }
        if (lane == 31) part[warp] = up;
        __syncthreads();
        int all = 0;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w == warp) up += all;
            all += part[w];
        }
        int at = done + up - n;
        for (unsigned m = gone; m; m &= m - 1, ++at) {
            const int page = __ldg(a.block_table + (row0 + __ffs(m) - 1) * a.max_pages + c);
            if (at < inside) mine[at] = page;
            else a.free_out[left + given_before + at - inside] = page;
        }
        done += all;
        __syncthreads();
    }
    __syncthreads();
    if (tid < K) {
        const int64_t row = row0 + tid;
        const int from = r.parent[tid], n = from < 0 || bad ? 0 : r.len[from];
        const bool copy = !bad && ((r.copies >> tid) & 1u);
        int src = -1, dst = -1, len = 0;
        if (copy) {
            const int rank = __popc(r.copies & ((1u << tid) - 1u)), c = n / a.page_size;
            src = __ldg(a.block_table + (row0 + from) * a.max_pages + c);
            dst = rank < inside ? mine[rank] : __ldg(a.free_pages + n_free - 1 - taken_before - (rank - inside));
            len = n % a.page_size;
            a.table_out[row * a.max_pages + c] = dst;
            if (dst < 0 || dst >= a.n_pages) atomicOr(a.status, kPlanBadPage);
        }
        a.kv_len_out[row] = n;
        a.copy_from[row] = src;
        a.copy_to[row] = dst;
        a.copy_len[row] = len;
    }
}

__global__ void __launch_bounds__(kThreads)
beam_place_kernel(const ReorderParams p) {
    __shared__ Request r;
    __shared__ int part[4 * kThreads / 32];
    __shared__ int mine[kMaxBeams];                              // pages that the request's own new rows take over
    const ReorderArgs& a = p.a;
    read_request(a, blockIdx.x, r);                              // (inputs only: may run ahead of the counts)
    const int n_free = __ldg(a.n_free);
    bool held = false;
    for (int k = 0; k < a.beams; ++k) held = held || (int)threadIdx.x < r.held[k];
    const unsigned first = held ? pages_gone(a, r, (int64_t)blockIdx.x * a.beams, threadIdx.x) : 0u;
    grid_dependency_wait();
    place_pages(a, r, blockIdx.x, p.counts, n_free, first, part, mine);
}

// Few requests: every CTA counts for all of them itself, its warps shared out, so one launch does it.  1 / 4 / 8 requests of four beams with up to 2000 tokens, with the copies of
// 24 layers: called from Python 21.9 / 21.8 / 21.9 us against 24.6 / 24.4 / 24.3 with two launches, replayed from a graph, where a launch costs the host nothing, 8.3 / 13.8 / 15.5
// against 9.0 / 12.4 / 13.3: calls gain 3 us with up to four requests, replays lose up to 1.4 with more than one.
__global__ void __launch_bounds__(kThreads)
beam_reorder_kernel(const ReorderParams p) {
    __shared__ Request all[kFew];
    __shared__ int32_t counts[2 * kFew];
    __shared__ int part[4 * kThreads / 32];
    __shared__ unsigned gone_s[kThreads];                        // of this CTA's request, by column
    __shared__ int mine[kMaxBeams];
    const ReorderArgs& a = p.a;
    const int b = blockIdx.x, K = a.beams, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (blockIdx.y > 0) {
        read_request(a, b, all[0]);
        move_rows(a, all[0], (int64_t)b * K, blockIdx.y - 1, gridDim.y - 1);
        return;
    }
    const int n_free = __ldg(a.n_free);
    if (tid < 2 * a.batch) counts[tid] = 0;
    gone_s[tid] = 0;
    if (warp < a.batch) read_request_warp(a, warp, all[warp]);
    __syncthreads();
    const int share = kThreads / 32 / a.batch, of = warp / share;          // warps of a request
    if (of < a.batch) {
        const Request& r = all[of];
        int most = 0, n = 0;
        for (int k = 0; k < K; ++k) most = max(most, r.held[k]);
        for (int c = (warp - of * share) * 32 + lane; c < most; c += 32 * share) {
            const unsigned gone = pages_gone(a, r, (int64_t)of * K, c);
            if (of == b) gone_s[c] = gone;
            n += __popc(gone);
        }
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) {
            atomicAdd(counts + 2 * of, n);
            if (warp == of * share) counts[2 * of + 1] = __popc(r.copies);
            if (warp == b * share && r.status) atomicOr(a.status, r.status);
        }
    }
    __syncthreads();
    place_pages(a, all[b], b, counts, n_free, gone_s[tid], part, mine);
}

// ---- copies ---------------------------------------------------------------------------------------------------------
struct CopyParams {
    void* kv[2 * kCopyLayers];               // k and v of every layer
    PagedCache shape;                        // strides and sizes of all of them, in elements
    const int32_t *from, *to, *len;
    int32_t* err_flag;
    int row_shift;                           // log2 of the 16-byte chunks of a head
    int slots_inside;                        // a head's slots stand closer than a slot's heads: walk them first
};

// A CTA copies a share of a page's slots in one layer's K or V: rows of d_head elements, four 16-byte chunks of a thread in flight.
__global__ void __launch_bounds__(kThreads)
cache_copy_kernel(const CopyParams p) {
    const int row = blockIdx.x, len = __ldg(p.len + row);
    if (len == 0) return;
    const int from = __ldg(p.from + row), to = __ldg(p.to + row);
    if (len < 0 || len > p.shape.page_size || from < 0 || from >= p.shape.n_pages || to < 0 || to >= p.shape.n_pages || from == to) {
        if (threadIdx.x == 0) atomicExch(p.err_flag, kErrBadPage);
        return;
    }
    const int chunks = 1 << p.row_shift, chunk = threadIdx.x & (chunks - 1), step = kThreads >> p.row_shift;
    const int inner = p.slots_inside ? len : p.shape.n_kv_heads, total = len * p.shape.n_kv_heads;
    const int e = p.shape.type == kTypeF32 ? 4 : 2;
    uint8_t* base = static_cast<uint8_t*>(p.kv[blockIdx.y]) + 16 * chunk;
    const uint8_t* src = base + from * p.shape.page_stride * e;
    uint8_t* dst = base + to * p.shape.page_stride * e;
    const int64_t outer_stride = (p.slots_inside ? p.shape.head_stride : p.shape.slot_stride) * e, inner_stride = (p.slots_inside ? p.shape.slot_stride : p.shape.head_stride) * e;
    for (int r0 = blockIdx.z * 4 * step + (threadIdx.x >> p.row_shift); r0 < total; r0 += gridDim.z * 4 * step) {
        uint4 w[4];
        int64_t at[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = r0 + u * step, o = r / inner;
            at[u] = o * outer_stride + (r - o * inner) * inner_stride;
            if (r < total) w[u] = *reinterpret_cast<const uint4*>(src + at[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (r0 + u * step < total) *reinterpret_cast<uint4*>(dst + at[u]) = w[u];
    }
}

}  // namespace

size_t beam_reorder_scratch_bytes(int batch) { return (size_t)batch * 2 * sizeof(int32_t); }

int launch_beam_reorder(const ReorderArgs& a, void* scratch, cudaStream_t s) {
    ReorderParams p{a, static_cast<int32_t*>(scratch)};
    const int y = 1 + (a.beams < 148 * 4 / a.batch ? a.beams : (a.beams + 3) / 4);
    // one launch while a request's warps get through its columns in a few rounds (the second launch costs the host 2 us and the device 4)
    if (a.batch <= kFew && a.max_pages <= kThreads) {
        if (launch_kernel(beam_reorder_kernel, dim3(a.batch, y), dim3(kThreads), 0, s, false, p) != cudaSuccess) return -1;
        count_launch();
        return 0;
    }
    if (launch_kernel(beam_count_kernel, dim3(a.batch, y), dim3(kThreads), 0, s, false, p) != cudaSuccess) return -1;
    count_launch();
    if (launch_kernel(beam_place_kernel, dim3(a.batch), dim3(kThreads), 0, s, true, p) != cudaSuccess) return -1;
    count_launch();
    return 0;
}

int launch_cache_copy(const PagedCache* caches, int n_layers, const int32_t* from, const int32_t* to, const int32_t* len, int rows, int32_t* err_flag,
                      cudaStream_t s) {
    for (int l0 = 0; l0 < n_layers;) {
        CopyParams p{};
        p.shape = caches[l0];
        int n = 0;
        for (; n < kCopyLayers && l0 + n < n_layers; ++n) {      // a launch takes the layers that look alike
            const PagedCache& c = caches[l0 + n];
            if (c.type != p.shape.type || c.n_pages != p.shape.n_pages || c.page_size != p.shape.page_size || c.n_kv_heads != p.shape.n_kv_heads ||
                c.d_head != p.shape.d_head || c.page_stride != p.shape.page_stride || c.slot_stride != p.shape.slot_stride || c.head_stride != p.shape.head_stride)
                break;
            p.kv[2 * n] = c.k;
            p.kv[2 * n + 1] = c.v;
        }
        p.from = from; p.to = to; p.len = len; p.err_flag = err_flag;
        const int bytes = p.shape.d_head * type_bytes(p.shape.type);
        p.row_shift = bytes == 512 ? 5 : (bytes == 256 ? 4 : 3);
        p.slots_inside = p.shape.slot_stride < p.shape.head_stride;
        const int64_t page = (int64_t)p.shape.page_size * p.shape.n_kv_heads * bytes;
        const int z = page <= 65536 ? 1 : (int)((page + 65535) / 65536 < 64 ? (page + 65535) / 65536 : 64);
        if (launch_kernel(cache_copy_kernel, dim3(rows, 2 * n, z), dim3(kThreads), 0, s, false, p) != cudaSuccess) return -1;
        count_launch();
        l0 += n;
    }
    return 0;
}

}  // namespace zq
