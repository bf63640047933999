// Work distribution of the attention kernels over a paged cache, shared by the CUDA-core and the tensor-core kernel.
//
// For request b with n new rows and L keys (C = L - n of them cached before this step, the drafts last) and g = n_heads /
// n_kv_heads query heads per key head, the queries that read one key head are the n * g vectors (draft i, head in group) in
// this order, cut into row tiles.  An item is (request, key head, row tile), its work the number of key tiles and a constant
// for opening and closing it (in tiles' time: without it the CTAs that get short contexts finish last; 16 x 32 heads of 100 to 2047
// keys at d_head 64, constants of 0 / 2 / 4 / 6: 98 / 70 / 62 / 61 us, 32 x 8 of 4096 at 128: 107 / 108 / 109 / 112).  All items' work, laid out one after the other, is cut into gridDim.x equal runs, one per CTA: long
// contexts are split over as many CTAs as it takes, short ones are packed, and no length is needed on the host.  Every CTA
// finds its run by scanning the requests' lengths.  A piece of an item that is not the whole item leaves (reference, sum, output) per
// query in the scratch, at most two pieces per CTA, and tree_combine_kernel joins them in the order of the keys, so results
// do not depend on timing.
#pragma once
#include "common.cuh"
#include "serve.cuh"
#include <cuda_fp16.h>

namespace zq {

constexpr int kKeys = 128;                               // keys of a key tile: the tensor-core kernels'
constexpr int kNarrowKeys = 32, kNarrowRows = 8, kNarrowWarps = 12;      // the warps' kernel (prefix_narrow.cu): a run per warp
constexpr int kF32Rows = 8, kF32Border = 32, kF32Warps = 10;             // its fp32 sibling (prefix_narrow_f32.cu); the border between parts

// A request's part of the work: n rows from row0 on, keys up to L, in n_rt row tiles and the key tiles [first_tile(), n_kt); n_rt * n_kt = 0: nothing to do.
// drafts(): how many of the last keys are the rows' own.  table(b): its row of the block table.
struct TreeRequest {
    int n, L, row0, n_rt, n_kt;
    __device__ __forceinline__ int first_tile() const { return 0; }
    __device__ __forceinline__ int drafts() const { return n; }
    __device__ __forceinline__ int table(int b) const { return b; }
};

struct TreeWork {
    using Request = TreeRequest;
    static constexpr bool kPrefix = false;
    const int32_t *kv_len, *row_start, *block_table;
    int batch, rows, n_kv, max_pages, page_size;
    int group;               // query heads per key head
    int tile_rows;           // queries per row tile
    int key_tile;            // keys per key tile
    int item_cost;           // work of an item besides its key tiles, in tiles
    int32_t* err_flag;
};

__device__ __forceinline__ TreeRequest tree_request(const TreeWork& w, int b) {
    TreeRequest r;
    r.row0 = __ldg(w.row_start + b);
    r.n = __ldg(w.row_start + b + 1) - r.row0;
    r.L = __ldg(w.kv_len + b);
    if (r.n <= 0 || r.row0 < 0 || r.n > r.L || r.row0 > w.rows - r.n || r.L > (long long)w.max_pages * w.page_size) {
        if (r.n != 0) atomicExch(w.err_flag, kErrBadRequest);
        r.n = r.n_rt = r.n_kt = 0;
        return r;
    }
    r.n_rt = (int)(((long long)r.n * w.group + w.tile_rows - 1) / w.tile_rows);
    r.n_kt = (r.L + w.key_tile - 1) / w.key_tile;
    return r;
}

// ---- a long prefix shared by groups of requests ---------------------------------------------------------------------
// The work list then holds, for every group, one part over the keys that all of its requests share - all their rows in row tiles, every key
// seen by all - and, for every request, one part over the keys behind them.  The border is the shared length rounded down to whole key
// tiles: the few shared keys behind it are read by every request through its own block table, which names the same pages (a border
// inside a tile would cost each request a tile with masked keys instead).  Both parts leave (reference, sum, output) of their rows, joined by
// prefix_join_kernel (prefix_attention.cu).
struct PrefixRequest : TreeRequest {
    int kt0, row, own;                       // first tile, row of the block table, 1: the part of one request
    __device__ __forceinline__ int first_tile() const { return kt0; }
    __device__ __forceinline__ int drafts() const { return own ? n : 0; }
    __device__ __forceinline__ int table(int) const { return row; }
};
struct PrefixWork : TreeWork {               // batch: parts in this launch
    using Request = PrefixRequest;
    static constexpr bool kPrefix = true;
    const int32_t *group_start, *prefix_len, *request_group;
    int groups, requests;
    int border;                              // keys that the border is a multiple of: a multiple of every key tile in use
    int first;                               // the launch's first part: 0 .. groups - 1 are groups, then come the requests
    int* row_sides;                          // [rows]
    bool late_wait;                          // the launch before left nothing that this one reads: waited for at the end
    // Where groups and requests go to different kernels, the two launches share the SMs out (prefix_share); other_time = 0: the launch has them all.
    int tile_time, other_time;               // of a key tile on an SM, here and in the other launch, in the same unit
    int other_rows, other_keys, other_cost;  // tile_rows, key_tile, item_cost of the other launch
    int2* entries;                           // [2][rows * heads]: where a query's shared (0) and own (1) pieces are
    float* partial;                          // [2][rows * heads][d_head + 4]: output, reference, sum of parts that one CTA finished
};
// a / b rounded down or up for a power of two b
__device__ __forceinline__ int prefix_down(int a, int b) { return a >> (31 - __clz(b)); }
__device__ __forceinline__ int prefix_up(int a, int b) { return (int)(((unsigned)a + (unsigned)b - 1u) >> (31 - __clz(b))); }

// A prefix is read through the table of the group's first request that has rows and holds its shared keys.  (The row of a request without rows says nothing: it may have ended, and
// its pages be others' by now.)  Where no request holds them, each contradicts the group, and no row takes what comes of the shared part: any row of the table will do.
// Not inlined: the attention kernels meet parts in many places, and all of this in each of them costs 4 us of 70 (8 groups of 32 queries a key head behind 8000 keys).
static __device__ __noinline__ int prefix_row(const int32_t* group_start, const int32_t* prefix_len, const int32_t* request_group, const int32_t* row_start, const int32_t* kv_len,
                                              int rows, long long most, int g) {
    const int b0 = __ldg(group_start + g), b1 = __ldg(group_start + g + 1), len = __ldg(prefix_len + g);
    for (int b = b0; b < b1; ++b) {
        const int at = __ldg(row_start + b), n = __ldg(row_start + b + 1) - at, have = __ldg(kv_len + b), of = __ldg(request_group + b);
        if (n > 0 && at >= 0 && at <= rows - n && of == g && have <= most && len <= (long long)have - n) return b;
        if (n != 0) continue;
        int lo = b, hi = b1;                 // a run of requests without rows: lo is the last one known of, or b1 - 1
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (__ldg(row_start + mid + 1) == at) lo = mid;
            else hi = mid;
        }
        b = lo;
    }
    return b0;
}
// The shared part of group g, its table not looked for; n_kt = 0: it has none, or (ok = false) its description contradicts itself.
__device__ __forceinline__ PrefixRequest prefix_shared(const PrefixWork& w, int g, bool& ok) {
    PrefixRequest r{};
    const int b0 = __ldg(w.group_start + g), b1 = __ldg(w.group_start + g + 1), len = __ldg(w.prefix_len + g);
    ok = b0 >= 0 && b1 >= b0 && b1 <= w.requests;
    if (!ok) return r;
    const int lo = __ldg(w.row_start + b0), n = __ldg(w.row_start + b1) - lo;
    if (n == 0) return r;                    // (a group without rows may have any length)
    ok = lo >= 0 && n > 0 && lo <= w.rows - n && len >= 0 && len <= (long long)w.max_pages * w.page_size;
    if (!ok) return r;
    r.row0 = lo; r.n = n;
    r.L = prefix_down(len, w.border) * w.border;
    r.n_rt = prefix_up(n * w.group, w.tile_rows);
    r.n_kt = prefix_down(r.L, w.key_tile);
    return r;
}
// The part of request b alone; its group's description is prefix_shared's to check.
__device__ __forceinline__ PrefixRequest prefix_own(const PrefixWork& w, int b, bool& ok) {
    PrefixRequest r{};
    const int g = __ldg(w.request_group + b), end = __ldg(w.row_start + b + 1);
    r.row0 = __ldg(w.row_start + b);
    r.L = __ldg(w.kv_len + b);
    const bool grouped = g >= 0 && g < w.groups;
    const int of = grouped ? g : 0, len = __ldg(w.prefix_len + of), b0 = __ldg(w.group_start + of), b1 = __ldg(w.group_start + of + 1);     // (all on their way at once)
    r.n = end - r.row0;
    r.row = b; r.own = 1;
    // (a request without rows may say anything: it may have ended)
    ok = r.n == 0 || (r.n > 0 && r.row0 >= 0 && r.row0 <= w.rows - r.n && r.L <= (long long)w.max_pages * w.page_size && grouped && b0 <= b && b < b1 && len >= 0 &&
                      len <= (long long)r.L - r.n);
    if (!ok || r.n == 0) { r.n = 0; return r; }
    r.kt0 = prefix_down(prefix_down(len, w.border) * w.border, w.key_tile);
    r.n_rt = prefix_up(r.n * w.group, w.tile_rows);
    r.n_kt = prefix_up(r.L, w.key_tile);
    return r;
}
__device__ __forceinline__ PrefixRequest tree_request(const PrefixWork& w, int part) {
    bool ok;
    part += w.first;
    const PrefixRequest r = part < w.groups ? prefix_shared(w, part, ok) : prefix_own(w, part - w.groups, ok);
    if (!ok) atomicExch(w.err_flag, kErrBadRequest);
    return r;
}
__device__ __forceinline__ void prefix_find_row(const PrefixWork& w, int part, PrefixRequest& r) {
    if (r.own || r.n_kt == 0) return;
    r.row = prefix_row(w.group_start, w.prefix_len, w.request_group, w.row_start, w.kv_len, w.rows, (long long)w.max_pages * w.page_size, w.first + part);
}
// Where the query's piece is: whole in `partial` (y = -1), or query y of the pieces of the CTAs x & 0xFFFF .. x >> 16.
__device__ __forceinline__ int64_t prefix_query(const PrefixWork& w, const PrefixRequest& r, int query, int h) {
    const int token = query / w.group;
    return ((int64_t)r.own * w.rows + r.row0 + token) * ((int64_t)w.n_kv * w.group) + (int64_t)h * w.group + (query - token * w.group);
}

// The prefix part of a work description: `parts` of them from `first` on.
inline void prefix_work(const PrefixAttnArgs& a, const PrefixScratch& at, int first, int parts, PrefixWork& w) {
    w.border = a.t.cache.type == kTypeF32 ? kF32Border : kKeys;
    w.group_start = a.group_start; w.prefix_len = a.prefix_len; w.request_group = a.request_group;
    w.groups = a.groups; w.requests = a.t.batch; w.first = first; w.batch = parts;
    w.entries = static_cast<int2*>(at.entries); w.partial = at.partial; w.row_sides = at.row_sides;
}

// Position in the sequence of key tiles.  next() moves on by one tile; tiles of requests without work do not exist.
template <class W> struct TreeCursorT {
    typename W::Request r;
    int b, h, rt, kt;
    __device__ __forceinline__ void load(const W& w) { r = tree_request(w, b); }
    // first query of the row tile and how many it has
    __device__ __forceinline__ int first_query(const W& w) const { return rt * w.tile_rows; }
    __device__ __forceinline__ int queries(const W& w) const { return min(w.tile_rows, r.n * w.group - rt * w.tile_rows); }
    __device__ __forceinline__ bool item_begins() const { return kt == r.first_tile(); }
    __device__ __forceinline__ bool item_ends() const { return kt == r.n_kt - 1; }
    __device__ __forceinline__ void next(const W& w) {
        if (++kt < r.n_kt) return;
        kt = r.first_tile();
        if (++rt < r.n_rt) return;
        rt = 0;
        if (++h < w.n_kv) return;
        h = 0;
        do { if (++b >= w.batch) return; load(w); } while (r.n_kt == 0);
        kt = r.first_tile();
    }
};
using TreeCursor = TreeCursorT<TreeWork>;
// next() for whoever looks pages up
__device__ __forceinline__ void tree_next(const TreeWork& w, TreeCursor& c) { c.next(w); }
__device__ __forceinline__ void tree_next(const PrefixWork& w, TreeCursorT<PrefixWork>& c) {
    const int b = c.b;
    c.next(w);
    if (c.b != b && c.b < w.batch) prefix_find_row(w, c.b, c.r);
}

// a / b for a >= 0, b > 0; almost always in 32 bits, which is several times faster
__device__ __forceinline__ long long tree_div(long long a, long long b) {
    return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}

// The run of a CTA: the tiles [begin, end) of all tiles in order.  tail_cta: where the item ends that the run's end cuts in two.
template <class W> struct TreeRunT { long long begin, end; int tail_cta; TreeCursorT<W> at; };
using TreeRun = TreeRunT<TreeWork>;

// Run c of `total` work in `ctas` runs begins here: the first total % ctas runs have one unit more than the others.
__device__ __forceinline__ long long tree_run_begin(long long total, int ctas, int c) {
    const long long q = tree_div(total, ctas), r = total - q * ctas;
    return q * c + (c < r ? c : r);
}
// The CTA whose run holds unit `x`.
__device__ __forceinline__ int tree_cta_of(long long x, long long total, int ctas) {
    const long long q = tree_div(total, ctas), r = total - q * ctas, wide = r * (q + 1);
    return (int)(x < wide ? tree_div(x, q + 1) : r + tree_div(x - wide, q));
}

// The run of this CTA; called by all threads of the block (part: two words per warp, out: shared).  Ends with a barrier.
// An item's units are its constant, then its tiles: a tile belongs to the CTA whose run holds its unit.
template <class W>
__device__ __forceinline__ void tree_find_run(const W& w, long long* part, TreeRunT<W>* out) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const int per = (w.batch + blockDim.x - 1) / blockDim.x;
    const int b0 = min(tid * per, w.batch), b1 = min(b0 + per, w.batch);
    long long tiles = 0, items = 0;
    for (int b = b0; b < b1; ++b) {
        const typename W::Request r = tree_request(w, b);
        const long long n = r.n_kt ? (long long)w.n_kv * r.n_rt : 0;
        items += n;
        tiles += n * (r.n_kt - r.first_tile());
    }
    long long up_tiles = tiles, up_items = items;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, up_tiles, o), v = __shfl_up_sync(0xffffffffu, up_items, o);
        if (lane >= o) { up_tiles += u; up_items += v; }
    }
    if (lane == 31) { part[2 * warp] = up_tiles; part[2 * warp + 1] = up_items; }
    __syncthreads();
    long long all_tiles = 0, all_items = 0;
    for (int k = 0; k < warps; ++k) {
        if (k == warp) { up_tiles += all_tiles; up_items += all_items; }
        all_tiles += part[2 * k];
        all_items += part[2 * k + 1];
    }
    const long long total = all_tiles + w.item_cost * all_items;
    const int ctas = total < (long long)gridDim.x ? (int)total : (int)gridDim.x;
    const bool idle = (int)blockIdx.x >= ctas;
    if (tid == 0 && idle) { out->begin = out->end = 0; }
    if (!idle) {
        const long long lo = (up_tiles - tiles) + w.item_cost * (up_items - items), hi = up_tiles + w.item_cost * up_items;   // this thread's units
        const long long edge[2] = {tree_run_begin(total, ctas, blockIdx.x), tree_run_begin(total, ctas, blockIdx.x + 1)};
        if (tid == 0 && edge[1] == total) { out->end = all_tiles; out->tail_cta = -1; }
#pragma unroll 1
        for (int e = 0; e < 2; ++e) {
            if (edge[e] < lo || edge[e] >= hi) continue;           // exactly one thread goes on (none for the end of the last run)
            long long rest = edge[e] - lo, at_tile = up_tiles - tiles, unit = lo;
            TreeCursorT<W> c;
            int cost = 1, tiles_of = 0;
            for (c.b = b0; c.b < b1; ++c.b) {
                c.load(w);
                if (c.r.n_kt == 0) continue;
                tiles_of = c.r.n_kt - c.r.first_tile();
                cost = tiles_of + w.item_cost;
                const long long n = (long long)w.n_kv * c.r.n_rt;
                if (rest < n * cost) break;
                rest -= n * cost;
                unit += n * cost;
                at_tile += n * tiles_of;
            }
            const long long item = tree_div(rest, cost), head = tree_div(item, c.r.n_rt);
            const int off = (int)(rest - item * cost);
            const int in = max(0, off - w.item_cost);
            c.kt = c.r.first_tile() + in;
            c.rt = (int)(item - head * c.r.n_rt);
            c.h = (int)head;
            at_tile += item * tiles_of + in;
            if (e == 0) { out->begin = at_tile; out->at = c; }
            else { out->end = at_tile; out->tail_cta = in > 0 ? tree_cta_of(unit + (item + 1) * cost - 1, total, ctas) : -1; }
        }
    }
    __syncthreads();
}

// How many of `grid` CTAs the groups' launch has, from the time of one SM that both need (the requests' launch has the others): both end at the same time then,
// and reading the keys of one overlaps the arithmetic of the other.  128 requests behind 16001 keys, 1 to 1500 own (128 queries a tile / a warp's runs), the groups' on 148 CTAs
// and the requests' on as many behind them 147 us, side by side on 64 + 84 / 80 + 68 / 96 + 52 CTAs 120 / 106 / 130; 8 x 8 beams behind 3000 to 16000 keys, 17 to 300 own (keys
// as rows / a warp's runs) 92 against 87 / 80 / 87 on 96 / 128 / 134 CTAs.  A single group has items of one length: a whole number of CTAs for each
// spares every CTA the second item that it would open (in the first example 72 CTAs, which is no multiple of 16 items, take 139 us).
__device__ __forceinline__ int prefix_share(long long shared, long long own, long long items, int grid, bool even) {
    if (shared == 0) return 0;
    const long long sum = shared + own;
    const int most = own ? grid - 1 : grid;
    int ctas = (int)((2 * grid * shared + sum) / (2 * sum));
    ctas = max(1, min(ctas, most));
    if (even && items <= ctas) ctas = min((ctas + (int)items / 2) / (int)items, most / (int)items) * (int)items;
    return ctas;
}

// The same for lists of parts, whose descriptions take several dependent reads: the threads keep those that they scanned in shared memory, and the edges of
// the runs are looked up side by side.  N workers per CTA (1, or its warps): out[0 .. N - 1] are their runs, *end the part in which the last of them ends.
struct PrefixScan {
    static constexpr int kMost = 384;        // threads of a block, and parts whose descriptions are kept
    long long units[kMost], tiles[kMost];    // before the parts of each thread
    PrefixRequest part[kMost];               // one part to a thread
    long long sums[4 * kMost / 32];
    int kept;                                // descriptions in `part`
};
__device__ __forceinline__ void prefix_load(const PrefixWork& w, const PrefixScan& scan, int b, PrefixRequest& r) {
    if (b < scan.kept) r = scan.part[b];
    else { r = tree_request(w, b); prefix_find_row(w, b, r); }
}
// What the joining launch needs to know of every row, so that it does not have to look for the row's request: 0 not a row of any (valid) request, 1 own keys only, 3 a
// shared part too.  By all threads of one CTA of the launch that has the requests' own parts.
__device__ __forceinline__ void prefix_map_rows(const PrefixWork& w, const PrefixScan& scan) {
    for (int r = threadIdx.x; r < w.rows; r += blockDim.x) w.row_sides[r] = 0;
    __syncthreads();
    for (int b = threadIdx.x; b < w.requests; b += blockDim.x) {
        PrefixRequest own, shared;
        prefix_load(w, scan, w.groups - w.first + b, own);
        if (own.n_kt == 0) continue;
        bool ok;
        shared = prefix_shared(w, __ldg(w.request_group + b), ok);
        // (rows that another request claims as well may get either's word)
        for (int i = 0; ok && i < own.n; ++i) w.row_sides[own.row0 + i] = shared.n_kt > 0 ? 3 : 1;
    }
}
// A cursor over tiles that looks parts up in the CTA's copies.
struct PrefixCursor {
    PrefixRequest r;
    int b, h, rt, kt;
    __device__ __forceinline__ void next(const PrefixWork& w, const PrefixScan& scan) {
        if (++kt < r.n_kt) return;
        if (++rt >= r.n_rt) {
            rt = 0;
            if (++h >= w.n_kv) {
                h = 0;
                do { if (++b >= w.batch) return; prefix_load(w, scan, b, r); } while (r.n_kt == 0);
            }
        }
        kt = r.kt0;
    }
};
// Returns how many CTAs have runs.
template <int N>
__device__ __forceinline__ int prefix_find_runs(const PrefixWork& w, PrefixScan& scan, TreeRunT<PrefixWork>* out) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const int per = (w.batch + blockDim.x - 1) / blockDim.x;
    const int b0 = min(tid * per, w.batch), b1 = min(b0 + per, w.batch);
    long long tiles = 0, items = 0;
    for (int b = b0; b < b1; ++b) {
        PrefixRequest r = tree_request(w, b);
        const long long n = r.n_kt ? (long long)w.n_kv * r.n_rt : 0;
        items += n;
        tiles += n * (r.n_kt - r.kt0);
        if (per == 1) {
            prefix_find_row(w, b, r);
            scan.part[b] = r;
        }
    }
    long long other_tiles = 0, other_items = 0;
    if (w.other_time) {
        PrefixWork o = w;
        o.tile_rows = w.other_rows; o.key_tile = w.other_keys;
        o.first = w.first ? 0 : w.groups;
        const int parts = w.first ? w.groups : w.requests;
        for (int b = blockDim.x - 1 - tid; b < parts; b += blockDim.x) {                 // (other warps than those that read this launch's few parts)
            const PrefixRequest r = tree_request(o, b);
            const long long n = r.n_kt ? (long long)w.n_kv * r.n_rt : 0;
            other_items += n;
            other_tiles += n * (r.n_kt - r.kt0);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            other_tiles += __shfl_xor_sync(0xffffffffu, other_tiles, o);
            other_items += __shfl_xor_sync(0xffffffffu, other_items, o);
        }
    }
    long long up_tiles = tiles, up_items = items;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, up_tiles, o), v = __shfl_up_sync(0xffffffffu, up_items, o);
        if (lane >= o) { up_tiles += u; up_items += v; }
    }
    if (lane == 31) { scan.sums[4 * warp] = up_tiles; scan.sums[4 * warp + 1] = up_items; scan.sums[4 * warp + 2] = other_tiles; scan.sums[4 * warp + 3] = other_items; }
    if (tid == 0) scan.kept = per == 1 ? w.batch : 0;
    __syncthreads();
    long long all_tiles = 0, all_items = 0;
    other_tiles = other_items = 0;
    for (int k = 0; k < warps; ++k) {
        if (k == warp) { up_tiles += all_tiles; up_items += all_items; }
        all_tiles += scan.sums[4 * k];
        all_items += scan.sums[4 * k + 1];
        other_tiles += scan.sums[4 * k + 2];
        other_items += scan.sums[4 * k + 3];
    }
    int ctas = gridDim.x, item_cost = w.item_cost;
    if (w.other_time) {
        const long long mine = w.tile_time * (all_tiles + item_cost * all_items), theirs = w.other_time * (other_tiles + w.other_cost * other_items);
        const bool even = w.groups == 1;
        if (w.first) ctas -= prefix_share(theirs, mine, other_items, gridDim.x, even);
        else {
            ctas = prefix_share(mine, theirs, all_items, gridDim.x, even);
            if (even && all_items > 0 && ctas >= all_items) {    // an item's units a multiple of its CTAs, so that runs begin where items do
                const int each = ctas / (int)all_items, units = (int)(all_tiles / all_items) + item_cost;
                item_cost += (units + each - 1) / each * each - units;
            }
        }
        if ((int)blockIdx.x >= ctas) {
            if (tid < N) { out[tid].begin = out[tid].end = 0; }
            __syncthreads();
            return ctas;
        }
    }
    scan.units[tid] = (up_tiles - tiles) + item_cost * (up_items - items);
    scan.tiles[tid] = up_tiles - tiles;
    const long long total = all_tiles + item_cost * all_items, most = (long long)ctas * N;
    const int workers = total < most ? (int)total : (int)most, me = blockIdx.x * N + tid;
    if (tid < N && me >= workers) { out[tid].begin = out[tid].end = 0; }
    if (tid < N && me == workers - 1) { out[tid].end = all_tiles; out[tid].tail_cta = -1; }
    __syncthreads();
    if (tid <= N && me < workers) {
        const long long edge = tree_run_begin(total, workers, me);
        int lo = 0, hi = blockDim.x;                           // the last thread whose parts begin at or before the edge
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (scan.units[mid] <= edge) lo = mid;
            else hi = mid;
        }
        long long rest = edge - scan.units[lo], at_tile = scan.tiles[lo], unit = scan.units[lo];
        TreeCursorT<PrefixWork> c;
        int cost = 1, tiles_of = 0;
        for (c.b = lo * per; c.b < w.batch; ++c.b) {
            prefix_load(w, scan, c.b, c.r);
            if (c.r.n_kt == 0) continue;
            tiles_of = c.r.n_kt - c.r.kt0;
            cost = tiles_of + item_cost;
            const long long n = (long long)w.n_kv * c.r.n_rt;
            if (rest < n * cost) break;
            rest -= n * cost;
            unit += n * cost;
            at_tile += n * tiles_of;
        }
        const long long item = tree_div(rest, cost), head = tree_div(item, c.r.n_rt);
        const int in = max(0, (int)(rest - item * cost) - item_cost);
        c.kt = c.r.kt0 + in;
        c.rt = (int)(item - head * c.r.n_rt);
        c.h = (int)head;
        at_tile += item * tiles_of + in;
        if (tid < N) { out[tid].begin = at_tile; out[tid].at = c; }
        if (tid > 0) { out[tid - 1].end = at_tile; out[tid - 1].tail_cta = in > 0 ? tree_cta_of(unit + (item + 1) * cost - 1, total, workers) : -1; }
    }
    __syncthreads();
    return ctas;
}

// ---- partial results ------------------------------------------------------------------------------------------------
// One descriptor per CTA, a word that says whether its front slot is in use, then 2 * G slots of [tile_rows] references, [tile_rows] sums and [tile_rows][d_head] outputs (fp32).
struct TreeTail { int last_cta, queries, row0, q0, h, pad[3]; };   // an item that begins in this CTA and ends in last_cta; -1: none
constexpr int kMaxTreeGrid = 2 * 148;                    // one or two CTAs per SM
constexpr size_t kTailBytes = 12288, kFrontOffset = kMaxTreeGrid * sizeof(TreeTail);
static_assert(kFrontOffset + kMaxTreeGrid * sizeof(int) <= kTailBytes, "descriptors");

__host__ __device__ inline size_t tree_slot_floats(int tile_rows, int dh) { return (size_t)tile_rows * (dh + 2); }

// which CTAs have a front piece: one that continues an item of an earlier CTA (slot 2 c; slot 2 c + 1: one that goes on in the next)
__device__ __forceinline__ int* tree_front(uint8_t* scratch) { return reinterpret_cast<int*>(scratch + kFrontOffset); }
// (parts of a shared prefix have no descriptors, their workers may be many)
constexpr int kMaxWorkers = kMaxTreeGrid / 2 * kNarrowWarps;
static_assert(kMaxWorkers * sizeof(int) <= kTailBytes && kMaxWorkers >= kMaxTreeGrid && kMaxWorkers < 32768, "front words, places of pieces");
__device__ __forceinline__ int* prefix_front(uint8_t* scratch) { return reinterpret_cast<int*>(scratch); }
// what a CTA says before its run
template <class W> __device__ __forceinline__ void tree_announce(uint8_t* scratch, bool front) {
    if (W::kPrefix) { prefix_front(scratch)[blockIdx.x] = front; return; }
    reinterpret_cast<TreeTail*>(scratch)[blockIdx.x].last_cta = -1;
    tree_front(scratch)[blockIdx.x] = front;
}
// The run of this CTA, as soon as the launch before has left what it reads; ends with a barrier.  scan: sizeof(PrefixScan) bytes of shared memory that are not in use
// yet (lists of parts only).
__device__ __forceinline__ void tree_start(const TreeWork& w, long long* part, TreeRun* run, void*) {
    grid_dependency_wait();
    tree_find_run(w, part, run);
}
__device__ __forceinline__ void tree_start(const PrefixWork& w, long long*, TreeRunT<PrefixWork>* run, void* scan) {
    if (!w.late_wait) grid_dependency_wait();
    grid_dependency_release();
    const int ctas = prefix_find_runs<1>(w, *static_cast<PrefixScan*>(scan), run);
    if ((int)blockIdx.x == max(ctas, 1) - 1 && w.first + w.batch > w.groups) prefix_map_rows(w, *static_cast<PrefixScan*>(scan));
}
__device__ __forceinline__ void tree_finish(const TreeWork&) {}
__device__ __forceinline__ void tree_finish(const PrefixWork& w) { if (w.late_wait) grid_dependency_wait(); }

__device__ __forceinline__ float* tree_slot(uint8_t* scratch, int index, int tile_rows, int dh) {
    return reinterpret_cast<float*>(scratch + kTailBytes) + (size_t)index * tree_slot_floats(tile_rows, dh);
}

__device__ __forceinline__ float tree_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <typename T> __device__ __forceinline__ T tree_round(float v);
template <> __device__ __forceinline__ float tree_round<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 tree_round<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half tree_round<__half>(float v) { return __float2half_rn(v); }

// Joins the pieces of split items: block (c, y) takes the item that begins in CTA c, queries y, y + gridDim.y, ...
// out = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p over its pieces p in key order per warp, the 8 warps' shares then in
// warp order; a query that saw no key gives zeros.  All of it in binary32, one rounding at the end.
template <typename T, int DH>
__global__ void __launch_bounds__(256)
tree_combine_kernel(uint8_t* scratch, int tile_rows, int group, T* out, int64_t out_stride) {
    constexpr int VPL = DH / 32;
    __shared__ float acc_s[8][DH], m_s[8], l_s[8];
    grid_dependency_wait();
    const TreeTail tail = reinterpret_cast<const TreeTail*>(scratch)[blockIdx.x];
    if (tail.last_cta < 0) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = blockIdx.x, pieces = tail.last_cta - c0 + 1;
    for (int q = blockIdx.y; q < tail.queries; q += gridDim.y) {
        float m = -INFINITY, l = 0.0f, acc[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j) acc[j] = 0.0f;
        for (int p0 = warp; p0 < pieces; p0 += 32) {          // four pieces of this warp in flight
            float pm[4], pl[4], po[4][VPL];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int p = p0 + 8 * u;
                pm[u] = -INFINITY; pl[u] = 0.0f;
#pragma unroll
                for (int j = 0; j < VPL; ++j) po[u][j] = 0.0f;
                if (p < pieces && (p == 0 || tree_front(scratch)[c0 + p])) {
                    const float* slot = tree_slot(scratch, p == 0 ? 2 * c0 + 1 : 2 * (c0 + p), tile_rows, DH);
                    pm[u] = slot[q];
                    pl[u] = slot[tile_rows + q];
                    const float* o = slot + 2 * tile_rows + (size_t)q * DH + lane * VPL;
#pragma unroll
                    for (int j = 0; j < VPL; ++j) po[u][j] = o[j];
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (pl[u] == 0.0f) continue;                   // nothing seen in this piece (NaN sums go on)
                const float top = fmaxf(m, pm[u]);
                const float fa = m == -INFINITY ? 0.0f : tree_ex2(m - top), fb = tree_ex2(pm[u] - top);
                l = l * fa + pl[u] * fb;
#pragma unroll
                for (int j = 0; j < VPL; ++j) acc[j] = acc[j] * fa + po[u][j] * fb;
                m = top;
            }
        }
        if (lane == 0) { m_s[warp] = m; l_s[warp] = l; }
#pragma unroll
        for (int j = 0; j < VPL; ++j) acc_s[warp][lane * VPL + j] = acc[j];
        __syncthreads();
        if (threadIdx.x < DH) {
            float top = -INFINITY, sum = 0.0f, o = 0.0f;
#pragma unroll
            for (int w = 0; w < 8; ++w) if (l_s[w] != 0.0f) top = fmaxf(top, m_s[w]);
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                if (l_s[w] == 0.0f) continue;
                const float f = tree_ex2(m_s[w] - top);
                sum += l_s[w] * f;
                o += acc_s[w][threadIdx.x] * f;
            }
            const int token = (tail.q0 + q) / group, head = tail.h * group + (tail.q0 + q - token * group);
            out[(int64_t)(tail.row0 + token) * out_stride + (int64_t)head * DH + threadIdx.x] = tree_round<T>(sum == 0.0f ? 0.0f : o / sum);
        }
        __syncthreads();
    }
}

}  // namespace zq
