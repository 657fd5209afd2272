// The bookkeeping of a serving step on the device: pages given out and taken back with the rows' positions and slots, what the
// drafted tokens of a tree see of one another, and the tokens of a tree that become part of their sequence.
//
// All three move a few kilobytes: what they cost is a launch and their chains of dependent steps, so each is one launch whose
// chains are short (a scan of all sequences in every block rather than a pass for the scan and one for its use).  Measured, us a call among others: pages
// of 4 sequences 4.5, of 256 with 5000 rows 6.8, masks of 256 trees 3.6 - 4.8, commit of 2 and of 256 trees 5.8 - 6.1.
#pragma once

#include <cooperative_groups.h>

#include "gva_common.cuh"

namespace gva {

constexpr int kTreeMost = 256;       // nodes of a tree

// ---- pages ---------------------------------------------------------------------------------------------------
struct AssignParams {
    const int32_t *used, *want, *pages_in;   // [B]; new_lens may be used, pages_out may be pages_in
    int32_t *pages_out, *block_table, *ring;
    const int32_t *free_in;                  // [2] first entry of the ring that holds a free page, and how many do
    int32_t *free_out, *new_lens, *cu_q, *positions, *slots;
    int32_t *dev_status;
    int max_pages, num_pages, max_rows, B, P;
    int rows_here;                           // 1: the rows' positions and slots too; 0: assign_rows_kernel follows
};
constexpr int kAssignItems = 8;      // sequences of a thread at most: 1024 threads serve 8192

// What a sequence asks for.
struct Asks {
    int used, pages, to, rows, take, give;
    bool fine;
};
__device__ __forceinline__ Asks sequence_asks(const AssignParams &p, int b, bool sound) {
    Asks a;
    a.used = p.used[b];
    a.pages = p.pages_in[b];
    const int want = p.want[b];
    a.fine = sound && a.used >= 0 && want >= 0 && a.pages >= 0 && a.pages <= p.max_pages && (long long)want <= (long long)p.max_pages * p.P &&
             (long long)a.used <= (long long)a.pages * p.P;
    a.to = a.fine ? (int)(((long long)want + p.P - 1) / p.P) : a.pages;
    a.rows = a.fine ? max(want - a.used, 0) : 0;
    a.take = max(a.to - a.pages, 0);
    a.give = max(a.pages - a.to, 0);
    return a;
}
// The slot of a row of sequence b, `at` tokens into its page.  A row on a bad page has none: appends take it for a padded row, so it is said here.
__device__ __forceinline__ int slot_of(const AssignParams &p, int b, int page, int at) {
    if (page >= 0 && page < p.num_pages) return page * p.P + at;
    report_error(p.dev_status, GVA_ERR_BAD_PAGE, b);
    return -1;
}
// Largest b in [0, B) with off[b] <= x, for off non-decreasing, off[0] <= x.
__device__ __forceinline__ int owner_of(const int *off, int B, int x) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (off[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}
// Largest b in [0, B) with off[b] <= x, by a whole warp: 32 candidates at a time (B <= 8192: three trips to memory at most).
__device__ __forceinline__ int warp_owner_of(const int32_t *off, int B, int x) {
    const int lane = threadIdx.x & 31;
    int lo = 0, n = B;                                   // the answer is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const unsigned below = __ballot_sync(0xffffffffu, lane * step < n && off[at] <= x);      // (a prefix of the lanes, the first among them)
        const int k = 31 - __clz(below);
        n = min(step, lo + n - (lo + k * step));
        lo += k * step;
    }
    return lo;
}
// An entry of the ring, `at` behind the first free page: num_pages is below 2^26 (slots are below 2^31), and `at` at most num_pages.
__device__ __forceinline__ int ring_entry(const AssignParams &p, int first, int at) {
    at += first;
    if (at >= p.num_pages) at -= p.num_pages;
    return at >= p.num_pages ? at - p.num_pages : at;
}
// Returned page i of the call, and whose it was.
__device__ __forceinline__ int returned_page(const AssignParams &p, const int *s_give, const int *s_to, int i, int &b) {
    b = owner_of(s_give, p.B, i);
    return p.block_table[(size_t)b * p.max_pages + s_to[b] + (i - s_give[b])];
}
// The ring's end where some of the n returned pages are bad: the good ones in their order, as many as there is room for, by one
// block, a page a thread at a time.  How many are good.  (Only an unsound block table leads here.)
__device__ __forceinline__ int return_good_pages(const AssignParams &p, const int *s_give, const int *s_to, int n, int first, int count, int *s_warp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int before = 0;
    for (int base = 0; base < n; base += blockDim.x) {
        const int i = base + threadIdx.x;
        int page = -1, b;
        if (i < n) page = returned_page(p, s_give, s_to, i, b);
        const bool good = page >= 0 && page < p.num_pages;
        const unsigned those = __ballot_sync(0xffffffffu, good);
        __syncthreads();
        if (lane == 0) s_warp[warp] = __popc(those);
        __syncthreads();
        int at = before + __popc(those & ((1u << lane) - 1));
        for (int w = 0; w < warps; ++w) {
            if (w < warp) at += s_warp[w];
            before += s_warp[w];
        }
        if (good && at < p.num_pages - count) p.ring[ring_entry(p, first, count + at)] = page;
    }
    return before;
}
// Inclusive sums over the block's threads of four values, in place; s_part holds 4 x 32 words.  The last value's total is returned.
struct Sums {
    long long v[4];
};
__device__ __forceinline__ long long block_scan(Sums &x, int wanted, long long (*s_part)[32]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long y = __shfl_up_sync(0xffffffffu, x.v[i], o);
            if (lane >= o) x.v[i] += y;
        }
    if (lane == 31)
#pragma unroll
        for (int i = 0; i < 4; ++i) s_part[i][warp] = x.v[i];
    __syncthreads();
    long long w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = lane < warps ? s_part[i][lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long y = __shfl_up_sync(0xffffffffu, w[i], o);
            if (lane >= o) w[i] += y;
        }
    long long total = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long before = __shfl_sync(0xffffffffu, w[i], (warp + 31) & 31), all = __shfl_sync(0xffffffffu, w[i], 31);
        if (warp > 0) x.v[i] += before;
        if (i == wanted) total = all;
    }
    return total;
}

// One cluster.  Every block scans all sequences for itself (ITEMS a thread) and keeps the offsets in shared memory; once all
// of them have read the inputs -- outputs may be the same buffers -- they share out rows, taken and returned pages among
// their threads, which find their sequence by bisection.  Growing sequences are served in order until one does not fit, so the
// sums before a served one are sums over all growing ones before it, and what is served needs no second scan.
template <int ITEMS>
__global__ void __launch_bounds__(1024)
assign_pages_kernel(AssignParams p) {
    grid_dependency_launch();
    extern __shared__ int s_mem[];
    int *s_row = s_mem, *s_take = s_row + p.B, *s_give = s_take + p.B, *s_used = s_give + p.B, *s_pages = s_used + p.B, *s_to = s_pages + p.B;
    __shared__ long long s_part[4][32];
    __shared__ int s_served[3];      // rows, pages taken, pages returned by growing sequences: of those served
    __shared__ int s_bad, s_warp[32];        // (of the first block:) whether any block has met a bad page; scratch of a scan
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, nt = blockDim.x, rank = (int)cluster.block_rank(), wide = (int)cluster.num_blocks();
    const int per = (p.B + nt - 1) / nt;
    if (tid < 3) s_served[tid] = 0;
    if (tid == 3) s_bad = 0;
    grid_dependency_wait();
    const int first = p.free_in[0], count = p.free_in[1];
    const bool sound = first >= 0 && first < p.num_pages && count >= 0 && count <= p.num_pages;    // else all stays as it is
    if (!sound && rank == 0 && tid == 0) report_error(p.dev_status, GVA_ERR_BAD_PAGE, 0);
    Asks a[ITEMS];
    long long rows = 0, take = 0, give = 0, back = 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int b = tid * per + i;
        if (i >= per || b >= p.B) continue;
        a[i] = sequence_asks(p, b, sound);
        rows += a[i].rows;
        take += a[i].take;
        if (a[i].rows > 0) back += a[i].give;
        else give += a[i].give;
        if (!a[i].fine && sound && rank == 0) report_error(p.dev_status, GVA_ERR_SEQ_LEN, b);
    }
    Sums to = {{rows, take, give, back}};
    const long long give_all = block_scan(to, 2, s_part);
    {
        int most_rows = 0, most_take = 0, most_back = 0;        // of this thread's sequences that are served
        long long r = to.v[0] - rows, t = to.v[1] - take, g = to.v[2] - give, k = to.v[3] - back;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int b = tid * per + i;
            if (i >= per || b >= p.B) continue;
            const bool grows = a[i].rows > 0;
            const bool served = !grows || (t + a[i].take <= count && r + a[i].rows <= p.max_rows);
            // (sums past what is served are past what fits: cut off here and below)
            s_row[b] = (int)min(r, (long long)p.max_rows);
            s_take[b] = (int)min(t, (long long)count);
            s_give[b] = (int)min(g, (long long)p.num_pages);
            s_to[b] = (int)min(k, (long long)p.num_pages);     // (for a moment: returned before it by growing sequences)
            s_used[b] = a[i].used;
            s_pages[b] = a[i].pages;
            r += a[i].rows;
            t += a[i].take;
            if (grows) k += a[i].give;
            else g += a[i].give;
            if (grows && served) {
                most_rows = (int)r;
                most_take = (int)t;
                most_back = (int)min(k, (long long)p.num_pages);
            }
            if (!served) {
                if (rank == 0) report_error(p.dev_status, GVA_ERR_NO_ROOM, b);
                a[i].to = a[i].pages;
                a[i].rows = -1;                                // stays as it is
            }
        }
        most_rows = __reduce_max_sync(0xffffffffu, most_rows);
        most_take = __reduce_max_sync(0xffffffffu, most_take);
        most_back = __reduce_max_sync(0xffffffffu, most_back);
        if ((tid & 31) == 0) {
            atomicMax(&s_served[0], most_rows);
            atomicMax(&s_served[1], most_take);
            atomicMax(&s_served[2], most_back);
        }
    }
    __syncthreads();
    const int n_rows = s_served[0], n_take = s_served[1], n_back = s_served[2];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int b = tid * per + i;
        if (i >= per || b >= p.B) continue;
        s_row[b] = min(s_row[b], n_rows);
        s_take[b] = min(s_take[b], n_take);
        s_give[b] = (int)min((long long)s_give[b] + min(s_to[b], n_back), (long long)p.num_pages);
        s_to[b] = a[i].to;
    }
    int want[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int b = tid * per + i;
        if (i < per && b < p.B) want[i] = p.want[b];
    }
    const int n_give = (int)min(give_all + n_back, (long long)p.num_pages + 1);
    // every block of the cluster has read its inputs (and this block's offsets are whole) before anything is written
    cluster.sync();
    const int me = rank * nt + tid, all = wide * nt, room = p.num_pages - count;
    auto entry = [&](int at) { return ring_entry(p, first, at); };
    if (rank == 0) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int b = tid * per + i;
            if (i >= per || b >= p.B) continue;
            p.pages_out[b] = a[i].to;
            p.new_lens[b] = !a[i].fine || a[i].rows < 0 ? a[i].used : want[i];
            p.cu_q[b] = s_row[b];
        }
        if (tid == 0) {
            p.cu_q[p.B] = n_rows;
            p.free_out[0] = sound ? entry(n_take) : first;
            p.free_out[1] = sound ? count - n_take + min(n_give, room) : count;
        }
    }
    for (int i = me; i < n_take; i += all) {                     // (none of these without a sound ring)
        const int b = owner_of(s_take, p.B, i);
        p.block_table[(size_t)b * p.max_pages + s_pages[b] + (i - s_take[b])] = p.ring[entry(i)];
    }
    bool bad = false;
    for (int i = me; i < n_give && i < room; i += all) {
        int b;
        const int page = returned_page(p, s_give, s_to, i, b);
        if (page >= 0 && page < p.num_pages) {
            p.ring[entry(count + i)] = page;
        } else {
            bad = true;
            report_error(p.dev_status, GVA_ERR_BAD_PAGE, b);
        }
    }
    for (int i = p.rows_here ? me : n_rows; i < n_rows; i += all) {
        const int b = owner_of(s_row, p.B, i);
        const int t = s_used[b] + (i - s_row[b]), j = t / p.P;
        const int page = j < s_pages[b] ? p.block_table[(size_t)b * p.max_pages + j]
                                        : p.ring[entry(s_take[b] + (j - s_pages[b]))];
        p.positions[i] = t;
        p.slots[i] = slot_of(p, b, page, t % p.P);
    }
    if (n_give == 0) return;                                     // (the same for the whole cluster)
    // a returned page that is outside the pool goes to nobody: where any block has met one, the first lays the ring's end out anew
    bad = __syncthreads_or(bad);
    if (wide > 1) {
        if (bad && tid == 0) *cluster.map_shared_rank(&s_bad, 0) = 1;
        cluster.sync();
        bad = s_bad != 0;
    }
    if (rank > 0) return;
    const int n_kept = bad ? return_good_pages(p, s_give, s_to, min(n_give, p.num_pages), first, count, s_warp) : n_give;
    if (tid == 0) {
        if (bad) p.free_out[1] = count - n_take + min(n_kept, room);
        // a ring that would overflow held pages twice: it takes no more than fit
        if (n_kept > room || n_give > p.num_pages) report_error(p.dev_status, GVA_ERR_BAD_PAGE, 0);
    }
}

// Positions and slots of many rows, from what assign_pages_kernel has left (0.2 M rows of 48 prompts: 8.4 - 9.3 us with that kernel, 33 in its one
// cluster).  A block has 1024 rows in a row, of as few sequences as these lie in.
constexpr int kAssignRows = 1024, kAssignRowThreads = 256;
__global__ void __launch_bounds__(kAssignRowThreads)
assign_rows_kernel(AssignParams p) {
    grid_dependency_launch();
    __shared__ int s_b[2];
    grid_dependency_wait();
    const int r0 = blockIdx.x * kAssignRows, total = p.cu_q[p.B];
    if (r0 >= total) return;
    const int end = r0 + min(kAssignRows, total - r0), warp = threadIdx.x >> 5;         // (rows are numbers of 32 bits: up to 2^31 - 32 of them)
    if (warp < 2) {
        const int b = warp_owner_of(p.cu_q, p.B, warp == 0 ? r0 : end - 1);
        if ((threadIdx.x & 31) == 0) s_b[warp] = b;
    }
    __syncthreads();
    const int b0 = s_b[0], n = s_b[1] - b0 + 1;
#pragma unroll
    for (int k = 0; k < kAssignRows / kAssignRowThreads; ++k) {
        const int i = r0 + k * kAssignRowThreads + threadIdx.x;
        if (i >= end) continue;
        const int b = b0 + owner_of(p.cu_q + b0, n, i), t = p.new_lens[b] - (p.cu_q[b + 1] - i), j = t / p.P;
        const int page = p.block_table[(size_t)b * p.max_pages + j];
        p.positions[i] = t;
        p.slots[i] = slot_of(p, b, page, t - j * p.P);
    }
}

// ---- trees ---------------------------------------------------------------------------------------------------
// One block per sequence: bits of a node and its ancestors, and its position ctx + depth.  A thread walks up from its node
// through the parents in shared memory: as many dependent steps as the tree is deep.
struct TreeMaskParams {
    const int32_t *parents, *cu_q, *ctx_lens;
    uint32_t *mask;
    int32_t *positions;              // nullable
    int32_t *dev_status;
    int words, most;                 // words of a row, nodes of a tree at most
};
// Loads a tree's parents (n of them) into s_parents; whether they are sound: the first -1 or any node's below its own number.
__device__ __forceinline__ bool load_parents(const int32_t *parents, int n, int *s_parents) {
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int par = parents[i];
        bad |= par < -1 || par >= i;
        s_parents[i] = par;
    }
    return !__syncthreads_or(bad);
}
__global__ void __launch_bounds__(kTreeMost)
tree_masks_kernel(TreeMaskParams p) {
    grid_dependency_launch();
    __shared__ int s_parents[kTreeMost];
    grid_dependency_wait();
    const int b = blockIdx.x, r0 = p.cu_q[b], n = p.cu_q[b + 1] - r0;
    if (n <= 0) return;
    if (n > p.most || !load_parents(p.parents + r0, n, s_parents)) {
        if (threadIdx.x == 0) report_error(p.dev_status, GVA_ERR_TREE, b);
        return;
    }
    const int ctx = p.positions ? p.ctx_lens[b] : 0;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        uint32_t bits[kTreeMost / 32];
#pragma unroll
        for (int w = 0; w < kTreeMost / 32; ++w) bits[w] = 0;
        int depth = -1;
        for (int at = i; at >= 0; at = s_parents[at], ++depth)
#pragma unroll
            for (int w = 0; w < kTreeMost / 32; ++w) bits[w] |= (at >> 5) == w ? 1u << (at & 31) : 0u;
        uint32_t *row = p.mask + (size_t)(r0 + i) * p.words;
#pragma unroll
        for (int w = 0; w < kTreeMost / 32; ++w)
            if (w < p.words) row[w] = bits[w];
        if (p.positions) p.positions[r0 + i] = ctx + depth;
    }
}

// ---- commit --------------------------------------------------------------------------------------------------
// One block per sequence.  Node 0 is accepted; of an accepted node the first child whose token is the one that was chosen
// after it is.  Every node looks at once whether it is such a child (the smallest wins), then one thread walks.  The path's nodes
// ascend, so rows only move down, and a row is overwritten by a row further along the path only: a thread that takes its
// 16-byte column of all rows in the path's order, loads of a batch before its stores, never reads what it has written.
struct TreeCommitParams {
    uint8_t *v_pool, *kr_pool;       // kr_pool may be null
    const int32_t *block_table;      // nullable
    const int32_t *parents, *tokens, *chosen, *cu_q, *ctx_lens;    // new_lens may be ctx_lens
    int32_t *path, *new_lens, *last;
    int32_t *dev_status;
    int v_bytes, kr_bytes;           // of a row
    int G, P, num_pages, max_pages, most;
};
constexpr int kCommitThreads = 128, kCommitBatch = 8;
__global__ void __launch_bounds__(kCommitThreads)
tree_commit_kernel(TreeCommitParams p) {
    grid_dependency_launch();
    __shared__ int s_parents[kTreeMost], s_next[kTreeMost], s_path[kTreeMost], s_chosen[kTreeMost];
    __shared__ int2 s_from[kTreeMost], s_to[kTreeMost];           // page and slot of every row of the path, and of where it goes
    __shared__ int s_count, s_page[kTreeMost / 32 + 1];          // (pages of 32 tokens at least)
    grid_dependency_wait();
    const int b = blockIdx.x, tid = threadIdx.x;
    const int r0 = p.cu_q[b], n = max(p.cu_q[b + 1] - r0, 0), ctx = p.ctx_lens[b];
    int code = GVA_OK;
    if (ctx < 0 || (long long)ctx + n > (long long)p.max_pages * p.P) code = GVA_ERR_SEQ_LEN;
    else if (n > p.most) code = GVA_ERR_TREE;
    int count = 0; int token[kTreeMost / kCommitThreads];
    if (code == GVA_OK) {                                         // everything the walk needs, in one trip
#pragma unroll
        for (int k = 0; k < kTreeMost / kCommitThreads; ++k) {
            const int i = tid + k * kCommitThreads;
            if (i >= n) continue;
            token[k] = p.tokens[r0 + i];
            s_chosen[i] = p.chosen[r0 + i];
            s_next[i] = n;
        }
        const int first = ctx / p.P, pages = n > 0 ? (ctx + n - 1) / p.P - first + 1 : 0;
        for (int j = tid; j < pages; j += kCommitThreads) {
            const long long page = p.block_table ? (long long)p.block_table[(size_t)b * p.max_pages + first + j] : (long long)b * p.max_pages + first + j;
            s_page[j] = page < 0 || page >= p.num_pages ? -1 : (int)page;
        }
        if (!load_parents(p.parents + r0, n, s_parents)) code = GVA_ERR_TREE;
    }
    if (code == GVA_OK && n > 0) {
#pragma unroll
        for (int k = 0; k < kTreeMost / kCommitThreads; ++k) {
            const int i = tid + k * kCommitThreads, par = i < n ? s_parents[i] : -1;
            if (par >= 0 && token[k] == s_chosen[par]) atomicMin(&s_next[par], i);
        }
        __syncthreads();
        if (tid == 0) {
            int k = 0;
            for (int at = 0; at < n; at = s_next[at]) s_path[k++] = at;
            s_count = k;
        }
        __syncthreads();
        count = s_count;
        bool bad = false;
        for (int i = tid; i < count; i += kCommitThreads) {
            auto place = [&](int t) {
                const int j = t / p.P, page = s_page[j - ctx / p.P];
                bad |= page < 0;
                return make_int2(page, t - j * p.P);
            };
            if (s_path[i] == i) continue;
            s_from[i] = place(ctx + s_path[i]);
            s_to[i] = place(ctx + i);
        }
        if (__syncthreads_or(bad)) {
            code = GVA_ERR_BAD_PAGE;
            count = 0;
        }
    }
    if (code != GVA_OK && tid == 0) report_error(p.dev_status, code, b);
    for (int i = tid; i < n; i += kCommitThreads) p.path[r0 + i] = i < count ? s_path[i] : -1;
    if (tid == 0) {
        p.new_lens[b] = ctx + count;
        p.last[b] = count > 0 ? s_chosen[s_path[count - 1]] : -1;
    }
    int begin = 0;                                                // the path's beginning stays where it is
    while (begin < count && s_path[begin] == begin) ++begin;
    if (begin == count) return;
    const int v_cols = p.v_bytes / 16, cols = p.G * v_cols + (p.kr_pool ? p.kr_bytes / 16 : 0);
    for (int c = tid; c < cols; c += kCommitThreads) {
        const bool v = c < p.G * v_cols;
        const int g = v ? c / v_cols : 0, at = (v ? c - g * v_cols : c - p.G * v_cols) * 16;
        auto address = [&](const int2 &x) {
            return v ? p.v_pool + (((size_t)x.x * p.G + g) * p.P + x.y) * p.v_bytes + at : p.kr_pool + ((size_t)x.x * p.P + x.y) * p.kr_bytes + at;
        };
        for (int i0 = begin; i0 < count; i0 += kCommitBatch) {
            uint4 row[kCommitBatch];
#pragma unroll
            for (int u = 0; u < kCommitBatch; ++u)
                if (i0 + u < count) row[u] = *reinterpret_cast<const uint4 *>(address(s_from[i0 + u]));
#pragma unroll
            for (int u = 0; u < kCommitBatch; ++u)
                if (i0 + u < count) *reinterpret_cast<uint4 *>(address(s_to[i0 + u])) = row[u];
        }
    }
}

}  // namespace gva
