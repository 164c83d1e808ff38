// Row, page and cache bookkeeping of drafted token trees: page tables from
// sequence lengths, drafted trees as the rows of a stage call, greedy acceptance,
// and the move of the accepted K/V.  All but the move are bound by latency
// (a few KB to a few hundred KB per call), so each is one or two launches whose
// workgroups recompute the small prefix sums they need instead of waiting for
// one another.
#include <algorithm>

#include "cdb_internal.h"

namespace cdb {

// Inclusive prefix sum over a 256-thread workgroup; *total = the whole sum.
// red: 4 ints of LDS, free again after the call's last barrier.
__device__ __forceinline__ int block_scan256(int v, int* red, int* total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 63) red[w] = v;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i < w) before += red[i];
        all += red[i];
    }
    *total = all;
    return v + before;
}

// ------------------------------------------------------------------ page tables
// One workgroup row (blockIdx.x) per sequence, blockIdx.y shares its entries.
struct MapArgs {
    int32_t* table;
    int S, P, planes;          // sequences, pages per plane, r_max + 2
    int width[3];              // distinct pages per token page in the pools (0: the stage has no layers)
    int first[3], n_planes[3]; // planes of each pool
    int own[3];                // first planes of the pool with a page of their own: plane k of it has page min(k, width - 1)
    int32_t* free_ids[3];
    int32_t* free_count[3];
    int capacity[3];
    const int32_t* len;
    int32_t* mapped;
    int32_t* old_pages;   // scratch [S]: mapped before the call
    int32_t* old_count;   // scratch [3]: stack heights before the call
    int* err;
};

__device__ __forceinline__ int pages_wanted(const MapArgs& a, int s, int old, bool& bad) {
    const int l = a.len[s];
    if (old < 0 || old > a.P) bad = true;
    if (l < 0) return old;
    if (l > a.P * kPage) bad = true;
    return (int)(((unsigned)l + kPage - 1) / kPage);
}

struct MapSums {
    int back, more;          // pages of sequences before this one that go back / are taken
    int all_back, all_more;
    int code;                // 0, or why nothing may change
};
// Every workgroup sums the page counts of all sequences itself.
__device__ __forceinline__ MapSums map_sums(const MapArgs& a, const int32_t* pages, const int32_t* count, int s) {
    __shared__ int red[4][4];
    __shared__ int s_bad;
    if (threadIdx.x == 0) s_bad = 0;
    __syncthreads();
    int v[4] = {0, 0, 0, 0};
    bool bad = false;
    for (int i = threadIdx.x; i < a.S; i += 256) {
        const int old = pages[i], now = pages_wanted(a, i, old, bad);
        const int b = old > now ? old - now : 0, m = now > old ? now - old : 0;
        v[2] += b;
        v[3] += m;
        if (i < s) {
            v[0] += b;
            v[1] += m;
        }
    }
    if (bad) s_bad = 1;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v[k] += __shfl_xor(v[k], o, 64);
        if ((threadIdx.x & 63) == 0) red[k][threadIdx.x >> 6] = v[k];
    }
    __syncthreads();
    MapSums r;
    r.back = red[0][0] + red[0][1] + red[0][2] + red[0][3];
    r.more = red[1][0] + red[1][1] + red[1][2] + red[1][3];
    r.all_back = red[2][0] + red[2][1] + red[2][2] + red[2][3];
    r.all_more = red[3][0] + red[3][1] + red[3][2] + red[3][3];
    r.code = s_bad ? CDB_DEV_BAD_INDEX : 0;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        if (!a.width[k]) continue;
        const int c = count[k], up = c + r.all_back * a.width[k];
        if (c < 0 || c > a.capacity[k])
            r.code = CDB_DEV_BAD_INDEX;
        else if (!r.code && (up > a.capacity[k] || up < r.all_more * a.width[k]))
            r.code = CDB_DEV_NO_PAGES;
    }
    return r;
}

// Entry e of the pages p0.. of sequence s in pool k, in (page, plane) order over
// the planes with a page of their own: the table's cell.
__device__ __forceinline__ size_t map_cell(const MapArgs& a, int k, int s, int p, int plane) {
    return ((size_t)s * a.planes + a.first[k] + plane) * a.P + p;
}

// Pages past the wanted count go back: stack position count + (all - 1 - rank),
// table entries -1.  Also keeps the counts as they were for k_map_take.
__global__ __launch_bounds__(256) void k_map_release(MapArgs a) {
    const int s = blockIdx.x;
    const bool lead = s == 0 && blockIdx.y == 0;
    bool bad = false;
    const int old = a.mapped[s], now = pages_wanted(a, s, old, bad);
    if (blockIdx.y == 0 && threadIdx.x == 0) a.old_pages[s] = old;
    int count[3] = {0, 0, 0};
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (a.width[k]) count[k] = *a.free_count[k];
    if (lead && threadIdx.x < 3) a.old_count[threadIdx.x] = count[threadIdx.x];
    if (old <= now && !lead) return;
    const MapSums m = map_sums(a, a.mapped, count, s);
    if (m.code) {
        if (lead && threadIdx.x == 0) set_err(a.err, m.code);
        return;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const int w = a.width[k];
        if (!w) continue;
        const int top = count[k] + m.all_back * w - 1 - m.back * w;
        for (int e = blockIdx.y * 256 + threadIdx.x; e < (old - now) * w; e += gridDim.y * 256) {
            const int p = now + e / w, plane = e % w;
            const int id = a.table[map_cell(a, k, s, p, plane)];
            if (id < 0) set_err(a.err, CDB_DEV_UNMAPPED_PAGE);
            a.free_ids[k][top - e] = id;
            a.table[map_cell(a, k, s, p, plane)] = -1;
            if (plane == w - 1)
                for (int q = w; q < a.n_planes[k]; ++q) a.table[map_cell(a, k, s, p, q)] = -1;
        }
    }
}

// New pages come off the stacks; then the counts take their new values.
__global__ __launch_bounds__(256) void k_map_take(MapArgs a) {
    const int s = blockIdx.x;
    const bool lead = s == 0 && blockIdx.y == 0;
    bool bad = false;
    const int old = a.old_pages[s], now = pages_wanted(a, s, old, bad);
    if (old == now && !lead) return;
    int count[3] = {0, 0, 0};
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (a.width[k]) count[k] = a.old_count[k];
    const MapSums m = map_sums(a, a.old_pages, count, s);
    if (m.code) return;
    if (blockIdx.y == 0 && threadIdx.x == 0) a.mapped[s] = now;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const int w = a.width[k];
        if (!w) continue;
        const int up = count[k] + m.all_back * w;
        if (lead && threadIdx.x == 0) *a.free_count[k] = up - m.all_more * w;
        const int top = up - 1 - m.more * w;
        for (int e = blockIdx.y * 256 + threadIdx.x; e < (now - old) * w; e += gridDim.y * 256) {
            const int p = old + e / w, plane = e % w;
            const int id = a.free_ids[k][top - e];
            if (id < 0) set_err(a.err, CDB_DEV_UNMAPPED_PAGE);
            a.table[map_cell(a, k, s, p, plane)] = id;
            if (plane == w - 1)
                for (int q = w; q < a.n_planes[k]; ++q) a.table[map_cell(a, k, s, p, q)] = id;
        }
    }
}

hipError_t launch_map_pages(const cdb_model_desc& md, int32_t* table, int S, int P, const cdb_page_pool* const* pools,
                            int core_width, const int32_t* len, int32_t* mapped, int32_t* scratch, int* err,
                            hipStream_t st) {
    if (S <= 0) return hipSuccess;
    MapArgs a{};
    a.table = table;
    a.S = S;
    a.P = P;
    a.planes = md.r_max + 2;
    const int layers[3] = {md.n_prelude, md.n_core, md.n_coda};
    const int first[3] = {0, 1, md.r_max + 1}, n[3] = {1, md.r_max, 1}, width[3] = {1, core_width, 1};
    int entries = 0;
    for (int k = 0; k < 3; ++k) {
        a.first[k] = first[k];
        a.n_planes[k] = n[k];
        if (!layers[k]) continue;
        a.width[k] = width[k];
        a.free_ids[k] = pools[k]->free_ids;
        a.free_count[k] = pools[k]->free_count;
        a.capacity[k] = pools[k]->capacity;
        entries = std::max(entries, P * width[k]);
    }
    a.len = len;
    a.mapped = mapped;
    a.old_count = scratch;
    a.old_pages = scratch + 4;
    a.err = err;
    // a whole sequence may come or go: at most 8 entries a thread, and 16 workgroups
    const dim3 grid(S, std::min(16, std::max(1, (entries + 2047) / 2048)));
    k_map_release<<<grid, 256, 0, st>>>(a);
    k_map_take<<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

// ------------------------------------------------------------------ drafted trees as rows
// One wave per tree, lane = node; every workgroup sums all trees' node counts.
// A node's ancestors by doubling: with m = the nodes seen so far and p = the
// node they end at, m |= m of p, p = p of p, six times for up to 64 nodes.
__device__ __forceinline__ uint64_t shfl64(uint64_t v, int src) {
    const uint32_t lo = __shfl((uint32_t)v, src, 64), hi = __shfl((uint32_t)(v >> 32), src, 64);
    return (uint64_t)hi << 32 | lo;
}

__global__ __launch_bounds__(256) void k_tree_rows(cdb_drafts dr, cdb_row_map out, int* err) {
    __shared__ __align__(16) int s_seq[CDB_TREE_MAX_TREES];
    __shared__ int s_len[CDB_TREE_MAX_TREES], s_n[CDB_TREE_MAX_TREES], s_end[CDB_TREE_MAX_TREES];
    __shared__ int red[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool lead = blockIdx.x == 0;
    // this wave's tree, before its node count is known
    const int t = blockIdx.x * 4 + wave;
    const bool inside = t < dr.n_trees && lane < dr.max_nodes;
    int p = inside ? dr.parent[(size_t)t * dr.max_nodes + lane] : -1;
    const int token = inside ? dr.tokens[(size_t)t * dr.max_nodes + lane] : 0;
    int n = 0;
    {
        const int q = tid < dr.n_trees ? dr.seq[tid] : -1;
        s_seq[tid] = q;
        bool ok = q >= 0 && q < dr.max_seqs;
        const int l = ok ? dr.len[q] : -1;
        if (tid < dr.n_trees) n = dr.n_nodes[tid];
        ok = ok && l >= 0 && l <= 0x7fffffff - CDB_TREE_MAX_NODES && n >= 0 && n <= dr.max_nodes;
        __syncthreads();
        if (tid < dr.n_trees) {
            bool twice = false;  // an earlier tree of this sequence
            for (int u = 0; u < dr.n_trees; u += 8) {
                int4 a[2];
                a[0] = *reinterpret_cast<const int4*>(s_seq + u);
                a[1] = *reinterpret_cast<const int4*>(s_seq + u + 4);
                const int b[8] = {a[0].x, a[0].y, a[0].z, a[0].w, a[1].x, a[1].y, a[1].z, a[1].w};
#pragma unroll
                for (int k = 0; k < 8; ++k) twice |= (u + k < tid) & (b[k] == q);
            }
            if (!ok || twice) {
                if (lead) set_err(err, CDB_DEV_BAD_INDEX);
                n = 0;
            }
            s_len[tid] = l;
        }
    }
    int total;
    const int end = block_scan256(n, red, &total);
    s_n[tid] = n;
    s_end[tid] = end;
    __syncthreads();
    // trees fit as long as their last row does
    if (lead && tid < dr.n_trees) {
        const bool fits = end <= out.capacity;
        out.row0[tid] = fits ? end - n : -1;
        if (!fits) set_err(err, CDB_DEV_BAD_INDEX);
        if (fits && (tid == dr.n_trees - 1 || s_end[tid + 1] > out.capacity)) *out.n_rows = end;
        if (!fits && tid == 0) *out.n_rows = 0;
    }
    if (lead && tid == 0 && dr.n_trees == 0) *out.n_rows = 0;
    if (t >= dr.n_trees || s_end[t] > out.capacity) return;
    const int nt = s_n[t], row0 = s_end[t] - nt, base = s_len[t];
    const bool live = lane < nt;
    if (!live) p = -1;
    if (live && (p < -1 || p >= lane)) {
        set_err(err, CDB_DEV_BAD_INDEX);
        p = -1;
    }
    uint64_t m = 1ull << lane;
#pragma unroll
    for (int i = 0; i < 6; ++i) {
        const uint64_t pm = shfl64(m, p & 63);
        const int pp = __shfl(p, p & 63, 64);
        if (p >= 0) {
            m |= pm;
            p = pp;
        }
    }
    if (live) {
        const int r = row0 + lane;
        out.seq[r] = s_seq[t];
        out.pos[r] = base + lane;
        out.base[r] = base;
        out.rope_pos[r] = base + __popcll(m) - 1;
        out.tokens[r] = token;
        out.mask[r] = m;
    }
}

hipError_t launch_tree_rows(const cdb_drafts& d, const cdb_row_map& out, int* err, hipStream_t st) {
    k_tree_rows<<<std::max(1, (d.n_trees + 3) / 4), 256, 0, st>>>(d, out, err);
    return hipGetLastError();
}

// ------------------------------------------------------------------ acceptance
// One wave per tree, lane = node: each step asks all nodes at once whether they
// hang below the current one and hold the wanted token.
__global__ __launch_bounds__(256) void k_tree_accept(cdb_drafts dr, const int32_t* __restrict__ row0,
                                                     const int32_t* __restrict__ next_ids, int n_rows,
                                                     const int32_t* __restrict__ first_ids, cdb_accepted out, int* err) {
    const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= dr.n_trees) return;
    const int r0 = row0[t];
    int n = dr.n_nodes[t];
    int want = first_ids[t];
    if (n < 0 || n > dr.max_nodes) n = 0;
    bool live = lane < n && r0 >= 0;
    if (live && r0 > n_rows - 1 - lane) {
        set_err(err, CDB_DEV_BAD_INDEX);
        live = false;
    }
    const size_t at = (size_t)t * dr.max_nodes + lane;
    const int p = live ? dr.parent[at] : -2, tok = live ? dr.tokens[at] : 0, says = live ? next_ids[r0 + lane] : 0;
    live = live && p < lane;
    int cur = -1, count = 0, path = -1;
    while (true) {
        const uint64_t hit = __ballot(live && p == cur && tok == want);
        if (!hit) break;
        cur = __ffsll((unsigned long long)hit) - 1;  // past the last one: its parent comes before it
        if (lane == count) path = cur;
        want = __shfl(says, cur, 64);
        ++count;
    }
    if (lane < dr.max_nodes) out.path[at] = path;
    if (lane == 0) {
        out.count[t] = count;
        out.next[t] = want;
    }
}

hipError_t launch_tree_accept(const cdb_drafts& d, const int32_t* row0, const int32_t* next_ids, int n_rows,
                              const int32_t* first_ids, const cdb_accepted& out, int* err, hipStream_t st) {
    if (d.n_trees <= 0) return hipSuccess;
    k_tree_accept<<<(d.n_trees + 3) / 4, 256, 0, st>>>(d, row0, next_ids, n_rows, first_ids, out, err);
    return hipGetLastError();
}

// ------------------------------------------------------------------ commit
// Workgroup (unit, tree): one layer of one plane.  Entry i of the path goes from
// position len + path[i] to len + i <= it.  Every wave reads what the move needs by
// itself (lane = path entry, page, or plane), so nothing waits at a barrier; the
// chain of dependent loads (path and sequence, length, page ids, data) bounds all
// but large calls.  A thread owns 16-byte columns of the (K/V, head, dim) entry and
// takes the moves in order, loading eight before it stores them: move i's
// destination is no later move's source (path[j] > path[i] >= i for j > i), so
// nothing is overwritten before it is read.
constexpr int kCommitBatch = 8;

__global__ __launch_bounds__(256) void k_tree_commit(int H, int hd, KvTarget kv, int plane0, int n_planes,
                                                     cdb_drafts dr, const int32_t* __restrict__ path_,
                                                     const int32_t* __restrict__ count_, int* err) {
    const int t = blockIdx.y, lane = threadIdx.x & 63;
    const int layer = blockIdx.x / n_planes, plane = plane0 + blockIdx.x % n_planes;
    const bool tells = blockIdx.x == 0 && threadIdx.x == 0;
    const int n = count_[t], sq = dr.seq[t];
    const int path = lane < dr.max_nodes ? path_[(size_t)t * dr.max_nodes + lane] : -1;
    bool bad = false;
    for (int k = lane; k < t; k += 64) bad |= dr.seq[k] == sq;  // an earlier tree of this sequence
    if (n == 0) return;
    bad |= n < 0 || n > dr.max_nodes || sq < 0 || sq >= kv.max_seqs || sq >= dr.max_seqs;
    const int before = __shfl_up(path, 1, 64);
    bad |= lane < n && (path < 0 || path >= dr.max_nodes || (lane > 0 && before >= path));
    if (__any(bad)) {
        if (tells) set_err(err, CDB_DEV_BAD_INDEX);
        return;
    }
    // the moves, in order: path increases, so from the first i with path[i] > i on all entries move
    const uint64_t moved = __ballot(lane < n && path != lane);
    const int base = dr.len[sq];
    const int top = __builtin_amdgcn_readlane(path, n - 1);  // the highest node of the path
    if (base < 0 || base > kv.max_pages * kPage || base + top >= kv.max_pages * kPage) {
        if (tells) set_err(err, CDB_DEV_BAD_INDEX);
        return;
    }
    if (!moved) return;
    const int i0 = __ffsll((unsigned long long)moved) - 1;
    const int pga = (base + i0) / kPage, pgb = (base + top) / kPage;  // pages the moves touch, at most 5
    const int32_t* pt = kv.page_table + (size_t)sq * kv.n_planes * kv.max_pages;
    // lane = page, then lane = plane of the pool with some, or all, of the same pages: the
    // lowest of those that share all moves them once
    const int pid = pga + lane <= pgb ? pt[(size_t)plane * kv.max_pages + pga + lane] : 0;
    int same = 0;
    if (lane < n_planes && plane0 + lane != plane) {
        const int32_t* other = pt + (size_t)(plane0 + lane) * kv.max_pages;
        const int32_t* own = pt + (size_t)plane * kv.max_pages;
        for (int g = pga; g <= pgb; ++g) same += other[g] == own[g];
    }
    if (__any(pid < 0 || pid >= kv.n_pages)) {
        if (threadIdx.x == 0) set_err(err, CDB_DEV_UNMAPPED_PAGE);
        return;
    }
    if (__any(same > 0 && same <= pgb - pga)) {
        if (threadIdx.x == 0) set_err(err, CDB_DEV_BAD_INDEX);
        return;
    }
    if (__any(same > 0 && plane0 + lane < plane)) return;
    const int vec_per_head = hd / 8, nvec = 2 * H * vec_per_head;
    auto entry = [&](int pos) {
        const int id = __builtin_amdgcn_readlane(pid, pos / kPage - pga);
        return kv.pool + kv_offset(layer, id, kv.n_pages, 0, 0, H, pos % kPage, hd);
    };
    for (int v0 = 0; v0 < nvec; v0 += 256) {  // whole waves stay in the loop: they read one another's lanes
        const int v = v0 + (int)threadIdx.x;
        const bool in = v < nvec;
        const int kvh = v / vec_per_head, e = v - kvh * vec_per_head;
        const size_t off = in ? (size_t)kvh * kPage * hd + e * 8 : 0;
        for (int b = i0; b < n; b += kCommitBatch) {
            u32x4 buf[kCommitBatch];  // past the last move: that one's source again
#pragma unroll
            for (int u = 0; u < kCommitBatch; ++u)
                buf[u] = *reinterpret_cast<const u32x4*>(entry(base + __builtin_amdgcn_readlane(path, min(b + u, n - 1))) + off);
#pragma unroll
            for (int u = 0; u < kCommitBatch; ++u)
                if (in && b + u < n) *reinterpret_cast<u32x4*>(entry(base + b + u) + off) = buf[u];
        }
    }
}

hipError_t launch_tree_commit(const cdb_model_desc& md, const KvTarget& kv, int plane0, int n_planes,
                              const cdb_drafts& d, const cdb_accepted& acc, int* err, hipStream_t st) {
    if (d.n_trees <= 0 || kv.n_layers <= 0) return hipSuccess;
    k_tree_commit<<<dim3(kv.n_layers * n_planes, d.n_trees), 256, 0, st>>>(md.n_heads, md.head_dim, kv, plane0, n_planes, d,
                                                                          acc.path, acc.count, err);
    return hipGetLastError();
}

}  // namespace cdb
