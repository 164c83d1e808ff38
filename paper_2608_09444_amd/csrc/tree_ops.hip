// Row, page and cache bookkeeping of drafted token trees: page tables from
// sequence lengths, drafted trees as the rows of a stage call, greedy acceptance,
// and the move of the accepted K/V.  All are bound by latency, so each is one launch
// (large page mappings two) whose workgroups recompute the small prefix sums they
// need instead of waiting for one another.
#include <algorithm>

#include "cdb_internal.h"

namespace cdb {

// Inclusive prefix sums over a 256-thread workgroup; total = the whole sums.
// red: 4 x N ints of LDS, free again after the call's last barrier.
template <int N>
__device__ __forceinline__ void block_scan256(int (&v)[N], int* red, int (&total)[N]) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int u = __shfl_up(v[k], o, 64);
            if (lane >= o) v[k] += u;
        }
    __syncthreads();
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < N; ++k) red[w * N + k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        int before = 0;
        total[k] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < w) before += red[i * N + k];
            total[k] += red[i * N + k];
        }
        v[k] += before;
    }
}

// ------------------------------------------------------------------ page tables
// Entries of the table to a workgroup, of up to 512.  Chosen when calls could not be
// taken back yet: 128 sequences of 32 planes leaving and coming took 20.1 us (two
// calls; 24.5 at 2048 entries, 21.8 at 256 workgroups), 64 that grow by 16 tokens and
// back 8.1 (8.5 at 2048; 7.3 in one workgroup, which takes 149 us for the former).
constexpr int kMapEntries = 512, kMapGroups = 512;
// Up to so many workgroups the last one takes a call back, above a second launch
// (k_map_pages says why): the former 28.1 us against 24.0 of that launch, the latter
// 9.4 against 11.5.  24 workgroups that leave and come, 4 planes: 13.3 against 14.1; 384
// that grow and are cut back, 32 planes: 20.1 against 21.3.
constexpr int kMapThrough = 64;
constexpr int kMapHole = 1 << 30;  // left in the workspace's header for the launch that takes back

struct MapArgs {
    int32_t* table;
    int S, P, planes;          // sequences, pages per plane, r_max + 2
    int width[3];              // distinct pages per token page in the pools (0: the stage has no layers)
    int first[3], n_planes[3]; // planes of each pool; plane k of it has page min(k, width - 1)
    int32_t* free_ids[3];
    int32_t* free_count[3];
    int capacity[3];
    const int32_t* len;
    int32_t* mapped;
    int* ws;                   // [0] error code, [kWsArrive] workgroups that are through
    bool through;              // stores go past this XCD's L2
    bool undo;                 // the second launch: take back what the first one did, if it met a hole
};

struct MapPages {
    int old, now;
};
__device__ __forceinline__ MapPages map_pages_of(const MapArgs& a, int s, bool& bad) {
    const int old = a.mapped[s], l = a.len[s];
    bad |= old < 0 || old > a.P || l > a.P * kPage;
    return {old, l < 0 ? old : (int)(((unsigned)l + kPage - 1) / kPage)};
}

// The cell of entry e of a side: pages given back (back) or taken, in (sequence,
// page, plane) order over the planes with a page of their own.  before[i] = pages
// of the sequences before i * per.
__device__ __forceinline__ size_t map_cell(const MapArgs& a, int k, const int* before, int per, int e, bool back) {
    const int w = a.width[k], page = e / w;
    int i = 0;
#pragma unroll
    for (int o = 128; o > 0; o >>= 1)
        if (before[i + o] <= page) i += o;
    int left = page - before[i], s = i * per, p = 0;
    for (; s < a.S; ++s) {  // always found
        bool bad = false;
        const MapPages m = map_pages_of(a, s, bad);
        const int n = back ? m.old - m.now : m.now - m.old;
        if (left < n) {
            p = (back ? m.now : m.old) + left;
            break;
        }
        left -= max(n, 0);
    }
    return ((size_t)min(s, a.S - 1) * a.planes + a.first[k] + (e - page * w)) * a.P + p;
}

__device__ __forceinline__ void map_store(const MapArgs& a, int32_t* p, int value) {
    if (a.through)
        __hip_atomic_store(p, value, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    else
        *p = value;
}
// Entry j's cell, and with the last page that a token page has the planes that share it.
__device__ __forceinline__ void map_put(const MapArgs& a, int k, size_t cell, int j, int value) {
    const int w = a.width[k];
    map_store(a, a.table + cell, value);
    if (j % w == w - 1)
        for (int q = w; q < a.n_planes[k]; ++q) map_store(a, a.table + cell + (size_t)(q - w + 1) * a.P, value);
}

// Every workgroup sums the page counts of all sequences itself (a
// thread `per` of them) and takes its share of the entries.  Entry j that is given
// back lands on the stack at count + all - 1 - j, and the j-th one that is taken
// comes from there, so its thread has it already; the others come off the stack
// below `count`, where this call writes nothing.  The workgroup that is through
// last writes mapped and the counts, which all have read by then.
//
// A page id below 0, in a cell to be given back or on the stack, shows only while
// entries move, and then the whole call is taken back: the ids that were given back
// all stand on the stack above `count`, so the last workgroup puts them into their
// cells again and unmaps the taken ones.  It must not be overtaken by the others'
// stores, so these go to memory (agent scope) and are through before a workgroup
// counts itself in; of large tables, whose scattered words cost more that way than
// another launch, a second launch of one workgroup takes back.
__global__ __launch_bounds__(256) void k_map_pages(MapArgs a) {
    __shared__ int s_back[256], s_more[256], red[8], s_bad, s_last, s_hole;
    const int tid = threadIdx.x, per = (a.S + 255) / 256;
    if (a.undo && a.ws[kWsArrive] != kMapHole) return;
    if (tid == 0) s_bad = s_hole = 0;
    int count[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) count[k] = a.width[k] ? *a.free_count[k] : 0;
    int v[2] = {0, 0}, all[2];
    bool bad = false;
    for (int s = tid * per; s < min(a.S, (tid + 1) * per); ++s) {
        const MapPages m = map_pages_of(a, s, bad);
        v[0] += max(m.old - m.now, 0);
        v[1] += max(m.now - m.old, 0);
    }
    const int own[2] = {v[0], v[1]};
    block_scan256(v, red, all);
    if (bad) s_bad = 1;
    s_back[tid] = v[0] - own[0];
    s_more[tid] = v[1] - own[1];
    __syncthreads();
    int code = s_bad ? CDB_DEV_BAD_INDEX : 0;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        if (!a.width[k]) continue;
        const int c = count[k], up = c + all[0] * a.width[k];
        if (c < 0 || c > a.capacity[k])
            code = CDB_DEV_BAD_INDEX;
        else if (!code && (up > a.capacity[k] || up < all[1] * a.width[k]))
            code = CDB_DEV_NO_PAGES;
    }
    if (!code && !a.undo)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int w = a.width[k];
            if (!w) continue;
            const int back = all[0] * w, more = all[1] * w, top = count[k] + back - 1;
            for (int j = blockIdx.x * 256 + tid; j < max(back, more); j += gridDim.x * 256) {
                int id;
                if (j < back) {
                    const size_t cell = map_cell(a, k, s_back, per, j, true);
                    id = a.table[cell];
                    map_put(a, k, cell, j, -1);
                    map_store(a, a.free_ids[k] + top - j, id);
                } else {
                    id = a.free_ids[k][top - j];
                }
                if (id < 0) s_hole = 1;
                if (j < more) map_put(a, k, map_cell(a, k, s_more, per, j, false), j, id);
            }
        }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's stores have reached memory
    __syncthreads();
    if (tid == 0) {  // workgroups that are through, those with a hole from bit 16 on
        const int own = 1 + (s_hole << 16), n = gridDim.x == 1 ? 0 : atomicAdd(a.ws + kWsArrive, own);
        s_last = (n & 0xffff) == (int)gridDim.x - 1;
        s_hole = (n + own) >> 16 | a.undo;
        if (s_last) {
            if (n || a.undo) atomicExch(a.ws + kWsArrive, s_hole && !a.through ? kMapHole : 0);
            if (code || s_hole) set_err(a.ws, code ? code : CDB_DEV_UNMAPPED_PAGE);
        }
    }
    __syncthreads();
    if (!s_last || code) return;
    if (s_hole && !a.through) return;
    if (s_hole) {
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int w = a.width[k], back = all[0] * w, more = all[1] * w, top = count[k] + back - 1;
            for (int j = tid; j < back; j += 256)
                map_put(a, k, map_cell(a, k, s_back, per, j, true), j,
                        __hip_atomic_load(a.free_ids[k] + top - j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
            for (int j = tid; j < more; j += 256) map_put(a, k, map_cell(a, k, s_more, per, j, false), j, -1);
        }
        return;
    }
    for (int s = tid; s < a.S; s += 256) {
        const MapPages m = map_pages_of(a, s, bad);
        if (m.now != m.old) a.mapped[s] = m.now;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (tid == k && a.width[k]) *a.free_count[k] = count[k] + (all[0] - all[1]) * a.width[k];
}

hipError_t launch_map_pages(const cdb_model_desc& md, int32_t* table, int S, int P, const cdb_page_pool* const* pools,
                            int core_width, const int32_t* len, int32_t* mapped, int* ws, hipStream_t st) {
    if (S <= 0) return hipSuccess;
    MapArgs a{};
    a.table = table;
    a.S = S;
    a.P = P;
    a.planes = md.r_max + 2;
    const int layers[3] = {md.n_prelude, md.n_core, md.n_coda};
    const int first[3] = {0, 1, md.r_max + 1}, n[3] = {1, md.r_max, 1}, width[3] = {1, core_width, 1};
    int64_t entries = 0;
    for (int k = 0; k < 3; ++k) {
        a.first[k] = first[k];
        a.n_planes[k] = n[k];
        if (!layers[k]) continue;
        a.width[k] = width[k];
        a.free_ids[k] = pools[k]->free_ids;
        a.free_count[k] = pools[k]->free_count;
        a.capacity[k] = pools[k]->capacity;
        entries = std::max(entries, (int64_t)S * P * width[k]);
    }
    a.len = len;
    a.mapped = mapped;
    a.ws = ws;
    // every sequence may come or go, but most calls change few of the pages
    const int groups = (int)std::min<int64_t>(kMapGroups, std::max<int64_t>(1, entries / kMapEntries));
    a.through = groups <= kMapThrough;
    k_map_pages<<<groups, 256, 0, st>>>(a);
    if (!a.through) {
        a.through = a.undo = true;
        k_map_pages<<<1, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

// ------------------------------------------------------------------ drafted trees as rows
// One wave per tree, lane = node; every workgroup sums all trees' node counts.
// Bound by latency (sequence, its length, the scan): 64 trees of 4 in 4.0 us, 4 of
// 64 in 3.0, where an empty kernel takes 1.7.
// A node's ancestors by doubling: with m = the nodes seen so far and p = the
// node they end at, m |= m of p, p = p of p, six times for up to 64 nodes.
__device__ __forceinline__ uint64_t shfl64(uint64_t v, int src) {
    const uint32_t lo = __shfl((uint32_t)v, src, 64), hi = __shfl((uint32_t)(v >> 32), src, 64);
    return (uint64_t)hi << 32 | lo;
}

// Positions of a tree behind l committed ones are in 32 bits.
__device__ __forceinline__ bool tree_length_ok(int l) { return l >= 0 && l <= 0x7fffffff - CDB_TREE_MAX_NODES; }

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
        ok = ok && tree_length_ok(l) && n >= 0 && n <= dr.max_nodes;
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
    int ends[1] = {n}, total[1];
    block_scan256(ends, red, total);
    const int end = ends[0];
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
// hang below the current one and hold the wanted token.  2.5 us for 64 trees of 4,
// 2.9 for 4 of 64.  A tree that got no rows because of its sequence or length stands
// in row0 where the next tree's rows begin, so both are looked at here as well (0.25
// us of it).
__global__ __launch_bounds__(256) void k_tree_accept(cdb_drafts dr, const int32_t* __restrict__ row0,
                                                     const int32_t* __restrict__ next_ids, int n_rows,
                                                     const int32_t* __restrict__ first_ids, cdb_accepted out, int* err) {
    const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= dr.n_trees) return;
    const int r0 = row0[t];
    int n = dr.n_nodes[t];
    int want = first_ids[t];
    bool refused = false;
    if (dr.seq) {
        const int sq = dr.seq[t];
        for (int k = lane; k < t; k += 64) refused |= dr.seq[k] == sq;  // an earlier tree of this sequence
        refused |= sq < 0 || sq >= dr.max_seqs;
        if (dr.len && !__any(refused)) refused = !tree_length_ok(dr.len[sq]);
        refused = __any(refused);
    }
    if (n < 0 || n > dr.max_nodes) n = 0;
    if (refused && n > 0) {
        if (lane == 0) set_err(err, CDB_DEV_BAD_INDEX);
        n = 0;
    }
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
// Workgroup (unit, tree): one layer of one plane of one stage.  Entry i of the path
// goes from position len + path[i] to len + i <= it.  Every wave reads what the move
// needs by itself (lane = path entry, page, or plane), so nothing waits at a
// barrier; the chain of dependent loads (path and sequence, length, page ids, data)
// bounds it (32 trees of 8 over 48 layer planes: 18 MB in 6.5 us, 2.8 TB/s).  A
// thread owns 16-byte columns of the (K/V, head, dim) entry, two at once, and takes
// the moves in order, loading eight before it stores them: move i's destination is
// no later move's source (path[j] > path[i] >= i for j > i), so nothing is
// overwritten before it is read.
constexpr int kCommitBatch = 8;
// Up to so many (unit, tree) pairs, workgroups share a unit's columns; by pairs, shared
// and not, trees of 8 over 48 layer planes of 16 x 128 heads: 240 4.1 and 4.2 us, 432 4.3
// both, 480 5.3 and 4.6, 768 6.4 and 5.0, 1536 8.8 and 6.5; over 34 of 55 x 96: 272 5.1 and
// 6.5, 408 5.2 and 5.6, 544 7.0 and 6.4; one tree of 24 over 96 of 16 x 128: 4.6 and 5.3.
constexpr int kCommitSplit = 448;

struct CommitStages {
    uint16_t* pool[3];
    int n_pages[3];
    int plane0[3], n_planes[3];
    int first[3];  // unit
    const int32_t* page_table;
    int max_seqs, max_pages, planes;
};

__global__ __launch_bounds__(256) void k_tree_commit(int H, int hd, CommitStages stages, cdb_drafts dr,
                                                     const int32_t* __restrict__ path_,
                                                     const int32_t* __restrict__ count_, int* err) {
    const int t = blockIdx.y, lane = threadIdx.x & 63;
    const int unit = blockIdx.x, stage = (unit >= stages.first[1]) + (unit >= stages.first[2]);
    const int plane0 = stages.plane0[stage], n_planes = stages.n_planes[stage], in_stage = unit - stages.first[stage];
    const int layer = in_stage / n_planes, plane = plane0 + in_stage % n_planes;
    struct {
        uint16_t* pool;
        int n_pages;
        const int32_t* page_table;
        int max_seqs, max_pages, n_planes;
    } kv{stages.pool[stage], stages.n_pages[stage], stages.page_table, stages.max_seqs, stages.max_pages,
         stages.planes};
    const bool tells = blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0;
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
    // two columns a thread; whole waves stay in the loop, as they read one another's lanes
    for (int v0 = blockIdx.z * 256; v0 < nvec; v0 += gridDim.z * 512) {
        size_t off[2];
        bool in[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int v = v0 + y * gridDim.z * 256 + (int)threadIdx.x;
            in[y] = v < nvec;
            const int kvh = v / vec_per_head, e = v - kvh * vec_per_head;
            off[y] = in[y] ? (size_t)kvh * kPage * hd + e * 8 : 0;
        }
        for (int b = i0; b < n; b += kCommitBatch) {
            u32x4 buf[2][kCommitBatch];
#pragma unroll
            for (int u = 0; u < kCommitBatch; ++u)
                if (b + u < n) {
                    const uint16_t* at = entry(base + __builtin_amdgcn_readlane(path, b + u));
#pragma unroll
                    for (int y = 0; y < 2; ++y) buf[y][u] = *reinterpret_cast<const u32x4*>(at + off[y]);
                }
#pragma unroll
            for (int u = 0; u < kCommitBatch; ++u)
                if (b + u < n) {
                    uint16_t* at = entry(base + b + u);
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        if (in[y]) *reinterpret_cast<u32x4*>(at + off[y]) = buf[y][u];
                }
        }
    }
}

hipError_t launch_tree_commit(const cdb_model_desc& md, const KvTarget (&kv)[3], const cdb_drafts& d,
                              const cdb_accepted& acc, int* err, hipStream_t st) {
    CommitStages s{};
    int units = 0;
    for (int k = 0; k < 3; ++k) {
        s.pool[k] = kv[k].pool;
        s.n_pages[k] = kv[k].n_pages;
        s.plane0[k] = k == 1 ? 1 : kv[k].plane_fixed;
        s.n_planes[k] = k == 1 ? md.r_max : 1;
        s.first[k] = units;
        units += std::max(0, kv[k].n_layers) * s.n_planes[k];
    }
    s.page_table = kv[0].page_table;
    s.max_seqs = kv[0].max_seqs;
    s.max_pages = kv[0].max_pages;
    s.planes = kv[0].n_planes;
    if (d.n_trees <= 0 || units == 0) return hipSuccess;
    const int parts = (int64_t)units * d.n_trees <= kCommitSplit ? (2 * md.n_heads * md.head_dim / 8 + 255) / 256 : 1;
    k_tree_commit<<<dim3(units, d.n_trees, parts), 256, 0, st>>>(md.n_heads, md.head_dim, s, d, acc.path, acc.count, err);
    return hipGetLastError();
}

}  // namespace cdb
