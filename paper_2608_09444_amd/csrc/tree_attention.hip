// Attention of drafted token trees over the paged, depth-indexed KV cache: row i
// attends to positions 0..base-1 of its sequence and to the positions base + j
// whose bit j of its mask is set (its ancestors and itself), in its own plane.
//
// The rows of one tree share their context, so its K and V are read once for up
// to 16, 32 or 64 of them and multiplied on MFMA (v_mfma_f32_16x16x32_bf16); with
// so few rows per byte the kernel is bound by HBM.
//
// k_tree_plan (one workgroup, once per stage call) cuts the rows into tiles:
// adjacent rows of one sequence, plane and base, at most 16 NT of them.  A tile's
// context is cut into segments (tree_segments, by its base alone), and a
// work item is one segment of one tile, for each head.
//
// k_tree_attn: a workgroup takes items in turn; its 4 waves deal the segment's
// pages among them in pairs (32 keys), and each keeps an online softmax of its
// own for the tile's rows.  Per pair:
//   S^T = K Q^T: A = the K rows as loaded from the cache (lane = key, 16 bytes of
//     it), B = q, split into bf16 hi + lo parts (about 16 bits of it).  A lane then
//     holds one row's scores at 4 keys of either page.
//   online softmax per row in the exp2 domain; the running maximum goes over the
//     four lanes of a row (two lane swaps), the sum stays apart until the end.
//   O^T += V^T P^T: B = P, hi + lo again, and already where the scores left it:
//     the order of the 32 keys in the product is free, so lane group g takes keys
//     4g..4g+3 of both pages.  A = V^T, read from the key-major rows in LDS with
//     the transposing read (ds_read_b64_tr_b16).
// The pair after the current one is in flight in registers meanwhile.  The waves'
// states are merged through LDS; several segments' through memory, by the
// workgroup that arrives last, in segment order.
//
// Masks: only pages that reach past base take the masked path.  There a score that
// a row does not see becomes -inf (p = 0), and V of keys that no row of the tile
// sees is cleared; a V that is not finite at a key that some rows see is taken out
// of the product, which would multiply it by the others' zeros, and added to those
// rows alone.
//
// Nothing in a row's arithmetic depends on the other rows: not its tile, not the
// segments, not the wave that takes a page.
#include <algorithm>

#include "cdb_internal.h"

namespace cdb {

constexpr int kTreeWaves = 8;
constexpr int kTreeSegs = 16;  // most segments of a context
constexpr int kTreeRows = 32;  // most rows of a workgroup

constexpr int kTreeSegPages = 128;  // pages of a segment, unless that makes too many

// Segments of a context whose last committed position is on page npg - 1, and the
// pages of each (the last one has the rest).
__host__ __device__ __forceinline__ int tree_segments(int npg, int* pages) {
    int n = (npg + kTreeSegPages - 1) / kTreeSegPages;
    n = n > kTreeSegs ? kTreeSegs : n;
    constexpr int round = 2 * kTreeWaves;  // the waves' pairs
    *pages = (npg + round * n - 1) / (round * n) * round;
    return (npg + *pages - 1) / *pages;
}

struct TreeItem {
    uint64_t seen;       // mask bits of any row of the tile
    int row0, n;         // the tile's rows
    int base;
    int seq, plane;
    int p0, p1;          // the segment's pages
    int seg, nseg;
    int pad[5];
};

struct TreeScratch {
    int* n_items;
    TreeItem* items;  // [rows][kTreeSegs]
    int* arrive;      // [rows][H], by a workgroup's first row, zero between launches
    float* part;      // [rows][H][kTreeSegs][hd + 2]: sums, maximum, weight
    size_t bytes;
};
static TreeScratch tree_scratch(void* at, int H, int hd, int rows) {
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    unsigned char* p = static_cast<unsigned char*>(at);
    size_t off = 256;
    TreeScratch t{};
    t.n_items = reinterpret_cast<int*>(p);
    t.items = reinterpret_cast<TreeItem*>(p + off);
    off = up(off + ((size_t)rows * kTreeSegs + 8) * sizeof(TreeItem));  // 8: read, not used, past the last
    t.arrive = reinterpret_cast<int*>(p + off);
    off = up(off + (size_t)rows * H * 4);
    t.part = reinterpret_cast<float*>(p + off);
    off = up(off + (size_t)rows * H * kTreeSegs * (hd + 2) * 4);
    t.bytes = off;
    return t;
}
size_t tree_scratch_bytes(const cdb_model_desc& d, int rows) {
    return rows > 0 ? tree_scratch(nullptr, d.n_heads, d.head_dim, rows).bytes : 0;
}

// ------------------------------------------------------------------ plan
// Thread = row.  cap = rows per tile.
__global__ __launch_bounds__(256) void k_tree_plan(KvTarget kv, const int32_t* __restrict__ seq, cdb_tree tree, int M,
                                                   int H, int cap, TreeScratch ts, int* err,
                                                   const int32_t* __restrict__ dn) {
    __shared__ int s_seq[256], s_plane[256], s_base[256];
    __shared__ uint64_t s_mask[256];
    __shared__ uint64_t s_run[4], s_end[4];  // by row: a run starts; a tile or a skipped row starts
    __shared__ int s_sum[4];
    const int i = threadIdx.x, lane = i & 63, w = i >> 6;
    const int n = live_rows(dn, M);
    const int limit = kv.max_pages * kPage;
    int sq = -1, plane = -1, base = 0;
    uint64_t mask = 0;
    bool ok = false;
    if (i < n) {
        sq = seq[i];
        base = tree.base[i];
        mask = tree.mask[i];
        plane = kv.c_row ? kv.c_row[i] + 1 : kv.plane_fixed;
        ok = sq >= 0 && sq < kv.max_seqs && base >= 0 && base <= limit &&
             (kv.c_row ? plane >= 1 && plane <= kv.n_planes - 2 : plane >= 0 && plane < kv.n_planes);
        ok = ok && (!mask || base + 63 - __clzll((long long)mask) < limit);
        if (!ok) set_err(err, CDB_DEV_UNMAPPED_PAGE);
    }
    s_seq[i] = ok ? sq : -1;
    s_plane[i] = plane;
    s_base[i] = base;
    s_mask[i] = mask;
    __syncthreads();
    const bool run = ok && !(i > 0 && s_seq[i - 1] == sq && s_plane[i - 1] == plane && s_base[i - 1] == base);
    const uint64_t runs = __ballot(run);
    if (lane == 0) s_run[w] = runs;
    __syncthreads();
    // the row at which i's run started
    int start = i;
    {
        uint64_t b = runs & (~0ull >> (63 - lane));
        int word = w;
        while (!b && word > 0) b = s_run[--word];
        if (b) start = word * 64 + 63 - __clzll((long long)b);
    }
    const bool first = ok && (i - start) % cap == 0;
    const uint64_t ends = __ballot(first || !ok);
    if (lane == 0) s_end[w] = ends;
    __syncthreads();
    int nseg = 0, rows = 0, npg = 0, sp = 0;
    uint64_t seen = 0;
    if (first) {
        uint64_t b = lane == 63 ? 0 : ends & (~0ull << (lane + 1));
        int word = w;
        while (!b && word < 3) b = s_end[++word];
        rows = (b ? word * 64 + __ffsll((unsigned long long)b) - 1 : 256) - i;
        for (int k = 0; k < rows; ++k) seen |= s_mask[i + k];
        const int last = seen ? base + 63 - __clzll((long long)seen) : base - 1;
        npg = last < 0 ? 0 : last / kPage + 1;
        nseg = tree_segments(base / kPage + 1, &sp);
    }
    // items in tile order
    int at = nseg;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(at, o, 64);
        if (lane >= o) at += u;
    }
    if (lane == 63) s_sum[w] = at;
    __syncthreads();
    int total = 0;
    for (int k = 0; k < 4; ++k) {
        if (k < w) at += s_sum[k];
        total += s_sum[k];
    }
    if (i == 0) *ts.n_items = total;
    at -= nseg;
    for (int sg = 0; sg < nseg; ++sg) {
        TreeItem it{};
        it.seen = seen;
        it.row0 = i;
        it.n = rows;
        it.base = base;
        it.seq = sq;
        it.plane = plane;
        it.p0 = sg * sp;
        it.p1 = sg == nseg - 1 ? npg : (sg + 1) * sp;
        it.seg = sg;
        it.nseg = nseg;
        ts.items[at + sg] = it;
    }
    if (nseg > 1)
        for (int r = 0; r < rows; r += kTreeRows)
            for (int h = 0; h < H; ++h) ts.arrive[(i + r) * H + h] = 0;
}

// ------------------------------------------------------------------ attention
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float over_rows_max(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float over_rows_sum(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Bits 0..3: whether positions base + off .. base + off + 3 are visible, those
// below base always.  (What follows from it is written as selects: out of
// branches the compiler has lost the write of a vector's last element.)
__device__ __forceinline__ uint32_t sees4(uint64_t mask, int off) {
    const int up = off < 0 ? 0 : off > 63 ? 63 : off, below = off < -4 ? 4 : off < 0 ? -off : 0;
    const uint32_t m = off > 63 ? 0 : (uint32_t)(mask >> up) & 15u;
    return (m << below | ((1u << below) - 1)) & 15u;
}

// 2^x by the hardware instruction: within an ulp, results below the smallest normal
// number are 0 (weights that far below the largest do not show in 32-bit sums).
__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// Rows of a page in LDS are padded so that what a read takes from several rows at
// once lies on different banks: K 16 bytes (16 rows at one 16-byte piece), V 32
// (8 rows at one 32-byte piece, by half a wave).
template <int HD>
constexpr int kKPitch = HD + 8;
template <int HD>
constexpr int kVPitch = HD + 16;

struct Work {
    TreeItem it;     // row0, n: this workgroup's rows
    int head;
    int p, mine;     // this wave's first page, and how many pairs of pages it has
};

template <int HD, int NT>
struct TreeState {
    floatx4 o[NT][HD / 16];
    float m[NT], l[NT];  // l: this lane's keys only
};

template <int HD, int NT, bool HALVES>
__global__ __launch_bounds__(kTreeWaves * 64) void k_tree_attn(
    const float* __restrict__ q, KvTarget kv, cdb_tree tree, int H, TreeScratch ts, uint16_t* __restrict__ out, int* err) {
    constexpr int NJ = HD / 32, NB = HD / 16, CPR = HD / 8;  // K steps, dim blocks, 16-byte pieces of a row
    constexpr int PITCH = HD + 4;
    constexpr int ROWS = 16 * NT, THREADS = kTreeWaves * 64;
    constexpr int REC = HD + 2;
    constexpr bool QLDS = NT > 1;
    // K and V of the waves' pairs, then the q operands; the waves' states take their place
    constexpr int KP = kKPitch<HD>, VP = kVPitch<HD>, KROWS = 2 * kPage;
    constexpr int VBYTES = kTreeWaves * KROWS * (KP + VP) * 2, QBYTES = QLDS ? NT * NJ * 2 * 1024 : 0;
    constexpr int OBYTES = kTreeWaves * ROWS * PITCH * 4;
    struct Factors {  // of the rows: the waves' maxima, weights and factors, the sum, the segments' factors
        float m[kTreeWaves][ROWS], l[kTreeWaves][ROWS], f[kTreeWaves][ROWS], den[ROWS], seg[kTreeSegs][ROWS];
    };
    constexpr int ABYTES = VBYTES + QBYTES, BBYTES = OBYTES + (int)sizeof(Factors);
    __shared__ __align__(16) unsigned char smem[ABYTES > BBYTES ? ABYTES : BBYTES];
    __shared__ int s_last;
    Factors& sf = *reinterpret_cast<Factors*>(smem + OBYTES);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int d = H * HD;
    const float qscale = 1.4426950408889634f / sqrtf((float)HD);
    uint16_t* sk = reinterpret_cast<uint16_t*>(smem) + wave * KROWS * (KP + VP);
    uint16_t* sv = sk + KROWS * KP;

    // Work w: with two halves, workgroups 8 apart, which run on one XCD at one time,
    // take the halves of a tile's rows, so that the second one's K and V come from
    // that XCD's L2.
    const int n_heads = *ts.n_items * H;  // items x heads
    const int n_work = !HALVES ? n_heads : (n_heads + 7) / 8 * 16;
    auto load_work = [&](int w) {
        const int ih = !HALVES ? w : w / 16 * 8 + w % 8, r = !HALVES ? 0 : w / 8 % 2 * kTreeRows;
        Work x;
        x.it = ts.items[ih / H];
        x.head = ih % H;
        x.it.row0 += r;
        x.it.n = ih < n_heads ? min(x.it.n - r, ROWS) : 0;  // at most 0: no rows
        x.p = x.it.p0 + 2 * wave;
        x.mine = x.it.n > 0 && x.it.p1 > x.p ? (x.it.p1 - x.p + 2 * kTreeWaves - 1) / (2 * kTreeWaves) : 0;
        return x;
    };
    // lane l: the id of page l % 2 of pair l / 2 from page `from` on
    auto page_ids = [&](const Work& x, int from) {
        const int pg = from + (lane >> 1) * (2 * kTreeWaves) + (lane & 1);
        return x.mine > 0 && pg < x.it.p1 ? kv.page_table[((size_t)x.it.seq * kv.n_planes + x.it.plane) * kv.max_pages + pg]
                            : -2;  // past the context
    };
    // The wave's pair i: whether its pages are there (bits 0, 1), and where they are.
    // A missing page's loads go to one that exists; what they bring is masked.
    struct Pair {
        int there;
        const char* at[2];
    };
    const size_t page_bytes = (size_t)2 * H * kPage * HD * 2;
    const uint32_t v_at = (uint32_t)H * kPage * HD * 2;
    auto pair_of = [&](const Work& x, int ids, int i) {
        const int p0 = __builtin_amdgcn_readlane(ids, 2 * (i & 31)), p1 = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + 1);
        const bool ok0 = p0 >= 0 && p0 < kv.n_pages, ok1 = p1 >= 0 && p1 < kv.n_pages;
        if (((!ok0 && p0 != -2) || (!ok1 && p1 != -2)) && lane == 0) set_err(err, CDB_DEV_UNMAPPED_PAGE);
        const int q0 = ok0 ? p0 : 0, q1 = ok1 ? p1 : q0;
        const char* pool = reinterpret_cast<const char*>(kv.pool + kv_offset(kv.layer, 0, kv.n_pages, 0, x.head, H, 0, HD));
        return Pair{(ok0 ? 1 : 0) | (ok1 ? 2 : 0), {pool + q0 * page_bytes, pool + q1 * page_bytes}};
    };
    // A pair's K and V, in 16-byte pieces as stored.  Each is read once by one
    // workgroup (past the caches' normal allocation), with halves by two.
    typedef u32x4 PairRegs[2][NJ];
    PairRegs kr, vr;
    const uint32_t lane16 = lane * 16;
    auto fetch = [&](const Pair& x) {
        auto load = [&](const char* page, int j) {  // uniform page + 32-bit lane offset + constant
            const u32x4* a = reinterpret_cast<const u32x4*>(page + (size_t)lane16 + 1024 * j);
            return HALVES ? *a : __builtin_nontemporal_load(a);
        };
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < NJ; ++j) kr[h][j] = load(x.at[h], j);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < NJ; ++j) vr[h][j] = load(x.at[h] + v_at, j);
    };

    // Each item's first pair is on its way before the item before it is written out.
    int work = blockIdx.x;  // the grid has no more workgroups than `items` has room for
    Work x = load_work(work);
    if (work >= n_work) return;
    int ids = page_ids(x, x.p);
    Pair pair{};
    if (x.mine > 0) {
        pair = pair_of(x, ids, 0);
        fetch(pair);
    }
    while (true) {
        const int next = work + gridDim.x;
        int ids2;
        {
            const Work x2 = load_work(next < n_work ? next : work);
            ids2 = page_ids(x2, x2.p);
        }
        const TreeItem& it = x.it;
        const int head = x.head;
        // A segment's record of a row: sums, maximum, weight.  Written through to memory
        // and read past the caches: the workgroups run on XCDs with L2s of their own.
        auto rec = [&](int row, int sg) {
            return ts.part + (((size_t)row * H + head) * kTreeSegs + sg) * REC;
        };
        auto put2 = [](float* at, float a, float b) {
            __hip_atomic_store(reinterpret_cast<uint64_t*>(at), (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a),
                               __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        };
        auto get2 = [](const float* at, float& a, float& b) {
            const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(at), __ATOMIC_RELAXED,
                                                 __HIP_MEMORY_SCOPE_AGENT);
            a = __uint_as_float((uint32_t)v);
            b = __uint_as_float((uint32_t)(v >> 32));
        };
        auto finish = [&](int row, int k, float a, float b, float den) {  // den 0: the row sees nothing
            *reinterpret_cast<uint32_t*>(out + frag_index(row, head * HD + k, d)) =
                den != 0.f ? pack_bf16(a / den, b / den) : 0u;
        };
        // q operands: row c of tile t, dims 32j + 8g .. + 7, scaled, hi + lo.  One tile's
        // stay in each wave's registers; two would cost the loop its second wave per
        // SIMD, so all waves read them from LDS.
        auto q_operand = [&](int t, int j, bf16x8& hi, bf16x8& lo) {
            const int row = it.row0 + min(t * 16 + c, it.n - 1);  // rows past the tile repeat its last one
            const float* src = q + (size_t)row * d + head * HD + 32 * j + 8 * g;
            floatx4 a, b;
            __builtin_memcpy(&a, src, 16);
            __builtin_memcpy(&b, src + 4, 16);
            const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            uint32_t hw[4], lw[4];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float x0 = x[e] * qscale, x1 = x[e + 1] * qscale;
                const uint32_t h = pack_bf16(x0, x1);
                hw[e / 2] = h;
                lw[e / 2] = pack_bf16(x0 - bflo(h), x1 - bfhi(h));
            }
            hi = __builtin_bit_cast(bf16x8, u32x4{hw[0], hw[1], hw[2], hw[3]});
            lo = __builtin_bit_cast(bf16x8, u32x4{lw[0], lw[1], lw[2], lw[3]});
        };
        u32x4* sq = reinterpret_cast<u32x4*>(smem + VBYTES) + lane;
        bf16x8 qr[2][QLDS ? 1 : NJ];  // hi, lo
        if constexpr (QLDS) {
            for (int f = wave; f < NT * NJ && it.n > 0; f += kTreeWaves) {
                bf16x8 hi, lo;
                q_operand(f / NJ, f % NJ, hi, lo);
                sq[f * 128] = __builtin_bit_cast(u32x4, hi);
                sq[f * 128 + 64] = __builtin_bit_cast(u32x4, lo);
            }
        } else {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                if (it.n > 0) q_operand(0, j, qr[0][j], qr[1][j]);
        }
        TreeState<HD, NT> st;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            st.m[t] = -1e30f;
            st.l[t] = 0.f;
#pragma unroll
            for (int b = 0; b < NB; ++b) st.o[t][b] = floatx4{0.f, 0.f, 0.f, 0.f};
        }

        if constexpr (QLDS) __syncthreads();
        int p = x.p;
        for (int i = 0; i < x.mine; ++i, p += 2 * kTreeWaves) {
            const Pair now = pair;
            const int there = now.there;
            const bool masked = there != 3 || p * kPage + 2 * kPage > it.base;  // wave-uniform
            bool odd = false;  // a V that is not finite where only some rows may see it
            if (masked) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        const int off = (p + h) * kPage + (j * 64 + lane) / CPR - it.base;
                        const uint32_t keep = (there >> h & 1) && (sees4(it.seen, off) & 1) ? ~0u : 0u;
                        const uint32_t part = off < 0 ? 0u : ~0u;  // committed positions: every row sees them
                        u32x4 x = vr[h][j] & keep;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t bad = ((x[e] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) |
                                                 ((x[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
                            odd |= (bad & part) != 0;
                            x[e] &= ~(bad & part);
                        }
                        vr[h][j] = x;
                    }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const int f = j * 64 + lane, r = f / CPR, ch = f - r * CPR;
                    *reinterpret_cast<u32x4*>(sk + (h * kPage + r) * KP + ch * 8) = kr[h][j];
                    *reinterpret_cast<u32x4*>(sv + (h * kPage + r) * VP + ch * 8) = vr[h][j];
                }
            const bool more = i + 1 < x.mine;
            if (more) {
                if (((i + 1) & 31) == 0) ids = page_ids(x, p + 2 * kTreeWaves);
                pair = pair_of(x, ids, i + 1);
                fetch(pair);
            }
            // A = K: key c of either page, dims 32j + 8g ..
            bf16x8 ka[2][NJ];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    ka[h][j] = *reinterpret_cast<const bf16x8*>(sk + (h * kPage + c) * KP + 32 * j + 8 * g);
            floatx4 s[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int part = 1; part >= 0; --part) {
                bf16x8 b[NT][NJ];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
                        if constexpr (QLDS)
                            b[t][j] = __builtin_bit_cast(bf16x8, sq[(t * NJ + j) * 128 + part * 64]);
                        else
                            b[t][j] = qr[part][j];
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            s[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[h][j], b[t][j], s[t][h], 0, 0, 0);
            }
            // A = V^T: dim 16b + c, keys 4g..4g+3 of both pages; lane c of group g points at key 4g + c/4, dims 4(c%4)..
            const int vk = 4 * g + (c >> 2);
            bf16x8 va[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint16_t* at = sv + vk * VP + b * 16 + (c & 3) * 4;
                const uint2 w0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                               (__attribute__((address_space(3))) s16x4*)at));
                const uint2 w1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                               (__attribute__((address_space(3))) s16x4*)(at + kPage * VP)));
                va[b] = __builtin_bit_cast(bf16x8, u32x4{w0.x, w0.y, w1.x, w1.y});
            }
            // The maximum that weights are taken against follows the row's own once it has
            // fallen 8 behind (weights stay below 2^8), so most pairs rescale nothing.
            bf16x8 ph[NT], pl[NT];
            bool up[NT], any_up = false;
            float mx[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (masked) {
                    const uint64_t mask = tree.mask[it.row0 + min(t * 16 + c, it.n - 1)];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t see = sees4(mask, (p + h) * kPage + 4 * g - it.base) & (there >> h & 1 ? 15u : 0u);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[t][h][e] = see >> e & 1 ? s[t][h][e] : -INFINITY;
                    }
                }
                mx[t] = fmaxf(s[t][0][0], s[t][0][1]);
#pragma unroll
                for (int e = 2; e < 8; ++e) mx[t] = fmaxf(mx[t], s[t][e >> 2][e & 3]);
                mx[t] = over_rows_max(mx[t]);
                up[t] = mx[t] > st.m[t] + 8.f;
                any_up |= up[t];
            }
            if (__any(any_up)) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const float m = up[t] ? mx[t] : st.m[t];
                    const float corr = up[t] ? exp2_raw(st.m[t] - m) : 1.f;
                    st.l[t] *= corr;
#pragma unroll
                    for (int b = 0; b < NB; ++b) st.o[t][b] *= corr;
                    st.m[t] = m;
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                uint32_t hw[4], lw[4];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float p0 = exp2_raw(s[t][e >> 2][e & 3] - st.m[t]);
                    const float p1 = exp2_raw(s[t][e >> 2][(e & 3) + 1] - st.m[t]);
                    st.l[t] += p0 + p1;
                    const uint32_t hi = pack_bf16(p0, p1);
                    hw[e / 2] = hi;
                    lw[e / 2] = pack_bf16(p0 - bflo(hi), p1 - bfhi(hi));
                }
                ph[t] = __builtin_bit_cast(bf16x8, u32x4{hw[0], hw[1], hw[2], hw[3]});
                pl[t] = __builtin_bit_cast(bf16x8, u32x4{lw[0], lw[1], lw[2], lw[3]});
            }
#pragma unroll
            for (int part = 1; part >= 0; --part)
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        st.o[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[b], part ? pl[t] : ph[t], st.o[t][b], 0, 0,
                                                                             0);
            if (masked && __any(odd)) {  // rare: the values taken out above, to the rows that see them
                for (int kk = 0; kk < 2 * kPage; ++kk) {
                    const int off = p * kPage + kk - it.base;
                    if (off < 0 || off >= 64 || !(it.seen >> off & 1) || !(there >> (kk >> 4) & 1)) continue;
                    const uint16_t* row =
                        reinterpret_cast<const uint16_t*>((kk < kPage ? now.at[0] : now.at[1]) + v_at) + (kk & 15) * HD;
                    const int w = (kk >> 4) * 2 + ((kk & 3) >> 1);  // p of key kk: word w, half kk % 2, of lane group kk % 16 / 4
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const u32x4 h4 = __builtin_bit_cast(u32x4, ph[t]), l4 = __builtin_bit_cast(u32x4, pl[t]);
                        uint32_t hw = 0, lw = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (e == w) {
                                hw = h4[e];
                                lw = l4[e];
                            }
                        const int from = c + 16 * ((kk & 15) >> 2);
                        hw = __shfl(hw, from, 64);
                        lw = __shfl(lw, from, 64);
                        const float pk = kk & 1 ? bfhi(hw) + bfhi(lw) : bflo(hw) + bflo(lw);
                        const bool see = tree.mask[it.row0 + min(t * 16 + c, it.n - 1)] >> off & 1;
#pragma unroll
                        for (int b = 0; b < NB; ++b)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t x = row[16 * b + 4 * g + e];
                                const float o = st.o[t][b][e];
                                st.o[t][b][e] = see && (x & 0x7f80u) == 0x7f80u ? fmaf(pk, bf2f((uint16_t)x), o) : o;
                            }
                    }
                }
            }
        }
        const Work x2 = load_work(next < n_work ? next : work);  // again: kept, it would crowd the loop's scalars
        if (next < n_work && x2.mine > 0) {
            pair = pair_of(x2, ids2, 0);
            fetch(pair);
        }

        // the waves' states: [page class][row][dim]
        __syncthreads();  // every wave is done with its V and q
        float* so = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float l = over_rows_sum(st.l[t]);
#pragma unroll
            for (int b = 0; b < NB; ++b)
                *reinterpret_cast<floatx4*>(so + (wave * ROWS + t * 16 + c) * PITCH + 16 * b + 4 * g) = st.o[t][b];
            if (g == 0) {
                sf.m[wave][t * 16 + c] = st.m[t];
                sf.l[wave][t * 16 + c] = l;
            }
        }
        __syncthreads();
        // row factors: waves of this segment
        if (tid < it.n) {
            float mx = sf.m[0][tid], den = 0.f;
#pragma unroll
            for (int w = 1; w < kTreeWaves; ++w) mx = fmaxf(mx, sf.m[w][tid]);
#pragma unroll
            for (int w = 0; w < kTreeWaves; ++w) {
                const float f = exp2_raw(sf.m[w][tid] - mx);
                sf.f[w][tid] = f;
                den = fmaf(f, sf.l[w][tid], den);
            }
            sf.den[tid] = den;
            if (it.nseg > 1) put2(rec(it.row0 + tid, it.seg) + HD, mx, den);
        }
        __syncthreads();
        // thread = two dims of a row, so that a wave's stores are one run
        for (int e = tid; e < it.n * (HD / 2); e += THREADS) {
            const int r = e / (HD / 2), k = 2 * (e - r * (HD / 2));
            float a = 0.f, b = 0.f;
#pragma unroll
            for (int w = 0; w < kTreeWaves; ++w) {
                const float2 o2 = *reinterpret_cast<const float2*>(so + (w * ROWS + r) * PITCH + k);
                a = fmaf(sf.f[w][r], o2.x, a);
                b = fmaf(sf.f[w][r], o2.y, b);
            }
            if (it.nseg == 1)
                finish(it.row0 + r, k, a, b, sf.den[r]);
            else
                put2(rec(it.row0 + r, it.seg) + k, a, b);
        }
        if (it.nseg > 1 && it.n > 0) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the wave's records have reached memory
            __syncthreads();
            if (tid == 0) {
                int* a = ts.arrive + it.row0 * H + head;
                s_last = __hip_atomic_fetch_add(a, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == it.nseg - 1;
                if (s_last) __hip_atomic_store(a, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (s_last) {
                if (tid < it.n) {
                    float sm[kTreeSegs], sl[kTreeSegs], mx = -1e30f, den = 0.f;
#pragma unroll
                    for (int sg = 0; sg < kTreeSegs; ++sg)  // past the last: the last again, with weight 0
                        get2(rec(it.row0 + tid, min(sg, it.nseg - 1)) + HD, sm[sg], sl[sg]);
#pragma unroll
                    for (int sg = 0; sg < kTreeSegs; ++sg) mx = fmaxf(mx, sm[sg]);
#pragma unroll
                    for (int sg = 0; sg < kTreeSegs; ++sg) {
                        const float f = exp2_raw(sm[sg] - mx);
                        sf.seg[sg][tid] = f;
                        den = sg < it.nseg ? fmaf(f, sl[sg], den) : den;
                    }
                    sf.den[tid] = den;
                }
                __syncthreads();
                for (int e = tid; e < it.n * (HD / 2); e += THREADS) {
                    const int r = e / (HD / 2), k = 2 * (e - r * (HD / 2));
                    const float* at = rec(it.row0 + r, 0) + k;
                    float a = 0.f, b = 0.f;
                    for (int s0 = 0; s0 < it.nseg; s0 += 8) {
                        float x[8], y[8];
#pragma unroll
                        for (int u = 0; u < 8; ++u) get2(at + min(s0 + u, it.nseg - 1) * REC, x[u], y[u]);
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            const bool in = s0 + u < it.nseg;
                            const float f = sf.seg[min(s0 + u, it.nseg - 1)][r];
                            a = in ? fmaf(f, x[u], a) : a;
                            b = in ? fmaf(f, y[u], b) : b;
                        }
                    }
                    finish(it.row0 + r, k, a, b, sf.den[r]);
                }
            }
        }
        if (next >= n_work) break;
        x = x2;
        ids = ids2;
        work = next;
        __syncthreads();  // the next item's V takes the place of the states
    }
}

// rows per tile
static int tree_rows_per_tile(int max_nodes) { return max_nodes <= 16 ? 16 : max_nodes <= 32 ? 32 : 64; }

hipError_t launch_tree_plan(const KvTarget& kv, const int32_t* seq, const cdb_tree& tree, int M, int H, int hd,
                            void* scratch, int* err, hipStream_t st, const int32_t* dn) {
    if (M <= 0) return hipSuccess;
    if (M > kMaxRows) return hipErrorInvalidValue;
    k_tree_plan<<<1, 256, 0, st>>>(kv, seq, tree, M, H, tree_rows_per_tile(tree.max_nodes),
                                   tree_scratch(scratch, H, hd, M), err, dn);
    return hipGetLastError();
}

template <int HD>
static void run_tree_attn(int rows, int most, const float* q, const KvTarget& kv, const cdb_tree& tree, int H,
                          const TreeScratch& ts, uint16_t* out, int* err, hipStream_t st) {
    // one resident workgroup of 8 waves per CU
    if (rows == 16)
        k_tree_attn<HD, 1, false><<<std::min(most, 256), kTreeWaves * 64, 0, st>>>(q, kv, tree, H, ts, out, err);
    else if (rows == 32)
        k_tree_attn<HD, 2, false><<<std::min(most, 256), kTreeWaves * 64, 0, st>>>(q, kv, tree, H, ts, out, err);
    else  // most <= items x heads; whole groups of 16
        k_tree_attn<HD, 2, true><<<std::min((most + 7) / 8 * 16, 256), kTreeWaves * 64, 0, st>>>(q, kv, tree, H, ts, out,
                                                                                                  err);
}

hipError_t launch_tree_attention(const float* q, const KvTarget& kv, const cdb_tree& tree, int M, int H, int hd,
                                 void* scratch, uint16_t* out, int* err, hipStream_t st) {
    if (M <= 0) return hipSuccess;
    const TreeScratch ts = tree_scratch(scratch, H, hd, M);
    const int rows = tree_rows_per_tile(tree.max_nodes);
    // no more workgroups than there can be items
    const int segs = std::min(kTreeSegs, kv.max_pages / kTreeSegPages + 1);
    const int most = M * H * segs;
    switch (hd) {
        case 64: run_tree_attn<64>(rows, most, q, kv, tree, H, ts, out, err, st); break;
        case 96: run_tree_attn<96>(rows, most, q, kv, tree, H, ts, out, err, st); break;
        case 128: run_tree_attn<128>(rows, most, q, kv, tree, H, ts, out, err, st); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace cdb
