// Attention of drafted token trees over the paged, depth-indexed KV cache: row i
// attends to positions 0..base-1 of its sequence and to the positions base + j
// whose bit j of its mask is set (its ancestors and itself), in its own plane.
//
// The rows of one tree share their context, so its K and V are read once for up
// to 64 of them and multiplied on MFMA (v_mfma_f32_16x16x32_bf16); with so few
// rows per byte large calls are bound by HBM (64 trees of 4 over 2048..4223
// positions, 16 x 128 heads: 1.63 GB in 261-277 us, 5.9-6.2 TB/s), wide trees by the
// instructions of two waves per SIMD (4 trees of 32-64 over 1024..2047, 55 x 96
// heads: 150 MB in 50-55 us) and small calls by latency (13 rows over 700: 12.2 us).
//
// Tiles: adjacent rows of one sequence, plane and base, at most 16, 32 or 64 of
// them (by cdb_tree.max_nodes).  A row's context is cut into segments
// (tree_segments, by its base alone).  Every wave works out all tiles itself at its
// start, which costs less than a launch that would do it once, or than barriers
// between waves that share it (12.4 us against 13.2, 13 rows over 700 positions;
// 256 rows lose a little: 20.0 against 19.5, 16 trees of 16 over 640).
//
// k_tree_attn: a workgroup takes works in turn: the segments of one tile and head,
// or, when that leaves CUs idle, a run of them.  Its 8 waves deal a segment's
// pages among them in pairs (32 keys), and each keeps an online softmax of its own
// for the tile's rows.  Per pair:
//   K and V come in whole lines into registers, a pair ahead, and go to LDS.
//   (Loads of K as operands, 64 bytes of a row at a time, kept a CU at half the
//   rate: 58 GB/s against 113.)
//   S^T = K Q^T: A = K (lane = key), B = q, split into bf16 hi + lo parts (about
//     16 bits of it).  A lane then holds one row's scores at 4 keys of either page.
//   online softmax per row in the exp2 domain; the running maximum goes over the
//     four lanes of a row (two lane swaps), the sum stays apart until the end.
//   O^T += V^T P^T: B = P, hi + lo again, and already where the scores left it:
//     the order of the 32 keys in the product is free, so lane group g takes keys
//     4g..4g+3 of both pages.  A = V^T, read from the key-major rows in LDS with
//     the transposing read (ds_read_b64_tr_b16).
// At a segment's end the waves' states are merged through LDS and folded into the
// row's total, in segment order: in registers, or, where the segments of a tile
// are spread over workgroups, from their records by k_tree_merge, with the same
// operations.
//
// 64-row tiles go to two workgroups of 32 rows that run on one XCD at one time:
// four 16-row tiles in one wave's registers left one wave per SIMD (77 us against
// 45 when that was measured, 4 trees of 64 over 1500 positions, 55 x 96 heads).
//
// Masks: only pages that reach past base take the masked path.  There a score that
// a row does not see becomes -inf (p = 0), and V of keys that no row of the tile
// sees is cleared; a V that is not finite at a key that some rows see is taken out
// of the product, which would multiply it by the others' zeros, and added to those
// rows alone.
//
// A row whose sums end as no number, or whose weights are all 0, is worked out again in
// plain fp32 (attend_plain), for the dims that are no number; looking for that takes 0
// to 0.4 us of a call.
//
// Nothing in a row's arithmetic depends on the other rows: not its tile, not the
// segments, not the wave that takes a page or the workgroup that takes a segment.
#include <algorithm>

#include "cdb_internal.h"

namespace cdb {

constexpr int kTreeWaves = 8;
constexpr int kTreeThreads = kTreeWaves * 64;
constexpr int kTreeSegs = 16;      // most segments of a context
constexpr int kTreeSegPages = 64;  // pages of a segment, unless that makes too many
constexpr int kTreeRows = 32;      // most rows of a workgroup
constexpr int kTreeCUs = 256;

// Segments of a context whose last committed position is on page npg - 1, and the
// pages of each (the last one has the rest); a multiple of the waves' pairs.
__host__ __device__ __forceinline__ int tree_segments(int npg, int* pages) {
    if (npg <= kTreeSegs * kTreeSegPages) {
        *pages = kTreeSegPages;
        return (npg + kTreeSegPages - 1) / kTreeSegPages;
    }
    constexpr int round = 2 * kTreeWaves;
    *pages = (npg + kTreeSegs * round - 1) / (kTreeSegs * round) * round;
    return (npg + *pages - 1) / *pages;
}

// Works that a tile and head is split into when there are n (tile, head, half)
// triples: as many as fit the CUs in one round.  Of the tiles, at least as many
// count as all rows of a call without a device row count make: whether the host
// launches k_tree_merge is decided by those, and rows that are skipped must not
// leave segments in records that nobody joins.
__host__ __device__ __forceinline__ int tree_runs(int n) {
    const int z = n > 0 ? kTreeCUs / n : 1;
    return z < 1 ? 1 : z > kTreeSegs ? kTreeSegs : z;
}

// Scratch of the segments' records: sums, maximum, weight.
struct TreeScratch {
    int* runs;    // tree_runs of the launch, for k_tree_merge
    float* part;  // [rows][H][kTreeSegs][hd + 2]
    size_t bytes;
};
static TreeScratch tree_scratch(void* at, int H, int hd, int rows) {
    unsigned char* p = static_cast<unsigned char*>(at);
    TreeScratch t{};
    t.runs = reinterpret_cast<int*>(p);
    t.part = reinterpret_cast<float*>(p + 256);
    t.bytes = 256 + (((size_t)rows * H * kTreeSegs * (hd + 2) * 4 + 255) & ~(size_t)255);
    return t;
}
size_t tree_scratch_bytes(const cdb_model_desc& d, int rows) {
    return rows > 0 ? tree_scratch(nullptr, d.n_heads, d.head_dim, rows).bytes : 0;
}

// What a row attends to, and whether that is in range.
struct RowSees {
    int seq, plane, base;
    uint64_t mask;
    bool ok;
};
__device__ __forceinline__ RowSees row_sees(const KvTarget& kv, const int32_t* seq, const cdb_tree& tree, int i) {
    RowSees r;
    r.seq = seq[i];
    r.base = tree.base[i];
    r.mask = tree.mask[i];
    r.plane = kv.c_row ? kv.c_row[i] + 1 : kv.plane_fixed;
    const int limit = kv.max_pages * kPage;
    r.ok = r.seq >= 0 && r.seq < kv.max_seqs && r.base >= 0 && r.base <= limit &&
           (kv.c_row ? r.plane >= 1 && r.plane <= kv.n_planes - 2 : r.plane >= 0 && r.plane < kv.n_planes);
    r.ok = r.ok && (!r.mask || r.base + 63 - __clzll((long long)r.mask) < limit);
    return r;
}

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

// Over groups of 8 lanes (quad swaps and a mirror of half a row); every lane gets it.
#define CDB_TREE_DPP(v, ctrl) \
    __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, (v)), (ctrl), 0xF, 0xF, true))
__device__ __forceinline__ float over_8_max(float v) {
    v = fmaxf(v, CDB_TREE_DPP(v, 0xB1));
    v = fmaxf(v, CDB_TREE_DPP(v, 0x4E));
    return fmaxf(v, CDB_TREE_DPP(v, 0x141));
}
__device__ __forceinline__ float over_8_sum(float v) {
    v += CDB_TREE_DPP(v, 0xB1);
    v += CDB_TREE_DPP(v, 0x4E);
    return v + CDB_TREE_DPP(v, 0x141);
}
// The lane before's value (lane 0: 0).
__device__ __forceinline__ int lane_before(int v) { return __builtin_amdgcn_update_dpp(0, v, 0x138, 0xF, 0xF, false); }
// Inclusive prefix sum: within 16 lanes, then lane 15 of each into the next 16, lane 31 into the upper half.
__device__ __forceinline__ int scan64(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
    return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
}
// Over the wave: quads, halves of 16, 16, 32, 64 lanes.
__device__ __forceinline__ uint64_t over_wave_or(uint64_t v) {
    uint32_t w[2] = {(uint32_t)v, (uint32_t)(v >> 32)};
#pragma unroll
    for (uint32_t& x : w) {
        x |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true);
        x |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true);
        x |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true);
        x |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, true);
        auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = r[0] | r[1];
        r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = __builtin_amdgcn_readfirstlane(r[0] | r[1]);
    }
    return (uint64_t)w[1] << 32 | w[0];
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
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
// (8 for V where LDS is full: two rows to a bank.)
template <int HD>
constexpr int kKPitch = HD + 8;
template <int HD, int NT>
constexpr int kVPitch = HD == 128 && NT == 2 ? HD + 8 : HD + 16;

struct Work {
    uint64_t seen;       // mask bits of any row of the tile
    int row0, n;         // the workgroup's rows; n 0: none
    int seq, plane, base, head;
    int sg0, sg1, nseg;  // the work's segments, those of the context
    int sp, npg;         // pages of a segment, of the context and the tree
    // from here on by wave: its first page, and how many pairs of pages it has
    int p, mine;
    __device__ __forceinline__ void by_wave(int wave) {
        p = sg0 * sp + 2 * wave;
        const int pe = sg1 == nseg ? npg : sg1 * sp;
        // at least one pair, of pages that are not there if need be: every work is fetched alike
        mine = pe > p ? (pe - p + 2 * kTreeWaves - 1) / (2 * kTreeWaves) : 1;
    }
};
constexpr int kWorkInts = 13;  // of Work, without the last two

template <int HD, int NT>
struct TreeState {
    floatx4 o[NT][HD / 16];
    float m[NT], l[NT];  // l: this lane's keys only
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            m[t] = -1e30f;
            l[t] = 0.f;
#pragma unroll
            for (int b = 0; b < HD / 16; ++b) o[t][b] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
    }
};

// The running total of a row: (m, l) and factors of the total so far and of the
// segment that joins it.  Used wherever segments are joined.
__device__ __forceinline__ void join_segment(float& tm, float& tl, float sm, float sl, float& a, float& b) {
    const float mx = fmaxf(tm, sm);
    a = exp2_raw(tm - mx);
    b = exp2_raw(sm - mx);
    tl = fmaf(tl, a, sl * b);
    tm = mx;
}
__device__ __forceinline__ float join_sum(float t, float s, float a, float b) { return fmaf(t, a, s * b); }

// One row and head in plain fp32, by one wave: lane = key for the scores, then two
// dims.  Three turns over the context (maximum, sum, weights already divided by it), as
// only rows take it whose sums in the products above are not to be had: an infinite K
// or V times the low part of q or p is not what it is times the whole, and sums of
// values that are themselves near the largest number overflow.  64 trees of 4 over
// 2048..4223 positions with every V infinite take 4.1 ms (261-277 us otherwise).
template <int HD>
__device__ __forceinline__ float2 attend_plain(const float* q, const KvTarget& kv, int seq, int plane, int base,
                                               uint64_t mask, int head, int H) {
    const int lane = threadIdx.x & 63, dim = 2 * min(lane, HD / 2 - 1);
    const int n = mask ? base + 64 - __clzll((long long)mask) : base;
    const int32_t* ids = kv.page_table + ((size_t)seq * kv.n_planes + plane) * kv.max_pages;
    const float qscale = 1.4426950408889634f / sqrtf((float)HD);
    float m = -INFINITY, l = 0.f, oa = 0.f, ob = 0.f;
    bool any = false;
#pragma unroll 1
    for (int turn = 0; turn < 3; ++turn) {
#pragma unroll 1
        for (int k0 = 0; k0 < n; k0 += 64) {
            const int key = k0 + lane, off = key - base;
            bool see = key < n && (off < 0 || (mask >> (off & 63) & 1));
            const int id = see ? ids[key / kPage] : -1;
            see = id >= 0 && id < kv.n_pages;
            const uint16_t* k = kv.pool + kv_offset(kv.layer, see ? id : 0, kv.n_pages, 0, head, H, key % kPage, HD);
            float s = 0.f;
#pragma unroll 2
            for (int j = 0; j < HD; j += 8) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(k + j);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s = fmaf(q[j + 2 * e], bflo(w[e]), s);
                    s = fmaf(q[j + 2 * e + 1], bfhi(w[e]), s);
                }
            }
            s *= qscale;
            if (turn == 0) {
                m = see ? fmaxf(m, s) : m;
                any |= see;
                continue;
            }
            float p = see ? exp2f(s - m) : 0.f;
            if (turn == 1) {
                l += p;
                continue;
            }
            p /= l;
            const uint64_t seen = __ballot(see);
#pragma unroll 1
            for (int u0 = 0; u0 < 64; u0 += 8) {
                uint32_t v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int at = __builtin_amdgcn_readlane(see ? id : 0, u0 + u);
                    v[u] = *reinterpret_cast<const uint32_t*>(
                        kv.pool + kv_offset(kv.layer, at, kv.n_pages, 1, head, H, (k0 + u0 + u) % kPage, HD) + dim);
                }
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (seen >> (u0 + u) & 1) {
                        const float pu = lane_value(p, u0 + u);
                        oa = fmaf(pu, bflo(v[u]), oa);
                        ob = fmaf(pu, bfhi(v[u]), ob);
                    }
            }
        }
        if (!__any(any)) break;
#pragma unroll 1
        for (int o = 1; o < 64 && turn < 2; o <<= 1) {
            const float x = __shfl_xor(turn ? l : m, o, 64);
            if (turn)
                l += x;
            else
                m = fmaxf(m, x);
        }
    }
    return make_float2(oa, ob);
}

// A row's values (a lane's two dims: sums over the sum of the weights) that are no
// numbers, because of the products or because all weights are 0, become what
// attend_plain finds; a row that sees nothing gets 0 from there.
__device__ __forceinline__ bool row_odd(float a, float b) { return !__builtin_isfinite(a) || !__builtin_isfinite(b); }
template <int HD>
__device__ __forceinline__ uint32_t row_plain(float a, float b, const float* q, const KvTarget& kv, int seq, int plane,
                                              int base, uint64_t mask, int head, int H) {
    const float2 v = attend_plain<HD>(q, kv, seq, plane, base, mask, head, H);
    return pack_bf16(__builtin_isfinite(a) ? a : v.x, __builtin_isfinite(b) ? b : v.y);
}

template <int HD, int NT, bool HALVES>
__global__ __launch_bounds__(kTreeThreads) void k_tree_attn(const float* __restrict__ q, KvTarget kv,
                                                            const int32_t* __restrict__ seq, cdb_tree tree, int M, int H,
                                                            TreeScratch ts, uint16_t* __restrict__ out, int* err,
                                                            const int32_t* __restrict__ dn, int least_tiles) {
    constexpr int NJ = HD / 32, NB = HD / 16, CPR = HD / 8;  // K steps, dim blocks, 16-byte pieces of a row
    constexpr int ROWS = 16 * NT, CAP = HALVES ? 2 * kTreeRows : ROWS;  // rows of a workgroup, of a tile
    constexpr int PITCH = HD + 4, REC = HD + 2;
    constexpr int NR = ROWS / kTreeWaves;  // rows whose totals a wave keeps: wave, wave + 8, ...; lane = two dims
    // K and V of the waves' pairs, then q operands.  At a segment's end the waves' states
    // and factors take the place of K and V.
    constexpr int KP = kKPitch<HD>, VP = kVPitch<HD, NT>, KROWS = 2 * kPage;
    constexpr int VBYTES = kTreeWaves * KROWS * (KP + VP) * 2, QBYTES = NT * NJ * 2 * 1024;
    constexpr int OBYTES = kTreeWaves * ROWS * PITCH * 4;
    struct States {  // the waves' maxima and weights
        float m[ROWS][kTreeWaves], l[ROWS][kTreeWaves];
    };
    static_assert(OBYTES + sizeof(States) <= VBYTES, "they leave q alone");
    __shared__ __align__(16) unsigned char smem[VBYTES + QBYTES];
    __shared__ uint8_t s_row[kMaxRows], s_plane[kMaxRows];  // by tile: its first row, its rows' plane,
    __shared__ int s_seq[kMaxRows], s_base[kMaxRows];       // sequence and base,
    __shared__ uint16_t s_before[kMaxRows];                 // and the works before it, if some tile has several
    __shared__ uint64_t s_mask[kMaxRows];                   // by row
    __shared__ uint64_t s_ends[kMaxRows / 64 + 2];          // bit: a row that starts a tile or has none
    __shared__ Work s_next[3];
    States& sf = *reinterpret_cast<States*>(smem + OBYTES);
    float* so = reinterpret_cast<float*>(smem);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int d = H * HD;
    const float qscale = 1.4426950408889634f / sqrtf((float)HD);

    // ---- tiles.  Every wave works them out by itself (lane = row of each 64), and all
    // leave the same values in LDS: no wave waits for another.
    int n_tiles = 0, runs, n_works = 0;
    {
        constexpr int WORDS = kMaxRows / 64;
        const int live = live_rows(dn, M);
        RowSees r[WORDS];
#pragma unroll
        for (int k = 0; k < WORDS; ++k)
            if (64 * k < M) r[k] = row_sees(kv, seq, tree, min(64 * k + lane, M - 1));
        int start = 0;  // the row at which the last run before these 64 started
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            uint64_t ends = ~0ull;
            if (64 * k < M) {
                const int row = 64 * k + lane;
                const bool ok = row < live && r[k].ok;
                if (row < live && !ok && wave == 0 && blockIdx.x == 0) set_err(err, CDB_DEV_UNMAPPED_PAGE);
                if (!ok) r[k].seq = -1;
                s_mask[row] = r[k].mask;
                int pseq = lane_before(r[k].seq), pplane = lane_before(r[k].plane), pbase = lane_before(r[k].base);
                if (k > 0) {
                    const RowSees& last = r[k > 0 ? k - 1 : 0];
                    pseq = lane > 0 ? pseq : __builtin_amdgcn_readlane(last.seq, 63);
                    pplane = lane > 0 ? pplane : __builtin_amdgcn_readlane(last.plane, 63);
                    pbase = lane > 0 ? pbase : __builtin_amdgcn_readlane(last.base, 63);
                }
                const uint64_t run =
                    __ballot(ok && !(row > 0 && pseq == r[k].seq && pplane == r[k].plane && pbase == r[k].base));
                const uint64_t b = run & (~0ull >> (63 - lane));
                const bool first = ok && (row - (b ? 64 * k + 63 - __clzll((long long)b) : start)) % CAP == 0;
                const uint64_t firsts = __ballot(first);
                ends = __ballot(first || !ok);
                if (run) start = 64 * k + 63 - __clzll((long long)run);
                if (first) {
                    const int tile = n_tiles + __builtin_amdgcn_mbcnt_hi((uint32_t)(firsts >> 32),
                                                                         __builtin_amdgcn_mbcnt_lo((uint32_t)firsts, 0));
                    s_row[tile] = (uint8_t)row;
                    s_seq[tile] = r[k].seq;
                    s_base[tile] = r[k].base;
                    s_plane[tile] = (uint8_t)r[k].plane;  // at most r_max + 1 <= 65
                }
                n_tiles += __popcll(firsts);
            }
            s_ends[k] = ends;
        }
        s_ends[WORDS] = s_ends[WORDS + 1] = ~0ull;
        runs = tree_runs(max(n_tiles, least_tiles) * H * (HALVES ? 2 : 1));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // what lanes have written, others read
        n_works = n_tiles;
        if (runs > 1) {
            n_works = 0;
            for (int t = 0; t < n_tiles; t += 64) {
                int sp;
                const int works =
                    t + lane < n_tiles ? min(runs, tree_segments(s_base[min(t + lane, kMaxRows - 1)] / kPage + 1, &sp)) : 0;
                const int at = scan64(works);
                if (t + lane < n_tiles) s_before[t + lane] = (uint16_t)(n_works + at - works);
                n_works += __builtin_amdgcn_readlane(at, 63);
            }
        }
        if (tid == 0 && blockIdx.x == 0) *ts.runs = runs;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // what lanes have written, others read
    }

    // Work w: with halves, workgroups 8 apart, which run on one XCD at one time, take
    // the halves of a tile's rows, so that the second one's K and V come from that
    // XCD's L2.
    const int n_heads = n_works * H;  // works x heads
    const int n_all = !HALVES ? n_heads : (n_heads + 7) / 8 * 16;
    auto load_work = [&](int w) {
        const int wh = !HALVES ? w : w / 16 * 8 + w % 8, r = !HALVES ? 0 : w / 8 % 2 * kTreeRows;
        Work x{};
        if (wh >= n_heads) {  // no rows: one pair of pages that are not there
            x.sg1 = x.nseg = 1;
            x.by_wave(wave);
            return x;
        }
        const int item = wh / H;
        x.head = wh - item * H;
        int tile = item, run = 0;
        if (runs > 1) {  // the last tile whose works start at or before `item`
            tile = -1;
            for (int k = 0; k < n_tiles; k += 64)
                tile += __popcll(__ballot(k + lane < n_tiles && s_before[min(k + lane, kMaxRows - 1)] <= item));
            run = item - s_before[tile];
        }
        const int tile0 = __builtin_amdgcn_readfirstlane((int)s_row[tile]), from = tile0 + 1;
        uint64_t ends = s_ends[from >> 6] >> (from & 63);
        if (from & 63) ends |= s_ends[(from >> 6) + 1] << (64 - (from & 63));
        const int rows = ends ? __ffsll((unsigned long long)ends) : 64;
        x.seq = __builtin_amdgcn_readfirstlane(s_seq[tile]);
        x.base = __builtin_amdgcn_readfirstlane(s_base[tile]);
        x.plane = __builtin_amdgcn_readfirstlane((int)s_plane[tile]);
        x.seen = over_wave_or(lane < rows ? s_mask[min(tile0 + lane, kMaxRows - 1)] : 0);
        x.nseg = tree_segments(x.base / kPage + 1, &x.sp);
        const int z = min(runs, x.nseg);
        if (z == x.nseg) {
            x.sg0 = run;
            x.sg1 = run + 1;
        } else {
            x.sg0 = run * x.nseg / z;
            x.sg1 = (run + 1) * x.nseg / z;
        }
        const int last = x.seen ? x.base + 63 - __clzll((long long)x.seen) : x.base - 1;
        x.npg = last < 0 ? 0 : last / kPage + 1;
        x.n = max(min(rows - r, ROWS), 0);
        x.row0 = x.n > 0 ? tile0 + r : tile0;
        // divisions leave these in vector registers
        for (int* f : {&x.head, &x.nseg, &x.sp, &x.sg0, &x.sg1, &x.npg, &x.row0, &x.n})
            *f = __builtin_amdgcn_readfirstlane(*f);
        x.by_wave(wave);
        return x;
    };
    // Wave 0 works a work out two turns ahead and leaves it in LDS.
    auto put_work = [&](int slot, int w) {
        if (wave != 0 || w >= n_all) return;
        const Work x = load_work(w);
        if (lane == 0) s_next[slot] = x;
    };
    auto get_work = [&](int slot) {
        int f[kWorkInts];
        __builtin_memcpy(f, &s_next[slot], sizeof f);
#pragma unroll
        for (int k = 0; k < kWorkInts; ++k) f[k] = __builtin_amdgcn_readfirstlane(f[k]);
        Work x;
        __builtin_memcpy(&x, f, sizeof f);
        x.by_wave(wave);
        return x;
    };
    // lane l: the id of page l % 2 of pair l / 2 from page `from` on; -2: past the context
    auto page_ids = [&](const Work& x, int from) {
        const int pg = from + (lane >> 1) * (2 * kTreeWaves) + (lane & 1);
        return x.n > 0 && pg < x.npg ? kv.page_table[((size_t)x.seq * kv.n_planes + x.plane) * kv.max_pages + pg] : -2;
    };
    // The wave's pair i: whether its pages are there (bits 0, 1), and where they are.
    // A missing page's loads go to one that exists; what they bring is masked.
    struct Pair {
        int there;
        const char* at[2];
    };
    const uint32_t v_at = (uint32_t)H * kPage * HD * 2, page_bytes = 2 * v_at;
    const char* pool = reinterpret_cast<const char*>(kv.pool + kv_offset(kv.layer, 0, kv.n_pages, 0, 0, H, 0, HD));
    auto pair_of = [&](int head, int ids, int i) {
        const int p0 = __builtin_amdgcn_readlane(ids, 2 * (i & 31)), p1 = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + 1);
        const bool ok0 = p0 >= 0 && p0 < kv.n_pages, ok1 = p1 >= 0 && p1 < kv.n_pages;
        if (((!ok0 && p0 != -2) || (!ok1 && p1 != -2)) && lane == 0) set_err(err, CDB_DEV_UNMAPPED_PAGE);
        const int q0 = ok0 ? p0 : 0, q1 = ok1 ? p1 : q0;
        const char* of_head = pool + (uint32_t)head * (kPage * HD * 2);
        return Pair{(ok0 ? 1 : 0) | (ok1 ? 2 : 0),
                    {of_head + (uint64_t)(uint32_t)q0 * page_bytes, of_head + (uint64_t)(uint32_t)q1 * page_bytes}};
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
    uint16_t* sk = reinterpret_cast<uint16_t*>(smem) + wave * KROWS * (KP + VP);
    uint16_t* sv = sk + KROWS * KP;

    // q: operand f = wave (dims 32j + 8g .. + 7 of row c of 16-row tile t, f = t NJ + j),
    // as loaded, then scaled, split into hi + lo, in LDS for all waves: in registers two
    // tiles of them would not leave room for a second wave per SIMD.
    static_assert(NT * NJ <= kTreeWaves, "one operand a wave");
    floatx4 qraw[2];
    auto fetch_q = [&](const Work& x) {
        if (wave >= NT * NJ || x.n <= 0) return;
        const int row = x.row0 + min(wave / NJ * 16 + c, x.n - 1);  // rows past the tile repeat its last one
        const float* src = q + (size_t)row * d + x.head * HD + 32 * (wave % NJ) + 8 * g;
        __builtin_memcpy(&qraw[0], src, 16);
        __builtin_memcpy(&qraw[1], src + 4, 16);
    };
    u32x4* sq = reinterpret_cast<u32x4*>(smem + VBYTES) + lane;
    auto stage_q = [&] {
        if (wave >= NT * NJ) return;
        const float v[8] = {qraw[0][0], qraw[0][1], qraw[0][2], qraw[0][3], qraw[1][0], qraw[1][1], qraw[1][2], qraw[1][3]};
        uint32_t hw[4], lw[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float v0 = v[e] * qscale, v1 = v[e + 1] * qscale;
            const uint32_t h = pack_bf16(v0, v1);
            hw[e / 2] = h;
            lw[e / 2] = pack_bf16(v0 - bflo(h), v1 - bfhi(h));
        }
        sq[wave * 128] = u32x4{hw[0], hw[1], hw[2], hw[3]};
        sq[wave * 128 + 64] = u32x4{lw[0], lw[1], lw[2], lw[3]};
    };

    // Each work's first pair and q are on their way before the work before it is written out.
    int work = blockIdx.x;
    if (work >= n_all) return;
    Work x = load_work(work);
    int ids = page_ids(x, x.p);
    qraw[0] = qraw[1] = floatx4{0.f, 0.f, 0.f, 0.f};
    fetch_q(x);
    Pair pair = pair_of(x.head, ids, 0);
    if (pair.there) fetch(pair);
    put_work(0, work + gridDim.x);
    // Waves w and w + 4 share a SIMD, and the older one wins ties.  Where a workgroup has
    // one work in which both have as many pairs (more than one), the younger goes first:
    // 13 rows over 700 positions 12.0 us against 12.5, one tree of 64 17.6 against 18.3, 16
    // of 16 over 640 20.2 against 20.7; over 620, 11.4 against 11.2.  With fewer pairs than
    // the older one (13 over 500) it took 12.3 against 11.2, with several works (64 of 4
    // over 100) 23.2 against 22.0.
    Work low = x;
    low.by_wave(wave % (kTreeWaves / 2));
    if (wave >= kTreeWaves / 2 && x.mine > 1 && x.mine == low.mine && work + (int)gridDim.x >= n_all)
        __builtin_amdgcn_s_setprio(1);
    stage_q();
    __syncthreads();
    for (int slot = 0;; slot = slot == 2 ? 0 : slot + 1) {
        const int next = work + gridDim.x;
        const int head = x.head;
        // the next work: its first pages and q; the rest of it stays in LDS
        int ids2 = -2;
        int head2 = 0;
        if (next < n_all) {
            const Work x2 = get_work(slot);
            ids2 = page_ids(x2, x2.p);
            fetch_q(x2);
            head2 = x2.head;
            put_work(slot == 2 ? 0 : slot + 1, next + gridDim.x);
        }
        float tot[NR][2], tm = -1e30f, tw = 0.f;  // totals; lanes 8k..: row k's maximum and weight
#pragma unroll
        for (int k = 0; k < NR; ++k) tot[k][0] = tot[k][1] = 0.f;
        TreeState<HD, NT> st;
        st.clear();
        const bool whole = x.sg0 == 0 && x.sg1 == x.nseg;  // else the segments are written as records
        int p = x.p, i = 0;
        for (int sg = x.sg0; sg < x.sg1; ++sg) {
            // pairs up to the segment's end (of the work's last one: all that are left)
            const int pairs = sg == x.sg1 - 1 ? x.mine : (sg + 1 - x.sg0) * (x.sp / (2 * kTreeWaves));
            for (; i < pairs; p += 2 * kTreeWaves, ++i) {
                const Pair now = pair;
                const int there = now.there;
                const bool masked = there && (there != 3 || p * kPage + 2 * kPage > x.base);  // wave-uniform
                uint32_t odd = 0;  // bits 15, 31: a V that is not finite where only some rows may see it
                if (masked) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if ((there >> h & 1) && (p + h + 1) * kPage <= x.base) continue;  // every row sees all of it
#pragma unroll
                        for (int j = 0; j < NJ; ++j) {
                            const int off = (p + h) * kPage + (j * 64 + lane) / CPR - x.base;
                            const uint64_t bit = off < 0 ? 1 : off < 64 ? x.seen >> (off & 63) : 0;
                            vr[h][j] &= (there >> h & 1) && (bit & 1) ? ~0u : 0u;
                            // an exponent of all ones carries into its half's top bit
                            uint32_t o = 0;
#pragma unroll
                            for (int e = 0; e < 4; ++e) o |= (vr[h][j][e] & 0x7f807f80u) + 0x00800080u;
                            odd |= off < 0 ? 0 : o;
                        }
                    }
                    odd = __any((odd & 0x80008000u) != 0) ? 1 : 0;
                    if (odd) {  // rare
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int j = 0; j < NJ; ++j) {
                                const int off = (p + h) * kPage + (j * 64 + lane) / CPR - x.base;
                                u32x4 v = vr[h][j];
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const uint32_t top = (v[e] & 0x7f807f80u) + 0x00800080u;
                                    const uint32_t bad = (top & 0x8000u ? 0xffffu : 0u) | (top >> 31 ? 0xffff0000u : 0u);
                                    v[e] &= off < 0 ? ~0u : ~bad;
                                }
                                vr[h][j] = v;
                            }
                    }
                }
                if (there) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int j = 0; j < NJ; ++j) {
                            const int f = j * 64 + lane, r = f / CPR, ch = f - r * CPR;
                            *reinterpret_cast<u32x4*>(sk + (h * kPage + r) * KP + ch * 8) = kr[h][j];
                            *reinterpret_cast<u32x4*>(sv + (h * kPage + r) * VP + ch * 8) = vr[h][j];
                        }
                }
                // the next pair, of this work or the next one
                const bool more = i + 1 < x.mine;
                if (more && ((i + 1) & 31) == 0) ids = page_ids(x, p + 2 * kTreeWaves);
                if (more || next < n_all) {
                    pair = pair_of(more ? head : head2, more ? ids : ids2, more ? i + 1 : 0);
                    if (pair.there) fetch(pair);
                }
                if (!there) continue;
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
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int part = 1; part >= 0; --part) {
                        bf16x8 b[NJ];
#pragma unroll
                        for (int j = 0; j < NJ; ++j)
                            b[j] = __builtin_bit_cast(bf16x8, sq[(t * NJ + j) * 128 + part * 64]);
#pragma unroll
                        for (int j = 0; j < NJ; ++j)
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                s[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[h][j], b[j], s[t][h], 0, 0, 0);
                    }
                // with two tiles of 128 dims no registers are left for V before the scores are done
                if constexpr (HD == 128 && NT == 2) __builtin_amdgcn_sched_barrier(0);
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
                        const uint64_t mask = s_mask[x.row0 + max(0, min(t * 16 + c, x.n - 1))];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t see = sees4(mask, (p + h) * kPage + 4 * g - x.base) & (there >> h & 1 ? 15u : 0u);
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
                if (odd) {  // rare: the values taken out above, to the rows that see them
                    for (int kk = 0; kk < 2 * kPage; ++kk) {
                        const int off = p * kPage + kk - x.base;
                        if (off < 0 || off >= 64 || !(x.seen >> off & 1) || !(there >> (kk >> 4) & 1)) continue;
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
                            const bool see = s_mask[x.row0 + max(0, min(t * 16 + c, x.n - 1))] >> off & 1;
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

            // the segment: the waves' states, [wave][row][dim]
            int tl = tid;
            asm volatile("" : "+v"(tl));  // addresses made here, not kept through the pairs
            const int ll = tl & 63, lc = tl & 15, lg = tl >> 4 & 3;
            __syncthreads();  // every wave is done with its K and V, and with q at the last segment
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float l = over_rows_sum(st.l[t]);
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    *reinterpret_cast<floatx4*>(so + (wave * ROWS + t * 16 + lc) * PITCH + 16 * b + 4 * lg) = st.o[t][b];
                if (lg == 0) {
                    sf.m[t * 16 + lc][wave] = st.m[t];
                    sf.l[t * 16 + lc][wave] = l;
                }
            }
            st.clear();
            if (sg == x.sg1 - 1 && next < n_all) stage_q();
            __syncthreads();
            // lane 8k + w: wave w's part in this wave's row k, wave + 8k
            const int at = (wave + kTreeWaves * (min(ll, 8 * NR - 1) >> 3)) * kTreeWaves + (ll & 7);
            const float sm = (&sf.m[0][0])[at];
            const float mx = over_8_max(sm), f = exp2_raw(sm - mx), den = over_8_sum(f * (&sf.l[0][0])[at]);
            float fa = 0.f, fb = 0.f;
            if (whole) join_segment(tm, tw, mx, den, fa, fb);
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                const int r = wave + kTreeWaves * k;
                if (r >= x.n) break;
                float a = 0.f, b = 0.f;
#pragma unroll
                for (int w = 0; w < kTreeWaves; ++w) {
                    const float2 o2 =
                        *reinterpret_cast<const float2*>(so + (w * ROWS + r) * PITCH + 2 * min(ll, HD / 2 - 1));
                    const float fw = lane_value(f, 8 * k + w);
                    a = fmaf(fw, o2.x, a);
                    b = fmaf(fw, o2.y, b);
                }
                if (whole) {
                    const float ta = lane_value(fa, 8 * k), tb = lane_value(fb, 8 * k);
                    tot[k][0] = join_sum(tot[k][0], a, ta, tb);
                    tot[k][1] = join_sum(tot[k][1], b, ta, tb);
                } else {
                    float* rec = ts.part + (((size_t)(x.row0 + r) * H + head) * kTreeSegs + sg) * REC;
                    if (2 * ll < HD) *reinterpret_cast<float2*>(rec + 2 * ll) = make_float2(a, b);
                    if (ll == 8 * k) *reinterpret_cast<float2*>(rec + HD) = make_float2(mx, den);
                }
            }
            __syncthreads();  // K and V take the place of the states
        }
        if (whole) {
            int tl = tid;
            asm volatile("" : "+v"(tl));
            const int dim = 2 * (tl & 63);
            uint32_t odd_rows = 0;
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                const int r = wave + kTreeWaves * k;
                const float den = lane_value(tw, 8 * k);
                tot[k][0] /= den;
                tot[k][1] /= den;
                if (r < x.n) {
                    odd_rows |= __any(row_odd(tot[k][0], tot[k][1])) ? 1u << k : 0u;
                    if (dim < HD)
                        *reinterpret_cast<uint32_t*>(out + frag_index(x.row0 + r, head * HD + dim, d)) =
                            pack_bf16(tot[k][0], tot[k][1]);
                }
            }
            while (__builtin_expect(odd_rows != 0, 0)) {  // rare
                const int at = __ffs(odd_rows) - 1, row = x.row0 + wave + kTreeWaves * at;
                odd_rows &= odd_rows - 1;
                float a = tot[0][0], b = tot[0][1];
#pragma unroll
                for (int k = 1; k < NR; ++k) {
                    a = at == k ? tot[k][0] : a;
                    b = at == k ? tot[k][1] : b;
                }
                const uint32_t o = row_plain<HD>(a, b, q + (size_t)row * d + head * HD, kv, x.seq, x.plane, x.base,
                                                 s_mask[row], head, H);
                if (dim < HD) *reinterpret_cast<uint32_t*>(out + frag_index(row, head * HD + dim, d)) = o;
            }
        }
        if (next >= n_all) break;
        x = get_work(slot);
        ids = ids2;
        work = next;
    }
}

// Rows whose segments went to several workgroups: their records joined, in segment
// order.  One wave per (row, head), lane = two dims.
template <int HD>
__global__ __launch_bounds__(256) void k_tree_merge(const float* __restrict__ q, KvTarget kv, const int32_t* __restrict__ seq, cdb_tree tree, int M,
                                                    int H, TreeScratch ts, uint16_t* __restrict__ out,
                                                    const int32_t* __restrict__ dn) {
    constexpr int REC = HD + 2;
    const int lane = threadIdx.x & 63, rh = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int row = rh / H, head = rh - row * H;
    const int runs = *ts.runs;
    if (row >= M) return;
    const RowSees s = row_sees(kv, seq, tree, row);
    if (runs == 1 || row >= live_rows(dn, M) || !s.ok) return;
    int sp;
    const int nseg = tree_segments(s.base / kPage + 1, &sp);
    if (nseg == 1) return;
    const float* rec = ts.part + ((size_t)row * H + head) * kTreeSegs * REC;
    const int at = min(lane, nseg - 1) * REC + HD;
    const float sm = rec[at], sl = rec[at + 1];
    const int dim = 2 * min(lane, HD / 2 - 1);
    float tm = -1e30f, tl = 0.f, ta = 0.f, tb = 0.f;
    for (int s0 = 0; s0 < nseg; s0 += 8) {
        float2 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const float2*>(rec + min(s0 + u, nseg - 1) * REC + dim);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (s0 + u >= nseg) break;
            float a, b;
            join_segment(tm, tl, __shfl(sm, s0 + u, 64), __shfl(sl, s0 + u, 64), a, b);
            ta = join_sum(ta, v[u].x, a, b);
            tb = join_sum(tb, v[u].y, a, b);
        }
    }
    ta /= tl;
    tb /= tl;
    uint32_t o = pack_bf16(ta, tb);
    if (__builtin_expect(__any(row_odd(ta, tb)), 0))
        o = row_plain<HD>(ta, tb, q + ((size_t)row * H + head) * HD, kv, s.seq, s.plane, s.base, s.mask, head, H);
    if (2 * lane < HD) *reinterpret_cast<uint32_t*>(out + frag_index(row, head * HD + dim, H * HD)) = o;
}

// rows per tile
static int tree_rows_per_tile(int max_nodes) { return max_nodes <= 16 ? 16 : max_nodes <= 32 ? 32 : 64; }

template <int HD>
static hipError_t run_tree_attn(const float* q, const KvTarget& kv, const int32_t* seq, const cdb_tree& tree, int M, int H,
                                const TreeScratch& ts, uint16_t* out, int* err, hipStream_t st, const int32_t* dn) {
    const int cap = tree_rows_per_tile(tree.max_nodes), halves = cap == 64 ? 2 : 1;
    int pages;
    const int segs = tree_segments(kv.max_pages + 1, &pages);  // the most a row's context may have
    const int least = dn ? 0 : (M + cap - 1) / cap;  // tiles of all rows, at least
    // no more workgroups than there can be works, and one resident per CU
    const int most = std::min(M * H * halves * segs, kTreeCUs);
    if (cap == 16)
        k_tree_attn<HD, 1, false><<<most, kTreeThreads, 0, st>>>(q, kv, seq, tree, M, H, ts, out, err, dn, least);
    else if (cap == 32)
        k_tree_attn<HD, 2, false><<<most, kTreeThreads, 0, st>>>(q, kv, seq, tree, M, H, ts, out, err, dn, least);
    else  // whole groups of 16
        k_tree_attn<HD, 2, true><<<(most + 15) / 16 * 16, kTreeThreads, 0, st>>>(q, kv, seq, tree, M, H, ts, out, err, dn, least);
    const bool split = segs > 1 && (dn || tree_runs(least * H * halves) > 1);
    if (split) k_tree_merge<HD><<<(M * H + 3) / 4, 256, 0, st>>>(q, kv, seq, tree, M, H, ts, out, dn);
    return hipGetLastError();
}

hipError_t launch_tree_attention(const float* q, const KvTarget& kv, const int32_t* seq, const cdb_tree& tree, int M,
                                 int H, int hd, void* scratch, uint16_t* out, int* err, hipStream_t st,
                                 const int32_t* dn) {
    if (M <= 0) return hipSuccess;
    if (M > kMaxRows) return hipErrorInvalidValue;
    const TreeScratch ts = tree_scratch(scratch, H, hd, M);
    switch (hd) {
        case 64: return run_tree_attn<64>(q, kv, seq, tree, M, H, ts, out, err, st, dn);
        case 96: return run_tree_attn<96>(q, kv, seq, tree, M, H, ts, out, err, st, dn);
        case 128: return run_tree_attn<128>(q, kv, seq, tree, M, H, ts, out, err, st, dn);
    }
    return hipErrorInvalidValue;
}

}  // namespace cdb
