// Causal attention of chunks of new tokens (several sequences, one to thousands of
// rows each) over the paged, depth-indexed KV cache.
//
//   out[i] = sum_{s <= p_i} 2^(x_is - m_i) V_s / sum_{s <= p_i} 2^(x_is - m_i),
//   x_is = q_i . K_s log2(e) / sqrt(hd),
//
// in one pass over the keys, with a running m_i and both sums scaled as it grows.
//
// Bound: 4 hd operations per (row, key, head) at the matrix rate where chunks are
// long, K and V once per chunk at the memory rate where they are short, and a chain of
// latencies (chunk, page id, K, scores, weights, V, join) where there is little of either.
// Workgroup = (head, tile of 128 rows, segment of the context), a wave to 32 rows: K and V
// are staged in LDS once for four waves, and with 32x32x16 products an operand read from
// LDS serves 32 rows.  S^T = K q^T leaves a row's scores in two lanes, so that maxima and sums
// need one exchange, and in the registers that the second product takes its weights from.
// The three parts of a half step (scores of the next 32 keys, weights of these, products
// of the ones before) do not depend on one another and stand interleaved in one block: a
// wave's exponentials run under its own products.  One barrier per 64 keys.
//
// Measured (bf16 q; us, with the join of segments; ranges over inputs and machines): 4 chunks of 2048 rows behind
// 4096 positions, 16 x 128 heads: 346-372, 925-993 TFLOP/s (a large library product reaches 1220-1230
// here; the instructions of a half alone take 690 cycles, of which the products 512); 62 single rows
// and 2 chunks of 700-1000 behind 2048-4100: 301-306, 5.6 TB/s of K and V; 9 chunks of
// 33-333 behind up to 2047, 55 x 96 heads: 89-102, 480-555 TFLOP/s; 13 rows behind 700: 12.6-13.6,
// latency; fp32 q, 512 rows behind 512: 29-34.
#include <algorithm>
#include <type_traits>

#include "cdb_internal.h"

namespace cdb {

constexpr int kTileRows = 128;  // rows of a workgroup: 32 to each of its 4 waves
constexpr int kNoVmem = 0xf70;  // s_waitcnt: vector memory loads 0, the others any
constexpr int kStep = 64;       // keys that a workgroup stages at a time, a page to each wave

// How contexts are cut (us; 16 x 128 heads where nothing else is said).
// Enough segments that there are kWant (tile, head, segment) triples, one to a compute unit: none against 256
// against 1024 of them, 13 rows behind 700 21.3 / 13.5 / 13.9, 512 fp32 rows behind 512 46.5 / 33.4 / 36.9, 2
// chunks of 700-1000 rows behind 2048-4100 89.4 / 71.9 / 75.4, 9 chunks of 33-333, 55 x 96 heads
// 97 / 97 / 114, 2 of 1024 behind 2048, 55 x 96 heads 153 / 149 / 182.  Segments of kFill positions at least: of 512
// the first two take 18.8 and 39.6.
// Longer segments than kLong positions are cut also where the launch is large, so that one long context does not
// outlast the others; at 1536 the records cost long chunks more than that gives (62 rows and 2 chunks 347 against
// 305, the last case above 187 against 149).  A chunk of kFewRows rows or fewer, one wave's, writes little of
// them: 64 single rows behind 3000-4000 take 332 with kLongFew, 360 without.
// All as far as there are records, which every row of a call has as many of: kChunkRecordRows / n_rows, so 2 up to 2048 rows and
// none above, where a workgroup takes a head's whole context: 2048 rows take 53, one more behind 32768 makes it 537, and
// alone that one takes 48.
constexpr int kWant = 256, kFill = 64;
constexpr int kLong = 8192, kLongFew = 1536, kFewRows = 32;

// From here on a scaled score's last place is worth 64 and more.
constexpr float kFar = 1073741824.f;

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Segments that a context of `keys` positions (1 or more, up to 2^31 - 1) is to be cut into: as many as the launch wants to
// fill the GPU (of kFill positions at least), and none longer than kLong positions, or kLongFew where few rows make records
// that cost little.  Not fewer for a longer context or for fewer rows.
__host__ __device__ __forceinline__ int segments_wanted(int keys, int rows, const ChunkSplit& s) {
    const int last = keys - 1, fill = last / kFill + 1;
    const int n = last / (rows <= kFewRows ? kLongFew : kLong) + 1, filling = fill < s.want ? fill : s.want;
    return n < filling ? filling : n;
}

// Segments that a chunk's context is cut into, as far as there are records for them.  *len: positions of a segment, whole
// steps, up to 2^31 of them.
__device__ __forceinline__ int chunk_segments(int keys, int rows, const ChunkSplit& s, uint32_t* len) {
    const int last = keys - 1, n = min(segments_wanted(keys, rows, s), s.most);
    *len = ((uint32_t)(last / n) / kStep + 1) * kStep;
    return (uint32_t)last / *len + 1;
}

ChunkSplit chunk_split(int H, int n_chunks, int n_rows, int max_pages) {
    ChunkSplit s{1, 1};
    const int tiles = std::max(n_chunks, (n_rows + kTileRows - 1) / kTileRows);
    s.want = std::max(1, (kWant + tiles * H - 1) / std::max(1, tiles * H));
    s.most = std::max(1, std::min(kChunkSegments, kChunkRecordRows / std::max(1, n_rows)));
    // no more than the longest context that the tables hold may be cut into: the grid has a workgroup for each
    s.most = std::min(s.most, segments_wanted(std::max(1, max_pages * kPage), 1, s));
    return s;
}

size_t chunk_scratch_bytes(const cdb_model_desc& d, int rows) {
    const int64_t n = std::min<int64_t>((int64_t)rows * kChunkSegments, kChunkRecordRows);
    return (size_t)n * d.n_heads * (d.head_dim + 2) * 4;
}

struct ChunkAttnArgs {
    cdb_chunks ch;
    KvTarget kv;
    const void* q;
    uint16_t* out;
    int order, H, xcd_heads;
    ChunkSplit split;
    float* part;  // [rows][H][split.most][hd], then maxima and weights [rows][H][split.most][2]
    float2* ml;
    int* err;
};

// A tile of one chunk's rows, and a segment of its context.
struct ChunkTile {
    int row, n;     // first row in the call's buffers, rows
    int pos;        // position of the first row
    int seq, plane;
    int seg;
    uint32_t seg_len;
    int found;
};

// Whether a chunk of n rows is in range.
__device__ __forceinline__ bool chunk_ok(const KvTarget& kv, int seq, int pos, int c, int n) {
    return seq >= 0 && seq < kv.max_seqs && pos >= 0 && pos <= kv.max_pages * kPage - n &&
           (!kv.c_row || (c >= 0 && c < kv.n_planes - 2));
}

// The work-th (tile, segment) pair from the end (later tiles of a chunk see longer contexts, so they come first).
// Run by all 256 threads, thread = chunk; false: there is no such pair.  Workgroups without one come
// last, when others have all of the work.
__device__ __forceinline__ bool chunk_tile(const ChunkAttnArgs& a, int work, ChunkTile* s_tile, int* s_red, bool tells) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int r0 = 0, r1 = 0, seq = -1, pos = 0, c = 0;
    if (tid < a.ch.n_chunks) {
        r0 = a.ch.row0[tid];
        r1 = a.ch.row0[tid + 1];
        seq = a.ch.seq[tid];
        pos = a.ch.pos0[tid];
        if (a.kv.c_row) c = a.kv.c_row[tid];
    }
    const bool bad = r0 < 0 || r1 < r0 || r1 > a.ch.n_rows;
    const int n = r1 - r0;
    const bool ok = !bad && n > 0 && chunk_ok(a.kv, seq, pos, c, n);
    if (tells && !bad && n > 0 && !ok) set_err(a.err, CDB_DEV_BAD_INDEX);
    uint32_t len = 0;
    const int segs = ok ? chunk_segments(pos + n, n, a.split, &len) : 0, works = ok ? (n + kTileRows - 1) / kTileRows * segs : 0;
    int v = works;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    const bool any_bad = __any(bad);
    if (lane == 63) s_red[w] = any_bad ? 1 << 24 : v;
    if (tid == 0) s_tile->found = 0;
    __syncthreads();
    int total = 0, before = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i < w) before += s_red[i];
        total += s_red[i];
    }
    if (total >= 1 << 24) {
        if (tells && tid == 0) set_err(a.err, CDB_DEV_BAD_INDEX);
        return false;
    }
    const int at = total - 1 - work, first = before + v - works;
    if (at < 0) return false;
    if (at >= first && at < first + works) {
        const int tile = (at - first) / segs, skip = tile * kTileRows;
        *s_tile = ChunkTile{r0 + skip, min(kTileRows, n - skip), pos + skip, seq, a.kv.c_row ? c + 1 : a.kv.plane_fixed,
                            at - first - tile * segs, len, 1};
    }
    __syncthreads();
    return s_tile->found;
}

// (head, rest) of a workgroup.  Workgroups go round the 8 XCDs by their index, so
// with xcd_heads a head stays on one of them, whose L2 then holds its K and V for
// all tiles (55 x 96 heads: 149 against 160 us for 2 chunks of 1024, 97 against 102 for 9 of
// 33-333).  Taken while rounding the heads up to eights leaves at most an eighth of the workgroups idle.
__device__ __forceinline__ bool chunk_head(const ChunkAttnArgs& a, int id, int* head, int* rest) {
    if (!a.xcd_heads) {
        *head = id % a.H;
        *rest = id / a.H;
        return true;
    }
    const int slot = id >> 3;
    *head = (slot % a.xcd_heads) * 8 + (id & 7);
    *rest = slot / a.xcd_heads;
    return *head < a.H;
}

__device__ __forceinline__ uint16_t* chunk_out(const ChunkAttnArgs& a, int row, int k, int d) {
    return a.out + (a.order == CDB_ORDER_ROWS ? (size_t)row * d + k : frag_index(row, k, d));
}

__device__ __forceinline__ bool odd_words(u32x4 x) {  // an infinity or NaN among 8 bf16 values
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) odd |= (x[i] & 0x7f80u) == 0x7f80u || (x[i] & 0x7f800000u) == 0x7f800000u;
    return odd;
}

// Eight weights times a power of two.
__device__ __forceinline__ bf16x8 scaled(bf16x8 p, float f) {
    u32x4 w = __builtin_bit_cast(u32x4, p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(bflo(w[i]) * f, bfhi(w[i]) * f);
    return __builtin_bit_cast(bf16x8, w);
}

// PER_CU: workgroups that a compute unit can hold.  Two leave a wave 256 registers, 17 too few for heads of 128 with q in two
// parts; one leaves it all it needs.  fp32 q, one against two (us; 16 heads): 2048 rows 72 / 90, 1024 behind 4096 93 / 114, 2
// of 2048 behind 2048 208 / 227, 1024 rows 36 / 37, but 512 behind 512 34.6 / 33.8, 12 chunks of 100-300 93 / 84, 65 single
// rows 359 / 340, where loads and starts are to be covered.  So long chunks take one (kLongChunk rows each on average).
constexpr int kLongChunk = 1024;
template <int HD, bool SPLIT, int PER_CU>
__global__ __launch_bounds__(256, PER_CU) void k_chunk_attn(ChunkAttnArgs a) {
    constexpr int NT = HD / 16, NB = HD / 32, NL = HD / 32, CPK = HD / 8;
    // Row pitches, and how many banks apart (mod 64) consecutive keys are in heads of 64, 96 and 128.  Conflicts, of the
    // cycles that LDS is read or written in: none, 5.7% (9 ragged chunks), none.
    constexpr int KP = HD + 8;                   // K: 36, 52, 4
    constexpr int VP = HD == 96 ? HD : HD + 32;  // V: 48, 48, 16
    __shared__ __align__(16) uint16_t sk[2][kStep * KP];
    __shared__ __align__(16) uint16_t sv[2][kStep * VP];
    __shared__ __align__(16) int s_there[2][4];  // by page of a step: whether it is mapped
    __shared__ int s_odd;                        // whether stage_v took something out
    __shared__ ChunkTile s_tile;
    __shared__ int s_red[4];
    int head, rest;
    if (!chunk_head(a, blockIdx.x, &head, &rest)) return;
    if (!chunk_tile(a, rest, &s_tile, s_red, blockIdx.x == 0)) return;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, c32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t_row = __builtin_amdgcn_readfirstlane(s_tile.row), t_n = __builtin_amdgcn_readfirstlane(s_tile.n);
    const int t_pos = __builtin_amdgcn_readfirstlane(s_tile.pos);
    const int last = t_pos + t_n - 1;  // the last position that any row sees
    const int seg = __builtin_amdgcn_readfirstlane(s_tile.seg);
    const uint32_t seg_len = __builtin_amdgcn_readfirstlane(s_tile.seg_len);
    const int segs = (uint32_t)last / seg_len + 1;  // of this tile
    if (seg >= segs) return;
    // positions reach 2^31 - 81, so that a step behind them does not pass 32 bits, and two do
    const int k0 = seg * seg_len, k1 = min(last + 1u, k0 + seg_len);
    const int steps = (k1 - k0 + kStep - 1) / kStep;
    const int d = a.H * HD;
    const int my = w * 32 + c32;  // this lane's row in the tile
    const int qpos = t_pos + min(my, t_n - 1);
    const int w_first = t_pos + min(w * 32, t_n - 1);           // position of the wave's first row
    const int w_last = t_pos + min(t_n, w * 32 + 32) - 1;       // and of its last one
    const int na = w * 32 < t_n && w_last >= k0 ? min(2 * steps, (w_last - k0) / 32 + 1) : -1;  // halves with keys that it sees
    // the table by scalar loads: a page id is asked for a step before it is used, and vector loads would make its
    // use wait for the K and V that are on their way
    const auto* pt = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.kv.page_table + ((size_t)__builtin_amdgcn_readfirstlane(s_tile.seq) * a.kv.n_planes +
                                           __builtin_amdgcn_readfirstlane(s_tile.plane)) * a.kv.max_pages);

    // staging: wave w takes page w of a step
    u32x4 kr[NL], vr[NL];
    const int tables = a.kv.max_pages - 1;
    const int page0 = k0 / kPage + w;
    auto entry_of = [&](int t) { return pt[min(page0 + t * (kStep / kPage), tables)]; };
    auto page_of = [&](int t, int pid) {  // -2: behind the segment, -1: not mapped
        return page0 + t * (kStep / kPage) > (k1 - 1) / kPage ? -2 : pid >= 0 && pid < a.kv.n_pages ? pid : -1;
    };
    const uint16_t* pool = a.kv.pool + kv_offset(a.kv.layer, 0, a.kv.n_pages, 0, head, a.H, 0, HD) + lane * 8;
    const size_t page_len = (size_t)2 * a.H * kPage * HD, v_off = (size_t)a.H * kPage * HD;
    auto fetch_page = [&](u32x4 (&r)[NL], int pid, size_t off) __attribute__((always_inline)) {
        const uint16_t* at = pool + pid * page_len + off;
#pragma unroll
        for (int i = 0; i < NL; ++i) r[i] = *reinterpret_cast<const u32x4*>(at + i * 512);
    };
    auto fetch = [&](u32x4 (&r)[NL], int pid, size_t off) __attribute__((always_inline)) {
        if (pid >= 0) {
            fetch_page(r, pid, off);
        } else {
#pragma unroll
            for (int i = 0; i < NL; ++i) r[i] = u32x4{0, 0, 0, 0};
        }
    };
    auto put_k = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int f = i * 64 + lane;
            *reinterpret_cast<u32x4*>(&sk[b][(w * kPage + f / CPK) * KP + f % CPK * 8]) = kr[i];
        }
    };
    auto stage_k = [&](int pid, int b) __attribute__((always_inline)) {
        if (lane == 0) s_there[b][w] = pid >= 0;
        put_k(b);
    };
    auto put_v = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int f = i * 64 + lane;
            *reinterpret_cast<u32x4*>(&sv[b][(w * kPage + f / CPK) * VP + f % CPK * 8]) = vr[i];
        }
    };
    // Of a step whose keys not all rows see, V behind the last position becomes 0, and a V that is not finite too
    // (at the end it is added to the rows that see it).
    auto stage_v = [&](int t, int pid, int b) __attribute__((always_inline)) {
        bool odd = false;
        if (k0 + t * kStep + kStep - 1 > t_pos && pid >= 0)
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int key = k0 + t * kStep + w * kPage + (i * 64 + lane) / CPK;
                const bool gone = key > last, o = !gone && odd_words(vr[i]);
                odd |= o;
                if (gone) vr[i] = u32x4{0, 0, 0, 0};
                if (o)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        if ((vr[i][x] & 0x7f80u) == 0x7f80u) vr[i][x] &= 0xffff0000u;
                        if ((vr[i][x] & 0x7f800000u) == 0x7f800000u) vr[i][x] &= 0xffffu;
                    }
            }
        if (odd) s_odd = 1;
        put_v(b);
    };
    // bits: the step's pages whose word is set
    auto bits = [&](const int* f) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(f);
        return __builtin_amdgcn_readfirstlane((int)(v[0] | v[1] << 1 | v[2] << 2 | v[3] << 3));
    };

    // whether every page of the segment is mapped
    bool hole = false;
    for (int i = tid; i < (k1 - k0 + kPage - 1) / kPage; i += 256) {
        const int id = pt[k0 / kPage + i];
        hole |= id < 0 || id >= a.kv.n_pages;
    }
    if (hole) set_err(a.err, CDB_DEV_UNMAPPED_PAGE);
    const int pid0 = page_of(0, entry_of(0));
    int entry = entry_of(1);
    fetch(kr, pid0, 0);
    fetch(vr, pid0, v_off);

    // q as the B operand: dims 16 t + 8 half + e of row c32; in two parts it takes the scale along
    const float scale = 1.4426950408889634f / sqrtf((float)HD);
    bf16x8 qh[NT], ql[SPLIT ? NT : 1];
    {
        const bool live = my < t_n;
        const size_t at = (size_t)(t_row + (live ? my : 0)) * d + head * HD + half * 8;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (SPLIT) {
                const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at + t * 16);
                const float4 x = src[0], y = src[1];
                const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                uint32_t hw[4], lw[4];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float v0 = v[e] * scale, v1 = v[e + 1] * scale;
                    const uint32_t h = pack_bf16(v0, v1);
                    hw[e / 2] = h;
                    lw[e / 2] = pack_bf16(v0 - bflo(h), v1 - bfhi(h));
                }
                qh[t] = __builtin_bit_cast(bf16x8, u32x4{hw[0], hw[1], hw[2], hw[3]});
                ql[t] = __builtin_bit_cast(bf16x8, u32x4{lw[0], lw[1], lw[2], lw[3]});
            } else {
                qh[t] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + at + t * 16));
            }
        }
    }
    const float s_scale = SPLIT ? 1.f : scale;

    floatx16 o[NB], s0, s1;  // s0, s1: scores of first and second halves
#pragma unroll
    for (int j = 0; j < 16; ++j) s0[j] = s1[j] = 0.f;
#pragma unroll
    for (int x = 0; x < NB; ++x) o[x] = s0;
    float m = -INFINITY, l = 0.f;
    // bf16 queries: m follows a score that is above lim; rows at kFar or beyond (far: which of the wave) have their maximum in
    // lim, scores less it, and m = 0
    float lim = -INFINITY;
    uint64_t far = 0;
    bf16x8 ph[2], pl[2];  // weights of the half before
    ph[0] = ph[1] = pl[0] = pl[1] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});

    const int k_at = c32 * KP + half * 8;
    const int v_at = (4 * half + ((lane & 15) >> 2)) * VP + (lane >> 4 & 1) * 16 + (lane & 3) * 4;
    auto k_operand = [&](const uint16_t* k, int t) { return *reinterpret_cast<const bf16x8*>(k + k_at + t * 16); };
    auto v_operand = [&](const uint16_t* v, int st, int x) {
        const uint16_t* at = v + v_at + st * 16 * VP + x * 32;
        const uint2 w0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at));
        const uint2 w1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * VP)));
        return __builtin_bit_cast(bf16x8, u32x4{w0.x, w0.y, w1.x, w1.y});
    };
    auto scores = [&](const uint16_t* k) __attribute__((always_inline)) {
        floatx16 r;
#pragma unroll
        for (int j = 0; j < 16; ++j) r[j] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const bf16x8 ka = k_operand(k, t);
            if constexpr (SPLIT) r = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, ql[t], r, 0, 0, 0);
            r = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qh[t], r, 0, 0, 0);
        }
        return r;
    };
    auto product = [&](const uint16_t* v, int st, int x, const bf16x8 (&h)[2], const bf16x8 (&lo)[2]) __attribute__((always_inline)) {
        const bf16x8 va = v_operand(v, st, x);
        if constexpr (SPLIT) o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, lo[st], o[x], 0, 0, 0);
        o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, h[st], o[x], 0, 0, 0);
    };
    auto products = [&](const uint16_t* v) __attribute__((always_inline)) {
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int x = 0; x < NB; ++x) product(v, st, x, ph, pl);
    };
    // Half i (32 keys from k, scores in s): scores of the next one, weights of this one, products of the one before, which
    // do not depend on one another.  there: this half's two pages.
    // PLAIN: every row sees all of this half and of the one before.
    auto run_half = [&](auto plain, int i, int k, floatx16& s, floatx16& next, const uint16_t* k_next, const uint16_t* v_before,
                        int there) __attribute__((always_inline)) {
        constexpr bool PLAIN = decltype(plain)::value;
        if (PLAIN ? na < 0 : i > na) return;  // half na: nothing of it is seen
        if (!PLAIN && (k + 31 > w_first || there != 3))
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (k + (j >> 2) * 8 + half * 4 + (j & 3) > qpos || !(there >> (j >> 3) & 1)) s[j] = -INFINITY;
        // The maximum that a row's weights are taken against is a whole number (of powers of two) and follows the
        // row's own once that is 8 above: what is scaled then, the weights at hand among it, stays exact.
        float mx = fmaxf(s[0], s[1]);
#pragma unroll
        for (int j = 2; j < 16; ++j) mx = fmaxf(mx, s[j]);
        float top;
        {
            const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            top = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
        }
        mx = top * s_scale;
        bool up = mx > (SPLIT ? m + 8.f : lim);
        if ((__ballot(up) | far) != 0) {
            const float limit = lim;
            float was = m;
            // A bf16 row's scores are scaled with the subtraction of the maximum, in one rounding, and against a maximum that was
            // rounded itself the largest weight may be any 2^(half its last place).  So from kFar on a row's maximum is a
            // quarter of its largest score, unscaled and exact: above (below, if negative) every other row's kind of maximum,
            // and in the scores' own order.  Different scores are 64 powers of two apart there, so that only equal ones
            // count, as many as there are, in one segment and where segments are joined.
            if constexpr (!SPLIT) {
                if (__builtin_expect((far | __ballot(fabsf(mx) >= kFar)) != 0, 0)) {
                    was = fabsf(limit) >= kFar ? limit : was;
                    mx = fabsf(mx) >= kFar ? top * 0.25f : mx;
                    up = mx > limit;
                }
            }
            const float now = up ? ceilf(mx) : was;
            const float corr = up ? __builtin_amdgcn_exp2f(was - now) : 1.f;
            m = now;
            l *= corr;
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[x][j] *= corr;
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                ph[st] = scaled(ph[st], corr);
                if constexpr (SPLIT) pl[st] = scaled(pl[st], corr);
            }
            if constexpr (!SPLIT) {
                lim = now + 8.f;  // now itself from kFar on
                const bool mine = fabsf(now) >= kFar && now > -INFINITY;
                far = __ballot(mine);
                if (__builtin_expect(far != 0, 0)) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) s[j] = mine ? fmaf(-4.f, now, s[j]) : s[j];
                    m = mine ? 0.f : now;
                }
            }
        }
        const float m0 = !PLAIN && m == -INFINITY ? 0.f : m;  // nothing seen yet: every weight 0
        const bf16x8 h[2] = {ph[0], ph[1]}, lo[2] = {pl[0], pl[1]};
#pragma unroll
        for (int j = 0; j < 16; ++j) next[j] = 0.f;
        uint32_t hw[8], lw[8];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            if (t < NT) {
                const bf16x8 ka = k_operand(k_next, t);
                if constexpr (SPLIT) next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, ql[t], next, 0, 0, 0);
                next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qh[t], next, 0, 0, 0);
                product(v_before, t / NB, t % NB, h, lo);
            }
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[2 * t], s_scale, -m0));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(s[2 * t + 1], s_scale, -m0));
            hw[t] = pack_bf16(p0, p1);
            // With few keys the sum is that of the weights as the product takes them, so that their rounding drops out of a
            // row that sees one key (0 against 2^-9, 0.0019 against 0.0023 of the values with 32 keys); over many keys it
            // makes no difference, and costs two instructions a pair.
            l += SPLIT || PLAIN ? p0 + p1 : bflo(hw[t]) + bfhi(hw[t]);
            if constexpr (SPLIT) lw[t] = pack_bf16(p0 - bflo(hw[t]), p1 - bfhi(hw[t]));
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            ph[st] = __builtin_bit_cast(bf16x8, u32x4{hw[st * 4], hw[st * 4 + 1], hw[st * 4 + 2], hw[st * 4 + 3]});
            if constexpr (SPLIT) pl[st] = __builtin_bit_cast(bf16x8, u32x4{lw[st * 4], lw[st * 4 + 1], lw[st * 4 + 2], lw[st * 4 + 3]});
        }
        __builtin_amdgcn_s_setprio(0);
        // here, next to the products, and not sunk to where the weights are used
        asm volatile("" : "+v"(ph[0]), "+v"(ph[1]), "+v"(l));
        if constexpr (SPLIT) asm volatile("" : "+v"(pl[0]), "+v"(pl[1]));
    };

    if (tid == 0) s_odd = 0;
    __syncthreads();
    // V of the half before the first: zeros
    for (int i = tid; i < 32 * VP / 8; i += 256) *reinterpret_cast<u32x4*>(&sv[1][32 * VP + i * 8]) = u32x4{0, 0, 0, 0};
    stage_k(pid0, 0);
    stage_v(0, pid0, 0);
    // nothing is on its way here (q among it), so that no use of q in the loop waits for later loads
    __builtin_amdgcn_s_waitcnt(kNoVmem);
    int pid_k = page_of(1, entry), pid_v = pid_k;
    entry = entry_of(2);
    fetch(kr, pid_k, 0);
    fetch(vr, pid_v, v_off);
    const bool all_there = !__syncthreads_or(hole);
    if (na >= 0) s0 = scores(sk[0]);
    // A step's first half needs nothing that was staged since the last barrier, and its barrier stands before the
    // second half, which needs K of the next step and V of this one.
    int t = 0;
    // Steps that every row sees, with another such one behind them (its V is staged here) and two whole ones: they
    // need neither masks nor flags, and the buffers of two of them are constants (4 chunks of 2048 rows behind
    // 4096: 360 us against 397 with the general steps alone).
    const int plain = all_there ? min(steps - 3, (t_pos + 1 - k0) / kStep - 1) : 0;
    auto plain_step = [&](auto buffer) __attribute__((always_inline)) {
        constexpr int b = decltype(buffer)::value;
        const std::true_type yes;
        const int pid_next = entry;  // of step t + 2
        entry = entry_of(t + 3);
        put_k(b ^ 1);
        fetch_page(kr, pid_next, 0);
        run_half(yes, 2 * t, 0, s0, s1, sk[b] + 32 * KP, sv[b ^ 1] + 32 * VP, 3);
        __syncthreads();
        put_v(b ^ 1);
        fetch_page(vr, pid_next, v_off);
        run_half(yes, 2 * t + 1, 0, s1, s0, sk[b ^ 1], sv[b], 3);
        ++t;
    };
    while (t + 2 <= plain) {
        plain_step(std::integral_constant<int, 0>{});
        plain_step(std::integral_constant<int, 1>{});
    }
    const int t_first = t;
    int there = 15;
    if (t_first > 0)
        pid_k = pid_v = 0;  // mapped, whichever it is
    else
        there = bits(s_there[0]);
    for (; t < steps; ++t) {
        const int k = k0 + t * kStep, b = t & 1;
        const bool more = t + 1 < steps;
        const std::false_type no;
        const int pid_next = page_of(t + 2, entry);
        entry = entry_of(t + 3);
        if (more) {
            stage_k(pid_k, b ^ 1);
            pid_k = pid_next;
            fetch(kr, pid_k, 0);
        }
        run_half(no, 2 * t, k, s0, s1, sk[b] + 32 * KP, sv[b ^ 1] + 32 * VP, there & 3);
        __syncthreads();
        const int there_next = bits(s_there[b ^ 1]);
        if (more) {
            stage_v(t + 1, pid_v, b ^ 1);
            pid_v = pid_next;
            fetch(vr, pid_v, v_off);
        }
        run_half(no, 2 * t + 1, k + 32, s1, s0, sk[b ^ 1], sv[b], there >> 2);
        there = there_next;
    }
    if (na == 2 * steps) {
        products(sv[(steps - 1) & 1] + 32 * VP);
    }

    {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    __syncthreads();
    if (my >= t_n) return;
    if (s_odd) {  // rare
#pragma unroll
        for (int x = 0; x < NB; ++x) {
            floatx16 more;
#pragma unroll
            for (int j = 0; j < 16; ++j) more[j] = 0.f;
#pragma unroll 1
            for (int key = max(k0, t_pos + 1 - kStep); key < k1; ++key) {
                const int id = pt[key / kPage];
                if (id < 0 || id >= a.kv.n_pages) continue;
                const uint16_t* at = a.kv.pool + kv_offset(a.kv.layer, id, a.kv.n_pages, 1, head, a.H, key % kPage, HD) + half * 4;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const uint16_t v = at[x * 32 + (j >> 2) * 8 + (j & 3)];
                    if ((v & 0x7f80) == 0x7f80 && key <= qpos) more[j] += bf2f(v);
                }
            }
            o[x] += more;
        }
    }
    const int row = t_row + my;
    if (segs == 1) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                uint2 v;
                v.x = pack_bf16(o[x][j] * inv, o[x][j + 1] * inv);
                v.y = pack_bf16(o[x][j + 2] * inv, o[x][j + 3] * inv);
                *reinterpret_cast<uint2*>(chunk_out(a, row, head * HD + x * 32 + j * 2 + half * 4, d)) = v;
            }
        return;
    }
    const size_t rec = ((size_t)row * a.H + head) * a.split.most + seg;
    if (half == 0) a.ml[rec] = make_float2(!SPLIT && fabsf(lim) >= kFar ? lim : m, l);
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int j = 0; j < 16; j += 4)
            *reinterpret_cast<float4*>(a.part + rec * HD + x * 32 + j * 2 + half * 4) =
                make_float4(o[x][j], o[x][j + 1], o[x][j + 2], o[x][j + 3]);
}

// Segments of a row joined, in order: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.  Workgroup = row; its threads
// take eight values of a head each.  A launch of its own, 4.2-5.5 us for small calls of which 2 are its launch; a
// join by the last workgroup of each (tile, head) was slower (13 rows behind 700: 14.3 against 13.1).
constexpr int kBatch = 8;  // records on their way at a time
template <int HD>
__global__ __launch_bounds__(256) void k_chunk_merge(ChunkAttnArgs a) {
    __shared__ int s_segs;
    const int tid = threadIdx.x, row = blockIdx.x;
    if (tid == 0) s_segs = 1;
    int r0 = 0, r1 = 0, seq = -1, pos = 0, c = 0;
    if (tid < a.ch.n_chunks) {
        r0 = a.ch.row0[tid];
        r1 = a.ch.row0[tid + 1];
        seq = a.ch.seq[tid];
        pos = a.ch.pos0[tid];
        if (a.kv.c_row) c = a.kv.c_row[tid];
    }
    if (__syncthreads_or(r0 < 0 || r1 < r0 || r1 > a.ch.n_rows)) return;
    if (row >= r0 && row < r1) {
        const int n = r1 - r0;
        if (chunk_ok(a.kv, seq, pos, c, n)) {
            uint32_t len;
            chunk_segments(pos + n, n, a.split, &len);
            s_segs = (uint32_t)(pos + min(n, ((row - r0) / kTileRows + 1) * kTileRows) - 1) / len + 1;
        }
    }
    __syncthreads();
    const int segs = s_segs;
    if (segs == 1) return;
    const int d = a.H * HD;
    for (int i = tid; i < d / 8; i += 256) {
        const size_t rec = ((size_t)row * a.H + i / (HD / 8)) * a.split.most;
        const float* part = a.part + rec * HD + i % (HD / 8) * 8;
        // every record is asked for before the first one is used: the kernel is a chain of memory latencies
        float2 ml[kChunkSegments];
#pragma unroll
        for (int s = 0; s < kChunkSegments; ++s) ml[s] = s < segs ? a.ml[rec + s] : make_float2(-INFINITY, 0.f);
        float num[8] = {}, den = 0.f, top = -INFINITY;
#pragma unroll
        for (int s0 = 0; s0 < kChunkSegments; s0 += kBatch) {
            if (s0 >= segs) break;
            float4 u[kBatch], v[kBatch];
#pragma unroll
            for (int s = 0; s < kBatch; ++s)
                if (s0 + s < segs) {
                    const float4* p = reinterpret_cast<const float4*>(part + (s0 + s) * HD);
                    u[s] = p[0];
                    v[s] = p[1];
                }
            if (s0 == 0)
#pragma unroll
                for (int s = 0; s < kChunkSegments; ++s) top = fmaxf(top, ml[s].x);
#pragma unroll
            for (int s = 0; s < kBatch; ++s)
                if (s0 + s < segs) {
                    // 1 where no segment has a score above -inf: sums are 0, or NaN where scores were
                    const float f = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[s0 + s].x - top);
                    den += f * ml[s0 + s].y;
                    const float y[8] = {u[s].x, u[s].y, u[s].z, u[s].w, v[s].x, v[s].y, v[s].z, v[s].w};
#pragma unroll
                    for (int e = 0; e < 8; ++e) num[e] += f * y[e];
                }
        }
        const float inv = den == 0.f ? 0.f : 1.f / den;
        u32x4 out;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = pack_bf16(num[2 * e] * inv, num[2 * e + 1] * inv);
        *reinterpret_cast<u32x4*>(chunk_out(a, row, i * 8, d)) = out;
    }
}

template <int HD>
static void launch_hd(const ChunkAttnArgs& a, bool split, int groups, hipStream_t st) {
    if (!split)
        k_chunk_attn<HD, false, 2><<<groups, 256, 0, st>>>(a);
    else if (HD == 128 && a.ch.n_rows / kLongChunk >= a.ch.n_chunks)
        k_chunk_attn<HD, true, HD == 128 ? 1 : 2><<<groups, 256, 0, st>>>(a);
    else
        k_chunk_attn<HD, true, 2><<<groups, 256, 0, st>>>(a);
    if (a.split.most > 1) k_chunk_merge<HD><<<a.ch.n_rows, 256, 0, st>>>(a);
}

hipError_t launch_chunk_attention(const cdb_chunks& ch, const KvTarget& kv, const void* q, int q_type, int H, int hd,
                                  void* scratch, uint16_t* out, int order, int* err, hipStream_t st) {
    if (ch.n_chunks <= 0 || ch.n_rows <= 0) return hipSuccess;
    ChunkAttnArgs a{};
    a.ch = ch;
    a.kv = kv;
    a.q = q;
    a.out = out;
    a.order = order;
    a.H = H;
    a.xcd_heads = (H + 7) / 8 * 8 * 8 <= H * 9 ? (H + 7) / 8 : 0;
    a.split = chunk_split(H, ch.n_chunks, ch.n_rows, kv.max_pages);
    a.part = static_cast<float*>(scratch);
    a.ml = reinterpret_cast<float2*>(a.part + (size_t)ch.n_rows * H * a.split.most * hd);
    a.err = err;
    // every chunk has one tile that is not full at most
    const int tiles = std::min(ch.n_chunks, ch.n_rows) + ch.n_rows / kTileRows;
    const int groups = (a.xcd_heads ? a.xcd_heads * 8 : H) * tiles * a.split.most;
    switch (hd) {
        case 64: launch_hd<64>(a, q_type == CDB_F32, groups, st); break;
        case 96: launch_hd<96>(a, q_type == CDB_F32, groups, st); break;
        case 128: launch_hd<128>(a, q_type == CDB_F32, groups, st); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace cdb
