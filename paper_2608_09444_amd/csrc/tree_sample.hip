// Sampled acceptance of drafted trees from given random numbers.
//
// r_0 = p, the target's probabilities after a node, q the drafter's.  A child with token x is
// accepted if u q(x) < r_k(x); if not, r_{k+1} = max(r_k - q, 0) / Z_{k+1} stands for its next sibling, and
// at the end for the token that follows.  Without a drafter's probabilities q is 1 at the child's token.
// Probabilities and sums are in 64 bits: which token's interval of the cumulated
// probabilities holds u is decided at borders that lie 1e-5 to 1e-12 apart.
//
// Bound: every row of logits once (the drafter's only where a node has children), 14 64-bit
// operations for each, about 0.5 us of them for 10^6; then a chain per tree.  A rejection's Z needs the whole
// vocabulary and the next one needs Z, so sums cannot be taken ahead: k_sample_walk joins as many workgroups
// as a row has pieces for the first ones.  Nothing of the probabilities is stored, 2^x is cheaper
// than reading it back.
// Measured (statistics + walk, us): 64 trees of 4, 49152 tokens 26 + 25; 4 trees of 32-64, 65536 tokens
// 25 + 2 x 21-22; 20 trees of 5-9, a sure drafter 9-9.5 + 14.5; one tree of 13 4.8 + 2 x 7.2-7.4.
#include <algorithm>

#include "cdb_internal.h"

namespace cdb {

constexpr int kPiece = 4096;  // logits of a workgroup's part of a row, 16 to each of its 256 threads
// Most launches of k_sample_walk.  Each takes one rejection's sum with all pieces' workgroups, and one workgroup takes
// those that follow in the last (17 us each of 65536 tokens).  A second one costs 1.4 us where nobody needs it (one tree of 13
// nodes: 17.6 against 16.2), and saves 18 of 83 us with 4 trees of 32-64; trees of at most 4 nodes rarely
// have two rejections in a row (64 trees of 4: 51.3 with it, 50.0 without).
constexpr int kRounds = 2;
constexpr int kTrees = CDB_TREE_MAX_TREES;

struct SampleArgs {
    cdb_drafts dr;
    const int32_t* row0;
    const int32_t* first_ids;
    cdb_sampling sm;
    cdb_accepted out;
    int n_rows, V, pieces;
    double2* stats;  // [target, drafter][n_rows][pieces] maximum, sum of exp((l - maximum) / temperature)
    double* rest;    // [trees][pieces] what a rejection leaves of a piece
    double* left;    // [kRounds][trees] and of all pieces
    int* arrive;     // [kRounds][trees] pieces that are summed
    int* done;       // [trees] whether the walk is over
    int round, rounds;
    int* err;
};

static int sample_pieces(const cdb_model_desc& d) { return (d.vocab + kPiece - 1) / kPiece; }
size_t tree_sample_bytes(const cdb_model_desc& d, int rows) {
    const size_t doubles = ((size_t)4 * rows + kTrees) * sample_pieces(d) + kTrees * kRounds;
    return doubles * 8 + (size_t)kTrees * (kRounds + 1) * 4;
}

// By its bits: a ballot of x < INFINITY was compiled to one that a NaN passes.
__device__ __forceinline__ bool is_finite(double x) { return (__double2hiint(x) & 0x7ff00000) != 0x7ff00000; }

// 2^y for y <= 0 (or a little above): 2^n 2^f with f in [-1/2, 1/2], the latter by the polynomial that meets it at the
// nine Chebyshev points, within 1.1e-12 of the value everywhere.  Adding 1.5 x 2^52 leaves y's nearest
// whole number in the low word; below -1000 the result is 0, or, without EXACT, 2^-1000.
template <bool EXACT = true>
__device__ __forceinline__ double exp2_64(double y) {
    constexpr double kRound = 6755399441055744.0;
    const double v = EXACT ? y : fmax(y, -1000.0), t = v + kRound, f = v - (t - kRound);
    double p = 1.3255224878668817e-06;
    p = fma(p, f, 1.5310079402249296e-05);
    p = fma(p, f, 1.5403455852453838e-04);
    p = fma(p, f, 1.3333450568000645e-03);
    p = fma(p, f, 9.6181291594025584e-03);
    p = fma(p, f, 5.5504109412059327e-02);
    p = fma(p, f, 2.4022650695812989e-01);
    p = fma(p, f, 6.9314718054593349e-01);
    p = fma(p, f, 1.0);
    const double r = __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
    return EXACT && !(y >= -1000.0) ? 0.0 : r;
}
// With the denormal results too: a drafted token of the smallest probability is still a possible one.
__device__ __forceinline__ double exp2_64_tail(double y) {
    return y < -900.0 ? exp2_64(y + 200.0) * 0x1p-200 : exp2_64(y);
}
constexpr double kLog2e = 1.4426950408889634;

__device__ __forceinline__ bool tree_len_ok(int l) { return l >= 0 && l <= 0x7fffffff - CDB_TREE_MAX_NODES; }

__device__ __forceinline__ bool temperature_ok(float t) { return t > 0.f && t < INFINITY; }

__device__ __forceinline__ float4 logits4(const float* row, int i, int V) {
    return i < V ? *reinterpret_cast<const float4*>(row + i) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
}

// Lane exchanges of 64-bit values by data-parallel moves, which take a tenth of the time of shuffles through LDS.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double dpp64(double x) {  // lanes without a source read 0
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, ROWS, 0xf, true);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, ROWS, 0xf, true);
    return __hiloint2double(hi, lo);
}
// Sum over the wave, the same in every lane.
__device__ __forceinline__ double wave_sum(double x) {
    x += dpp64<0xb1>(x);   // lanes of a pair
    x += dpp64<0x4e>(x);   // pairs of a quad
    x += dpp64<0x141>(x);  // quads of 8 (mirrored)
    x += dpp64<0x140>(x);  // halves of 16 (mirrored)
    auto lo = __builtin_amdgcn_permlane16_swap(__double2loint(x), __double2loint(x), false, false);
    auto hi = __builtin_amdgcn_permlane16_swap(__double2hiint(x), __double2hiint(x), false, false);
    x = __hiloint2double(hi[0], lo[0]) + __hiloint2double(hi[1], lo[1]);
    lo = __builtin_amdgcn_permlane32_swap(__double2loint(x), __double2loint(x), false, false);
    hi = __builtin_amdgcn_permlane32_swap(__double2hiint(x), __double2hiint(x), false, false);
    return __hiloint2double(hi[0], lo[0]) + __hiloint2double(hi[1], lo[1]);
}
// Sums over the lanes up to this one.
__device__ __forceinline__ double wave_scan(double x) {
    x += dpp64<0x111>(x);  // from 1, 2, 4 and 8 lanes below in 16
    x += dpp64<0x112>(x);
    x += dpp64<0x114>(x);
    x += dpp64<0x118>(x);
    x += dpp64<0x142, 0xa>(x);  // the last lane of 16 to the next 16
    x += dpp64<0x143, 0xc>(x);  // lane 31 to the upper half
    return x;
}
template <int CTRL>
__device__ __forceinline__ float dpp32(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, dpp32<0xb1>(x));
    x = fmaxf(x, dpp32<0x4e>(x));
    x = fmaxf(x, dpp32<0x141>(x));
    x = fmaxf(x, dpp32<0x140>(x));
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Maxima and sums of the pieces of every row that a tree has; of the drafter's rows those of nodes with children,
// which are known before their logits are read.  Workgroup = (piece, row, target or drafter): 16 logits to a thread, in
// four loads at once.  26 us for 448 rows of 49152 (3.4 TB/s): the 64-bit operations take about 10 of it, and
// loads, maximum, powers and sum follow one another in each workgroup; a loop over
// pieces with the next one's loads ahead took 32 us, 1024 threads a workgroup 36.
__global__ __launch_bounds__(256) void k_sample_stats(SampleArgs a) {
    __shared__ int s_tree, s_kids;
    __shared__ float s_max[4];
    __shared__ double s_sum[4];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int piece = blockIdx.x, row = blockIdx.y;
    const bool target = blockIdx.z == 0;
    const float* src = target ? a.sm.logits + (size_t)row * a.sm.logits_stride : a.sm.draft_logits + (size_t)row * a.sm.draft_stride;
    float4 x[4];
    auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = logits4(src, piece * kPiece + i * 1024 + tid * 4, a.V);
    };
    if (target) fetch();
    if (tid == 0) {
        s_tree = -1;
        s_kids = 0;
    }
    if (piece + row + blockIdx.z == 0)  // for the launches of k_sample_walk
        for (int i = tid; i < kTrees * (kRounds + 1); i += 256) a.arrive[i] = 0;
    __syncthreads();
    if (tid < a.dr.n_trees) {
        const int first = a.row0[tid], n = a.dr.n_nodes[tid];
        // a tree that was refused stands where rows of later trees begin
        if (first >= 0 && n > 0 && n <= a.dr.max_nodes && row >= first && row < first + n) atomicMax(&s_tree, tid);
    }
    __syncthreads();
    const int t = s_tree;
    if (t < 0) return;
    if (!target) {
        const int node = row - a.row0[t];
        if (tid < a.dr.max_nodes && tid < a.dr.n_nodes[t] && a.dr.parent[(size_t)t * a.dr.max_nodes + tid] == node) s_kids = 1;
        __syncthreads();
        if (!s_kids) return;
        fetch();
    }
    const float* temps = target ? a.sm.temperature : a.sm.draft_temperature;
    const double scale = temps ? kLog2e / (double)temps[t] : kLog2e;
    float m = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m = fmaxf(fmaxf(fmaxf(m, x[i].x), fmaxf(x[i].y, x[i].z)), x[i].w);
        nan |= __builtin_isunordered(x[i].x, x[i].y) || __builtin_isunordered(x[i].z, x[i].w);
    }
    m = wave_max(m);
    if (lane == 0) s_max[w] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    double s = nan || m == INFINITY ? NAN : 0.0;
    if (m > -INFINITY) {
        // The difference first: the product of a mask's lowest value, or of a low temperature, is rounded in its whole places.
        const double top = m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s += exp2_64<false>(((double)x[i].x - top) * scale) + exp2_64<false>(((double)x[i].y - top) * scale);
            s += exp2_64<false>(((double)x[i].z - top) * scale) + exp2_64<false>(((double)x[i].w - top) * scale);
        }
    }
    s = wave_sum(s);
    if (lane == 0) s_sum[w] = s;
    __syncthreads();
    if (tid == 0)
        a.stats[((size_t)(target ? 0 : a.n_rows) + row) * a.pieces + piece] = make_double2(m, s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]);
}

// One workgroup per tree, or, for a drafter's probabilities, per (piece, tree).  Wave 0 walks (lane = node), up to
// the first rejection whose sum is not known yet, the round-th one; each workgroup then sums what that leaves of its
// own piece, and the one that is through last has all sums and walks on alone.  Where that meets
// another rejection, it leaves it to the next round, or, in the last one, sums by itself.
__global__ __launch_bounds__(256, 3) void k_sample_walk(SampleArgs a) {
    extern __shared__ double s_sum[];  // [pieces] what is left of the target's probabilities at the current node
    double* s_part = s_sum + a.pieces; // [pieces][4] the waves' parts
    __shared__ double s_m[2][CDB_TREE_MAX_NODES], s_inv[2][CDB_TREE_MAX_NODES];  // each node's maximum, 1 / sum
    __shared__ double s_z[CDB_TREE_MAX_NODES + 1];  // 1 / Z_k after k rejections at the current node
    __shared__ double s_seg[16];
    __shared__ int s_out[CDB_TREE_MAX_NODES];       // the tokens of the rejections
    __shared__ double s_drop[CDB_TREE_MAX_NODES];   // and, of a sure drafter, what each took out of r
    __shared__ int s_exact;                         // whether s_sum is what the last of them left
    __shared__ int s_kid[CDB_TREE_MAX_NODES];  // whether the node has children
    __shared__ int s_cur, s_k, s_todo, s_pick[1];
    const int t = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    if (a.round > 0 && a.done[t]) return;
    const bool dense = a.sm.draft_logits != nullptr, tells = blockIdx.x == 0;
    const int N = a.dr.max_nodes;
    const size_t at = (size_t)t * N + lane;
    // all that does not depend on another load
    const int r0 = a.row0[t];
    int n = a.dr.n_nodes[t], next = a.first_ids[t];
    const float temp = a.sm.temperature ? a.sm.temperature[t] : 1.f;
    const float dtemp = dense && a.sm.draft_temperature ? a.sm.draft_temperature[t] : 1.f;
    const float un = a.sm.u_next[t];
    int par = lane < N ? a.dr.parent[at] : -2, token = lane < N ? a.dr.tokens[at] : 0;
    const double u = lane < N ? a.sm.u_node[at] : 0.f;
    bool refused = false;
    if (a.dr.seq) {
        const int sq = a.dr.seq[t];
        for (int i = lane; i < t; i += 64) refused |= a.dr.seq[i] == sq;
        refused |= sq < 0 || sq >= a.dr.max_seqs;
        if (a.dr.len && !__any(refused)) refused = !tree_len_ok(a.dr.len[sq]);
    }
    refused = __any(refused);
    const double scale[2] = {kLog2e / (double)temp, kLog2e / (double)dtemp};
    auto target_row = [&](int node) { return a.sm.logits + (size_t)(r0 + node) * a.sm.logits_stride; };
    auto draft_row = [&](int node) { return a.sm.draft_logits + (size_t)(r0 + node) * a.sm.draft_stride; };
    if (n < 0 || n > N) n = 0;
    bool live = lane < n && r0 >= 0;
    if (n > 0 && (refused || !temperature_ok(temp) || !temperature_ok(dtemp))) {
        if (tells && tid == 0) set_err(a.err, refused ? CDB_DEV_BAD_INDEX : CDB_DEV_BAD_VALUE);
        live = false;
    }
    if (live && r0 > a.n_rows - 1 - lane) {
        if (tells && w == 0) set_err(a.err, CDB_DEV_BAD_INDEX);
        live = false;
    }
    live = live && par < lane;
    if (live && (token < 0 || token >= a.V)) {
        if (tells && w == 0) set_err(a.err, CDB_DEV_BAD_INDEX);
        live = false;
    }
    if (!live) par = -2;
    float lp = 0.f, lq = 0.f;  // this node's token after its parent
    if (w == 0 && par >= 0) {
        lp = target_row(par)[token];
        if (dense) lq = draft_row(par)[token];
    }
    const uint64_t lives = __ballot(live);
    if (w == 0) {
        s_kid[lane] = 0;
        if (par >= 0) s_kid[par] = 1;
    }
    __syncthreads();
    {  // statistics of the nodes' rows: four threads to a node
        const int node = tid >> 2, sub = tid & 3;
        const bool here = lives >> node & 1;
        const bool has[2] = {here, here && dense && s_kid[node]};
        double m[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0, 0.0};
        for (int i0 = 0; i0 < a.pieces; i0 += 16) {
            double2 x[2][4];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const double2* st = a.stats + ((size_t)(z ? a.n_rows : 0) + r0 + node) * a.pieces;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int piece = i0 + i * 4 + sub;
                    x[z][i] = has[z] && piece < a.pieces ? st[piece] : make_double2(-INFINITY, 0.0);
                }
            }
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const double top = fmax(fmax(fmax(m[z], x[z][0].x), fmax(x[z][1].x, x[z][2].x)), x[z][3].x);
                // a piece of nothing but -inf has the sum 0, one with NaN the sum NaN
                if (i0 && m[z] > -INFINITY) sum[z] *= exp2_64((m[z] - top) * scale[z]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const double e = exp2_64((x[z][i].x - top) * scale[z]);
                    sum[z] += x[z][i].x > -INFINITY ? x[z][i].y * e : x[z][i].y;
                }
                m[z] = top;
            }
        }
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            double top = fmax(m[z], dpp64<0xb1>(m[z]));
            top = fmax(top, dpp64<0x4e>(top));
            const double e = exp2_64((m[z] - top) * scale[z]);
            if (m[z] > -INFINITY) sum[z] *= e;
            sum[z] += dpp64<0xb1>(sum[z]);
            sum[z] += dpp64<0x4e>(sum[z]);
            if (sub == 0) {
                s_m[z][node] = top;
                s_inv[z][node] = top < INFINITY ? 1.0 / sum[z] : NAN;  // NaN or infinite: no distribution
            }
        }
    }
    __syncthreads();
    double pj = 0.0, qj = 1.0;
    uint64_t good_p = 0, good_q = 0;
    if (w == 0) {
        const int from = max(par, 0);
        pj = exp2_64_tail(((double)lp - s_m[0][from]) * scale[0]) * s_inv[0][from];
        if (dense) qj = exp2_64_tail(((double)lq - s_m[1][from]) * scale[1]) * s_inv[1][from];
        good_p = __ballot(is_finite(s_inv[0][lane]));
        good_q = __ballot(!dense || is_finite(s_inv[1][lane]));
    }

    // What is left of the target's probabilities of tokens i .. i + 3 after k rejections at node cur.
    auto left4 = [&](float4 x, float4 y, int i, int cur, int k, double (&r)[4]) {
        const float p[4] = {x.x, x.y, x.z, x.w};
        const double m = s_m[0][cur], inv = s_inv[0][cur];
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = exp2_64(((double)p[j] - m) * scale[0]) * inv;
        if (dense && k) {
            const float d[4] = {y.x, y.y, y.z, y.w};
            const double mq = s_m[1][cur], invq = s_inv[1][cur];
            double q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = exp2_64(((double)d[j] - mq) * scale[1]) * invq;
            for (int s = 1; s < k; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = fmax(r[j] - q[j], 0.0) * s_z[s];
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = fmax(r[j] - q[j], 0.0);
        } else if (!dense) {
            for (int s = 0; s < k; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = i + j == s_out[s] ? 0.0 : r[j];
        }
    };
    // s_sum's total, the same bits in every thread
    auto total = [&]() {
        double z = 0.0;
        for (int i = lane; i < a.pieces; i += 64) z += s_sum[i];
        return wave_sum(z);
    };

    int path = -1, count = 0, cur = -1, tried = -1, k = 0, rejected = 0;
    double mass = 1.0;  // what a sure drafter's rejections left of p
    bool bad = false, alone = !dense, exact = dense;
    for (;;) {
        // the walk needs sums after a rejection (1), or a token (2), or is over (3)
        if (w == 0) {
            int todo = 0;
            while (!todo) {
                const uint64_t kids = __ballot(par == cur && lane > tried);
                if (cur >= 0 && (!(good_p >> cur & 1) || (kids && !(good_q >> cur & 1)))) {
                    bad = true;
                    todo = 3;
                    break;
                }
                if (!kids) {
                    todo = cur < 0 ? 3 : 2;
                    break;
                }
                const int j = __ffsll((unsigned long long)kids) - 1;
                tried = j;
                const int x = __builtin_amdgcn_readlane(token, j);
                bool yes;
                double r = pj;
                if (cur < 0) {
                    yes = x == next;
                } else {
                    if (dense) {
                        for (int s = 1; s <= k; ++s) r = fmax(r - qj, 0.0) * s_z[s];
                    } else {
                        for (int s = 0; s < k; ++s) r = s_out[s] == token ? 0.0 : r;
                    }
                    yes = __ballot(u * qj < (dense || !k ? r : r * s_z[k])) >> j & 1;
                }
                if (yes) {
                    if (lane == count) path = j;
                    ++count;
                    cur = j;
                    k = 0;
                    mass = 1.0;
                } else if (cur >= 0) {
                    if (lane == 0) s_out[k] = x;
                    ++k;
                    if (rejected < a.round) {  // an earlier round's
                        const double z = a.left[(size_t)rejected * kTrees + t];
                        if (!(z > 0.0))
                            --k;
                        else if (lane == 0)
                            s_z[k] = 1.0 / z;
                    } else if (dense) {
                        todo = 1;
                    } else {
                        const double gone = __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(r), j),
                                                             __builtin_amdgcn_readlane(__double2loint(r), j));
                        mass -= gone;
                        // Probabilities are within 1.1e-12 of their values, the difference within 2^-33 of its own as
                        // long as this much is left; else the rest is summed.
                        exact = mass < 1.0 / 64;
                        todo = exact;
                        if (lane == 0) {
                            s_drop[k - 1] = gone;
                            if (!exact) s_z[k] = 1.0 / mass;
                        }
                    }
                    ++rejected;
                }
            }
            if (lane == 0) {
                s_cur = cur;
                s_k = k;
                s_todo = todo;
                s_exact = exact;
            }
        }
        __syncthreads();
        const int todo = s_todo, c = s_cur;
        int kk = s_k;
        if (todo != 1 && !alone) {  // every workgroup of the tree came to the same
            if (!tells) return;
            alone = true;
        }
        if (todo == 3 || (todo == 2 && kk > 0 && s_exact)) break;  // the sums are there
        if (todo == 1 && dense && alone && a.round + 1 < a.rounds) return;  // the next round's
        const bool shared = todo == 1 && !alone;
        for (bool again = true; again;) {
            int from = 0, to = 0;
            if (todo == 1 && kk > 0) {
                if (shared && kk == s_k)
                    from = blockIdx.x, to = from + 1;
                else
                    to = a.pieces;
            }
            if (todo == 2 || kk == 0) {  // from the statistics
                for (int i = tid; i < a.pieces; i += 256) {
                    const double2 x = a.stats[(size_t)(r0 + c) * a.pieces + i];
                    s_sum[i] = x.x > -INFINITY ? x.y * exp2_64((x.x - s_m[0][c]) * scale[0]) * s_inv[0][c] : 0.0;
                }
                __syncthreads();
                if (kk > 0) {  // without the tokens that are out
                    if (tid == 0) {
                        bool thin = false;
                        for (int s = 0; s < kk; ++s) s_sum[s_out[s] / kPiece] -= s_drop[s];
                        for (int s = 0; s < kk; ++s) thin |= s_sum[s_out[s] / kPiece] < 1e-9;
                        s_exact = thin;
                    }
                    __syncthreads();
                    if (s_exact) to = a.pieces;  // what is left of a piece may be the rounding alone
                }
            }
            if (from < to) {
                const float *tp = target_row(c), *tq = dense ? draft_row(c) : tp;
                float4 p[4], q[4];  // the next four of 1024 logits each are on their way
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[i] = logits4(tp, from * kPiece + i * 1024 + tid * 4, a.V);
                    q[i] = logits4(tq, from * kPiece + i * 1024 + tid * 4, a.V);
                }
                for (int piece = from; piece < to; ++piece) {
                    double s = 0.0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int e = piece * kPiece + i * 1024 + tid * 4;
                        const float4 x = p[i], y = q[i];
                        if (piece + 1 < to) {
                            p[i] = logits4(tp, e + kPiece, a.V);
                            q[i] = logits4(tq, e + kPiece, a.V);
                        }
                        double r[4];
                        left4(x, y, e, c, kk, r);
                        s += (r[0] + r[1]) + (r[2] + r[3]);
                    }
                    s = wave_sum(s);
                    if (lane == 0) s_part[piece * 4 + w] = s;
                }
                __syncthreads();
                for (int i = from + tid; i < to; i += 256)
                    s_sum[i] = s_part[i * 4] + s_part[i * 4 + 1] + s_part[i * 4 + 2] + s_part[i * 4 + 3];
                __syncthreads();
                if (shared && kk == s_k) {
                    if (tid == 0) {
                        __hip_atomic_store(a.rest + (size_t)t * a.pieces + from, s_sum[from], __ATOMIC_RELAXED,
                                           __HIP_MEMORY_SCOPE_AGENT);
                        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the sum has reached memory
                        s_pick[0] = __hip_atomic_fetch_add(a.arrive + a.round * kTrees + t, 1, __ATOMIC_RELAXED,
                                                           __HIP_MEMORY_SCOPE_AGENT);
                    }
                    __syncthreads();
                    if (s_pick[0] != a.pieces - 1) return;
                    alone = true;
                    for (int i = tid; i < a.pieces; i += 256)
                        s_sum[i] = __hip_atomic_load(a.rest + (size_t)t * a.pieces + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    __syncthreads();
                }
            }
            again = false;
            if (todo == 1) mass = total();
            if (todo == 1 && kk == s_k) {
                const double z = mass;
                if (tid == 0 && a.round + 1 < a.rounds) a.left[(size_t)a.round * kTrees + t] = z;
                if (z > 0.0) {
                    if (tid == 0) s_z[kk] = 1.0 / z;
                } else {  // nothing is left: the rejection does not count, what was there before is summed again
                    --kk;
                    again = true;
                    __syncthreads();
                }
            }
        }
        if (todo == 2) break;
        k = kk;
        __syncthreads();
    }
    if (s_todo == 2) {
        // the piece in which the cumulated sum passes u_next, then the logit; u_next may be 1 to rounding: the last
        // one with anything
        const int c = s_cur, kk = s_k;
        const double aim = (double)un * total();
        double start = 0.0, before = 0.0;
        int piece = 0;
        for (int i0 = 0; i0 < a.pieces; i0 += 64) {
            const double own = i0 + lane < a.pieces ? s_sum[i0 + lane] : 0.0;
            const double v = wave_scan(own);
            const uint64_t hit = __ballot(before + v > aim && own > 0.0), some = __ballot(own > 0.0);
            if (some) {
                const int j = hit ? __ffsll((unsigned long long)hit) - 1 : 63 - __clzll((long long)some);
                piece = i0 + j;
                start = before + __shfl(v - own, j, 64);
                if (hit) break;
            }
            before += __shfl(v, 63, 64);
        }
        const float *tp = target_row(c), *tq = dense ? draft_row(c) : tp;
        float4 p[4], q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = logits4(tp, piece * kPiece + i * 1024 + tid * 4, a.V);
            q[i] = logits4(tq, piece * kPiece + i * 1024 + tid * 4, a.V);
        }
        double r[4][4], own[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            left4(p[i], q[i], piece * kPiece + i * 1024 + tid * 4, c, kk, r[i]);
            own[i] = (r[i][0] + r[i][1]) + (r[i][2] + r[i][3]);
            const double z = wave_sum(own[i]);
            if (lane == 0) s_seg[i * 4 + w] = z;  // 256 logits in a row
        }
        __syncthreads();
        // the segment, as the piece above; its wave looks for the logit
        int seg = 0;
        bool found = false;
        double from = start;
        before = start;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const double x = s_seg[i];
            if (x > 0.0 && !found) {
                seg = i;
                from = before;
                found = before + x > aim;
            }
            before += x;
        }
        if ((seg & 3) == w) {
            double x[4], mine = 0.0;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = 0.0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (seg >> 2 == i) {
                    mine = own[i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = r[i][j];
                }
            double run = from + (wave_scan(mine) - mine);
            const int e = piece * kPiece + seg * 256 + lane * 4;
            int pick = -1, last = -1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                run += x[j];
                if (x[j] > 0.0) {
                    last = e + j;
                    if (pick < 0 && run > aim) pick = e + j;
                }
            }
            const uint64_t hit = __ballot(pick >= 0), some = __ballot(last >= 0);
            if (hit)
                pick = __builtin_amdgcn_readlane(pick, __ffsll((unsigned long long)hit) - 1);
            else
                pick = some ? __builtin_amdgcn_readlane(last, 63 - __clzll((long long)some)) : 0;
            if (lane == 0) s_pick[0] = pick;
        }
        __syncthreads();
        next = s_pick[0];
    }
    if (w != 0) return;
    if (bad) {
        if (lane == 0) set_err(a.err, CDB_DEV_BAD_VALUE);
        next = -1;
    }
    if (lane < N) a.out.path[at] = path;
    if (lane == 0) {
        a.out.count[t] = count;
        a.out.next[t] = next;
        a.done[t] = 1;
    }
}

hipError_t launch_tree_sample(const cdb_model_desc& md, const cdb_drafts& d, const int32_t* row0, int n_rows,
                              const int32_t* first_ids, const cdb_sampling& sm, const cdb_accepted& out, void* scratch,
                              int* err, hipStream_t st) {
    if (d.n_trees <= 0) return hipSuccess;
    SampleArgs a{};
    a.dr = d;
    a.row0 = row0;
    a.first_ids = first_ids;
    a.sm = sm;
    a.out = out;
    a.n_rows = n_rows;
    a.V = md.vocab;
    a.pieces = sample_pieces(md);
    a.stats = static_cast<double2*>(scratch);
    a.rest = reinterpret_cast<double*>(a.stats + (size_t)2 * n_rows * a.pieces);
    a.left = a.rest + (size_t)kTrees * a.pieces;
    a.arrive = reinterpret_cast<int*>(a.left + kTrees * kRounds);
    a.done = a.arrive + kTrees * kRounds;
    a.err = err;
    a.rounds = sm.draft_logits && n_rows > 0 && d.max_nodes > 4 ? kRounds : 1;
    if (n_rows > 0) k_sample_stats<<<dim3(a.pieces, n_rows, sm.draft_logits ? 2 : 1), 256, 0, st>>>(a);
    const int split = sm.draft_logits ? a.pieces : 1;
    for (a.round = 0; a.round < a.rounds; ++a.round)
        k_sample_walk<<<dim3(split, d.n_trees), 256, 5 * a.pieces * sizeof(double), st>>>(a);
    return hipGetLastError();
}

}  // namespace cdb
