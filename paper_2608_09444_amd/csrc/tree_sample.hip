// Sampled acceptance of drafted trees from given random numbers.
//
// r_0 = p, the target's probabilities after a node, q the drafter's.  A child with token x is
// accepted if u q(x) < r_k(x); if not, r_{k+1} = max(r_k - q, 0) / Z_{k+1} stands for its next sibling, and
// at the end for the token that follows.  Without a drafter's probabilities q is 1 at the child's token.
// Probabilities and sums are in 64 bits: which token's interval of the cumulated
// probabilities holds u is decided at borders that lie 1e-5 to 1e-12 apart.
#include <algorithm>

#include "cdb_internal.h"

namespace cdb {

constexpr int kPiece = 4096;  // logits of a workgroup's part of a row, 16 to each of its 256 threads

struct SampleArgs {
    cdb_drafts dr;
    const int32_t* row0;
    const int32_t* first_ids;
    cdb_sampling sm;
    cdb_accepted out;
    int n_rows, V, pieces;
    double2* stats;  // [target, drafter][n_rows][pieces] maximum, sum of exp((l - maximum) / temperature)
    double* rest;    // [trees][pieces] what the first rejection leaves of a piece
    int* arrive;     // [trees] pieces of it that are summed, 0 between launches
    int* err;
};

static int sample_pieces(const cdb_model_desc& d) { return (d.vocab + kPiece - 1) / kPiece; }
size_t tree_sample_bytes(const cdb_model_desc& d, int rows) {
    return ((size_t)2 * rows * sizeof(double2) + CDB_TREE_MAX_TREES * sizeof(double)) * sample_pieces(d) +
           CDB_TREE_MAX_TREES * sizeof(int);
}

// 2^y for y <= 0 (or a little above): 2^n 2^f with f in [-1/2, 1/2], the latter by its Taylor
// series, whose rest is below (ln 2 / 2)^11 / 11! = 2.2e-13.
__device__ __forceinline__ double exp2_64(double y) {
    y = fmax(y, -1100.0);
    const double n = rint(y), f = y - n;
    double p = 7.0549116208011209e-09;  // ln(2)^k / k!, k = 10 .. 0
    p = fma(p, f, 1.0178086009239696e-07);
    p = fma(p, f, 1.3215486790144305e-06);
    p = fma(p, f, 1.5252733804059838e-05);
    p = fma(p, f, 1.5403530393381606e-04);
    p = fma(p, f, 1.3333558146428441e-03);
    p = fma(p, f, 9.6181291076284769e-03);
    p = fma(p, f, 5.5504108664821576e-02);
    p = fma(p, f, 2.4022650695910069e-01);
    p = fma(p, f, 6.9314718055994529e-01);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n);
}
constexpr double kLog2e = 1.4426950408889634;

__device__ __forceinline__ bool tree_len_ok(int l) { return l >= 0 && l <= 0x7fffffff - CDB_TREE_MAX_NODES; }

// Whether cdb_tree_rows gave tree t no rows because of its sequence or length.  By one thread.
__device__ __forceinline__ bool tree_refused(const cdb_drafts& dr, int t) {
    if (!dr.seq) return false;
    const int sq = dr.seq[t];
    if (sq < 0 || sq >= dr.max_seqs) return true;
    for (int k = 0; k < t; ++k)
        if (dr.seq[k] == sq) return true;
    return dr.len && !tree_len_ok(dr.len[sq]);
}

__device__ __forceinline__ bool temperature_ok(float t) { return t > 0.f && t < INFINITY; }

__device__ __forceinline__ float4 logits4(const float* row, int i, int V) {
    return i < V ? *reinterpret_cast<const float4*>(row + i) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
}

template <typename T, typename F>
__device__ __forceinline__ T wave_all(T v, F f) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = f(v, __shfl_xor(v, o, 64));
    return v;
}

// Workgroup = (piece, row, target or drafter).
__global__ __launch_bounds__(256) void k_sample_stats(SampleArgs a) {
    __shared__ int s_found, s_tree, s_kids;
    __shared__ float s_max[4];
    __shared__ double s_sum[4];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int piece = blockIdx.x, row = blockIdx.y;
    const bool target = blockIdx.z == 0;
    const float* src = target ? a.sm.logits + (size_t)row * a.sm.logits_stride : a.sm.draft_logits + (size_t)row * a.sm.draft_stride;
    float4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = logits4(src, piece * kPiece + i * 1024 + tid * 4, a.V);
    if (tid == 0) s_found = s_kids = 0;
    if (piece + row + blockIdx.z == 0) a.arrive[tid] = 0;  // CDB_TREE_MAX_TREES = 256 of them
    __syncthreads();
    bool mine = false;
    int first = 0;
    if (tid < a.dr.n_trees) {
        first = a.row0[tid];
        const int n = a.dr.n_nodes[tid];
        mine = first >= 0 && n > 0 && n <= a.dr.max_nodes && row >= first && row < first + n;
    }
    if (mine) {
        s_tree = tid;
        atomicAdd(&s_found, 1);
    }
    __syncthreads();
    if (s_found == 0) return;
    if (s_found > 1) {  // a tree that was refused stands where the next one's rows begin
        if (mine && !tree_refused(a.dr, tid)) s_tree = tid;
        __syncthreads();
    }
    const int t = s_tree, node = row - a.row0[t];
    if (!target) {  // the drafter's probabilities count where there are children
        if (tid < a.dr.max_nodes && tid < a.dr.n_nodes[t] && a.dr.parent[(size_t)t * a.dr.max_nodes + tid] == node) s_kids = 1;
        __syncthreads();
        if (!s_kids) return;
    }
    const float* temps = target ? a.sm.temperature : a.sm.draft_temperature;
    const double scale = temps ? kLog2e / (double)temps[t] : kLog2e;
    float m = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m = fmaxf(fmaxf(fmaxf(m, x[i].x), fmaxf(x[i].y, x[i].z)), x[i].w);
        nan |= x[i].x != x[i].x || x[i].y != x[i].y || x[i].z != x[i].z || x[i].w != x[i].w;
    }
    m = wave_all(m, [](float p, float q) { return fmaxf(p, q); });
    if (lane == 0) s_max[w] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    double s = nan || m == INFINITY ? NAN : 0.0;
    if (m > -INFINITY) {
        const double mc = -scale * m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s += exp2_64(fma((double)x[i].x, scale, mc)) + exp2_64(fma((double)x[i].y, scale, mc));
            s += exp2_64(fma((double)x[i].z, scale, mc)) + exp2_64(fma((double)x[i].w, scale, mc));
        }
    }
    s = wave_all(s, [](double p, double q) { return p + q; });
    if (lane == 0) s_sum[w] = s;
    __syncthreads();
    if (tid == 0)
        a.stats[((size_t)(target ? 0 : a.n_rows) + row) * a.pieces + piece] = make_double2(m, s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]);
}

// One workgroup per tree, or, for a drafter's probabilities, per (piece, tree).  Wave 0 walks (lane = node).  All
// workgroups of a tree walk alike up to its first rejection; each then sums what that leaves of its own
// piece, and the one that is through last has all sums and goes on alone.
__global__ __launch_bounds__(256) void k_sample_walk(SampleArgs a) {
    extern __shared__ double s_sum[];  // [pieces] what is left of the target's probabilities at the current node
    __shared__ double s_m[2][CDB_TREE_MAX_NODES], s_inv[2][CDB_TREE_MAX_NODES];  // each node's maximum x scale, 1 / sum
    __shared__ double s_z[CDB_TREE_MAX_NODES + 1];  // 1 / Z_k after k rejections at the current node
    __shared__ double s_red[4];
    __shared__ int s_out[CDB_TREE_MAX_NODES];  // the tokens of the rejections
    __shared__ int s_par[CDB_TREE_MAX_NODES];
    __shared__ int s_cur, s_k, s_todo, s_pick[4];
    const int t = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const bool dense = a.sm.draft_logits != nullptr;
    const float temp = a.sm.temperature ? a.sm.temperature[t] : 1.f;
    const float dtemp = dense && a.sm.draft_temperature ? a.sm.draft_temperature[t] : 1.f;
    const double scale[2] = {kLog2e / (double)temp, kLog2e / (double)dtemp};
    const int r0 = a.row0[t], N = a.dr.max_nodes;
    const bool tells = blockIdx.x == 0;
    // the nodes, in every wave
    int n = a.dr.n_nodes[t];
    if (n < 0 || n > N) n = 0;
    const size_t at = (size_t)t * N + lane;
    int par = lane < n ? a.dr.parent[at] : -2;
    const int token = lane < n ? a.dr.tokens[at] : 0;
    const double u = lane < n ? a.sm.u_node[at] : 0.0;
    int next = a.first_ids[t];
    bool live = lane < n && r0 >= 0;
    if (n > 0) {
        bool refused = false;
        if (a.dr.seq) {
            const int s = a.dr.seq[t];
            for (int i = lane; i < t; i += 64) refused |= a.dr.seq[i] == s;
            refused |= s < 0 || s >= a.dr.max_seqs;
            if (a.dr.len && !__any(refused)) refused = !tree_len_ok(a.dr.len[s]);
        }
        refused = __any(refused);
        const bool cold = !temperature_ok(temp) || !temperature_ok(dtemp);
        if (refused || cold) {
            if (tells && tid == 0) set_err(a.err, refused ? CDB_DEV_BAD_INDEX : CDB_DEV_BAD_VALUE);
            live = false;
        }
    }
    if (live && r0 > a.n_rows - 1 - lane) {
        if (tells && w == 0) set_err(a.err, CDB_DEV_BAD_INDEX);
        live = false;
    }
    live = live && par < lane;
    if (live && par >= 0 && (token < 0 || token >= a.V)) {
        if (tells && w == 0) set_err(a.err, CDB_DEV_BAD_INDEX);
        live = false;
    }
    if (!live) par = -2;
    const uint64_t lives = __ballot(live);
    if (w == 0) s_par[lane] = par;
    __syncthreads();
    // statistics of the nodes' rows: four threads to a node
    {
        const int node = tid >> 2, sub = tid & 3;
        const bool here = lives >> node & 1;
        bool kids = false;
        if (here && dense)
            for (int j = node + 1; j < n; ++j) kids |= s_par[j] == node;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            double m = -INFINITY, sum = 0.0;
            if (here && (z == 0 || kids)) {
                const double2* st = a.stats + ((size_t)(z ? a.n_rows : 0) + r0 + node) * a.pieces;
#pragma unroll 4
                for (int i = sub; i < a.pieces; i += 4) m = fmax(m, st[i].x);
                m = fmax(m, __shfl_xor(m, 1, 64));
                m = fmax(m, __shfl_xor(m, 2, 64));
#pragma unroll 4
                for (int i = sub; i < a.pieces; i += 4) {
                    const double2 x = st[i];  // of a piece of nothing but -inf (or NaN): 0 (or NaN)
                    sum += x.x > -INFINITY ? x.y * exp2_64((x.x - m) * scale[z]) : x.y;
                }
                sum += __shfl_xor(sum, 1, 64);
                sum += __shfl_xor(sum, 2, 64);
            }
            if (sub == 0) {
                s_m[z][node] = m * scale[z];
                s_inv[z][node] = m < INFINITY ? 1.0 / sum : NAN;  // NaN or infinite: no distribution
            }
        }
    }
    __syncthreads();
    // what is left of the target's probability of token i after k rejections at the current node
    auto left = [&](float lp, float lq, int i, int cur, int k) {
        double r = exp2_64(fma((double)lp, scale[0], -s_m[0][cur])) * s_inv[0][cur];
        if (dense) {
            if (k) {
                const double q = exp2_64(fma((double)lq, scale[1], -s_m[1][cur])) * s_inv[1][cur];
                for (int s = 1; s < k; ++s) r = fmax(r - q, 0.0) * s_z[s];
                r = fmax(r - q, 0.0);
            }
        } else {
            for (int s = 0; s < k; ++s) r = i == s_out[s] ? 0.0 : r;
        }
        return r;
    };
    auto target_row = [&](int cur) { return a.sm.logits + (size_t)(r0 + cur) * a.sm.logits_stride; };
    auto draft_row = [&](int cur) { return a.sm.draft_logits + (size_t)(r0 + cur) * a.sm.draft_stride; };
    // a piece's sum, in s_red[0] for all; by the whole workgroup
    auto piece_sum = [&](int piece, int cur, int k) {
        double s = 0.0;
        float4 x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = piece * kPiece + i * 1024 + tid * 4;
            x[i] = logits4(target_row(cur), e, a.V);
            y[i] = dense && k ? logits4(draft_row(cur), e, a.V) : x[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = piece * kPiece + i * 1024 + tid * 4;
            s += left(x[i].x, y[i].x, e, cur, k) + left(x[i].y, y[i].y, e + 1, cur, k);
            s += left(x[i].z, y[i].z, e + 2, cur, k) + left(x[i].w, y[i].w, e + 3, cur, k);
        }
        s = wave_all(s, [](double p, double q) { return p + q; });
        __syncthreads();
        if (lane == 0) s_red[w] = s;
        __syncthreads();
        return s_red[0] + s_red[1] + s_red[2] + s_red[3];
    };

    // this node's token after its parent (wave 0)
    double pj = 0.0, qj = 1.0;
    bool bad = false;
    if (w == 0) {
        if (live && par >= 0) {
            const float lp = target_row(par)[token], lq = dense ? draft_row(par)[token] : 0.f;
            pj = exp2_64(fma((double)lp, scale[0], -s_m[0][par])) * s_inv[0][par];
            if (dense) qj = exp2_64(fma((double)lq, scale[1], -s_m[1][par])) * s_inv[1][par];
        }
    }
    int path = -1, count = 0, cur = -1, tried = -1, k = 0;
    bool alone = !dense;
    for (;;) {
        // the walk needs sums after a rejection (1), or a token (2), or is over (3)
        if (w == 0) {
            int todo = 0;
            while (!todo) {
                const uint64_t kids = __ballot(par == cur && lane > tried && live);
                if (cur >= 0 && (!(s_inv[0][cur] < INFINITY) || (dense && kids && !(s_inv[1][cur] < INFINITY)))) {
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
                bool yes;
                if (cur < 0) {
                    yes = __shfl(token, j, 64) == next;
                } else {
                    double r = pj;
                    if (dense) {
                        for (int s = 1; s <= k; ++s) r = fmax(r - qj, 0.0) * s_z[s];
                    } else {
                        for (int s = 0; s < k; ++s) r = s_out[s] == token ? 0.0 : r;
                        if (k) r *= s_z[k];
                    }
                    yes = __shfl((int)(u * qj < r), j, 64);
                }
                if (yes) {
                    if (lane == count) path = j;
                    ++count;
                    cur = j;
                    k = 0;
                } else if (cur >= 0) {
                    const int x = __shfl(token, j, 64);
                    if (lane == 0) s_out[k] = x;
                    ++k;
                    todo = 1;
                }
            }
            if (lane == 0) {
                s_cur = cur;
                s_k = k;
                s_todo = todo;
            }
        }
        __syncthreads();
        const int todo = s_todo, c = s_cur;
        int kk = s_k;
        if (todo != 1 && !alone) {  // no rejection so far: every workgroup of the tree knows the same
            if (!tells) return;
            alone = true;
        }
        if (todo == 3) break;
        // sums at a node that nothing was rejected at, from the statistics
        auto fresh = [&]() {
            for (int i = tid; i < a.pieces; i += 256) {
                const double2 x = a.stats[(size_t)(r0 + c) * a.pieces + i];
                s_sum[i] = x.x > -INFINITY ? x.y * exp2_64(fma(x.x, scale[0], -s_m[0][c])) * s_inv[0][c] : 0.0;
            }
            __syncthreads();
        };
        auto total = [&]() {  // every thread's own, in order
            double z = 0.0;
            for (int i = 0; i < a.pieces; ++i) z += s_sum[i];
            return z;
        };
        if (todo == 2) {
            if (kk == 0) fresh();
            break;
        }
        double z;
        if (dense && !alone) {
            const double own = piece_sum(blockIdx.x, c, kk);
            if (tid == 0) {
                __hip_atomic_store(a.rest + (size_t)t * a.pieces + blockIdx.x, own, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_pick[0] = __hip_atomic_fetch_add(a.arrive + t, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (s_pick[0] != a.pieces - 1) return;
            alone = true;
            for (int i = tid; i < a.pieces; i += 256)
                s_sum[i] = __hip_atomic_load(a.rest + (size_t)t * a.pieces + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
        } else if (dense) {
            for (int i = 0; i < a.pieces; ++i) {
                const double own = piece_sum(i, c, kk);
                if (tid == 0) s_sum[i] = own;
            }
            __syncthreads();
        } else {  // a piece without the rejected token
            if (kk == 1) fresh();
            const int i = s_out[kk - 1] / kPiece;
            const double own = piece_sum(i, c, kk);
            if (tid == 0) s_sum[i] = own;
            __syncthreads();
        }
        z = total();
        __syncthreads();
        if (!(z > 0.0)) {  // nothing is left: the rejection does not count
            --kk;
            if (kk == 0) {
                fresh();
            } else if (dense) {
                for (int i = 0; i < a.pieces; ++i) {
                    const double own = piece_sum(i, c, kk);
                    if (tid == 0) s_sum[i] = own;
                }
                __syncthreads();
            } else {
                const int i = s_out[kk] / kPiece;
                const double own = piece_sum(i, c, kk);
                if (tid == 0) s_sum[i] = own;
                __syncthreads();
            }
        } else if (tid == 0) {
            s_z[kk] = 1.0 / z;
        }
        k = kk;
        if (tid == 0) s_k = kk;
        __syncthreads();
    }
    if (s_todo == 2) {
        // the piece in which the cumulated sum passes u_next, then the logit
        const int c = s_cur, kk = s_k;
        double aim = 0.0;
        for (int i = 0; i < a.pieces; ++i) aim += s_sum[i];
        aim *= (double)a.sm.u_next[t];
        double before = 0.0, start = 0.0;
        int piece = -1;
        for (int i = 0; i < a.pieces; ++i) {
            const double own = s_sum[i];
            if (own > 0.0) {
                piece = i;
                start = before;
                if (before + own > aim) break;
            }
            before += own;
        }  // none (u_next is 1 to rounding): the last one with anything
        piece = piece < 0 ? 0 : piece;
        const int e = piece * kPiece + tid * 16;
        double r[16], own = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 x = logits4(target_row(c), e + i * 4, a.V), y = dense && kk ? logits4(draft_row(c), e + i * 4, a.V) : x;
            r[i * 4] = left(x.x, y.x, e + i * 4, c, kk);
            r[i * 4 + 1] = left(x.y, y.y, e + i * 4 + 1, c, kk);
            r[i * 4 + 2] = left(x.z, y.z, e + i * 4 + 2, c, kk);
            r[i * 4 + 3] = left(x.w, y.w, e + i * 4 + 3, c, kk);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) own += r[i];
        double v = own;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double x = __shfl_up(v, o, 64);
            if (lane >= o) v += x;
        }
        if (lane == 63) s_red[w] = v;
        __syncthreads();
        double run = start;
        for (int i = 0; i < w; ++i) run += s_red[i];
        run += v - own;
        int pick = 0x7fffffff, last = -1;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            run += r[i];
            if (r[i] > 0.0) {
                last = e + i;
                if (run > aim && pick == 0x7fffffff) pick = e + i;
            }
        }
        pick = wave_all(pick, [](int p, int q) { return min(p, q); });
        last = wave_all(last, [](int p, int q) { return max(p, q); });
        if (lane == 0) s_pick[w] = pick;
        __syncthreads();
        pick = min(min(s_pick[0], s_pick[1]), min(s_pick[2], s_pick[3]));
        __syncthreads();
        if (lane == 0) s_pick[w] = last;
        __syncthreads();
        last = max(max(s_pick[0], s_pick[1]), max(s_pick[2], s_pick[3]));
        next = pick != 0x7fffffff ? pick : last < 0 ? 0 : last;
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
    a.arrive = reinterpret_cast<int*>(a.rest + (size_t)CDB_TREE_MAX_TREES * a.pieces);
    a.err = err;
    if (n_rows > 0) k_sample_stats<<<dim3(a.pieces, n_rows, sm.draft_logits ? 2 : 1), 256, 0, st>>>(a);
    const int split = sm.draft_logits ? a.pieces : 1;
    k_sample_walk<<<dim3(split, d.n_trees), 256, a.pieces * sizeof(double), st>>>(a);
    return hipGetLastError();
}

}  // namespace cdb
