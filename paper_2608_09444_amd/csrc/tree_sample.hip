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

constexpr int kPiece = 4096;  // logits of a workgroup's part of a row
constexpr int kFinish = 1024; // threads that finish a tree

struct SampleArgs {
    cdb_drafts dr;
    const int32_t* row0;
    const int32_t* first_ids;
    cdb_sampling sm;
    cdb_accepted out;
    int n_rows, V, pieces;
    double2* stats;  // [target, drafter][n_rows][pieces] maximum, sum of exp((l - maximum) / temperature)
    int* err;
};

static size_t sample_stats_bytes(int rows, int V) { return (size_t)2 * rows * ((V + kPiece - 1) / kPiece) * sizeof(double2); }
size_t tree_sample_bytes(const cdb_model_desc& d, int rows) { return sample_stats_bytes(rows, d.vocab); }

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
    const double inv = temps ? 1.0 / (double)temps[t] : 1.0;
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(fmaxf(fmaxf(m, x[i].x), fmaxf(x[i].y, x[i].z)), x[i].w);
    m = wave_all(m, [](float p, float q) { return fmaxf(p, q); });
    if (lane == 0) s_max[w] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    double s = 0.0;
    if (m > -INFINITY)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s += exp(((double)x[i].x - m) * inv) + exp(((double)x[i].y - m) * inv);
            s += exp(((double)x[i].z - m) * inv) + exp(((double)x[i].w - m) * inv);
        }
    else  // nothing but -inf, or NaN
#pragma unroll
        for (int i = 0; i < 4; ++i) s += x[i].x != x[i].x || x[i].y != x[i].y || x[i].z != x[i].z || x[i].w != x[i].w ? NAN : 0.0;
    s = wave_all(s, [](double p, double q) { return p + q; });
    if (lane == 0) s_sum[w] = s;
    __syncthreads();
    if (tid == 0)
        a.stats[((size_t)(target ? 0 : a.n_rows) + row) * a.pieces + piece] = make_double2(m, s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]);
}

// A row's maximum and 1 / sum; 1 / sum is NaN or infinite where the row is no distribution.
struct RowStat {
    double m, inv;
};
__device__ __forceinline__ RowStat row_stat(const double2* s, int pieces, double inv_t) {
    double m = -INFINITY;
    for (int i = 0; i < pieces; ++i) m = fmax(m, s[i].x);
    double z = 0.0;
    for (int i = 0; i < pieces; ++i) z += s[i].y * (s[i].x > -INFINITY ? exp((s[i].x - m) * inv_t) : 1.0);
    return {m, m < INFINITY ? 1.0 / z : NAN};
}

// One workgroup per tree: wave 0 walks (lane = node), all sum what a rejection leaves.
__global__ __launch_bounds__(kFinish) void k_sample_finish(SampleArgs a) {
    constexpr int W = kFinish / 64, E = kFinish * 4;  // waves; logits a round
    extern __shared__ double s_sum[];  // [rounds][W]
    __shared__ double s_z[CDB_TREE_MAX_NODES + 1];  // 1 / Z_k after k rejections at the current node
    __shared__ int s_out[CDB_TREE_MAX_NODES];        // their tokens
    __shared__ int s_cur, s_k, s_end;
    __shared__ double s_pm, s_pinv, s_qm, s_qinv, s_total;
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const bool dense = a.sm.draft_logits != nullptr;
    const double inv_t = a.sm.temperature ? 1.0 / (double)a.sm.temperature[t] : 1.0;
    const double inv_d = dense && a.sm.draft_temperature ? 1.0 / (double)a.sm.draft_temperature[t] : 1.0;
    const int rounds = (a.V + E - 1) / E, r0 = a.row0[t];

    // wave 0: the nodes
    const size_t at = (size_t)t * a.dr.max_nodes + lane;
    bool live = false;
    int par = -2, token = 0, path = -1, count = 0, cur = -1, tried = -1, k = 0;
    int next = 0;
    double u = 0.0, pj = 0.0, qj = 1.0;
    RowStat sp{0.0, 0.0}, sq{0.0, 0.0};
    bool bad_p = false, bad_q = false;
    if (w == 0) {
        int n = a.dr.n_nodes[t];
        next = a.first_ids[t];
        if (n < 0 || n > a.dr.max_nodes) n = 0;
        if (n > 0) {
            bool refused = false;
            if (a.dr.seq) {
                const int s = a.dr.seq[t];
                for (int i = lane; i < t; i += 64) refused |= a.dr.seq[i] == s;
                refused |= s < 0 || s >= a.dr.max_seqs;
                if (a.dr.len && !__any(refused)) refused = !tree_len_ok(a.dr.len[s]);
            }
            if (__any(refused)) {
                if (lane == 0) set_err(a.err, CDB_DEV_BAD_INDEX);
                n = 0;
            } else if ((a.sm.temperature && !temperature_ok(a.sm.temperature[t])) ||
                       (dense && a.sm.draft_temperature && !temperature_ok(a.sm.draft_temperature[t]))) {
                if (lane == 0) set_err(a.err, CDB_DEV_BAD_VALUE);
                n = 0;
            }
        }
        live = lane < n && r0 >= 0;
        if (live && r0 > a.n_rows - 1 - lane) {
            set_err(a.err, CDB_DEV_BAD_INDEX);
            live = false;
        }
        if (live) {
            par = a.dr.parent[at];
            token = a.dr.tokens[at];
            u = a.sm.u_node[at];
        }
        live = live && par < lane;
        if (live && par >= 0 && (token < 0 || token >= a.V)) {
            set_err(a.err, CDB_DEV_BAD_INDEX);
            live = false;
        }
        bool kids = false;
        for (int j = 1; j < a.dr.max_nodes; ++j) kids |= __shfl(live ? par : -2, j, 64) == lane;
        if (live) {
            sp = row_stat(a.stats + (size_t)(r0 + lane) * a.pieces, a.pieces, inv_t);
            bad_p = !(sp.inv < INFINITY);
            if (dense && kids) {
                sq = row_stat(a.stats + (size_t)(a.n_rows + r0 + lane) * a.pieces, a.pieces, inv_d);
                bad_q = !(sq.inv < INFINITY);
            }
        }
        // this node's token after its parent
        const int from = live && par >= 0 ? par : lane;
        const double pm = __shfl(sp.m, from, 64), pi = __shfl(sp.inv, from, 64);
        const double qm = __shfl(sq.m, from, 64), qi = __shfl(sq.inv, from, 64);
        if (live && par >= 0) {
            pj = exp(((double)a.sm.logits[(size_t)(r0 + par) * a.sm.logits_stride + token] - pm) * inv_t) * pi;
            if (dense) qj = exp(((double)a.sm.draft_logits[(size_t)(r0 + par) * a.sm.draft_stride + token] - qm) * inv_d) * qi;
        }
    }
    // what is left of the target's probability of token i at the current node after k rejections
    auto left = [&](float lp, float lq, int i, int k) {
        double r = exp(((double)lp - s_pm) * inv_t) * s_pinv;
        if (dense) {
            if (k) {
                const double q = exp(((double)lq - s_qm) * inv_d) * s_qinv;
                for (int s = 1; s < k; ++s) r = fmax(r - q, 0.0) * s_z[s];
                r = fmax(r - q, 0.0);
            }
        } else {
            for (int s = 0; s < k; ++s) r = i == s_out[s] ? 0.0 : r;
        }
        return r;
    };
    for (;;) {
        // 0: walk on; the walk needs sums (1: after a rejection, 2: at the end) or is over (3)
        if (w == 0) {
            int todo = 0;
            while (!todo) {
                const uint64_t kids = __ballot(live && par == cur && lane > tried);
                if (!kids) {
                    todo = cur < 0 ? 3 : 2;
                    if (todo == 2 && __shfl(bad_p, cur, 64)) {
                        if (lane == 0) set_err(a.err, CDB_DEV_BAD_VALUE);
                        next = -1;
                        todo = 3;
                    }
                    break;
                }
                const int j = __ffsll((unsigned long long)kids) - 1;
                tried = j;
                bool yes;
                if (cur < 0) {
                    yes = __shfl(token, j, 64) == next;
                } else {
                    if (__shfl(bad_p || bad_q, cur, 64)) {
                        if (lane == 0) set_err(a.err, CDB_DEV_BAD_VALUE);
                        next = -1;
                        todo = 3;
                        break;
                    }
                    double r = pj;
                    if (dense) {
                        for (int s = 1; s <= k; ++s) r = fmax(r - qj, 0.0) * s_z[s];
                    } else {
                        bool out = false;
                        for (int s = 0; s < k; ++s) out |= s_out[s] == token;
                        r = out ? 0.0 : k ? r * s_z[k] : r;
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
            const int from = cur < 0 ? 0 : cur;
            const double v0 = __shfl(sp.m, from, 64), v1 = __shfl(sp.inv, from, 64), v2 = __shfl(sq.m, from, 64), v3 = __shfl(sq.inv, from, 64);
            if (lane == 0) {
                s_cur = cur;
                s_k = k;
                s_end = todo;
                s_pm = v0, s_pinv = v1, s_qm = v2, s_qinv = v3;
            }
        }
        __syncthreads();
        const int todo = s_end;
        int kk = s_k;
        if (todo == 3) break;
        const float* lp = a.sm.logits + (size_t)(r0 + s_cur) * a.sm.logits_stride;
        const float* lq = a.sm.draft_logits + (size_t)(r0 + s_cur) * a.sm.draft_stride;
        for (bool again = todo == 1 || kk == 0; again;) {
            for (int i = 0; i < rounds; ++i) {
                const int e = i * E + tid * 4;
                const float4 x = logits4(lp, e, a.V), y = dense && kk ? logits4(lq, e, a.V) : x;
                double s = left(x.x, y.x, e, kk) + left(x.y, y.y, e + 1, kk);
                s += left(x.z, y.z, e + 2, kk) + left(x.w, y.w, e + 3, kk);
                s = wave_all(s, [](double p, double q) { return p + q; });
                if (lane == 0) s_sum[i * W + w] = s;
            }
            __syncthreads();
            if (w == 0) {
                double z = 0.0;
                for (int i = lane; i < rounds * W; i += 64) z += s_sum[i];
                z = wave_all(z, [](double p, double q) { return p + q; });
                if (lane == 0) {
                    s_total = z;
                    s_z[kk] = 1.0 / z;
                }
            }
            __syncthreads();
            // nothing is left: the rejection does not count, what was there before is summed again
            again = kk > 0 && !(s_total > 0.0);
            if (again) --kk;
        }
        if (w == 0) {
            k = kk;
            if (lane == 0) s_k = kk;
        }
        __syncthreads();
        if (todo == 2) break;
    }
    if (w != 0) return;
    if (s_end == 2) {
        // the first 256 logits whose cumulated sum passes u, then the first logit
        const double aim = (double)a.sm.u_next[t] * s_total;
        double before = 0.0, start = 0.0;
        int seg = -1, some = 0;
        double some_start = 0.0;
        for (int i = 0; i < rounds * W && seg < 0; i += 64) {
            const double own = i + lane < rounds * W ? s_sum[i + lane] : 0.0;
            double v = own;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const double x = __shfl_up(v, o, 64);
                if (lane >= o) v += x;
            }
            const uint64_t hit = __ballot(before + v > aim && own > 0.0), has = __ballot(own > 0.0);
            if (hit) {
                const int j = __ffsll((unsigned long long)hit) - 1;
                seg = i + j;
                start = before + __shfl(v - own, j, 64);
            }
            if (has) {
                const int j = 63 - __clzll((long long)has);
                some = i + j;
                some_start = before + __shfl(v - own, j, 64);
            }
            before += __shfl(v, 63, 64);
        }
        if (seg < 0) seg = some, start = some_start;  // u is 1 to rounding: the last logit with a probability
        const float* lp = a.sm.logits + (size_t)(r0 + s_cur) * a.sm.logits_stride;
        const float* lq = a.sm.draft_logits + (size_t)(r0 + s_cur) * a.sm.draft_stride;
        const int e = seg * 256 + lane * 4;
        const float4 x = logits4(lp, e, a.V), y = dense && s_k ? logits4(lq, e, a.V) : x;
        const double r[4] = {left(x.x, y.x, e, s_k), left(x.y, y.y, e + 1, s_k), left(x.z, y.z, e + 2, s_k),
                             left(x.w, y.w, e + 3, s_k)};
        const double own = r[0] + r[1] + r[2] + r[3];
        double v = own;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double z = __shfl_up(v, o, 64);
            if (lane >= o) v += z;
        }
        double c = start + (v - own);
        int pick = -1, last = -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c += r[i];
            if (r[i] > 0.0) last = e + i;
            if (pick < 0 && r[i] > 0.0 && c > aim) pick = e + i;
        }
        const uint64_t hit = __ballot(pick >= 0), has = __ballot(last >= 0);
        if (hit)
            next = __shfl(pick, __ffsll((unsigned long long)hit) - 1, 64);
        else
            next = has ? __shfl(last, 63 - __clzll((long long)has), 64) : 0;
    }
    if (lane < a.dr.max_nodes) a.out.path[at] = path;
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
    a.pieces = (md.vocab + kPiece - 1) / kPiece;
    a.stats = static_cast<double2*>(scratch);
    a.err = err;
    if (n_rows > 0) k_sample_stats<<<dim3(a.pieces, n_rows, sm.draft_logits ? 2 : 1), 256, 0, st>>>(a);
    const int rounds = (md.vocab + kFinish * 4 - 1) / (kFinish * 4);
    k_sample_finish<<<d.n_trees, kFinish, (size_t)rounds * (kFinish / 64) * sizeof(double), st>>>(a);
    return hipGetLastError();
}

}  // namespace cdb
