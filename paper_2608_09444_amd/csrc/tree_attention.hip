// Attention of drafted token trees over the paged, depth-indexed KV cache: row i
// attends to positions 0..base-1 of its sequence and to the positions base + j
// whose bit j of its mask is set (its ancestors and itself), in its own plane.
#include "cdb_internal.h"

namespace cdb {

// One wave per (row, head), 64 positions at a time: lane = position for the
// scores, lane = dim for the weighted sum of V.
template <int HD>
__global__ __launch_bounds__(64) void k_tree_attn(const float* __restrict__ q, KvTarget kv,
                                                  const int32_t* __restrict__ seq, cdb_tree tree, int M, int H,
                                                  uint16_t* __restrict__ out, int* err,
                                                  const int32_t* __restrict__ dn) {
    __shared__ float s_q[HD];
    const int head = blockIdx.x, m = blockIdx.y, lane = threadIdx.x;
    const int d = H * HD;
    if (m >= live_rows(dn, M)) return;
    const float qscale = 1.4426950408889634f / sqrtf((float)HD);
    for (int k = lane; k < HD; k += 64) s_q[k] = q[(size_t)m * d + head * HD + k] * qscale;
    __syncthreads();
    const int sq = seq[m], base = tree.base[m];
    const uint64_t mask = tree.mask[m];
    const int plane = kv.c_row ? kv.c_row[m] + 1 : kv.plane_fixed;
    const bool plane_ok = kv.c_row ? (plane >= 1 && plane <= kv.n_planes - 2) : (plane >= 0 && plane < kv.n_planes);
    const int cap = kv.max_pages * kPage;
    const int last = base + (mask ? 63 - __clzll((long long)mask) : -1);
    if (sq < 0 || sq >= kv.max_seqs || !plane_ok || base < 0 || base > cap || last >= cap) {
        if (lane == 0) set_err(err, CDB_DEV_UNMAPPED_PAGE);
        return;
    }
    const int32_t* pt = kv.page_table + ((size_t)sq * kv.n_planes + plane) * kv.max_pages;
    float mx = -1e30f, l = 0.f, acc[2] = {0.f, 0.f};
    for (int p0 = 0; p0 <= last; p0 += 64) {
        const int p = p0 + lane;
        bool see = p <= last && (p < base || (mask >> (p - base) & 1));
        const uint16_t* row = nullptr;
        float s = -1e30f;
        if (p <= last) {
            const int pid = pt[p / kPage];
            if (pid < 0 || pid >= kv.n_pages) {
                set_err(err, CDB_DEV_UNMAPPED_PAGE);
                see = false;
            }
            if (see) {
                row = kv.pool + kv_offset(kv.layer, pid, kv.n_pages, 0, head, H, p % kPage, HD);
                s = 0.f;
                for (int k = 0; k < HD; ++k) s = fmaf(s_q[k], bf2f(row[k]), s);
            }
        }
        float mn = s;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) mn = fmaxf(mn, __shfl_xor(mn, o, 64));
        mn = fmaxf(mn, mx);
        const float corr = exp2f(mx - mn), w = see ? exp2f(s - mn) : 0.f;
        mx = mn;
        l = l * corr + w;
        acc[0] *= corr;
        acc[1] *= corr;
        const size_t vofs = (size_t)H * kPage * HD;
        for (int j = 0; j < 64; ++j) {
            const float wj = __shfl(w, j, 64);
            const uint64_t rj = (uint64_t)__shfl((int)((uint64_t)row >> 32), j, 64) << 32 |
                                (uint32_t)__shfl((int)(uint64_t)row, j, 64);
            const uint16_t* vr = reinterpret_cast<const uint16_t*>(rj);
            if (!vr) continue;
            acc[0] = fmaf(wj, bf2f(vr[vofs + lane]), acc[0]);
            if (lane + 64 < HD) acc[1] = fmaf(wj, bf2f(vr[vofs + lane + 64]), acc[1]);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
#pragma unroll
    for (int u = 0; u < 2; ++u)
        if (lane + 64 * u < HD)
            out[frag_index(m, head * HD + lane + 64 * u, d)] = f2bf(l != 0.f ? acc[u] / l : 0.f);
}

size_t tree_scratch_bytes(const cdb_model_desc&, int) { return 0; }

hipError_t launch_tree_attention(const float* q, const KvTarget& kv, const int32_t* seq, const cdb_tree& tree, int M,
                                 int H, int hd, uint16_t* out, int* err, hipStream_t st, const int32_t* dn) {
    if (M <= 0) return hipSuccess;
    const dim3 grid(H, M);
    switch (hd) {
        case 64: k_tree_attn<64><<<grid, 64, 0, st>>>(q, kv, seq, tree, M, H, out, err, dn); break;
        case 96: k_tree_attn<96><<<grid, 64, 0, st>>>(q, kv, seq, tree, M, H, out, err, dn); break;
        case 128: k_tree_attn<128><<<grid, 64, 0, st>>>(q, kv, seq, tree, M, H, out, err, dn); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace cdb
