// Queries, keys and values of chunks of new tokens: RMSNorm of every query and key
// head, rotation, and the write into the paged cache.
//
//   x' = g x / sqrt(mean(x^2) + eps);   (a, b) -> (a cos t - b sin t, b cos t + a sin t)
//
// for a = x'[j], b = x'[j + hd / 2], t = position * base^(-2 j / hd).
// Bound: every value is read and written once, and for few rows the chain row -> chunk ->
// page id -> write.  Measured: 8 rows 4.2-4.3 us, of which 1.7 are the launch's own; 7 chunks of 3-201 rows, fp32,
// 55 x 96 heads 17.4 us, 4.7 TB/s; 16 chunks of 384-512, bf16, 16 x 128 heads 31.2-32.2 us, 5.5 TB/s
// (a large copy: 5.1); 13 rows of 65536, the others nobody's, 23-25 us.
#include <cmath>

#include "cdb_internal.h"

namespace cdb {

struct QkvArgs {
    cdb_chunks ch;
    KvTarget kv;
    cdb_qkv in;
    void* q_out;
    int H;
    float eps;
    double log2_base;
    int* err;
};

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bflo(a[i]), v[2 * i + 1] = bfhi(a[i]);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
    u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<u32x4*>(p) = a;
}

// Workgroup = (row, kTasks of its 3 H heads of q, k and v).  Eight lanes (four for heads of 64) take one head: a
// lane 8 values of its first half and the 8 that are rotated with them.  Chunks follow one another, so the ends of
// row0 tell by scalar loads whether any has the row; then its values are asked for, so that they come
// while its chunk, its page and its angles are found.  Two heads to a group of lanes: the angles
// (in 64 bits: a position of 10^5 keeps 2^-24 of a turn) and the search are paid once for 64 heads of 128, and enough
// workgroups are left.  1, 2, 4 heads (graphs): 8 rows 4.0, 4.3, 4.5 us; 7 ragged chunks 18.6, 17.2, 17.7; 16 prompts 31.4, 31.1, 35.5.
constexpr int kTasks = 2;

template <int HD, typename IN, typename OUT>
__global__ __launch_bounds__(256) void k_chunk_qkv(QkvArgs a) {
    constexpr int G = HD == 64 ? 4 : 8, HALF = HD / 2, NG = 256 / G;
    __shared__ int s_pos, s_turn, s_pid;
    __shared__ float2 s_cs[HALF];
    const int tid = threadIdx.x, row = blockIdx.x, e = tid % G;
    const bool on = e * 16 < HD;  // heads of 96 leave two of eight lanes idle
    const auto* ends = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)a.ch.row0;
    const bool outside = row < ends[0] || row >= ends[a.ch.n_chunks];
    if (outside && blockIdx.x + blockIdx.y != 0) return;  // the first workgroup tells what is wrong with row0
    if (tid == 0) s_pos = -1;
    int r0 = 0, r1 = 0, seq = -1, pos = 0, c = 0;
    if (tid < a.ch.n_chunks) {
        r0 = a.ch.row0[tid];
        r1 = a.ch.row0[tid + 1];
        seq = a.ch.seq[tid];
        pos = a.ch.pos0[tid];
        if (a.kv.c_row) c = a.kv.c_row[tid];
    }
    float x[kTasks][8], y[kTasks][8];
#pragma unroll
    for (int t = 0; t < kTasks; ++t) {
        const int i = (blockIdx.y * kTasks + t) * NG + tid / G, head = i % a.H, part = i / a.H;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[t][k] = y[t][k] = 0.f;
        if (on && part < 3 && !outside) {
            const int64_t stride = part == 0 ? a.in.q_stride : part == 1 ? a.in.k_stride : a.in.v_stride;
            const IN* src = static_cast<const IN*>(part == 0 ? a.in.q : part == 1 ? a.in.k : a.in.v) + row * stride + head * HD + e * 8;
            load8(src, x[t]);
            load8(src + HALF, y[t]);
        }
    }
    const double turn = exp2(a.log2_base * (-2.0 / HD) * tid);  // of pair tid, radians per position
    if (__syncthreads_or(r0 < 0 || r1 < r0 || r1 > a.ch.n_rows)) {
        if (blockIdx.x + blockIdx.y == 0 && tid == 0) set_err(a.err, CDB_DEV_BAD_INDEX);
        return;
    }
    int pid = -1;
    const bool mine = row >= r0 && row < r1;
    if (mine) {
        const bool ok = seq >= 0 && seq < a.kv.max_seqs && pos >= 0 && pos <= a.kv.max_pages * kPage - (r1 - r0) &&
                        (!a.kv.c_row || (c >= 0 && c < a.kv.n_planes - 2));
        if (ok) {
            const int p = pos + (row - r0), plane = a.kv.c_row ? c + 1 : a.kv.plane_fixed;
            pid = a.kv.page_table[((size_t)seq * a.kv.n_planes + plane) * a.kv.max_pages + p / kPage];
            s_pos = p;
            s_turn = a.in.rope_pos ? a.in.rope_pos[row] : p;
        } else {
            set_err(a.err, CDB_DEV_BAD_INDEX);
        }
    }
    __syncthreads();
    if (s_pos < 0) return;
    if (tid < HALF) {
        double sn, cs;
        sincos((double)s_turn * turn, &sn, &cs);
        s_cs[tid] = make_float2((float)cs, (float)sn);
    }
    if (mine) {
        if (pid < 0 || pid >= a.kv.n_pages) {
            set_err(a.err, CDB_DEV_UNMAPPED_PAGE);
            pid = -1;
        }
        s_pid = pid;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTasks; ++t) {
        const int i = (blockIdx.y * kTasks + t) * NG + tid / G, head = i % a.H, part = i / a.H;
        if (part < 2) {
            if (a.in.norm) {
                float ss = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) ss += x[t][k] * x[t][k] + y[t][k] * y[t][k];
#pragma unroll
                for (int o = 1; o < G; o <<= 1) ss += __shfl_xor(ss, o, G);
                const float f = 1.f / sqrtf(ss * (1.f / HD) + a.eps);
                const uint16_t* gain = static_cast<const uint16_t*>(part == 0 ? a.in.q_gain : a.in.k_gain);
                float gx[8], gy[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) gx[k] = gy[k] = 1.f;
                if (gain && on) {
                    load8(gain + e * 8, gx);
                    load8(gain + HALF + e * 8, gy);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) x[t][k] *= f * gx[k], y[t][k] *= f * gy[k];
            }
            if (on)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float2 cs = s_cs[e * 8 + k];
                    const float u = fmaf(x[t][k], cs.x, -(y[t][k] * cs.y));
                    y[t][k] = fmaf(y[t][k], cs.x, x[t][k] * cs.y);
                    x[t][k] = u;
                }
        }
        if (!on || part > 2) continue;
        if (part == 0) {
            OUT* dst = static_cast<OUT*>(a.q_out) + (size_t)row * a.H * HD + head * HD + e * 8;
            store8(dst, x[t]);
            store8(dst + HALF, y[t]);
        } else if (s_pid >= 0) {
            uint16_t* dst = a.kv.pool + kv_offset(a.kv.layer, s_pid, a.kv.n_pages, part - 1, head, a.H, s_pos % kPage, HD) + e * 8;
            store8(dst, x[t]);
            store8(dst + HALF, y[t]);
        }
    }
}

template <int HD, typename IN, typename OUT>
static void launch_qkv(const QkvArgs& a, hipStream_t st) {
    constexpr int each = 256 / (HD == 64 ? 4 : 8) * kTasks;
    k_chunk_qkv<HD, IN, OUT><<<dim3(a.ch.n_rows, (3 * a.H + each - 1) / each), 256, 0, st>>>(a);
}
template <int HD>
static void launch_qkv_types(const QkvArgs& a, int q_type, hipStream_t st) {
    if (a.in.type == CDB_F32)
        q_type == CDB_F32 ? launch_qkv<HD, float, float>(a, st) : launch_qkv<HD, float, uint16_t>(a, st);
    else
        q_type == CDB_F32 ? launch_qkv<HD, uint16_t, float>(a, st) : launch_qkv<HD, uint16_t, uint16_t>(a, st);
}

hipError_t launch_chunk_qkv(const cdb_model_desc& md, const cdb_chunks& ch, const KvTarget& kv, const cdb_qkv& in,
                            void* q_out, int q_type, int* err, hipStream_t st) {
    if (ch.n_chunks <= 0 || ch.n_rows <= 0) return hipSuccess;
    const QkvArgs a{ch, kv, in, q_out, md.n_heads, md.rms_eps, std::log2((double)md.rope_base), err};
    switch (md.head_dim) {
        case 64: launch_qkv_types<64>(a, q_type, st); break;
        case 96: launch_qkv_types<96>(a, q_type, st); break;
        case 128: launch_qkv_types<128>(a, q_type, st); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace cdb
