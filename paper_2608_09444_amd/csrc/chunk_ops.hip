// Queries, keys and values of chunks of new tokens: RMSNorm of every query and key
// head, rotation, and the write into the paged cache.
#include "cdb_internal.h"

namespace cdb {

struct QkvArgs {
    cdb_chunks ch;
    KvTarget kv;
    cdb_qkv in;
    void* q_out;
    int H;
    float eps, base;
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

// Workgroup = ROWS rows.  Eight lanes (four for heads of 64) take one head of q, k
// or v: a lane 8 values of its first half and the 8 that are rotated with them.
template <int HD, typename IN, typename OUT, int ROWS>
__global__ __launch_bounds__(256) void k_chunk_qkv(QkvArgs a) {
    constexpr int G = HD == 64 ? 4 : 8, HALF = HD / 2;
    struct Row {
        int pos, turn, pid, ok;
    };
    __shared__ Row s_row[ROWS];
    __shared__ float2 s_cs[ROWS][HALF];
    const int tid = threadIdx.x, row0 = blockIdx.x * ROWS;
    if (tid < ROWS) s_row[tid].ok = 0;
    int r0 = 0, r1 = 0;
    if (tid < a.ch.n_chunks) {
        r0 = a.ch.row0[tid];
        r1 = a.ch.row0[tid + 1];
    }
    if (__syncthreads_or(r0 < 0 || r1 < r0 || r1 > a.ch.n_rows)) {
        if (blockIdx.x == 0 && tid == 0) set_err(a.err, CDB_DEV_BAD_INDEX);
        return;
    }
    if (r0 < row0 + ROWS && r1 > row0) {
        const int seq = a.ch.seq[tid], pos = a.ch.pos0[tid], c = a.kv.c_row ? a.kv.c_row[tid] : 0;
        const int plane = a.kv.c_row ? c + 1 : a.kv.plane_fixed;
        const bool ok = seq >= 0 && seq < a.kv.max_seqs && pos >= 0 && pos <= a.kv.max_pages * kPage - (r1 - r0) &&
                        (!a.kv.c_row || (c >= 0 && c < a.kv.n_planes - 2));
        if (!ok) set_err(a.err, CDB_DEV_BAD_INDEX);
        if (ok)
            for (int r = max(r0, row0); r < min(r1, row0 + ROWS); ++r) {
                const int p = pos + (r - r0);
                const int pid = a.kv.page_table[((size_t)seq * a.kv.n_planes + plane) * a.kv.max_pages + p / kPage];
                const bool there = pid >= 0 && pid < a.kv.n_pages;
                if (!there) set_err(a.err, CDB_DEV_UNMAPPED_PAGE);
                s_row[r - row0] = Row{p, a.in.rope_pos ? a.in.rope_pos[r] : p, there ? pid : -1, 1};
            }
    }
    __syncthreads();
    for (int i = tid; i < ROWS * HALF; i += 256) {
        const int r = i / HALF, j = i % HALF;
        if (!s_row[r].ok) continue;
        const double ang = (double)s_row[r].turn * pow((double)a.base, -2.0 * j / HD);
        double sn, cs;
        sincos(ang, &sn, &cs);
        s_cs[r][j] = make_float2((float)cs, (float)sn);
    }
    __syncthreads();
    const int e = tid % G;
    const bool on = e * 16 < HD;  // heads of 96 leave two of eight lanes idle
    for (int i = tid / G; i < ROWS * 3 * a.H; i += 256 / G) {
        const int head = i % a.H, rp = i / a.H, part = rp % 3, r = rp / 3;
        const Row w = s_row[r];
        if (!w.ok) continue;
        const int64_t stride = part == 0 ? a.in.q_stride : part == 1 ? a.in.k_stride : a.in.v_stride;
        const IN* src = static_cast<const IN*>(part == 0 ? a.in.q : part == 1 ? a.in.k : a.in.v) + (row0 + r) * stride +
                        head * HD + e * 8;
        float x[8] = {}, y[8] = {};
        if (on) {
            load8(src, x);
            load8(src + HALF, y);
        }
        if (part < 2) {
            if (a.in.norm) {
                float ss = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) ss += x[k] * x[k] + y[k] * y[k];
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
                for (int k = 0; k < 8; ++k) x[k] *= f * gx[k], y[k] *= f * gy[k];
            }
            if (on)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float2 cs = s_cs[r][e * 8 + k];
                    const float u = fmaf(x[k], cs.x, -(y[k] * cs.y));
                    y[k] = fmaf(y[k], cs.x, x[k] * cs.y);
                    x[k] = u;
                }
        }
        if (!on) continue;
        if (part == 0) {
            OUT* dst = static_cast<OUT*>(a.q_out) + (size_t)(row0 + r) * a.H * HD + head * HD + e * 8;
            store8(dst, x);
            store8(dst + HALF, y);
        } else if (w.pid >= 0) {
            uint16_t* dst = a.kv.pool + kv_offset(a.kv.layer, w.pid, a.kv.n_pages, part - 1, head, a.H, w.pos % kPage, HD) + e * 8;
            store8(dst, x);
            store8(dst + HALF, y);
        }
    }
}

template <int HD, typename IN, typename OUT>
static void launch_qkv(const QkvArgs& a, hipStream_t st) {
    if (a.ch.n_rows <= 1024)
        k_chunk_qkv<HD, IN, OUT, 1><<<a.ch.n_rows, 256, 0, st>>>(a);
    else
        k_chunk_qkv<HD, IN, OUT, 4><<<(a.ch.n_rows + 3) / 4, 256, 0, st>>>(a);
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
    const QkvArgs a{ch, kv, in, q_out, md.n_heads, md.rms_eps, md.rope_base, err};
    switch (md.head_dim) {
        case 64: launch_qkv_types<64>(a, q_type, st); break;
        case 96: launch_qkv_types<96>(a, q_type, st); break;
        case 128: launch_qkv_types<128>(a, q_type, st); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace cdb
