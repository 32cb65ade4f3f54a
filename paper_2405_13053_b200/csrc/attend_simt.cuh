// Pieces of attention on CUDA cores: fp32 caches, and heads whose rows are no whole 16-byte vectors.
//
// A CTA of 128 threads walks its share of the tiles (attend.cuh), units of 16 rows, 64 keys held in shared memory as fp32.  Scores:
// a thread has two rows and four keys, 32 FMAs for six 16-byte reads.  Weighted sum: a thread has its entries of all rows,
// one read of a value for 16 FMAs.  A key that a row does not see has weight 0 and is left out of that row's sum, whatever
// its value holds.
//
// Bound by shared-memory reads and FMAs: it stands for exactness in fp32 and for shapes that nothing else takes, not for speed.
#pragma once

#include "attend.cuh"

namespace meteora {

constexpr int kSimtRows = 16;

// floats of a row in shared memory: rows of neighbouring keys start four banks apart
__host__ __device__ inline int simt_pitch(int dim) { return (dim + 3) / 4 * 4 + ((dim + 3) / 4 * 4 % 32 == 0 ? 4 : 0); }
inline size_t attend_simt_bytes(int dim) { return (size_t)((2 * kAttendTile + kSimtRows) * simt_pitch(dim) + kAttendTile * 20 + 32) * 4 + kAttendTile * 8; }

template <typename E>
__global__ void __launch_bounds__(128) k_attend_simt(const __grid_constant__ AttendParams p) {
    extern __shared__ __align__(16) float s_all[];
    const int pitch = simt_pitch(p.dim), quads = (p.dim + 3) / 4;
    float* const s_k = s_all;                                  // [64][pitch]
    float* const s_v = s_k + kAttendTile * pitch;
    float* const s_q = s_v + kAttendTile * pitch;              // [16][pitch]
    float* const s_p = s_q + kSimtRows * pitch;                // [64][20] weights, rows fastest
    float* const s_f = s_p + kAttendTile * 20;                 // [16] factors of the sums so far, then [16] the rows' limits
    long long* const s_off = reinterpret_cast<long long*>(s_f + 32);
    const int tid = threadIdx.x, lane = tid & 31;
    launch_begins(p);
    Walk w = start_walk<1>(p, 0);
    const int ra = (tid >> 4) * 2, kq = tid & 15;              // rows ra, ra + 1 and keys kq + 16 i
    while (w.left > 0) {
        const Walk u = w;                                      // the unit at hand
        const int rows_used = (int)min((long long)kSimtRows, (long long)u.tokens * p.group - (long long)u.rt * kSimtRows);
        __syncthreads();
        for (int i = tid; i < kSimtRows * pitch; i += 128) {
            const int r = i / pitch, e = i - r * pitch;
            int t, g;
            float v = 0.f;
            if (e < p.dim && row_place(p, u, r, t, g))
                v = to_f32(((const E*)p.q)[t * p.q_t + (int64_t)(u.h * p.group + g) * p.q_h + e]) * p.scale_log2;
            s_q[i] = v;
        }
        const PageList pages = page_list(p.batch, u.b);
        int lim[2], t0, g0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int t, g;
            lim[i] = row_place(p, u, ra + i, t, g) ? row_limit(u, t) : 0;
        }
        if (kq == 0) reinterpret_cast<int2*>(s_f + 16)[ra / 2] = make_int2(lim[0], lim[1]);
        row_place(p, u, 0, t0, g0);
        const int lim_all = row_limit(u, t0);
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[2][kSimtRows];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < kSimtRows; ++r) o[i][r] = 0.f;
        bool more = true;
        while (more) {
            const int key0 = w.tile * kAttendTile;
            __syncthreads();
            if (tid < kAttendTile) s_off[tid] = key0 + tid < u.hi ? key_row(pages, p.batch, p.by_page, key0 + tid, p.kv_heads, u.h) : -1ll;
            __syncthreads();
            if (sizeof(E) == 4 && p.dim % 4 == 0) {
                for (int i = tid; i < kAttendTile * quads; i += 128) {
                    const int r = i / quads, c = (i - r * quads) * 4;
                    const long long row = s_off[r];
                    float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
                    if (row >= 0) {
                        a = *reinterpret_cast<const float4*>((const float*)p.k + row * p.dim + c);
                        b = *reinterpret_cast<const float4*>((const float*)p.v + row * p.dim + c);
                    }
                    *reinterpret_cast<float4*>(s_k + r * pitch + c) = a;
                    *reinterpret_cast<float4*>(s_v + r * pitch + c) = b;
                }
            } else {
                for (int i = tid; i < kAttendTile * quads * 4; i += 128) {
                    const int r = i / (quads * 4), c = i - r * quads * 4;
                    const long long row = s_off[r];
                    const bool real = row >= 0 && c < p.dim;
                    s_k[r * pitch + c] = real ? to_f32(((const E*)p.k)[row * p.dim + c]) : 0.f;
                    s_v[r * pitch + c] = real ? to_f32(((const E*)p.v)[row * p.dim + c]) : 0.f;
                }
            }
            __syncthreads();
            if (ra < rows_used) {
                float s[2][4] = {};
                for (int c = 0; c < quads; ++c) {
                    const float4 qa = *reinterpret_cast<const float4*>(s_q + ra * pitch + 4 * c);
                    const float4 qb = *reinterpret_cast<const float4*>(s_q + (ra + 1) * pitch + 4 * c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4 k = *reinterpret_cast<const float4*>(s_k + (kq + 16 * i) * pitch + 4 * c);
                        s[0][i] = fmaf(qa.x, k.x, fmaf(qa.y, k.y, fmaf(qa.z, k.z, fmaf(qa.w, k.w, s[0][i]))));
                        s[1][i] = fmaf(qb.x, k.x, fmaf(qb.y, k.y, fmaf(qb.z, k.z, fmaf(qb.w, k.w, s[1][i]))));
                    }
                }
                const unsigned peers = 0xFFFFu << (lane & 16);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float top = m[j];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = key0 + kq + 16 * i;
                        if (s_off[kq + 16 * i] < 0 || key >= lim[j]) s[j][i] = -INFINITY;
                        top = fmaxf(top, s[j][i]);
                    }
#pragma unroll
                    for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(peers, top, x));
                    const float base = top == -INFINITY ? 0.f : top;
                    const float f = m[j] == -INFINITY ? 0.f : exp2f(m[j] - top);
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float w = exp2f(s[j][i] - base);
                        s_p[(kq + 16 * i) * 20 + ra + j] = w;
                        sum += w;
                    }
                    l[j] = fmaf(l[j], f, sum);
                    m[j] = top;
                    if (kq == 0) s_f[ra + j] = f;
                }
            }
            __syncthreads();
            const int n = min(kAttendTile, u.hi - key0);
            const bool masked = key0 + kAttendTile > lim_all;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int e = tid + 128 * i;
                if (e >= p.dim) continue;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (q * 4 >= rows_used) continue;
                    const float4 f = *reinterpret_cast<const float4*>(s_f + q * 4);
                    float4 a = make_float4(o[i][4 * q] * f.x, o[i][4 * q + 1] * f.y, o[i][4 * q + 2] * f.z, o[i][4 * q + 3] * f.w);
                    if (masked) {
                        const int4 until = *reinterpret_cast<const int4*>(s_f + 16 + q * 4);
                        for (int kk = 0; kk < n; ++kk) {
                            const float v = s_v[kk * pitch + e];
                            const float4 w = *reinterpret_cast<const float4*>(s_p + kk * 20 + q * 4);
                            const int key = key0 + kk;
                            if (key < until.x) a.x = fmaf(w.x, v, a.x);
                            if (key < until.y) a.y = fmaf(w.y, v, a.y);
                            if (key < until.z) a.z = fmaf(w.z, v, a.z);
                            if (key < until.w) a.w = fmaf(w.w, v, a.w);
                        }
                    } else {
#pragma unroll 8
                        for (int kk = 0; kk < n; ++kk) {
                            const float v = s_v[kk * pitch + e];
                            const float4 w = *reinterpret_cast<const float4*>(s_p + kk * 20 + q * 4);
                            a.x = fmaf(w.x, v, a.x);
                            a.y = fmaf(w.y, v, a.y);
                            a.z = fmaf(w.z, v, a.z);
                            a.w = fmaf(w.w, v, a.w);
                        }
                    }
                    o[i][4 * q] = a.x;
                    o[i][4 * q + 1] = a.y;
                    o[i][4 * q + 2] = a.z;
                    o[i][4 * q + 3] = a.w;
                }
            }
            more = w.next(p) && w.unit == u.unit;
        }
        if (u.unit + (int)blockIdx.x >= p.here.pieces) continue;
        const size_t piece = (size_t)(u.unit + (int)blockIdx.x) * kSimtRows;
        const unsigned peers = 0xFFFFu << (lane & 16);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float sum = l[j];
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(peers, sum, x);
            if (ra + j < rows_used && kq == 0) p.here.ml[piece + ra + j] = make_float2(m[j], sum);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = tid + 128 * i;
            if (e >= p.dim) continue;
#pragma unroll
            for (int r = 0; r < kSimtRows; ++r)
                if (r < rows_used) p.here.o[(piece + r) * p.dim + e] = o[i][r];
        }
    }
    launch_ends(p);
}

}  // namespace meteora
