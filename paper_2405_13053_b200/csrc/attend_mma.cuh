// Pieces of attention on bf16 caches for few rows: a stream of keys and values through warp-level matrix instructions.
//
// A CTA of four warps takes a tile of rows (16, or 64 where a sequence brings more) and walks a piece's keys in tiles of 64,
// fetched by asynchronous 16-byte copies, kStages - 1 tiles ahead, each key's row found through its page.  WM = 1: the
// warps share the 16 rows and take 16 of a tile's keys each, their running maxima and sums apart until they join at the
// end; WM = 4: each warp has 16 rows of its own and takes all 64 keys.  Scores and weighted sums are m16n8k16 products with
// fp32 accumulators; the weights 2^(s - m) are rounded to bf16 for the second product, and l sums the ROUNDED weights, so
// that the result is an exact average with weights that are off by 2^-8 at most, not one whose weights miss a sum of 1.
// Bound by HBM in a decode batch: 64 keys of 128 entries are 32 KB, and two CTAs of an SM hold 128 KB in flight.
#pragma once

#include "attend.cuh"

namespace meteora {

template <int DP, int WM> struct AttendMmaShape {
    static constexpr int kChunks = DP / 8;                         // 16-byte chunks of a row
    static constexpr int kRows = 16 * WM;
    static constexpr int kTileBytes = kAttendTile * DP * 2;        // keys or values of a tile
    static constexpr int kStages = DP == 64 ? 4 : WM == 4 ? 2 : 3;     // (64 rows: two CTAs per SM instead of a third stage)
    static constexpr int kOffs = kStages + 1;
    static constexpr bool kHoldQ = DP <= 128;                      // queries stay in registers
    static constexpr int kWeightBytes = kHoldQ ? 0 : kRows * kAttendTile * 2;      // (else they lie in the queries' place)
    static constexpr int kBytes = 2 * kStages * kTileBytes + kRows * DP * 2 + kWeightBytes + kOffs * kAttendTile * 8;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two weights rounded to bf16 (a in the lower half); they come back as the values they were rounded to.
__device__ __forceinline__ uint32_t round_pair(float& a, float& b) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    a = __uint_as_float(r << 16);
    b = __uint_as_float(r & 0xFFFF0000u);
    return r;
}

template <int DP, int WM>
__global__ void __launch_bounds__(128) k_attend_mma(const __grid_constant__ AttendParams p) {
    typedef AttendMmaShape<DP, WM> S;
    constexpr int kRows = S::kRows, KB = WM == 1 ? 1 : 4;          // 16-key blocks of a tile that a warp takes
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t* const s_kv = smem;                                    // [stage][K, V][64][DP], chunks swizzled by row
    uint8_t* const s_q = smem + 2 * S::kStages * S::kTileBytes;    // [kRows][DP]
    uint32_t* const s_w = reinterpret_cast<uint32_t*>(s_q + (S::kHoldQ ? 0 : kRows * DP * 2));     // [kRows][32] pairs of weights
    long long* const s_off = reinterpret_cast<long long*>(s_q + kRows * DP * 2 + S::kWeightBytes); // [kOffs][64] rows of keys
    const uint32_t kv0 = (uint32_t)__cvta_generic_to_shared(s_kv), q0 = (uint32_t)__cvta_generic_to_shared(s_q);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const AttendItem it = attend_item(p, blockIdx.x);
    const int rows_used = it.tile_tokens * it.tile_heads;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    auto swz = [](int row, int chunk) { return (uint32_t)(row * DP * 2 + ((chunk ^ (row & 7)) << 4)); };
    // queries, rows past the tile's and entries past the head's zero
    {
        const __nv_bfloat16* q = (const __nv_bfloat16*)p.q;
        for (int i = tid; i < kRows * S::kChunks; i += 128) {
            const int r = i / S::kChunks, c = i - r * S::kChunks;
            const int t = it.t0 + r / it.tile_heads, g = it.g0 + r % it.tile_heads;
            uint4 val = make_uint4(0u, 0u, 0u, 0u);
            if (r < rows_used && t < p.batch.T && g < p.group && c * 8 < p.dim) {
                const __nv_bfloat16* src = q + t * p.q_t + (int64_t)(it.h * p.group + g) * p.q_h + c * 8;
                if (((uintptr_t)src & 15) == 0) {
                    val = *reinterpret_cast<const uint4*>(src);
                } else {
                    __nv_bfloat16 e[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) e[j] = src[j];
                    memcpy(&val, e, 16);
                }
            }
            *reinterpret_cast<uint4*>(s_q + swz(r, c)) = val;
        }
    }

    constexpr bool kHoldQ = S::kHoldQ;
    uint32_t qf[kHoldQ ? DP / 16 : 1][4];
    const int q_row = (WM == 1 ? 0 : warp * 16) + (lane & 15);
    __syncthreads();
    if (kHoldQ) {
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) ldsm4(q0 + swz(q_row, ks * 2 + (lane >> 4)), qf[kHoldQ ? ks : 0]);
    }

    int t_seg = it.t0;                                             // first token of the sequence at hand in the tile
    const int t_end = min(p.batch.T, it.t0 + it.tile_tokens);
    while (t_seg < t_end) {
        OwnRange seg = {-1, 0, 0, t_end, it.piece * p.prefix_piece, min(p.batch.prefix, (it.piece + 1) * p.prefix_piece)};
        if (!it.prefix) {
            const int b = sequence_of(p.batch, t_seg, lane);
            if (b < 0) {                                           // (tokens before the first or behind the last sequence)
                ++t_seg;
                continue;
            }
            seg = own_range(p, b, it.piece, t_seg, t_end);
        }
        const int lo = seg.lo, hi = seg.hi, t_next = seg.t_next;
        if (lo >= hi) {                                            // nothing that these rows see in this piece
            t_seg = t_next;
            continue;
        }
        const PageList pages = page_list(p.batch, seg.b);
        const int tiles = (hi - lo + kAttendTile - 1) / kAttendTile;
        auto place = [&](int tile) {                               // by threads 0 .. 63
            const int key = lo + tile * kAttendTile + tid;
            return tile < tiles && key < hi ? key_row(pages, p.batch, key, p.kv_heads, it.h) : -1ll;
        };
        auto fetch = [&](int tile) {
            const uint32_t dst = kv0 + (tile % S::kStages) * 2 * S::kTileBytes;
            const long long* off = s_off + (tile % S::kOffs) * kAttendTile;
            if (tile < tiles) {
#pragma unroll
                for (int i = 0; i < kAttendTile * S::kChunks / 128; ++i) {
                    const int x = tid + i * 128, r = x / S::kChunks, c = x % S::kChunks;
                    const long long row = off[r];
                    const bool real = row >= 0 && c * 8 < p.dim;
                    const size_t at = real ? (size_t)row * p.dim + c * 8 : 0;
                    cp_async16(dst + swz(r, c), (const __nv_bfloat16*)p.k + at, real);
                    cp_async16(dst + S::kTileBytes + swz(r, c), (const __nv_bfloat16*)p.v + at, real);
                }
            }
            cp_async_commit();
        };
        __syncthreads();                                           // (the join of the sequence before is done with the stages)
        if (tid < kAttendTile) {
#pragma unroll
            for (int i = 0; i < S::kStages; ++i) s_off[i * kAttendTile + tid] = place(i);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < S::kStages - 1; ++i) fetch(i);

        float o[DP / 8][4];
#pragma unroll
        for (int i = 0; i < DP / 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        const int row0 = (WM == 1 ? 0 : warp * 16) + (lane >> 2);  // this thread's rows: row0 and row0 + 8
        int lim[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int t = it.t0 + (row0 + 8 * i) / it.tile_heads;
            const bool mine = row0 + 8 * i < rows_used && t >= t_seg && t < t_next;
            lim[i] = !mine ? 0 : it.prefix ? hi : own_limit(seg, t);
        }
        // first key that some row of the tile does not see: tiles below it need no comparison with lim
        const int lim_all = it.prefix ? hi : own_limit(seg, t_seg);

        for (int tile = 0; tile < tiles; ++tile) {
            cp_async_wait<S::kStages - 2>();
            __syncthreads();
            const long long next_off = tid < kAttendTile ? place(tile + S::kStages) : 0;
            fetch(tile + S::kStages - 1);
            const uint32_t kt = kv0 + (tile % S::kStages) * 2 * S::kTileBytes, vt = kt + S::kTileBytes;
            const long long* off = s_off + (tile % S::kOffs) * kAttendTile;
            const int key0 = lo + tile * kAttendTile, kb0 = WM == 1 ? warp : 0;
            float s[KB * 2][4];
#pragma unroll
            for (int i = 0; i < KB * 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll
            for (int ks = 0; ks < DP / 16; ++ks) {
                uint32_t qa[4];
                if (kHoldQ) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) qa[j] = qf[kHoldQ ? ks : 0][j];
                } else {
                    ldsm4(q0 + swz(q_row, ks * 2 + (lane >> 4)), qa);
                }
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    uint32_t kf[4];                                // keys 0-7 and 8-15 of the block, 16 entries each
                    ldsm4(kt + swz((kb0 + kb) * 16 + (lane & 7) + ((lane >> 4) << 3), ks * 2 + ((lane >> 3) & 1)), kf);
                    mma_bf16(s[kb * 2], qa, kf[0], kf[1]);
                    mma_bf16(s[kb * 2 + 1], qa, kf[2], kf[3]);
                }
            }
            // scores in units of log2; keys without a place or past a row's limit count as -inf
            float top[2] = {m[0], m[1]};
            const bool masked = key0 + kAttendTile > lim_all;
#pragma unroll
            for (int i = 0; i < KB * 2; ++i) {
                const int kk = kb0 * 16 + i * 8 + (lane & 3) * 2;
                const longlong2 places = *reinterpret_cast<const longlong2*>(off + kk);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = key0 + kk + (j & 1);
                    const bool there = ((j & 1) ? places.y : places.x) >= 0;
                    const bool seen = there && (!masked || key < lim[j >> 1]);
                    s[i][j] = seen ? s[i][j] * p.scale_log2 : -INFINITY;
                    top[j >> 1] = fmaxf(top[j >> 1], s[i][j]);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xFFFFFFFFu, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xFFFFFFFFu, top[i], 2));
            }
            if (__any_sync(0xFFFFFFFFu, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float f = m[i] == -INFINITY ? 0.f : exp2_fast(m[i] - top[i]);
                    m[i] = top[i];
                    l[i] *= f;
#pragma unroll
                    for (int d = 0; d < DP / 8; ++d) {
                        o[d][2 * i] *= f;
                        o[d][2 * i + 1] *= f;
                    }
                }
            }
            const float base[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
            uint32_t pf[KB][4];
#pragma unroll
            for (int i = 0; i < KB * 2; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i][j] = exp2_fast(s[i][j] - base[j >> 1]);
                pf[i >> 1][(i & 1) * 2] = round_pair(s[i][0], s[i][1]);
                pf[i >> 1][(i & 1) * 2 + 1] = round_pair(s[i][2], s[i][3]);
                l[0] += s[i][0] + s[i][1];
                l[1] += s[i][2] + s[i][3];
            }
            // A product with weight 0 is no good where the value is no finite number: a tile with keys that some of the rows
            // do not see, and such a value among them, is summed key by key.
            bool plain = false;
            if (masked && !it.prefix && t_next - t_seg > 1) {
                bool odd = false;
#pragma unroll 4
                for (int i = 0; i < kAttendTile * S::kChunks / 128; ++i) {
                    const uint4 v = *reinterpret_cast<const uint4*>(s_kv + (vt - kv0) + (tid + i * 128) * 16);
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) odd |= (w[j] & 0x7F80u) == 0x7F80u || (w[j] & 0x7F800000u) == 0x7F800000u;
                }
                plain = __syncthreads_or(odd);
            }
            if (plain) {
#pragma unroll
                for (int i = 0; i < KB * 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) s_w[(row0 + 8 * j) * 32 + kb0 * 8 + i * 4 + (lane & 3)] = pf[i >> 1][(i & 1) * 2 + j];
                __syncwarp();
                for (int kk = kb0 * 16; kk < (kb0 + KB) * 16; ++kk) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (key0 + kk >= lim[j]) continue;
                        const uint32_t pair = s_w[(row0 + 8 * j) * 32 + (kk >> 1)];
                        const float w = __uint_as_float((kk & 1) ? pair & 0xFFFF0000u : pair << 16);
#pragma unroll
                        for (int d = 0; d < DP / 8; ++d) {
                            const uint32_t v = *reinterpret_cast<const uint32_t*>(s_kv + (vt - kv0) + swz(kk, d) + (lane & 3) * 4);
                            o[d][2 * j] = fmaf(w, __uint_as_float(v << 16), o[d][2 * j]);
                            o[d][2 * j + 1] = fmaf(w, __uint_as_float(v & 0xFFFF0000u), o[d][2 * j + 1]);
                        }
                    }
                }
                __syncwarp();
            } else {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
                    for (int d = 0; d < DP / 16; ++d) {
                        uint32_t vf[4];
                        ldsm4_trans(vt + swz((kb0 + kb) * 16 + (lane & 15), d * 2 + (lane >> 4)), vf);
                        mma_bf16(o[2 * d], pf[kb], vf[0], vf[1]);
                        mma_bf16(o[2 * d + 1], pf[kb], vf[2], vf[3]);
                    }
                }
            }
            if (tid < kAttendTile) s_off[((tile + S::kStages) % S::kOffs) * kAttendTile + tid] = next_off;
        }
        cp_async_wait<0>();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 1);
            l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 2);
        }
        const size_t all_rows = (size_t)p.batch.T * p.q_heads;
        auto out_row = [&](int r, bool& mine) {                    // slot and row of tile row r
            const int t = it.t0 + r / it.tile_heads, g = it.g0 + r % it.tile_heads;
            mine = r < rows_used && t >= t_seg && t < t_next && g < p.group;
            return (size_t)it.slot * all_rows + (size_t)t * p.q_heads + it.h * p.group + g;
        };
        if (WM == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                bool mine;
                const size_t row = out_row(row0 + 8 * i, mine);
                if (!mine) continue;
                if ((lane & 3) == 0) p.part_ml[row] = make_float2(m[i], l[i]);
#pragma unroll
                for (int d = 0; d < DP / 8; ++d) {
                    const int e = d * 8 + (lane & 3) * 2;
                    if (e < p.dim) *reinterpret_cast<float2*>(p.part_o + row * p.dim + e) = make_float2(o[d][2 * i], o[d][2 * i + 1]);
                }
            }
        } else {
            __syncthreads();                                       // every warp has read its last tile
            float* const s_o = reinterpret_cast<float*>(s_kv);     // [warp][16][DP], then (m, l) [warp][16]
            float2* const s_ml = reinterpret_cast<float2*>(s_o + 4 * 16 * DP);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = (lane >> 2) + 8 * i;
                if (r >= rows_used) continue;
                if ((lane & 3) == 0) s_ml[warp * 16 + r] = make_float2(m[i], l[i]);
#pragma unroll
                for (int d = 0; d < DP / 8; ++d)
                    *reinterpret_cast<float2*>(s_o + (warp * 16 + r) * DP + d * 8 + (lane & 3) * 2) = make_float2(o[d][2 * i], o[d][2 * i + 1]);
            }
            __syncthreads();
            for (int x = tid; x < rows_used * (DP / 4); x += 128) {
                const int r = x / (DP / 4), e = x % (DP / 4) * 4;
                bool mine;
                const size_t row = out_row(r, mine);
                if (!mine || e >= p.dim) continue;
                float2 ml[4];
                float M = -INFINITY, L = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    ml[w] = s_ml[w * 16 + r];
                    M = fmaxf(M, ml[w].x);
                }
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float f = piece_factor(ml[w], M == -INFINITY ? 0.f : M);
                    if (f == 0.f) continue;
                    const float4 v = *reinterpret_cast<const float4*>(s_o + (w * 16 + r) * DP + e);
                    L = fmaf(f, ml[w].y, L);
                    acc.x = fmaf(f, v.x, acc.x);
                    acc.y = fmaf(f, v.y, acc.y);
                    acc.z = fmaf(f, v.z, acc.z);
                    acc.w = fmaf(f, v.w, acc.w);
                }
                if (e == 0) p.part_ml[row] = make_float2(M, L);
                *reinterpret_cast<float4*>(p.part_o + row * p.dim + e) = acc;
            }
        }
        t_seg = t_next;
    }
}

}  // namespace meteora
