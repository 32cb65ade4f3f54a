// Attention on bf16 caches for units of 64 rows (a sequence with more than 16 rows, where the tensor-core kernel does not take
// the prefix: that too), through warp-level matrix instructions.
//
// A CTA of four warps walks its share of the tiles (attend.cuh), 64 keys each, fetched by asynchronous 16-byte copies kStages - 1
// tiles ahead, across units too: each key's row is found through its page, a new unit's queries come with its first
// tile.  A warp has 16 of the rows and takes all 64 keys.  Scores and weighted sums are m16n8k16 products with fp32
// accumulators; the weights 2^(s - m) are rounded to bf16 for the second product, and l sums the ROUNDED weights, so that
// the result is an exact average with weights that are off by 2^-8 at most, not one whose weights miss a sum of 1.
#pragma once

#include "attend_ops.cuh"

namespace meteora {

template <int DP> struct AttendMmaShape {
    static constexpr int kChunks = DP / 8;                         // 16-byte chunks of a row
    static constexpr int kRows = 64;
    static constexpr int kTileBytes = kAttendTile * DP * 2;        // keys or values of a tile
    static constexpr int kStages = DP == 64 ? 4 : 2;               // (two CTAs per SM instead of a third stage)
    static constexpr int kOffs = kStages + 1;
    static constexpr bool kHoldQ = DP <= 128;                      // queries stay in registers
    static constexpr int kQBytes = kRows * DP * 2;                 // of a unit; kStages units can be under way
    static constexpr int kWeightBytes = kHoldQ ? 0 : kRows * kAttendTile * 2;      // (else they lie in the queries' place)
    static constexpr int kInfoInts = 12;
    static constexpr int kBytes = 2 * kStages * kTileBytes + kStages * kQBytes + kWeightBytes + kOffs * (kAttendTile * 8 + kInfoInts * 4);
};

template <int DP>
__global__ void __launch_bounds__(128) k_attend_mma(const __grid_constant__ AttendParams p) {
    typedef AttendMmaShape<DP> S;
    constexpr int kRows = S::kRows, KB = 4;                        // 16-key blocks of a tile
    constexpr bool kHoldQ = S::kHoldQ;
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t* const s_kv = smem;                                    // [stage][K, V][64][DP], chunks swizzled by row
    uint8_t* const s_qs = smem + 2 * S::kStages * S::kTileBytes;   // [unit % kStages][kRows][DP]
    long long* const s_off = reinterpret_cast<long long*>(s_qs + S::kStages * S::kQBytes + S::kWeightBytes);   // [kOffs][64] rows of keys
    int* const s_info = reinterpret_cast<int*>(s_off + S::kOffs * kAttendTile);        // [kOffs][kInfoInts]
    const uint32_t kv0 = (uint32_t)__cvta_generic_to_shared(s_kv), q0 = (uint32_t)__cvta_generic_to_shared(s_qs);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    launch_begins(p);
    Walk w = start_walk<1>(p, 0);                                  // runs ahead: where the places of keys are looked up
    const int cta = (int)blockIdx.x;

    auto swz = [](int row, int chunk) { return (uint32_t)(row * DP * 2 + ((chunk ^ (row & 7)) << 4)); };
    const bool q_wide = (((uintptr_t)p.q | (uintptr_t)(p.q_t * 2) | (uintptr_t)(p.q_h * 2)) & 15) == 0;
    int made = 0, units = 0;                                       // tiles looked up, units among them
    bool fresh = true;                                             // the walk is at its first tile of a unit
    // The next tile: the place of key `tid` (returned), and what the tile is (kept in thread 0 until both are stored).
    int info[S::kInfoInts];
    auto look_up = [&]() {
        const int key = w.tile * kAttendTile + tid;
        long long row = -1;
        if (tid < kAttendTile && key < w.hi) row = key_row(page_list(p.batch, w.b), p.batch, p.by_page, key, p.kv_heads, w.h);
        if (fresh) ++units;
        info[0] = w.b, info[1] = w.rt, info[2] = w.h, info[3] = w.unit, info[4] = w.tile * kAttendTile, info[5] = w.hi;
        info[6] = w.first, info[7] = w.tokens, info[8] = w.held, info[9] = fresh, info[11] = (units - 1) % S::kStages;
        const int unit = w.unit;
        fresh = !w.next(p) || w.unit != unit;
        info[10] = fresh;                                          // last of its unit
        return row;
    };
    auto store_place = [&](long long row) {
        const int slot = made % S::kOffs;
        if (tid < kAttendTile) s_off[slot * kAttendTile + tid] = row;
        if (tid == 0)
#pragma unroll
            for (int i = 0; i < S::kInfoInts; ++i) s_info[slot * S::kInfoInts + i] = info[i];
        ++made;
    };
    auto view = [&](int tile, Walk& v) {                           // a tile's unit, as row_place and row_limit need it
        const int* q = s_info + tile % S::kOffs * S::kInfoInts;
        v.b = q[0], v.rt = q[1], v.h = q[2], v.unit = q[3], v.hi = q[5], v.first = q[6], v.tokens = q[7], v.held = q[8];
        return q;
    };
    auto fetch = [&](int tile) {
        if (tile < made) {
            const uint32_t dst = kv0 + tile % S::kStages * 2 * S::kTileBytes;
            const long long* off = s_off + tile % S::kOffs * kAttendTile;
#pragma unroll
            for (int i = 0; i < kAttendTile * S::kChunks / 128; ++i) {
                const int x = tid + i * 128, r = x / S::kChunks, c = x % S::kChunks;
                const long long row = off[r];
                const bool real = row >= 0 && c * 8 < p.dim;
                const size_t at = real ? (size_t)row * p.dim + c * 8 : 0;
                cp_async16(dst + swz(r, c), (const __nv_bfloat16*)p.k + at, real);
                cp_async16(dst + S::kTileBytes + swz(r, c), (const __nv_bfloat16*)p.v + at, real);
            }
            Walk u;
            const int* q = view(tile, u);
            if (q[9]) {                                            // a new unit's queries; rows and entries that are none are zero
                const int buf = q[11] * S::kQBytes;
                for (int i = tid; i < kRows * S::kChunks; i += 128) {
                    const int r = i / S::kChunks, c = i - r * S::kChunks;
                    int t, g;
                    const bool real = row_place(p, u, r, t, g) && c * 8 < p.dim;
                    const __nv_bfloat16* src = (const __nv_bfloat16*)p.q + (real ? t * p.q_t + (int64_t)(u.h * p.group + g) * p.q_h + c * 8 : 0);
                    if (q_wide) {
                        cp_async16(q0 + buf + swz(r, c), src, real);
                    } else {
                        __nv_bfloat16 e[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) e[j] = real ? src[j] : __float2bfloat16_rn(0.f);
                        memcpy(s_qs + buf + swz(r, c), e, 16);
                    }
                }
            }
        }
        cp_async_commit();
    };
    for (int i = 0; i < S::kStages && w.left > 0; ++i) store_place(look_up());
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::kStages - 1; ++i) fetch(i);

    float o[DP / 8][4], m[2], l[2];
    uint32_t qf[kHoldQ ? DP / 16 : 1][4];
    Walk u;                                                        // the unit at hand
    int lim[2], lim_all = 0, q_buf = 0;
    const int row0 = warp * 16 + (lane >> 2);      // this thread's rows of it: row0 and row0 + 8
    const int q_row = warp * 16 + (lane & 15);
    for (int tile = 0; tile < made; ++tile) {
        cp_async_wait<S::kStages - 2>();
        __syncthreads();
        const bool more = w.left > 0;
        const long long next_row = more ? look_up() : 0;
        fetch(tile + S::kStages - 1);
        const uint32_t kt = kv0 + tile % S::kStages * 2 * S::kTileBytes, vt = kt + S::kTileBytes;
        const long long* off = s_off + tile % S::kOffs * kAttendTile;
        const int* const q_info = s_info + tile % S::kOffs * S::kInfoInts;
        const int key0 = q_info[4];
        const bool last = q_info[10];
        if (q_info[9]) {
            view(tile, u);
            q_buf = q_info[11] * S::kQBytes;
            if (kHoldQ) {
#pragma unroll
                for (int ks = 0; ks < DP / 16; ++ks) ldsm4(q0 + q_buf + swz(q_row, ks * 2 + (lane >> 4)), qf[kHoldQ ? ks : 0]);
            }
#pragma unroll
            for (int i = 0; i < DP / 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                m[i] = -INFINITY, l[i] = 0.f;
                int t, g;
                lim[i] = row_place(p, u, row0 + 8 * i, t, g) ? row_limit(u, t) : 0;
            }
            int t, g;
            row_place(p, u, 0, t, g);
            lim_all = row_limit(u, t);                          // every row of the unit sees the keys below it
        }
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
                            ldsm4(q0 + q_buf + swz(q_row, ks * 2 + (lane >> 4)), qa);
                        }
#pragma unroll
                        for (int kb = 0; kb < KB; ++kb) {
                            uint32_t kf[4];                                // keys 0-7 and 8-15 of the block, 16 entries each
                            ldsm4(kt + swz(kb * 16 + (lane & 7) + ((lane >> 4) << 3), ks * 2 + ((lane >> 3) & 1)), kf);
                            mma_bf16(s[kb * 2], qa, kf[0], kf[1]);
                            mma_bf16(s[kb * 2 + 1], qa, kf[2], kf[3]);
                        }
                    }
                    // scores in units of log2; keys without a place or past a row's limit count as -inf
                    float top[2] = {m[0], m[1]};
                    const bool masked = key0 + kAttendTile > lim_all;
#pragma unroll
                    for (int i = 0; i < KB * 2; ++i) {
                        const int kk = i * 8 + (lane & 3) * 2;
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
                    if (masked && u.b >= 0 && u.tokens > 1) {
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
            uint32_t* const s_w = reinterpret_cast<uint32_t*>(kHoldQ ? s_qs + q_buf : s_qs + S::kStages * S::kQBytes);   // [kRows][32] pairs
#pragma unroll
                        for (int i = 0; i < KB * 2; ++i)
#pragma unroll
                            for (int j = 0; j < 2; ++j) s_w[(row0 + 8 * j) * 32 + i * 4 + (lane & 3)] = pf[i >> 1][(i & 1) * 2 + j];
                        __syncwarp();
                        for (int kk = 0; kk < kAttendTile; ++kk) {
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
                                ldsm4_trans(vt + swz(kb * 16 + (lane & 15), d * 2 + (lane >> 4)), vf);
                                mma_bf16(o[2 * d], pf[kb], vf[0], vf[1]);
                                mma_bf16(o[2 * d + 1], pf[kb], vf[2], vf[3]);
                            }
                        }
                    }
        if (last) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 1);
                l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 2);
            }
            const size_t piece = (size_t)(u.unit + cta) * kRows;
            if (u.unit + cta < p.here.pieces) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    int t, g;
                    if (!row_place(p, u, row0 + 8 * i, t, g)) continue;
                    const size_t row = piece + row0 + 8 * i;
                    if ((lane & 3) == 0) p.here.ml[row] = make_float2(m[i], l[i]);
#pragma unroll
                    for (int d = 0; d < DP / 8; ++d) {
                        const int e = d * 8 + (lane & 3) * 2;
                        if (e < p.dim) *reinterpret_cast<float2*>(p.here.o + row * p.dim + e) = make_float2(o[d][2 * i], o[d][2 * i + 1]);
                    }
                }
            }
        }
        if (more) store_place(next_row);
    }
    cp_async_wait<0>();
    launch_ends(p);
}

}  // namespace meteora
