// Attention on bf16 caches for units of 64 rows (sequences with more than 16 that the tensor-core kernel does not take, and the prefix
// where it takes none), through warp-level matrix instructions.  Included by wgemm_tcgen05.cu after the device helpers it uses.
//
// A CTA of four warps walks its share of the tiles (attend.cuh), 64 keys each, kStages of them in shared memory; a warp has
// 16 of the rows and takes all 64 keys.  Where pages are whole multiples of 8 keys and a head's entries of 64 (kTma), a
// tile comes as TMA boxes, its page numbers asked for a tile before; else as 16-byte copies, every key's row looked up.
// The products and the rounding of the weights are those of attend_warp.cuh; a row's reference m stays until the maximum is 8
// above it, as in attend_prefix.cuh.
//
// Bound by what two CTAs of an SM (252 registers a thread) issue: 16 sequences of 10 to 100 tokens on 300, 40 heads of their own
// (164 MB of keys and values at most, 6 GFLOP and half as much again in masked parts of tiles): 68 us, 0.3 instructions per
// scheduler and cycle, matrix pipes a quarter busy.
#pragma once

#include "attend_ops.cuh"

namespace meteora {

template <int DP, bool kTma>
__global__ void __launch_bounds__(128)
k_attend_mma(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ AttendParams p, const int box_shift) {
    typedef AttendMmaShape<DP> S;
    constexpr int KB = kAttendTile / 16;                           // 16-key blocks of a tile
    constexpr bool kHoldQ = DP <= 128;                             // queries stay in registers
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), ring0 = (raw + 1023u) & ~1023u;
    uint8_t* const ring = smem_raw + (ring0 - raw);                // [stage][K, V][entries / 64][64 keys][128 bytes], chunks swizzled by key
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_id();
    uint8_t* const s_q = ring + S::kStages * 2 * S::kTileBytes + warp * S::kWarpBytes;     // this warp's [DP / 64][16][128 bytes], if not held
    uint32_t* const s_w = reinterpret_cast<uint32_t*>(s_q + (kHoldQ ? 0 : 16 * DP * 2));   // and [16][32] pairs of weights
    const uint32_t q0 = ring0 + (uint32_t)(s_q - ring);
    long long* const s_off = reinterpret_cast<long long*>(ring + S::kStages * 2 * S::kTileBytes + 4 * S::kWarpBytes);    // [kInfos][64]
    TileInfo* const s_info = reinterpret_cast<TileInfo*>(s_off + S::kInfos * kAttendTile);
    const uint32_t bar = ring0 + S::kBarOff;
    if (kTma && tid == 0) {
#pragma unroll
        for (int i = 0; i < S::kStages; ++i) mbar_init(bar + i * 8, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    launch_begins(p);
    Walk w = start_walk<1>(p, 0);                                  // runs ahead: the tile whose pages are asked for
    const int cta = (int)blockIdx.x;

    auto swz = [](int row, int chunk) { return (uint32_t)((chunk >> 3) * (kAttendTile * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4)); };
    auto swq = [](int row, int chunk) { return (uint32_t)((chunk >> 3) * 2048 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4)); };
    int asked = 0, fetched = 0;
    bool fresh = true, more = w.left > 0;
    // A tile is asked for: what it is and (kTma: in lane i of warp 0, for box i) its pages, or the place of key `tid`.
    struct Asked {
        long long found;
        int key0, keys, h;
        bool real;
    };
    auto ask = [&]() {
        Asked a;
        a.real = more;
        a.found = -1;
        if (!more) return a;
        a.key0 = w.tile * kAttendTile;
        a.keys = min(kAttendTile, w.hi - a.key0);
        a.h = w.h;
        const PageList pages = page_list(p.batch, w.b);
        TileInfo* const q = s_info + asked % S::kInfos;
        if (kTma) {
            const int key = a.key0 + (lane << box_shift), slot = (int)p.by_page.of((unsigned)key);
            if (warp == 0 && (lane << box_shift) < a.keys && slot < pages.n) a.found = (unsigned)__ldg(pages.pages + slot);
        } else {
            if (tid < a.keys) a.found = key_row(pages, p.batch, p.by_page, a.key0 + tid, p.kv_heads, w.h);
            if (tid < kAttendTile) s_off[asked % S::kInfos * kAttendTile + tid] = a.found;
            const unsigned there = __ballot_sync(0xFFFFFFFFu, a.found >= 0);
            if (lane == 0 && warp < 2) q->there[warp] = there;
        }
        const int4 x = make_int4(w.b, w.rt, w.h, w.unit), y = make_int4(w.first, w.tokens, w.held, w.hi);
        int4 z = make_int4(a.key0, fresh, 0, 0);
        const int unit = w.unit;
        more = w.next(p);
        fresh = !more || w.unit != unit;
        z.z = fresh;                                               // last of its unit
        if (tid == 0) q->x = x, q->y = y, q->z = z;
        ++asked;
        return a;
    };
    auto fetch = [&](const Asked& a) {                             // (every warp is done with the stage)
        if (a.real) {
            const int stage = fetched % S::kStages;
            const uint32_t dst = ring0 + stage * 2 * S::kTileBytes;
            TileInfo* const q = s_info + fetched % S::kInfos;
            if (kTma) {
                if (warp == 0) {
                    const int rows = 1 << box_shift, key = a.key0 + lane * rows;
                    const bool ok = a.found >= 0 && a.found < p.batch.n_pages;
                    const unsigned boxes = __ballot_sync(0xFFFFFFFFu, ok);
                    if (lane == 0) mbar_expect_tx(bar + stage * 8, (uint32_t)__popc(boxes) * rows * DP * 4);
                    __syncwarp();
                    if (ok) {
                        const int at = key - (int)p.by_page.of((unsigned)key) * p.batch.page, plane = (int)a.found * p.kv_heads + a.h;
#pragma unroll
                        for (int c = 0; c < DP / 64; ++c) {
                            const uint32_t to = dst + c * (kAttendTile * 128) + lane * rows * 128;
                            tma_load_4d(to, &tmK, 0, at, c, plane, bar + stage * 8);
                            tma_load_4d(to + S::kTileBytes, &tmV, 0, at, c, plane, bar + stage * 8);
                        }
                    }
                    // lane i: keys 2 i and 2 i + 1
                    const int k0 = 2 * lane;
                    const unsigned bits = (boxes >> (k0 >> box_shift) & 1u) ? (k0 < a.keys ? 1u : 0u) | (k0 + 1 < a.keys ? 2u : 0u) : 0u;
                    unsigned lo = lane < 16 ? bits << k0 : 0u, hi = lane < 16 ? 0u : bits << (k0 - 32);
                    lo = __reduce_or_sync(0xFFFFFFFFu, lo);
                    hi = __reduce_or_sync(0xFFFFFFFFu, hi);
                    if (lane == 0) q->there[0] = lo, q->there[1] = hi;
                }
            } else {
                const long long* off = s_off + fetched % S::kInfos * kAttendTile;
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
            ++fetched;
        }
        if (!kTma) cp_async_commit();
    };
    {
        Asked first[S::kStages];
#pragma unroll
        for (int i = 0; i < S::kStages; ++i) first[i] = ask();     // (their page numbers are under way together)
        __syncthreads();
#pragma unroll
        for (int i = 0; i < S::kStages; ++i) fetch(first[i]);
        __syncthreads();
    }

    const bool q_even = (((uintptr_t)p.q & 3) | ((uintptr_t)(p.q_t | p.q_h) & 1)) == 0;        // pairs of entries in one load
    const int row0 = warp * 16 + (lane >> 2), col = (lane & 3) * 2;    // this thread's rows of a unit: row0 and row0 + 8
    float o[DP / 8][4], m[2], l[2];
    uint32_t qf[kHoldQ ? DP / 16 : 1][4];
    int lim[2], lim_all = 0, tokens = 0, unit = 0;
    bool ok = true;
    for (int tile = 0; tile < asked; ++tile) {
        const int stage = tile % S::kStages;
        const Asked next = ask();
        if (kTma) {
            ok = mbar_wait_warp(bar + stage * 8, tile / S::kStages & 1);
            if (__syncthreads_or(!ok)) {                           // (all warps or none)
                ok = false;
                break;
            }
        } else {
            cp_async_wait<S::kStages - 1>();
            __syncthreads();
        }
        const TileInfo info = s_info[tile % S::kInfos];
        const int key0 = info.z.x;
        if (info.z.y) {                                            // a new unit
            Walk u;
            u.b = info.x.x, u.rt = info.x.y, u.h = info.x.z, u.first = info.y.x, u.tokens = info.y.y, u.held = info.y.z, u.hi = info.y.w;
            unit = info.x.w;
            tokens = u.b < 0 ? 1 : u.tokens;
            int t, g;
            row_place(p, u, 0, t, g);
            lim_all = row_limit(u, t);                             // every row sees the keys below it
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bool real = row_place(p, u, row0 + 8 * i, t, g);
                lim[i] = real ? row_limit(u, t) : 0;
                m[i] = -INFINITY, l[i] = 0.f;
                const __nv_bfloat16* src = (const __nv_bfloat16*)p.q + (real ? t * p.q_t + (int64_t)(u.h * p.group + g) * p.q_h : 0);
#pragma unroll
                for (int ks = 0; ks < DP / 16; ++ks)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int e = ks * 16 + j * 8 + col;
                        uint32_t v = 0;
                        if (real && e < p.dim) {
                            if (q_even) v = *reinterpret_cast<const uint32_t*>(src + e);
                            else v = (uint32_t)__bfloat16_as_ushort(src[e]) | (uint32_t)__bfloat16_as_ushort(src[e + 1]) << 16;
                        }
                        if (kHoldQ) qf[kHoldQ ? ks : 0][2 * j + i] = v;
                        else *reinterpret_cast<uint32_t*>(s_q + swq((lane >> 2) + 8 * i, ks * 2 + j) + (lane & 3) * 4) = v;
                    }
            }
            __syncwarp();
#pragma unroll
            for (int d = 0; d < DP / 8; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[d][j] = 0.f;
        }
        const uint32_t kt = ring0 + stage * 2 * S::kTileBytes, vt = kt + S::kTileBytes;
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
                ldsm4(q0 + swq(lane & 15, ks * 2 + (lane >> 4)), qa);
            }
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                uint32_t kf[4];                                    // keys 0-7 and 8-15 of the block, 16 entries each
                ldsm4(kt + swz(kb * 16 + (lane & 7) + ((lane >> 4) << 3), ks * 2 + ((lane >> 3) & 1)), kf);
                mma_bf16(s[kb * 2], qa, kf[0], kf[1]);
                mma_bf16(s[kb * 2 + 1], qa, kf[2], kf[3]);
            }
        }
        // Keys without a place or past a row's limit count as -inf; a row's reference m stays until a score is 8 above it.
        const bool masked = key0 + kAttendTile > lim_all, some = masked || (info.there[0] & info.there[1]) != 0xFFFFFFFFu;
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < KB * 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int kk = i * 8 + col + (j & 1);
                s[i][j] *= p.scale_log2;
                if (some && (!(info.there[i >> 2] >> (kk & 31) & 1u) || key0 + kk >= lim[j >> 1])) s[i][j] = -INFINITY;
                top[j >> 1] = fmaxf(top[j >> 1], s[i][j]);
            }
        if (__any_sync(0xFFFFFFFFu, top[0] > m[0] + 8.f || top[1] > m[1] + 8.f)) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xFFFFFFFFu, top[i], 1));
                top[i] = fmaxf(m[i], fmaxf(top[i], __shfl_xor_sync(0xFFFFFFFFu, top[i], 2)));
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
        if (kTma && (info.there[0] & info.there[1]) != 0xFFFFFFFFu) {  // what lies in the place of keys that there are not
            for (int r = warp * 16; r < warp * 16 + 16; ++r)
                if (!(info.there[r >> 5] >> (r & 31) & 1u) && lane < S::kChunks)
                    *reinterpret_cast<uint4*>(ring + (vt - ring0) + swz(r, lane)) = make_uint4(0u, 0u, 0u, 0u);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncthreads();
        }
        // A product with weight 0 is no good where the value is no finite number: a tile with keys that some of the rows do
        // not see, and such a value among them, is summed key by key.
        bool plain = false;
        if (masked && tokens > 1) {
            bool odd = false;
#pragma unroll 4
            for (int i = 0; i < kAttendTile * S::kChunks / 128; ++i) {
                const uint4 v = *reinterpret_cast<const uint4*>(ring + (vt - ring0) + (tid + i * 128) * 16);
                const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) odd |= (x[j] & 0x7F80u) == 0x7F80u || (x[j] & 0x7F800000u) == 0x7F800000u;
            }
            plain = __syncthreads_or(odd);
        }
        if (plain) {
#pragma unroll
            for (int i = 0; i < KB * 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) s_w[((lane >> 2) + 8 * j) * 32 + i * 4 + (lane & 3)] = pf[i >> 1][(i & 1) * 2 + j];
            __syncwarp();
            for (int kk = 0; kk < kAttendTile; ++kk) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (key0 + kk >= lim[j]) continue;
                    const uint32_t pair = s_w[((lane >> 2) + 8 * j) * 32 + (kk >> 1)];
                    const float x = __uint_as_float((kk & 1) ? pair & 0xFFFF0000u : pair << 16);
#pragma unroll
                    for (int d = 0; d < DP / 8; ++d) {
                        const uint32_t v = *reinterpret_cast<const uint32_t*>(ring + (vt - ring0) + swz(kk, d) + (lane & 3) * 4);
                        o[d][2 * j] = fmaf(x, __uint_as_float(v << 16), o[d][2 * j]);
                        o[d][2 * j + 1] = fmaf(x, __uint_as_float(v & 0xFFFF0000u), o[d][2 * j + 1]);
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
        __syncthreads();                                           // the stage is free
        fetch(next);
        if (info.z.z && unit + cta < p.here.pieces) {
            const size_t piece = (size_t)(unit + cta) * S::kRows;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 1);
                l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 2);
                if (lim[i] == 0) continue;                         // no row
                const size_t row = piece + row0 + 8 * i;
                if ((lane & 3) == 0) p.here.ml[row] = make_float2(m[i], l[i]);
#pragma unroll
                for (int d = 0; d < DP / 8; ++d) {
                    const int e = d * 8 + col;
                    if (e < p.dim) *reinterpret_cast<float2*>(p.here.o + row * p.dim + e) = make_float2(o[d][2 * i], o[d][2 * i + 1]);
                }
            }
        }
    }
    if (!kTma) cp_async_wait<0>();
    if (!ok) {
        if (tid == 0) {
            atomicExch(p.status, 1);
            atomicExch(p.status + 1, 4700);
        }
        for (int i = max(0, fetched - S::kStages); i < fetched; ++i) mbar_wait_warp(bar + i % S::kStages * 8, i / S::kStages & 1);   // copies under way land
    }
    launch_ends(p);
}

}  // namespace meteora
