// Attention on bf16 caches for units of up to 16 rows: a stream of keys and values through warp-level matrix instructions.
// Included by wgemm_tcgen05.cu after the device helpers it uses.
//
// Every warp is a worker of its own (attend.cuh): it walks its share of the tiles, 16 keys each, with a ring of kStages tiles in
// shared memory that it alone fills and reads, so there is no barrier between warps.  Where pages are whole multiples of 8
// keys and a head's entries of 64 (kTma), a tile comes as TMA boxes of 64 entries by 8 or 16 keys, 128-byte swizzled, its
// page numbers asked for a tile before; else as 16-byte copies, every key's row looked up.  Scores and weighted sums are
// m16n8k16 products with fp32 accumulators; the weights 2^(s - m) are rounded to bf16 for the second product, and l sums
// the ROUNDED weights, so that the result is an exact average with weights that are off by 2^-8 at most, not one whose
// weights miss a sum of 1.
//
// In a decode batch every key is read once for the rows of its kv head: 12 warps of an SM (heads of 128: 168 registers a thread,
// 66 KB a CTA), each with a tile of 8 KB under way behind the one it works on.  128 sequences of 524 own tokens, 8 kv heads
// (275 MB): 60 us = 4.6 TB/s; a tile is a chain of some 250 instructions, 1300 cycles, that 3 warps of a scheduler overlap
// (8 warps of an SM with three stages 70 us).  Forms that were slower: four warps on one tile of 64 keys with block
// barriers 93 us; 16-byte copies for all shapes, 1200 cycles of address work per tile, 67 us.
#pragma once

#include "attend_ops.cuh"

namespace meteora {

template <int DP, bool kTma>
__global__ void __launch_bounds__(128, DP == 256 ? 1 : 3)
k_attend_warp(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ AttendParams p, const int box_shift) {
    typedef AttendWarpShape<DP> S;
    extern __shared__ uint8_t smem_raw[];
    const int lane = threadIdx.x & 31, warp = warp_id();
    const uint32_t raw = smem_u32(smem_raw), base0 = (raw + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base0 - raw);
    uint8_t* const ring = smem + warp * S::kWarpBytes;             // [stage][K, V][entries / 64][16 keys][128 bytes], chunks swizzled by key
    int4* const s_units = reinterpret_cast<int4*>(smem + 4 * S::kWarpBytes) + warp * S::kInfos * 2;
    int2* const s_tiles = reinterpret_cast<int2*>(smem + 4 * (S::kWarpBytes + S::kInfos * 32)) + warp * S::kInfos;
    const uint32_t ring0 = base0 + warp * S::kWarpBytes;
    const uint32_t bar = base0 + 4 * (S::kWarpBytes + S::kInfos * 40) + warp * S::kStages * 8;
    if (kTma && lane == 0) {
#pragma unroll
        for (int i = 0; i < S::kStages; ++i) mbar_init(bar + i * 8, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    launch_begins(p);
    Walk w = start_walk<4>(p, warp);                               // runs ahead: the tile whose page is asked for
    const int worker = (int)blockIdx.x * 4 + warp;
    if (w.left <= 0) {
        launch_ends(p);
        return;
    }

    auto swz = [](int row, int chunk) { return (uint32_t)((chunk >> 3) * (kWarpTile * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4)); };
    constexpr int kCopies = kWarpTile * S::kChunks / 32;           // 16-byte copies of a lane, for keys and values each

    // A tile is asked for (its page numbers or its keys' places are under way), fetched an iteration later, and used when it has
    // arrived.  What a fetch needs stays in registers, and nothing in it waits; what the use needs goes through shared
    // memory: a line per tile, and one per unit when it starts.
    struct Asked {
        int page0, page1;          // kTma: pages of the tile's halves (one where a page holds both), not looked at yet
        int in_page;               // kTma: its first key in page0
        long long place;           // else: of key `lane`
        int key0, keys, h;
        bool real, fresh;
    };
    int asked = 0, fetched = 0, units = 0;
    bool fresh = true, more = true;
    int slot = 0, in_page = 0, page = -1;                          // of the tile asked for last, where a page holds whole tiles
    PageList pages = {};
    auto ask = [&]() {
        Asked a;
        a.real = more;
        a.page0 = a.page1 = -1;
        a.place = -1;
        if (!more) return a;
        a.key0 = w.tile * kWarpTile;
        a.keys = min(kWarpTile, w.hi - a.key0);
        a.h = w.h;
        a.fresh = fresh;
        if (fresh) {
            pages = page_list(p.batch, w.b);
            slot = (int)p.by_page.of((unsigned)a.key0);
            in_page = a.key0 - slot * p.batch.page;
            ++units;
            if (lane == 0) {
                int4* const q = s_units + units % S::kInfos * 2;            // (a tile names its unit by this place alone)
                q[0] = make_int4(w.b, w.rt, w.h, w.first);
                q[1] = make_int4(w.tokens, w.held, w.hi, w.unit);
            }
        }
        if (kTma) {
            if (box_shift == 4) {
                if (in_page >= p.batch.page) in_page = 0, ++slot;
                if (in_page == 0 || fresh) page = slot < pages.n ? __ldg(pages.pages + slot) : -1;
                a.page0 = page;
                a.in_page = in_page;
                in_page += kWarpTile;
            } else {
                const int slot0 = (int)p.by_page.of((unsigned)a.key0), slot1 = (int)p.by_page.of((unsigned)a.key0 + 8u);
                a.in_page = a.key0 - slot0 * p.batch.page;
                if (slot0 < pages.n) a.page0 = __ldg(pages.pages + slot0);
                if (slot1 < pages.n && a.keys > 8) a.page1 = __ldg(pages.pages + slot1);
            }
        } else if (lane < a.keys) {
            a.place = key_row(pages, p.batch, p.by_page, a.key0 + lane, p.kv_heads, w.h);
        }
        const bool inside = w.left > 1 && a.key0 + kWarpTile < w.hi;     // the unit goes on in this share
        if (lane == 0) s_tiles[asked % S::kInfos] = make_int2(a.key0, (fresh ? 1 << 16 : 0) | (inside ? 0 : 1 << 17) | units % S::kInfos << 18);
        if (inside) {
            --w.left;
            ++w.tile;
        } else {
            more = w.next(p);
        }
        fresh = !inside;
        ++asked;
        return a;
    };
    auto view = [&](int at, Walk& u) {                             // the unit at a place, as row_place and row_limit need it
        const int4* const q = s_units + at * 2;
        const int4 x = q[0], y = q[1];
        u.b = x.x, u.rt = x.y, u.h = x.z, u.first = x.w, u.tokens = y.x, u.held = y.y, u.hi = y.z, u.unit = y.w;
    };
    auto fetch = [&](const Asked& a) {
        if (a.real) {
            const int stage = fetched % S::kStages;
            const uint32_t dst = ring0 + stage * 2 * S::kTileBytes, full = bar + stage * 8;
            unsigned there;                                        // keys that there are
            if (kTma) {
                const bool ok0 = (unsigned)a.page0 < (unsigned)p.batch.n_pages, ok1 = (unsigned)a.page1 < (unsigned)p.batch.n_pages;
                if (elect_one()) {
                    const uint32_t box = DP * 4u << box_shift;     // bytes of a box of keys and one of values
                    mbar_expect_tx(full, (ok0 ? box : 0u) + (ok1 ? box : 0u));
                    if (ok0) {
                        const int plane = a.page0 * p.kv_heads + a.h;
                        if (box_shift == 4) {
                            tma_load_4d(dst, &tmK, 0, a.in_page, 0, plane, full);
                            tma_load_4d(dst + S::kTileBytes, &tmV, 0, a.in_page, 0, plane, full);
                        } else {
#pragma unroll
                            for (int c = 0; c < DP / 64; ++c) {    // (a box of 8 keys fills half of a swizzled block: 64 entries at a time)
                                tma_load_4d(dst + c * (kWarpTile * 128), &tmK, 0, a.in_page, c, plane, full);
                                tma_load_4d(dst + S::kTileBytes + c * (kWarpTile * 128), &tmV, 0, a.in_page, c, plane, full);
                            }
                        }
                    }
                    if (ok1) {                                     // the tile's second half, in pages of 8, 24, ...
                        const int key = a.key0 + 8, at = key - (int)p.by_page.of((unsigned)key) * p.batch.page, plane = a.page1 * p.kv_heads + a.h;
#pragma unroll
                        for (int c = 0; c < DP / 64; ++c) {
                            tma_load_4d(dst + c * (kWarpTile * 128) + 1024, &tmK, 0, at, c, plane, full);
                            tma_load_4d(dst + S::kTileBytes + c * (kWarpTile * 128) + 1024, &tmV, 0, at, c, plane, full);
                        }
                    }
                }
                __syncwarp();
                there = ((ok0 ? box_shift == 4 ? 0xFFFFu : 0xFFu : 0u) | (ok1 ? 0xFF00u : 0u)) & (0xFFFFu >> (kWarpTile - a.keys));
            } else {
                there = __ballot_sync(0xFFFFFFFFu, a.place >= 0);
#pragma unroll
                for (int i = 0; i < kCopies; ++i) {
                    const int x = lane + 32 * i, r = x / S::kChunks, c = x % S::kChunks;
                    const long long row = __shfl_sync(0xFFFFFFFFu, a.place, r);
                    const bool real = row >= 0 && c * 8 < p.dim;
                    const size_t at = real ? (size_t)row * p.dim + c * 8 : 0;
                    cp_async16(dst + swz(r, c), (const __nv_bfloat16*)p.k + at, real);
                    cp_async16(dst + S::kTileBytes + swz(r, c), (const __nv_bfloat16*)p.v + at, real);
                }
            }
            if (lane == 0) s_tiles[fetched % S::kInfos].y |= (int)there;
            if (a.fresh && lane < kWarpRows) {                     // a new unit: its queries towards L1
                Walk u;
                view(s_tiles[fetched % S::kInfos].y >> 18, u);
                int t, g;
                if (row_place(p, u, lane, t, g)) {
                    const char* src = (const char*)((const __nv_bfloat16*)p.q + t * p.q_t + (int64_t)(u.h * p.group + g) * p.q_h);
#pragma unroll
                    for (int i = 0; i < DP * 2; i += 128)
                        if (i < p.dim * 2) asm volatile("prefetch.global.L1 [%0];" ::"l"(src + i));
                }
            }
            ++fetched;
        }
        if (!kTma) cp_async_commit();
    };
    Asked pending;
    {
        Asked first[S::kStages];
#pragma unroll
        for (int i = 0; i < S::kStages; ++i) first[i] = ask();     // (their page numbers are under way together)
        __syncwarp();
#pragma unroll
        for (int i = 0; i < S::kStages - 1; ++i) fetch(first[i]);
        pending = first[S::kStages - 1];
    }

    const bool q_even = (((uintptr_t)p.q & 3) | ((uintptr_t)(p.q_t | p.q_h) & 1)) == 0;        // pairs of entries in one load
    const int row0 = lane >> 2, col = (lane & 3) * 2;              // this thread's rows of a unit: row0 and row0 + 8
    float o[DP / 8][4], m[2], l[2];
    uint32_t qf[DP / 16][4];
    int lim[2], lim_all = 0, tokens = 0, unit = 0;
    bool ok = true;
    for (int tile = 0; tile < asked; ++tile) {
        const int stage = tile % S::kStages;
        if (kTma) ok = mbar_wait_warp(bar + stage * 8, tile / S::kStages & 1);
        else cp_async_wait<S::kStages - 2>();
        if (!ok) break;
        __syncwarp();
        fetch(pending);
        pending = ask();
        const int2 at = s_tiles[tile % S::kInfos];                 // first key; keys that there are, first and last of its unit, the unit's place
        const bool last = at.y >> 17 & 1;
        if (at.y >> 16 & 1) {                                      // a new unit
            Walk u;
            view(at.y >> 18, u);
            unit = u.unit;
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
                        qf[ks][2 * j + i] = v;
                    }
            }
#pragma unroll
            for (int d = 0; d < DP / 8; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[d][j] = 0.f;
        }
        const uint32_t kt = ring0 + stage * 2 * S::kTileBytes, vt = kt + S::kTileBytes;
        float s[2][4] = {}, s2[2][4] = {};                         // (two sums each: half the chain of dependent products)
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) {
            uint32_t kf[4];                                        // keys 0-7 and 8-15, 16 entries each
            ldsm4(kt + swz((lane & 7) + ((lane >> 4) << 3), ks * 2 + ((lane >> 3) & 1)), kf);
            mma_bf16(ks & 1 ? s2[0] : s[0], qf[ks], kf[0], kf[1]);
            mma_bf16(ks & 1 ? s2[1] : s[1], qf[ks], kf[2], kf[3]);
        }
        // Keys without a place or past a row's limit count as -inf.  A row's reference m (in units of log2) stays until a
        // score is 8 above it: weights stay below 2^8, and most tiles need neither the row's maximum nor a new scale of o.
        const bool masked = at.x + kWarpTile > lim_all, some = masked || (at.y & 0xFFFF) != 0xFFFF;
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int kk = i * 8 + col + (j & 1);
                s[i][j] = (s[i][j] + s2[i][j]) * p.scale_log2;
                if (some && (!(at.y >> kk & 1) || at.x + kk >= lim[j >> 1])) s[i][j] = -INFINITY;
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
        uint32_t pf[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = exp2_fast(s[i][j] - base[j >> 1]);
            pf[i * 2] = round_pair(s[i][0], s[i][1]);
            pf[i * 2 + 1] = round_pair(s[i][2], s[i][3]);
            l[0] += s[i][0] + s[i][1];
            l[1] += s[i][2] + s[i][3];
        }
        if (kTma && (at.y & 0xFFFF) != 0xFFFF) {                              // what lies in the place of keys that there are not
#pragma unroll
            for (int r = 0; r < kWarpTile; ++r)
                if (!(at.y >> r & 1) && lane < S::kChunks) *reinterpret_cast<uint4*>(ring + (vt - ring0) + swz(r, lane)) = make_uint4(0u, 0u, 0u, 0u);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
        }
        // A product with weight 0 is no good where the value is no finite number: a tile with keys that some of the rows do
        // not see, and such a value among them, is summed key by key.
        bool plain = false;
        if (masked && tokens > 1) {
            bool odd = false;
#pragma unroll 4
            for (int i = 0; i < kCopies; ++i) {
                const uint4 v = *reinterpret_cast<const uint4*>(ring + (vt - ring0) + (lane + 32 * i) * 16);
                const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) odd |= (x[j] & 0x7F80u) == 0x7F80u || (x[j] & 0x7F800000u) == 0x7F800000u;
            }
            plain = __any_sync(0xFFFFFFFFu, odd);
        }
        if (plain) {
            for (int kk = 0; kk < kWarpTile; ++kk) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    // the weight of this row and key, from the lane that has it
                    const uint32_t pair = __shfl_sync(0xFFFFFFFFu, kk < 8 ? pf[j] : pf[2 + j], (lane & ~3) | ((kk & 7) >> 1));
                    const float x = __uint_as_float(kk & 1 ? pair & 0xFFFF0000u : pair << 16);
                    if (at.x + kk >= lim[j]) continue;
#pragma unroll
                    for (int d = 0; d < DP / 8; ++d) {
                        const uint32_t v = *reinterpret_cast<const uint32_t*>(ring + (vt - ring0) + swz(kk, d) + (lane & 3) * 4);
                        o[d][2 * j] = fmaf(x, __uint_as_float(v << 16), o[d][2 * j]);
                        o[d][2 * j + 1] = fmaf(x, __uint_as_float(v & 0xFFFF0000u), o[d][2 * j + 1]);
                    }
                }
            }
        } else {
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                uint32_t vf[4];
                ldsm4_trans(vt + swz(lane & 15, d * 2 + (lane >> 4)), vf);
                mma_bf16(o[2 * d], pf, vf[0], vf[1]);
                mma_bf16(o[2 * d + 1], pf, vf[2], vf[3]);
            }
        }
        if (last && unit + worker < p.here.pieces) {
            const size_t piece = (size_t)(unit + worker) * kWarpRows;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 1);
                l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 2);
                if (lim[i] == 0) continue;                         // no row (every row of a unit that is visited sees a key)
                const size_t row = piece + row0 + 8 * i;
                if ((lane & 3) == 0) p.here.ml[row] = make_float2(m[i], l[i]);
#pragma unroll
                for (int d = 0; d < DP / 8; ++d) {
                    const int e = d * 8 + col;
                    if (e < p.dim) *reinterpret_cast<float2*>(p.here.o + row * p.dim + e) = make_float2(o[d][2 * i], o[d][2 * i + 1]);
                }
            }
        }
        __syncwarp();
    }
    if (!kTma) cp_async_wait<0>();
    if (!ok) {
        if (lane == 0) {
            atomicExch(p.status, 1);
            atomicExch(p.status + 1, 4600);
        }
        for (int i = max(0, fetched - S::kStages); i < fetched; ++i) mbar_wait_warp(bar + i % S::kStages * 8, i / S::kStages & 1);   // copies under way land
    }
    launch_ends(p);
}

}  // namespace meteora
