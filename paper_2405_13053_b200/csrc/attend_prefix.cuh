// Attention on the tensor cores, for bf16 caches (attend.cuh has the mathematics and where the pieces go): the shared prefix, rows of
// all sequences against its keys, and (kOwn) own tokens of sequences that bring more than 64 rows on the average.
// Included by wgemm_tcgen05.cu after the device helpers it uses.
//
// A unit of work is 256 rows (token, head of one kv head's group) x their keys, in tiles of 128 keys; the tiles are dealt to
// one CTA per SM in even shares (the prefix's units of one kv head follow one another: their CTAs read the same keys at about the
// same time).
//
// The rows are two tiles of 128 with a softmax group of eight warps each, two threads per row, 64 of a tile's keys each.
// Scores S = Q K^T go to TMEM, the group turns them into weights 2^(s - m), rounded to bf16 and stored over the scores they
// came from, and the second product O += P V takes P from there (A operand in TMEM) and V as it lies (its entries
// contiguous: the MN-major form of B).  While one group works on its scores the tensor core has the other tile's products:
// S and PV of a tile are 512 cycles each (128 x 128 x 128), a tile's 16384 exponentials 1024 at 16 per cycle, so at 256
// rows tensor core and exponentials are nearly even.  Measured, heads of 128: 512 rows of 8 kv heads over 32768 keys (69 GFLOP)
// 84 us, 880 rows of 40 heads over 8192 keys (148 GFLOP) 171 us = 0.86 PFLOP/s.  With the softmax left out (wrong results) the
// copies and products alone are 57 and 122 us, twice the products' cycles: every 256 rows read their 64 KB of a tile
// through L2, 5.9 TB/s over all SMs (1013 MB in the 171 us), and that bounds this form; a pair of SMs with 512 rows would halve it.  Slower or even:
// maxima exchanged a tile later and a polynomial for a part of the exponentials 87 us (of 82); one thread per row, 8 warps
// of softmax instead of 16, within 5%.
// A row's reference m is not its running maximum: it stays until the maximum is 8 above it, which leaves weights below 2^8
// and spares nearly all rescaling of O.  The two threads of a row need the same m: their warps exchange one word that says
// whether any of their rows needs a new one, and only then the maxima themselves (through unused columns of TMEM).
//
// A page that is not there and the keys behind the last count as -inf, and their values are zeroed in shared memory: what
// the cache holds there (an infinity, a NaN) would pass a weight of 0.  So would a value that is no finite number of an own
// token that only some of the rows see: in tiles with such tokens those values are zeroed too, and added to the rows that
// see them when the unit is done.
#pragma once

#include "attend.cuh"

namespace meteora {

constexpr int kPfxKeys = kPrefixTile, kPfxRows = kPrefixRows;
constexpr int kPfxThreads = 576;                     // warp 0: copies, warp 1: products, 16 warps of softmax
constexpr int kPfxUnits = 16;                        // units described (more than the ring holds, so that copies seldom wait for a place)
constexpr int kPfxOdd = 2 * kPfxUnits;               // units whose zeroed values are remembered (a group is at most kPfxUnits ahead of the other)
constexpr int kPfxMasks = 16;                        // tiles whose page masks are remembered (more than the ring holds)

template <int D> struct PrefixShape {
    static constexpr int kTileBytes = kPfxKeys * D * 2;
    static constexpr int kStages = D == 128 ? 5 : 11;              // of keys or values of one tile
    static constexpr int kBarOff = (2 + kStages) * kTileBytes;     // barriers, then page masks, TMEM slot
    static constexpr int kBars = 2 * kStages + 19 + 2 * kPfxUnits;
    static constexpr int kWords = kBarOff + kBars * 8;             // page masks [kPfxMasks], growth [16], zeroed [kPfxOdd], TMEM slot, then the units
    static constexpr int kUnitOff = (kWords + (kPfxMasks + kPfxOdd + 17) * 4 + 15) / 16 * 16;
    static constexpr int kSmem = 1024 + kUnitOff + kPfxUnits * 48;
};

struct PrefixTcParams {
    AttendParams a;
    int box_rows, box_shift;                         // keys per copy: divides the page and the tile
    int sign;                                        // of the scale (-1, 0, 1): the queries are multiplied by it, scale_log2 is above 0 (a
                                                     // masked score, -inf, stays one)
};

// A_i P^T: A from TMEM, B from shared memory.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
          "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st1(uint32_t taddr, float v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "r"(__float_as_uint(v)) : "memory");
}
__device__ __forceinline__ float tmem_ld1(uint32_t taddr) {
    uint32_t r;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    return __uint_as_float(r);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
        "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
        "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void add2(unsigned long long& a, unsigned long long b) { asm("add.rn.f32x2 %0, %0, %1;" : "+l"(a) : "l"(b)); }
__device__ __forceinline__ unsigned long long pair2(float a, float b) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair2(unsigned long long v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ unsigned long long fma2_of(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Two bf16 times 0: NaN where one is no finite number.
__device__ __forceinline__ uint32_t times_zero(uint32_t v) {
    return ((v & 0x7F80u) == 0x7F80u ? 0x7FFFu : 0u) | ((v & 0x7F800000u) == 0x7F800000u ? 0x7FFF0000u : 0u);
}

// The units of a CTA's share, one after the other; the copies' warp walks them and leaves each one's description.
struct __align__(16) TcUnit {
    int id, b, h, row0;                              // id < 0: no more; b: sequence or -1; rows [row0, row0 + rows) of its
    int rows, first, held, tile0;                    // tokens' and heads'; first token; own tokens held before
    int count, hi, none[2];                          // tiles of keys, from tile0; keys that any of the rows sees
    // keys that the row-th row of the unit sees
    __device__ __forceinline__ int limit(const AttendParams& p, int row) const {
        return b < 0 ? hi : min(hi, held + (int)p.by_group.of((unsigned)(row0 + row)) + 1);
    }
};
template <bool kOwn> struct TcUnits {
    Walk w;
    int x, x_hi, unit_tiles, pair_tiles, rows_all;
    __device__ __forceinline__ bool next(const AttendParams& p, TcUnit& u) {
        if (kOwn) {
            if (w.left <= 0) return false;
            u.id = w.unit, u.b = w.b, u.h = w.h, u.row0 = w.rt * kPfxRows, u.rows = min(kPfxRows, w.tokens * p.group - u.row0);
            u.first = w.first, u.held = w.held, u.tile0 = w.tile, u.hi = w.hi;
            u.count = min(w.left, (w.hi + kPfxKeys - 1) / kPfxKeys - w.tile);
            w.left -= u.count;
            w.tile += u.count;
            w.settle(p);
            return true;
        }
        if (x >= x_hi) return false;
        u.id = x / unit_tiles, u.b = -1, u.h = u.id / pair_tiles, u.row0 = u.id % pair_tiles * kPfxRows, u.rows = min(kPfxRows, rows_all - u.row0);
        u.first = 0, u.held = 0, u.tile0 = x - u.id * unit_tiles, u.hi = p.batch.prefix;
        u.count = min(x_hi, (u.id + 1) * unit_tiles) - x;
        x += u.count;
        return true;
    }
};

template <int D, bool kOwn>
__global__ void __launch_bounds__(kPfxThreads, 1)
k_attend_tc(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PrefixTcParams pp) {
    typedef PrefixShape<D> S;
    constexpr int kHalves = D / 64;
    const AttendParams& p = pp.a;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* const base_ptr = smem_raw + (base - raw);
    const uint32_t s_q = base, ring = base + 2 * S::kTileBytes;
    const uint32_t bar_full = base + S::kBarOff, bar_free = bar_full + S::kStages * 8, bar_s = bar_free + S::kStages * 8, bar_p = bar_s + 16,
                   bar_o = bar_p + 16, bar_ofree = bar_o + 16, bar_q = bar_ofree + 16, bar_x = bar_q + 16, bar_tail = bar_x + 64, bar_u = bar_tail + 8,
                   bar_ufree = bar_u + kPfxUnits * 8;
    volatile uint32_t* const s_mask = reinterpret_cast<volatile uint32_t*>(base_ptr + S::kWords);
    volatile uint32_t* const s_grow = s_mask + kPfxMasks;          // [tile of rows][half][quarter]
    volatile uint32_t* const s_odd = s_grow + 16;                  // [unit of the share % kPfxOdd]: its id + 1, if values were zeroed in it
    uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + S::kWords + (kPfxMasks + kPfxOdd + 16) * 4);
    int4* const s_unit = reinterpret_cast<int4*>(base_ptr + S::kUnitOff);
    const int warp = warp_id(), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(bar_full + i * 8, 1);
            mbar_init(bar_free + i * 8, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_s + i * 8, 1);
            mbar_init(bar_p + i * 8, 8);
            mbar_init(bar_o + i * 8, 1);
            mbar_init(bar_ofree + i * 8, 8);
            mbar_init(bar_q + i * 8, 8);
        }
        for (int i = 0; i < 8; ++i) mbar_init(bar_x + i * 8, 2);
        mbar_init(bar_tail, 1);
        for (int i = 0; i < kPfxUnits; ++i) {
            mbar_init(bar_u + i * 8, 1);
            mbar_init(bar_ufree + i * 8, 17);
        }
        for (int i = 0; i < kPfxOdd; ++i) s_odd[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_slot);    // S of both tiles, then O of both
    launch_begins(p);
    bool ok = true;
    int where = 0;
    const PieceSpace& space = kOwn ? p.own : p.prefix;
    TcUnits<kOwn> units;
    if (kOwn) {
        units.w = start_walk<1>(p, 0);
    } else {
        const Shares shares((uint32_t)p.prefix.total, gridDim.x);
        units.x = (int)shares.start(blockIdx.x), units.x_hi = (int)shares.start(blockIdx.x + 1);
        units.unit_tiles = (p.batch.prefix + kPfxKeys - 1) / kPfxKeys;
        units.rows_all = p.batch.T * p.group, units.pair_tiles = (units.rows_all + kPfxRows - 1) / kPfxRows;
    }

    if (warp == 0) {
        // ---- copies: K then V of every tile, page by page
        int n = 0, tails = 0, done = 0, told = 0;
        // (a place is free when the products and both groups have read it: a group that has no rows in the units which follow one
        // holds up no copy, and would find a later unit's description)
        const auto tell = [&](const TcUnit& u) {
            const int slot = told % kPfxUnits;
            if (told >= kPfxUnits && !mbar_wait_warp(bar_ufree + slot * 8, (told / kPfxUnits & 1) ^ 1)) return false;
            if (lane == 0) {
                const int4* const from = reinterpret_cast<const int4*>(&u);
                s_unit[slot * 3] = from[0], s_unit[slot * 3 + 1] = from[1], s_unit[slot * 3 + 2] = from[2];
                mbar_arrive(bar_u + slot * 8);
            }
            ++told;
            return true;
        };
        TcUnit u = {};
        while (ok && units.next(p, u)) {
        if (!tell(u)) {
            ok = false, where = 13;
            break;
        }
        const PageList pages = page_list(p.batch, u.b);
        for (int r = lane; r < u.rows; r += 32) {                              // the unit's queries towards L2
            const int j = (int)p.by_group.of((unsigned)(u.row0 + r)), g = u.row0 + r - j * p.group;
            const char* src = (const char*)((const __nv_bfloat16*)p.q + (u.first + j) * p.q_t + (int64_t)(u.h * p.group + g) * p.q_h);
#pragma unroll
            for (int c = 0; c < D * 2; c += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(src + c));
        }
        for (int tile = u.tile0; tile < u.tile0 + u.count && ok; ++tile, ++done) {
            const int key0 = tile * kPfxKeys, boxes = kPfxKeys >> pp.box_shift, h = u.h;
            const int limit = min(kPfxKeys, u.hi - key0);                      // keys of the tile that there are
            long long page = -1;
            int at = 0;
            if (lane < boxes && lane * pp.box_rows < limit) {
                const int key = key0 + lane * pp.box_rows, slot = (int)p.by_page.of((unsigned)key);
                at = key - slot * p.batch.page;
                if (slot < pages.n) page = __ldg(pages.pages + slot);
                if (page < 0 || page >= p.batch.n_pages) page = -1;
            }
            const uint32_t mask = __ballot_sync(0xFFFFFFFFu, page >= 0);
            const bool whole = limit == kPfxKeys && __popc(mask) == boxes;
            if (lane == 0) s_mask[done % kPfxMasks] = mask;
            for (int which = 0; which < 2 && ok; ++which, ++n) {
                const int st = n % S::kStages, round = n / S::kStages;
                if (round > 0 && !mbar_wait_warp(bar_free + st * 8, (round & 1) ^ 1)) {
                    ok = false, where = 1;
                    break;
                }
                const uint32_t dst = ring + st * S::kTileBytes;
                const bool slow = which == 1 && !whole;                        // values that have to be zeroed
                const uint32_t bar = slow ? bar_tail : bar_full + st * 8;
                if (lane == 0) mbar_expect_tx(bar, (uint32_t)__popc(mask) * pp.box_rows * D * 2);
                __syncwarp();
                if (page >= 0) {
                    const CUtensorMap* tm = which ? &tmV : &tmK;
#pragma unroll
                    for (int c = 0; c < kHalves; ++c)
                        tma_load_4d(dst + c * (kPfxKeys * 128) + lane * pp.box_rows * 128, tm, 0, at, c, (int)page * p.kv_heads + h, bar);
                }
                __syncwarp();
                if (slow) {
                    if (!mbar_wait_warp(bar_tail, tails & 1)) {
                        ok = false, where = 2;
                        break;
                    }
                    ++tails;
                    for (int r = 0; r < kPfxKeys; ++r) {
                        if (r < limit && (mask >> (r >> pp.box_shift) & 1u)) continue;
                        if (lane < kHalves * 8)
                            *reinterpret_cast<uint4*>(base_ptr + (dst - base) + (lane >> 3) * (kPfxKeys * 128) + r * 128 + (lane & 7) * 16) =
                                make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_full + st * 8);
                }
            }
        }
        }
        u.id = -1;
        if (ok && !tell(u)) ok = false, where = 13;                            // (without it the others' waits run out)
        if (!ok)                                                               // copies in flight land before the CTA leaves
            for (int q = max(0, n - S::kStages); q < n; ++q) mbar_wait_warp(bar_full + (q % S::kStages) * 8, (q / S::kStages) & 1);
    } else if (warp == 1) {
        // ---- products
        const uint32_t idesc_s = instr_desc_bf16(kPfxKeys), idesc_o = instr_desc_bf16(D) | (1u << 16);
        int n = 0, tiles_of[2] = {0, 0}, segs_of[2] = {0, 0}, heard = 0;
        auto scores = [&](int i, uint32_t k_tile) {
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < D / kUmmaK; ++kk) {
                    const uint32_t off = (kk >> 2) * (kPfxKeys * 128);
                    umma_bf16(tmem + i * 128, smem_desc_sw128(s_q + i * S::kTileBytes + off) + (uint64_t)((kk & 3) * 2),
                              smem_desc_sw128(k_tile + off) + (uint64_t)((kk & 3) * 2), idesc_s, kk != 0);
                }
                umma_commit(bar_s + i * 8);
            }
            __syncwarp();
        };
        auto sums = [&](int i, uint32_t v_tile, bool first) {
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < kPfxKeys / kUmmaK; ++kk) {
                    // 16 keys: two groups of eight rows of 128 bytes, 1024 apart; the next 64 entries a half tile on
                    const uint64_t db = (smem_desc_sw128(v_tile + kk * 2048) & ~((uint64_t)0x3FFF << 16)) | ((uint64_t)((kPfxKeys * 128) >> 4) << 16);
                    umma_bf16_ts(tmem + 256 + i * 128, tmem + i * 128 + kk * 8, db, idesc_o, !(first && kk == 0));
                }
            }
            __syncwarp();
        };
        auto release = [&](int stage) {
            if (elect_one()) umma_commit(bar_free + stage * 8);
            __syncwarp();
        };
        auto wait_full = [&](int i) { return mbar_wait_warp(bar_full + (i % S::kStages) * 8, (i / S::kStages) & 1); };
        while (ok) {
            ok = mbar_wait_warp(bar_u + heard % kPfxUnits * 8, heard / kPfxUnits & 1);
            if (!ok) {
                where = 11;
                break;
            }
            const TcUnit& u = reinterpret_cast<const TcUnit*>(s_unit)[heard % kPfxUnits];
            const int count = u.count, active = u.rows > 128 ? 2 : 1;
            if (u.id < 0) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_ufree + heard % kPfxUnits * 8);
            ++heard;
            ok = wait_full(n);
            for (int i = 0; i < active && ok; ++i) ok = mbar_wait_warp(bar_q + i * 8, segs_of[i] & 1);
            if (!ok) {
                where = 3;
                break;
            }
            tc_fence_after();
            for (int i = 0; i < active; ++i) scores(i, ring + n % S::kStages * S::kTileBytes);
            release(n % S::kStages);
            for (int j = 0; j < count && ok; ++j, n += 2) {
                ok = wait_full(n + 1) && (j + 1 == count || wait_full(n + 2));
                const uint32_t v_tile = ring + (n + 1) % S::kStages * S::kTileBytes, k_next = ring + (n + 2) % S::kStages * S::kTileBytes;
                for (int i = 0; i < active && ok; ++i) {
                    if (j == 0 && segs_of[i] > 0) ok = mbar_wait_warp(bar_ofree + i * 8, (segs_of[i] - 1) & 1);
                    ok = ok && mbar_wait_warp(bar_p + i * 8, tiles_of[i] & 1);
                    if (!ok) break;
                    tc_fence_after();
                    ++tiles_of[i];
                    sums(i, v_tile, j == 0);
                    if (j + 1 < count) {
                        scores(i, k_next);
                    } else {
                        if (elect_one()) umma_commit(bar_o + i * 8);
                        __syncwarp();
                    }
                }
                if (!ok) {
                    where = 4;
                    break;
                }
                release((n + 1) % S::kStages);
                if (j + 1 < count) release((n + 2) % S::kStages);
            }
            for (int i = 0; i < active; ++i) ++segs_of[i];
        }
    } else {
        // ---- softmax: four groups of four warps, (tile of rows, half of the keys); a warp's TMEM lanes are those of its number mod 4
        const int i = (warp - 2) >> 3, half = (warp - 2) >> 2 & 1, quad = warp & 3;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint32_t t_s = tmem + lanes + i * 128, t_o = tmem + lanes + 256 + i * 128;
        const uint32_t bar_pair = bar_x + (i * 4 + quad) * 8;
        volatile uint32_t* const grow_mine = s_grow + (i * 2 + half) * 4 + quad;
        volatile uint32_t* const grow_other = s_grow + (i * 2 + 1 - half) * 4 + quad;
        constexpr int kCols = kPfxKeys / 2, kPart = D / 4;         // scores of a thread; entries of O that leave at a time
        int tiles = 0, segs = 0, done = 0, pairs = 0, heard = 0;
        // The two warps of 32 rows wait for each other.
        auto meet = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_pair);
            const bool met = mbar_wait_warp(bar_pair, pairs & 1);
            ++pairs;
            return met;
        };
        while (ok) {
            ok = mbar_wait_warp(bar_u + heard % kPfxUnits * 8, heard / kPfxUnits & 1);
            if (!ok) {
                where = 12;
                break;
            }
            const TcUnit u = reinterpret_cast<const TcUnit*>(s_unit)[heard % kPfxUnits];
            if (u.id < 0) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_ufree + heard % kPfxUnits * 8);
            ++heard;
            const int count = u.count, h = u.h;
            if (i == 1 && u.rows <= 128) {                                     // no rows for the second tile
                done += count;
                continue;
            }
            const int row = i * 128 + quad * 32 + lane, lim = min(u.hi, row < u.rows ? u.limit(p, row) : 0);     // keys this row sees
            const int lim_all = u.limit(p, 0);                                 // and the first one, so all of them
            // queries: a warp 16 of the 32 rows, each row's chunks by neighbouring lanes
            {
                constexpr int kChunks = D / 8, kAtOnce = 32 / kChunks;
                const uint32_t flip = pp.sign < 0 ? 0x80008000u : 0u;
                const int c = lane % kChunks;
                uint4 v[16 / kAtOnce];
#pragma unroll
                for (int q = 0; q < 16 / kAtOnce; ++q) {
                    const int at = i * 128 + quad * 32 + half * 16 + q * kAtOnce + lane / kChunks;
                    v[q] = make_uint4(0u, 0u, 0u, 0u);
                    if (at < u.rows) {
                        const int j = (int)p.by_group.of((unsigned)(u.row0 + at)), g = u.row0 + at - j * p.group, t = u.first + j;
                        const __nv_bfloat16* src = (const __nv_bfloat16*)p.q + t * p.q_t + (int64_t)(h * p.group + g) * p.q_h + c * 8;
                        if (((uintptr_t)src & 15) == 0) {
                            v[q] = *reinterpret_cast<const uint4*>(src);
                        } else {
                            __nv_bfloat16 e[8];
#pragma unroll
                            for (int y = 0; y < 8; ++y) e[y] = src[y];
                            memcpy(&v[q], e, 16);
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < 16 / kAtOnce; ++q) {
                    const int rr = quad * 32 + half * 16 + q * kAtOnce + lane / kChunks;
                    if (pp.sign == 0) v[q] = make_uint4(times_zero(v[q].x), times_zero(v[q].y), times_zero(v[q].z), times_zero(v[q].w));
                    v[q].x ^= flip, v[q].y ^= flip, v[q].z ^= flip, v[q].w ^= flip;
                    *reinterpret_cast<uint4*>(base_ptr + i * S::kTileBytes + (c >> 3) * (kPfxKeys * 128) + rr * 128 + (((c & 7) ^ (rr & 7)) << 4)) = v[q];
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_q + i * 8);
            }
            float ref = -INFINITY, l = 0.f;
            for (int j = 0; j < count; ++j, ++tiles, ++done) {
                if (!mbar_wait_warp(bar_s + i * 8, tiles & 1)) {
                    ok = false, where = 5;
                    break;
                }
                tc_fence_after();
                const uint32_t mask = s_mask[done % kPfxMasks];
                const int key0 = (u.tile0 + j) * kPfxKeys + half * kCols;       // of this half
                float s[kCols];
                tmem_ld32(t_s + half * kCols, s);
                tmem_ld32(t_s + half * kCols + 32, s + 32);
                tmem_wait_ld();
                if (key0 + kCols > lim_all) {                                  // keys that this row does not see
                    const int n = lim - key0;
#pragma unroll
                    for (int k = 0; k < kCols; ++k) s[k] = k < n ? s[k] : -INFINITY;
                }
                if (__popc(mask) < (kPfxKeys >> pp.box_shift)) {               // keys of pages that are not there
#pragma unroll
                    for (int k = 0; k < kCols; k += 8)
                        if (!(mask >> ((half * kCols + k) >> pp.box_shift) & 1u))
#pragma unroll
                            for (int q = 0; q < 8; ++q) s[k + q] = -INFINITY;
                }
                float top[2] = {max3(s[0], s[2], s[4]), max3(s[1], s[3], s[5])};
#pragma unroll
                for (int k = 6; k + 3 < kCols; k += 4) {
                    top[0] = max3(top[0], s[k], s[k + 2]);
                    top[1] = max3(top[1], s[k + 1], s[k + 3]);
                }
                float high = max3(top[0], top[1], fmaxf(s[kCols - 2], s[kCols - 1])) * p.scale_log2;
                bool grow = high > ref + 8.f || (ref == -INFINITY && high > -INFINITY);
                const bool any = __any_sync(0xFFFFFFFFu, grow);
                if (lane == 0) *grow_mine = any;
                tc_fence_before();
                ok = meet();                                                   // (and both have their scores: the weights may take their place)
                tc_fence_after();
                if (ok && (any || *grow_other)) {                              // (the same on both sides)
                    tmem_st1(t_s + 64 + half, high);
                    tmem_wait_st();
                    tc_fence_before();
                    ok = meet();
                    tc_fence_after();
                    high = fmaxf(high, tmem_ld1(t_s + 65 - half));
                    grow = high > ref + 8.f || (ref == -INFINITY && high > -INFINITY);
                    const float f = grow ? exp2_fast(ref - high) : 1.f;
                    l *= f;
                    if (j > 0 && ok) {                                         // this half of the entries of O
#pragma unroll
                        for (int c = 0; c < D / 2; c += 16) {
                            uint32_t w[16];
                            float o[16];
                            tmem_ld16(t_o + half * (D / 2) + c, o);
#pragma unroll
                            for (int q = 0; q < 16; ++q) w[q] = __float_as_uint(o[q] * f);
                            tmem_st16(t_o + half * (D / 2) + c, w);
                        }
                    }
                    if (grow) ref = high;
                }
                if (!ok) {
                    where = 7;
                    break;
                }
                const float m = ref == -INFINITY ? 0.f : ref;
                const unsigned long long sc2 = pair2(p.scale_log2, p.scale_log2), m2 = pair2(-m, -m);
                unsigned long long sum2[2] = {0ull, 0ull};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int q = 0; q < 16; ++q) {
                        float a, b;
                        unpair2(fma2_of(pair2(s[c * 32 + 2 * q], s[c * 32 + 2 * q + 1]), sc2, m2), a, b);
                        a = exp2_fast(a);
                        b = exp2_fast(b);
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[q]) : "f"(b), "f"(a));
                        add2(sum2[q & 1], bf16x2_to_f32x2(w[q]));
                    }
                    tmem_st16(t_s + half * 32 + c * 16, w);
                }
                add2(sum2[0], sum2[1]);
                float a, b;
                unpair2(sum2[0], a, b);
                l += a + b;
                tmem_wait_st();
                if (kOwn && lim_all < u.hi && (u.tile0 + j + 1) * kPfxKeys > lim_all) {
                    // keys that some rows do not see: values that are no finite numbers become zeros (by both tiles of rows alike)
                    const int st = (2 * done + 1) % S::kStages;
                    if (!mbar_wait_warp(bar_full + st * 8, (2 * done + 1) / S::kStages & 1)) {
                        ok = false, where = 10;
                        break;
                    }
                    uint4* const v = reinterpret_cast<uint4*>(base_ptr + (ring - base) + st * S::kTileBytes);
                    for (int e = (half * 4 + quad) * 32 + lane; e < S::kTileBytes / 16; e += 256) {
                        uint4 x = v[e];
                        uint32_t* const w = reinterpret_cast<uint32_t*>(&x);
                        bool odd = false;
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            if ((w[q] & 0x7F80u) == 0x7F80u) w[q] &= 0xFFFF0000u, odd = true;
                            if ((w[q] & 0x7F800000u) == 0x7F800000u) w[q] &= 0xFFFFu, odd = true;
                        }
                        if (odd) {                                             // (the other tile of rows finds zeros: it sees the word before them)
                            s_odd[(heard - 1) % kPfxOdd] = (uint32_t)u.id + 1u;
                            __threadfence_block();
                            v[e] = x;
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_p + i * 8);
            }
            if (!ok) break;
            if (!mbar_wait_warp(bar_o + i * 8, segs & 1)) {
                ok = false, where = 6;
                break;
            }
            tc_fence_after();
            // kPart entries at a time through the place of the queries, so that a store is whole lines of several rows; a
            // thread's own row straight from its registers takes 32 of them
            const size_t piece = (size_t)(u.id + (int)blockIdx.x) * kPfxRows + i * 128 + quad * 32;
            const int rows_here = u.id + (int)blockIdx.x < space.pieces ? min(32, u.rows - i * 128 - quad * 32) : 0;
            // the row's sum: the halves' sums through a column of TMEM that no product uses any more
            if (half == 1) {
                tmem_st1(t_s + 64, l);
                tmem_wait_st();
            }
            tc_fence_before();
            if (!meet()) {
                ok = false, where = 8;
                break;
            }
            tc_fence_after();
            if (half == 0) {
                l += tmem_ld1(t_s + 64);
                if (lane < rows_here) space.ml[piece + lane] = make_float2(ref, l);
            }
            uint8_t* const turn = base_ptr + i * S::kTileBytes + (D == 128 ? half * (kPfxKeys * 128) : half * 2048) + quad * 4096;
            constexpr int kQuads = kPart / 4, kRowsAtOnce = 32 / kQuads;       // 16-byte pieces of a row
#pragma unroll
            for (int c = 0; c < D / 2; c += kPart) {
                float o[kPart];
#pragma unroll
                for (int q = 0; q < kPart; q += 16) tmem_ld16(t_o + half * (D / 2) + c + q, *reinterpret_cast<float(*)[16]>(o + q));
                if (kOwn && s_odd[(heard - 1) % kPfxOdd] == (uint32_t)u.id + 1u) {     // what was zeroed, to the rows that see it
                    const PageList pages = page_list(p.batch, u.b);
                    const int from = max(u.tile0, lim_all / kPfxKeys) * kPfxKeys, to = min(lim, (u.tile0 + count) * kPfxKeys);
                    for (int key = from; key < to; ++key) {
                        const long long at = key_row(pages, p.batch, p.by_page, key, p.kv_heads, h);
                        const __nv_bfloat16* v = (const __nv_bfloat16*)p.v + at * D + half * (D / 2) + c;
                        for (int q = 0; at >= 0 && q < kPart; q += 2) {
                            const uint32_t w = *reinterpret_cast<const uint32_t*>(v + q);
                            const float a = (w & 0x7F80u) == 0x7F80u ? __uint_as_float(w << 16) : 0.f;
                            const float b = (w & 0x7F800000u) == 0x7F800000u ? __uint_as_float(w & 0xFFFF0000u) : 0.f;
                            if (a != 0.f || b != 0.f) {
#pragma unroll
                                for (int e = 0; e < kPart; e += 2)
                                    if (e == q) o[e] += a, o[e + 1] += b;
                            }
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < kQuads; ++q)
                    *reinterpret_cast<float4*>(turn + lane * (kPart * 4) + ((q ^ (lane & (kQuads - 1))) << 4)) =
                        make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
                __syncwarp();
#pragma unroll
                for (int q = 0; q < kQuads; ++q) {
                    const int rr = q * kRowsAtOnce + lane / kQuads, e = lane % kQuads;
                    const float4 v = *reinterpret_cast<const float4*>(turn + rr * (kPart * 4) + ((e ^ (rr & (kQuads - 1))) << 4));
                    if (rr < rows_here) *reinterpret_cast<float4*>(space.o + (piece + rr) * D + half * (D / 2) + c + e * 4) = v;
                }
                __syncwarp();
            }
            tc_fence_before();
            if (!meet()) {                                                     // (the other half's queries may take this one's place)
                ok = false, where = 9;
                break;
            }
            if (lane == 0) mbar_arrive(bar_ofree + i * 8);
            ++segs;
        }
    }
    if (!ok && where && lane == 0) {
        atomicExch(p.status, 1);
        atomicExch(p.status + 1, 4500 + where);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    launch_ends(p);
}

}  // namespace meteora
