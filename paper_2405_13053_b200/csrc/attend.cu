// Attention for a batch whose sequences share a prefix, over a paged cache: the plan of a call and its launches.
#include <algorithm>

#include "attend_ops.cuh"
#include "attend_simt.cuh"
#include "launch_heads.cuh"

namespace meteora {

// A row's pieces of one launch: the first one's row, and how many there are, `rows` of the space apart.
struct RowPieces {
    long long row;
    int n;
};
__device__ __forceinline__ RowPieces row_pieces(const PieceSpace& s, int W, uint32_t x0, int tiles, int unit, int r) {
    if (tiles <= 0 || W <= 0) return RowPieces{0, 0};
    const Shares shares((uint32_t)W, share_count(s, (uint32_t)W));
    const int c0 = (int)shares.of(x0), n = (int)shares.of(x0 + (uint32_t)tiles - 1) - c0 + 1;
    const bool there = unit + c0 >= 0 && (long long)unit + c0 + n <= s.pieces;    // (a cu_tokens that does not ascend)
    return RowPieces{there ? (long long)(unit + c0) * s.rows + r : 0, there ? n : 0};
}

// Whether any page of the prefix or of the first `seen` own tokens of sequence b is there, by a whole warp.  (Not inlined: rare, and five registers of
// the join otherwise, 280 instead of 276 us for 880 tokens of 40 heads.)
__device__ __noinline__ bool sees_keys(const AttendParams& p, int b, int seen, int lane) {
    bool any = false;
    for (int which = 0; which < 2 && !any; ++which) {
        const PageList l = page_list(p.batch, which ? b : -1);
        const int n = which ? min(l.n, (int)(((long long)seen + p.batch.page - 1) / p.batch.page)) : l.n;
        for (int i = lane; i < n && !any; i += 32) {
            const int page = __ldg(l.pages + i);
            any = page >= 0 && page < p.batch.n_pages;
        }
        any = __any_sync(0xFFFFFFFFu, any);
    }
    return any;
}

// The pieces of one token's heads joined, kAhead of them at a time, by a running maximum like the pieces themselves, in their
// order.  kWarps == 1: a warp takes `heads_each` heads one after the other (a lane works out each one's pieces beforehand).
// kWarps > 1, where the rows are too few to hide one another's latency: a CTA per row, warp w joins pieces w, w + kWarps,
// ..., then the warps in order.  kWide: heads of more than 128 entries.
template <typename E, int kWarps, bool kWide>
__global__ void __launch_bounds__(kWarps == 1 ? 128 : 32 * kWarps) k_attend_join(const __grid_constant__ AttendParams p, const int heads_each) {
    constexpr int kParts = kWide ? 2 : 1, kAhead = kWide ? 4 : 8;
    __shared__ float4 s_acc[kWarps == 1 ? 1 : kWarps][32 * kParts];
    __shared__ float2 s_ml[kWarps == 1 ? 1 : kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = kWarps == 1 ? 0 : warp;
    const int t = blockIdx.x, h0 = (kWarps == 1 ? (int)blockIdx.y * 4 + warp : (int)blockIdx.y) * heads_each;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (h0 >= p.q_heads) return;
    const int b = sequence_of(p.batch, t, lane);
    if (b < 0) return;
    const int W0 = p.prefix.total >= 0 ? p.prefix.total : p.total[0], W1 = p.total[1], first_tile = p.first_tile[b], first_unit = p.first_unit[b];
    const SequenceView s = sequence_view(p.batch, b);
    if (s.held < 0 || t >= s.first + s.tokens) return;
    const int seen = min(s.held + (t - s.first) + 1, s.all);
    RowPieces early = {}, late = {};
    if (lane < heads_each && h0 + lane < p.q_heads) {
        const int h = h0 + lane, kv = (int)p.by_group.of((unsigned)h), g = h - kv * p.group;
        if (p.batch.prefix > 0) {
            const int i = t * p.group + g, rt = (int)((unsigned)i / (unsigned)p.prefix.rows), n_rt = row_tiles(p, p.batch.T, p.prefix.rows);
            const int tiles = (p.batch.prefix + (1 << p.prefix.shift) - 1) >> p.prefix.shift;
            const int unit = p.tc ? kv * n_rt + rt : rt * p.kv_heads + kv;
            early = row_pieces(p.prefix, W0, (uint32_t)unit * (uint32_t)tiles, tiles, unit, i - rt * p.prefix.rows);
        }
        if (seen > 0) {
            const int i = (t - s.first) * p.group + g, rt = (int)((unsigned)i / (unsigned)p.own.rows), in = rt * p.kv_heads + kv;
            const int up = (1 << p.own.shift) - 1;
            const uint32_t x0 = (uint32_t)first_tile + (uint32_t)in * (uint32_t)((s.all + up) >> p.own.shift);
            late = row_pieces(p.own, W1, x0, (seen + up) >> p.own.shift, first_unit + in, i - rt * p.own.rows);
        }
    }
    const bool quads = p.dim % 4 == 0;
    for (int head = 0; head < heads_each && h0 + head < p.q_heads; ++head) {
        const int h = h0 + head;
        const int early_n = __shfl_sync(0xFFFFFFFFu, early.n, head), n = early_n + __shfl_sync(0xFFFFFFFFu, late.n, head);
        const long long early_row = __shfl_sync(0xFFFFFFFFu, early.row, head), late_row = __shfl_sync(0xFFFFFFFFu, late.row, head);
        float M = -INFINITY, L = 0.f;
        float4 acc[kParts];
#pragma unroll
        for (int c = 0; c < kParts; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i0 = part; i0 < n; i0 += kAhead * kWarps) {
            float4 v[kAhead][kParts];
            float2 ml[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int i = i0 + a * kWarps;
                ml[a] = make_float2(-INFINITY, 0.f);
#pragma unroll
                for (int c = 0; c < kParts; ++c) v[a][c] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (i >= n) continue;
                const bool is_early = i < early_n;
                const long long row = is_early ? early_row + (long long)i * p.prefix.rows : late_row + (long long)(i - early_n) * p.own.rows;
                const float* o = (is_early ? p.prefix.o : p.own.o) + row * p.dim;
                ml[a] = (is_early ? p.prefix.ml : p.own.ml)[row];
#pragma unroll
                for (int c = 0; c < kParts; ++c) {
                    const int e = (lane + 32 * c) * 4;
                    if (e >= p.dim) continue;
                    if (quads) {
                        v[a][c] = *reinterpret_cast<const float4*>(o + e);
                    } else {
                        v[a][c].x = o[e];
                        if (e + 1 < p.dim) v[a][c].y = o[e + 1];
                        if (e + 2 < p.dim) v[a][c].z = o[e + 2];
                        if (e + 3 < p.dim) v[a][c].w = o[e + 3];
                    }
                }
            }
            float high = M;
#pragma unroll
            for (int a = 0; a < kAhead; ++a) high = fmaxf(high, ml[a].x);
            const float base = high == -INFINITY ? 0.f : high, f0 = M == -INFINITY ? (L != L ? L : 0.f) : exp2_fast(M - base);
            M = high;
            L = L * f0;
#pragma unroll
            for (int c = 0; c < kParts; ++c) acc[c] = make_float4(acc[c].x * f0, acc[c].y * f0, acc[c].z * f0, acc[c].w * f0);
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const float f = piece_factor(ml[a], base);           // (of 0 too: a value that is no number passes a weight next to nothing)
                L = fmaf(f, ml[a].y, L);
#pragma unroll
                for (int c = 0; c < kParts; ++c) {
                    acc[c].x = fmaf(f, v[a][c].x, acc[c].x);
                    acc[c].y = fmaf(f, v[a][c].y, acc[c].y);
                    acc[c].z = fmaf(f, v[a][c].z, acc[c].z);
                    acc[c].w = fmaf(f, v[a][c].w, acc[c].w);
                }
            }
        }
        if (kWarps > 1) {                                            // (one head)
#pragma unroll
            for (int c = 0; c < kParts; ++c) s_acc[part][lane + 32 * c] = acc[c];
            if (lane == 0) s_ml[part] = make_float2(M, L);
            __syncthreads();
            if (warp > 0) return;
            float high = -INFINITY;
#pragma unroll
            for (int x = 0; x < kWarps; ++x) high = fmaxf(high, s_ml[x].x);
            const float base = high == -INFINITY ? 0.f : high;
            M = high, L = 0.f;
#pragma unroll
            for (int c = 0; c < kParts; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int x = 0; x < kWarps; ++x) {
                if (x >= n) continue;
                const float f = piece_factor(s_ml[x], base);
                L = fmaf(f, s_ml[x].y, L);
#pragma unroll
                for (int c = 0; c < kParts; ++c) {
                    const float4 v = s_acc[x][lane + 32 * c];
                    acc[c] = make_float4(fmaf(f, v.x, acc[c].x), fmaf(f, v.y, acc[c].y), fmaf(f, v.z, acc[c].z), fmaf(f, v.w, acc[c].w));
                }
            }
        }
        // a row that sees nothing: zeros, and the logarithm of an empty sum; one that sees scores of -inf alone: 0 / 0
        float inv = 1.f / L;
        if (M == -INFINITY && L == 0.f) inv = sees_keys(p, b, seen, lane) ? NAN : 0.f;
        E* const out = (E*)p.out + t * p.out_t + h * p.out_h;
        const bool wide = quads && ((uintptr_t)p.out | (uintptr_t)(p.out_t * sizeof(E)) | (uintptr_t)(p.out_h * sizeof(E))) % (4 * sizeof(E)) == 0;
#pragma unroll
        for (int c = 0; c < kParts; ++c) {
            const int e = (lane + 32 * c) * 4;
            const float v[4] = {acc[c].x * inv, acc[c].y * inv, acc[c].z * inv, acc[c].w * inv};
            if (e >= p.dim) continue;
            if (wide) {
                const f32x2 pairs[2] = {make_pair2(v[0], v[1]), make_pair2(v[2], v[3])};
                HeadVec<E, 4>::store(out + e, HeadVec<E, 4>::pack(pairs));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (e + j < p.dim) {
                        if constexpr (sizeof(E) == 2) out[e + j] = __float2bfloat16_rn(v[j]);
                        else out[e + j] = v[j];
                    }
            }
        }
        if (p.lse && lane == 0) p.lse[(size_t)t * p.q_heads + h] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
    }
}

// ---------------------------------------------------------------------------------------------
// Plan
// ---------------------------------------------------------------------------------------------
struct AttendPlan {
    AttendParams p;                      // sizes, and the workspace's places from a null base
    bool mma, together;                  // matrix instructions; prefix and own tokens in one launch
    bool fits;                           // fewer than 2^31 tiles
    size_t bytes;
};

// The kernel that takes units of `rows` rows: its shared memory per CTA and, with 148 SMs, the workers that run at a time
// (4 CTAs of an SM at most, by registers).
static size_t pieces_smem(const AttendSizes& z, bool mma, int rows) {
    if (!mma) return attend_simt_bytes(z.head_dim);
    const bool wide = rows == 64;
    if (z.head_dim <= 64) return wide ? AttendMmaShape<64>::kBytes : AttendWarpShape<64>::kBytes;
    if (z.head_dim <= 128) return wide ? AttendMmaShape<128>::kBytes : AttendWarpShape<128>::kBytes;
    return wide ? AttendMmaShape<256>::kBytes : AttendWarpShape<256>::kBytes;
}
static void set_kernel(PieceSpace& s, const AttendSizes& z, bool mma) {
    const int ctas = 148 * std::max(1, std::min(4, (int)(228 * 1024 / (pieces_smem(z, mma, s.rows) + 1024))));
    const bool warps = mma && s.rows == kWarpRows;
    s.workers = warps ? 4 * ctas : ctas;
    s.shift = warps ? 4 : 6;
    s.least_shift = warps ? 1 : 0;               // (32 keys: a piece of fewer costs the join more than it saves)
    s.total = -1;
}

static AttendPlan plan_attend(const AttendSizes& z, void* workspace) {
    AttendPlan plan = {};
    AttendParams& p = plan.p;
    p.q_heads = z.q_heads;
    p.kv_heads = z.kv_heads;
    p.group = z.q_heads / z.kv_heads;
    p.dim = z.head_dim;
    p.by_group = fixed_div((uint32_t)p.group);
    p.by_page = fixed_div((uint32_t)z.page_size);
    plan.mma = z.dtype == METEORA_BF16 && z.head_dim % 8 == 0;
    const long long rows = (long long)z.T * p.group, mean = std::max(1, z.B > 0 ? z.T / z.B : 1);    // mean: new tokens of a sequence
    // More than 16 rows at a time: on the tensor cores where these take the shape, else 64; of the prefix all rows, of own
    // tokens a sequence's mean.  Own tokens of up to 64 rows per sequence stay with the 64-row kernel: a unit of the other
    // costs about 20 us / SM to start and end (us, own tokens alone, 64-row kernel / tensor cores: 16 sequences of 55 rows, 355
    // keys, 40 heads 79 / 108; 64 of 24 rows, 1024 keys, 40 heads 429 / 445; with 8 kv heads, 32 of 64 rows, 516 keys 56 / 80; 32
    // of 128 rows, 532 keys 83 / 83; 16 of 512 rows, 628 keys 143 / 95; 2 of 8000 rows, 2000 keys 598 / 215).
    p.tc = z.prefix_len > 0 && attend_tc_supported(z, rows);
    p.own_tc = mean * p.group > 64 && attend_tc_supported(z, mean * p.group);
    p.prefix.rows = p.tc ? kPrefixRows : plan.mma && rows > 16 ? 64 : 16;
    p.own.rows = p.own_tc ? kPrefixRows : plan.mma && mean * p.group > 16 ? 64 : 16;
    plan.together = !p.tc && z.prefix_len > 0 && p.prefix.rows == p.own.rows;
    const auto units = [&](int r) { return (rows + r - 1) / r * z.kv_heads; };
    size_t off = kHeaderBytes;
    const auto take = [&](size_t bytes) {
        uint8_t* at = workspace ? (uint8_t*)workspace + off : nullptr;
        off += align_up(bytes, 256);
        return at;
    };
    const auto space = [&](PieceSpace& s, long long n_units) {
        s.pieces = n_units + s.workers;
        s.o = (float*)take((size_t)s.pieces * s.rows * z.head_dim * 4);
        s.ml = (float2*)take((size_t)s.pieces * s.rows * 8);
    };
    const long long prefix_units = z.prefix_len > 0 ? units(p.prefix.rows) : 0;
    const auto set_tc = [](PieceSpace& s) {      // one CTA per SM
        s.shift = 7;
        s.least_shift = 0;
        s.workers = 148;
        s.total = -1;
    };
    if (p.own_tc) set_tc(p.own);
    else set_kernel(p.own, z, plan.mma);
    space(p.own, units(p.own.rows) + (long long)z.B * z.kv_heads + (plan.together ? prefix_units : 0));
    if (plan.together) {
        p.prefix = p.own;
    } else if (z.prefix_len > 0) {
        if (p.tc) {
            set_tc(p.prefix);
            p.prefix.total = (int)(prefix_units * ((z.prefix_len + kPrefixTile - 1) / kPrefixTile));
            // (two tiles each at least: 64 rows of 32 heads over 2048 keys, with 64 sequences' own tokens and the join, 44.8 us; one
            // each, 16 pieces for a row instead of 8, 49.3; four 49.4)
            p.prefix.workers = std::max(1, std::min(148, p.prefix.total >> 1));
        } else {
            set_kernel(p.prefix, z, plan.mma);
        }
        space(p.prefix, prefix_units);
    }
    p.total = (int32_t*)take(8);
    p.first_tile = (int32_t*)take((size_t)z.B * 4);
    p.first_unit = (int32_t*)take((size_t)z.B * 4);
    p.status = (int32_t*)workspace;
    plan.bytes = off;
    // tiles of a launch at most, by the tables' room
    const auto most = [&](const PieceSpace& s, long long n_units, long long keys) { return n_units * ((keys >> s.shift) + 1); };
    const long long own_most = most(p.own, units(p.own.rows) + (long long)z.B * z.kv_heads, (long long)z.table_width * z.page_size);
    plan.fits = own_most + (z.prefix_len > 0 ? most(p.prefix, prefix_units, z.prefix_len) : 0) < (1LL << 31);
    return plan;
}

size_t attend_workspace_bytes(const AttendSizes& z) {
    const AttendPlan plan = plan_attend(z, nullptr);
    return plan.fits ? plan.bytes : 0;
}

template <typename E>
static int launch_join(const AttendParams& p, cudaStream_t st) {
    const long long rows = (long long)p.batch.T * p.q_heads;
    // a CTA per SM at most: of 16 warps (us, the whole call with 8 / 16 / 32: one token of 16 heads over 16500 keys, 515 pieces a
    // row, 30.2 / 21.0 / 22.0; of 32 heads over 2085 keys 15.9 / 15.5 / 17.8)
    if (rows <= 148)
        return p.dim > 128 ? launch_dependent<k_attend_join<E, 16, true>>(dim3(p.batch.T, p.q_heads), 512, 0, st, p, 1)
                           : launch_dependent<k_attend_join<E, 16, false>>(dim3(p.batch.T, p.q_heads), 512, 0, st, p, 1);
    if (rows <= 1184)                            // 8 CTAs per SM
        return p.dim > 128 ? launch_dependent<k_attend_join<E, 8, true>>(dim3(p.batch.T, p.q_heads), 256, 0, st, p, 1)
                           : launch_dependent<k_attend_join<E, 8, false>>(dim3(p.batch.T, p.q_heads), 256, 0, st, p, 1);
    const int each = (int)std::max(1LL, std::min(32LL, rows / (148 * 24)));       // heads per warp: as many as leave every SM 24 warps
    const int warps = (p.q_heads + each - 1) / each;
    const dim3 grid(p.batch.T, (warps + 3) / 4);
    return p.dim > 128 ? launch_dependent<k_attend_join<E, 1, true>>(grid, 128, 0, st, p, each)
                       : launch_dependent<k_attend_join<E, 1, false>>(grid, 128, 0, st, p, each);
}

int launch_prefix_attention(const meteora_heads_t& q, const meteora_heads_t& out, float* lse, const meteora_cache_t& cache,
                            const BatchView& batch, const AttendSizes& z, float scale, void* workspace, cudaStream_t st) {
    AttendPlan plan = plan_attend(z, workspace);
    AttendParams& p = plan.p;
    p.batch = batch;
    p.q = q.data;
    p.q_t = q.stride_token;
    p.q_h = q.stride_head;
    p.out = out.data;
    p.out_t = out.stride_token;
    p.out_h = out.stride_head;
    p.lse = lse;
    p.k = cache.k;
    p.v = cache.v;
    p.scale_log2 = scale * 1.4426950408889634f;
    const auto pieces = [&](bool prefix, bool own) -> int {
        AttendParams a = p;
        a.with_prefix = prefix;
        a.with_own = own;
        a.here = own ? p.own : p.prefix;
        a.beside = own && !prefix && z.prefix_len > 0;
        if (own ? p.own_tc : p.tc) return launch_attend_tc(a, own, st);
        if (plan.mma) return launch_attend_warps(a, p.dim <= 64 ? 64 : p.dim <= 128 ? 128 : 256, st);
        if (z.dtype == METEORA_BF16) return launch_dependent<k_attend_simt<__nv_bfloat16>>(dim3(a.here.workers), 128, attend_simt_bytes(p.dim), st, a);
        return launch_dependent<k_attend_simt<float>>(dim3(a.here.workers), 128, attend_simt_bytes(p.dim), st, a);
    };
    int rc = METEORA_OK;
    if (z.prefix_len > 0 && !plan.together) rc = pieces(true, false);
    if (rc == METEORA_OK) rc = pieces(plan.together, true);
    if (rc != METEORA_OK) return rc;
    return z.dtype == METEORA_BF16 ? launch_join<__nv_bfloat16>(p, st) : launch_join<float>(p, st);
}

}  // namespace meteora
