// Attention for a batch whose sequences share a prefix, over a paged cache: the plan of a call and its launches.
#include <algorithm>

#include "attend_mma.cuh"
#include "attend_simt.cuh"
#include "launch_heads.cuh"

namespace meteora {

// A row's slots joined, one warp per row: the common maximum first, then sums in the order of the slots.
template <typename E>
__global__ void __launch_bounds__(128) k_attend_join(const __grid_constant__ AttendParams p) {
    const int lane = threadIdx.x & 31;
    const size_t all_rows = (size_t)p.batch.T * p.q_heads;
    const size_t row = (size_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (row >= all_rows) return;
    const int t = (int)(row / p.q_heads), h = (int)(row - (size_t)t * p.q_heads);
    const int b = sequence_of(p.batch, t, lane);
    if (b < 0) return;
    const SequenceView s = sequence_view(p.batch, b);
    if (s.held < 0) return;
    const int all = (int)min((long long)s.held + s.tokens, table_keys(p.batch));
    const int seen = (int)min((long long)s.held + (t - s.first) + 1, (long long)all);
    const int piece = own_piece(all, p.own_slots, p.own_min);
    int early = p.prefix_slots;                                      // pieces of the prefix, then those of the own tokens
    if (p.tc.ctas > 0) {
        const int kv = h / p.group, tiles = p.tc.units / p.kv_heads;
        const long long x = ((long long)kv * tiles + ((long long)t * p.group + h - kv * p.group) / kPrefixRows) * p.tc.tiles;
        early = share_of(p.tc, x + p.tc.tiles - 1) - share_of(p.tc, x) + 1;
    }
    const int slots = early + (seen + piece - 1) / piece, skip = p.prefix_slots - early;
    float M = -INFINITY;
    for (int i = lane; i < slots; i += 32) M = fmaxf(M, p.part_ml[(i + (i < early ? 0 : skip)) * all_rows + row].x);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, x));
    const float base = M == -INFINITY ? 0.f : M;
    const bool quads = p.dim % 4 == 0;
    float L = 0.f;
    float4 acc[2] = {};
    for (int i0 = 0; i0 < slots; i0 += 32) {
        float2 ml = make_float2(-INFINITY, 0.f);
        if (i0 + lane < slots) ml = p.part_ml[(i0 + lane + (i0 + lane < early ? 0 : skip)) * all_rows + row];
        const float w = piece_factor(ml, base);
        const int n = min(32, slots - i0);
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            const float f = __shfl_sync(0xFFFFFFFFu, w, i), fl = __shfl_sync(0xFFFFFFFFu, ml.y, i);
            if (f == 0.f) continue;              // (a piece in which the row sees nothing; NaN goes on)
            L = fmaf(f, fl, L);
            const float* o = p.part_o + ((i0 + i + (i0 + i < early ? 0 : skip)) * all_rows + row) * p.dim;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int e = (lane + 32 * c) * 4;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (quads) {
                    if (e < p.dim) v = *reinterpret_cast<const float4*>(o + e);
                } else {
                    if (e < p.dim) v.x = o[e];
                    if (e + 1 < p.dim) v.y = o[e + 1];
                    if (e + 2 < p.dim) v.z = o[e + 2];
                    if (e + 3 < p.dim) v.w = o[e + 3];
                }
                acc[c].x = fmaf(f, v.x, acc[c].x);
                acc[c].y = fmaf(f, v.y, acc[c].y);
                acc[c].z = fmaf(f, v.z, acc[c].z);
                acc[c].w = fmaf(f, v.w, acc[c].w);
            }
        }
    }
    // a row that sees nothing: zeros, and the logarithm of an empty sum
    const float inv = M == -INFINITY && L == 0.f ? 0.f : 1.f / L;
    E* const out = (E*)p.out + t * p.out_t + h * p.out_h;
    const bool wide = quads && ((uintptr_t)p.out | (uintptr_t)(p.out_t * sizeof(E)) | (uintptr_t)(p.out_h * sizeof(E))) % (4 * sizeof(E)) == 0;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int e = (lane + 32 * c) * 4;
        const float v[4] = {acc[c].x * inv, acc[c].y * inv, acc[c].z * inv, acc[c].w * inv};
        if (e >= p.dim) continue;
        if (wide) {
            HeadVec<E, 4>::store(out + e, HeadVec<E, 4>::pack(v));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e + j < p.dim) {
                    if constexpr (sizeof(E) == 2) out[e + j] = __float2bfloat16_rn(v[j]);
                    else out[e + j] = v[j];
                }
        }
    }
    if (p.lse && lane == 0) p.lse[row] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------------------------------------
// Plan
// ---------------------------------------------------------------------------------------------
constexpr int kTargetCtas = 296;         // two CTAs per SM
constexpr int kMaxOwnItems = 8192;       // a piece that its sequence does not reach is a CTA that leaves at once

struct AttendPlan {
    AttendParams p;                      // sizes, tiles, pieces
    bool mma;
    int dp;                              // entries of a head as the matrix kernel pads them
    int wide[2];                         // 64 rows a tile for the prefix / own tokens
    size_t slots;
};

static void set_tile(AttendParams& p, int which, int rows, int tokens) {
    p.tile_heads[which] = std::min(p.group, rows);
    p.tile_tokens[which] = std::max(1, std::min(rows / p.tile_heads[which], std::max(1, tokens)));
    p.t_tiles[which] = std::max(1, (int)(((long long)p.batch.T + p.tile_tokens[which] - 1) / p.tile_tokens[which]));   // (T = 0: sizes only)
    p.g_tiles[which] = (p.group + p.tile_heads[which] - 1) / p.tile_heads[which];
}

static AttendPlan plan_attend(const AttendSizes& z) {
    AttendPlan plan = {};
    AttendParams& p = plan.p;
    p.q_heads = z.q_heads;
    p.kv_heads = z.kv_heads;
    p.group = z.q_heads / z.kv_heads;
    p.dim = z.head_dim;
    p.batch.B = z.B;
    p.batch.T = z.T;
    p.batch.width = z.table_width;
    p.batch.page = z.page_size;
    p.batch.prefix = z.prefix_len;
    plan.mma = z.dtype == METEORA_BF16 && z.head_dim % 8 == 0;
    plan.dp = z.head_dim <= 64 ? 64 : z.head_dim <= 128 ? 128 : 256;
    const int mean = std::max(1, z.B > 0 ? z.T / z.B : 1);          // new tokens per sequence
    plan.wide[0] = plan.mma && (long long)z.T * p.group > 16;
    plan.wide[1] = plan.mma && (long long)mean * p.group > 16;
    set_tile(p, 0, plan.wide[0] ? 64 : 16, z.T);
    set_tile(p, 1, plan.wide[1] ? 64 : 16, mean);
    const auto round_up = [](long long v) { return (v + kAttendTile - 1) / kAttendTile * kAttendTile; };
    if (prefix_tc_supported(z)) {
        // even shares of whole tiles: no more CTAs than SMs, and pieces of two tiles at least where there are as many
        const long long tiles_of_rows = ((long long)z.T * p.group + kPrefixRows - 1) / kPrefixRows;
        p.tc.units = (int)(tiles_of_rows * p.kv_heads);
        p.tc.tiles = (z.prefix_len + 127) / 128;
        p.tc.ctas = (int)std::max(1LL, std::min(148LL, (long long)p.tc.units * p.tc.tiles));
        for (int u = 0; u < p.tc.units; ++u) {
            const long long x = (long long)u * p.tc.tiles;
            p.prefix_slots = std::max(p.prefix_slots, share_of(p.tc, x + p.tc.tiles - 1) - share_of(p.tc, x) + 1);
        }
    } else if (z.prefix_len > 0) {
        const long long units = (long long)p.kv_heads * p.t_tiles[0] * p.g_tiles[0];
        const long long want = std::max(1LL, std::min({(kTargetCtas + units - 1) / units, round_up(z.prefix_len) / kAttendTile, 64LL}));
        p.prefix_piece = (int)round_up((z.prefix_len + want - 1) / want);
        p.prefix_slots = (z.prefix_len + p.prefix_piece - 1) / p.prefix_piece;
    }
    const long long keys = (long long)z.table_width * z.page_size, units = (long long)p.kv_heads * p.t_tiles[1] * p.g_tiles[1];
    p.own_min = (int)std::min(512LL, std::max((long long)kAttendTile, round_up(keys * units / kTargetCtas)));
    p.own_slots = (int)std::max(1LL, std::min({(keys + p.own_min - 1) / p.own_min, std::max(8LL, kMaxOwnItems / units), 64LL}));
    plan.slots = (size_t)p.prefix_slots + (keys > 0 ? p.own_slots : 0);
    return plan;
}

size_t attend_workspace_bytes(const AttendSizes& z) {
    const AttendPlan plan = plan_attend(z);
    const size_t rows = plan.slots * z.T * z.q_heads;
    return kHeaderBytes + align_up(rows * z.head_dim * 4, 256) + align_up(rows * 8, 256);
}

template <int DP>
static int launch_mma(bool wide, const AttendParams& p, cudaStream_t st) {
    if (wide) return launch_dependent<k_attend_mma<DP, 4>>(dim3((unsigned)p.items), 128, AttendMmaShape<DP, 4>::kBytes, st, p);
    return launch_dependent<k_attend_mma<DP, 1>>(dim3((unsigned)p.items), 128, AttendMmaShape<DP, 1>::kBytes, st, p);
}

int launch_prefix_attention(const meteora_heads_t& q, const meteora_heads_t& out, float* lse, const meteora_cache_t& cache,
                            const BatchView& batch, const AttendSizes& z, float scale, void* workspace, cudaStream_t st) {
    AttendPlan plan = plan_attend(z);
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
    p.status = (int32_t*)workspace;
    const size_t rows = plan.slots * z.T * z.q_heads;
    p.part_o = (float*)((uint8_t*)workspace + kHeaderBytes);
    p.part_ml = (float2*)((uint8_t*)p.part_o + align_up(rows * z.head_dim * 4, 256));
    const long long prefix_items = p.tc.ctas > 0 ? 0 : (long long)p.prefix_slots * p.kv_heads * p.t_tiles[0] * p.g_tiles[0];
    const long long own_items = z.table_width > 0 ? (long long)p.own_slots * p.kv_heads * p.t_tiles[1] * p.g_tiles[1] : 0;
    if (prefix_items + own_items >= (1LL << 31)) return METEORA_ERR_UNSUPPORTED_SHAPE;
    int rc = METEORA_OK;
    auto pieces = [&](long long n_prefix, long long n_own, bool wide) -> int {
        if (n_prefix + n_own == 0) return METEORA_OK;
        AttendParams a = p;
        a.prefix_items = (int)n_prefix;
        a.items = (int)(n_prefix + n_own);
        if (plan.mma) return plan.dp == 64 ? launch_mma<64>(wide, a, st) : plan.dp == 128 ? launch_mma<128>(wide, a, st) : launch_mma<256>(wide, a, st);
        if (z.dtype == METEORA_BF16) return launch_dependent<k_attend_simt<__nv_bfloat16>>(dim3((unsigned)a.items), 128, attend_simt_bytes(p.dim), st, a);
        return launch_dependent<k_attend_simt<float>>(dim3((unsigned)a.items), 128, attend_simt_bytes(p.dim), st, a);
    };
    if (p.tc.ctas > 0 && (rc = launch_prefix_tc(p, st)) != METEORA_OK) return rc;
    if (plan.wide[0] == plan.wide[1]) {
        rc = pieces(prefix_items, own_items, plan.wide[0]);
    } else {
        rc = pieces(prefix_items, 0, plan.wide[0]);
        if (rc == METEORA_OK) rc = pieces(0, own_items, plan.wide[1]);
    }
    if (rc != METEORA_OK) return rc;
    const long long join = ((long long)z.T * z.q_heads + 3) / 4;
    if (z.dtype == METEORA_BF16) return launch_dependent<k_attend_join<__nv_bfloat16>>(dim3((unsigned)join), 128, 0, st, p);
    return launch_dependent<k_attend_join<float>>(dim3((unsigned)join), 128, 0, st, p);
}

}  // namespace meteora
