// Rotary positions, norms of query and key heads, and the append to a paged cache: one pass over rows of heads.
//
// A row is one head of one token.  A group of lanes holds it in registers as items of two vectors (heads.cuh): the two
// entries of a pair are in one thread, the norm's sum is a few shuffles.  A CTA takes a token (its rows, or a share
// of them where there are few tokens), so that the cos and sin of the token's pairs are computed once, by rot/2 threads, and
// read from shared memory by all its heads: sincospif for every row would take as long as the row's bytes.
// Bound by HBM: every entry is read once and written once.
#include <algorithm>

#include "heads.cuh"
#include "launch_heads.cuh"

namespace meteora {

constexpr int kHeadThreads = 256;
constexpr int kMaxPairs = METEORA_MAX_HEAD_DIM / 2;

struct HeadSeg {
    const void* in;
    void* out;               // paged: the cache
    int64_t in_t, in_h, out_t, out_h;
    const void* gain;
    int heads, paged, turn;
};

struct HeadPassParams {
    HeadSeg seg[3];
    int rows, rows_per_cta, groups, lanes, items;
    int T, dim, p64, batched, inverse;
    const void* positions;
    float eps;
    BatchView batch;
    meteora_rotary_t rot;    // dim 0: no rotation
};

template <typename E, int VE, int NI>
__global__ void __launch_bounds__(kHeadThreads) k_head_pass(const __grid_constant__ HeadPassParams p) {
    typedef HeadVec<E, VE> V;
    __shared__ float2 s_cs[kMaxPairs];
    __shared__ int s_at[2];
    __shared__ long long s_pos;
    const int tid = threadIdx.x, lane = tid & (p.lanes - 1), group = tid / p.lanes;
    const int t = blockIdx.x;
    const int row_lo = blockIdx.y * p.rows_per_cta, row_hi = min(p.rows, row_lo + p.rows_per_cta);
    const HeadItems it(p.dim, p.rot.dim, p.rot.layout == METEORA_ROTARY_HALF, VE);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    typename V::Raw a[NI], b[NI];
    auto seg_of = [&](int r, int& h) {
        int s = 0;
        h = r;
        if (h >= p.seg[0].heads) h -= p.seg[0].heads, s = 1;
        if (s == 1 && h >= p.seg[1].heads) h -= p.seg[1].heads, s = 2;
        return s;
    };
    auto load_row = [&](int r) {
        if (r >= row_hi) return;
        int h;
        const HeadSeg& g = p.seg[seg_of(r, h)];
        const E* src = (const E*)g.in + t * g.in_t + h * g.in_h;
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            const int i = lane + n * p.lanes;
            a[n] = b[n] = V::zero();
            if (i < p.items) {
                a[n] = V::load(src + it.a(i, VE));
                if (it.b(i, VE) < p.dim) b[n] = V::load(src + it.b(i, VE));
            }
        }
    };
    load_row(row_lo + group);                   // on its way while the token's place and angles are worked out

    if (p.batched) {
        if (tid < 32) {
            const int seq = sequence_of(p.batch, t, tid);
            if (tid == 0) {
                int held = seq >= 0 ? __ldg(p.batch.lengths + seq) : -1;
                long long i = -1, page = -1;
                if (held >= 0) {
                    i = (long long)held + (p.batch.cu ? t - __ldg(p.batch.cu + seq) : 0);
                    const long long slot = i / p.batch.page;
                    if (slot < p.batch.width) page = __ldg(p.batch.table + (size_t)seq * p.batch.width + slot);
                    if (page >= p.batch.n_pages) page = -1;
                }
                s_pos = p.batch.prefix + i;
                s_at[0] = held >= 0 ? (int)page : -2;
                s_at[1] = held >= 0 ? (int)(i % p.batch.page) : 0;
            }
        }
        __syncthreads();
        if (s_at[0] == -2) return;              // no sequence: nothing of this token is written
    }
    if (p.rot.dim > 0) {
        const long long pos = p.batched ? s_pos
                              : p.p64   ? __ldg((const long long*)p.positions + t)
                                        : (long long)__ldg((const int32_t*)p.positions + t);
        for (int i = tid; i < p.rot.dim / 2; i += blockDim.x)
            s_cs[i] = rotary_pair(p.rot.turns[i], pos, p.inverse != 0, p.rot.scale);
        __syncthreads();
    }
    const bool has_place = !p.batched || s_at[0] >= 0;
    // (whole warps stay in the loop: the norm's shuffles need every lane)
    for (int r0 = row_lo; r0 < row_hi; r0 += p.groups) {
        const int r = r0 + group;
        const bool live = r < row_hi && group < p.groups;
        int h = 0;
        const HeadSeg& g = p.seg[live ? seg_of(r, h) : 0];
        typename V::Raw ya[NI], yb[NI];
        float sum = 0.f;
        float xa[NI][VE], xb[NI][VE];
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            ya[n] = a[n];
            yb[n] = b[n];
            V::unpack(a[n], xa[n]);
            V::unpack(b[n], xb[n]);
#pragma unroll
            for (int j = 0; j < VE; ++j) sum = fmaf(xa[n][j], xa[n][j], fmaf(xb[n][j], xb[n][j], sum));
        }
        load_row(r + p.groups);
        const bool norm = live && g.gain != nullptr;
        if (p.seg[0].gain || p.seg[1].gain) sum = lanes_sum(sum, p.lanes);
        const float rs = norm ? 1.f / sqrtf(sum / (float)p.dim + p.eps) : 1.f;
        if (!live || (g.paged && !has_place)) continue;
        E* dst = g.paged ? (E*)g.out + (((int64_t)s_at[0] * g.heads + h) * p.batch.page + s_at[1]) * p.dim
                         : (E*)g.out + t * g.out_t + h * g.out_h;
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            const int i = lane + n * p.lanes;
            if (i >= p.items) continue;
            const int oa = it.a(i, VE), ob = it.b(i, VE);
            if (norm) {
                float ga[VE], gb[VE];
                V::unpack(V::load((const E*)g.gain + oa), ga);
                V::unpack(ob < p.dim ? V::load((const E*)g.gain + ob) : V::zero(), gb);
#pragma unroll
                for (int j = 0; j < VE; ++j) xa[n][j] *= rs * ga[j], xb[n][j] *= rs * gb[j];
            }
            if (g.turn && i < it.nr) {
                float2 cs[VE];
#pragma unroll
                for (int j = 0; j < VE; ++j) cs[j] = s_cs[i * VE + j];
                turn_item<VE>(xa[n], xb[n], cs, it.half);
            }
            if (norm || (g.turn && i < it.nr)) {
                ya[n] = V::pack(xa[n]);
                yb[n] = V::pack(xb[n]);
            }
            V::store(dst + oa, ya[n]);
            if (ob < p.dim) V::store(dst + ob, yb[n]);
        }
    }
}

// Gradients of the norm with the rotation.  CTAs [0, q_ctas) take q, the others k; a CTA walks its share of the tokens,
// kTokTile at a time (their angles by all its threads at once), and keeps its rows' sum of dn * n in registers: one row
// of partial sums per CTA goes to the workspace, and k_gain_sums adds those up in their order.
constexpr int kTokTile = 4;

struct HeadGradSeg {
    const void* dy;
    const void* x;
    void* dx;
    const void* gain;
    int64_t dy_t, dy_h, x_t, x_h, dx_t, dx_h;
    int heads;
};
struct HeadGradParams {
    HeadGradSeg seg[2];
    int q_ctas, groups, lanes, items;
    int T, dim, p64;
    const void* positions;
    float eps;
    float* part;             // [CTAs][dim]
    meteora_rotary_t rot;
};

template <typename E, int VE, int NI>
__global__ void __launch_bounds__(kHeadThreads) k_head_grad(const __grid_constant__ HeadGradParams p) {
    typedef HeadVec<E, VE> V;
    __shared__ float2 s_cs[kTokTile][kMaxPairs];
    __shared__ float s_sum[METEORA_MAX_HEAD_DIM];
    const int tid = threadIdx.x, lane = tid & (p.lanes - 1), group = tid / p.lanes;
    const bool is_k = (int)blockIdx.x >= p.q_ctas;
    const HeadGradSeg& g = p.seg[is_k ? 1 : 0];
    const int ctas = is_k ? gridDim.x - p.q_ctas : p.q_ctas, cta = is_k ? blockIdx.x - p.q_ctas : blockIdx.x;
    const int t_lo = (int)((long long)p.T * cta / ctas), t_hi = (int)((long long)p.T * (cta + 1) / ctas);
    const HeadItems it(p.dim, p.rot.dim, p.rot.layout == METEORA_ROTARY_HALF, VE);
    const int pairs = p.rot.dim / 2;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    float ga[NI][VE], gb[NI][VE], da[NI][VE], db[NI][VE];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int i = lane + n * p.lanes;
        V::unpack(i < p.items ? V::load((const E*)g.gain + it.a(i, VE)) : V::zero(), ga[n]);
        V::unpack(i < p.items && it.b(i, VE) < p.dim ? V::load((const E*)g.gain + it.b(i, VE)) : V::zero(), gb[n]);
#pragma unroll
        for (int j = 0; j < VE; ++j) da[n][j] = db[n][j] = 0.f;
    }
    for (int t0 = t_lo; t0 < t_hi; t0 += kTokTile) {
        const int nt = min(kTokTile, t_hi - t0);
        __syncthreads();
        for (int i = tid; i < nt * pairs; i += blockDim.x) {
            const int tt = i / pairs, q = i - tt * pairs;
            const long long pos = p.p64 ? __ldg((const long long*)p.positions + t0 + tt)
                                        : (long long)__ldg((const int32_t*)p.positions + t0 + tt);
            s_cs[tt][q] = rotary_pair(p.rot.turns[q], pos, true, p.rot.scale);
        }
        __syncthreads();
        const int rows = nt * g.heads;
        for (int r0 = 0; r0 < rows; r0 += p.groups) {
            const int r = r0 + group;
            const bool live = r < rows && group < p.groups;
            const int tt = live ? r / g.heads : 0, h = live ? r - tt * g.heads : 0;
            const int64_t t = t0 + tt;
            const E* x = (const E*)g.x + t * g.x_t + h * g.x_h;
            const E* dy = (const E*)g.dy + t * g.dy_t + h * g.dy_h;
            float xa[NI][VE], xb[NI][VE], ya[NI][VE], yb[NI][VE];
            typename V::Raw ra[NI], rb[NI], sa[NI], sb[NI];
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int i = lane + n * p.lanes;
                const bool in = live && i < p.items, in_b = in && it.b(i, VE) < p.dim;
                ra[n] = in ? V::load(x + it.a(i, VE)) : V::zero();
                sa[n] = in ? V::load(dy + it.a(i, VE)) : V::zero();
                rb[n] = in_b ? V::load(x + it.b(i, VE)) : V::zero();
                sb[n] = in_b ? V::load(dy + it.b(i, VE)) : V::zero();
            }
            float sq = 0.f, dot = 0.f;
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int i = lane + n * p.lanes;
                V::unpack(ra[n], xa[n]);
                V::unpack(rb[n], xb[n]);
                V::unpack(sa[n], ya[n]);
                V::unpack(sb[n], yb[n]);
                if (i < it.nr) {
                    float2 cs[VE];
#pragma unroll
                    for (int j = 0; j < VE; ++j) cs[j] = s_cs[tt][i * VE + j];
                    turn_item<VE>(ya[n], yb[n], cs, it.half);
                }
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    sq = fmaf(xa[n][j], xa[n][j], fmaf(xb[n][j], xb[n][j], sq));
                    dot = fmaf(ga[n][j] * ya[n][j], xa[n][j], fmaf(gb[n][j] * yb[n][j], xb[n][j], dot));
                }
            }
            sq = lanes_sum(sq, p.lanes);
            dot = lanes_sum(dot, p.lanes);
            if (!live) continue;
            const float rs = 1.f / sqrtf(sq / (float)p.dim + p.eps);
            const float mean = dot * rs / (float)p.dim;             // mean of gain * dn * n
            E* dx = (E*)g.dx + t * g.dx_t + h * g.dx_h;
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int i = lane + n * p.lanes;
                if (i >= p.items) continue;
                float oa[VE], ob[VE];
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const float na = xa[n][j] * rs, nb = xb[n][j] * rs;
                    da[n][j] = fmaf(ya[n][j], na, da[n][j]);
                    db[n][j] = fmaf(yb[n][j], nb, db[n][j]);
                    oa[j] = rs * (ga[n][j] * ya[n][j] - na * mean);
                    ob[j] = rs * (gb[n][j] * yb[n][j] - nb * mean);
                }
                V::store(dx + it.a(i, VE), V::pack(oa));
                if (it.b(i, VE) < p.dim) V::store(dx + it.b(i, VE), V::pack(ob));
            }
        }
    }
    // the groups' sums, group by group in order
    for (int s = 0; s < p.groups; ++s) {
        if (group == s) {
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int i = lane + n * p.lanes;
                if (i >= p.items) continue;
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const int oa = it.a(i, VE) + j, ob = it.b(i, VE) + j;
                    s_sum[oa] = s ? s_sum[oa] + da[n][j] : da[n][j];
                    if (ob < p.dim) s_sum[ob] = s ? s_sum[ob] + db[n][j] : db[n][j];
                }
            }
        }
        __syncthreads();
    }
    for (int d = tid; d < p.dim; d += blockDim.x) p.part[(size_t)blockIdx.x * p.dim + d] = s_sum[d];
}

// Column sums of the partial rows: 32 columns per CTA, 32 threads per column, then a tree.  CTAs [0, col_ctas) for q.
__global__ void __launch_bounds__(1024) k_gain_sums(const float* part, int q_ctas, int k_ctas, int dim, float* dq_gain, float* dk_gain) {
    __shared__ float s[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int col_ctas = (dim + 31) / 32;
    const bool is_k = (int)blockIdx.x >= col_ctas;
    const int d = (blockIdx.x - (is_k ? col_ctas : 0)) * 32 + x;
    const int lo = is_k ? q_ctas : 0, n = is_k ? k_ctas : q_ctas;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    float v = 0.f;
    if (d < dim)
        for (int r = y; r < n; r += 32) v += part[(size_t)(lo + r) * dim + d];
    s[y][x] = v;
    __syncthreads();
    for (int o = 16; o > 0; o >>= 1) {
        if (y < o) s[y][x] += s[y + o][x];
        __syncthreads();
    }
    if (y == 0 && d < dim) (is_k ? dk_gain : dq_gain)[d] = s[0][x];
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
static int pow2_at_least(int v) {
    int l = 1;
    while (l < v) l *= 2;
    return l;
}

// Whether a tensor's rows can be read as vectors of `bytes`.
static bool vector_rows(const void* p, int64_t st, int64_t sh, int es, int bytes) {
    return (uintptr_t)p % bytes == 0 && st * es % bytes == 0 && sh * es % bytes == 0;
}

// Entries per vector: 16 bytes where both halves of an item start on a multiple of it in every tensor, then 8 (bf16 only:
// 40 rotated entries of 80, say), else one entry at a time.
template <typename F>
static int vector_entries(meteora_dtype_t dtype, int dim, int rot, F all_aligned) {
    const int es = (int)elem_size(dtype);
    for (int ve = 16 / es; ve >= 4; ve /= 2)
        if (dim % ve == 0 && rot % (2 * ve) == 0 && all_aligned(ve * es)) return ve;
    return 1;
}

static int items_of(int dim, int rot, int ve) { return rot / 2 / ve + ((dim - rot) / ve + 1) / 2; }

int launch_head_pass(const HeadRows* segs, int n_segs, const HeadPassArgs& args, cudaStream_t st) {
    if (args.T == 0) return METEORA_OK;
    HeadPassParams p = {};
    for (int i = 0; i < n_segs; ++i) {
        const HeadRows& r = segs[i];
        p.seg[i] = HeadSeg{r.in.data, r.out, r.in.stride_token, r.in.stride_head, r.out_t, r.out_h, r.gain, r.in.heads, r.paged, r.turn && args.rot};
        p.rows += r.in.heads;
    }
    if (p.rows == 0) return METEORA_OK;
    p.T = args.T;
    p.dim = args.head_dim;
    p.p64 = args.positions_64;
    p.positions = args.positions;
    p.inverse = args.inverse;
    p.eps = args.eps;
    if (args.batch) {
        p.batched = 1;
        p.batch = *args.batch;
    }
    if (args.rot) p.rot = *args.rot;
    const int es = (int)elem_size(args.dtype);
    const int ve = vector_entries(args.dtype, p.dim, p.rot.dim, [&](int bytes) {
        for (int i = 0; i < n_segs; ++i) {
            const HeadSeg& s = p.seg[i];
            if (!vector_rows(s.in, s.in_t, s.in_h, es, bytes)) return false;
            if (!(s.paged ? (uintptr_t)s.out % bytes == 0 : vector_rows(s.out, s.out_t, s.out_h, es, bytes))) return false;
            if ((uintptr_t)s.gain % bytes != 0) return false;
        }
        return true;
    });
    p.items = items_of(p.dim, p.rot.dim, ve);
    p.lanes = std::min(32, pow2_at_least(p.items));
    // A token's rows in as few rounds of 256 threads as they take, evenly; where there are fewer tokens than the device
    // holds CTAs the rows are dealt over several CTAs.
    int rounds = (p.rows * p.lanes + kHeadThreads - 1) / kHeadThreads;
    int split = 1;
    while (split < rounds && (long long)args.T * (split + 1) <= 592) ++split;
    p.rows_per_cta = (p.rows + split - 1) / split;
    split = (p.rows + p.rows_per_cta - 1) / p.rows_per_cta;
    rounds = (p.rows_per_cta * p.lanes + kHeadThreads - 1) / kHeadThreads;
    p.groups = (p.rows_per_cta + rounds - 1) / rounds;
    const int threads = (p.groups * p.lanes + 31) / 32 * 32;
    const dim3 grid(args.T, split);
    if (args.dtype == METEORA_BF16) {
        if (ve == 8) return launch_dependent<k_head_pass<__nv_bfloat16, 8, 1>>(grid, threads, 0, st, p);
        if (ve == 4) return launch_dependent<k_head_pass<__nv_bfloat16, 4, 1>>(grid, threads, 0, st, p);
        return launch_dependent<k_head_pass<__nv_bfloat16, 1, 4>>(grid, threads, 0, st, p);
    }
    if (ve == 4) return launch_dependent<k_head_pass<float, 4, 1>>(grid, threads, 0, st, p);
    return launch_dependent<k_head_pass<float, 1, 4>>(grid, threads, 0, st, p);
}

// CTAs of the gradient kernel: a few per SM, each with at least a tile of tokens; q and k get shares as their heads are.
static void grad_ctas(int T, int q_heads, int k_heads, int* q_ctas, int* k_ctas) {
    const int tiles = (T + kTokTile - 1) / kTokTile, budget = 148 * 4;
    const int rows = std::max(1, q_heads + k_heads);
    *q_ctas = q_heads ? std::max(1, std::min(tiles, (int)((long long)budget * q_heads / rows))) : 0;
    *k_ctas = k_heads ? std::max(1, std::min(tiles, (int)((long long)budget * k_heads / rows))) : 0;
}

size_t head_grad_workspace_bytes(int T, int q_heads, int k_heads, int head_dim) {
    int q = 0, k = 0;
    grad_ctas(T, q_heads, k_heads, &q, &k);
    return align_up((size_t)(q + k) * head_dim * 4, 256);
}

int launch_head_grad(const meteora_heads_t* dy, const meteora_heads_t* x, const void* const* gain, const meteora_heads_t* dx,
                     float* dq_gain, float* dk_gain, const HeadPassArgs& args, float* part, cudaStream_t st) {
    HeadGradParams p = {};
    for (int i = 0; i < 2; ++i)
        p.seg[i] = HeadGradSeg{dy[i].data, x[i].data, dx[i].data, gain[i], dy[i].stride_token, dy[i].stride_head, x[i].stride_token,
                               x[i].stride_head, dx[i].stride_token, dx[i].stride_head, x[i].heads};
    int k_ctas = 0;
    grad_ctas(args.T, x[0].heads, x[1].heads, &p.q_ctas, &k_ctas);
    p.T = args.T;
    p.dim = args.head_dim;
    p.p64 = args.positions_64;
    p.positions = args.positions;
    p.eps = args.eps;
    p.part = part;
    if (args.rot) p.rot = *args.rot;
    const int es = (int)elem_size(args.dtype);
    const int ve = vector_entries(args.dtype, p.dim, p.rot.dim, [&](int bytes) {
        for (int i = 0; i < 2; ++i) {
            const HeadGradSeg& s = p.seg[i];
            if (s.heads == 0) continue;
            if (!vector_rows(s.dy, s.dy_t, s.dy_h, es, bytes) || !vector_rows(s.x, s.x_t, s.x_h, es, bytes) ||
                !vector_rows(s.dx, s.dx_t, s.dx_h, es, bytes) || (uintptr_t)s.gain % bytes != 0)
                return false;
        }
        return true;
    });
    p.items = items_of(p.dim, p.rot.dim, ve);
    p.lanes = std::min(32, pow2_at_least(p.items));
    p.groups = kHeadThreads / p.lanes;
    const dim3 grid(p.q_ctas + k_ctas);
    int rc = METEORA_OK;
    if (args.dtype == METEORA_BF16)
        rc = ve == 8   ? launch_dependent<k_head_grad<__nv_bfloat16, 8, 1>>(grid, kHeadThreads, 0, st, p)
             : ve == 4 ? launch_dependent<k_head_grad<__nv_bfloat16, 4, 1>>(grid, kHeadThreads, 0, st, p)
                       : launch_dependent<k_head_grad<__nv_bfloat16, 1, 4>>(grid, kHeadThreads, 0, st, p);
    else
        rc = ve == 4 ? launch_dependent<k_head_grad<float, 4, 1>>(grid, kHeadThreads, 0, st, p)
                     : launch_dependent<k_head_grad<float, 1, 4>>(grid, kHeadThreads, 0, st, p);
    if (rc != METEORA_OK) return rc;
    const dim3 sums((x[1].heads ? 2 : 1) * ((p.dim + 31) / 32));
    return launch_dependent<k_gain_sums>(sums, 1024, 0, st, (const float*)part, p.q_ctas, k_ctas, p.dim, dq_gain, dk_gain);
}

}  // namespace meteora
