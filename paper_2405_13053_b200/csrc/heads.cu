// Rotary positions, norms of query and key heads, and the append to a paged cache: one pass over rows of heads.
//
// A row is one head of one token.  A group of lanes holds it in registers as items of two vectors (heads.cuh): the two
// entries of a pair are in one thread, the norm's sum is a few shuffles.  A CTA takes a few tokens: their places and the cos
// and sin of their pairs are worked out once, by all its threads, and read from shared memory by all their heads
// (sincospif for every row would take as long as the row's bytes); then its groups, each with one token whose
// angles it keeps in registers, walk their rows, kAhead of them under way through shared memory (16 KB per CTA, 64 KB per SM;
// through registers, half as many, 20.5 us for 4096 tokens of 32 + 8 heads of 128), the first asked for before the angles.  Few
// tokens: one per CTA, its rows dealt over several CTAs.
// Every entry is read once and written once: 84 MB there, 15.5 us = 5.4 TB/s for the rotation.  With the norm instructions bound
// it (361 for a warp's four rows, 0.66 issued per scheduler and cycle): 19.9 us; gains and places kept in registers from row to
// row save a fifth of them and cost the fourth CTA of an SM or spills, 22 to 32 us.
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

constexpr int kMaxTokens = 4;      // of a CTA
constexpr int kAhead = 2;          // rows of a group under way

struct HeadPassParams {
    HeadSeg seg[3];
    int rows, rows_per_cta, tokens, groups, groups_per_token, lanes, lane_shift, items;
    int T, dim, p64, batched, inverse;
    const void* positions;
    float eps, inv_dim;
    BatchView batch;
    meteora_rotary_t rot;    // dim 0: no rotation
};

// The i-th of what stands `stride` apart.  Strides of kernels with vectors are below 2^31 (vector_rows), which makes a place one
// instruction: with products of 64 bits the norm's pass over 4096 tokens took 20.9 us instead of 19.9, its gradient 32.5
// instead of 30.5.
template <int VE> __device__ __forceinline__ int64_t away(int i, int64_t stride) { return VE == 1 ? i * stride : (int64_t)i * (int)stride; }

template <typename E, int VE, int NI, bool kNorm>
__global__ void __launch_bounds__(kHeadThreads, NI > 1 ? 2 : 4) k_head_pass(const __grid_constant__ HeadPassParams p) {
    typedef HeadVec<E, VE> V;
    extern __shared__ __align__(16) uint8_t s_rows[];           // [kAhead][2 NI][threads] vectors
    __shared__ __align__(16) float s_cs[kMaxTokens][2 * kMaxPairs];
    __shared__ int s_page[kMaxTokens], s_in_page[kMaxTokens];
    __shared__ long long s_pos[kMaxTokens];
    const int tid = threadIdx.x, lane = tid & (p.lanes - 1), group = tid >> p.lane_shift;
    const int t0 = blockIdx.x * p.tokens, nt = min(p.tokens, p.T - t0);
    const int row_lo = blockIdx.y * p.rows_per_cta, rows = min(p.rows, row_lo + p.rows_per_cta) - row_lo;    // of each token
    const HeadItems it(p.dim, p.rot.dim, p.rot.layout == METEORA_ROTARY_HALF, VE);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    int oa[NI], ob[NI];                         // where this thread's items start; no second vector: ob >= dim
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int i = lane + n * p.lanes;
        oa[n] = i < p.items ? it.a(i, VE) : p.dim;
        ob[n] = i < p.items ? it.b(i, VE) : p.dim;
    }
    typedef typename V::Raw Raw;
    typedef typename V::P P;
    const auto place = [&](int slot, int v) { return reinterpret_cast<Raw*>(s_rows) + (slot * 2 * NI + v) * blockDim.x + tid; };
    const auto seg_of = [&](int r, int& h) {
        h = row_lo + r;
        if (h < p.seg[0].heads) return 0;
        h -= p.seg[0].heads;
        if (h < p.seg[1].heads) return 1;
        h -= p.seg[1].heads;
        return 2;
    };
    // a group's rows: every stride-th of token tt of the CTA's; `far` runs kAhead of them ahead
    const int stride = p.groups_per_token, tt = group / stride;
    const bool mine = tt < nt && group < p.groups;               // (not: a token past the end, lanes that fill the last warp)
    int rr = group - tt * stride, far = mine ? rr : rows, asked = 0;
    const auto ask = [&]() {
        if (far < rows) {
            int h;
            const HeadSeg& g = p.seg[seg_of(far, h)];
            const E* src = (const E*)g.in + away<VE>(t0 + tt, g.in_t) + away<VE>(h, g.in_h);
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                if (oa[n] < p.dim) row_copy(place(asked % kAhead, 2 * n), src + oa[n]);
                if (ob[n] < p.dim) row_copy(place(asked % kAhead, 2 * n + 1), src + ob[n]);
            }
            far += stride;
        }
        ++asked;
        row_commit();
    };
#pragma unroll
    for (int q = 0; q < kAhead; ++q) ask();

    if (p.batched) {
        for (int k = tid >> 5; k < nt; k += blockDim.x >> 5) {
            const int t = t0 + k, seq = sequence_of(p.batch, t, tid & 31);
            if ((tid & 31) == 0) {
                const int held = seq >= 0 ? __ldg(p.batch.lengths + seq) : -1;
                long long i = -1, page = -1;
                if (held >= 0) {
                    i = (long long)held + (p.batch.cu ? t - max(0, __ldg(p.batch.cu + seq)) : 0);     // (as in attention)
                    const long long slot = i / p.batch.page;
                    if (slot < p.batch.width) page = __ldg(p.batch.table + (size_t)seq * p.batch.width + slot);
                    if (page >= p.batch.n_pages || page < 0) page = -1;
                }
                s_pos[k] = p.batch.prefix + i;
                s_page[k] = held >= 0 ? (int)page : -2;
                s_in_page[k] = held >= 0 ? (int)(i % p.batch.page) : 0;
            }
        }
        __syncthreads();
    }
    const int pairs = p.rot.dim / 2;
    if (pairs > 0) {
        for (int i = tid, k = 0; i < nt * pairs; i += blockDim.x) {
            k = i / pairs;
            const long long pos = p.batched ? s_pos[k]
                                  : p.p64   ? __ldg((const long long*)p.positions + t0 + k)
                                            : (long long)__ldg((const int32_t*)p.positions + t0 + k);
            const int q = i - k * pairs;
            store_angle<VE>(s_cs[k], it, q, rotary_pair(p.rot.turns[q], pos, p.inverse != 0, p.rot.scale));
        }
        __syncthreads();
    }
    ItemAngles<VE> angles[NI];
#pragma unroll
    for (int n = 0; n < NI; ++n)
        if (mine && lane + n * p.lanes < it.nr) angles[n].load(s_cs[tt], it, lane + n * p.lanes);
    const int page = p.batched && mine ? s_page[tt] : 0;             // -2: no sequence, -1: no page
    // (whole warps stay in the loop: the norm's shuffles need every lane)
    int used = 0;
    for (int done = 0; done < rows; done += stride, rr += stride, ++used) {
        row_wait<kAhead - 1>();
        const bool live = mine && rr < rows;
        int h = 0;
        const HeadSeg& g = p.seg[live ? seg_of(rr, h) : 0];
        Raw a[NI], b[NI];
        P xa[NI][V::N], xb[NI][V::N];
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            a[n] = live && oa[n] < p.dim ? *place(used % kAhead, 2 * n) : V::zero();
            b[n] = live && ob[n] < p.dim ? *place(used % kAhead, 2 * n + 1) : V::zero();
            V::unpack(a[n], xa[n]);
            V::unpack(b[n], xb[n]);
        }
        ask();
        if (kNorm) {
            P sum2;
            splat(sum2, 0.f);
#pragma unroll
            for (int n = 0; n < NI; ++n)
#pragma unroll
                for (int j = 0; j < V::N; ++j) sum2 = fma_p(xa[n][j], xa[n][j], fma_p(xb[n][j], xb[n][j], sum2));
            const float sum = lanes_sum(total(sum2), p.lanes);
            if (g.gain) {
                P rs;
                splat(rs, rsqrtf(fmaf(sum, p.inv_dim, p.eps)));
#pragma unroll
                for (int n = 0; n < NI; ++n) {
                    P ga[V::N], gb[V::N];
                    V::unpack(oa[n] < p.dim ? V::load((const E*)g.gain + oa[n]) : V::zero(), ga);
                    V::unpack(ob[n] < p.dim ? V::load((const E*)g.gain + ob[n]) : V::zero(), gb);
#pragma unroll
                    for (int j = 0; j < V::N; ++j) xa[n][j] = mul_p(mul_p(xa[n][j], rs), ga[j]), xb[n][j] = mul_p(mul_p(xb[n][j], rs), gb[j]);
                }
            }
        }
        if (live && page > -2 && (page >= 0 || !g.paged)) {
            E* const dst = g.paged ? (E*)g.out + (((int64_t)page * g.heads + h) * p.batch.page + s_in_page[tt]) * p.dim
                                   : (E*)g.out + away<VE>(t0 + tt, g.out_t) + away<VE>(h, g.out_h);
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                if (oa[n] >= p.dim) continue;
                const int i = lane + n * p.lanes;
                const bool turn = g.turn && i < it.nr;
                if (turn) angles[n].turn(xa[n], xb[n], it.half);
                const bool same = !turn && !(kNorm && g.gain);           // bit for bit
                V::store(dst + oa[n], same ? a[n] : V::pack(xa[n]));
                if (ob[n] < p.dim) V::store(dst + ob[n], same ? b[n] : V::pack(xb[n]));
            }
        }
    }
}

// Gradients of the norm with the rotation.  A CTA takes an even share of the tokens, kGradTokens at a time (their angles by all
// its threads at once); its first warps take the query heads, the others the key heads, as many as their heads ask for.
// A group keeps its rows' sum of dn * n in registers: one row of partial sums per CTA and tensor goes to the workspace,
// and k_gain_sums adds those up in their order.  With u = dn * x and c = r^3 mean(gain * u):
//     dgain += r u,   dx = (gain r) dn - c x.
// x and dy are read once, dx written once: 126 MB for 4096 tokens of 32 + 8 heads of 128, 30.5 us = 4.1 TB/s.  Bound by
// instructions (481 for a warp's four rows) that 15 warps of an SM, at 128 registers a thread, issue at 0.55 per scheduler and
// cycle.  Slower: rows of one token after the other in a group, its angles in registers, 35.5 us.
constexpr int kGradTokens = 16;

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
    int q_warps, lanes, lane_shift, items;
    int T, dim, p64;
    const void* positions;
    float eps, inv_dim;
    float* part;             // [2][CTAs][dim]
    meteora_rotary_t rot;
};

template <typename E, int VE, int NI>
__global__ void __launch_bounds__(kHeadThreads, 2) k_head_grad(const __grid_constant__ HeadGradParams p) {
    typedef HeadVec<E, VE> V;
    typedef typename V::Raw Raw;
    typedef typename V::P P;
    constexpr int kWarps = kHeadThreads / 32;
    __shared__ __align__(16) float s_cs[kGradTokens][2 * kMaxPairs];
    __shared__ float s_sum[kWarps][METEORA_MAX_HEAD_DIM];
    extern __shared__ __align__(16) uint8_t s_rows[];           // [kAhead][4 NI][threads] vectors
    const int tid = threadIdx.x, lane = tid & (p.lanes - 1), warp = tid >> 5;
    const bool is_k = warp >= p.q_warps;
    const HeadGradSeg& g = p.seg[is_k ? 1 : 0];
    const int group = (tid - (is_k ? p.q_warps * 32 : 0)) >> p.lane_shift;
    const int groups = (is_k ? kWarps - p.q_warps : p.q_warps) * (32 >> p.lane_shift);
    const int t_lo = (int)((long long)p.T * blockIdx.x / gridDim.x), t_hi = (int)((long long)p.T * (blockIdx.x + 1) / gridDim.x);
    const HeadItems it(p.dim, p.rot.dim, p.rot.layout == METEORA_ROTARY_HALF, VE);
    const int pairs = p.rot.dim / 2, heads = g.heads;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int oa[NI], ob[NI];
    Raw gain_a[NI], gain_b[NI];
    P da[NI][V::N], db[NI][V::N];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int i = lane + n * p.lanes;
        oa[n] = i < p.items ? it.a(i, VE) : p.dim;
        ob[n] = i < p.items ? it.b(i, VE) : p.dim;
        gain_a[n] = heads > 0 && oa[n] < p.dim ? V::load((const E*)g.gain + oa[n]) : V::zero();
        gain_b[n] = heads > 0 && ob[n] < p.dim ? V::load((const E*)g.gain + ob[n]) : V::zero();
#pragma unroll
        for (int j = 0; j < V::N; ++j) splat(da[n][j], 0.f), splat(db[n][j], 0.f);
    }
    const auto step = [&](int& t, int& h) {
        h += groups;
        while (h >= heads) h -= heads, ++t;
    };
    const auto place = [&](int slot, int v) { return reinterpret_cast<Raw*>(s_rows) + (slot * 4 * NI + v) * kHeadThreads + tid; };
    // a group's rows: token t, head h; `far` runs kAhead rows ahead
    int next_t = heads > 0 ? t_lo : t_hi, next_h = group, asked = 0, used = 0;
    while (heads > 0 && next_h >= heads) next_h -= heads, ++next_t;
    int far_t = next_t, far_h = next_h;
    const auto ask = [&]() {
        if (far_t < t_hi) {
            const E* x = (const E*)g.x + away<VE>(far_t, g.x_t) + away<VE>(far_h, g.x_h);
            const E* dy = (const E*)g.dy + away<VE>(far_t, g.dy_t) + away<VE>(far_h, g.dy_h);
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                if (oa[n] < p.dim) {
                    row_copy(place(asked % kAhead, 4 * n), x + oa[n]);
                    row_copy(place(asked % kAhead, 4 * n + 1), dy + oa[n]);
                }
                if (ob[n] < p.dim) {
                    row_copy(place(asked % kAhead, 4 * n + 2), x + ob[n]);
                    row_copy(place(asked % kAhead, 4 * n + 3), dy + ob[n]);
                }
            }
            step(far_t, far_h);
        }
        ++asked;
        row_commit();
    };
#pragma unroll
    for (int q = 0; q < kAhead; ++q) ask();
    for (int t0 = t_lo; t0 < t_hi; t0 += kGradTokens) {
        const int nt = min(kGradTokens, t_hi - t0);
        if (pairs > 0) {
            __syncthreads();
            for (int i = tid; i < nt * pairs; i += kHeadThreads) {
                const int k = i / pairs, q = i - k * pairs;
                const long long pos = p.p64 ? __ldg((const long long*)p.positions + t0 + k)
                                            : (long long)__ldg((const int32_t*)p.positions + t0 + k);
                store_angle<VE>(s_cs[k], it, q, rotary_pair(p.rot.turns[q], pos, true, p.rot.scale));
            }
            __syncthreads();
        }
        // (whole warps stay in the loop: the sums' shuffles need every lane)
        while (__any_sync(0xFFFFFFFFu, next_t < t0 + nt)) {
            const bool live = next_t < t0 + nt;
            const int t = next_t, h = next_h;
            P xa[NI][V::N], xb[NI][V::N], ya[NI][V::N], yb[NI][V::N], sq2, dot2;
            splat(sq2, 0.f);
            splat(dot2, 0.f);
            row_wait<kAhead - 1>();
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int i = lane + n * p.lanes;
                const bool in = live && oa[n] < p.dim, in_b = live && ob[n] < p.dim;
                V::unpack(in ? *place(used % kAhead, 4 * n) : V::zero(), xa[n]);
                V::unpack(in ? *place(used % kAhead, 4 * n + 1) : V::zero(), ya[n]);
                V::unpack(in_b ? *place(used % kAhead, 4 * n + 2) : V::zero(), xb[n]);
                V::unpack(in_b ? *place(used % kAhead, 4 * n + 3) : V::zero(), yb[n]);
                if (i < it.nr && live) {
                    ItemAngles<VE> angles;
                    angles.load(s_cs[t - t0], it, i);
                    angles.turn(ya[n], yb[n], it.half);
                }
                P ga[V::N], gb[V::N];
                V::unpack(gain_a[n], ga);
                V::unpack(gain_b[n], gb);
#pragma unroll
                for (int j = 0; j < V::N; ++j) {
                    sq2 = fma_p(xa[n][j], xa[n][j], fma_p(xb[n][j], xb[n][j], sq2));
                    dot2 = fma_p(ga[j], mul_p(ya[n][j], xa[n][j]), fma_p(gb[j], mul_p(yb[n][j], xb[n][j]), dot2));
                }
            }
            if (live) {
                step(next_t, next_h);
                ++used;
                ask();
            }
            const float sq = lanes_sum(total(sq2), p.lanes), dot = lanes_sum(total(dot2), p.lanes);
            if (!live) continue;
            const float r = rsqrtf(fmaf(sq, p.inv_dim, p.eps));
            P rs, c;
            splat(rs, r);
            splat(c, -(r * (r * (r * (dot * p.inv_dim)))));           // (r^3 alone leaves fp32 where heads are small or large)
            E* dx = (E*)g.dx + away<VE>(t, g.dx_t) + away<VE>(h, g.dx_h);
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                P ga[V::N], gb[V::N];
                V::unpack(gain_a[n], ga);
                V::unpack(gain_b[n], gb);
#pragma unroll
                for (int j = 0; j < V::N; ++j) {
                    da[n][j] = fma_p(rs, mul_p(ya[n][j], xa[n][j]), da[n][j]);
                    db[n][j] = fma_p(rs, mul_p(yb[n][j], xb[n][j]), db[n][j]);
                    xa[n][j] = fma_p(mul_p(ga[j], rs), ya[n][j], mul_p(c, xa[n][j]));
                    xb[n][j] = fma_p(mul_p(gb[j], rs), yb[n][j], mul_p(c, xb[n][j]));
                }
                if (oa[n] < p.dim) V::store(dx + oa[n], V::pack(xa[n]));
                if (ob[n] < p.dim) V::store(dx + ob[n], V::pack(xb[n]));
            }
        }
    }
    // the groups' sums: inside a warp by shuffles, then warp by warp in order
    float fa[NI][VE], fb[NI][VE];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        memcpy(fa[n], da[n], sizeof(fa[n]));
        memcpy(fb[n], db[n], sizeof(fb[n]));
#pragma unroll
        for (int j = 0; j < VE; ++j)
            for (int o = p.lanes; o < 32; o <<= 1) {
                fa[n][j] += __shfl_xor_sync(0xFFFFFFFFu, fa[n][j], o);
                fb[n][j] += __shfl_xor_sync(0xFFFFFFFFu, fb[n][j], o);
            }
        if ((tid & 31) < p.lanes) {
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                if (oa[n] < p.dim) s_sum[warp][oa[n] + j] = fa[n][j];
                if (ob[n] < p.dim) s_sum[warp][ob[n] + j] = fb[n][j];
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < 2 * p.dim; i += kHeadThreads) {
        const int which = i >= p.dim, d = i - which * p.dim, w0 = which ? p.q_warps : 0, w1 = which ? kWarps : p.q_warps;
        float v = 0.f;
        for (int w = w0; w < w1; ++w) v += s_sum[w][d];
        p.part[((size_t)which * gridDim.x + blockIdx.x) * p.dim + d] = v;
    }
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

// Whether a tensor's rows can be read as vectors of `bytes`, with strides of 31 bits.
static bool vector_rows(const void* p, int64_t st, int64_t sh, int es, int bytes) {
    return std::max(st, sh) < (1LL << 31) && (uintptr_t)p % bytes == 0 && st * es % bytes == 0 && sh * es % bytes == 0;
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

template <typename E, bool kNorm>
static int launch_pass(int ve, dim3 grid, int threads, const HeadPassParams& p, cudaStream_t st) {
    const size_t smem = (size_t)kAhead * 2 * (ve == 1 ? 4 : 1) * threads * ve * sizeof(E);
    if (ve == 16 / (int)sizeof(E)) return launch_dependent<k_head_pass<E, 16 / (int)sizeof(E), 1, kNorm>>(grid, threads, smem, st, p);
    if constexpr (sizeof(E) == 2)
        if (ve == 4) return launch_dependent<k_head_pass<E, 4, 1, kNorm>>(grid, threads, smem, st, p);
    return launch_dependent<k_head_pass<E, 1, 4, kNorm>>(grid, threads, smem, st, p);
}

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
    p.inv_dim = 1.f / (float)args.head_dim;
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
    while ((1 << p.lane_shift) < p.lanes) ++p.lane_shift;
    // Up to four tokens per CTA; few tokens: the rows of each dealt over several CTAs.
    constexpr int kWave = 148 * 4;
    p.tokens = std::min(4, (args.T + kWave - 1) / kWave);
    int rounds = (p.rows * p.lanes + kHeadThreads - 1) / kHeadThreads, split = 1;
    while (split < rounds && (long long)args.T * (split + 1) <= kWave) ++split;
    p.rows_per_cta = (p.rows + split - 1) / split;
    split = (p.rows + p.rows_per_cta - 1) / p.rows_per_cta;
    p.groups_per_token = std::min(kHeadThreads / p.lanes / p.tokens, p.rows_per_cta);
    p.groups = p.groups_per_token * p.tokens;
    const int threads = (p.groups * p.lanes + 31) / 32 * 32;
    const dim3 grid((args.T + p.tokens - 1) / p.tokens, split);
    bool norm = false;
    for (int i = 0; i < n_segs; ++i) norm |= segs[i].gain != nullptr;
    if (args.dtype == METEORA_BF16) return norm ? launch_pass<__nv_bfloat16, true>(ve, grid, threads, p, st) : launch_pass<__nv_bfloat16, false>(ve, grid, threads, p, st);
    return norm ? launch_pass<float, true>(ve, grid, threads, p, st) : launch_pass<float, false>(ve, grid, threads, p, st);
}

// CTAs of the gradient kernel: two per SM (by registers), a token each at least.
static int grad_ctas(int T) { return std::max(1, std::min(T, 148 * 2)); }

size_t head_grad_workspace_bytes(int T, int head_dim) { return align_up((size_t)2 * grad_ctas(T) * head_dim * 4, 256); }

int launch_head_grad(const meteora_heads_t* dy, const meteora_heads_t* x, const void* const* gain, const meteora_heads_t* dx,
                     float* dq_gain, float* dk_gain, const HeadPassArgs& args, float* part, cudaStream_t st) {
    HeadGradParams p = {};
    for (int i = 0; i < 2; ++i)
        p.seg[i] = HeadGradSeg{dy[i].data, x[i].data, dx[i].data, gain[i], dy[i].stride_token, dy[i].stride_head, x[i].stride_token,
                               x[i].stride_head, dx[i].stride_token, dx[i].stride_head, x[i].heads};
    const int ctas = grad_ctas(args.T), warps = kHeadThreads / 32, all = x[0].heads + x[1].heads;
    p.q_warps = x[1].heads == 0 ? warps : std::max(1, std::min(warps - 1, (warps * x[0].heads + all / 2) / all));
    p.T = args.T;
    p.dim = args.head_dim;
    p.p64 = args.positions_64;
    p.positions = args.positions;
    p.eps = args.eps;
    p.inv_dim = 1.f / (float)args.head_dim;
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
    while ((1 << p.lane_shift) < p.lanes) ++p.lane_shift;
    const dim3 grid(ctas);
    const size_t smem = (size_t)kAhead * 4 * (ve == 1 ? 4 : 1) * kHeadThreads * ve * es;
    int rc = METEORA_OK;
    if (args.dtype == METEORA_BF16)
        rc = ve == 8   ? launch_dependent<k_head_grad<__nv_bfloat16, 8, 1>>(grid, kHeadThreads, smem, st, p)
             : ve == 4 ? launch_dependent<k_head_grad<__nv_bfloat16, 4, 1>>(grid, kHeadThreads, smem, st, p)
                       : launch_dependent<k_head_grad<__nv_bfloat16, 1, 4>>(grid, kHeadThreads, smem, st, p);
    else
        rc = ve == 4 ? launch_dependent<k_head_grad<float, 4, 1>>(grid, kHeadThreads, smem, st, p)
                     : launch_dependent<k_head_grad<float, 1, 4>>(grid, kHeadThreads, smem, st, p);
    if (rc != METEORA_OK) return rc;
    const dim3 sums((x[1].heads ? 2 : 1) * ((p.dim + 31) / 32));
    return launch_dependent<k_gain_sums>(sums, 1024, 0, st, (const float*)part, ctas, ctas, p.dim, dq_gain, dk_gain);
}

}  // namespace meteora
