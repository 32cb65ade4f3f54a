// Shared by the kernels on query, key and value heads: the rotary table of a token, rows of heads as vectors, and where a
// token of a batch stands in the paged cache.
#pragma once

#include <type_traits>

#include "common.cuh"

namespace meteora {

// (cos, sin) of pair i at a position.  position * turns modulo 2^64 is the angle as a fraction of a turn, exactly; its
// upper half is cut into the nearest quarter and a rest of at most an eighth of a turn, which fp32 holds to 2^-28 turns.
__device__ __forceinline__ float2 rotary_pair(uint64_t turns, long long position, bool inverse, float scale) {
    const int32_t a = (int32_t)(((uint64_t)position * turns) >> 32);
    const int32_t quarter = (int32_t)((uint32_t)a + 0x20000000u) >> 30;                 // -2 .. 1
    const int32_t rest = (int32_t)((uint32_t)a - ((uint32_t)quarter << 30));            // [-2^29, 2^29]
    float s, c;
    sincospif((float)rest * 0x1p-31f, &s, &c);
    if (quarter & 1) {
        const float t = c;
        c = -s;
        s = t;
    }
    if (quarter & 2) {
        c = -c;
        s = -s;
    }
    return make_float2(c * scale, (inverse ? -s : s) * scale);
}

template <int bytes> struct RawVec;
template <> struct RawVec<16> { typedef uint4 type; };
template <> struct RawVec<8> { typedef uint2 type; };
template <> struct RawVec<4> { typedef uint32_t type; };
template <> struct RawVec<2> { typedef uint16_t type; };

// Arithmetic on two fp32 in a register pair (one instruction each on this architecture), or on one.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 make_pair2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split_pair2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 mul_p(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma_p(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float mul_p(float a, float b) { return a * b; }
__device__ __forceinline__ float fma_p(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ void splat(f32x2& r, float v) { r = make_pair2(v, v); }
__device__ __forceinline__ void splat(float& r, float v) { r = v; }
__device__ __forceinline__ float total(f32x2 v) {
    float a, b;
    split_pair2(v, a, b);
    return a + b;
}
__device__ __forceinline__ float total(float v) { return v; }

// A vector of VE entries: as it lies in memory, and as VE / 2 register pairs (one float where it is one entry).
template <typename E, int VE> struct HeadVec {
    typedef typename RawVec<VE * sizeof(E)>::type Raw;
    typedef typename std::conditional<VE == 1, float, f32x2>::type P;
    static constexpr int N = VE == 1 ? 1 : VE / 2;
    static __device__ __forceinline__ Raw load(const E* p) { return *reinterpret_cast<const Raw*>(p); }
    static __device__ __forceinline__ void store(E* p, const Raw& r) { *reinterpret_cast<Raw*>(p) = r; }
    static __device__ __forceinline__ Raw zero() {
        Raw r;
        memset(&r, 0, sizeof(r));
        return r;
    }
    static __device__ __forceinline__ void unpack(const Raw& r, P (&v)[N]) {
        if constexpr (VE == 1) {
            E e;
            memcpy(&e, &r, sizeof(e));
            v[0] = to_f32(e);
        } else if constexpr (sizeof(E) == 2) {
            uint32_t w[N];
            memcpy(w, &r, sizeof(r));
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = bf16x2_to_f32x2(w[i]);
        } else {
            memcpy(v, &r, sizeof(r));
        }
    }
    static __device__ __forceinline__ Raw pack(const P (&v)[N]) {
        Raw r;
        if constexpr (VE == 1) {
            E e;
            if constexpr (sizeof(E) == 2) e = __float2bfloat16_rn(v[0]);
            else e = v[0];
            memcpy(&r, &e, sizeof(e));
        } else if constexpr (sizeof(E) == 2) {
            uint32_t w[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float a, b;
                split_pair2(v[i], a, b);
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(b), "f"(a));
            }
            memcpy(&r, w, sizeof(r));
        } else {
            memcpy(&r, v, sizeof(r));
        }
        return r;
    }
};

// A vector from global memory to a place in shared memory that this thread alone reads, on its way until row_wait (an entry of
// two bytes is too small for that and arrives at once).
template <typename Raw>
__device__ __forceinline__ void row_copy(Raw* dst, const void* src) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    if constexpr (sizeof(Raw) == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
    else if constexpr (sizeof(Raw) >= 4) asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(d), "l"(src), "n"(sizeof(Raw)) : "memory");
    else *dst = *(const Raw*)src;
}
__device__ __forceinline__ void row_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void row_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// A head's entries as items of two vectors, so that a pair is in one thread and neighbouring lanes have neighbouring vectors:
// item i < nr is vector i of either half of the rotated part, later items vectors of either half of the rest.  In the half
// layout a pair is an entry of the first vector and the same one of the second, in the interleaved one two entries of a
// vector (with vectors of one entry: the first and the second, 2 i and 2 i + 1).
struct HeadItems {
    int nr, np, half, rot;
    __device__ __forceinline__ HeadItems(int dim, int rot_dim, bool half_layout, int ve)
        : nr(rot_dim / 2 / ve), np(((dim - rot_dim) / ve + 1) / 2), half(half_layout), rot(rot_dim) {}
    __device__ __forceinline__ int a(int i, int ve) const { return i < nr ? (half || ve > 1 ? i * ve : 2 * i) : rot + (i - nr) * ve; }
    __device__ __forceinline__ int b(int i, int ve) const {                  // at or past the head's end: there is none
        return i < nr ? (half || ve > 1 ? rot / 2 + i * ve : 2 * i + 1) : rot + (np + i - nr) * ve;
    }
    // Where cos of pair q stands in a token's table, its sin `sin_off` further: an item's pairs two and two as (cos, cos, sin,
    // sin), first vector first, 16 nr bytes apart, so that lanes read neighbours (vectors of one entry: as (cos, sin)).
    __device__ __forceinline__ int table(int q, int ve) const {
        if (ve == 1) return 2 * q;
        int i = q / ve, j = q % ve;
        if (!half) {
            const int v = ve / 2, second = q >= rot / 4, r = second ? q - rot / 4 : q;
            i = r / v, j = second * v + r % v;
        }
        return ((j >> 1) * nr + i) * 4 + (j & 1);
    }
    static __device__ __forceinline__ int sin_off(int ve) { return ve == 1 ? 1 : 2; }
};

// The angles of a token as it is needed: table[] as above, by `threads` threads of which this is `tid`.
template <int VE>
__device__ __forceinline__ void store_angle(float* table, const HeadItems& it, int q, float2 cs) {
    float* const at = table + it.table(q, VE);
    at[0] = cs.x;
    at[HeadItems::sin_off(VE)] = cs.y;
}

// Angles of an item, in registers for the rows of a token, and its two vectors turned by them.
template <int VE> struct ItemAngles {
    static constexpr int N = VE == 1 ? 1 : VE / 2;
    typedef typename std::conditional<VE == 1, float2, float4>::type Cell;
    Cell t[N];
    __device__ __forceinline__ void load(const float* table, const HeadItems& it, int i) {
#pragma unroll
        for (int j = 0; j < N; ++j) t[j] = *reinterpret_cast<const Cell*>(table + (j * it.nr + i) * (sizeof(Cell) / 4));
    }
    template <typename P>
    __device__ __forceinline__ void turn(P (&a)[N], P (&b)[N], bool half) const {
        if constexpr (VE == 1) {
            const float2 cs = t[0];
            const float x = a[0], y = b[0];
            a[0] = fmaf(y, -cs.y, __fmul_rn(x, cs.x));             // (rounded as the pairs below are)
            b[0] = fmaf(x, cs.y, __fmul_rn(y, cs.x));
        } else if (half) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const f32x2 c = make_pair2(t[j].x, t[j].y), s = make_pair2(t[j].z, t[j].w), m = make_pair2(-t[j].z, -t[j].w), x = a[j], y = b[j];
                a[j] = fma_p(y, m, mul_p(x, c));
                b[j] = fma_p(x, s, mul_p(y, c));
            }
        } else {
            // an entry pair is (x, y) -> (x c - y s, y c + x s) = (x, y) * (c, c) + (y, x) * (-s, s)
#pragma unroll
            for (int j = 0; j < N; ++j) {                          // t[j]: pairs 2 j and 2 j + 1 of the item
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int e = 2 * j + k;                       // of the first vector's pairs, then the second's
                    P& v = e < N ? a[e < N ? e : 0] : b[e < N ? 0 : e - N];
                    const float c = k ? t[j].y : t[j].x, s = k ? t[j].w : t[j].z;
                    float x, y;
                    split_pair2(v, x, y);
                    v = fma_p(make_pair2(y, x), make_pair2(-s, s), mul_p(v, make_pair2(c, c)));
                }
            }
        }
    }
};

// Sum over the `lanes` (a power of two) neighbouring lanes that share a row.
__device__ __forceinline__ float lanes_sum(float a, int lanes) {
    if (lanes == 8) {              // 64 to 128 entries in vectors of 8: the usual head
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
    } else {
        for (int o = lanes >> 1; o > 0; o >>= 1) a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
    }
    return a;
}

// A batch over a paged cache, as the kernels take it.
struct BatchView {
    const int32_t* cu;          // [B + 1] or nullptr: one token each
    const int32_t* lengths;
    const int32_t* table;
    const int32_t* prefix_pages;
    int B, T, width, page, prefix;
    long long n_pages;
};

// The sequence of token t by a whole warp (all its lanes call with the same t), -1 where it has none.  Each step
// looks at 32 places of cu at once, so that 4096 sequences take three dependent loads.
__device__ __forceinline__ int sequence_of(const BatchView& v, int t, int lane) {
    if (!v.cu) return t < v.B ? t : -1;
    if (t < __ldg(v.cu) || t >= __ldg(v.cu + v.B)) return -1;
    int lo = 0, hi = v.B;                       // cu[lo] <= t < cu[hi]
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const unsigned le = __ballot_sync(0xFFFFFFFFu, at < hi && __ldg(v.cu + at) <= t);
        const int last = 31 - __clz(le | 1u);   // (lane 0 is at lo, which holds; an order that does not ascend still ends)
        lo += last * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

}  // namespace meteora
