// Shared by the kernels on query, key and value heads: the rotary table of a token, rows of heads as vectors, and where a
// token of a batch stands in the paged cache.
#pragma once

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

template <typename E, int VE> struct HeadVec {
    typedef typename RawVec<VE * sizeof(E)>::type Raw;
    static __device__ __forceinline__ Raw load(const E* p) { return *reinterpret_cast<const Raw*>(p); }
    static __device__ __forceinline__ void store(E* p, const Raw& r) { *reinterpret_cast<Raw*>(p) = r; }
    static __device__ __forceinline__ Raw zero() {
        Raw r;
        memset(&r, 0, sizeof(r));
        return r;
    }
    static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[VE]) {
        E e[VE];
        memcpy(e, &r, sizeof(r));
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = to_f32(e[i]);
    }
    static __device__ __forceinline__ Raw pack(const float (&v)[VE]) {
        E e[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            if constexpr (sizeof(E) == 2) e[i] = __float2bfloat16_rn(v[i]);
            else e[i] = v[i];
        }
        Raw r;
        memcpy(&r, e, sizeof(r));
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
    // Where pair q's (cos, sin) stands: those of an item, first vector first, nr apart, so that lanes read neighbours.
    __device__ __forceinline__ int table(int q, int ve) const {
        if (half || ve == 1) return q % ve * nr + q / ve;
        const int v = ve / 2, second = q >= rot / 4, r = second ? q - rot / 4 : q;
        return (second * v + r % v) * nr + r / v;
    }
};

template <int VE>
__device__ __forceinline__ void turn_item(float (&a)[VE], float (&b)[VE], const float2 (&cs)[VE], bool half) {
    if (VE == 1 || half) {
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const float x = a[j], y = b[j];
            a[j] = x * cs[j].x - y * cs[j].y;
            b[j] = y * cs[j].x + x * cs[j].y;
        }
    } else {
#pragma unroll
        for (int j = 0; j + 1 < VE; j += 2) {
            const float2 ca = cs[j / 2], cb = cs[VE / 2 + j / 2];
            const float x = a[j], y = a[j + 1], z = b[j], w = b[j + 1];
            a[j] = x * ca.x - y * ca.y;
            a[j + 1] = y * ca.x + x * ca.y;
            b[j] = z * cb.x - w * cb.y;
            b[j + 1] = w * cb.x + z * cb.y;
        }
    }
}

// Sums over the `lanes` (a power of two) neighbouring lanes that share a row.
__device__ __forceinline__ void lanes_sum(float& a, float& b, int lanes) {
    if (lanes == 8) {              // 64 to 128 entries in vectors of 8: the usual head
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) a += __shfl_xor_sync(0xFFFFFFFFu, a, o), b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
    } else {
        for (int o = lanes >> 1; o > 0; o >>= 1) a += __shfl_xor_sync(0xFFFFFFFFu, a, o), b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
    }
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
