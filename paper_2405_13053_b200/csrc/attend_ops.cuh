// Copies and warp-level products of the attention kernels.
#pragma once

#include "attend.cuh"

namespace meteora {

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two weights rounded to bf16 (a in the lower half); they come back as the values they were rounded to.
__device__ __forceinline__ uint32_t round_pair(float& a, float& b) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    a = __uint_as_float(r << 16);
    b = __uint_as_float(r & 0xFFFF0000u);
    return r;
}

// What the 64-row kernel and the warp kernel need to be planned: their shared memory.
struct TileInfo {
    int4 x, y, z;                  // sequence, tile of rows, kv head, unit; first token, tokens, held, keys the unit sees; first key, first and last of its unit
    unsigned there[2];             // keys that there are
    unsigned none[2];
};
template <int DP> struct AttendMmaShape {
    static constexpr int kChunks = DP / 8;                         // 16-byte chunks of a row
    static constexpr int kRows = 64;
    static constexpr int kTileBytes = kAttendTile * DP * 2;        // keys or values of a tile
    static constexpr int kStages = DP == 64 ? 4 : DP == 128 ? 3 : 2;
    static constexpr int kInfos = kStages + 1;
    static constexpr int kWarpBytes = (DP == 256 ? 16 * DP * 2 : 0) + 16 * kAttendTile * 2;     // queries that registers do not hold; weights
    static constexpr int kBarOff = 2 * kStages * kTileBytes + 4 * kWarpBytes + kInfos * (kAttendTile * 8 + (int)sizeof(TileInfo));
    static constexpr int kBytes = 1024 + kBarOff + kStages * 8;
};

template <int DP> struct AttendWarpShape {
    static constexpr int kChunks = DP / 8;                         // 16-byte chunks of a row
    static constexpr int kTileBytes = kWarpTile * DP * 2;          // keys or values of a tile
    static constexpr int kStages = DP == 128 ? 2 : 3;
    static constexpr int kInfos = 4;                               // tiles described: one more than kStages
    static constexpr int kWarpBytes = 2 * kStages * kTileBytes;
    static constexpr int kBytes = 1024 + 4 * (kWarpBytes + kInfos * 40 + kStages * 8);
};

}  // namespace meteora
