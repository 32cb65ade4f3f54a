// Attention over a paged cache with a shared prefix: what its kernels have in common.
//
// softmax over the keys a query sees is joined from pieces: for a set K of keys and a row of scores s (in units of log2),
//     m = max_K s,  l = sum_K 2^(s - m),  o = sum_K 2^(s - m) v,
// and the pieces of disjoint sets join by the common maximum: o = sum_i 2^(m_i - M) o_i, l likewise, result o / l.  So the
// prefix is computed once for the rows of all sequences together (its keys are read once per tile of rows, not once per
// sequence) and every sequence's own pages for its own rows.
//
// A unit of work is a tile of rows of one kv head against its keys, in tiles of keys.  The tiles of all units stand in one
// row and are dealt to the workers (CTAs or warps) in even shares, whatever the sequences' lengths: no worker waits behind a
// long sequence, and it goes from unit to unit with its copies ahead.  Where a share starts or ends inside a unit, the unit comes in
// pieces: share c's part of unit u is piece u + c (going along the row, either grows by one at a time), a tile of (o, m, l)
// in fp32 in the workspace, and k_attend_join adds a row's pieces in their order.  Everything follows from lengths that are on
// the device, so a captured call goes on as they grow.
#pragma once

#include "heads.cuh"

namespace meteora {

constexpr int kAttendTile = 64;    // keys per tile of the kernels whose CTA is one worker
constexpr int kWarpTile = 16;      // of the one whose warps are
constexpr int kWarpRows = 16;      // rows of a unit of that one
constexpr int kPrefixRows = 256;   // rows of a unit of the tensor-core kernel
constexpr int kPrefixTile = 128;   // its keys per tile

// Share c of W tiles dealt to C <= W workers: the first W % C have a tile more.  (W < 2^31: 64-bit divisions were most of a short
// call's instructions.)
struct Shares {
    uint32_t each, rest;
    __host__ __device__ Shares(uint32_t W, uint32_t C) : each(W / C), rest(W - W / C * C) {}
    __host__ __device__ uint32_t start(uint32_t c) const { return each * c + (c < rest ? c : rest); }
    __host__ __device__ uint32_t of(uint32_t x) const {            // the share that tile x is in
        const uint32_t longer = rest * (each + 1);
        return x < longer ? x / (each + 1) : rest + (x - longer) / each;
    }
};

// Where a launch leaves its pieces.
struct PieceSpace {
    float* o;                      // [pieces][rows][dim]
    float2* ml;                    // [pieces][rows] (m, l)
    int rows, shift;               // rows of a unit; keys of a tile as a power of two
    int workers, least_shift;      // workers at most; a worker gets 2^least_shift tiles at least (less where that is all)
    long long pieces;              // room (units + workers; tokens counted twice by a cu_tokens that does not ascend find none)
    int total;                     // tiles; -1: written by the launch to AttendParams::total
};
__host__ __device__ inline uint32_t share_count(const PieceSpace& s, uint32_t W) {
    const uint32_t c = W >> s.least_shift;
    return c < 1 ? 1 : c < (uint32_t)s.workers ? c : (uint32_t)s.workers;
}

// Division by a fixed d >= 1 of numbers below 2^31.
struct FixedDiv {
    uint32_t mul, shift;
    __device__ __forceinline__ uint32_t of(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
};
inline FixedDiv fixed_div(uint32_t d) {
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    return FixedDiv{(uint32_t)(((1ull << 32) * ((1ull << l) - d)) / d + 1), l};
}

struct AttendParams {
    const void* q;
    void* out;
    float* lse;                    // [T, q_heads] or nullptr
    int64_t q_t, q_h, out_t, out_h;
    const void* k;
    const void* v;
    BatchView batch;
    int q_heads, kv_heads, group;  // group = q_heads / kv_heads
    int dim;
    FixedDiv by_group, by_page;
    float scale_log2;              // scale * log2(e)
    PieceSpace prefix, own;        // (the same where one launch has both)
    int tc, own_tc;                // the prefix / the own tokens run on the tensor-core kernel
    // of this launch: which parts it has, its pieces, and whether it may run beside the launch ahead (the prefix's)
    int with_prefix, with_own, beside;
    PieceSpace here;
    int32_t* total;                // [2] tiles of the launch with the prefix / with the own tokens
    int32_t* first_tile;           // [B] where a sequence's own tiles start in their launch
    int32_t* first_unit;           // [B] and its units
    int32_t* status;
};

// The order of launches.  A kernel waits for the launches ahead before it touches memory; the own tokens' launch behind the
// prefix's needs nothing of that one, which has let it start after its own wait: it waits at its end instead, so that the
// join, which waits for this launch alone, finds both done.
__device__ __forceinline__ void launch_begins(const AttendParams& p) {
    if (!p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
__device__ __forceinline__ void launch_ends(const AttendParams& p) {
    if (p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// What a sequence has: own tokens [0, held + tokens), of which the table holds `all`.
struct SequenceView {
    int first, tokens, held;       // held < 0: padding
    int all;
};
__device__ __forceinline__ SequenceView sequence_view(const BatchView& v, int b) {
    SequenceView s;
    s.held = __ldg(v.lengths + b);
    s.first = v.cu ? __ldg(v.cu + b) : b;
    s.first = max(0, s.first);
    s.tokens = v.cu ? max(0, min(max(0, __ldg(v.cu + b + 1)), v.T) - s.first) : 1;     // (both at least 0: no difference wraps)
    // (the table holds fewer than 2^29 keys: what lies past it does not exist, and sums stay inside 31 bits)
    s.held = min(s.held, 0x1FFFFFFF);
    s.tokens = min(s.tokens, 0x1FFFFFFF);
    s.all = s.held < 0 ? 0 : (int)min((long long)s.held + s.tokens, (long long)v.width * v.page);
    return s;
}

// Places of keys in the cache, for one list of pages.
struct PageList {
    const int32_t* pages;
    int n;                         // pages in the list
};
__device__ __forceinline__ PageList page_list(const BatchView& v, int b) {
    PageList l;
    l.pages = b < 0 ? v.prefix_pages : v.table + (size_t)b * v.width;
    l.n = b < 0 ? (v.prefix + v.page - 1) / v.page : v.width;
    return l;
}
// Row of [page * kv_heads][page_size] that holds a key of kv head h, -1 where there is none.
__device__ __forceinline__ long long key_row(const PageList& l, const BatchView& v, const FixedDiv& by_page, int key, int kv_heads, int h) {
    const unsigned slot = by_page.of((unsigned)key), at = (unsigned)key - slot * (unsigned)v.page;
    if ((int)slot >= l.n) return -1;
    const long long page = __ldg(l.pages + slot);
    if (page < 0 || page >= v.n_pages) return -1;
    return (page * kv_heads + h) * v.page + at;
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Factor of a piece when it joins others whose largest maximum is `base`: none where the row saw nothing there; a sum that is
// NaN stays one.
__device__ __forceinline__ float piece_factor(float2 ml, float base) {
    return ml.y != ml.y ? ml.y : ml.x == -INFINITY ? 0.f : exp2_fast(ml.x - base);
}

__device__ __forceinline__ int row_tiles(const AttendParams& p, int tokens, int rows) {
    return (int)(((unsigned)tokens * (unsigned)p.group + (unsigned)rows - 1u) / (unsigned)rows);     // (T * q_heads < 2^31 - 2^8)
}

// A place in the row of tiles of a launch: the prefix's units first, then sequence by sequence; a sequence's units are its
// tiles of rows, for each of them the kv heads, each as many tiles as the sequence has keys.  The walk visits the tiles of
// a share in order and leaves out those behind the last key that any row of a unit sees.
struct Walk {
    int left;                      // tiles of the share, this one included
    int b;                         // -1: the prefix
    int rt, h, tile, unit;         // tile of rows, kv head, tile of keys, unit
    int n_rt, tiles;               // of this sequence
    int first, tokens, held, hi;   // hi: keys that the unit's rows see, at most

    __device__ __forceinline__ void enter(const AttendParams& p, int seq) {        // sizes of a sequence
        b = seq;
        int keys = p.batch.prefix;
        if (b < 0) {
            first = 0, tokens = p.batch.T, held = 0;
        } else {
            const SequenceView s = sequence_view(p.batch, b);
            first = s.first, tokens = s.tokens, held = s.held, keys = s.all;
        }
        n_rt = row_tiles(p, tokens, p.here.rows);
        tiles = (keys + (1 << p.here.shift) - 1) >> p.here.shift;
    }
    __device__ __forceinline__ void limit(const AttendParams& p) {                 // keys that the unit's rows see
        if (b < 0) {
            hi = p.batch.prefix;
            return;
        }
        const int last = min(tokens - 1, (int)p.by_group.of((unsigned)(rt + 1) * (unsigned)p.here.rows - 1u));
        hi = min((int)min((long long)p.batch.width * p.batch.page, 0x3FFFFFFFll), held + last + 1);
    }
    __device__ __forceinline__ void next_unit(const AttendParams& p) {
        tile = 0;
        ++unit;
        if (++h < p.kv_heads) return;
        h = 0;
        if (++rt < n_rt) {
            limit(p);
            return;
        }
        rt = 0;
        if (b + 1 >= p.batch.B || !p.with_own) {                                   // (no more; shares never get here)
            left = 0;
            return;
        }
        do enter(p, b + 1);
        while ((n_rt == 0 || tiles == 0) && b + 1 < p.batch.B);
        limit(p);
    }
    // To the next tile that has keys; false behind the share's end.
    __device__ __forceinline__ bool settle(const AttendParams& p) {
        while (left > 0 && (tile >= tiles || (long long)tile << p.here.shift >= hi)) {
            left -= tiles - tile;
            if (left > 0) next_unit(p);
        }
        return left > 0;
    }
    __device__ __forceinline__ bool next(const AttendParams& p) {
        --left;
        ++tile;
        return settle(p);
    }
};

// The start of a worker's share, worked out by the first 128 threads of its CTA, which all call it, for its kWorkers workers
// (this thread's is `mine`).  For the
// join CTA 0 leaves the totals, and whoever has a sequence's first tile its start.
template <int kWorkers>
__device__ __forceinline__ Walk start_walk(const AttendParams& p, int mine) {
    constexpr int kThreadsOf = 128, kWarps = kThreadsOf / 32;
    __shared__ long long s_tiles[kWarps];
    __shared__ uint32_t s_x[kWorkers];
    __shared__ int s_units[kWarps], s_b[kWorkers], s_unit[kWorkers];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int B = p.with_own ? p.batch.B : 0, per = (B + kThreadsOf - 1) / kThreadsOf;
    const int b_lo = min(B, tid * per), b_hi = tid < kThreadsOf ? min(B, b_lo + per) : b_lo;
    Walk w;
    long long before = 0;          // tiles and units of the prefix
    int units_before = 0;
    if (p.with_prefix) {
        w.enter(p, -1);
        units_before = w.n_rt * p.kv_heads;
        before = (long long)units_before * w.tiles;
    }
    long long tiles = 0;
    int units = 0;
    for (int b = b_lo; b < b_hi; ++b) {
        w.enter(p, b);
        if (w.tiles == 0) continue;
        units += w.n_rt * p.kv_heads;
        tiles += (long long)w.n_rt * p.kv_heads * w.tiles;
    }
    // (the host has bounded the sum; one that a cu_tokens which does not ascend makes larger is cut off)
    constexpr long long kMost = 0x7FFFFFFF;
    long long x64 = min(tiles, kMost);
    int u = units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xFFFFFFFFu, x64, o);
        const int v = __shfl_up_sync(0xFFFFFFFFu, u, o);
        if (lane >= o) x64 += y, u += v;
    }
    if (lane == 31 && warp < kWarps) s_tiles[warp] = x64, s_units[warp] = u;
    if (tid < kWorkers) s_b[tid] = -2;
    __syncthreads();
    long long W64 = before;
    x64 += before - min(tiles, kMost);
    u += units_before - units;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        if (i < warp) x64 += s_tiles[i], u += s_units[i];
        W64 += s_tiles[i];
    }
    const uint32_t W = (uint32_t)min(W64, kMost);
    uint32_t x = (uint32_t)min(x64, kMost);
    const uint32_t C = W > 0 ? share_count(p.here, W) : 1;
    const Shares shares(W, C);
    const uint32_t c0 = blockIdx.x * kWorkers;
    const auto start = [&](uint32_t c) { return c < C ? shares.start(c) : W; };
    if (blockIdx.x == 0 && tid == 0) {
        if (p.with_prefix) p.total[0] = (int)W;
        if (p.with_own) p.total[1] = (int)W;
    }
    if (tid < kWorkers && start(c0 + tid) < before) s_b[tid] = -1, s_x[tid] = 0, s_unit[tid] = 0;
    if (b_hi > b_lo && x < start(c0 + kWorkers) && x + min(tiles, kMost) > start(c0)) {
        for (int b = b_lo; b < b_hi; ++b) {
            w.enter(p, b);
            if (w.tiles == 0 || w.n_rt == 0) continue;
            if (x >= W) break;         // (behind the cut)
            const uint32_t n = (uint32_t)(w.n_rt * p.kv_heads) * (uint32_t)w.tiles;
            if (x >= start(c0) && x < start(c0 + kWorkers)) p.first_tile[b] = (int)x, p.first_unit[b] = u;
#pragma unroll
            for (int i = 0; i < kWorkers; ++i) {
                const uint32_t lo = start(c0 + i);
                if (x <= lo && lo < x + n) s_b[i] = b, s_x[i] = x, s_unit[i] = u;
            }
            x += n;
            u += w.n_rt * p.kv_heads;
        }
    }
    __syncthreads();
    const uint32_t lo = start(c0 + mine);
    w.left = (int)(start(c0 + mine + 1) - lo);
    if (w.left <= 0 || s_b[mine] == -2) {
        w.left = 0;
        return w;
    }
    w.enter(p, s_b[mine]);
    const uint32_t in = lo - s_x[mine], unit = in / (uint32_t)w.tiles;
    w.tile = (int)(in - unit * (uint32_t)w.tiles);
    w.rt = (int)(unit / (uint32_t)p.kv_heads);
    w.h = (int)(unit - (uint32_t)w.rt * (uint32_t)p.kv_heads);
    w.unit = s_unit[mine] + (int)unit;
    w.limit(p);
    w.settle(p);
    return w;
}

// Row r of a tile of rows: its token and head in the group; false where there is none.
__device__ __forceinline__ bool row_place(const AttendParams& p, const Walk& w, int r, int& t, int& g) {
    const unsigned i = (unsigned)w.rt * (unsigned)p.here.rows + (unsigned)r, j = p.by_group.of(i);
    g = (int)(i - j * (unsigned)p.group);
    t = w.first + (int)j;
    return (int)j < w.tokens;
}
// Keys below this limit are seen by that row.
__device__ __forceinline__ int row_limit(const Walk& w, int t) { return w.b < 0 ? w.hi : min(w.hi, w.held + (t - w.first) + 1); }

}  // namespace meteora
