// Attention over a paged cache with a shared prefix: what its kernels have in common.
//
// softmax over the keys a query sees is joined from pieces: for a set K of keys and a row of scores s (in units of log2),
//     m = max_K s,  l = sum_K 2^(s - m),  o = sum_K 2^(s - m) v,
// and the pieces of disjoint sets join by the common maximum: o = sum_i 2^(m_i - M) o_i, l likewise, result o / l.  So the
// prefix is computed once for the rows of all sequences together (its keys are read once per tile of rows, not once per
// sequence), every sequence's own pages for its own rows, and both may be cut along the keys where rows are few.  A
// piece leaves (o, m, l) in fp32 in its slot of the workspace; k_attend_join adds the slots of a row in their order.
//
// Slots: [0, prefix_slots) pieces of the prefix, then own_slots pieces of the own tokens.  The pieces of sequence b are
// own_piece(tokens of b) keys long, so a row's number of pieces follows from its own length alone, wherever it runs.
#pragma once

#include "heads.cuh"

namespace meteora {

// The tensor-core kernel's tiles of the prefix (attend_prefix.cuh), `tiles` per unit of rows, dealt to `ctas` CTAs in even
// shares: share c is tiles [share_start(c), share_start(c + 1)) of all units in a row.
struct PrefixShare {
    int ctas;                      // 0: the prefix runs elsewhere
    int units, tiles;
};
__host__ __device__ inline long long share_start(const PrefixShare& s, int c) { return (long long)s.units * s.tiles * c / s.ctas; }
// The share that tile x is in: the largest c with share_start(c) <= x.
__host__ __device__ inline int share_of(const PrefixShare& s, long long x) {
    return (int)(((x + 1) * s.ctas - 1) / ((long long)s.units * s.tiles));
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
    float scale_log2;              // scale * log2(e)
    int prefix_slots, prefix_piece;    // prefix_piece: keys per piece, a multiple of the tile
    int own_slots, own_min;            // own_min: shortest piece, a multiple of the tile
    // rows of a tile, [0] for the prefix and [1] for own tokens: tokens x heads of one kv head; and the tiles there are
    int tile_tokens[2], tile_heads[2], t_tiles[2], g_tiles[2];
    int prefix_items, items;           // of this launch; items [0, prefix_items) are pieces of the prefix
    PrefixShare tc;
    float* part_o;                 // [slots][T * q_heads][dim]
    float2* part_ml;               // [slots][T * q_heads] (m, l)
    int32_t* status;
};

constexpr int kAttendTile = 64;    // keys per tile
constexpr int kPrefixRows = 256;   // rows of a unit of the tensor-core kernel

__host__ __device__ inline int own_piece(int tokens, int own_slots, int own_min) {
    const int even = ((tokens + own_slots - 1) / own_slots + kAttendTile - 1) / kAttendTile * kAttendTile;
    return even > own_min ? even : own_min;
}

// What a sequence's tokens see: its keys are own tokens [0, held + tokens).
struct SequenceView {
    int first, tokens, held;       // held < 0: padding
};
__device__ __forceinline__ SequenceView sequence_view(const BatchView& v, int b) {
    SequenceView s;
    s.held = __ldg(v.lengths + b);
    s.first = v.cu ? __ldg(v.cu + b) : b;
    s.tokens = v.cu ? max(0, __ldg(v.cu + b + 1) - s.first) : 1;
    // (the table holds fewer than 2^29 keys: what lies past it does not exist, and sums stay inside 31 bits)
    s.held = min(s.held, 0x1FFFFFFF);
    s.tokens = min(s.tokens, 0x1FFFFFFF);
    return s;
}
// Own keys there can be at all.
__device__ __forceinline__ long long table_keys(const BatchView& v) { return (long long)v.width * v.page; }

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
__device__ __forceinline__ long long key_row(const PageList& l, const BatchView& v, int key, int kv_heads, int h) {
    const unsigned slot = (unsigned)key / (unsigned)v.page, at = (unsigned)key - slot * (unsigned)v.page;
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

// One piece of work: the rows of a tile against a range of keys.
struct AttendItem {
    bool prefix;
    int slot, piece, h, t0, g0, tile_tokens, tile_heads;
};
__device__ __forceinline__ AttendItem attend_item(const AttendParams& p, int i) {
    AttendItem it;
    it.prefix = i < p.prefix_items;
    const int own = it.prefix ? 0 : 1;
    if (own) i -= p.prefix_items;
    it.tile_tokens = p.tile_tokens[own];
    it.tile_heads = p.tile_heads[own];
    it.h = i % p.kv_heads;
    i /= p.kv_heads;
    it.g0 = i % p.g_tiles[own] * it.tile_heads;
    i /= p.g_tiles[own];
    it.t0 = i % p.t_tiles[own] * it.tile_tokens;
    it.piece = i / p.t_tiles[own];
    it.slot = own * p.prefix_slots + it.piece;
    return it;
}

// The keys of own pages that the tile's rows of one sequence see in a piece, and the limits that hold inside it.
struct OwnRange {
    int b, first, held, t_next, lo, hi;
};
__device__ __forceinline__ OwnRange own_range(const AttendParams& p, int b, int piece, int t_seg, int t_end) {
    OwnRange r;
    const SequenceView s = sequence_view(p.batch, b);
    r.b = b;
    r.first = s.first;
    r.held = s.held;
    r.t_next = min(t_end, max(t_seg + 1, s.first + s.tokens));
    r.lo = r.hi = 0;
    if (s.held >= 0) {
        const int all = (int)min((long long)s.held + s.tokens, table_keys(p.batch));
        const int keys = own_piece(all, p.own_slots, p.own_min);
        const long long start = (long long)piece * keys;
        r.lo = (int)min(start, (long long)all);
        r.hi = (int)min(min(start + keys, (long long)all), (long long)s.held + (r.t_next - s.first));
    }
    return r;
}
// Own keys below this limit are seen by token t of a sequence.
__device__ __forceinline__ int own_limit(const OwnRange& r, int t) { return (int)min((long long)r.held + (t - r.first) + 1, (long long)r.hi); }

}  // namespace meteora
