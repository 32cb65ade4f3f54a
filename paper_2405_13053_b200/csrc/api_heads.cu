// C ABI of the operators on heads (declared in include/meteora.h): argument validation and dispatch.
#include <math.h>

#include "launch_heads.cuh"

namespace meteora {

static bool known_dtype(meteora_dtype_t t) { return t == METEORA_F32 || t == METEORA_BF16; }
static bool element_aligned(const void* p, meteora_dtype_t t) { return (uintptr_t)p % elem_size(t) == 0; }

// Token counts stay so far below 2^31 that a launch may round them up to whole tiles or add a step to them.
constexpr int kMostTokens = INT32_MAX - 4096;

// A tensor x[T, heads, head_dim]; an output's entries must not coincide.
static int check_heads(const meteora_heads_t* h, int T, int head_dim, meteora_dtype_t dtype, bool output) {
    if (!h || h->heads < 1 || h->stride_token < 0 || h->stride_head < 0) return METEORA_ERR_INVALID_ARG;
    if (h->heads > 65535) return METEORA_ERR_UNSUPPORTED_SHAPE;
    if (T == 0) return METEORA_OK;
    if (!h->data) return METEORA_ERR_INVALID_ARG;
    if (!element_aligned(h->data, dtype)) return METEORA_ERR_MISALIGNED;
    if (output) {
        const int64_t st = h->stride_token, sh = h->stride_head, n = h->heads;
        const bool tokens_outer = (n == 1 || sh >= head_dim) && (T == 1 || st >= (n - 1) * sh + head_dim);
        const bool heads_outer = (T == 1 || st >= head_dim) && (n == 1 || sh >= (int64_t)(T - 1) * st + head_dim);
        if (!tokens_outer && !heads_outer) return METEORA_ERR_INVALID_ARG;
    }
    return METEORA_OK;
}

static int check_rotary(const meteora_rotary_t* rot, int head_dim) {
    if (!rot) return METEORA_OK;
    if (rot->dim < 2 || rot->dim % 2 != 0 || rot->dim > head_dim) return METEORA_ERR_INVALID_ARG;
    if (rot->layout != METEORA_ROTARY_HALF && rot->layout != METEORA_ROTARY_INTERLEAVED) return METEORA_ERR_INVALID_ARG;
    return isfinite(rot->scale) ? METEORA_OK : METEORA_ERR_INVALID_ARG;
}

static int check_sizes(int T, int head_dim, meteora_dtype_t dtype) {
    if (T < 0 || head_dim < 1 || !known_dtype(dtype)) return METEORA_ERR_INVALID_ARG;
    return head_dim <= METEORA_MAX_HEAD_DIM && T <= kMostTokens ? METEORA_OK : METEORA_ERR_UNSUPPORTED_SHAPE;
}

static HeadRows rows_of(const meteora_heads_t& in, const meteora_heads_t& out, const void* gain) {
    return HeadRows{in, out.data, out.stride_token, out.stride_head, gain, 0, 1};
}

static int check_attend_sizes(const meteora_cache_t* c, const meteora_batch_t* b, int q_heads, AttendSizes* z) {
    if (!c || !b || c->kv_heads < 1 || c->page_size < 1 || q_heads < 1 || q_heads % c->kv_heads != 0) return METEORA_ERR_INVALID_ARG;
    if (b->T < 0 || b->B < 0 || b->table_width < 0 || b->prefix_len < 0) return METEORA_ERR_INVALID_ARG;
    if (!known_dtype(c->dtype) || c->head_dim < 1) return METEORA_ERR_INVALID_ARG;
    if (c->head_dim > METEORA_MAX_HEAD_DIM || q_heads > 65535 || b->B > METEORA_MAX_BATCH || c->page_size > (1 << 24))
        return METEORA_ERR_UNSUPPORTED_SHAPE;
    if ((long long)b->table_width * c->page_size >= (1LL << 29) || b->prefix_len >= (1 << 29)) return METEORA_ERR_UNSUPPORTED_SHAPE;
    if ((long long)b->T * q_heads >= (1LL << 31) - 4096) return METEORA_ERR_UNSUPPORTED_SHAPE;
    *z = AttendSizes{b->T, b->B, q_heads, c->kv_heads, c->head_dim, c->page_size, b->table_width, b->prefix_len, c->n_pages, c->dtype};
    return METEORA_OK;
}

#define METEORA_TRY(call)                       \
    do {                                        \
        const int rc_ = (call);                 \
        if (rc_ != METEORA_OK) return rc_;      \
    } while (0)

// q and k in, q and k out: the rotation and the norm with it.
static int head_pass(const meteora_heads_t* q, const meteora_heads_t* k, const void* q_gain, const void* k_gain,
                     const meteora_heads_t* q_out, const meteora_heads_t* k_out, const HeadPassArgs& args, cudaStream_t st) {
    METEORA_TRY(check_sizes(args.T, args.head_dim, args.dtype));
    METEORA_TRY(check_rotary(args.rot, args.head_dim));
    if ((k == nullptr) != (k_out == nullptr)) return METEORA_ERR_INVALID_ARG;
    METEORA_TRY(check_heads(q, args.T, args.head_dim, args.dtype, false));
    METEORA_TRY(check_heads(q_out, args.T, args.head_dim, args.dtype, true));
    if (q->heads != q_out->heads) return METEORA_ERR_INVALID_ARG;
    if (k) {
        METEORA_TRY(check_heads(k, args.T, args.head_dim, args.dtype, false));
        METEORA_TRY(check_heads(k_out, args.T, args.head_dim, args.dtype, true));
        if (k->heads != k_out->heads) return METEORA_ERR_INVALID_ARG;
    }
    if (args.T == 0) return METEORA_OK;
    if (args.rot && !args.positions) return METEORA_ERR_INVALID_ARG;
    if (args.rot && (uintptr_t)args.positions % (args.positions_64 ? 8 : 4) != 0) return METEORA_ERR_MISALIGNED;
    HeadRows segs[2];
    segs[0] = rows_of(*q, *q_out, q_gain);
    if (k) segs[1] = rows_of(*k, *k_out, k_gain);
    return launch_head_pass(segs, k ? 2 : 1, args, st);
}

static int check_cache(const meteora_cache_t* c) {
    if (!c || c->n_pages < 0 || c->kv_heads < 1 || c->page_size < 1) return METEORA_ERR_INVALID_ARG;
    METEORA_TRY(check_sizes(0, c->head_dim, c->dtype));
    if (c->n_pages >= (1LL << 31) || c->kv_heads > 65535 || c->page_size > (1 << 24)) return METEORA_ERR_UNSUPPORTED_SHAPE;
    if (c->n_pages > 0 && (!c->k || !c->v)) return METEORA_ERR_INVALID_ARG;
    if ((uintptr_t)c->k % 16 != 0 || (uintptr_t)c->v % 16 != 0) return METEORA_ERR_MISALIGNED;
    return METEORA_OK;
}

static int check_batch(const meteora_batch_t* b) {
    if (!b || b->B < 0 || b->T < 0 || b->table_width < 0 || b->prefix_len < 0) return METEORA_ERR_INVALID_ARG;
    if (b->B > METEORA_MAX_BATCH || b->T > kMostTokens) return METEORA_ERR_UNSUPPORTED_SHAPE;
    if (!b->cu_tokens && b->T != b->B) return METEORA_ERR_INVALID_ARG;
    if (b->T == 0 || b->B == 0) return METEORA_OK;
    if (!b->lengths || (b->table_width > 0 && !b->page_table)) return METEORA_ERR_INVALID_ARG;
    if ((uintptr_t)b->cu_tokens % 4 != 0 || (uintptr_t)b->lengths % 4 != 0 || (uintptr_t)b->page_table % 4 != 0 ||
        (uintptr_t)b->prefix_pages % 4 != 0)
        return METEORA_ERR_MISALIGNED;
    return METEORA_OK;
}

static BatchView view_of(const meteora_batch_t& b, const meteora_cache_t& c) {
    return BatchView{b.cu_tokens, b.lengths, b.page_table, b.prefix_pages, b.B, b.T, b.table_width, c.page_size, b.prefix_len, c.n_pages};
}

}  // namespace meteora

using namespace meteora;

extern "C" {

int meteora_rotary_init(const meteora_rotary_spec_t* spec, meteora_rotary_t* rot) {
    if (!spec || !rot) return METEORA_ERR_INVALID_ARG;
    const meteora_rotary_spec_t& s = *spec;
    if (s.dim < 2 || s.dim % 2 != 0) return METEORA_ERR_INVALID_ARG;
    if (s.dim > METEORA_MAX_HEAD_DIM) return METEORA_ERR_UNSUPPORTED_SHAPE;
    if (s.layout != METEORA_ROTARY_HALF && s.layout != METEORA_ROTARY_INTERLEAVED) return METEORA_ERR_INVALID_ARG;
    if (!(s.theta > 0.0) || !isfinite(s.theta) || !isfinite(s.attention_scale)) return METEORA_ERR_INVALID_ARG;
    if (s.scaling != METEORA_ROTARY_NONE && s.scaling != METEORA_ROTARY_LINEAR && s.scaling != METEORA_ROTARY_BANDS)
        return METEORA_ERR_INVALID_ARG;
    if (s.scaling != METEORA_ROTARY_NONE && (!(s.factor > 0.0) || !isfinite(s.factor))) return METEORA_ERR_INVALID_ARG;
    if (s.scaling == METEORA_ROTARY_BANDS &&
        (!(s.original_context > 0.0) || !isfinite(s.original_context) || !(s.low < s.high) || !isfinite(s.low) || !isfinite(s.high)))
        return METEORA_ERR_INVALID_ARG;
    const long double two_pi = 6.283185307179586476925286766559005768L;
    meteora_rotary_t out = {};
    for (int i = 0; i < s.dim / 2; ++i) {
        long double f = powl((long double)s.theta, -2.0L * i / s.dim);
        if (s.scaling == METEORA_ROTARY_LINEAR) f /= s.factor;
        if (s.scaling == METEORA_ROTARY_BANDS) {
            long double keep = (s.original_context * f / two_pi - s.low) / ((long double)s.high - s.low);
            keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
            f = keep * f + (1.0L - keep) * f / s.factor;
        }
        const long double turns = f / two_pi, part = turns - floorl(turns);     // whole turns leave no trace at whole positions
        if (!isfinite((double)turns)) return METEORA_ERR_INVALID_ARG;
        const long double scaled = roundl(ldexpl(part, 64));
        out.turns[i] = scaled >= 0x1p64L ? 0 : (uint64_t)scaled;
    }
    out.dim = s.dim;
    out.layout = s.layout;
    out.scale = s.attention_scale;
    *rot = out;
    return METEORA_OK;
}

int meteora_rotary(const meteora_heads_t* q, const meteora_heads_t* k, const meteora_heads_t* q_out, const meteora_heads_t* k_out,
                   const void* positions, int positions_64, int T, int head_dim, meteora_dtype_t dtype, const meteora_rotary_t* rot,
                   int inverse, void* stream) {
    if (!rot) return METEORA_ERR_INVALID_ARG;
    const HeadPassArgs args = {T, head_dim, dtype, positions, positions_64, rot, inverse, 0.f, nullptr};
    return head_pass(q, k, nullptr, nullptr, q_out, k_out, args, (cudaStream_t)stream);
}

int meteora_head_norm_rotary(const meteora_heads_t* q, const meteora_heads_t* k, const void* q_gain, const void* k_gain,
                             const meteora_heads_t* q_out, const meteora_heads_t* k_out, const void* positions, int positions_64,
                             int T, int head_dim, meteora_dtype_t dtype, const meteora_rotary_t* rot, float eps, void* stream) {
    if (!(eps >= 0.f) || !isfinite(eps)) return METEORA_ERR_INVALID_ARG;
    if (T != 0 && (!q_gain || (k && !k_gain))) return METEORA_ERR_INVALID_ARG;
    if (known_dtype(dtype) && (!element_aligned(q_gain, dtype) || !element_aligned(k_gain, dtype))) return METEORA_ERR_MISALIGNED;
    const HeadPassArgs args = {T, head_dim, dtype, positions, positions_64, rot, 0, eps, nullptr};
    return head_pass(q, k, q_gain, k_gain, q_out, k_out, args, (cudaStream_t)stream);
}

size_t meteora_head_norm_rotary_backward_workspace_bytes(int T, int q_heads, int k_heads, int head_dim) {
    if (T < 0 || T > kMostTokens || q_heads < 1 || k_heads < 0 || head_dim < 1 || head_dim > METEORA_MAX_HEAD_DIM || q_heads > 65535 || k_heads > 65535) return 0;
    return head_grad_workspace_bytes(T, head_dim);
}

int meteora_head_norm_rotary_backward(const meteora_heads_t* dq_out, const meteora_heads_t* dk_out, const meteora_heads_t* q,
                                      const meteora_heads_t* k, const void* q_gain, const void* k_gain, const meteora_heads_t* dq,
                                      const meteora_heads_t* dk, float* dq_gain, float* dk_gain, const void* positions,
                                      int positions_64, int T, int head_dim, meteora_dtype_t dtype, const meteora_rotary_t* rot,
                                      float eps, void* workspace, size_t workspace_bytes, void* stream) {
    METEORA_TRY(check_sizes(T, head_dim, dtype));
    METEORA_TRY(check_rotary(rot, head_dim));
    if (!(eps >= 0.f) || !isfinite(eps)) return METEORA_ERR_INVALID_ARG;
    const bool has_k = k != nullptr;
    if (has_k != (dk_out != nullptr) || has_k != (dk != nullptr) || has_k != (dk_gain != nullptr)) return METEORA_ERR_INVALID_ARG;
    meteora_heads_t dy[2] = {}, x[2] = {}, dx[2] = {};
    for (int i = 0; i < (has_k ? 2 : 1); ++i) {
        const meteora_heads_t *a = i ? dk_out : dq_out, *b = i ? k : q, *c = i ? dk : dq;
        METEORA_TRY(check_heads(a, T, head_dim, dtype, false));
        METEORA_TRY(check_heads(b, T, head_dim, dtype, false));
        METEORA_TRY(check_heads(c, T, head_dim, dtype, true));
        if (a->heads != b->heads || b->heads != c->heads) return METEORA_ERR_INVALID_ARG;
        dy[i] = *a, x[i] = *b, dx[i] = *c;
    }
    if (!q_gain || !dq_gain || (has_k && !k_gain) || !workspace) return METEORA_ERR_INVALID_ARG;
    if (T > 0 && rot && !positions) return METEORA_ERR_INVALID_ARG;
    if (!element_aligned(q_gain, dtype) || !element_aligned(k_gain, dtype) || (uintptr_t)dq_gain % 4 != 0 ||
        (uintptr_t)dk_gain % 4 != 0 || (uintptr_t)workspace % 16 != 0 || (rot && (uintptr_t)positions % (positions_64 ? 8 : 4) != 0))
        return METEORA_ERR_MISALIGNED;
    if (workspace_bytes < head_grad_workspace_bytes(T, head_dim)) return METEORA_ERR_WORKSPACE_TOO_SMALL;
    const HeadPassArgs args = {T, head_dim, dtype, positions, positions_64, rot, 1, eps, nullptr};
    const void* const gain[2] = {q_gain, has_k ? k_gain : nullptr};
    return launch_head_grad(dy, x, gain, dx, dq_gain, dk_gain, args, (float*)workspace, (cudaStream_t)stream);
}

int meteora_cache_append(const meteora_heads_t* k, const meteora_heads_t* v, const meteora_heads_t* q, const meteora_heads_t* q_out,
                         const void* q_gain, const void* k_gain, float eps, const meteora_rotary_t* rot, const meteora_cache_t* cache,
                         const meteora_batch_t* batch, void* stream) {
    METEORA_TRY(check_cache(cache));
    METEORA_TRY(check_batch(batch));
    METEORA_TRY(check_rotary(rot, cache->head_dim));
    const int T = batch->T, D = cache->head_dim;
    if ((q == nullptr) != (q_out == nullptr) || (q_gain && !q)) return METEORA_ERR_INVALID_ARG;
    if (!(eps >= 0.f) || !isfinite(eps)) return METEORA_ERR_INVALID_ARG;
    METEORA_TRY(check_heads(k, T, D, cache->dtype, false));
    METEORA_TRY(check_heads(v, T, D, cache->dtype, false));
    if (k->heads != cache->kv_heads || v->heads != cache->kv_heads) return METEORA_ERR_INVALID_ARG;
    if (q) {
        METEORA_TRY(check_heads(q, T, D, cache->dtype, false));
        METEORA_TRY(check_heads(q_out, T, D, cache->dtype, true));
        if (q->heads != q_out->heads) return METEORA_ERR_INVALID_ARG;
    }
    if (!element_aligned(q_gain, cache->dtype) || !element_aligned(k_gain, cache->dtype)) return METEORA_ERR_MISALIGNED;
    if (T == 0 || batch->B == 0) return METEORA_OK;
    const BatchView view = view_of(*batch, *cache);
    const HeadPassArgs args = {T, D, cache->dtype, nullptr, 0, rot, 0, eps, &view};
    HeadRows segs[3] = {};
    int n = 0;
    if (q) segs[n++] = rows_of(*q, *q_out, q_gain);
    segs[n++] = HeadRows{*k, cache->k, 0, 0, k_gain, 1, 1};
    segs[n++] = HeadRows{*v, cache->v, 0, 0, nullptr, 1, 0};
    return launch_head_pass(segs, n, args, (cudaStream_t)stream);
}

size_t meteora_prefix_attention_workspace_bytes(const meteora_cache_t* cache, const meteora_batch_t* batch, int q_heads) {
    AttendSizes z;
    return check_attend_sizes(cache, batch, q_heads, &z) == METEORA_OK ? attend_workspace_bytes(z) : 0;
}

int meteora_prefix_attention(const meteora_heads_t* q, const meteora_cache_t* cache, const meteora_batch_t* batch, float scale,
                             const meteora_heads_t* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    METEORA_TRY(check_cache(cache));
    METEORA_TRY(check_batch(batch));
    const int T = batch->T, D = cache->head_dim;
    METEORA_TRY(check_heads(q, T, D, cache->dtype, false));
    METEORA_TRY(check_heads(out, T, D, cache->dtype, true));
    if (q->heads != out->heads || !isfinite(scale)) return METEORA_ERR_INVALID_ARG;
    AttendSizes z;
    METEORA_TRY(check_attend_sizes(cache, batch, q->heads, &z));
    if (T == 0 || batch->B == 0) return METEORA_OK;
    if (!workspace || (batch->prefix_len > 0 && !batch->prefix_pages)) return METEORA_ERR_INVALID_ARG;
    if ((uintptr_t)workspace % 16 != 0 || (uintptr_t)lse % 4 != 0) return METEORA_ERR_MISALIGNED;
    const size_t need = attend_workspace_bytes(z);
    if (need == 0) return METEORA_ERR_UNSUPPORTED_SHAPE;
    if (workspace_bytes < need) return METEORA_ERR_WORKSPACE_TOO_SMALL;
    return launch_prefix_attention(*q, *out, lse, *cache, view_of(*batch, *cache), z, scale, workspace, (cudaStream_t)stream);
}

}  // extern "C"
