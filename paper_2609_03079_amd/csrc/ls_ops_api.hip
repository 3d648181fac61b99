// ls_ops_api.hip - the C entry points of include/ls_ops.h: context, checks of arguments, launches.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <utility>

#include "ls_ops_internal.h"

struct ls_ops {
    int device = 0;
    int n_cu = 0;
    hipStream_t stream = nullptr;
    uint8_t* ws = nullptr;
    size_t ws_bytes = 0;
    ls_status sticky = LS_OK;
    char err[256] = "";
};

namespace {

thread_local char g_ops_error[256] = "";

ls_status fail(ls_ops* c, ls_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(c ? c->err : g_ops_error, 256, fmt, ap);
    va_end(ap);
    if (c && st == LS_E_DEVICE) c->sticky = LS_E_DEVICE;
    return st;
}

ls_status launched(ls_ops* c, hipError_t e, const char* what) {
    return e == hipSuccess ? LS_OK : fail(c, LS_E_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

// The context is usable and on its own device.
ls_status check_ctx(ls_ops* c) {
    if (!c) return LS_E_INVAL;
    if (c->sticky != LS_OK) {
        std::snprintf(c->err, sizeof c->err, "context is in a failed state after an earlier device error");
        return c->sticky;
    }
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return launched(c, e, "hipGetDevice");
    if (dev != c->device) return fail(c, LS_E_STATE, "the context belongs to device %d, the current device is %d", c->device, dev);
    return LS_OK;
}

bool is_float(ls_dtype t) { return t == LS_F32 || t == LS_F16 || t == LS_BF16; }
bool element_aligned(const void* p, ls_dtype t) { return ls::aligned(p, ls::type_size(t)); }

#define LS_REQUIRE(cond, ...)                                      \
    do {                                                           \
        if (!(cond)) return fail(c, LS_E_INVAL, __VA_ARGS__);      \
    } while (0)

// What a cache of either kind has to be.
ls_status check_pages(ls_ops* c, const ls_kv_cache* kv) {
    LS_REQUIRE(kv->n_pages >= 1, "cache: n_pages must be >= 1");
    LS_REQUIRE(kv->page_size >= 1 && kv->page_size <= 4096 && !(kv->page_size & (kv->page_size - 1)),
               "cache: page_size must be a power of two in 1..4096");
    LS_REQUIRE((int64_t)kv->n_pages * kv->page_size < (int64_t)1 << 31, "cache: n_pages * page_size must be below 2^31");
    LS_REQUIRE(kv->n_kv_heads >= 1 && kv->n_kv_heads <= 4096, "cache: n_kv_heads must be in 1..4096");
    LS_REQUIRE(kv->head_dim >= 1 && kv->head_dim <= 1024, "cache: head_dim must be in 1..1024");
    LS_REQUIRE(kv->page_stride >= 0 && kv->head_stride >= 0 && kv->token_stride >= 0, "cache: negative stride");
    return LS_OK;
}

ls_status check_cache(ls_ops* c, const ls_kv_cache* kv) {
    LS_REQUIRE(kv, "cache is NULL");
    LS_REQUIRE(kv->k && kv->v, "cache: k or v is NULL");
    LS_REQUIRE(is_float(kv->dtype), "cache: bad dtype");
    const ls_status st = check_pages(c, kv);
    if (st != LS_OK) return st;
    LS_REQUIRE(element_aligned(kv->k, kv->dtype) && element_aligned(kv->v, kv->dtype), "cache: k or v is not aligned to its type");
    return LS_OK;
}

ls_status check_kvq(ls_ops* c, const ls_kvq_cache* kv, ls_dtype type) {
    LS_REQUIRE(kv, "cache is NULL");
    LS_REQUIRE(kv->k && kv->v && kv->k_scale && kv->v_scale, "cache: k, v or their scales are NULL");
    LS_REQUIRE(kv->code == LS_FP4 || kv->code == LS_FP8, "cache: code must be LS_FP4 or LS_FP8");
    LS_REQUIRE(is_float(type), "bad type");
    const ls_kv_cache shape = ls::shape_of(*kv, type);
    const ls_status st = check_pages(c, &shape);
    if (st != LS_OK) return st;
    LS_REQUIRE(kv->head_dim % 8 == 0, "cache: head_dim must be a multiple of 8");
    LS_REQUIRE(kv->scale_page_stride >= 0 && kv->scale_head_stride >= 0 && kv->scale_token_stride >= 0, "cache: negative stride of the scales");
    const int64_t eight = kv->code == LS_FP4 ? 4 : 8;  // bytes of eight codes
    LS_REQUIRE(ls::aligned(kv->k, eight) && ls::aligned(kv->v, eight) && kv->page_stride % eight == 0 && kv->head_stride % eight == 0 &&
                   kv->token_stride % eight == 0,
               "cache: codes and their strides must be multiples of %d bytes", (int)eight);
    return LS_OK;
}

ls_status check_append(ls_ops* c, int head_dim, ls_dtype type, const ls_append_args* a) {
    LS_REQUIRE(a, "args is NULL");
    LS_REQUIRE(a->n_tokens >= 0, "n_tokens must be >= 0");
    LS_REQUIRE(a->n_heads >= 0 && a->n_heads <= 4096, "n_heads must be in 0..4096");
    LS_REQUIRE(a->rot_dim >= 0 && a->rot_dim % 2 == 0 && a->rot_dim <= head_dim, "rot_dim must be even and at most head_dim");
    LS_REQUIRE(a->style == LS_ROPE_HALF || a->style == LS_ROPE_PAIR, "bad style");
    LS_REQUIRE(a->n_tokens == 0 || ((a->q != nullptr) == (a->n_heads > 0) && (a->q_out != nullptr) == (a->n_heads > 0)),
               "q and q_out go with n_heads > 0, and only with it");
    if (a->n_tokens == 0) return LS_OK;
    LS_REQUIRE(a->k && a->v && a->slots, "k, v or slots is NULL");
    LS_REQUIRE(a->rot_dim == 0 || (a->positions && a->cos_sin && a->n_pos >= 1), "a rotation needs positions and cos_sin of n_pos >= 1 rows");
    for (int64_t s : {a->k_token_stride, a->k_head_stride, a->v_token_stride, a->v_head_stride, a->q_token_stride, a->q_head_stride,
                      a->q_out_token_stride, a->q_out_head_stride})
        LS_REQUIRE(s >= 0, "negative stride");
    LS_REQUIRE(element_aligned(a->k, type) && element_aligned(a->v, type) && element_aligned(a->q, type) &&
                   element_aligned(a->q_out, type) && ls::aligned(a->positions, 4) && ls::aligned(a->slots, 4) && ls::aligned(a->cos_sin, 4),
               "a pointer is not aligned to its type");
    return LS_OK;
}

ls_status check_attend(ls_ops* c, const ls_kv_cache* kv, const ls_attend_args* a, const char* no_f32) {
    LS_REQUIRE(a, "args is NULL");
    if (kv->dtype == LS_F32) return fail(c, LS_E_UNSUPPORTED, "%s", no_f32);
    LS_REQUIRE(kv->head_dim % 8 == 0 && kv->head_dim <= 256, "head_dim must be a multiple of 8, at most 256");
    LS_REQUIRE(a->n_seqs >= 0, "n_seqs must be >= 0");
    LS_REQUIRE(a->n_q >= 1 && a->n_q <= 16, "n_q must be in 1..16");
    LS_REQUIRE(a->n_heads >= 1 && a->n_heads <= 4096 && a->n_heads % kv->n_kv_heads == 0, "n_heads must be a multiple of n_kv_heads, at most 4096");
    LS_REQUIRE(a->prefix_len >= 0 && a->prefix_len < 1 << 22 && a->max_len >= 0 && a->max_len < 1 << 22,
               "prefix_len and max_len must be in 0..2^22 - 1");
    LS_REQUIRE(std::isfinite(a->scale) && a->scale > 0.f, "scale must be finite and > 0");
    if (a->n_seqs == 0) return LS_OK;
    LS_REQUIRE(a->q && a->out && a->lens, "q, out or lens is NULL");
    LS_REQUIRE(a->prefix_len == 0 || a->prefix_pages, "prefix_pages is NULL");
    LS_REQUIRE(a->max_len == 0 || a->pages, "pages is NULL");
    LS_REQUIRE(a->max_len == 0 || (a->pages_stride >= 1 && a->pages_stride >= ls::ceil_div(a->max_len, kv->page_size)),
               "pages_stride pages hold fewer than max_len keys");
    for (int64_t s : {a->q_token_stride, a->q_head_stride, a->out_token_stride, a->out_head_stride})
        LS_REQUIRE(s >= 0 && s % 8 == 0, "strides must be multiples of 8 elements");
    LS_REQUIRE(ls::aligned(a->q, 16) && ls::aligned(a->out, 16), "q, out, k and v must be 16-byte aligned");
    LS_REQUIRE(ls::aligned(a->prefix_pages, 4) && ls::aligned(a->pages, 4) && ls::aligned(a->lens, 4), "a pointer is not aligned to its type");
    return LS_OK;
}

// No two rows of n elements overlap, `a` of them that are by_a apart in each of `b` that are by_b apart.
bool rows_apart(int64_t a, int64_t by_a, int64_t b, int64_t by_b, int64_t n) {
    if (a == 1 || b == 1) return a == b || (a == 1 ? by_b : by_a) >= n;
    const int64_t outer = std::max(by_a, by_b), inner = std::min(by_a, by_b), of_inner = by_a < by_b ? a : b;
    if (inner < n) return false;
    if ((outer - n) / inner >= of_inner - 1) return true;  // one nested in the other
    // otherwise two rows that are j of the b apart: the nearest are as many of the a apart the other way, or one more
    for (int64_t j = 1; j < b; ++j) {
        const __int128 off = (__int128)j * by_b;
        const int64_t i = (int64_t)std::min<__int128>(a - 1, off / by_a);
        if (off - (__int128)i * by_a < n || (i + 1 < a && (__int128)(i + 1) * by_a - off < n)) return false;
    }
    return true;
}

// Launches an attention that was found right, in as many pieces as it takes.
template <typename Plan, typename Launch>
ls_status attend_pieces(ls_ops* c, ls_dtype type, const ls_attend_args* a, const char* what, Plan plan_of, Launch launch) {
    ls_status st;
    // A launch holds fewer than 2^32 threads: more rows than 2^20 (at most 2^21 workgroups for a part) are taken in pieces.
    const int64_t piece = std::max<int64_t>(1, (1 << 20) / ((int64_t)a->n_q * a->n_heads)), es = (int64_t)ls::type_size(type);
    for (int64_t s = 0; s < a->n_seqs; s += piece) {
        ls_attend_args b = *a;
        b.n_seqs = (int32_t)std::min<int64_t>(piece, a->n_seqs - s);
        b.q = static_cast<const char*>(a->q) + s * a->n_q * a->q_token_stride * es;
        b.out = static_cast<char*>(a->out) + s * a->n_q * a->out_token_stride * es;
        if (b.pages) b.pages += s * a->pages_stride;
        b.lens += s;
        ls::AttendPlan plan;
        if (!plan_of(b, &plan))
            return fail(c, LS_E_CAPACITY, "the partial results do not fit the workspace of %zu bytes", c->ws_bytes);
        if ((st = launched(c, launch(b, plan), what)) != LS_OK) return st;
    }
    return LS_OK;
}

}  // namespace

extern "C" {

ls_status ls_ops_create(const ls_ops_desc* desc, ls_ops** out) {
    if (!out) return fail(nullptr, LS_E_INVAL, "out is NULL");
    *out = nullptr;
    if (!desc) return fail(nullptr, LS_E_INVAL, "desc is NULL");
    if (desc->debug_flags != 0) return fail(nullptr, LS_E_INVAL, "debug_flags must be 0");
    const size_t bytes = desc->workspace_bytes ? desc->workspace_bytes : LS_OPS_WORKSPACE_DEFAULT;
    if (bytes < (1u << 20)) return fail(nullptr, LS_E_INVAL, "workspace_bytes must be 0 or at least 1 MiB");
    ls_ops* c = new (std::nothrow) ls_ops();
    if (!c) return fail(nullptr, LS_E_NOMEM, "host allocation failed");
    c->stream = static_cast<hipStream_t>(desc->stream);
    hipError_t e = hipGetDevice(&c->device);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&c->n_cu, hipDeviceAttributeMultiprocessorCount, c->device);
    if (e != hipSuccess) {
        delete c;
        return fail(nullptr, LS_E_DEVICE, "no HIP device: %s", hipGetErrorString(e));
    }
    if (hipMalloc(reinterpret_cast<void**>(&c->ws), bytes) != hipSuccess) {
        (void)hipGetLastError();
        delete c;
        return fail(nullptr, LS_E_NOMEM, "device allocation of the workspace failed (%zu bytes)", bytes);
    }
    c->ws_bytes = bytes;
    *out = c;
    return LS_OK;
}

ls_status ls_ops_destroy(ls_ops* c) {
    if (!c) return LS_E_INVAL;
    (void)hipStreamSynchronize(c->stream);
    (void)hipFree(c->ws);
    delete c;
    return LS_OK;
}

ls_status ls_ops_sync(ls_ops* c) {
    ls_status st = check_ctx(c);
    if (st != LS_OK) return st;
    return launched(c, hipStreamSynchronize(c->stream), "hipStreamSynchronize");
}

const char* ls_ops_last_error(const ls_ops* c) { return c ? c->err : g_ops_error; }

ls_status ls_norm_residual(ls_ops* c, const ls_norm_args* a) {
    ls_status st = check_ctx(c);
    if (st != LS_OK) return st;
    LS_REQUIRE(a, "args is NULL");
    LS_REQUIRE(is_float(a->dtype), "bad dtype");
    LS_REQUIRE(a->n_tokens >= 0, "n_tokens must be >= 0");
    LS_REQUIRE(a->d >= 1 && a->d <= 32768, "d must be in 1..32768");
    LS_REQUIRE((a->post_norm == 0 || a->post_norm == 1) && (a->pre_norm == 0 || a->pre_norm == 1), "post_norm and pre_norm must be 0 or 1");
    LS_REQUIRE(a->eps >= 0.f, "eps must be >= 0");
    if (a->n_tokens == 0) return LS_OK;
    LS_REQUIRE(a->y || !(a->gate || a->post_weight || a->post_norm), "a gate or a norm of y without y");
    LS_REQUIRE(a->post_norm || !a->post_weight, "post_weight without post_norm");
    LS_REQUIRE((a->pre_norm && a->h) || !a->pre_weight, "pre_weight without a pre_norm that writes h");
    LS_REQUIRE(a->x_out || a->h, "x_out and h are both NULL");
    LS_REQUIRE(a->x, "x is NULL");
    // rows of several tokens must not overlap (a read may repeat one row: stride 0)
    const int64_t rows = a->n_tokens > 1 ? a->d : 0;
    LS_REQUIRE(a->x_stride >= 0 && a->y_stride >= 0 && a->gate_stride >= 0, "negative stride");
    LS_REQUIRE(!a->x_out || a->x_out_stride >= rows, "x_out_stride is shorter than a row");
    LS_REQUIRE(!a->h || a->h_stride >= rows, "h_stride is shorter than a row");
    LS_REQUIRE(ls::aligned(a->x, 4) && ls::aligned(a->x_out, 4) && element_aligned(a->y, a->dtype) &&
                   element_aligned(a->gate, a->dtype) && element_aligned(a->post_weight, a->dtype) &&
                   element_aligned(a->pre_weight, a->dtype) && element_aligned(a->h, a->dtype),
               "a pointer is not aligned to its type");
    return launched(c, ls::launch_norm(*a, c->stream), "ls_norm_residual");
}

ls_status ls_linear_i8(ls_ops* c, const ls_linear_i8_args* a) {
    ls_status st = check_ctx(c);
    if (st != LS_OK) return st;
    LS_REQUIRE(a, "args is NULL");
    LS_REQUIRE(a->x_type == LS_I8 || is_float(a->x_type), "bad x_type");
    LS_REQUIRE(is_float(a->out_type), "bad out_type");
    LS_REQUIRE(a->n_tokens >= 0, "n_tokens must be >= 0");
    LS_REQUIRE(a->k >= 16 && a->k % 16 == 0 && a->k <= 131056, "k must be a multiple of 16 in 16..131056");
    LS_REQUIRE(a->n >= 1, "n must be >= 1");
    LS_REQUIRE(a->n_tokens == 0 || (a->x_type == LS_I8) == (a->x_scale != nullptr), "x_scale goes with LS_I8 inputs, and only with them");
    if (a->n_tokens == 0) return LS_OK;
    LS_REQUIRE(a->x && a->w && a->w_scale && a->out, "x, w, w_scale or out is NULL");
    LS_REQUIRE(a->x_stride >= 0 && a->w_stride >= 0, "negative stride");
    LS_REQUIRE(a->n_tokens == 1 || a->out_stride >= a->n, "out_stride is shorter than a row");
    const int64_t es = (int64_t)ls::type_size(a->x_type);
    LS_REQUIRE(ls::aligned(a->x, 16) && (a->x_stride * es) % 16 == 0, "rows of x must be 16-byte aligned");
    LS_REQUIRE(ls::aligned(a->w, 16) && a->w_stride % 16 == 0, "rows of w must be 16-byte aligned");
    LS_REQUIRE(ls::aligned(a->w_scale, 4) && ls::aligned(a->x_scale, 4) && ls::aligned(a->bias, 4) && element_aligned(a->out, a->out_type),
               "a pointer is not aligned to its type");
    LS_REQUIRE(a->x_type == LS_I8 || a->n_tokens < 1 << 23, "n_tokens must be below 2^23 where x is quantised on the way");
    const size_t need = ls::linear_workspace(*a);
    if (need > c->ws_bytes)
        return fail(c, LS_E_CAPACITY, "the quantised tokens take %zu bytes, the workspace has %zu", need, c->ws_bytes);
    return launched(c, ls::launch_linear(*a, c->ws, c->ws_bytes, c->n_cu, c->stream), "ls_linear_i8");
}

ls_status ls_kv_append(ls_ops* c, const ls_kv_cache* kv, const ls_append_args* a) {
    ls_status st = check_ctx(c);
    if (st != LS_OK) return st;
    if ((st = check_cache(c, kv)) != LS_OK) return st;
    if ((st = check_append(c, kv->head_dim, kv->dtype, a)) != LS_OK || a->n_tokens == 0) return st;
    return launched(c, ls::launch_append(*kv, *a, c->stream), "ls_kv_append");
}

ls_status ls_attend(ls_ops* c, const ls_kv_cache* kv, const ls_attend_args* a) {
    ls_status st = check_ctx(c);
    if (st != LS_OK) return st;
    if ((st = check_cache(c, kv)) != LS_OK) return st;
    if ((st = check_attend(c, kv, a, "ls_attend takes f16 and bf16 caches")) != LS_OK || a->n_seqs == 0) return st;
    for (int64_t s : {kv->page_stride, kv->head_stride, kv->token_stride}) LS_REQUIRE(s % 8 == 0, "strides must be multiples of 8 elements");
    LS_REQUIRE(ls::aligned(kv->k, 16) && ls::aligned(kv->v, 16), "q, out, k and v must be 16-byte aligned");
    auto plan = [&](const ls_attend_args& b, ls::AttendPlan* out) { return ls::plan_attend(*kv, b, c->ws_bytes, c->n_cu, out); };
    return attend_pieces(c, kv->dtype, a, "ls_attend", plan, [&](const ls_attend_args& b, const ls::AttendPlan& plan) {
        return ls::launch_attend(*kv, b, plan, c->ws, c->stream);
    });
}

ls_status ls_kvq_append(ls_ops* c, const ls_kvq_cache* kv, ls_dtype type, const ls_append_args* a) {
    ls_status st = check_ctx(c);
    if (st != LS_OK) return st;
    if ((st = check_kvq(c, kv, type)) != LS_OK) return st;
    if ((st = check_append(c, kv->head_dim, type, a)) != LS_OK || a->n_tokens == 0) return st;
    return launched(c, ls::launch_kvq_append(*kv, type, *a, c->stream), "ls_kvq_append");
}

ls_status ls_kvq_read(ls_ops* c, const ls_kvq_cache* kv, const ls_kvq_read_args* a) {
    ls_status st = check_ctx(c);
    if (st != LS_OK) return st;
    LS_REQUIRE(a, "args is NULL");
    if ((st = check_kvq(c, kv, a->type)) != LS_OK) return st;
    LS_REQUIRE(a->n_tokens >= 0, "n_tokens must be >= 0");
    if (a->n_tokens == 0) return LS_OK;
    LS_REQUIRE(a->k && a->v && a->slots, "k, v or slots is NULL");
    for (int64_t s : {a->k_token_stride, a->k_head_stride, a->v_token_stride, a->v_head_stride}) LS_REQUIRE(s >= 0, "negative stride");
    for (const auto& x : {std::make_pair(a->k_token_stride, a->k_head_stride), std::make_pair(a->v_token_stride, a->v_head_stride)})
        LS_REQUIRE(rows_apart(a->n_tokens, x.first, kv->n_kv_heads, x.second, kv->head_dim), "k or v: rows overlap");
    LS_REQUIRE(element_aligned(a->k, a->type) && element_aligned(a->v, a->type) && ls::aligned(a->slots, 4), "a pointer is not aligned to its type");
    return launched(c, ls::launch_kvq_read(*kv, *a, c->stream), "ls_kvq_read");
}

ls_status ls_kvq_attend(ls_ops* c, const ls_kvq_cache* kv, ls_dtype type, const ls_attend_args* a) {
    ls_status st = check_ctx(c);
    if (st != LS_OK) return st;
    if ((st = check_kvq(c, kv, type)) != LS_OK) return st;
    const ls_kv_cache shape = ls::shape_of(*kv, type);
    if ((st = check_attend(c, &shape, a, "ls_kvq_attend takes f16 and bf16 queries")) != LS_OK || a->n_seqs == 0) return st;
    auto plan = [&](const ls_attend_args& b, ls::AttendPlan* out) { return ls::plan_attend_codes(*kv, b, c->ws_bytes, c->n_cu, out); };
    return attend_pieces(c, type, a, "ls_kvq_attend", plan, [&](const ls_attend_args& b, const ls::AttendPlan& plan) {
        const bool half = type == LS_F16;
        return kv->code == LS_FP4 ? (half ? ls::launch_attend_fp4_f16 : ls::launch_attend_fp4_bf16)(*kv, b, plan, c->ws, c->stream)
                                  : (half ? ls::launch_attend_fp8_f16 : ls::launch_attend_fp8_bf16)(*kv, b, plan, c->ws, c->stream);
    });
}

ls_status ls_verify(ls_ops* c, const ls_verify_args* a) {
    ls_status st = check_ctx(c);
    if (st != LS_OK) return st;
    LS_REQUIRE(a, "args is NULL");
    LS_REQUIRE(is_float(a->type), "bad type");
    LS_REQUIRE(a->n_seqs >= 0, "n_seqs must be >= 0");
    LS_REQUIRE(a->n_drafts >= 0 && a->n_drafts <= 63, "n_drafts must be in 0..63");
    LS_REQUIRE(a->vocab >= 1 && a->vocab <= 1 << 30, "vocab must be in 1..2^30");
    if (a->n_seqs == 0) return LS_OK;
    LS_REQUIRE(a->target && a->sample && a->tokens && a->n_accepted, "target, sample, tokens or n_accepted is NULL");
    LS_REQUIRE(a->n_drafts == 0 || (a->drafts && a->accept), "drafts or accept is NULL");
    for (int64_t s : {a->target_seq_stride, a->target_token_stride, a->draft_seq_stride, a->draft_token_stride, a->drafts_stride, a->accept_stride})
        LS_REQUIRE(s >= 0, "negative stride");
    LS_REQUIRE(a->n_seqs == 1 || a->tokens_stride > a->n_drafts, "tokens_stride is shorter than a row");
    LS_REQUIRE(element_aligned(a->target, a->type) && element_aligned(a->draft, a->type) && ls::aligned(a->drafts, 4) && ls::aligned(a->counts, 4) &&
                   ls::aligned(a->accept, 4) && ls::aligned(a->sample, 4) && ls::aligned(a->tokens, 4) && ls::aligned(a->n_accepted, 4),
               "a pointer is not aligned to its type");
    return launched(c, ls::launch_verify(*a, c->ws, c->ws_bytes, c->n_cu, c->stream), "ls_verify");
}

}  // extern "C"
