// C ABI of the token operators (see include/int8t.h): argument checks, scratch, the order of the launches.
#include "../../include/int8t.h"
#include "tokens.h"

using namespace int8t;

namespace {

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
inline int pad16(int v) { return (v + 15) & ~15; }
inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned(p, 16); }
inline bool type_ok(int8t_dtype t) { return t == INT8T_F32 || t == INT8T_BF16 || t == INT8T_F16; }
inline size_t bytes_of(int8t_dtype t) { return t == INT8T_F32 ? 4 : 2; }

// codes of rows x cols: 32-bit indices in the kernels
inline bool codes_ok(int rows, int cols) {
    return rows > 0 && cols > 0 && cols <= 0x7ffffff0 && (unsigned long long)rows * (unsigned long long)pad16(cols) < (1ull << 31);
}
// ... of rows: long ones are passed kLongSpan values at a time, counted in an int
inline bool rows_ok(int rows, int cols) { return codes_ok(rows, cols) && cols <= 0x7fffffff - kLongSpan + 1 && rows <= kMostRows; }
inline size_t code_bytes(int rows, int cols) { return align256((size_t)rows * pad16(cols)); }
inline int8t_status launched(hipError_t e) { return e == hipSuccess ? INT8T_OK : INT8T_ERR_RUNTIME; }

size_t cols_bytes(int rows, int cols) { return 2 * align256((size_t)quantize_cols_parts(rows, cols) * cols * sizeof(float)); }

ColsArgs cols_args(const void* x, int type, int rows, int cols, size_t pitch, const float* factor, int stochastic, uint64_t seed, int8_t* q, float* scale,
                   float* sum, void* ws) {
    ColsArgs a{x, pitch, type, rows, cols, factor, stochastic, seed, q, scale, sum, nullptr, nullptr, quantize_cols_parts(rows, cols)};
    a.part_max = static_cast<float*>(ws);
    a.part_sum = a.part_max + align256((size_t)a.parts * cols * sizeof(float)) / sizeof(float);
    return a;
}

int8t_status linear_ok(const int8t_linear_desc* d, bool backward) {
    if (!d) return INT8T_ERR_NULL;
    if (!type_ok(d->type) || !type_ok(d->wtype)) return INT8T_ERR_ARG;
    if (d->M < 0 || (backward && d->M == 0) || d->K <= 0 || d->N <= 0 || d->K > INT8T_MAX_REDUCTION) return INT8T_ERR_SHAPE;
    if (!codes_ok(d->N, d->K) || (d->M > 0 && (!codes_ok(d->M, d->K) || !codes_ok(d->M, d->N)))) return INT8T_ERR_SHAPE;
    if (backward && (d->N > INT8T_MAX_REDUCTION || d->M > INT8T_MAX_REDUCTION || !codes_ok(d->K, d->N) || !codes_ok(d->K, d->M) || !codes_ok(d->N, d->M)))
        return INT8T_ERR_SHAPE;
    return INT8T_OK;
}

// scratch of the two directions, carved in order
struct Carve {
    unsigned char* at;
    size_t used = 0;
    template <typename T>
    T* take(size_t bytes) {
        T* p = at ? reinterpret_cast<T*>(at + used) : nullptr;
        used += align256(bytes);
        return p;
    }
};
struct FwdScratch {
    int8_t* xq;
    float* sx;
    void* product;
    size_t product_bytes, bytes;
};
// served: no codes of x are kept, those of W are there
FwdScratch fwd_scratch(const int8t_linear_desc* d, bool served, void* ws) {
    Carve c{static_cast<unsigned char*>(ws)};
    FwdScratch s{};
    if (served && few_tokens(d->M, pad16(d->K))) return s;
    s.xq = c.take<int8_t>(code_bytes(d->M, d->K));
    s.sx = c.take<float>((size_t)d->M * 4);
    s.product_bytes = product_scratch(d->M, d->N, pad16(d->K));
    s.product = c.take<void>(s.product_bytes);
    s.bytes = c.used;
    return s;
}
struct BwdScratch {
    int8_t *gq, *wqt, *hq, *xqt;
    float *sg, *sh;
    void *cols, *product;
    size_t product_bytes, bytes;
};
BwdScratch bwd_scratch(const int8t_linear_desc* d, void* ws) {
    Carve c{static_cast<unsigned char*>(ws)};
    BwdScratch s{};
    s.gq = c.take<int8_t>(code_bytes(d->M, d->N));
    s.wqt = c.take<int8_t>(code_bytes(d->K, d->N));
    s.hq = c.take<int8_t>(code_bytes(d->N, d->M));
    s.xqt = c.take<int8_t>(code_bytes(d->K, d->M));
    s.sg = c.take<float>((size_t)d->M * 4);
    s.sh = c.take<float>((size_t)d->N * 4);
    s.cols = c.take<void>(cols_bytes(d->M, d->N));
    const size_t px = product_scratch(d->M, d->K, pad16(d->N)), pw = product_scratch(d->N, d->K, pad16(d->M));
    s.product_bytes = px > pw ? px : pw;
    s.product = c.take<void>(s.product_bytes);
    s.bytes = c.used;
    return s;
}

int8t_status cache_ok(const int8t_cache* c) {
    if (!c || !c->kq || !c->vq || !c->ks || !c->vs) return INT8T_ERR_NULL;
    if (c->pages <= 0 || c->page_size <= 0 || c->heads <= 0 || c->dim <= 0 || c->dim > 256 || (c->dim & 15) || c->heads > 65535) return INT8T_ERR_SHAPE;
    if ((long long)c->pages * c->page_size > 0x7fffffffll) return INT8T_ERR_SHAPE;
    if (!aligned16(c->kq) || !aligned16(c->vq) || !aligned16(c->ks) || !aligned16(c->vs)) return INT8T_ERR_ARG;
    return INT8T_OK;
}
CacheArgs cache_args(const int8t_cache* c) {
    return CacheArgs{c->kq, c->vq, c->ks, c->vs, c->pages, c->page_size, c->heads, c->dim, fast_div((unsigned)c->page_size), (long long)c->pages * c->page_size};
}

int8t_status attend_ok(const int8t_cache* c, const int8t_attend_desc* d) {
    const int8t_status s = cache_ok(c);
    if (s != INT8T_OK) return s;
    if (!d) return INT8T_ERR_NULL;
    if (!type_ok(d->type) || (d->causal != 0 && d->causal != 1) || !(d->scale - d->scale == 0.0f)) return INT8T_ERR_ARG;
    if (d->tokens < 0 || d->requests < 0 || d->group <= 0 || d->table_width < 0 || d->longest < 0) return INT8T_ERR_SHAPE;
    if ((unsigned long long)d->tokens * (unsigned long long)c->heads * (unsigned long long)d->group > 0x7fffffffull) return INT8T_ERR_SHAPE;
    if ((unsigned long long)d->tokens * (unsigned long long)d->group / 16 + (unsigned long long)d->requests > 0x7fffffull) return INT8T_ERR_SHAPE;
    if (((unsigned long long)d->tokens * (unsigned long long)d->group / 16 + (unsigned long long)d->requests) * (unsigned long long)c->heads > 0x7fffffffull) return INT8T_ERR_SHAPE;
    if ((long long)d->table_width * c->page_size > kMostKeys || d->table_pitch < (size_t)d->table_width) return INT8T_ERR_SHAPE;
    return INT8T_OK;
}
AttendArgs attend_args(const int8t_cache* c, const int8t_attend_desc* d) {
    AttendArgs a{};
    a.c = cache_args(c);
    a.q_token = d->q_token_pitch;
    a.q_head = d->q_head_pitch;
    a.table_pitch = d->table_pitch;
    a.tokens = d->tokens;
    a.requests = d->requests;
    a.group = d->group;
    a.by_group = fast_div((unsigned)d->group);
    a.by_heads = fast_div((unsigned)c->heads);
    a.width = d->table_width;
    a.type = d->type;
    a.causal = d->causal;
    a.scale = d->scale;
    const int most = d->table_width * c->page_size;
    a.splits = 1;
    if (d->tokens && d->requests) attend_plan(&a, d->longest > 0 && d->longest < most ? d->longest : most);
    return a;
}
size_t attend_bytes(const AttendArgs& a) {
    if (a.splits <= 1) return 0;
    const size_t rows = (size_t)a.splits * a.tokens * a.c.heads * a.group;
    return align256(rows * a.c.dim * sizeof(float)) + align256(2 * rows * sizeof(float));
}

}  // namespace

extern "C" int8t_status int8t_quantize_rows(const void* x_dev, int8t_dtype type, int rows, int cols, size_t pitch, const float* factor_dev, int8t_round mode,
                                            uint64_t seed, int8_t* q_dev, float* scale_dev, void* stream) {
    if (!x_dev || !q_dev || !scale_dev) return INT8T_ERR_NULL;
    if (!rows_ok(rows, cols) || pitch < (size_t)cols) return INT8T_ERR_SHAPE;
    if (!type_ok(type) || (mode != INT8T_ROUND_NEAREST_EVEN && mode != INT8T_ROUND_STOCHASTIC)) return INT8T_ERR_ARG;
    if (!aligned(x_dev, bytes_of(type)) || !aligned16(factor_dev) || !aligned16(q_dev) || !aligned16(scale_dev)) return INT8T_ERR_ARG;
    const RowsArgs a{x_dev, pitch, type, rows, cols, factor_dev, mode == INT8T_ROUND_STOCHASTIC, seed, q_dev, scale_dev};
    return launched(launch_quantize_rows(a, (hipStream_t)stream));
}

extern "C" size_t int8t_quantize_cols_workspace_bytes(int rows, int cols) { return codes_ok(cols, rows) && codes_ok(rows, cols) ? cols_bytes(rows, cols) : 0; }

extern "C" int8t_status int8t_quantize_cols(const void* x_dev, int8t_dtype type, int rows, int cols, size_t pitch, const float* factor_dev, int8t_round mode,
                                            uint64_t seed, int8_t* q_dev, float* scale_dev, float* sum_dev, void* ws_dev, size_t ws_bytes, void* stream) {
    if (!x_dev || !q_dev || !scale_dev || !ws_dev) return INT8T_ERR_NULL;
    if (!codes_ok(rows, cols) || !codes_ok(cols, rows) || rows > 8 * INT8T_MAX_REDUCTION || pitch < (size_t)cols) return INT8T_ERR_SHAPE;
    if (!type_ok(type) || (mode != INT8T_ROUND_NEAREST_EVEN && mode != INT8T_ROUND_STOCHASTIC)) return INT8T_ERR_ARG;
    if (!aligned(x_dev, bytes_of(type)) || !aligned(factor_dev, 4) || !aligned16(q_dev) || !aligned16(scale_dev) || !aligned(sum_dev, 4) || !aligned16(ws_dev))
        return INT8T_ERR_ARG;
    if (ws_bytes < cols_bytes(rows, cols)) return INT8T_ERR_WORKSPACE;
    return launched(launch_quantize_cols(cols_args(x_dev, type, rows, cols, pitch, factor_dev, mode == INT8T_ROUND_STOCHASTIC, seed, q_dev, scale_dev, sum_dev, ws_dev),
                                         (hipStream_t)stream));
}

extern "C" int8t_status int8t_transpose_codes(const int8_t* q_dev, int rows, int cols, int8_t* qt_dev, void* stream) {
    if (!q_dev || !qt_dev) return INT8T_ERR_NULL;
    if (!codes_ok(rows, cols) || !codes_ok(cols, rows) || rows > 8 * INT8T_MAX_REDUCTION) return INT8T_ERR_SHAPE;
    if (!aligned16(q_dev) || !aligned16(qt_dev)) return INT8T_ERR_ARG;
    return launched(launch_transpose_codes(q_dev, rows, cols, qt_dev, (hipStream_t)stream));
}

extern "C" size_t int8t_product_workspace_bytes(int M, int N, int K) {
    return codes_ok(M, K) && codes_ok(N, K) && K <= INT8T_MAX_REDUCTION ? product_scratch(M, N, pad16(K)) : 0;
}

extern "C" int8t_status int8t_product(const int8_t* a_dev, const float* sa_dev, const int8_t* b_dev, const float* sb_dev, int M, int N, int K,
                                      const float* bias_dev, void* y_dev, int8t_dtype type, size_t pitch, void* ws_dev, size_t ws_bytes, void* stream) {
    if (!a_dev || !sa_dev || !b_dev || !y_dev) return INT8T_ERR_NULL;
    if (!codes_ok(M, K) || !codes_ok(N, K) || K > INT8T_MAX_REDUCTION || pitch < (size_t)N || !product_fits(M, N, pad16(K))) return INT8T_ERR_SHAPE;
    if (!type_ok(type) || !aligned16(a_dev) || !aligned16(b_dev) || !aligned(sa_dev, 4) || !aligned(sb_dev, 4) || !aligned(bias_dev, 4) ||
        !aligned(y_dev, bytes_of(type)) || !aligned16(ws_dev))
        return INT8T_ERR_ARG;
    ProductArgs a{};
    a.a = a_dev; a.b = b_dev; a.sa = sa_dev; a.sb = sb_dev; a.bias = bias_dev;
    a.M = M; a.N = N; a.Kp = pad16(K); a.y = y_dev; a.pitch = pitch; a.type = type;
    a.part = static_cast<int32_t*>(ws_dev);
    return launched(launch_product(a, ws_dev ? ws_bytes : 0, (hipStream_t)stream));
}

extern "C" size_t int8t_linear_workspace_bytes(const int8t_linear_desc* d, int direction) {
    if (direction < 0 || direction > 2 || linear_ok(d, direction == 1) != INT8T_OK) return 0;
    return direction == 1 ? bwd_scratch(d, nullptr).bytes : fwd_scratch(d, direction == 2, nullptr).bytes;
}

extern "C" int8t_status int8t_linear_fwd(const int8t_linear_desc* d, const int8t_linear_buffers* b, void* stream) {
    const int8t_status ok = linear_ok(d, false);
    if (ok != INT8T_OK) return ok;
    if (!b || !b->wq || !b->sw) return INT8T_ERR_NULL;
    if (b->w && b->w_pitch < (size_t)d->K) return INT8T_ERR_SHAPE;
    if (!aligned16(b->wq) || !aligned16(b->sw) || !aligned(b->w, bytes_of(d->wtype)) || !aligned(b->bias, 4)) return INT8T_ERR_ARG;
    const bool served = !b->w && !b->xq;
    const FwdScratch s = fwd_scratch(d, served, b->ws);
    if (d->M > 0) {
        if (!b->x || !b->y || (!b->ws && s.bytes > 0) || (!b->xq != !b->sx)) return INT8T_ERR_NULL;
        if (b->x_pitch < (size_t)d->K || b->y_pitch < (size_t)d->N) return INT8T_ERR_SHAPE;
        if (!aligned(b->x, bytes_of(d->type)) || !aligned(b->y, bytes_of(d->type)) || !aligned16(b->xq) || !aligned16(b->sx) || !aligned16(b->ws)) return INT8T_ERR_ARG;
        if (b->ws_bytes < s.bytes) return INT8T_ERR_WORKSPACE;
    }
    const hipStream_t st = (hipStream_t)stream;
    const bool few = served && few_tokens(d->M, pad16(d->K));
    if ((b->w && d->N > kMostRows) || (!few && d->M > kMostRows)) return INT8T_ERR_SHAPE;
    const RowsArgs w{b->w, b->w_pitch, d->wtype, d->N, d->K, nullptr, 0, 0, b->wq, b->sw};
    if (d->M == 0) return b->w ? launched(launch_quantize_rows(w, st)) : INT8T_OK;
    if (few) {
        const int wide = (((uintptr_t)b->x | b->x_pitch * bytes_of(d->type)) & 15) == 0;
        return launched(launch_few_tokens(FewArgs{b->x, b->x_pitch, d->type, d->M, d->K, pad16(d->K), d->N, wide, b->wq, b->sw, b->bias, b->y, b->y_pitch}, st));
    }
    const RowsArgs x{b->x, b->x_pitch, d->type, d->M, d->K, nullptr, 0, 0, b->xq ? b->xq : s.xq, b->sx ? b->sx : s.sx};
    const bool together = b->w && d->wtype == d->type && (long long)d->M + d->N <= kMostRows;
    hipError_t e = b->w && !together ? launch_quantize_rows(w, st) : hipSuccess;
    if (e == hipSuccess) e = launch_quantize_rows(x, st, together ? &w : nullptr);
    if (e != hipSuccess) return INT8T_ERR_RUNTIME;
    ProductArgs a{};
    a.a = x.q; a.sa = x.scale; a.b = b->wq; a.sb = b->sw; a.bias = b->bias;
    a.M = d->M; a.N = d->N; a.Kp = pad16(d->K); a.y = b->y; a.pitch = b->y_pitch; a.type = d->type;
    a.part = static_cast<int32_t*>(s.product);
    return launched(launch_product(a, s.product_bytes, st));
}

extern "C" int8t_status int8t_linear_bwd(const int8t_linear_desc* d, const int8t_linear_buffers* b, uint64_t seed, void* stream) {
    const int8t_status ok = linear_ok(d, true);
    if (ok != INT8T_OK) return ok;
    if (!b || !b->dy || !b->ws || (!b->dx && !b->dw && !b->db)) return INT8T_ERR_NULL;
    if ((b->dx && (!b->wq || !b->sw)) || (b->dw && (!b->xq || !b->sx))) return INT8T_ERR_NULL;
    if (b->dy_pitch < (size_t)d->N) return INT8T_ERR_SHAPE;
    if (!aligned(b->dy, bytes_of(d->type)) || !aligned(b->dx, bytes_of(d->type)) || !aligned(b->dw, bytes_of(d->wtype)) || !aligned(b->db, 4) ||
        !aligned16(b->wq) || !aligned16(b->sw) || !aligned16(b->xq) || !aligned16(b->sx) || !aligned16(b->ws))
        return INT8T_ERR_ARG;
    const BwdScratch s = bwd_scratch(d, b->ws);
    if (b->ws_bytes < s.bytes) return INT8T_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    const RowsArgs g{b->dy, b->dy_pitch, d->type, d->M, d->N, b->sw, 1, seed, s.gq, s.sg};
    const ColsArgs h = cols_args(b->dy, d->type, d->M, d->N, b->dy_pitch, b->dw ? b->sx : nullptr, 1, seed ^ (1ull << 63), b->dw ? s.hq : nullptr, s.sh, b->db, s.cols);
    ProductArgs px{}, pw{};
    px.part = pw.part = static_cast<int32_t*>(s.product);
    px.a = s.gq; px.sa = s.sg; px.b = s.wqt;
    px.M = d->M; px.N = d->K; px.Kp = pad16(d->N); px.y = b->dx; px.pitch = (size_t)d->K; px.type = d->type;
    pw.a = s.hq; pw.sa = s.sh; pw.b = s.xqt;
    pw.M = d->N; pw.N = d->K; pw.Kp = pad16(d->M); pw.y = b->dw; pw.pitch = (size_t)d->K; pw.type = d->wtype;
    hipError_t e = hipSuccess;
    if (b->dx && b->dw && gradient_together(d->N)) {
        e = launch_quantize_gradient(g, h, Transpose{b->wq, d->N, d->K, s.wqt}, Transpose{b->xq, d->M, d->K, s.xqt}, st);
        if (e == hipSuccess) e = launch_products(px, pw, s.product_bytes, st);
        return launched(e);
    }
    if (b->dx) {
        e = launch_quantize_rows(g, st);
        if (e == hipSuccess) e = launch_transpose_codes(b->wq, d->N, d->K, s.wqt, st);
        if (e == hipSuccess) e = launch_product(px, s.product_bytes, st);
        if (e != hipSuccess) return INT8T_ERR_RUNTIME;
    }
    if (b->dw || b->db) e = launch_quantize_cols(h, st);
    if (b->dw && e == hipSuccess) {
        e = launch_transpose_codes(b->xq, d->M, d->K, s.xqt, st);
        if (e == hipSuccess) e = launch_product(pw, s.product_bytes, st);
    }
    return launched(e);
}

extern "C" int8t_status int8t_cache_write(const int8t_cache* cache, const void* k_dev, const void* v_dev, int8t_dtype type, int tokens, size_t k_token_pitch,
                                          size_t k_head_pitch, size_t v_token_pitch, size_t v_head_pitch, const int64_t* slots_dev, void* stream) {
    const int8t_status ok = cache_ok(cache);
    if (ok != INT8T_OK) return ok;
    if (tokens < 0 || (long long)tokens * cache->heads > 0x7fffffffll) return INT8T_ERR_SHAPE;
    if (!type_ok(type)) return INT8T_ERR_ARG;
    if (tokens == 0) return INT8T_OK;
    if (!k_dev || !v_dev || !slots_dev) return INT8T_ERR_NULL;
    const size_t e = bytes_of(type);
    if (!aligned(k_dev, e) || !aligned(v_dev, e) || !aligned(slots_dev, 8)) return INT8T_ERR_ARG;
    CacheMoveArgs a{cache_args(cache), const_cast<void*>(k_dev), const_cast<void*>(v_dev), k_token_pitch, k_head_pitch, v_token_pitch, v_head_pitch,
                    reinterpret_cast<const long long*>(slots_dev), tokens, type, 0};
    a.wide = (((uintptr_t)k_dev | (uintptr_t)v_dev | (k_token_pitch | k_head_pitch | v_token_pitch | v_head_pitch) * e) & 15) == 0;
    return launched(launch_cache_write(a, (hipStream_t)stream));
}

extern "C" int8t_status int8t_cache_read(const int8t_cache* cache, const int64_t* slots_dev, int tokens, void* k_dev, void* v_dev, int8t_dtype type, void* stream) {
    const int8t_status ok = cache_ok(cache);
    if (ok != INT8T_OK) return ok;
    if (tokens < 0 || (long long)tokens * cache->heads > 0x7fffffffll) return INT8T_ERR_SHAPE;
    if (!type_ok(type)) return INT8T_ERR_ARG;
    if (tokens == 0) return INT8T_OK;
    if (!k_dev || !v_dev || !slots_dev) return INT8T_ERR_NULL;
    const size_t e = bytes_of(type), row = (size_t)cache->heads * cache->dim;
    if (!aligned(k_dev, e) || !aligned(v_dev, e) || !aligned(slots_dev, 8)) return INT8T_ERR_ARG;
    const CacheMoveArgs a{cache_args(cache), k_dev, v_dev, row, (size_t)cache->dim, row, (size_t)cache->dim, reinterpret_cast<const long long*>(slots_dev), tokens, type,
                          aligned16(k_dev) && aligned16(v_dev)};
    return launched(launch_cache_read(a, (hipStream_t)stream));
}

extern "C" size_t int8t_cache_attend_workspace_bytes(const int8t_cache* cache, const int8t_attend_desc* desc) {
    return attend_ok(cache, desc) == INT8T_OK ? attend_bytes(attend_args(cache, desc)) : 0;
}

extern "C" int8t_status int8t_cache_attend(const int8t_cache* cache, const int8t_attend_desc* desc, const void* q_dev, const int* starts_dev,
                                           const int* lengths_dev, const int* table_dev, void* out_dev, float* lse_dev, void* ws_dev, size_t ws_bytes,
                                           void* stream) {
    const int8t_status ok = attend_ok(cache, desc);
    if (ok != INT8T_OK) return ok;
    if (desc->tokens == 0) return INT8T_OK;
    if (desc->requests == 0) return INT8T_ERR_SHAPE;
    if (!q_dev || !starts_dev || !lengths_dev || (!table_dev && desc->table_width > 0) || !out_dev) return INT8T_ERR_NULL;
    const size_t e = bytes_of(desc->type);
    if (!aligned(q_dev, e) || !aligned(starts_dev, 4) || !aligned(lengths_dev, 4) || !aligned(table_dev, 4) || !aligned16(out_dev) || !aligned(lse_dev, 4) ||
        !aligned16(ws_dev))
        return INT8T_ERR_ARG;
    AttendArgs a = attend_args(cache, desc);
    const size_t need = attend_bytes(a);
    if (need > 0 && !ws_dev) return INT8T_ERR_NULL;
    if (ws_bytes < need) return INT8T_ERR_WORKSPACE;
    a.q = q_dev;
    a.starts = starts_dev;
    a.lengths = lengths_dev;
    a.table = table_dev;
    a.out = out_dev;
    a.lse = lse_dev;
    a.wide_q = (((uintptr_t)q_dev | (desc->q_token_pitch | desc->q_head_pitch) * e) & 15) == 0;
    a.part_o = static_cast<float*>(ws_dev);
    a.part_ml = a.part_o ? a.part_o + align256((size_t)a.splits * a.tokens * a.c.heads * a.group * a.c.dim * sizeof(float)) / sizeof(float) : nullptr;
    return launched(launch_attend(a, (hipStream_t)stream));
}

extern "C" int8t_status int8t_product_division(int M, int N, int K, size_t ws_bytes, int8t_division* out) {
    if (!out) return INT8T_ERR_NULL;
    if (!codes_ok(M, K) || !codes_ok(N, K) || K > INT8T_MAX_REDUCTION || !product_fits(M, N, pad16(K))) return INT8T_ERR_SHAPE;
    product_division(M, N, pad16(K), ws_bytes, &out->rows, &out->waves, &out->stages, &out->shares);
    return INT8T_OK;
}

extern "C" int8t_status int8t_cache_attend_division(const int8t_cache* cache, const int8t_attend_desc* desc, int8t_division* out) {
    const int8t_status ok = attend_ok(cache, desc);
    if (ok != INT8T_OK) return ok;
    if (!out) return INT8T_ERR_NULL;
    if (desc->tokens == 0 || desc->requests == 0) return INT8T_ERR_SHAPE;
    const AttendArgs a = attend_args(cache, desc);
    *out = int8t_division{a.rows, a.waves, 0, a.splits};
    return INT8T_OK;
}
