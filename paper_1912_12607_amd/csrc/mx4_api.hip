// C ABI of the microscaled 4-bit operators, rotary positions and page tables (see include/int8t.h): argument checks, scratch, the order of the launches.
#include "../../include/int8t.h"
#include "mx4.h"
#include "positions.h"
#include "token_api.h"

using namespace int8t;

namespace {

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned(p, 16); }
inline bool type_ok(int8t_dtype t) { return t == INT8T_F32 || t == INT8T_BF16 || t == INT8T_F16; }
inline size_t bytes_of(int8t_dtype t) { return t == INT8T_F32 ? 4 : 2; }
inline int8t_status launched(hipError_t e) { return e == hipSuccess ? INT8T_OK : INT8T_ERR_RUNTIME; }

// rows of codes whose blocks lie along cols: 32-bit indices and counts of threads (eight values each) in the kernels
inline bool codes_ok(int rows, int cols) {
    return rows > 0 && cols > 0 && cols <= INT8T_MAX_REDUCTION && (unsigned long long)rows * (unsigned long long)mx_panels(cols) * 256 < (1ull << 31);
}
inline size_t code_bytes(int rows, int cols) { return align256((size_t)rows * mx_row_bytes(cols)); }
inline size_t scale_bytes(int rows, int cols) { return align256((size_t)mx_panels(cols) * rows * 8); }
inline size_t part_bytes(int rows, int cols) { return align256((size_t)mx_sum_parts(rows) * cols * sizeof(float)); }

int8t_status linear_ok(const int8t_linear_desc* d, bool backward) {
    if (!d) return INT8T_ERR_NULL;
    if (!type_ok(d->type) || !type_ok(d->wtype)) return INT8T_ERR_ARG;
    if (d->M < 0 || (backward && d->M == 0) || d->K <= 0 || d->N <= 0) return INT8T_ERR_SHAPE;
    if (!codes_ok(d->N, d->K) || (d->M > 0 && (!codes_ok(d->M, d->K) || (unsigned long long)d->M * (unsigned long long)d->N >= (1ull << 31)))) return INT8T_ERR_SHAPE;
    if (backward && (!codes_ok(d->M, d->N) || !codes_ok(d->K, d->N) || !codes_ok(d->K, d->M) || !codes_ok(d->N, d->M))) return INT8T_ERR_SHAPE;
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
    uint8_t *xq, *sx, *wq, *sw;
    void* product;
    size_t product_bytes, bytes;
};
// laid_out: W's codes are there;  few: nothing is needed (mx_few_tokens())
FwdScratch fwd_scratch(const int8t_linear_desc* d, bool laid_out, bool few, void* ws) {
    Carve c{static_cast<unsigned char*>(ws)};
    FwdScratch s{};
    if (few) return s;
    s.xq = c.take<uint8_t>(code_bytes(d->M, d->K));
    s.sx = c.take<uint8_t>(scale_bytes(d->M, d->K));
    if (!laid_out) {
        s.wq = c.take<uint8_t>(code_bytes(d->N, d->K));
        s.sw = c.take<uint8_t>(scale_bytes(d->N, d->K));
    }
    s.product_bytes = d->M > 0 ? mx_product_scratch(d->M, d->N, mx_row_bytes(d->K)) : 0;
    s.product = c.take<void>(s.product_bytes);
    s.bytes = c.used;
    return s;
}
struct BwdScratch {
    uint8_t *gq, *sg, *hq, *sh;
    float* part;
    void* product;
    size_t product_bytes, bytes;
};
BwdScratch bwd_scratch(const int8t_linear_desc* d, void* ws) {
    Carve c{static_cast<unsigned char*>(ws)};
    BwdScratch s{};
    s.gq = c.take<uint8_t>(code_bytes(d->M, d->N));
    s.sg = c.take<uint8_t>(scale_bytes(d->M, d->N));
    s.hq = c.take<uint8_t>(code_bytes(d->N, d->M));
    s.sh = c.take<uint8_t>(scale_bytes(d->N, d->M));
    s.part = c.take<float>(part_bytes(d->M, d->N));
    const size_t px = mx_product_scratch(d->M, d->K, mx_row_bytes(d->N)), pw = mx_product_scratch(d->N, d->K, mx_row_bytes(d->M));
    s.product_bytes = px > pw ? px : pw;
    s.product = c.take<void>(s.product_bytes);
    s.bytes = c.used;
    return s;
}

int8t_status cache_ok(const int8t_mx4_cache* c) {
    if (!c || !c->kq || !c->vq || !c->ks || !c->vs) return INT8T_ERR_NULL;
    if (c->pages <= 0 || c->page_size <= 0 || c->heads <= 0 || c->dim <= 0 || c->dim > 256 || (c->dim & 15) || c->heads > 65535) return INT8T_ERR_SHAPE;
    if ((long long)c->pages * c->page_size > 0x7fffffffll) return INT8T_ERR_SHAPE;
    if (!aligned16(c->kq) || !aligned16(c->vq) || !aligned16(c->ks) || !aligned16(c->vs)) return INT8T_ERR_ARG;
    return INT8T_OK;
}
CacheArgs cache_args(const int8t_mx4_cache* c) {
    return CacheArgs{reinterpret_cast<int8_t*>(c->kq), reinterpret_cast<int8_t*>(c->vq), reinterpret_cast<float*>(c->ks), reinterpret_cast<float*>(c->vs),
                     c->pages, c->page_size, c->heads, c->dim, fast_div((unsigned)c->page_size), (long long)c->pages * c->page_size};
}
int8t_status attend_ok(const int8t_mx4_cache* c, const int8t_attend_desc* d) {
    const int8t_status s = cache_ok(c);
    if (s != INT8T_OK) return s;
    return attend_desc_ok(d, c->heads, c->page_size);
}

int8t_status pages_ok(const int8t_pages_desc* d) {
    if (!d) return INT8T_ERR_NULL;
    if (d->requests < 0 || d->width < 0 || d->page_size <= 0 || d->pages < 0 || d->tokens < 0 || d->tokens > 0x7fffffff - 4096) return INT8T_ERR_SHAPE;
    if ((long long)d->width * d->page_size > 0x7fffffffll || d->table_pitch < (size_t)d->width) return INT8T_ERR_SHAPE;
    return INT8T_OK;
}

}  // namespace

extern "C" size_t int8t_mx4_quantize_workspace_bytes(int rows, int cols) { return codes_ok(cols, rows) ? part_bytes(rows, cols) : 0; }

extern "C" int8t_status int8t_mx4_quantize(const void* x_dev, int8t_dtype type, int rows, int cols, size_t pitch, int8t_round mode, uint64_t seed, uint8_t* q_dev,
                                           uint8_t* s_dev, uint8_t* qt_dev, uint8_t* st_dev, float* sum_dev, void* ws_dev, size_t ws_bytes, void* stream) {
    if (!x_dev || !q_dev != !s_dev || !qt_dev != !st_dev || (!q_dev && !qt_dev && !sum_dev) || (sum_dev && !ws_dev)) return INT8T_ERR_NULL;
    if (rows <= 0 || cols <= 0 || pitch < (size_t)cols || (q_dev && !codes_ok(rows, cols)) || ((qt_dev || sum_dev) && !codes_ok(cols, rows))) return INT8T_ERR_SHAPE;
    if (!type_ok(type) || (mode != INT8T_ROUND_NEAREST_EVEN && mode != INT8T_ROUND_STOCHASTIC)) return INT8T_ERR_ARG;
    if (!aligned(x_dev, bytes_of(type)) || !aligned16(q_dev) || !aligned16(s_dev) || !aligned16(qt_dev) || !aligned16(st_dev) || !aligned(sum_dev, 4) || !aligned16(ws_dev))
        return INT8T_ERR_ARG;
    if (sum_dev && ws_bytes < part_bytes(rows, cols)) return INT8T_ERR_WORKSPACE;
    const MxArgs a{x_dev, pitch, type, rows, cols, mode == INT8T_ROUND_STOCHASTIC, seed, q_dev, s_dev, qt_dev, st_dev, sum_dev, static_cast<float*>(ws_dev)};
    return launched(launch_mx_quantize(a, (hipStream_t)stream));
}

extern "C" size_t int8t_mx4_product_workspace_bytes(int M, int N, int K) { return codes_ok(M, K) && codes_ok(N, K) ? mx_product_scratch(M, N, mx_row_bytes(K)) : 0; }

extern "C" int8t_status int8t_mx4_product(const uint8_t* a_dev, const uint8_t* sa_dev, const uint8_t* b_dev, const uint8_t* sb_dev, int M, int N, int K, const float* bias_dev,
                                          void* y_dev, int8t_dtype type, size_t pitch, void* ws_dev, size_t ws_bytes, void* stream) {
    if (!a_dev || !sa_dev || !b_dev || !sb_dev || !y_dev) return INT8T_ERR_NULL;
    if (!codes_ok(M, K) || !codes_ok(N, K) || pitch < (size_t)N || !mx_product_fits(M, N, mx_row_bytes(K))) return INT8T_ERR_SHAPE;
    if (!type_ok(type) || !aligned16(a_dev) || !aligned16(b_dev) || !aligned16(sa_dev) || !aligned16(sb_dev) || !aligned(bias_dev, 4) || !aligned(y_dev, bytes_of(type)) ||
        !aligned16(ws_dev))
        return INT8T_ERR_ARG;
    MxProductArgs a{};
    a.a = a_dev; a.b = b_dev; a.sa = sa_dev; a.sb = sb_dev; a.bias = bias_dev;
    a.M = M; a.N = N; a.Kb = mx_row_bytes(K); a.y = y_dev; a.pitch = pitch; a.type = type;
    a.part = static_cast<float*>(ws_dev);
    return launched(launch_mx_product(a, ws_dev ? ws_bytes : 0, (hipStream_t)stream));
}

extern "C" size_t int8t_mx4_linear_workspace_bytes(const int8t_linear_desc* d, int direction) {
    if (direction < 0 || direction > 2 || linear_ok(d, direction == 1) != INT8T_OK) return 0;
    return direction == 1 ? bwd_scratch(d, nullptr).bytes : fwd_scratch(d, direction == 2, direction == 2 && mx_few_tokens(d->M, d->N, mx_row_bytes(d->K)), nullptr).bytes;
}

extern "C" int8t_status int8t_mx4_linear_fwd(const int8t_linear_desc* d, const int8t_mx4_linear_buffers* b, void* stream) {
    const int8t_status ok = linear_ok(d, false);
    if (ok != INT8T_OK) return ok;
    if (!b || !b->wq != !b->sw || !b->wt != !b->swt || !b->xt != !b->sxt || (!b->w && (!b->wq || b->wt))) return INT8T_ERR_NULL;
    if ((b->w && b->w_pitch < (size_t)d->K) || (b->wt && !codes_ok(d->K, d->N))) return INT8T_ERR_SHAPE;
    if (!aligned16(b->wq) || !aligned16(b->sw) || !aligned16(b->wt) || !aligned16(b->swt) || !aligned(b->w, bytes_of(d->wtype)) || !aligned(b->bias, 4)) return INT8T_ERR_ARG;
    const bool few = !b->w && !b->xt && mx_few_tokens(d->M, d->N, mx_row_bytes(d->K));
    const FwdScratch s = fwd_scratch(d, !b->w, few, b->ws);
    const size_t need = few || (d->M == 0 && (!b->w || b->wq)) ? 0 : s.bytes;
    if (need > 0 && !b->ws) return INT8T_ERR_NULL;
    if (d->M > 0) {
        if (!b->x || !b->y) return INT8T_ERR_NULL;
        if (b->x_pitch < (size_t)d->K || b->y_pitch < (size_t)d->N || (b->xt && !codes_ok(d->K, d->M)) || (!few && !mx_product_fits(d->M, d->N, mx_row_bytes(d->K))))
            return INT8T_ERR_SHAPE;
        if (!aligned(b->x, bytes_of(d->type)) || !aligned(b->y, bytes_of(d->type)) || !aligned16(b->xt) || !aligned16(b->sxt) || !aligned16(b->ws)) return INT8T_ERR_ARG;
    }
    if (b->ws_bytes < need) return INT8T_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    if (few && d->M > 0) {
        const int wide = (((uintptr_t)b->x | b->x_pitch * bytes_of(d->type)) & 15) == 0;
        return launched(launch_mx_few_tokens(MxFewArgs{b->x, b->x_pitch, d->type, d->M, d->K, mx_row_bytes(d->K), d->N, wide, b->wq, b->sw, b->bias, b->y, b->y_pitch}, st));
    }
    uint8_t *const wq = b->wq ? b->wq : s.wq, *const sw = b->wq ? b->sw : s.sw;
    const MxArgs w{b->w, b->w_pitch, d->wtype, d->N, d->K, 0, 0, wq, sw, b->wt, b->swt, nullptr, nullptr};
    const MxArgs x{b->x, b->x_pitch, d->type, d->M, d->K, 0, 0, s.xq, s.sx, b->xt, b->sxt, nullptr, nullptr};
    if (d->M == 0) return b->w ? launched(launch_mx_quantize(w, st)) : INT8T_OK;
    const bool together = b->w && d->wtype == d->type;
    hipError_t e = b->w && !together ? launch_mx_quantize(w, st) : hipSuccess;
    if (e == hipSuccess) e = launch_mx_quantize(x, st, together ? &w : nullptr);
    if (e != hipSuccess) return INT8T_ERR_RUNTIME;
    MxProductArgs a{};
    a.a = s.xq; a.sa = s.sx; a.b = wq; a.sb = sw; a.bias = b->bias;
    a.M = d->M; a.N = d->N; a.Kb = mx_row_bytes(d->K); a.y = b->y; a.pitch = b->y_pitch; a.type = d->type;
    a.part = static_cast<float*>(s.product);
    return launched(launch_mx_product(a, s.product_bytes, st));
}

extern "C" int8t_status int8t_mx4_linear_bwd(const int8t_linear_desc* d, const int8t_mx4_linear_buffers* b, uint64_t seed, void* stream) {
    const int8t_status ok = linear_ok(d, true);
    if (ok != INT8T_OK) return ok;
    if (!b || !b->dy || !b->ws || (!b->dx && !b->dw && !b->db)) return INT8T_ERR_NULL;
    if ((b->dx && (!b->wt || !b->swt)) || (b->dw && (!b->xt || !b->sxt))) return INT8T_ERR_NULL;
    if (b->dy_pitch < (size_t)d->N || (b->dx && !mx_product_fits(d->M, d->K, mx_row_bytes(d->N))) || (b->dw && !mx_product_fits(d->N, d->K, mx_row_bytes(d->M)))) return INT8T_ERR_SHAPE;
    if (!aligned(b->dy, bytes_of(d->type)) || !aligned(b->dx, bytes_of(d->type)) || !aligned(b->dw, bytes_of(d->wtype)) || !aligned(b->db, 4) || !aligned16(b->wt) ||
        !aligned16(b->swt) || !aligned16(b->xt) || !aligned16(b->sxt) || !aligned16(b->ws))
        return INT8T_ERR_ARG;
    const BwdScratch s = bwd_scratch(d, b->ws);
    if (b->ws_bytes < s.bytes) return INT8T_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    const MxArgs g{b->dy, b->dy_pitch, d->type, d->M, d->N, 1, seed, b->dx ? s.gq : nullptr, s.sg, b->dw ? s.hq : nullptr, s.sh, b->db, s.part, b->dw != nullptr};
    hipError_t e = launch_mx_quantize(g, st);
    if (e != hipSuccess) return INT8T_ERR_RUNTIME;
    MxProductArgs px{}, pw{};
    px.part = pw.part = static_cast<float*>(s.product);
    px.a = s.gq; px.sa = s.sg; px.b = b->wt; px.sb = b->swt;
    px.M = d->M; px.N = d->K; px.Kb = mx_row_bytes(d->N); px.y = b->dx; px.pitch = (size_t)d->K; px.type = d->type;
    pw.a = s.hq; pw.sa = s.sh; pw.b = b->xt; pw.sb = b->sxt;
    pw.M = d->N; pw.N = d->K; pw.Kb = mx_row_bytes(d->M); pw.y = b->dw; pw.pitch = (size_t)d->K; pw.type = d->wtype;
    if (b->db && b->dw && mx_sum_parts(d->M) > 1) {
        pw.sum_part = s.part; pw.sum = b->db; pw.sum_parts = mx_sum_parts(d->M);
    }
    if (b->dx && b->dw) e = launch_mx_products(px, pw, s.product_bytes, st);
    else if (b->dx) e = launch_mx_product(px, s.product_bytes, st);
    else if (b->dw) e = launch_mx_product(pw, s.product_bytes, st);
    return launched(e);
}

extern "C" int8t_status int8t_mx4_cache_write(const int8t_mx4_cache* cache, const void* k_dev, const void* v_dev, int8t_dtype type, int tokens, size_t k_token_pitch,
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
    return launched(launch_mx_cache_write(a, (hipStream_t)stream));
}

extern "C" int8t_status int8t_mx4_cache_read(const int8t_mx4_cache* cache, const int64_t* slots_dev, int tokens, void* k_dev, void* v_dev, int8t_dtype type, void* stream) {
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
    return launched(launch_mx_cache_read(a, (hipStream_t)stream));
}

extern "C" size_t int8t_mx4_cache_attend_workspace_bytes(const int8t_mx4_cache* cache, const int8t_attend_desc* desc) {
    return attend_ok(cache, desc) == INT8T_OK ? attend_bytes(attend_args(cache_args(cache), desc, 1)) : 0;
}

extern "C" int8t_status int8t_mx4_cache_attend(const int8t_mx4_cache* cache, const int8t_attend_desc* desc, const void* q_dev, const int* starts_dev, const int* lengths_dev,
                                               const int* table_dev, void* out_dev, float* lse_dev, void* ws_dev, size_t ws_bytes, void* stream) {
    const int8t_status ok = attend_ok(cache, desc);
    if (ok != INT8T_OK) return ok;
    return attend_call(attend_args(cache_args(cache), desc, 1), desc, q_dev, starts_dev, lengths_dev, table_dev, out_dev, lse_dev, ws_dev, ws_bytes, stream);
}

extern "C" int8t_status int8t_mx4_product_division(int M, int N, int K, size_t ws_bytes, int8t_division* out) {
    if (!out) return INT8T_ERR_NULL;
    if (!codes_ok(M, K) || !codes_ok(N, K) || !mx_product_fits(M, N, mx_row_bytes(K))) return INT8T_ERR_SHAPE;
    mx_product_division(M, N, mx_row_bytes(K), ws_bytes, &out->rows, &out->waves, &out->stages, &out->shares);
    return INT8T_OK;
}

extern "C" int8t_status int8t_mx4_cache_attend_division(const int8t_mx4_cache* cache, const int8t_attend_desc* desc, int8t_division* out) {
    const int8t_status ok = attend_ok(cache, desc);
    if (ok != INT8T_OK) return ok;
    if (!out) return INT8T_ERR_NULL;
    if (desc->tokens == 0 || desc->requests == 0) return INT8T_ERR_SHAPE;
    const AttendArgs a = attend_args(cache_args(cache), desc, 1);
    *out = int8t_division{a.rows, a.waves, 0, a.splits};
    return INT8T_OK;
}

extern "C" int8t_status int8t_rotate(const int8t_rotate_desc* d, const int8t_rotate_tensor* first, const int8t_rotate_tensor* second, const int* positions_dev,
                                     const double* turns_dev, void* stream) {
    if (!d || !first) return INT8T_ERR_NULL;
    if (!type_ok(d->type) || (d->interleaved != 0 && d->interleaved != 1) || (d->back != 0 && d->back != 1) || !(d->amplitude - d->amplitude == 0.0f)) return INT8T_ERR_ARG;
    if (d->tokens < 0 || d->dim <= 0 || d->rot <= 0 || d->rot > d->dim || (d->rot & 1) || d->dim > 65536) return INT8T_ERR_SHAPE;
    RotateArgs a{};
    long long heads = 0;
    const size_t e = bytes_of(d->type);
    const int8t_rotate_tensor* const ts[2] = {first, second};
    for (int i = 0; i < 2; ++i) {
        const int8t_rotate_tensor* const t = ts[i];
        if (!t || (i == 1 && t->heads == 0)) continue;
        if (t->heads <= 0) return INT8T_ERR_SHAPE;
        heads += t->heads;
        if (d->tokens == 0) continue;
        if (!t->x || !t->y) return INT8T_ERR_NULL;
        if (t->x == t->y && (t->x_token_pitch != t->y_token_pitch || t->x_head_pitch != t->y_head_pitch)) return INT8T_ERR_ARG;
        if (!aligned(t->x, e) || !aligned(t->y, e)) return INT8T_ERR_ARG;
        a.t[i] = RotateTensor{t->x, t->y, t->x_token_pitch, t->x_head_pitch, t->y_token_pitch, t->y_head_pitch, t->heads,
                              (((uintptr_t)t->x | (t->x_token_pitch | t->x_head_pitch) * e) & 15) == 0, (((uintptr_t)t->y | (t->y_token_pitch | t->y_head_pitch) * e) & 15) == 0};
    }
    if ((long long)d->tokens * heads * ((d->dim + 15) / 16 + 1) > 0x7fffff00ll) return INT8T_ERR_SHAPE;
    if (d->tokens == 0) return INT8T_OK;
    if (!positions_dev || !turns_dev) return INT8T_ERR_NULL;
    if (!aligned(positions_dev, 4) || !aligned(turns_dev, 8)) return INT8T_ERR_ARG;
    a.positions = positions_dev;
    a.turns = turns_dev;
    a.tokens = d->tokens; a.dim = d->dim; a.rot = d->rot; a.type = d->type;
    a.interleaved = d->interleaved; a.back = d->back; a.amplitude = d->amplitude;
    return launched(launch_rotate(a, (hipStream_t)stream));
}

extern "C" int8t_status int8t_pages_extend(const int8t_pages_desc* d, const int* have_dev, const int* add_dev, int* table_dev, const int* free_dev, const int* available_dev,
                                           int* lengths_dev, int* left_dev, int* starts_dev, int64_t* slots_dev, int* positions_dev, int* without_dev, void* stream) {
    const int8t_status ok = pages_ok(d);
    if (ok != INT8T_OK) return ok;
    if ((d->requests > 0 && (!have_dev || !add_dev || !lengths_dev || (!table_dev && d->width > 0))) || (!free_dev && d->pages > 0) || !available_dev || !left_dev || !starts_dev ||
        (d->tokens > 0 && (!slots_dev || !positions_dev)) || !without_dev)
        return INT8T_ERR_NULL;
    for (const void* p : {(const void*)have_dev, (const void*)add_dev, (const void*)table_dev, (const void*)free_dev, (const void*)available_dev, (const void*)lengths_dev,
                          (const void*)left_dev, (const void*)starts_dev, (const void*)positions_dev, (const void*)without_dev})
        if (!aligned(p, 4)) return INT8T_ERR_ARG;
    if (!aligned(slots_dev, 8) || (lengths_dev && (lengths_dev == have_dev || lengths_dev == add_dev)) || left_dev == available_dev) return INT8T_ERR_ARG;
    PagesArgs a{};
    a.have = have_dev; a.add = add_dev; a.table = table_dev; a.table_pitch = d->table_pitch; a.free = free_dev; a.available = available_dev;
    a.requests = d->requests; a.width = d->width; a.page_size = d->page_size; a.pages = d->pages; a.tokens = d->tokens;
    a.by_page = fast_div((unsigned)d->page_size);
    a.lengths = lengths_dev; a.left = left_dev; a.starts = starts_dev; a.positions = positions_dev; a.without = without_dev;
    a.slots = reinterpret_cast<long long*>(slots_dev);
    return launched(launch_pages_extend(a, (hipStream_t)stream));
}

extern "C" int8t_status int8t_pages_shrink(const int8t_pages_desc* d, const int* stay_dev, int* lengths_dev, const int* table_dev, int* free_dev, int* available_dev, void* stream) {
    const int8t_status ok = pages_ok(d);
    if (ok != INT8T_OK) return ok;
    if ((d->requests > 0 && (!stay_dev || !lengths_dev || (!table_dev && d->width > 0))) || (!free_dev && d->pages > 0) || !available_dev) return INT8T_ERR_NULL;
    for (const void* p : {(const void*)stay_dev, (const void*)lengths_dev, (const void*)table_dev, (const void*)free_dev, (const void*)available_dev})
        if (!aligned(p, 4)) return INT8T_ERR_ARG;
    PagesArgs a{};
    a.have = lengths_dev; a.add = stay_dev; a.table = const_cast<int*>(table_dev); a.table_pitch = d->table_pitch; a.free = free_dev; a.available = available_dev;
    a.requests = d->requests; a.width = d->width; a.page_size = d->page_size; a.pages = d->pages;
    a.by_page = fast_div((unsigned)d->page_size);
    a.lengths = lengths_dev; a.left = available_dev;
    return launched(launch_pages_shrink(a, (hipStream_t)stream));
}
