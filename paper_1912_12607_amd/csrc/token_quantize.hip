// Codes of tokens: a scale for each row, or for each column with the codes transposed (Eq.1 / Eq.3 of the per-tensor quantizer, c the
// maximum of the row or column), and the transposition of codes.
#include <type_traits>

#include "device_common.h"
#include "tokens.h"

namespace int8t {
namespace {

inline int pad16(int v) { return (v + 15) & ~15; }

// Keeps the computation of eight values in front of a change of the rounding mode.
__device__ __forceinline__ void pin8(float v[8]) {
    asm volatile("" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(v[4]), "+v"(v[5]), "+v"(v[6]), "+v"(v[7]));
}

// Stochastic codes of values below 2^-93 go by 2^40 times the values, and by inv in units that much smaller: inv 2^24 would pass fp32's range.
__device__ __forceinline__ bool tiny_values(float inv) { return inv > 0x1p100f; }
__device__ __forceinline__ float stochastic_inv(float inv) { return __fmul_rn(inv, tiny_values(inv) ? 0x1p-16f : kTwo24); }
__device__ __forceinline__ void raise8(float v[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], 0x1p40f);
}

// Codes of eight neighbouring values.  STOCH: in the round-down mode, inv times 2^24 (see stoch_fixed()).
template <bool STOCH>
__device__ __forceinline__ uint2 codes8(const float v[8], float inv, uint32_t kx, uint32_t ka, uint32_t index, uint32_t step) {
    int c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = quantize_one<STOCH>(v[i], inv, kx, ka, index + (uint32_t)i * step);
    return make_uint2(pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7]));
}

// One pass: a row's values are loaded once, stay in registers while their maximum is found, and leave as codes.  TPR lanes have a
// row (256 x 2048 and 1000 x 2048 in fp32: 256 lanes 6.2 us, a wave 6.8); rows beyond 32768 values (LONG) are read a second time, from the caches.
// Bound by memory where codes go to the nearest (8192 and 4096 rows of 4096 values, bf16: 30 us, 5.0 TB/s), by memory and the draws together where
// they are stochastic (8192 rows: 34 us).
template <int TYPE, bool STOCH, int TPR, int CH, bool LONG>
__device__ __forceinline__ void rows_body(const RowsArgs& a, const int block, const int wide, const uint32_t kx, const uint32_t ka) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1, SPAN = TPR * 8 * CH;
    static_assert(!LONG || SPAN == kLongSpan, "the step that the limit of columns goes by");
    const int t = (int)threadIdx.x % TPR;
    const int row = block * RPB + (int)threadIdx.x / TPR;
    const bool live = row < a.rows;            // (all lanes stay for the reductions)
    const int Kp = (a.cols + 15) & ~15;
    const T* __restrict__ x = static_cast<const T*>(a.x) + (size_t)(live ? row : 0) * a.pitch;
    const int cols = live ? a.cols : 0;
    float v[CH][8];
    auto fetch = [&](int base) {
#pragma unroll
        for (int u = 0; u < CH; ++u) {
            const int c = base + (u * TPR + t) * 8;
            load8<TYPE>(x + c, cols - c, wide, v[u]);
        }
        if (a.factor) {
#pragma unroll
            for (int u = 0; u < CH; ++u) {
                const int c = base + (u * TPR + t) * 8;
                float f[8];
                load8<kF32>(a.factor + c, cols - c, true, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] = __fmul_rn(v[u][i], f[i]);
            }
        }
    };
    float m = 0.0f;
    for (int base = 0; base < (LONG ? a.cols : 1); base += SPAN) {
        fetch(base);
#pragma unroll
        for (int u = 0; u < CH; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) m = most(m, fabsf(v[u][i]));
    }
    m = wave_maximum(m);
    if constexpr (TPR > 64) {
        __shared__ float lds[TPR / 64];
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
        __syncthreads();
        m = lds[0];
#pragma unroll
        for (int i = 1; i < TPR / 64; ++i) m = most(m, lds[i]);
    }
    float inv = inv_scale_of(m), sc = token_scale_of(m);
    if (live && t == 0) a.scale[row] = sc;
    const bool tiny = STOCH && tiny_values(inv);
    if (STOCH) inv = stochastic_inv(inv);
    int8_t* __restrict__ q = a.q + (size_t)(live ? row : 0) * Kp;
    for (int base = 0; base < (LONG ? a.cols : 1); base += SPAN) {
        if (LONG) fetch(base);
        if (tiny) {
#pragma unroll
            for (int u = 0; u < CH; ++u) raise8(v[u]);
        }
#pragma unroll
        for (int u = 0; u < CH; ++u) pin8(v[u]);
        if (STOCH) fp32_round_down_mode(inv, sc);
#pragma unroll
        for (int u = 0; u < CH; ++u) {
            const int c = base + (u * TPR + t) * 8;
            const uint2 o = codes8<STOCH>(v[u], inv, kx, ka, (uint32_t)row * (uint32_t)a.cols + (uint32_t)c, 1u);
            if (live && c < Kp) *reinterpret_cast<uint2*>(q + c) = o;      // (values beyond the row are zero, and so are their codes)
        }
        if (STOCH) fp32_round_nearest_mode(inv);
    }
}

// Two matrices of as many columns in one launch (tokens and weights; a launch more costs small layers as much as either): blocks from `first` on
// have the second's rows.
template <int TYPE, bool STOCH, int TPR, int CH, bool LONG>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void quantize_rows_kernel(const RowsArgs a, const RowsArgs b, const int first, const int wide, const uint32_t kx,
                                                                              const uint32_t ka) {
    if ((int)blockIdx.x < first) rows_body<TYPE, STOCH, TPR, CH, LONG>(a, (int)blockIdx.x, wide, kx, ka);
    else rows_body<TYPE, STOCH, TPR, CH, LONG>(b, (int)blockIdx.x - first, wide, kx, ka);
}

inline int row_blocks(int rows, int tpr) { return tpr < 256 ? (rows + 256 / tpr - 1) / (256 / tpr) : rows; }

// Calls f(lanes of a row, chunks of eight values a lane, whether a row is longer): as few lanes as hold a row, at least a wave.
template <typename F>
void for_row_length(int cols, F f) {
    if (cols <= 512) f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>(), std::false_type());
    else if (cols <= 1024) f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>(), std::false_type());
    else if (cols <= 2048) f(std::integral_constant<int, 256>(), std::integral_constant<int, 1>(), std::false_type());
    else if (cols <= 4096) f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>(), std::false_type());
    else if (cols <= 8192) f(std::integral_constant<int, 256>(), std::integral_constant<int, 4>(), std::false_type());
    else if (cols <= 16384) f(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>(), std::false_type());
    else if (cols <= 32768) f(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>(), std::false_type());
    else f(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>(), std::true_type());
}

template <int TYPE, bool STOCH>
void rows_of(const RowsArgs& a, const RowsArgs* b, int wide, hipStream_t st) {
    KernelTimer kt(KID_TOKEN_ROWS, st);
    const uint32_t kx = seed_key_x(a.seed), ka = seed_key_a(a.seed);
    for_row_length(a.cols, [&](auto tpr, auto ch, auto more) {
        constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value;
        const int first = row_blocks(a.rows, TPR);
        launch_timed(kt, (quantize_rows_kernel<TYPE, STOCH, TPR, CH, decltype(more)::value>), dim3(first + (b ? row_blocks(b->rows, TPR) : 0)), dim3(TPR < 256 ? 256 : TPR), 0,
                     st, a, b ? *b : a, first, wide, kx, ka);
    });
}

inline int wide_rows(const void* x, size_t pitch, int type) {
    return (((uintptr_t)x | (pitch * (type == kF32 ? 4 : 2))) & 15) == 0;
}

// ---- scales of columns -----------------------------------------------------------------------
// First pass: maxima of |x factor| and sums of x over a part of the rows, for 256 columns of a block: lane (c, r) has the columns
// 8 c .. + 7 of every eighth row.  Bound by memory (8192 x 4096, bf16: 17 us).
template <int TYPE>
__device__ __forceinline__ void cols_max_body(const ColsArgs& a, const int bx, const int part, const int wide) {
    typedef typename ElemOf<TYPE>::type T;
    __shared__ float lds[8][257];
    const int cg = (int)threadIdx.x & 31, r0 = (int)threadIdx.x >> 5;
    const int col = bx * 256 + cg * 8;
    const int from = (int)((long long)a.rows * part / a.parts), to = (int)((long long)a.rows * (part + 1) / a.parts);
    float m[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int r = from + r0; r < to; r += 8) {
        float v[8];
        load8<TYPE>(static_cast<const T*>(a.x) + (size_t)r * a.pitch + col, a.cols - col, wide, v);
        const float f = a.factor ? a.factor[r] : 1.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[i] += v[i];
            m[i] = most(m[i], fabsf(__fmul_rn(v[i], f)));
        }
    }
    const int c = bx * 256 + (int)threadIdx.x;
#pragma unroll
    for (int i = 0; i < 8; ++i) lds[r0][cg * 8 + i] = m[i];
    __syncthreads();
    if (c < a.cols) {
        float t = lds[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < 8; ++i) t = most(t, lds[i][threadIdx.x]);
        a.part_max[(size_t)part * a.cols + c] = t;
    }
    if (!a.sum) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) lds[r0][cg * 8 + i] = s[i];
    __syncthreads();
    if (c < a.cols) {
        float t = lds[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < 8; ++i) t += lds[i][threadIdx.x];
        a.part_sum[(size_t)part * a.cols + c] = t;
    }
}

__device__ __forceinline__ float parts_sum(const ColsArgs& a, const int c) {
    double s = 0.0;
#pragma unroll 8
    for (int p = 0; p < a.parts; ++p) s += (double)a.part_sum[(size_t)p * a.cols + c];
    return (float)s;
}

template <int TYPE>
__global__ __launch_bounds__(256) void cols_max_kernel(const ColsArgs a, const int wide) {
    cols_max_body<TYPE>(a, (int)blockIdx.x, (int)blockIdx.y, wide);
}

// Sums alone (a bias without its weights): those of the parts, as the second pass forms them.
__global__ __launch_bounds__(256) void cols_sum_kernel(const ColsArgs a) {
    const int c = (int)(blockIdx.x * 256 + threadIdx.x);
    if (c < a.cols) a.sum[c] = parts_sum(a, c);
}

// Tiles of 128 rows, turned in LDS: the codes of four neighbouring rows of a column are one word, 32 words a column, and leave in runs of 128
// bytes along the rows.  A lane has four rows of eight or sixteen columns; words 8, 16, 24 are exchanged by the column so that a wave's lanes
// use all banks.
constexpr int CT_R = 128, CT_PITCH = CT_R + 16;
__device__ __forceinline__ int tile_word(int c, int w) { return c * (CT_PITCH / 4) + (w ^ (((c >> 4) & 3) << 3)); }
template <int COLS>
__device__ __forceinline__ void tile_out(const uint32_t* tile, int8_t* __restrict__ q, int row0, int col0, int rows_p, int cols) {
    const int g = (int)threadIdx.x & 7;
#pragma unroll
    for (int u = 0; u < COLS / 32; ++u) {
        const int c = ((int)threadIdx.x >> 3) + 32 * u;
        const int r = row0 + 16 * g;
        if (col0 + c < cols && r < rows_p) *reinterpret_cast<uint4*>(q + (size_t)(col0 + c) * rows_p + r) = *reinterpret_cast<const uint4*>(tile + tile_word(c, 4 * g));
    }
}
// Second pass: codes of a tile of 128 rows x 64 columns.  Bound by the draws and by memory (8192 x 4096, bf16: 35 us).
constexpr int CT_C = 64;
template <int TYPE, bool STOCH>
__device__ __forceinline__ void cols_codes_body(uint32_t* const tile, const ColsArgs& a, const int bx, const int by, const int wide, const uint32_t kx, const uint32_t ka) {
    typedef typename ElemOf<TYPE>::type T;
    __shared__ __attribute__((aligned(16))) float invs[CT_C];
    const int col0 = bx * CT_C, row0 = by * CT_R;
    // (on their way while the maxima are found)
    const int cg = (int)threadIdx.x & 7, rq = (int)threadIdx.x >> 3;
    const int col = col0 + cg * 8, row = row0 + 4 * rq;
    float v[4][8], f[4], inv[8];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const bool in = row + u < a.rows;
        load8<TYPE>(static_cast<const T*>(a.x) + (size_t)(in ? row + u : 0) * a.pitch + col, in ? a.cols - col : 0, wide, v[u]);
        f[u] = a.factor && in ? a.factor[row + u] : 1.0f;
    }
    // the parts' maxima: four lanes a column
    __shared__ float tops[4][CT_C];
    {
        const int c = (int)threadIdx.x & (CT_C - 1), p0 = (int)threadIdx.x / CT_C;
        const float* const part = a.part_max + (col0 + c < a.cols ? col0 + c : 0);
        float m = 0.0f;
#pragma unroll 8
        for (int p = p0; p < a.parts; p += 4) m = most(m, part[(size_t)p * a.cols]);
        tops[p0][c] = m;
    }
    __syncthreads();
    if (threadIdx.x < CT_C) {
        const int c = col0 + (int)threadIdx.x;
        const float m = most(most(tops[0][threadIdx.x], tops[1][threadIdx.x]), most(tops[2][threadIdx.x], tops[3][threadIdx.x]));
        if (by == 0 && c < a.cols) {
            a.scale[c] = token_scale_of(m);
            if (a.sum) a.sum[c] = parts_sum(a, c);
        }
        const float inv = inv_scale_of(m);
        invs[threadIdx.x] = inv;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] = __fmul_rn(v[u][i], f[u]);
        pin8(v[u]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) inv[i] = invs[cg * 8 + i];
    if (STOCH) {
        float highest = inv[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) highest = fmaxf(highest, inv[i]);
        if (__any(tiny_values(highest))) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float up = tiny_values(inv[i]) ? 0x1p40f : 1.0f;
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u][i] = __fmul_rn(v[u][i], up);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) pin8(v[u]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) inv[i] = stochastic_inv(inv[i]);
    }
    float dummy = 0.0f;
    if (STOCH) {
        pin8(inv);
        fp32_round_down_mode(inv[0], dummy);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        int c[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            c[u] = quantize_one<STOCH>(v[u][i], inv[i], kx, ka, (uint32_t)(row + u) * (uint32_t)a.cols + (uint32_t)(col + i));
        tile[tile_word(cg * 8 + i, rq)] = pack4(c[0], c[1], c[2], c[3]);
    }
    __syncthreads();
    tile_out<CT_C>(tile, a.q, row0, col0, (a.rows + 15) & ~15, a.cols);
}

template <int TYPE, bool STOCH>
__global__ __launch_bounds__(256) void cols_codes_kernel(const ColsArgs a, const int wide, const uint32_t kx, const uint32_t ka) {
    __shared__ __attribute__((aligned(16))) uint32_t tile[CT_C * CT_PITCH / 4];
    cols_codes_body<TYPE, STOCH>(tile, a, (int)blockIdx.x, (int)blockIdx.y, wide, kx, ka);
}

template <int TYPE>
void cols_of(const ColsArgs& a, int wide, hipStream_t st) {
    {
        KernelTimer kt(KID_TOKEN_COLS, st);
        launch_timed(kt, cols_max_kernel<TYPE>, dim3((a.cols + 255) / 256, a.parts), dim3(256), 0, st, a, wide);
    }
    KernelTimer kt(KID_TOKEN_COLS, st);
    if (!a.q) {
        launch_timed(kt, cols_sum_kernel, dim3((a.cols + 255) / 256), dim3(256), 0, st, a);
        return;
    }
    const dim3 grid((a.cols + CT_C - 1) / CT_C, (a.rows + CT_R - 1) / CT_R);
    const uint32_t kx = seed_key_x(a.seed), ka = seed_key_a(a.seed);
    if (a.stochastic) launch_timed(kt, (cols_codes_kernel<TYPE, true>), grid, dim3(256), 0, st, a, wide, kx, ka);
    else launch_timed(kt, (cols_codes_kernel<TYPE, false>), grid, dim3(256), 0, st, a, wide, kx, ka);
}

// Codes [rows][pad16(cols)] -> [cols][pad16(rows)], tiles of 128 x 128.  Bound by memory (8192 x 4096: 13 us).
constexpr int TT_C = 128;
__device__ __forceinline__ void transpose_body(uint32_t* const tile, const int8_t* __restrict__ q, const int rows, const int cols, int8_t* __restrict__ qt, const int bx,
                                               const int by) {
    const int col0 = bx * TT_C, row0 = by * CT_R;
    const int Kp = (cols + 15) & ~15;
    const int g = (int)threadIdx.x & 7, rq = (int)threadIdx.x >> 3;
    const int c = col0 + 16 * g, row = row0 + 4 * rq;
    uint4 t[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        t[u] = make_uint4(0u, 0u, 0u, 0u);
        if (row + u < rows && c < Kp) t[u] = *reinterpret_cast<const uint4*>(q + (size_t)(row + u) * Kp + c);
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t d[4] = {w == 0 ? t[0].x : w == 1 ? t[0].y : w == 2 ? t[0].z : t[0].w, w == 0 ? t[1].x : w == 1 ? t[1].y : w == 2 ? t[1].z : t[1].w,
                               w == 0 ? t[2].x : w == 1 ? t[2].y : w == 2 ? t[2].z : t[2].w, w == 0 ? t[3].x : w == 1 ? t[3].y : w == 2 ? t[3].z : t[3].w};
        uint32_t o[4];
        transpose4x4_bytes(d, o);
#pragma unroll
        for (int i = 0; i < 4; ++i) tile[tile_word(16 * g + 4 * w + i, rq)] = o[i];
    }
    __syncthreads();
    tile_out<TT_C>(tile, qt, row0, col0, (rows + 15) & ~15, cols);
}
__global__ __launch_bounds__(256) void transpose_codes_kernel(const int8_t* __restrict__ q, const int rows, const int cols, int8_t* __restrict__ qt) {
    __shared__ __attribute__((aligned(16))) uint32_t tile[TT_C * CT_PITCH / 4];
    transpose_body(tile, q, rows, cols, qt, (int)blockIdx.x, (int)blockIdx.y);
}

// ---- a gradient's codes for both products, in two launches -------------------------------------
// First: codes of its rows (bound by the draws) beside the maxima of its columns (bound by memory); then: codes of its columns (draws) beside the
// transposition of the other operands' codes (memory).  8192 x 4096, bf16, with weights 4096 x 4096: 45 and 41 us, as much as one after the other; 256 x 1000,
// fp32, with weights 1000 x 2048: 5.8 and 6.3 us, where five launches took 30.  Blocks of either kind take turns in proportion to their numbers: of n + m blocks, those where
// floor((i + 1) n / (n + m)) steps up have the first kind.
__device__ __forceinline__ bool take_turn(int i, int n, int all, int* at) {
    const int before = (int)((long long)i * n / all), after = (int)((long long)(i + 1) * n / all);
    *at = after > before ? before : i - before;
    return after > before;
}
template <int TYPE, int TPR, int CH>
__global__ __launch_bounds__(256) void gradient_first_kernel(const RowsArgs r, const ColsArgs c, const int rblocks, const int cx, const int wide, const uint32_t kx,
                                                             const uint32_t ka) {
    int at;
    if (take_turn((int)blockIdx.x, rblocks, (int)gridDim.x, &at)) rows_body<TYPE, true, TPR, CH, false>(r, at, wide, kx, ka);
    else cols_max_body<TYPE>(c, at % cx, at / cx, wide);
}
template <int TYPE>
__global__ __launch_bounds__(256) void gradient_second_kernel(const ColsArgs c, const int cx, const int cblocks, const Transpose w, const int wx, const int wblocks,
                                                              const Transpose x, const int xx, const int wide, const uint32_t kx, const uint32_t ka) {
    __shared__ __attribute__((aligned(16))) uint32_t tile[TT_C * CT_PITCH / 4];
    int at;
    if (take_turn((int)blockIdx.x, cblocks, (int)gridDim.x, &at)) cols_codes_body<TYPE, true>(tile, c, at % cx, at / cx, wide, kx, ka);
    else if (at < wblocks) transpose_body(tile, w.q, w.rows, w.cols, w.qt, at % wx, at / wx);
    else transpose_body(tile, x.q, x.rows, x.cols, x.qt, (at - wblocks) % xx, (at - wblocks) / xx);
}
inline int over(int n, int d) { return (n + d - 1) / d; }
template <int TYPE>
void gradient_of(const RowsArgs& r, const ColsArgs& c, const Transpose& w, const Transpose& x, int wide, hipStream_t st) {
    const int maxima = over(c.cols, 256);
    for_row_length(r.cols, [&](auto tpr, auto ch, auto) {
        if constexpr (decltype(tpr)::value <= 256) {
            KernelTimer kt(KID_TOKEN_ROWS, st);
            const int rblocks = row_blocks(r.rows, decltype(tpr)::value);
            launch_timed(kt, (gradient_first_kernel<TYPE, decltype(tpr)::value, decltype(ch)::value>), dim3(rblocks + maxima * c.parts), dim3(256), 0, st, r, c, rblocks, maxima,
                         wide, seed_key_x(r.seed), seed_key_a(r.seed));
        }
    });
    KernelTimer kt(KID_TOKEN_COLS, st);
    const int cx = over(c.cols, CT_C), cblocks = cx * over(c.rows, CT_R);
    const int wx = over(w.cols, TT_C), wblocks = wx * over(w.rows, CT_R), xx = over(x.cols, TT_C), xblocks = xx * over(x.rows, CT_R);
    launch_timed(kt, gradient_second_kernel<TYPE>, dim3(cblocks + wblocks + xblocks), dim3(256), 0, st, c, cx, cblocks, w, wx, wblocks, x, xx, wide, seed_key_x(c.seed),
                 seed_key_a(c.seed));
}

}  // namespace

hipError_t launch_quantize_rows(const RowsArgs& a, hipStream_t st, const RowsArgs* b) {
    const int wide = wide_rows(a.x, a.pitch, a.type) && (!b || wide_rows(b->x, b->pitch, b->type));
#define LAUNCH(TY) a.stochastic ? rows_of<TY, true>(a, b, wide, st) : rows_of<TY, false>(a, b, wide, st)
    if (a.type == kF32) LAUNCH(kF32);
    else if (a.type == kBF16) LAUNCH(kBF16);
    else LAUNCH(kF16);
#undef LAUNCH
    return hipGetLastError();
}

// parts of the rows in the first pass: blocks of 256 columns times parts fill the chip, a part has 32 rows at least
int quantize_cols_parts(int rows, int cols) {
    const int want = 1024 / ((cols + 255) / 256), most = (rows + 31) / 32;
    return want < 1 ? 1 : want > 64 ? (most < 64 ? most : 64) : (most < want ? most : want);
}
hipError_t launch_quantize_cols(const ColsArgs& a, hipStream_t st) {
    const int wide = wide_rows(a.x, a.pitch, a.type);
    if (a.type == kF32) cols_of<kF32>(a, wide, st);
    else if (a.type == kBF16) cols_of<kBF16>(a, wide, st);
    else cols_of<kF16>(a, wide, st);
    return hipGetLastError();
}
bool gradient_together(int cols) { return cols <= 8192; }
hipError_t launch_quantize_gradient(const RowsArgs& r, const ColsArgs& c, const Transpose& w, const Transpose& x, hipStream_t st) {
    const int wide = wide_rows(r.x, r.pitch, r.type);
    if (r.type == kF32) gradient_of<kF32>(r, c, w, x, wide, st);
    else if (r.type == kBF16) gradient_of<kBF16>(r, c, w, x, wide, st);
    else gradient_of<kF16>(r, c, w, x, wide, st);
    return hipGetLastError();
}
hipError_t launch_transpose_codes(const int8_t* q, int rows, int cols, int8_t* qt, hipStream_t st) {
    KernelTimer kt(KID_TOKEN_TRANSPOSE, st);
    launch_timed(kt, transpose_codes_kernel, dim3((cols + TT_C - 1) / TT_C, (rows + CT_R - 1) / CT_R), dim3(256), 0, st, q, rows, cols, qt);
    return hipGetLastError();
}

}  // namespace int8t
