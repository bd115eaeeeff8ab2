// Shared by the token operators (scales per token and output channel, paged cache, attention): element types, argument structs,
// launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "profile.h"

namespace int8t {

// Element types of the floating tensors (the values of int8t_dtype)
constexpr int kF32 = 0, kBF16 = 1, kF16 = 2;

typedef _Float16 tk_h2 __attribute__((ext_vector_type(2)));
typedef _Float16 tk_h8 __attribute__((ext_vector_type(8)));
typedef float tk_f4 __attribute__((ext_vector_type(4)));
typedef float tk_f16 __attribute__((ext_vector_type(16)));

template <int TYPE> struct ElemOf;
template <> struct ElemOf<kF32> { typedef float type; };
template <> struct ElemOf<kBF16> { typedef __bf16 type; };
template <> struct ElemOf<kF16> { typedef _Float16 type; };

// Eight elements from p, of which the first `left` exist (left <= 0: none); the others are zero.  `wide`: p is 16-byte aligned
// wherever left >= 8.
template <int TYPE>
__device__ __forceinline__ void load8(const typename ElemOf<TYPE>::type* __restrict__ p, int left, bool wide, float v[8]) {
    typedef typename ElemOf<TYPE>::type T;
    if (wide && left >= 8) {
        if constexpr (TYPE == kF32) {
            const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            typedef T V8 __attribute__((ext_vector_type(8)));
            const V8 a = *reinterpret_cast<const V8*>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? (float)p[i] : 0.0f;
    }
}
// Eight results, each rounded once (to nearest even) to the type
template <int TYPE>
__device__ __forceinline__ void store8(typename ElemOf<TYPE>::type* __restrict__ p, int left, bool wide, const float v[8]) {
    typedef typename ElemOf<TYPE>::type T;
    if (wide && left >= 8) {
        if constexpr (TYPE == kF32) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            typedef T V8 __attribute__((ext_vector_type(8)));
            V8 a;
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = (T)v[i];
            *reinterpret_cast<V8*>(p) = a;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (T)v[i];
    }
}

// Maxima that keep NaN (v_maximum3_f32, as fast as the other), and the scale that belongs to one: a token, channel or column that holds NaN gets codes of 0 and a
// scale of NaN, one that holds an infinity codes of 0 and an infinite scale, so that what is computed from either is NaN.
__device__ __forceinline__ float most(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float token_scale_of(float c) { return c > 0.0f ? __fdiv_rn(c, 127.0f) : c; }

// ---- token_quantize.hip ------------------------------------------------------------------------
struct RowsArgs {            // codes of rows x cols values, a scale for each row
    const void* x;
    size_t pitch;            // elements between rows
    int type, rows, cols;
    const float* factor;     // cols, or null: values are multiplied first
    int stochastic;
    uint64_t seed;
    int8_t* q;               // [rows][pad16(cols)]
    float* scale;            // rows
};
constexpr int kLongSpan = 32768;         // values of a row that a block holds; longer rows are passed in steps of so many: at most 2^31 - kLongSpan columns
constexpr int kMostRows = (1 << 26) - 4;  // a launch has fewer than 2^32 threads, a row 64 at least
// with b (as many columns, the same type and rounding to nearest in both): two matrices in one launch
hipError_t launch_quantize_rows(const RowsArgs& a, hipStream_t st, const RowsArgs* b = nullptr);

struct ColsArgs {            // ... a scale for each column, codes transposed
    const void* x;
    size_t pitch;
    int type, rows, cols;
    const float* factor;     // rows, or null
    int stochastic;
    uint64_t seed;
    int8_t* q;               // [cols][pad16(rows)]; null: sums alone
    float* scale;            // cols
    float* sum;              // cols, or null: sums of x (without the factor)
    float *part_max, *part_sum;   // [parts][cols]
    int parts;
};
int quantize_cols_parts(int rows, int cols);
hipError_t launch_quantize_cols(const ColsArgs& a, hipStream_t st);
hipError_t launch_transpose_codes(const int8_t* q, int rows, int cols, int8_t* qt, hipStream_t st);
struct Transpose {
    const int8_t* q;
    int rows, cols;
    int8_t* qt;
};
// A gradient's codes by rows and by columns, stochastic, and two transpositions, in two launches: where gradient_together(its columns), a block of
// 256 lanes holding a row at least.
bool gradient_together(int cols);
hipError_t launch_quantize_gradient(const RowsArgs& r, const ColsArgs& c, const Transpose& w, const Transpose& x, hipStream_t st);

// ---- token_product.hip -------------------------------------------------------------------------
struct ProductArgs {         // y[m][n] = (sum_k a[m][k] b[n][k]) * (sa[m] * sb[n]) + bias[n]
    const int8_t *a, *b;     // [M][Kp], [N][Kp], Kp = pad16(K), the padding zero in one of them at least
    const float *sa, *sb;    // sb null: ones
    const float* bias;       // null: none
    int M, N, Kp;
    void* y;
    size_t pitch;
    int type;
    int32_t* part;           // partial sums of a split reduction, or null
    int splits;
};
struct FewArgs {             // the same from x itself, codes made on the way: few_tokens(M, Kp)
    const void* x;
    size_t x_pitch;
    int type, M, K, Kp, N, wide;
    const int8_t* wq;
    const float *sw, *bias;
    void* y;
    size_t y_pitch;
};
bool few_tokens(int M, int Kp);
hipError_t launch_few_tokens(const FewArgs& a, hipStream_t st);
bool product_fits(int M, int N, int Kp);      // its blocks fit a launch
void product_division(int M, int N, int Kp, size_t scratch_bytes, int* rows, int* waves, int* stages, int* shares);
size_t product_scratch(int M, int N, int Kp);
hipError_t launch_product(ProductArgs a, size_t scratch_bytes, hipStream_t st);
// Two products, in one launch where both take the same tiles whole.  They share the scratch.
hipError_t launch_products(ProductArgs a, ProductArgs b, size_t scratch_bytes, hipStream_t st);

// ---- token_cache.hip ---------------------------------------------------------------------------
struct CacheArgs {
    int8_t *kq, *vq;         // [pages][heads][page_size][dim]
    float *ks, *vs;          // [pages][heads][page_size]
    int pages, page_size, heads, dim;
    FastDiv by_page;
    long long places;        // pages * page_size
};
struct CacheMoveArgs {       // tokens to (write) or from (read) their places
    CacheArgs c;
    void *k, *v;
    size_t k_token, k_head, v_token, v_head;      // pitches, elements
    const long long* slots;
    int tokens, type;
    int wide;                // 16-byte accesses
};
hipError_t launch_cache_write(const CacheMoveArgs& a, hipStream_t st);
hipError_t launch_cache_read(const CacheMoveArgs& a, hipStream_t st);

// ---- token_attend.hip, token_attend_chunk.hip --------------------------------------------------------------------------
// Keys that a table may have: the kernels look at the pages of tiles ahead, some 300 keys behind the last, and round lengths up to a share of 2048, in an int.
constexpr long long kMostKeys = 0x7fffffffll - 4096;
struct AttendArgs {
    CacheArgs c;
    const void* q;
    size_t q_token, q_head;
    const int *starts, *lengths, *table;
    size_t table_pitch;
    int tokens, requests, group, width, type, causal;
    FastDiv by_group, by_heads;
    float scale;
    void* out;               // [tokens][heads * group][dim]
    float* lse;              // [tokens][heads * group], or null
    int rows, waves;         // of a block: attend_plan()
    int splits;              // blocks per row tile; blocks of 16 rows: the last one has what is left
    int share;               // keys of one, blocks of 16 rows (a multiple of 32)
    float *part_o, *part_ml; // [splits][tokens * heads * group][dim], [..][2]
    int wide_q;
};
void attend_plan(AttendArgs* a, int longest);       // rows, splits
hipError_t launch_attend_chunk(const AttendArgs& a, hipStream_t st);      // (blocks of 128 or 256 rows; does not join)
hipError_t launch_attend(const AttendArgs& a, hipStream_t st);

}  // namespace int8t
