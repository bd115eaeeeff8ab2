// Microscaled 4-bit codes: blocks of 32 values share a power of two 2^e, codes stand for 0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives (two exponent bits,
// one of mantissa).  Shared by the quantisers, products and the cache.
#pragma once
#include "device_common.h"
#include "tokens.h"

namespace int8t {

// ---- sizes of the layouts (host and device) ---------------------------------------------------------------------------
__host__ __device__ constexpr int mx_blocks(int values) { return (int)(((long long)values + 31) >> 5); }
__host__ __device__ constexpr int mx_row_bytes(int values) { return mx_blocks(values) * 16; }
__host__ __device__ constexpr int mx_panels(int values) { return (mx_blocks(values) + 7) >> 3; }      // of eight blocks

// ---- codes ------------------------------------------------------------------------------------------------------------
// The byte of a block from its largest magnitude: e + 127 with e the least integer of [-127, 127] for which m <= 6 2^e.  6 = 1.5 * 2^2, so one more than the
// exponent of m less two where its mantissa is beyond 1.5: no value is clipped, the nearest code is off by half a step at most and a drawn one is unbiased.
// Infinities and NaN: 255.
__device__ __forceinline__ uint32_t mx_byte_of(float m) {
    const uint32_t bits = __float_as_uint(m);
    const int b = (int)((bits + 0x3fffffu) >> 23) - 2;
    return bits >= 0x7f800000u ? 255u : (uint32_t)max(b, 0);
}
// 2^(byte - 127); NaN of 255
__device__ __forceinline__ float mx_power(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23);
}
// The same of 0 .. 254, in two operations (254 itself is not a quantiser's)
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(max(byte << 23, 0x00400000u)); }
// Two values as codes in byte SEL of `into`, to the nearest (ties to even): x / scale, scale 2^e
template <int SEL>
__device__ __forceinline__ uint32_t mx_pair(uint32_t into, float x0, float x1, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(into, x0, x1, scale, SEL);
}
__device__ __forceinline__ uint32_t mx_codes8(const float v[8], float scale) {
    uint32_t w = mx_pair<0>(0u, v[0], v[1], scale);
    w = mx_pair<1>(w, v[2], v[3], scale);
    w = mx_pair<2>(w, v[4], v[5], scale);
    return mx_pair<3>(w, v[6], v[7], scale);
}
// What the eight codes of a word stand for, without their scale
__device__ __forceinline__ void mx_values8(uint32_t w, float v[8]) {
    typedef float V2 __attribute__((ext_vector_type(2)));
    const V2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
    const V2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
    v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
}
// Codes drawn: a magnitude counts 2^-22 of a step -- below 1 steps are .5, from there on a float's bits count them, two steps to each power of two --, the upper 22
// bits of a word drawn are added, and what is whole is the code.  |x| inv <= 6 exactly, inv 2^-e.  The bits of a + max(a, 1) are that count in either range, if the sum is
// rounded toward zero: draws_begin() switches the wave to that, and gives the 1 that keeps the sums behind it.
__device__ __forceinline__ float draws_begin() {
    float one = 1.0f;
    asm volatile("s_setreg_imm32_b32 hwreg(HW_REG_MODE, 0, 2), 3\n\ts_nop 3" : "+v"(one)::"memory");
    return one;
}
__device__ __forceinline__ void draws_end() { asm volatile("s_setreg_imm32_b32 hwreg(HW_REG_MODE, 0, 2), 0\n\ts_nop 3" ::: "memory"); }
// w shifted up by one code, and x's below: the count 64 times in a word, where the draw's lower bits reach nothing, and 127's bits by the 2 above the draw
__device__ __forceinline__ uint32_t mx_drawn(uint32_t w, float x, float inv, float one, uint32_t draw32) {
    const float a = __fmul_rn(fabsf(x), inv);
    const uint32_t count = (__float_as_uint(a + fmaxf(a, one)) << 6) + __builtin_amdgcn_alignbit(2u, draw32, 4);
    uint32_t top;
    asm("v_bfi_b32 %0, %1, %2, %3" : "=v"(top) : "s"(0x7fffffffu), "v"(count), "v"(x));      // (left to itself, the compiler masks both)
    return __builtin_amdgcn_alignbit(w, top, 28);
}
// 2^-e from 2^e's byte (0 .. 253)
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// ---- mx4_quantize.hip -------------------------------------------------------------------------------------------------
struct MxArgs {              // codes of rows x cols values
    const void* x;
    size_t pitch;            // elements between rows
    int type, rows, cols;
    int stochastic;
    uint64_t seed;           // of the rows' codes, columns' go by it with the highest bit flipped
    uint8_t *q, *s;          // blocks along the columns: [rows][mx_row_bytes(cols)], [mx_panels(cols)][rows][8]; or null
    uint8_t *qt, *st;        // blocks along the rows: [cols][mx_row_bytes(rows)], [mx_panels(rows)][cols][8]; or null
    float* sum;              // cols, or null: sums of the columns
    float* part;             // [parts][cols], with sum (one part: not used)
    bool parts_only = false; // parts are left for the product that follows (MxProductArgs)
};
int mx_sum_parts(int rows);
// with b (the same type and rounding to nearest in both): two matrices in one launch
hipError_t launch_mx_quantize(const MxArgs& a, hipStream_t st, const MxArgs* b = nullptr);

// ---- mx4_product.hip --------------------------------------------------------------------------------------------------
struct MxProductArgs {       // y[m][n] = sum_k a[m][k] b[n][k] + bias[n]
    const uint8_t *a, *b;    // [M][Kb], [N][Kb]: Kb bytes, two values each
    const uint8_t *sa, *sb;  // [panels][M][8], [panels][N][8]
    const float* bias;       // null: none
    int M, N, Kb;
    void* y;
    size_t pitch;
    int type;
    float* part;             // partial sums of a split reduction, or null
    int splits;
    const float* sum_part;   // [sum_parts][M] sums to join beside the product, in sum; or null
    float* sum;
    int sum_parts;
};
// Parts in their order, in 64 bits
__device__ __forceinline__ float mx_join(const float* part, int parts, size_t pitch) {
    double s = 0.0;
#pragma unroll 8
    for (int p = 0; p < parts; ++p) s += (double)part[(size_t)p * pitch];
    return (float)s;
}
struct MxFewArgs {           // the same from x itself, codes made on the way: mx_few_tokens(M, N, Kb)
    const void* x;
    size_t x_pitch;
    int type, M, K, Kb, N, wide;
    const uint8_t *wq, *sw;
    const float* bias;
    void* y;
    size_t y_pitch;
};
bool mx_few_tokens(int M, int N, int Kb);
hipError_t launch_mx_few_tokens(const MxFewArgs& a, hipStream_t st);
bool mx_product_fits(int M, int N, int Kb);
void mx_product_division(int M, int N, int Kb, size_t scratch_bytes, int* rows, int* waves, int* stages, int* shares);
size_t mx_product_scratch(int M, int N, int Kb);
hipError_t launch_mx_product(MxProductArgs a, size_t scratch_bytes, hipStream_t st);
hipError_t launch_mx_products(MxProductArgs a, MxProductArgs b, size_t scratch_bytes, hipStream_t st);

// ---- mx4_cache.hip ----------------------------------------------------------------------------------------------------
// Codes and scales of CacheArgs' pointers: kq, vq [pages][heads][page_size][mx_row_bytes(dim)], ks, vs bytes [pages][heads][page_size][mx_blocks(dim)].
hipError_t launch_mx_cache_write(const CacheMoveArgs& a, hipStream_t st);
hipError_t launch_mx_cache_read(const CacheMoveArgs& a, hipStream_t st);

}  // namespace int8t
