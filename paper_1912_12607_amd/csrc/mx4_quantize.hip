// Microscaled 4-bit codes of matrices: blocks along the rows' values, or along the columns' with the codes transposed, or both from one pass.
#include <type_traits>

#include "mx4.h"

namespace int8t {
namespace {

// The word whose upper 24 bits are rng24()
__device__ __forceinline__ uint32_t draw32(uint32_t key_x, uint32_t key_a, uint32_t index) {
    uint32_t at;
    asm("v_xad_u32 %0, %1, %2, %3" : "=v"(at) : "v"(index), "v"(key_x), "s"(key_a));
    return rng_mix32(at);
}

// Four neighbouring lanes have a block, eight values each; their largest goes round by lane exchanges of a quad.  Rows are lanes in whole panels (256
// values), so that the scales behind the last block are written (zeros).  Bound by memory: 16384 x 4096 bf16 34 to 36 us, 170 MB at 4.7 to 5 TB/s, a large copy's rate.
template <int TYPE, bool STOCH>
__global__ __launch_bounds__(256) void mx_rows_kernel(const MxArgs a, const FastDiv by_row, const int groups, const int wide, const uint32_t kx, const uint32_t ka) {
    typedef typename ElemOf<TYPE>::type T;
    const int at = (int)(blockIdx.x * 256 + threadIdx.x);
    const int row = div_by(at, by_row), g = at - row * groups;          // (a row has a multiple of 32 lanes)
    const bool live = row < a.rows;
    const int c = g * 8;
    float v[8];
    load8<TYPE>(static_cast<const T*>(a.x) + (size_t)(live ? row : 0) * a.pitch + c, live ? a.cols - c : 0, wide, v);
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = most(m, fabsf(v[i]));
    m = most(m, dpp_of<kDppSwap1>(m));
    m = most(m, dpp_of<kDppSwap2>(m));
    if (!live) return;
    const uint32_t byte = mx_byte_of(m);
    const int block = g >> 2, blocks = mx_blocks(a.cols);
    if ((g & 3) == 0) a.s[((size_t)(block >> 3) * a.rows + row) * 8 + (block & 7)] = block < blocks ? (uint8_t)byte : (uint8_t)0;
    if (block >= blocks) return;
    uint32_t w = 0;
    if (STOCH) {
        const float inv = mx_inverse(byte), one = draws_begin();
        const uint32_t index = (uint32_t)row * (uint32_t)a.cols + (uint32_t)c;
#pragma unroll
        for (int i = 7; i >= 0; --i) w = mx_drawn(w, v[i], inv, one, draw32(kx, ka, index + (uint32_t)i));
        // (values behind the row are zero and stay zero: a draw alone does not reach a step)
    } else {
        w = mx_codes8(v, mx_scale(byte));
    }
    *reinterpret_cast<uint32_t*>(a.q + (size_t)row * (16 * blocks) + 4 * g) = byte < 255u ? w : 0u;
}

// Both directions from one pass: tiles of 256 rows by 128 bytes (64 columns, 32 of fp32), a lane has eight rows of 16 bytes, four lanes above each other a block of
// rows, four or eight side by side one of columns; the largest goes round by lane exchanges.  Codes along the rows' axis are turned in registers -- the eight rows
// of a lane's column are a word -- and go through LDS, so that a column's 256 rows leave as one line.  An XCD takes a run of tiles side by side: what two of them
// write of a line meets in its L2.
// To the nearest it is bound by memory (8192 x 4096 and 4096 x 4096 bf16, a layer's x and W, in one launch: 39 to 41 us, 3.9 TB/s);
// draws, two for each value, by vector arithmetic: 8192 x 4096 bf16 45 to 50 us (2.3 TB/s), instructions issued in 71 % of the cycles, of which 13 of a value's 20 are a draw's,
// two of them products of 32 bits at a quarter of the rate.  A pass for each direction took 155 us where one took 105 (these two launches, when draws took 60).
constexpr int QT_R = 256, QT_PITCH = QT_R / 2 + 16;
template <int TYPE, bool STOCH>
__device__ __forceinline__ void tile_body(const MxArgs& a, const int block, const int total, const int wide, const uint32_t kx, const uint32_t ka, const uint32_t tx, const uint32_t ta) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int C = 16 / (int)sizeof(T), TC = 8 * C;
    __shared__ __attribute__((aligned(16))) uint8_t turned[TC * QT_PITCH], turned_s[TC * 8];
    __shared__ float sums[4][TC];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = lane & 7, rg = tid >> 3;
    const int tiles_c = ((a.q ? mx_panels(a.cols) * 256 : a.cols) + TC - 1) / TC, per = (total + 7) >> 3, tile = (block & 7) * per + (block >> 3);
    if ((block >> 3) >= per || tile >= total) return;
    const int row0 = tile / tiles_c * QT_R, col0 = (tile - tile / tiles_c * tiles_c) * TC;
    const int row = row0 + 8 * rg, col = col0 + cg * C;
    // (a tile inside of the matrix needs no look at its ends)
    const auto tile_of = [&](auto inside) __attribute__((always_inline)) {
        constexpr bool IN = decltype(inside)::value;
        T v[8][C];
        const T* const x = static_cast<const T*>(a.x);
        const bool whole = IN || (wide && col + C <= a.cols);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const bool in = IN || row + r < a.rows;
            const T* const at = x + (size_t)(in ? row + r : 0) * a.pitch + col;
            if (whole) {
                typedef T V __attribute__((ext_vector_type(C)));
                const V t = *reinterpret_cast<const V*>(at);
#pragma unroll
                for (int j = 0; j < C; ++j) v[r][j] = in ? t[j] : (T)0.0f;
            } else {
#pragma unroll
                for (int j = 0; j < C; ++j) v[r][j] = in && col + j < a.cols ? at[j] : (T)0.0f;
            }
        }
        if (a.sum) {
#pragma unroll
            for (int j = 0; j < C; ++j) {
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < 8; ++r) sum += (float)v[r][j];
                sum += dpp_of<kDppRor8>(sum);
                const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
                sum = __uint_as_float(b[0]) + __uint_as_float(b[1]);
                const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
                sum = __uint_as_float(h[0]) + __uint_as_float(h[1]);
                if (lane < 8) sums[wave][cg * C + j] = sum;
            }
        }
        float one = 1.0f;
        if (STOCH) one = draws_begin();
        if (a.q) {
            const int block_c = col >> 5, blocks = mx_blocks(a.cols);
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                float m = 0.0f, f[8];
#pragma unroll
                for (int j = 0; j < C; ++j) {
                    f[j] = (float)v[r][j];
                    m = most(m, fabsf(f[j]));
                }
                m = most(m, dpp_of<kDppSwap1>(m));
                m = most(m, dpp_of<kDppSwap2>(m));
                if (C == 4) m = most(m, dpp_of<0x141>(m));             // (row_half_mirror: the quads of eight lanes)
                const uint32_t byte = mx_byte_of(m);
                uint32_t w = 0;
                if (STOCH) {
                    const float inv = mx_inverse(byte);
#pragma unroll
                    for (int j = C - 1; j >= 0; --j) w = mx_drawn(w, f[j], inv, one, draw32(kx, ka, (uint32_t)(row + r) * (uint32_t)a.cols + (uint32_t)(col + j)));
                } else {
#pragma unroll
                    for (int j = C; j < 8; ++j) f[j] = 0.0f;
                    w = mx_codes8(f, mx_scale(byte));
                }
                w = byte < 255u ? w : 0u;
                if (IN || (row + r < a.rows && block_c < blocks)) {
                    uint8_t* const q = a.q + (size_t)(row + r) * (16 * blocks) + col / 2;
                    if (C == 8) *reinterpret_cast<uint32_t*>(q) = w;
                    else *reinterpret_cast<uint16_t*>(q) = (uint16_t)w;
                    if ((col & 31) == 0) a.s[((size_t)(block_c >> 3) * a.rows + row + r) * 8 + (block_c & 7)] = (uint8_t)byte;
                }
                // (behind the last block, the rest of its panel)
                if (!IN && row + r < a.rows && block_c >= blocks && block_c < ((blocks + 7) & ~7) && (col & 31) == 0)
                    a.s[((size_t)(block_c >> 3) * a.rows + row + r) * 8 + (block_c & 7)] = 0;
            }
        }
        if (a.qt) {
#pragma unroll
            for (int j = 0; j < C; ++j) {
                float m = 0.0f, f[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    f[r] = (float)v[r][j];
                    m = most(m, fabsf(f[r]));
                }
                m = most(m, dpp_of<kDppRor8>(m));
                const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
                m = most(__uint_as_float(b[0]), __uint_as_float(b[1]));
                const uint32_t byte = mx_byte_of(m);
                uint32_t w = 0;
                if (STOCH) {
                    const float inv = mx_inverse(byte);
#pragma unroll
                    for (int r = 7; r >= 0; --r) w = mx_drawn(w, f[r], inv, one, draw32(tx, ta, (uint32_t)(row + r) * (uint32_t)a.cols + (uint32_t)(col + j)));
                } else {
                    w = mx_codes8(f, mx_scale(byte));
                }
                *reinterpret_cast<uint32_t*>(turned + (cg * C + j) * QT_PITCH + 4 * rg) = byte < 255u ? w : 0u;
                if ((rg & 3) == 0) turned_s[(cg * C + j) * 8 + (rg >> 2)] = (uint8_t)byte;
            }
        }
        if (STOCH) draws_end();
    };
    if (wide && row0 + QT_R <= a.rows && col0 + TC <= a.cols) tile_of(std::true_type());
    else tile_of(std::false_type());
    if (a.qt || a.sum) {
        __syncthreads();
        if (a.qt) {
            const int blocks = mx_blocks(a.rows), b0 = row0 >> 5;
#pragma unroll
            for (int u = 0; u < TC * 8 / 256; ++u) {
                const int c = (tid >> 3) + 32 * u, b = tid & 7;
                if (col0 + c < a.cols && b0 + b < blocks)
                    *reinterpret_cast<uint4*>(a.qt + ((size_t)(col0 + c) * blocks + b0 + b) * 16) = *reinterpret_cast<const uint4*>(turned + c * QT_PITCH + 16 * b);
            }
            // (a tile's rows are a panel; blocks behind the last have largest values of zero, and bytes of zero)
            if (tid < TC && col0 + tid < a.cols)
                *reinterpret_cast<uint2*>(a.st + ((size_t)(b0 >> 3) * a.cols + col0 + tid) * 8) = *reinterpret_cast<const uint2*>(turned_s + tid * 8);
        }
        if (a.sum && tid < TC && col0 + tid < a.cols) {
            const float s = (sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid]);
            if (a.rows <= QT_R) a.sum[col0 + tid] = s;
            else a.part[(size_t)(row0 / QT_R) * a.cols + col0 + tid] = s;
        }
    }
}
// Two matrices in one launch: blocks from `first` (a multiple of eight) on have the second's tiles.
template <int TYPE, bool STOCH>
__global__ __launch_bounds__(256) void mx_tiles_kernel(const MxArgs a, const MxArgs b, const int first, const int total_a, const int total_b, const int wide_a, const int wide_b,
                                                       const uint32_t kx, const uint32_t ka, const uint32_t tx, const uint32_t ta) {
    const bool second = (int)blockIdx.x >= first;
    const MxArgs m = second ? b : a;
    tile_body<TYPE, STOCH>(m, (int)blockIdx.x - (second ? first : 0), second ? total_b : total_a, second ? wide_b : wide_a, kx, ka, tx, ta);
}

// Sums of columns from those of the blocks of rows (where no product follows)
__global__ __launch_bounds__(256) void mx_sum_kernel(const MxArgs a, const int parts) {
    const int c = (int)(blockIdx.x * 256 + threadIdx.x);
    if (c >= a.cols) return;
    a.sum[c] = mx_join(a.part + c, parts, (size_t)a.cols);
}

inline int wide_rows(const MxArgs& a) { return (((uintptr_t)a.x | (a.pitch * (a.type == kF32 ? 4 : 2))) & 15) == 0; }
inline long long tiles_of(const MxArgs& a) {
    const int tc = a.type == kF32 ? 32 : 64, cols = a.q ? mx_panels(a.cols) * 256 : a.cols;      // (whole panels: the scales behind the last block are written)
    return (long long)((a.rows + QT_R - 1) / QT_R) * ((cols + tc - 1) / tc);
}

template <int TYPE, bool STOCH>
hipError_t quantize_of(const MxArgs& a, const MxArgs* b, hipStream_t st) {
    const uint64_t turned = a.seed ^ (1ull << 63);
    if (!a.qt && !a.sum && !b) {
        const int groups = mx_panels(a.cols) * 32;
        KernelTimer kt(KID_MX_QUANTIZE, st);
        launch_timed(kt, (mx_rows_kernel<TYPE, STOCH>), dim3((unsigned)(((long long)a.rows * groups + 255) / 256)), dim3(256), 0, st, a, fast_div((unsigned)groups), groups,
                     wide_rows(a), seed_key_x(a.seed), seed_key_a(a.seed));
        return hipGetLastError();
    }
    {
        const int ta = (int)tiles_of(a), tb = b ? (int)tiles_of(*b) : 0, first = (ta + 7) & ~7;
        KernelTimer kt(KID_MX_QUANTIZE, st);
        launch_timed(kt, (mx_tiles_kernel<TYPE, STOCH>), dim3((unsigned)(first + ((tb + 7) & ~7))), dim3(256), 0, st, a, b ? *b : a, first, ta, tb, wide_rows(a), b ? wide_rows(*b) : 0,
                     seed_key_x(a.seed), seed_key_a(a.seed), seed_key_x(turned), seed_key_a(turned));
    }
    if (a.sum && a.rows > QT_R && !a.parts_only) {
        KernelTimer kt(KID_MX_QUANTIZE, st);
        launch_timed(kt, mx_sum_kernel, dim3((unsigned)((a.cols + 255) / 256)), dim3(256), 0, st, a, mx_sum_parts(a.rows));
    }
    return hipGetLastError();
}
template <int TYPE>
hipError_t quantize_type(const MxArgs& a, const MxArgs* b, hipStream_t st) { return a.stochastic ? quantize_of<TYPE, true>(a, b, st) : quantize_of<TYPE, false>(a, b, st); }

}  // namespace

int mx_sum_parts(int rows) { return (rows + QT_R - 1) / QT_R; }
hipError_t launch_mx_quantize(const MxArgs& a, hipStream_t st, const MxArgs* b) {
    if (a.type == kF32) return quantize_type<kF32>(a, b, st);
    if (a.type == kBF16) return quantize_type<kBF16>(a, b, st);
    return quantize_type<kF16>(a, b, st);
}

}  // namespace int8t
