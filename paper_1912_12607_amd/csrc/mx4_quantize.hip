// Microscaled 4-bit codes of matrices: blocks along the rows' values, or along the columns' with the codes transposed, or both from one pass.
#include "mx4.h"

namespace int8t {
namespace {

// Four neighbouring lanes have a block, eight values each; their largest goes round by lane exchanges of a quad.  Rows are lanes in whole panels (256
// values), so that the scales behind the last block are written (zeros).
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
    if (byte < 255u) {
        if (STOCH) {
            const float inv = mx_inverse(byte);
            const uint32_t index = (uint32_t)row * (uint32_t)a.cols + (uint32_t)c;
#pragma unroll
            for (int i = 0; i < 8; ++i) w |= mx_drawn(v[i], inv, rng24(kx, ka, index + (uint32_t)i)) << (4 * i);
            // (values behind the row are zero and stay zero: a draw alone does not reach a step)
        } else {
            w = mx_codes8(v, mx_power(byte));
        }
    }
    *reinterpret_cast<uint32_t*>(a.q + (size_t)row * (16 * blocks) + 4 * g) = w;
}

// Blocks along the rows' axis: a lane has 16 bytes of 32 neighbouring rows in registers, RB blocks of rows and 64 / RB groups of columns a wave.
template <int TYPE, bool STOCH, int RB>
__global__ __launch_bounds__(256) void mx_cols_kernel(const MxArgs a, const int wide, const uint32_t kx, const uint32_t ka) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int C = 16 / (int)sizeof(T), CG = 64 / RB;               // columns of a lane, groups of a wave
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int col = (((int)blockIdx.x * 4 + wave) * CG + lane % CG) * C, block = (int)blockIdx.y * RB + lane / CG;
    const int blocks = mx_blocks(a.rows), row0 = block * 32;
    if (col >= a.cols) return;
    if (block >= blocks) {
        if (a.qt && block < (blocks + 7) / 8 * 8)
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (col + j < a.cols) a.st[((size_t)(block >> 3) * a.cols + col + j) * 8 + (block & 7)] = 0;
        return;
    }
    T v[32][C];
    const bool whole = wide && col + C <= a.cols;
    const T* const x = static_cast<const T*>(a.x) + (size_t)row0 * a.pitch + col;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const bool in = row0 + i < a.rows;
        if (whole) {
            typedef T V __attribute__((ext_vector_type(C)));
            V t = *reinterpret_cast<const V*>(x + (in ? (size_t)i * a.pitch : 0));
#pragma unroll
            for (int j = 0; j < C; ++j) v[i][j] = in ? t[j] : (T)0.0f;
        } else {
#pragma unroll
            for (int j = 0; j < C; ++j) v[i][j] = in && col + j < a.cols ? x[(size_t)i * a.pitch + j] : (T)0.0f;
        }
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
        if (col + j >= a.cols) break;
        float m = 0.0f, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            m = most(m, fabsf((float)v[i][j]));
            sum += (float)v[i][j];
        }
        if (a.sum) a.part[(size_t)block * a.cols + col + j] = sum;
        if (!a.qt) continue;
        const uint32_t byte = mx_byte_of(m);
        a.st[((size_t)(block >> 3) * a.cols + col + j) * 8 + (block & 7)] = (uint8_t)byte;
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        if (byte < 255u) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = (float)v[8 * u + i][j];
                if (STOCH) {
                    const float inv = mx_inverse(byte);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        w[u] |= mx_drawn(f[i], inv, rng24(kx, ka, (uint32_t)(row0 + 8 * u + i) * (uint32_t)a.cols + (uint32_t)(col + j))) << (4 * i);
                } else {
                    w[u] = mx_codes8(f, mx_power(byte));
                }
            }
        }
        *reinterpret_cast<uint4*>(a.qt + ((size_t)(col + j) * blocks + block) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Sums of columns from those of the blocks of rows
__global__ __launch_bounds__(256) void mx_sum_kernel(const MxArgs a, const int parts) {
    const int c = (int)(blockIdx.x * 256 + threadIdx.x);
    if (c >= a.cols) return;
    double s = 0.0;
#pragma unroll 8
    for (int p = 0; p < parts; ++p) s += (double)a.part[(size_t)p * a.cols + c];
    a.sum[c] = (float)s;
}

template <int TYPE, bool STOCH>
hipError_t quantize_of(const MxArgs& a, hipStream_t st) {
    const int wide = (((uintptr_t)a.x | (a.pitch * (TYPE == kF32 ? 4 : 2))) & 15) == 0;
    if (a.q) {
        const int groups = mx_panels(a.cols) * 32;
        KernelTimer kt(KID_MX_QUANTIZE, st);
        launch_timed(kt, (mx_rows_kernel<TYPE, STOCH>), dim3((unsigned)(((long long)a.rows * groups + 255) / 256)), dim3(256), 0, st, a, fast_div((unsigned)groups), groups, wide,
                     seed_key_x(a.seed), seed_key_a(a.seed));
    }
    if (a.qt || a.sum) {
        constexpr int C = TYPE == kF32 ? 4 : 8;
        const uint64_t seed = a.seed ^ (1ull << 63);
        const int blocks = mx_panels(a.rows) * 8;
        KernelTimer kt(KID_MX_QUANTIZE, st);
        launch_timed(kt, (mx_cols_kernel<TYPE, STOCH, 8>), dim3((unsigned)((a.cols + 32 * C - 1) / (32 * C)), (unsigned)(blocks / 8)), dim3(256), 0, st, a, wide, seed_key_x(seed),
                     seed_key_a(seed));
    }
    if (a.sum) {
        KernelTimer kt(KID_MX_QUANTIZE, st);
        launch_timed(kt, mx_sum_kernel, dim3((unsigned)((a.cols + 255) / 256)), dim3(256), 0, st, a, mx_sum_parts(a.rows));
    }
    return hipGetLastError();
}
template <int TYPE>
hipError_t quantize_type(const MxArgs& a, hipStream_t st) { return a.stochastic ? quantize_of<TYPE, true>(a, st) : quantize_of<TYPE, false>(a, st); }

}  // namespace

int mx_sum_parts(int rows) { return mx_blocks(rows); }
hipError_t launch_mx_quantize(const MxArgs& a, hipStream_t st) {
    if (a.type == kF32) return quantize_type<kF32>(a, st);
    if (a.type == kBF16) return quantize_type<kBF16>(a, st);
    return quantize_type<kF16>(a, st);
}

}  // namespace int8t
