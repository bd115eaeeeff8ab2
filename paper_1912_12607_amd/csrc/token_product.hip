// Products of 8-bit codes with a scale for each row of either operand:  y[m][n] = (float)(sum_k a[m][k] b[n][k]) * (sa[m] sb[n]) + bias[n].
#include "device_common.h"
#include "lds_dma.h"
#include "tokens.h"

namespace int8t {
namespace {

typedef int tp_v4i __attribute__((ext_vector_type(4)));
typedef int tp_v16i __attribute__((ext_vector_type(16)));

// Output tile of WM x WN waves, each MI x NJ products of 32 x 32; stages of 128 reduction bytes, two of them in LDS: while one is
// multiplied, the next is on its way (buffer loads into LDS, rows beyond the operand and bytes beyond the reduction read as zeros).
template <int TYPE, int WM, int WN, int MI, int NJ>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(const ProductArgs a, const int mtiles, const int ntiles) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int KG = 8, NW = WM * WN, BM = WM * MI * 32, BN = WN * NJ * 32, STAGE = (BM + BN) * KG;
    constexpr int NLA = BM * KG / 64 / NW, NLB = BN * KG / 64 / NW, NL = NLA + NLB;
    static_assert((NW & 1) == 0, "the swizzle below needs an even wave count");
    extern __shared__ __attribute__((aligned(1024))) uint4 ring[];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;

    // Workgroup b runs on XCD b % 8: an XCD takes a run of tiles, eight tiles of rows by one of columns at a time, so that the operands
    // that its tiles share meet in its L2.
    const int total = mtiles * ntiles, per = (total + 7) >> 3;
    const int tile = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);
    if (((int)blockIdx.x >> 3) >= per || tile >= total) return;
    const int group = tile / (8 * ntiles), first = group * 8, height = mtiles - first < 8 ? mtiles - first : 8;
    const int in = tile - group * 8 * ntiles;
    const int row0 = (first + in % height) * BM, col0 = (in / height) * BN;

    const int rows = a.M - row0 < BM ? a.M - row0 : BM, cols = a.N - col0 < BN ? a.N - col0 : BN;
    const lds_dma_v4i ra = igd_rsrc(a.a + (size_t)row0 * a.Kp, (uint32_t)rows * (uint32_t)a.Kp);
    const lds_dma_v4i rb = igd_rsrc(a.b + (size_t)col0 * a.Kp, (uint32_t)cols * (uint32_t)a.Kp);
    const uint32_t lds_a = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(size_t)(ring + 64 * wave));
    const uint32_t lds_b = lds_a + BM * KG * 16;
    // load i of this wave covers 8 tile rows from 8 (wave + NW i); the lane's granule is the inverse of igd_slot<8>()
    const int lrow = lane >> 3;
    const int gran = (lane & 7) ^ (((lrow >> 1) & 3) | ((wave & 1) << 2));
    const uint32_t voff = (uint32_t)(8 * wave + lrow) * (uint32_t)a.Kp + (uint32_t)gran * 16u;
    const uint32_t vstep = (uint32_t)(8 * NW) * (uint32_t)a.Kp;
    const int nsteps = (a.Kp + 127) >> 7;
    auto issue = [&](int buf, int step) {
        const uint32_t boff = (uint32_t)buf * (STAGE * 16u);
        const uint32_t past = step * 128 + gran * 16 < a.Kp ? 0u : IGD_OOB;      // beyond the reduction
        const uint32_t k = (uint32_t)__builtin_amdgcn_readfirstlane(step * 128);
#pragma unroll
        for (int i = 0; i < NLA; ++i) igd_load_lds(ra, lds_a + boff + (uint32_t)i * (NW * 1024), (voff + (uint32_t)i * vstep) | past, k);
#pragma unroll
        for (int i = 0; i < NLB; ++i) igd_load_lds(rb, lds_b + boff + (uint32_t)i * (NW * 1024), (voff + (uint32_t)i * vstep) | past, k);
    };

    tp_v16i acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;

    issue(0, 0);
    for (int step = 0; step < nsteps; ++step) {
        igd_wait_vmcnt<0>();
        __syncthreads();         // the stage is in LDS, and the one before it has been read by all
        if (step + 1 < nsteps) issue((step + 1) & 1, step + 1);
        const uint4* __restrict__ sA = ring + (step & 1) * STAGE;
        const uint4* __restrict__ sB = sA + BM * KG;
#pragma unroll
        for (int kk = 0; kk < KG / 2; ++kk) {
            const int g = kk * 2 + (lane >> 5);
            tp_v4i fa[MI], fb[NJ];
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const uint4 t = sA[igd_slot<KG>((wm * MI + i) * 32 + (lane & 31), g)];
                fa[i] = tp_v4i{(int)t.x, (int)t.y, (int)t.z, (int)t.w};
            }
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const uint4 t = sB[igd_slot<KG>((wn * NJ + j) * 32 + (lane & 31), g)];
                fb[j] = tp_v4i{(int)t.x, (int)t.y, (int)t.z, (int)t.w};
            }
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[i], fb[j], acc[i][j], 0, 0, 0);
        }
    }

    T* const y = static_cast<T*>(a.y);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int n = col0 + (wn * NJ + j) * 32 + (lane & 31);
        if (n >= a.N) continue;
        const float sb = a.sb ? a.sb[n] : 1.0f, bias = a.bias ? a.bias[n] : 0.0f;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int m = row0 + (wm * MI + i) * 32 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
                if (m < a.M) {
                    float r = __fmul_rn((float)acc[i][j][v], __fmul_rn(a.sa[m], sb));
                    if (a.bias) r = __fadd_rn(r, bias);
                    y[(size_t)m * a.pitch + n] = (T)r;
                }
            }
    }
}

template <int TYPE, int WM, int WN, int MI, int NJ>
hipError_t product_of(const ProductArgs& a, hipStream_t st) {
    constexpr int BM = WM * MI * 32, BN = WN * NJ * 32, LDS = 2 * (BM + BN) * 128;
    static std::atomic<unsigned long long> done{0};
    const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(&product_kernel<TYPE, WM, WN, MI, NJ>), LDS, done);
    if (e != hipSuccess) return e;
    const int mt = (a.M + BM - 1) / BM, nt = (a.N + BN - 1) / BN;
    KernelTimer kt(KID_TOKEN_PRODUCT, st);
    launch_timed(kt, (product_kernel<TYPE, WM, WN, MI, NJ>), dim3((unsigned)((((size_t)mt * nt + 7) / 8) * 8)), dim3(64 * WM * WN), LDS, st, a, mt, nt);
    return hipGetLastError();
}

template <int TYPE>
hipError_t product_type(const ProductArgs& a, hipStream_t st) {
    return product_of<TYPE, 2, 2, 2, 2>(a, st);
}

}  // namespace

size_t product_scratch(int M, int N, int Kp) {
    (void)M; (void)N; (void)Kp;
    return 0;
}
hipError_t launch_product(ProductArgs a, size_t scratch_bytes, hipStream_t st) {
    (void)scratch_bytes;
    if (a.type == kF32) return product_type<kF32>(a, st);
    if (a.type == kBF16) return product_type<kBF16>(a, st);
    return product_type<kF16>(a, st);
}

}  // namespace int8t
