// Products of 8-bit codes with a scale for each row of either operand:  y[m][n] = (float)(sum_k a[m][k] b[n][k]) * (sa[m] sb[n]) + bias[n].
#include <type_traits>

#include "device_common.h"
#include "lds_dma.h"
#include "tokens.h"

namespace int8t {
namespace {

typedef int tp_v4i __attribute__((ext_vector_type(4)));
typedef int tp_v16i __attribute__((ext_vector_type(16)));
constexpr int kFewCodes = 32768;         // of few tokens, see few_tokens()

// Output tile of WM x WN waves, each MI x NJ products of 32 x 32; stages of 128 reduction bytes (whole lines; half as many: 7 % slower), NS of them in LDS: while one is
// multiplied, the next ones are on their way (buffer loads into LDS, rows beyond the operand and bytes beyond the reduction read as zeros).
// Bound by the matrix units and the power that they draw: 16384 x 4096 -> 4096 in 250 us (2.20 POP/s; a large library product reaches 2.16 here, products of
// registers alone 3.4 with random codes), 8192 x 4096 -> 4096 in 124, 1001 x 4096 -> 16384 in 64 (2.1); below about 500 tokens by the depth of the reduction,
// 0.26 us for each 128 bytes of it.
// SPLIT: the block has a share of the reduction and leaves its sums for product_reduce_kernel.
template <int TYPE, int WM, int WN, int MI, int NJ, int NS, bool SPLIT>
__device__ __forceinline__ void product_body(const ProductArgs& a, const int mtiles, const int ntiles, const int block) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int KG = 8, NW = WM * WN, BM = WM * MI * 32, BN = WN * NJ * 32, STAGE = (BM + BN) * KG;
    constexpr int NLA = BM * KG / 64 / NW, NLB = BN * KG / 64 / NW, NL = NLA + NLB;
    static_assert((NW & 1) == 0, "the swizzle below needs an even wave count");
    extern __shared__ __attribute__((aligned(1024))) uint4 ring[];
    __shared__ __attribute__((aligned(16))) float cscale[2 * BN];       // scales and biases of the tile's columns
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;

    // Workgroup b runs on XCD b % 8: an XCD takes a run of tiles, four tiles of rows by one of columns at a time, so that the operands
    // that its tiles share meet in its L2 (eight by one: 16384 tokens 4096 -> 4096 294 us instead of 285).  SPLIT: the shares of a tile's reduction
    // are tiles of their own.
    const int total = mtiles * ntiles * (SPLIT ? a.splits : 1), per = (total + 7) >> 3;
    int tile = (block & 7) * per + (block >> 3), share = 0;
    if ((block >> 3) >= per || tile >= total) return;
    if (SPLIT) {
        share = tile / (mtiles * ntiles);
        tile -= share * (mtiles * ntiles);
    }
    const int group = tile / (4 * ntiles), first = group * 4, height = mtiles - first < 4 ? mtiles - first : 4;
    const int in = tile - group * 4 * ntiles;
    const int row0 = (first + in % height) * BM, col0 = (in / height) * BN;

    const int rows = a.M - row0 < BM ? a.M - row0 : BM, cols = a.N - col0 < BN ? a.N - col0 : BN;
    const lds_dma_v4i ra = igd_rsrc(a.a + (size_t)row0 * a.Kp, (uint32_t)rows * (uint32_t)a.Kp);
    const lds_dma_v4i rb = igd_rsrc(a.b + (size_t)col0 * a.Kp, (uint32_t)cols * (uint32_t)a.Kp);
    const uint32_t lds_a = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(size_t)(ring + 64 * wave));
    const uint32_t lds_b = lds_a + BM * KG * 16;
    // load i of this wave covers RL tile rows from RL (wave + NW i); the lane's granule is the inverse of igd_slot<KG>()
    constexpr int RL = 64 / KG;
    const int lrow = lane / KG;
    const int gran = (lane & 7) ^ (((lrow >> 1) & 3) | ((wave & 1) << 2));
    const uint32_t voff = (uint32_t)(RL * wave + lrow) * (uint32_t)a.Kp + (uint32_t)gran * 16u;
    const uint32_t vstep = (uint32_t)(RL * NW) * (uint32_t)a.Kp;
    const int all_steps = (a.Kp + KG * 16 - 1) / (KG * 16);
    const int first_step = SPLIT ? all_steps * share / a.splits : 0, nsteps = SPLIT ? all_steps * (share + 1) / a.splits - first_step : all_steps;
    auto load = [&](int buf, int step, int u) __attribute__((always_inline)) {      // the u-th of this wave's NL loads of a stage
        const uint32_t boff = (uint32_t)buf * (STAGE * 16u);
        const int at = (first_step + step) * (KG * 16);
        const uint32_t past = at + gran * 16 < a.Kp ? 0u : IGD_OOB;      // beyond the reduction
        const uint32_t k = (uint32_t)__builtin_amdgcn_readfirstlane(at);
        if (u < NLA) igd_load_lds(ra, lds_a + boff + (uint32_t)u * (NW * 1024), (voff + (uint32_t)u * vstep) | past, k);
        else igd_load_lds(rb, lds_b + boff + (uint32_t)(u - NLA) * (NW * 1024), (voff + (uint32_t)(u - NLA) * vstep) | past, k);
    };

    for (int c = (int)threadIdx.x; c < BN; c += 64 * NW) {
        const bool in = c < cols;
        cscale[c] = in && a.sb ? a.sb[col0 + c] : 1.0f;
        cscale[BN + c] = in && a.bias ? a.bias[col0 + c] : 0.0f;
    }
    tp_v16i acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;

    // Operands of 32 reduction bytes are read while the 32 before them are multiplied, across the stages too: before a stage's last
    // products every wave has all of the stage's operands in registers, so behind the barrier that stands there the next stage can be
    // read and this one's place filled again.
    tp_v4i fa[2][MI], fb[2][NJ];
    const auto read = [&](int buf, int kk) __attribute__((always_inline)) {
        const uint4* __restrict__ sA = ring + buf * STAGE;
        const uint4* __restrict__ sB = sA + BM * KG;
        const int g = kk * 2 + (lane >> 5);
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const uint4 t = sA[igd_slot<KG>((wm * MI + i) * 32 + (lane & 31), g)];
            fa[kk & 1][i] = tp_v4i{(int)t.x, (int)t.y, (int)t.z, (int)t.w};
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const uint4 t = sB[igd_slot<KG>((wn * NJ + j) * 32 + (lane & 31), g)];
            fb[kk & 1][j] = tp_v4i{(int)t.x, (int)t.y, (int)t.z, (int)t.w};
        }
    };
    // (more: the loads of the NS - 2 stages behind the next one are still under way)
    const auto turn = [&](bool more) __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (NS > 2 && more) igd_wait_vmcnt<NS == 2 ? 0 : (NS - 2) * NL>();
        else igd_wait_vmcnt<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // The loads of a stage are dealt out between the products from the barrier on that frees their place, NQ products to a load, so that they
    // are under way at least a step before they are waited for: all at once they keep the waves from their products until the last has been taken.
    constexpr int NP = MI * NJ, NQ = NP * (NS > 2 ? KG / 2 : KG / 2 - 1) / NL > 0 ? NP * (NS > 2 ? KG / 2 : KG / 2 - 1) / NL : 1;
    static_assert((NL - 1) * NQ < NP * (KG / 2), "all loads of a stage are issued before the next barrier");
#pragma unroll
    for (int p = 0; p < NS - 1; ++p)
#pragma unroll
        for (int u = 0; u < NL; ++u)
            if (p < nsteps) load(p, p, u);
    turn(nsteps >= NS);
#pragma unroll
    for (int u = 0; u < NL; ++u)
        if (u * NQ < NP && NS - 1 < nsteps) load(NS - 1, NS - 1, u);
    read(0, 0);
    const auto stage = [&](const auto slot, int step) __attribute__((always_inline)) {
        constexpr int BUF = decltype(slot)::value;
#pragma unroll
        for (int kk = 0; kk < KG / 2; ++kk) {
            // from the last group on the loads of NS stages ahead go into this stage's place; they go on through the next stage's other groups
            const bool last = kk + 1 == KG / 2;
            if (!last) {
                read(BUF, kk + 1);
            } else if (step + 1 < nsteps) {
                turn(step + NS - 1 < nsteps);
                read((BUF + 1) % NS, 0);
            }
            const int into = last ? BUF : (BUF + NS - 1) % NS, which = last ? step + NS : step + NS - 1;
            const int done = last ? 0 : (kk + 1) * NP;                      // products since the barrier
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < NP; ++q) {
                const int i = q / NJ, j = q % NJ;
                if ((done + q) % NQ == 0 && (done + q) / NQ < NL && which < nsteps) load(into, which, (done + q) / NQ);
                acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[kk & 1][j], fa[kk & 1][i], acc[i][j], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int step = 0; step < nsteps; step += NS) {
        stage(std::integral_constant<int, 0>(), step);
        if (step + 1 < nsteps) stage(std::integral_constant<int, 1>(), step + 1);
        if constexpr (NS > 2) {
            if (step + 2 < nsteps) stage(std::integral_constant<int, 2 % NS>(), step + 2);
        }
        if constexpr (NS > 3) {
            if (step + 3 < nsteps) stage(std::integral_constant<int, 3 % NS>(), step + 3);
        }
    }

    if constexpr (SPLIT) {
        // [share][row][column], columns padded to four
        const int np = (a.N + 3) & ~3;
        int32_t* const part = a.part + (size_t)share * a.M * np;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m = row0 + (wm * MI + i) * 32 + (lane & 31);
            if (m >= a.M) continue;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = col0 + (wn * NJ + j) * 32 + 8 * q + 4 * (lane >> 5);
                    if (n < a.N) *reinterpret_cast<int4*>(part + (size_t)m * np + n) = make_int4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
                }
        }
        return;
    }

    // Results: a lane has four neighbouring columns of a row at a time (the products' rows are b's).  They go through LDS, 32 rows of the
    // wave at a time in a place of its own, and leave in pieces of 16 bytes, whole cache lines of a row together.
    __syncthreads();                 // the ring has been read by all
    constexpr int CW = NJ * 32, ES = (int)sizeof(T), RP = CW * ES + 16, VE = 16 / ES, LPR = CW / VE, RPI = 64 / LPR;
    static_assert(NW * 32 * RP <= NS * STAGE * 16, "the staged rows fit the ring");
    unsigned char* const stg = reinterpret_cast<unsigned char*>(ring) + wave * 32 * RP;
    const int n0 = col0 + wn * CW;
    const bool wide = ((uintptr_t)a.y & 15) == 0 && (a.pitch * ES & 15) == 0;
    T* const y = static_cast<T*>(a.y);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int m0 = row0 + (wm * MI + i) * 32;
        const int m = m0 + (lane & 31);
        const float sa = a.sa[m < a.M ? m : a.M - 1];
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = j * 32 + 8 * q + 4 * (lane >> 5);
                typedef T V4 __attribute__((ext_vector_type(4)));
                V4 o;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float sb = cscale[wn * CW + c + u];
                    float r = __fmul_rn((float)acc[i][j][4 * q + u], __fmul_rn(sa, sb));
                    if (a.bias) r = __fadd_rn(r, cscale[BN + wn * CW + c + u]);
                    o[u] = (T)r;
                }
                *reinterpret_cast<V4*>(stg + (lane & 31) * RP + c * ES) = o;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (the wave's own place: no other wave reads or writes it)
        const int pc = lane % LPR * VE, pr = lane / LPR;
#pragma unroll
        for (int p = 0; p < 32 / RPI; ++p) {
            const int r = m0 + p * RPI + pr, n = n0 + pc;
            typedef T VE_ __attribute__((ext_vector_type(VE)));
            const VE_ t = *reinterpret_cast<const VE_*>(stg + (p * RPI + pr) * RP + pc * ES);
            if (r >= a.M) continue;
            T* const to = y + (size_t)r * a.pitch + n;
            if (wide && n + VE <= a.N) {
                *reinterpret_cast<VE_*>(to) = t;
            } else {
#pragma unroll
                for (int u = 0; u < VE; ++u)
                    if (n + u < a.N) to[u] = t[u];
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// One product, or two whose blocks from `first` (a multiple of eight) on have the second one's tiles.
template <int TYPE, int WM, int WN, int MI, int NJ, int NS, bool SPLIT>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(const ProductArgs a, const ProductArgs b, const int first) {
    constexpr int BM = WM * MI * 32, BN = WN * NJ * 32;
    const bool second = (int)blockIdx.x >= first;
    const ProductArgs p = second ? b : a;
    product_body<TYPE, WM, WN, MI, NJ, NS, SPLIT>(p, (p.M + BM - 1) / BM, (p.N + BN - 1) / BN, (int)blockIdx.x - (second ? first : 0));
}

// ------------------------------------------------------------------------------------------------
// Few tokens (at most 16) through weights that are laid out: one launch, codes of the tokens included.  Every block makes them for itself
// in LDS -- the tokens are small and come from the caches -- and multiplies them with 16 channels at a time: a wave has an eighth of the
// reduction, loads its 16 bytes of 16 weight rows per lane straight into the products' operand (16 x 16 x 64), and the eight sums meet in
// LDS.  The first channels' weights are on their way while the codes are made.  Bound by reading the weights once, behind the codes: 1 token through
// 4096 x 4096 5.9 us (16.8 MB; 3.3 at a copy's rate), 9 through 1000 x 2048 7 (latency: values, maxima, codes, products one after the other).
// ------------------------------------------------------------------------------------------------
constexpr int FW = 8;            // waves
constexpr int FL = 8;            // weight loads of a lane in flight: 512 reduction bytes of a wave
__host__ __device__ constexpr int few_pitch(int Kp) { return ((Kp + 255) & ~255) + 16; }       // rows of codes 16 bytes apart modulo the banks
// Codes: WPR waves have a token, or ROWS of them (the second eight after the first), whose values stay in registers while their maximum is found where
// they are at most 512 WPR CH (beyond, they are read again).  One token by all eight waves, up to four by two each, others by a wave each, with no wait for
// one another.
template <int TYPE, int WPR, int ROWS, int CH>
__global__ __launch_bounds__(64 * FW, 4) void few_tokens_kernel(const FewArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    extern __shared__ __attribute__((aligned(1024))) int8_t codes[];      // [M][few_pitch]
    __shared__ float part[FW], scales[16];
    __shared__ __attribute__((aligned(16))) int sums[FW][4][64];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, kg = lane >> 4;
    const int pitch = few_pitch(a.Kp);
    // this wave's part of the reduction: whole 64s
    const int chunks = (a.Kp + 63) >> 6, c_from = chunks * wave / FW, c_to = chunks * (wave + 1) / FW;
    const int tiles = (a.N + 15) >> 4;

    uint4 w[FL];
    auto fetch = [&](int tile, int c0) __attribute__((always_inline)) {
        const int n = tile * 16 + n16;
        const int8_t* const row = a.wq + (size_t)(n < a.N ? n : a.N - 1) * a.Kp;
#pragma unroll
        for (int i = 0; i < FL; ++i) {
            const int k = (c0 + i) * 64 + kg * 16;
            w[i] = make_uint4(0u, 0u, 0u, 0u);
            if (c0 + i < c_to && k < a.Kp) w[i] = *reinterpret_cast<const uint4*>(row + k);
        }
    };
    int tile = (int)blockIdx.x;
    fetch(tile, c_from);

    // maxima, scales, codes of the tokens
    {
        constexpr int SPAN = 512 * WPR * CH;
        const T* const x = static_cast<const T*>(a.x);
        const int m0 = wave / WPR, t8 = (tid - m0 * 64 * WPR) * 8;
        float v[ROWS][CH][8], top[ROWS];
        const auto values = [&](int base) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const int m = m0 + FW / WPR * r;
#pragma unroll
                for (int u = 0; u < CH; ++u) {
                    const int c = base + u * 512 * WPR + t8;
                    load8<TYPE>(x + (size_t)(m < a.M ? m : 0) * a.x_pitch + c, m < a.M ? a.K - c : 0, a.wide, v[r][u]);
                }
            }
        };
#pragma unroll
        for (int r = 0; r < ROWS; ++r) top[r] = 0.0f;
        for (int base = 0; base < a.K; base += SPAN) {
            values(base);
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int u = 0; u < CH; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) top[r] = most(top[r], fabsf(v[r][u][i]));
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) top[r] = wave_maximum(top[r]);
        if (WPR > 1) {
            if (lane == 0) part[wave] = top[0];
            __syncthreads();
            top[0] = part[m0 * WPR];
#pragma unroll
            for (int i = 1; i < WPR; ++i) top[0] = most(top[0], part[m0 * WPR + i]);
        }
        for (int base = 0; base < a.Kp; base += SPAN) {
            if (a.K > SPAN) values(base);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const int m = m0 + FW / WPR * r;
                const float inv = inv_scale_of(top[r]);
                if (m >= a.M) continue;
                if (t8 == 0 && base == 0) scales[m] = token_scale_of(top[r]);
#pragma unroll
                for (int u = 0; u < CH; ++u) {
                    const int c = base + u * 512 * WPR + t8;
                    int q[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) q[i] = quantize_one<false>(v[r][u][i], inv, 0u, 0u, 0u);
                    if (c < a.Kp) *reinterpret_cast<uint2*>(codes + m * pitch + c) = make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7]));
                }
            }
        }
    }
    __syncthreads();

    const int8_t* const mine = codes + (n16 < a.M ? n16 : 0) * pitch + kg * 16;      // (columns of tokens that there are not: not stored)
    for (;;) {
        tp_v4i acc = {0, 0, 0, 0};
        for (int c0 = c_from; c0 < c_to; c0 += FL) {
            if (c0 > c_from) fetch(tile, c0);
#pragma unroll
            for (int i = 0; i < FL; ++i) {
                // (beyond the wave's part, and beyond the row, the weights are zero: any codes will do there)
                const int k = c0 + i < c_to ? (c0 + i) * 64 : 0;
                const uint4 t = *reinterpret_cast<const uint4*>(mine + k);
                acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(tp_v4i{(int)w[i].x, (int)w[i].y, (int)w[i].z, (int)w[i].w}, tp_v4i{(int)t.x, (int)t.y, (int)t.z, (int)t.w}, acc, 0, 0, 0);
            }
        }
        const int next = tile + (int)gridDim.x;
        if (next < tiles) fetch(next, c_from);
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][r][lane] = acc[r];
        __syncthreads();
        if (tid < 256) {
            // channel 4 (lane / 16) + r of token lane % 16: neighbouring threads take neighbouring channels
            const int n = tile * 16 + (tid & 15), m = tid >> 4, at = ((tid & 15) >> 2) * 16 + m, r = tid & 3;
            int s = 0;
#pragma unroll
            for (int i = 0; i < FW; ++i) s += sums[i][r][at];
            if (n < a.N && m < a.M) {
                float v = __fmul_rn((float)s, __fmul_rn(scales[m], a.sw[n]));
                if (a.bias) v = __fadd_rn(v, a.bias[n]);
                static_cast<T*>(a.y)[(size_t)m * a.y_pitch + n] = (T)v;
            }
        }
        if (next >= tiles) break;
        tile = next;
        __syncthreads();
    }
}

// Sums of the shares, scales, bias: four neighbouring results a lane
template <int TYPE>
__global__ __launch_bounds__(256) void product_reduce_kernel(const ProductArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    const int np = (a.N + 3) & ~3, quads = np >> 2;
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (size_t)a.M * quads) return;
    const int m = (int)(at / quads), n = (int)(at - (size_t)m * quads) * 4;
    int4 s = make_int4(0, 0, 0, 0);
    for (int p = 0; p < a.splits; ++p) {
        const int4 t = *reinterpret_cast<const int4*>(a.part + ((size_t)p * a.M + m) * np + n);
        s.x += t.x;
        s.y += t.y;
        s.z += t.z;
        s.w += t.w;
    }
    const int v[4] = {s.x, s.y, s.z, s.w};
    const float sa = a.sa[m];
    T* const y = static_cast<T*>(a.y) + (size_t)m * a.pitch;
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (n + u < a.N) {
            float r = __fmul_rn((float)v[u], __fmul_rn(sa, a.sb ? a.sb[n + u] : 1.0f));
            if (a.bias) r = __fadd_rn(r, a.bias[n + u]);
            y[n + u] = (T)r;
        }
}

template <int TYPE, int WM, int WN, int MI, int NJ, int NS, bool SPLIT>
hipError_t product_split(const ProductArgs& a, const ProductArgs* b, hipStream_t st) {
    constexpr int BM = WM * MI * 32, BN = WN * NJ * 32, LDS = NS * (BM + BN) * 128;
    static std::atomic<unsigned long long> done{0};
    const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(&product_kernel<TYPE, WM, WN, MI, NJ, NS, SPLIT>), LDS, done);
    if (e != hipSuccess) return e;
    const auto blocks = [](const ProductArgs& p) {
        return (unsigned)((((size_t)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN) * (SPLIT ? p.splits : 1) + 7) / 8) * 8);
    };
    const unsigned first = blocks(a);
    {
        KernelTimer kt(KID_TOKEN_PRODUCT, st);
        launch_timed(kt, (product_kernel<TYPE, WM, WN, MI, NJ, NS, SPLIT>), dim3(first + (b ? blocks(*b) : 0u)), dim3(64 * WM * WN), LDS, st, a, b ? *b : a, (int)first);
    }
    if (SPLIT) {
        KernelTimer kt(KID_TOKEN_REDUCE, st);
        launch_timed(kt, product_reduce_kernel<TYPE>, dim3((unsigned)(((size_t)a.M * ((a.N + 3) / 4) + 255) / 256)), dim3(256), 0, st, a);
    }
    return hipGetLastError();
}
template <int TYPE, int WM, int WN, int MI, int NJ, int NS>
hipError_t product_of(const ProductArgs& a, const ProductArgs* b, hipStream_t st) {
    return a.splits > 1 ? product_split<TYPE, WM, WN, MI, NJ, NS, true>(a, nullptr, st) : product_split<TYPE, WM, WN, MI, NJ, NS, false>(a, b, st);
}

// Tiles and shares of the reduction by an estimate, us: rounds of blocks times stages of 128 reduction bytes, plus what a block and the
// joining pass cost.  occ: blocks on a compute unit; busy: of its matrix units per stage; least: a stage of a block alone.  (Measured, one share,
// bf16 results, tiles of 256, 128 with two and three stages in LDS, 64: 16384 x 4096 -> 4096 250, 320, 369, -; 1001 x 4096 -> 16384 64, 83, 95, 113;
// 1001 x 4096 -> 4096 48, 31, 25, 29; 512 x 4096 -> 4096 -, 28, 22, 17; 128 x 4096 -> 4096 -, 23, 21, 10.)
struct ProductPlan {
    int tile, splits;          // 0: 256 x 256, 1: 128 x 128, 2: the same with three stages, 3: 64 x 64 with four
};
ProductPlan product_plan(int M, int N, int Kp, bool scratch) {
    static const struct { int bm, occ; double busy, least, fixed; } kTiles[4] = {{256, 1, 1.63, 1.63, 10.0}, {128, 2, 0.57, 0.85, 4.0}, {128, 1, 0.66, 0.66, 4.5}, {64, 4, 0.22, 0.26, 2.5}};
    const int steps = (Kp + 127) >> 7;
    ProductPlan best{0, 1};
    double least = 1e30;
    for (int t = 0; t < 4; ++t) {
        const long long tiles = (long long)((M + kTiles[t].bm - 1) / kTiles[t].bm) * ((N + kTiles[t].bm - 1) / kTiles[t].bm);
        for (int s = 1; s <= (scratch ? 16 : 1) && s <= steps; s *= 2) {
            const long long blocks = tiles * s, slots = 256ll * kTiles[t].occ;
            if (s > 1 && (tiles * s > 1024 || (size_t)M * N * s > (1u << 26))) break;
            const double together = blocks >= slots ? kTiles[t].occ : (double)((blocks + 255) / 256);
            const double stage = together * kTiles[t].busy > kTiles[t].least ? together * kTiles[t].busy : kTiles[t].least;
            double us = (double)((blocks + slots - 1) / slots) * ((steps + s - 1) / s * stage + kTiles[t].fixed);
            if (s > 1) us += 3.5 + 8e-6 * (double)s * M * N / 4;
            if (us < least) {
                least = us;
                best = ProductPlan{t, s};
            }
        }
    }
    return best;
}

template <int TYPE>
hipError_t product_type(const ProductArgs& a, const ProductArgs* b, int tile, hipStream_t st) {
    return tile == 0 ? product_of<TYPE, 2, 4, 4, 2, 2>(a, b, st) : tile == 1 ? product_of<TYPE, 2, 2, 2, 2, 2>(a, b, st)
           : tile == 2 ? product_of<TYPE, 2, 2, 2, 2, 3>(a, b, st) : product_of<TYPE, 2, 2, 1, 1, 4>(a, b, st);
}
hipError_t product_launch(const ProductArgs& a, const ProductArgs* b, int tile, hipStream_t st) {
    if (a.type == kF32) return product_type<kF32>(a, b, tile, st);
    if (a.type == kBF16) return product_type<kBF16>(a, b, tile, st);
    return product_type<kF16>(a, b, tile, st);
}
// the plan of a product, with shares only where their scratch is there
int planned(ProductArgs* a, size_t scratch_bytes) {
    const size_t need = product_scratch(a->M, a->N, a->Kp);
    const ProductPlan p = product_plan(a->M, a->N, a->Kp, need > 0 && a->part && scratch_bytes >= need);
    a->splits = p.splits;
    return p.tile;
}

template <int TYPE, int WPR, int ROWS, int CH>
hipError_t few_of(const FewArgs& a, hipStream_t st) {
    static_assert(kFewCodes + 16 * (255 + 16) + 12 * 1024 <= 64 * 1024, "the codes fit what a launch may ask for");
    const int tiles = (a.N + 15) / 16;
    KernelTimer kt(KID_TOKEN_FEW, st);
    launch_timed(kt, (few_tokens_kernel<TYPE, WPR, ROWS, CH>), dim3(tiles < 512 ? tiles : 512), dim3(64 * FW), (size_t)a.M * few_pitch(a.Kp), st, a);
    return hipGetLastError();
}

}  // namespace

// Up to so many codes it is cheaper that every block makes them for itself than a launch more (us, one launch / two: 8 x 4096 -> 4096 10.6/14.6,
// 4 x 8192 -> 1000 14.0/15.6, 16 x 2048 -> 4096 9.3/11.3; 16 x 4096 -> 1000 13.3/14.2, -> 4096 16.8/13.8, -> 16384 31/19, 8 x 8192 -> 8192 30/22).
bool few_tokens(int M, int Kp) { return M <= 16 && M * (long long)Kp <= kFewCodes; }
hipError_t launch_few_tokens(const FewArgs& a, hipStream_t st) {
#define LAUNCH(TY) return a.M == 1 ? few_of<TY, FW, 1, 2>(a, st) : a.M <= FW / 2 ? few_of<TY, 2, 1, 4>(a, st) : a.M <= FW ? few_of<TY, 1, 1, 8>(a, st) : few_of<TY, 1, 2, 4>(a, st)
    if (a.type == kF32) LAUNCH(kF32);
    if (a.type == kBF16) LAUNCH(kBF16);
    LAUNCH(kF16);
#undef LAUNCH
}

constexpr int kTileRows[4] = {256, 128, 128, 64}, kTileWaves[4] = {8, 4, 4, 4}, kTileStages[4] = {2, 2, 3, 4};
bool product_fits(int M, int N, int Kp) {
    for (const bool scratch : {false, true}) {
        const ProductPlan p = product_plan(M, N, Kp, scratch);
        const int rows = kTileRows[p.tile];
        const unsigned long long blocks = ((unsigned long long)M + rows - 1) / rows * (((unsigned long long)N + rows - 1) / rows) * p.splits;
        if ((blocks + 8) * 64 * kTileWaves[p.tile] >= 1ull << 32) return false;
    }
    return true;
}
void product_division(int M, int N, int Kp, size_t scratch_bytes, int* rows, int* waves, int* stages, int* shares) {
    ProductArgs a{};
    int32_t there = 0;
    a.M = M; a.N = N; a.Kp = Kp; a.part = scratch_bytes ? &there : nullptr;
    const int tile = planned(&a, scratch_bytes);
    *rows = kTileRows[tile];
    *waves = kTileWaves[tile];
    *stages = kTileStages[tile];
    *shares = a.splits;
}
size_t product_scratch(int M, int N, int Kp) {
    const ProductPlan p = product_plan(M, N, Kp, true);
    return p.splits > 1 ? (size_t)p.splits * M * ((N + 3) & ~3) * sizeof(int32_t) : 0;
}
hipError_t launch_product(ProductArgs a, size_t scratch_bytes, hipStream_t st) {
    const int tile = planned(&a, scratch_bytes);
    return product_launch(a, nullptr, tile, st);
}
hipError_t launch_products(ProductArgs a, ProductArgs b, size_t scratch_bytes, hipStream_t st) {
    const int ta = planned(&a, scratch_bytes), tb = planned(&b, scratch_bytes);
    if (ta == tb && a.type == b.type && a.splits == 1 && b.splits == 1) return product_launch(a, &b, ta, st);
    const hipError_t e = product_launch(a, nullptr, ta, st);
    return e != hipSuccess ? e : product_launch(b, nullptr, tb, st);
}

}  // namespace int8t
