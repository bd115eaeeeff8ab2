// Products of microscaled 4-bit codes:  y[m][n] = sum_k (a[m][k] 2^ea) (b[n][k] 2^eb) + bias[n], sums in fp32.
#include <type_traits>

#include "lds_dma.h"
#include "mx4.h"

namespace int8t {
namespace {

typedef int mp_v4i __attribute__((ext_vector_type(4)));
typedef int mp_v8i __attribute__((ext_vector_type(8)));
constexpr int kMxFewBytes = 24576;       // codes of few tokens, see mx_few_tokens()

// 32 x 32 sums of 64 products each: a lane has a block of a row (16 bytes), the lanes of the wave's other half another one; byte S of `sa`, `sb` is its scale.
template <int S>
__device__ __forceinline__ tk_f16 product32(const mp_v4i& a, const mp_v4i& b, const tk_f16& c, uint32_t sa, uint32_t sb) {
    const mp_v8i wa = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, wb = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wa, wb, c, 4, 4, S, (int)sa, S, (int)sb);
}
__device__ __forceinline__ tk_f16 product32_at(int s, const mp_v4i& a, const mp_v4i& b, const tk_f16& c, uint32_t sa, uint32_t sb) {
    return s == 0 ? product32<0>(a, b, c, sa, sb) : s == 1 ? product32<1>(a, b, c, sa, sb) : s == 2 ? product32<2>(a, b, c, sa, sb) : product32<3>(a, b, c, sa, sb);
}
// 16 x 16 sums of 128 products: a quarter of the wave's lanes has a block each
template <int S>
__device__ __forceinline__ tk_f4 product16(const uint4& a, const uint4& b, const tk_f4& c, uint32_t sa, uint32_t sb) {
    const mp_v8i wa = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, wb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, c, 4, 4, S, (int)sa, S, (int)sb);
}
// One wave-wide 4-byte-per-lane buffer load into LDS: lane l's word lands at lds_base + 4 l (see igd_load_lds()).
__device__ __forceinline__ void load_words_lds(const lds_dma_v4i& rsrc, uint32_t lds_base_uniform, uint32_t voff, uint32_t soff) {
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(lds_base_uniform), "v"(voff), "s"(rsrc), "s"(soff) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// Output tile of WM x WN waves, each MI x NJ products of 32 x 32; stages of 256 values (128 bytes of a row, whole lines, and a panel of eight scales), NS of them
// in LDS: while one is multiplied, the next ones are on their way (buffer loads into LDS, rows beyond the operand and bytes beyond the reduction read as zeros).
// A lane's blocks of a stage are four neighbours (4 half + kk for product kk), so that one word has their scales.
// SPLIT: the block has a share of the reduction and leaves its sums for mx_reduce_kernel.
// Bound by the matrix units and their power: tiles of 256 (four products of a wave for every eight blocks read from LDS) 16384 x 4096 -> 4096 136 to 148 us, 3.7 to 4.0 PFLOP/s, 8192 x 8192 ->
// 8192 270 us (4.05); the units are busy in 52 % of the cycles, at 1.7 GHz, and products of registers alone, busy all the time, reach 6.36 PFLOP/s at 1.5 GHz.  Blocks that
// went on to a next tile, its loads under way while the results leave, were slower (160 us); LDS reads that conflict take 5 % of the time.
template <int TYPE, int WM, int WN, int MI, int NJ, int NS, bool SPLIT>
__device__ __forceinline__ void product_body(const MxProductArgs& a, const int mtiles, const int ntiles, const int block) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int KG = 8, NW = WM * WN, BM = WM * MI * 32, BN = WN * NJ * 32, CODES = (BM + BN) * KG, STAGE = CODES + (BM + BN) / 2;      // (in pieces of 16 bytes)
    constexpr int NLA = BM * KG / 64 / NW, NLB = BN * KG / 64 / NW, NL = NLA + NLB;
    constexpr int SD = (BM + BN) * 8 / 256 / NW;           // loads of scales, 32 rows each: the first half of the waves a's, the others b's
    static_assert((NW & 1) == 0 && BM == BN && SD * 256 * NW == (BM + BN) * 8, "the swizzle below needs an even wave count, the scales' loads as many rows as columns");
    extern __shared__ __attribute__((aligned(1024))) uint4 ring[];
    __shared__ __attribute__((aligned(16))) float cbias[BN];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;

    // Workgroup b runs on XCD b % 8: an XCD takes a run of tiles, four tiles of rows by one of columns at a time, so that the operands that its tiles share
    // meet in its L2.  SPLIT: the shares of a tile's reduction are tiles of their own.
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
    const int all_steps = (a.Kb + KG * 16 - 1) / (KG * 16);
    const lds_dma_v4i ra = igd_rsrc(a.a + (size_t)row0 * a.Kb, (uint32_t)rows * (uint32_t)a.Kb);
    const lds_dma_v4i rb = igd_rsrc(a.b + (size_t)col0 * a.Kb, (uint32_t)cols * (uint32_t)a.Kb);
    const bool scales_a = wave < NW / 2;
    const int lines = scales_a ? a.M : a.N, line0 = scales_a ? row0 : col0;
    const lds_dma_v4i rs = igd_rsrc((scales_a ? a.sa : a.sb) + (size_t)line0 * 8, (uint32_t)(((size_t)all_steps * lines - line0) * 8));
    const uint32_t lds_a = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(size_t)(ring + 64 * wave));
    const uint32_t lds_b = lds_a + BM * KG * 16;
    const uint32_t lds_s = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(size_t)(ring + CODES + SD * 16 * wave));
    const int sline = (wave % (NW / 2)) * (SD * 32) + (lane >> 1);
    const uint32_t sv = (uint32_t)(sline * 8 + (lane & 1) * 4);
    // load i of this wave covers RL tile rows from RL (wave + NW i); the lane's granule is the inverse of igd_slot<KG>()
    constexpr int RL = 64 / KG;
    const int lrow = lane / KG;
    const int gran = (lane & 7) ^ (((lrow >> 1) & 3) | ((wave & 1) << 2));
    const uint32_t voff = (uint32_t)(RL * wave + lrow) * (uint32_t)a.Kb + (uint32_t)gran * 16u;
    const uint32_t vstep = (uint32_t)(RL * NW) * (uint32_t)a.Kb;
    const int first_step = SPLIT ? (int)((long long)all_steps * share / a.splits) : 0, nsteps = SPLIT ? (int)((long long)all_steps * (share + 1) / a.splits) - first_step : all_steps;
    // The u-th of this wave's NL loads of codes of a stage, scales with the first ones.  Stages behind the last are loaded too, as zeros: no branch stands between the
    // products, which the compiler would move behind it, operands and all (registers spilled, 16384 x 4096 -> 4096 1080 us).
    auto load = [&](int buf, int step, int u) __attribute__((always_inline)) {
        const uint32_t boff = (uint32_t)buf * (STAGE * 16u);
        const int at = (first_step + step) * (KG * 16);
        const uint32_t end = step < nsteps ? 0u : IGD_OOB;
        const uint32_t past = at + gran * 16 < a.Kb ? end : IGD_OOB;      // beyond the reduction
        const uint32_t k = (uint32_t)__builtin_amdgcn_readfirstlane(at);
        if (u < SD) {
            const uint32_t behind = line0 + sline + u * 32 < lines ? end : IGD_OOB;
            load_words_lds(rs, lds_s + boff + (uint32_t)u * 256u, (sv + (uint32_t)u * 256u) | behind, (uint32_t)__builtin_amdgcn_readfirstlane((first_step + step) * lines * 8));
        }
        if (u < NLA) igd_load_lds(ra, lds_a + boff + (uint32_t)u * (NW * 1024), (voff + (uint32_t)u * vstep) | past, k);
        else igd_load_lds(rb, lds_b + boff + (uint32_t)(u - NLA) * (NW * 1024), (voff + (uint32_t)(u - NLA) * vstep) | past, k);
    };

    for (int c = (int)threadIdx.x; c < BN; c += 64 * NW) cbias[c] = c < cols && a.bias ? a.bias[col0 + c] : 0.0f;
    tk_f16 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

    // Operands of 64 values are read while the 64 before them are multiplied, across the stages too: before a stage's last products every wave has all of the
    // stage's operands in registers, so behind the barrier that stands there the next stage can be read and this one's place filled again.
    mp_v4i fa[2][MI], fb[2][NJ];
    uint32_t ea[NS][MI], eb[NS][NJ];
    const int half = lane >> 5, l32 = lane & 31;
    const auto read = [&](const auto slot, int kk) __attribute__((always_inline)) {
        constexpr int BUF = decltype(slot)::value;
        const uint4* __restrict__ sA = ring + BUF * STAGE;
        const uint4* __restrict__ sB = sA + BM * KG;
        const uint32_t* __restrict__ sS = reinterpret_cast<const uint32_t*>(sA + CODES);
        const int g = 4 * half + kk;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int r = (wm * MI + i) * 32 + l32;
            const uint4 t = sA[igd_slot<KG>(r, g)];
            fa[kk & 1][i] = mp_v4i{(int)t.x, (int)t.y, (int)t.z, (int)t.w};
            if (kk == 0) ea[BUF][i] = sS[2 * r + half];
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int c = (wn * NJ + j) * 32 + l32;
            const uint4 t = sB[igd_slot<KG>(c, g)];
            fb[kk & 1][j] = mp_v4i{(int)t.x, (int)t.y, (int)t.z, (int)t.w};
            if (kk == 0) eb[BUF][j] = sS[2 * (BM + c) + half];
        }
    };
    // (the loads of the NS - 2 stages behind the next one are still under way)
    const auto turn = []() __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wait_loads<(NS - 2) * (NL + SD)>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // The loads of a stage are dealt out between the products from the barrier on that frees their place, NQ products to a load, so that they
    // are under way at least a step before they are waited for.
    constexpr int NP = MI * NJ, NQ = NP * (NS > 2 ? KG / 2 : KG / 2 - 1) / NL > 0 ? NP * (NS > 2 ? KG / 2 : KG / 2 - 1) / NL : 1;
    static_assert((NL - 1) * NQ < NP * (KG / 2), "all loads of a stage are issued before the next barrier");
#pragma unroll
    for (int p = 0; p < NS - 1; ++p)
#pragma unroll
        for (int u = 0; u < NL; ++u)
            load(p, p, u);
    turn();
#pragma unroll
    for (int u = 0; u < NL; ++u)
        if (u * NQ < NP) load(NS - 1, NS - 1, u);
    read(std::integral_constant<int, 0>(), 0);
    const auto stage = [&](const auto slot, int step) __attribute__((always_inline)) {
        constexpr int BUF = decltype(slot)::value;
#pragma unroll
        for (int kk = 0; kk < KG / 2; ++kk) {
            // from the last group on the loads of NS stages ahead go into this stage's place; they go on through the next stage's other groups
            const bool last = kk + 1 == KG / 2;
            if (!last) {
                read(slot, kk + 1);
            } else {
                turn();
                read(std::integral_constant<int, (BUF + 1) % NS>(), 0);
            }
            const int into = last ? BUF : (BUF + NS - 1) % NS, which = last ? step + NS : step + NS - 1;
            const int done = last ? 0 : (kk + 1) * NP;                      // products since the barrier
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < NP; ++q) {
                const int i = q / NJ, j = q % NJ;
                if ((done + q) % NQ == 0 && (done + q) / NQ < NL) load(into, which, (done + q) / NQ);
                acc[i][j] = product32_at(kk, fb[kk & 1][j], fa[kk & 1][i], acc[i][j], eb[BUF][j], ea[BUF][i]);
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

    wait_loads<0>();                 // (of the zeros behind the last stage)
    if constexpr (SPLIT) {
        // [share][row][column], columns padded to four
        const int np = (a.N + 3) & ~3;
        float* const part = a.part + (size_t)share * a.M * np;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m = row0 + (wm * MI + i) * 32 + l32;
            if (m >= a.M) continue;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = col0 + (wn * NJ + j) * 32 + 8 * q + 4 * half;
                    if (n < a.N) *reinterpret_cast<float4*>(part + (size_t)m * np + n) = make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
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
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = j * 32 + 8 * q + 4 * half;
                typedef T V4 __attribute__((ext_vector_type(4)));
                V4 o;
#pragma unroll
                for (int u = 0; u < 4; ++u) o[u] = (T)__fadd_rn(acc[i][j][4 * q + u], cbias[wn * CW + c + u]);
                *reinterpret_cast<V4*>(stg + l32 * RP + c * ES) = o;
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
__global__ __launch_bounds__(64 * WM * WN) void mx_product_kernel(const MxProductArgs a, const MxProductArgs b, const int first) {
    constexpr int BM = WM * MI * 32, BN = WN * NJ * 32;
    const bool second = (int)blockIdx.x >= first;
    const MxProductArgs p = second ? b : a;
    const int block = (int)blockIdx.x - (second ? first : 0);
    product_body<TYPE, WM, WN, MI, NJ, NS, SPLIT>(p, (p.M + BM - 1) / BM, (p.N + BN - 1) / BN, block);
    // (a launch of 4 us less; the first blocks have as many lanes as the product has rows)
    static_assert(64 * WM * WN >= BM, "a lane for each row");
    const long long m = (long long)block * (64 * WM * WN) + (int)threadIdx.x;
    if (p.sum && m < p.M) p.sum[m] = mx_join(p.sum_part + m, p.sum_parts, (size_t)p.M);
}

// ------------------------------------------------------------------------------------------------
// Few tokens (at most 16) through weights that are laid out: one launch, codes of the tokens included.  Every block makes them for itself in LDS -- the tokens are
// small and come from the caches -- and multiplies them with 16 channels at a time: a wave has an eighth of the reduction's panels, loads two blocks of 16 weight
// rows per lane straight into the products' operands (16 x 16 x 128), and the eight sums meet in LDS.  The first channels' weights are on their way while the
// codes are made.  1 x 4096 -> 4096 bf16 4.0 to 4.2 us, weights and scales of 8.9 MB at 2.1 TB/s: the launch, the first loads and the sums that follow each other are most of
// it; 16 channels are 256 blocks here, one for each compute unit.
// ------------------------------------------------------------------------------------------------
constexpr int XW = 8;            // waves
constexpr int XL = 4;            // panels of a lane's weights in flight
__host__ __device__ constexpr int few_pitch(int Kb) { return ((Kb + 127) & ~127) + 16; }       // rows of codes 16 bytes apart modulo the banks
__host__ __device__ constexpr int few_lds(int M, int Kb) { return M * few_pitch(Kb) + M * ((Kb + 127) / 128 * 8); }
template <int TYPE>
__global__ __launch_bounds__(64 * XW, 4) void mx_few_kernel(const MxFewArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    extern __shared__ __attribute__((aligned(1024))) uint8_t codes[];      // [M][few_pitch], scales [M][8 panels]
    __shared__ __attribute__((aligned(16))) float sums[XW][4][64];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, kg = lane >> 4;
    const int pitch = few_pitch(a.Kb), panels = (a.Kb + 127) >> 7, spitch = panels * 8;
    uint8_t* const scales = codes + a.M * pitch;
    // this wave's part of the reduction: whole panels
    const int p_from = panels * wave / XW, p_to = panels * (wave + 1) / XW;
    const int tiles = (a.N + 15) >> 4;

    uint4 w[XL][2];
    uint32_t sw[XL];
    auto fetch = [&](int tile, int p0) __attribute__((always_inline)) {
        const int n = min(tile * 16 + n16, a.N - 1);
        const uint8_t* const row = a.wq + (size_t)n * a.Kb;
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            sw[i] = 0u;
            if (p0 + i < p_to) sw[i] = *reinterpret_cast<const uint16_t*>(a.sw + ((size_t)(p0 + i) * a.N + n) * 8 + 2 * kg);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = (p0 + i) * 128 + kg * 32 + h * 16;
                w[i][h] = make_uint4(0u, 0u, 0u, 0u);
                if (p0 + i < p_to && k < a.Kb) w[i][h] = *reinterpret_cast<const uint4*>(row + k);
            }
        }
    };
    int tile = (int)blockIdx.x;
    fetch(tile, p_from);

    // the tokens' codes: four neighbouring lanes a block, in whole panels
    {
        const T* const x = static_cast<const T*>(a.x);
        const int groups = panels * 32, all = a.M * groups;
        for (int t = tid; t < all; t += 64 * XW) {          // (groups, and with it each step's end, are multiples of four lanes)
            const int m = t / groups, g = t - m * groups;
            float v[8];
            load8<TYPE>(x + (size_t)m * a.x_pitch + 8 * g, a.K - 8 * g, a.wide, v);
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = most(top, fabsf(v[i]));
            top = most(top, dpp_of<kDppSwap1>(top));
            top = most(top, dpp_of<kDppSwap2>(top));
            const uint32_t byte = mx_byte_of(top);
            *reinterpret_cast<uint32_t*>(codes + m * pitch + 4 * g) = byte < 255u ? mx_codes8(v, mx_power(byte)) : 0u;
            if ((g & 3) == 0) scales[m * spitch + (g >> 2)] = (uint8_t)byte;
        }
    }
    __syncthreads();

    // (columns of tokens that there are not: not stored)
    const uint8_t* const mine = codes + (n16 < a.M ? n16 : 0) * pitch + kg * 32;
    const uint8_t* const mine_s = scales + (n16 < a.M ? n16 : 0) * spitch + 2 * kg;
    for (;;) {
        tk_f4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int p0 = p_from; p0 < p_to; p0 += XL) {
            if (p0 > p_from) fetch(tile, p0);
#pragma unroll
            for (int i = 0; i < XL; ++i) {
                if (p0 + i >= p_to) break;
                const int p = p0 + i;
                const uint32_t sx = *reinterpret_cast<const uint16_t*>(mine_s + p * 8);
                const uint4 t0 = *reinterpret_cast<const uint4*>(mine + p * 128), t1 = *reinterpret_cast<const uint4*>(mine + p * 128 + 16);
                acc = product16<0>(w[i][0], t0, acc, sw[i], sx);
                acc = product16<1>(w[i][1], t1, acc, sw[i], sx);
            }
        }
        const int next = tile + (int)gridDim.x;
        if (next < tiles) fetch(next, p_from);
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][r][lane] = acc[r];
        __syncthreads();
        if (tid < 256) {
            // channel 4 (lane / 16) + r of token lane % 16: neighbouring threads take neighbouring channels
            const int n = tile * 16 + (tid & 15), m = tid >> 4, at = ((tid & 15) >> 2) * 16 + m, r = tid & 3;
            float s = sums[0][r][at];
#pragma unroll
            for (int i = 1; i < XW; ++i) s += sums[i][r][at];
            if (n < a.N && m < a.M) {
                if (a.bias) s = __fadd_rn(s, a.bias[n]);
                static_cast<T*>(a.y)[(size_t)m * a.y_pitch + n] = (T)s;
            }
        }
        if (next >= tiles) break;
        tile = next;
        __syncthreads();
    }
}

// Sums of the shares, bias: four neighbouring results a lane (17 x 8192 -> 512 bf16: products of four shares and this 8.6 us, one share
// 9.3)
template <int TYPE>
__global__ __launch_bounds__(256) void mx_reduce_kernel(const MxProductArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    const int np = (a.N + 3) & ~3, quads = np >> 2;
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (size_t)a.M * quads) return;
    const int m = (int)(at / quads), n = (int)(at - (size_t)m * quads) * 4;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < a.splits; ++p) {
        const float4 t = *reinterpret_cast<const float4*>(a.part + ((size_t)p * a.M + m) * np + n);
        v[0] += t.x;
        v[1] += t.y;
        v[2] += t.z;
        v[3] += t.w;
    }
    T* const y = static_cast<T*>(a.y) + (size_t)m * a.pitch;
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (n + u < a.N) y[n + u] = (T)(a.bias ? __fadd_rn(v[u], a.bias[n + u]) : v[u]);
}

template <int TYPE, int WM, int WN, int MI, int NJ, int NS, bool SPLIT>
hipError_t product_split(const MxProductArgs& a, const MxProductArgs* b, hipStream_t st) {
    constexpr int BM = WM * MI * 32, BN = WN * NJ * 32, LDS = NS * (BM + BN) * (128 + 8);
    static std::atomic<unsigned long long> done{0};
    const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(&mx_product_kernel<TYPE, WM, WN, MI, NJ, NS, SPLIT>), LDS, done);
    if (e != hipSuccess) return e;
    const auto blocks = [](const MxProductArgs& p) {
        return (unsigned)((((size_t)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN) * (SPLIT ? p.splits : 1) + 7) / 8) * 8);
    };
    const unsigned first = blocks(a);
    {
        KernelTimer kt(KID_MX_PRODUCT, st);
        launch_timed(kt, (mx_product_kernel<TYPE, WM, WN, MI, NJ, NS, SPLIT>), dim3(first + (b ? blocks(*b) : 0u)), dim3(64 * WM * WN), LDS, st, a, b ? *b : a, (int)first);
    }
    if (SPLIT) {
        KernelTimer kt(KID_MX_REDUCE, st);
        launch_timed(kt, mx_reduce_kernel<TYPE>, dim3((unsigned)(((size_t)a.M * ((a.N + 3) / 4) + 255) / 256)), dim3(256), 0, st, a);
    }
    return hipGetLastError();
}
template <int TYPE, int WM, int WN, int MI, int NJ, int NS>
hipError_t product_of(const MxProductArgs& a, const MxProductArgs* b, hipStream_t st) {
    return a.splits > 1 ? product_split<TYPE, WM, WN, MI, NJ, NS, true>(a, nullptr, st) : product_split<TYPE, WM, WN, MI, NJ, NS, false>(a, b, st);
}

// Tiles and shares of the reduction by an estimate, us: rounds of blocks times stages of 256 values, plus what a block and the joining pass cost.  occ: blocks on
// a compute unit; a stage, and a block's start and end, take longer the fuller the chip is (first: one block alone, then all places taken).  (Measured, one share, bf16 results,
// tiles of 256, 128 with two and three stages in LDS, 64: 8192 x 4096 -> 4096 73, 86, 97, 127; 1001 x 4096 -> 16384 38, 46, 51, 65; 1001 x 4096 -> 4096 25, 14.6, 13.9, 19;
// 512 x 8192 -> 4096 45, 26, 20, 18; 128 x 8192 -> 4096 41, 18, 17, 9; shares hardly ever pay: 17 x 8192 -> 512 with four 8.6, with one 9.3.  Over 76 sizes from 17 x 256 -> 512
// to 8192 x 8192 -> 4096 the choice takes 1.2 % longer than the fastest.)
struct ProductPlan {
    int tile, splits;          // 0: 256 x 256, 1: 128 x 128, 2: the same with three stages, 3: 64 x 64 with four
};
ProductPlan find_plan(int M, int N, int Kb, bool scratch) {
    static const struct { int bm, occ; double stage, full_stage, fixed, full_fixed; } kTiles[4] = {
        {256, 1, 1.17, 1.76, 4.0, 9.5}, {128, 2, 0.41, 1.04, 4.0, 6.2}, {128, 1, 0.40, 0.57, 3.8, 4.5}, {64, 2, 0.20, 0.42, 2.5, 2.9}};
    const int steps = (Kb + 127) >> 7;
    ProductPlan best{0, 1};
    double least = 1e30;
    for (int t = 0; t < 4; ++t) {
        const long long tiles = (long long)((M + kTiles[t].bm - 1) / kTiles[t].bm) * ((N + kTiles[t].bm - 1) / kTiles[t].bm);
        for (int s = 1; s <= (scratch ? 16 : 1) && s <= steps; s *= 2) {
            const long long blocks = tiles * s, slots = 256ll * kTiles[t].occ;
            if (s > 1 && (tiles * s > 1024 || (size_t)M * N * s > (1u << 26))) break;
            const double load = blocks < slots ? (double)blocks / (double)slots : 1.0;
            const double stage = kTiles[t].stage + (kTiles[t].full_stage - kTiles[t].stage) * load, fixed = kTiles[t].fixed + (kTiles[t].full_fixed - kTiles[t].fixed) * load;
            double us = (double)((blocks + slots - 1) / slots) * ((steps + s - 1) / s * stage + fixed);
            if (s > 1) us += 4.5 + 0.1 * s + 3.6e-6 * (double)s * M * N;
            if (us < least) {
                least = us;
                best = ProductPlan{t, s};
            }
        }
    }
    return best;
}
// (a call asks for its plan several times: the last ones are kept, by sizes alone)
ProductPlan product_plan(int M, int N, int Kb, bool scratch) {
    struct Kept { int M, N, Kb, scratch; ProductPlan plan; };
    static thread_local Kept kept[64];
    Kept& k = kept[((unsigned)M * 0x9E3779B1u ^ (unsigned)N * 0x85EBCA77u ^ (unsigned)Kb * 0xC2B2AE3Du ^ (scratch ? 0x27D4EB2Fu : 0u)) >> 26];
    if (k.M != M || k.N != N || k.Kb != Kb || k.scratch != (int)scratch) k = Kept{M, N, Kb, (int)scratch, find_plan(M, N, Kb, scratch)};
    return k.plan;
}

template <int TYPE>
hipError_t product_type(const MxProductArgs& a, const MxProductArgs* b, int tile, hipStream_t st) {
    return tile == 0 ? product_of<TYPE, 2, 4, 4, 2, 2>(a, b, st) : tile == 1 ? product_of<TYPE, 2, 2, 2, 2, 2>(a, b, st)
           : tile == 2 ? product_of<TYPE, 2, 2, 2, 2, 3>(a, b, st) : product_of<TYPE, 2, 2, 1, 1, 4>(a, b, st);
}
hipError_t product_launch(const MxProductArgs& a, const MxProductArgs* b, int tile, hipStream_t st) {
    if (a.type == kF32) return product_type<kF32>(a, b, tile, st);
    if (a.type == kBF16) return product_type<kBF16>(a, b, tile, st);
    return product_type<kF16>(a, b, tile, st);
}
// the plan of a product, with shares only where their scratch is there
int planned(MxProductArgs* a, size_t scratch_bytes) {
    const size_t need = mx_product_scratch(a->M, a->N, a->Kb);
    const ProductPlan p = product_plan(a->M, a->N, a->Kb, need > 0 && a->part && scratch_bytes >= need);
    a->splits = p.splits;
    return p.tile;
}

template <int TYPE>
hipError_t few_of(const MxFewArgs& a, hipStream_t st) {
    static_assert(kMxFewBytes + 16 * (127 + 16) + (kMxFewBytes + 16 * 127) / 16 + 8 * 1024 <= 64 * 1024, "the codes fit what a launch may ask for");
    const int tiles = (a.N + 15) / 16;
    KernelTimer kt(KID_MX_FEW, st);
    launch_timed(kt, mx_few_kernel<TYPE>, dim3(tiles < 512 ? tiles : 512), dim3(64 * XW), (size_t)few_lds(a.M, a.Kb), st, a);
    return hipGetLastError();
}

}  // namespace

// Up to so many codes every block makes them for itself: a launch less, 4 us of the host's time or of a graph's, against 0.17 us for each 1024 bytes of codes, twice that where
// compute units have two blocks of 16 channels (bf16, us of one launch / two, by the host and in a graph: 16 x 2048 -> 1000 7.9/12 and 5.8/6.5, 8 x 4096 -> 4096 7.3/11.4 and
// 6.3/7.8, 16 x 4096 -> 4096 9.6/11.4 and 9.5/7.8, 8 x 4096 -> 16384 12.4/11.3 and 12.4/8.8, 16 x 4096 -> 16384 18/11.3 and 18/8.8, 8 x 8192 -> 8192 16.5/11.5 and 16.4/11.5).
bool mx_few_tokens(int M, int N, int Kb) { return M <= 16 && M * (long long)Kb * (N > 16 * 256 ? 2 : 1) <= kMxFewBytes; }
hipError_t launch_mx_few_tokens(const MxFewArgs& a, hipStream_t st) {
    if (a.type == kF32) return few_of<kF32>(a, st);
    if (a.type == kBF16) return few_of<kBF16>(a, st);
    return few_of<kF16>(a, st);
}

constexpr int kTileRows[4] = {256, 128, 128, 64}, kTileWaves[4] = {8, 4, 4, 4}, kTileStages[4] = {2, 2, 3, 4};
bool mx_product_fits(int M, int N, int Kb) {
    if (((unsigned long long)M + 63) / 64 * (((unsigned long long)N + 63) / 64) < (1u << 18)) return true;      // (with 16 shares and 512 lanes a block)
    for (const bool scratch : {false, true}) {
        const ProductPlan p = product_plan(M, N, Kb, scratch);
        const int rows = kTileRows[p.tile];
        const unsigned long long blocks = ((unsigned long long)M + rows - 1) / rows * (((unsigned long long)N + rows - 1) / rows) * p.splits;
        if ((blocks + 8) * 64 * kTileWaves[p.tile] >= 1ull << 32) return false;
    }
    return true;
}
void mx_product_division(int M, int N, int Kb, size_t scratch_bytes, int* rows, int* waves, int* stages, int* shares) {
    MxProductArgs a{};
    float there = 0;
    a.M = M; a.N = N; a.Kb = Kb; a.part = scratch_bytes ? &there : nullptr;
    const int tile = planned(&a, scratch_bytes);
    *rows = kTileRows[tile];
    *waves = kTileWaves[tile];
    *stages = kTileStages[tile];
    *shares = a.splits;
}
size_t mx_product_scratch(int M, int N, int Kb) {
    const ProductPlan p = product_plan(M, N, Kb, true);
    return p.splits > 1 ? (size_t)p.splits * M * ((N + 3) & ~3) * sizeof(float) : 0;
}
hipError_t launch_mx_product(MxProductArgs a, size_t scratch_bytes, hipStream_t st) {
    const int tile = planned(&a, scratch_bytes);
    return product_launch(a, nullptr, tile, st);
}
hipError_t launch_mx_products(MxProductArgs a, MxProductArgs b, size_t scratch_bytes, hipStream_t st) {
    const int ta = planned(&a, scratch_bytes), tb = planned(&b, scratch_bytes);
    if (ta == tb && a.type == b.type && a.splits == 1 && b.splits == 1) return product_launch(a, &b, ta, st);
    const hipError_t e = product_launch(a, nullptr, ta, st);
    return e != hipSuccess ? e : product_launch(b, nullptr, tb, st);
}

}  // namespace int8t
