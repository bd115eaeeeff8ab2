// Attention of new tokens over a paged cache of microscaled 4-bit codes (the formulas of token_attend.hip, keys and values 2^e times their codes): blocks of 16
// rows.  Larger ones are token_attend_chunk.hip's.
#include "mx4.h"
#include "token_attend.h"

namespace int8t {
namespace {

typedef __bf16 ma_b2 __attribute__((ext_vector_type(2)));
typedef __bf16 ma_b8 __attribute__((ext_vector_type(8)));

// Two codes of byte SEL of a word times 2^e, as bf16: exact (two bits of mantissa)
template <int SEL>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) { return __builtin_bit_cast(uint32_t, ma_b2{(__bf16)a, (__bf16)b}); }
// x in pieces of bf16, each the nearest to what the ones before leave: 8 bits of x each
template <int PARTS>
__device__ __forceinline__ void bf16_pieces(const float x[8], ma_b8 out[PARTS]) {
    uint32_t w[PARTS][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            w[p][i] = bf16_pair(a, b);
            a -= __uint_as_float(w[p][i] << 16);
            b -= __uint_as_float(w[p][i] & 0xffff0000u);
        }
    }
#pragma unroll
    for (int p = 0; p < PARTS; ++p) out[p] = __builtin_bit_cast(ma_b8, make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]));
}

// One wave-wide load into LDS, 16 or 4 bytes or one (as a word) a lane, lane l's at lds + 16 l or 4 l; `base` is the wave's, or the address is the lane's own.  The waits
// for them are placed by hand: the compiler does not count them.
__device__ __forceinline__ void load16_lds(uint32_t lds, const void* base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load16_lds(uint32_t lds, const void* at) { asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at) : "memory"); }
__device__ __forceinline__ void load4_lds(uint32_t lds, const void* at) { asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(at) : "memory"); }
__device__ __forceinline__ void load1_lds(uint32_t lds, const void* at) { asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_ubyte %1, off" ::"s"(lds), "v"(at) : "memory"); }
// The largest of the 16 lanes that have a key's dims
__device__ __forceinline__ uint32_t dims_max(uint32_t v) {
    v = max(v, (uint32_t)dpp_word<kDppSwap1>((int)v));
    v = max(v, (uint32_t)dpp_word<kDppSwap2>((int)v));
    v = max(v, (uint32_t)dpp_word<0x141>((int)v));           // (row_half_mirror: the quads of eight lanes)
    return max(v, (uint32_t)dpp_word<0x140>((int)v));        // (row_mirror: the eights)
}
// In a branch that is seldom taken: keeps the compiler from running what it holds every time and selecting.
__device__ __forceinline__ void rarely() { asm volatile(""); }
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// tile_request() of 16 rows, by a look of 64 lanes at a time: one load for up to 64 requests, two for 4096
__device__ __forceinline__ int block_request(const AttendArgs& a, int t, int lane) {
    int lo = 0, n = a.requests;                  // among requests lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 63) >> 6, at = lane * step;
        const bool before = at < n && (long long)a.starts[lo + at] * a.group / 16 + lo + at <= t;
        const int last = (int)__popcll(__ballot(before)) - 1;            // (ascending: the lanes before it too; the first one's always is)
        lo += max(last, 0) * step;
        n = min(step, n - max(last, 0) * step);
    }
    return lo;
}

// A wave's steps of 32 keys in LDS: codes of keys and values, then their scales.  WORDS: a key has four or eight blocks, its scales are loaded by words; else by bytes, which
// lie in words of their own.
constexpr int most_blocks(int DIM, bool words) { return DIM == 256 && !words ? 7 : DIM / 32; }
constexpr int step_bytes(int DIM, bool words) { return 2 * 32 * most_blocks(DIM, words) * (words ? 17 : 20); }
constexpr int steps_ahead(int DIM) { return DIM == 64 ? 4 : 2; }          // (dim 128 with three: a block less on a compute unit, 64 requests over 1 to 8192 keys 87 us, not 83)
constexpr int rows_lds(int DIM, bool words, int RW) {
    const int ring = RW * steps_ahead(DIM) * step_bytes(DIM, words), sums = RW * 16 * (DIM + 4 + 2) * 4;
    return ring > sums ? ring : sums;
}

// ------------------------------------------------------------------------------------------------
// Sixteen rows (tokens times heads of a group, in order) of one request and one head of the cache per block.  The request's keys are dealt
// out in shares of `share` to blocks and in each to RW waves, which run on their own, 32 keys at a time, and join their sums in LDS.  A wave's next steps are on their
// way into its own part of LDS meanwhile, 16 bytes a lane.
//   scores   S^T[key][row] = K Q^T (16 x 16 x 32 products): a lane has a quarter of a key's dims, its codes become bf16 with their block's power of two, exactly;
//   softmax  a lane's eight scores belong to one row; its unit (p = 2^(s - unit)) is shared by the row's four lanes and moves up when its scores pass it far;
//   values   O^T[dim][row] = V^T P^T: S^T's layout is P^T's operand layout if the keys of a 32 are numbered (lane group, tile, i), so
//            nothing is exchanged; a lane reads DIM / 16 dims of eight keys and turns them in registers.  Values lie in LDS with four keys in an order by their
//            group of four, so that the lanes' reads of four groups use all banks.
// bf16 has fp32's range, so that no scale leaves the codes; q and p are held in pieces of it: q exactly (bf16 1, fp16 2, fp32 3 pieces), p to 16 bits for bf16 and fp16
// tensors and to 24 for fp32 ones.
// Bound by memory where keys are many: a token each of 64 requests of 1 to 8192 keys, 8 heads of 128 with four rows each, bf16, 72 to 77 us (4.3 to 4.5 TB/s;
// equal lengths of 4096 in 60 to 62 with the joining pass); vector instructions are issued in 40 % of the cycles, most of them codes' way to bf16.  Values through registers, as the 8-bit cache's blocks take
// them, were 105: a wave's loads were too few to fill the way to memory.  Few requests are bound by a wave's steps in
// sequence (nine of up to 1500 keys, fp32, dim 64: 20 us in one share each).
// UNI: the page size is a multiple of 16 and DIM is the heads' dim (rounded up to blocks): whole tiles of 16 keys lie on a page and their address is scalar.
// ------------------------------------------------------------------------------------------------
template <int TYPE, int DIM, bool UNI, bool WORDS, int RW>
__global__ __launch_bounds__(64 * RW, 2) void mx_attend_rows_kernel(const AttendArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int QP = TYPE == kF32 ? 3 : TYPE == kF16 ? 2 : 1, PP = TYPE == kF32 ? 3 : 2;      // pieces
    constexpr int CB = DIM / 16, KW = DIM / 32, VW = DIM == 256 ? 2 : 1;       // a lane's dims of a value; words of a key, of a value
    constexpr int MOST = most_blocks(DIM, WORDS), STEP = step_bytes(DIM, WORDS), R = steps_ahead(DIM), NC = (MOST + 1) / 2;      // (loads of a step's codes, keys or values)
    constexpr int NL = WORDS ? 2 * NC + DIM / 128 : DIM == 256 ? 12 : 4 * NC;  // loads of a step, with its scales (five or six blocks of 256 dims have 12, seven 16)
    extern __shared__ __attribute__((aligned(1024))) float lds[];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n16 = lane & 15, kg = lane >> 4;
    // Heads first: an XCD has as few heads' keys in its L2 as can be.
    const int place = (int)((a.close ? blockIdx.z * gridDim.y * gridDim.x : 0u) + blockIdx.y * gridDim.x + blockIdx.x), group_of = div_by(place, a.by_heads);
    const int head = place - group_of * a.c.heads;
    const int D = a.c.dim, NB = UNI ? DIM / 32 : mx_blocks(D), RB = 16 * NB;

    Unit job;
    if (a.close) {
        if (!unit_of(a, group_of, 16, true, lane, &job)) return;
    } else {
        const int block = (int)gridDim.x - 1 - group_of;
        const int b = block_request(a, block, lane);
        job.rq = request_of(a, b);
        job.tile = (int)((long long)block - ((long long)a.starts[b] * a.group / 16 + b));
        job.share = (int)blockIdx.z;
        job.shares = shares_of(a, job.rq.length);
    }
    const Request& rq = job.rq;
    const int nrows = rq.tokens * a.group, tile = job.tile, split = job.share, shares = job.shares;
    if (tile < 0 || (long long)tile * 16 >= nrows) return;
    const int r0 = tile * 16;
    const int heads = a.c.heads * a.group;

    // the block's keys: of those that its last row sees
    const int last_token = div_by(min(r0 + 15, nrows - 1), a.by_group);
    const int behind = rq.length - rq.new_tokens;               // keys before the new tokens
    const int seen_end = max(0, a.causal ? min(rq.length, behind + last_token + 1) : rq.length);
    const int all = max(0, a.causal ? min(rq.length, behind + div_by(r0, a.by_group) + 1) : rq.length);      // keys that all of its rows see
    const int all_steps = (seen_end + 31) >> 5;
    const int each = (int)((uint32_t)all_steps / (uint32_t)shares), more = all_steps - each * shares;      // (shares of `each` steps, the first ones of one more)
    const int from = split < shares ? min(32 * (each * split + min(split, more)), seen_end) : seen_end;
    const int end = split < shares ? min(32 * (each * (split + 1) + min(split + 1, more)), seen_end) : seen_end;
    if (a.splits > 1) {
        // nothing here, or in the shares behind the request's last (which have blocks of their own where those are not close): the joining pass looks at m alone
        const bool none = from >= end && split != 0;
        const int lo = none ? split : shares, hi = none ? split + 1 : a.close && split == 0 ? a.splits : 0;
        for (int i = (int)threadIdx.x; i < 16 * (hi - lo); i += 64 * RW) {
            const int r = r0 + (i & 15), t = div_by(r, a.by_group);
            if (r < nrows) a.part_ml[2 * ((size_t)(lo + (i >> 4)) * a.tokens * heads + (size_t)(rq.token0 + t) * heads + head * a.group + (r - t * a.group))] = kNone;
        }
        if (none) return;
    }

    // this lane's row
    const int row = r0 + n16;
    const bool have = row < nrows;
    const int token = div_by(have ? row : r0, a.by_group), gh = (have ? row : r0) - token * a.group;
    const int limit = a.causal ? min(rq.length, behind + token + 1) : rq.length;

    // this wave's keys: whole 32s of the block's share
    const int steps = (end - from + 31) >> 5;
    const int s_from = steps * wave / RW, s_to = steps * (wave + 1) / RW;
    // Blocks of values up to this byte need no look: sums of p v with p up to 2^16, 2^16 6 2^(byte - 127) of each of the wave's keys, stay below 2^127.
    const uint32_t calm = 235u - (32u - (uint32_t)__builtin_clz(32 * max(s_to - s_from, 1)));

    // ---- loader: codes of keys and values and their scales, as they are, into the wave's steps in LDS
    const uint8_t *const kq = reinterpret_cast<const uint8_t*>(a.c.kq), *const vq = reinterpret_cast<const uint8_t*>(a.c.vq);
    const uint8_t *const ksb = reinterpret_cast<const uint8_t*>(a.c.ks), *const vsb = reinterpret_cast<const uint8_t*>(a.c.vs);
    constexpr int V_AT = 32 * MOST * 16, KS_AT = 2 * V_AT, VS_AT = KS_AT + 32 * MOST * (WORDS ? 1 : 4);
    const uint8_t* const mine = reinterpret_cast<const uint8_t*>(lds) + wave * (R * STEP);
    const uint32_t mine_lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(size_t)mine);
    const auto value_row = [](int r) __attribute__((always_inline)) { return (r & ~3) | (((r & 3) - (r >> 2)) & 3); };      // of the key at a place of the values' 16
    uint32_t ok[R] = {};                      // bit j: key j of the step is in the cache, and before `end`; [0]: of the step that is multiplied next
    // pages of the request from `page0` on, one a lane: looked at 64 at a time
    int page0 = div_by(from + s_from * 32, a.c.by_page), ids;
    const auto look = [&]() __attribute__((always_inline)) {
        const int p = page0 + lane;
        ids = (long long)p * a.c.page_size < end ? rq.pages[p] : -1;
    };
    const auto fetch = [&](int s, int slot) __attribute__((always_inline)) {
        const int j0 = from + s * 32;
        const uint32_t to = mine_lds + (uint32_t)slot * STEP;
        if (div_by(min(j0 + 31, end - 1), a.c.by_page) - page0 >= 64) {
            page0 = div_by(j0, a.c.by_page);
            look();
            __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0): the compiler knows of it, and waits nowhere else for these loads
        }
        if constexpr (UNI) {
            uint32_t there = 0;
            size_t at[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int j = j0 + 16 * t, page = div_by(j, a.c.by_page);
                const int id = __builtin_amdgcn_readlane(ids, min(page - page0, 63));
                const bool in = j < end && (unsigned)id < (unsigned)a.c.pages;
                at[t] = ((size_t)(in ? id : 0) * a.c.heads + head) * a.c.page_size + (in ? j - page * a.c.page_size : 0);
                if (in) there |= (j + 16 <= end ? 0xffffu : (1u << (end - j)) - 1u) << (16 * t);
            }
            ok[R - 1] = there;
            if constexpr (DIM == 64) {           // (two tiles a load)
                const size_t k = lane < 32 ? at[0] : at[1];
                const uint32_t g = (uint32_t)(lane & 31);
                load16_lds(to, kq + k * 32 + g * 16);
                load16_lds(to + V_AT, vq + k * 32 + (uint32_t)value_row((int)g >> 1) * 32u + (g & 1u) * 16u);
                load1_lds(to + KS_AT, ksb + k * 2 + g);
                load1_lds(to + VS_AT, vsb + k * 2 + g);
            } else {
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    const int t = i / (NC / 2), g = (DIM == 256 ? (i & 1) * 64 : 0) + lane, r = g / MOST;
                    load16_lds(to + (uint32_t)i * 1024u, kq + at[t] * RB, (uint32_t)g * 16u);
                    load16_lds(to + V_AT + (uint32_t)i * 1024u, vq + at[t] * RB, (uint32_t)(value_row(r) * RB + (g % MOST) * 16));
                }
                if constexpr (DIM == 128) {      // (a word a key, keys' and values')
                    const size_t k = (lane & 16 ? at[1] : at[0]) + (lane & 15);
                    load4_lds(to + KS_AT, (lane < 32 ? ksb : vsb) + k * 4);
                } else {
                    const size_t k = (lane < 32 ? at[0] : at[1]) * 8 + (lane & 31) * 4;
                    load4_lds(to + KS_AT, ksb + k);
                    load4_lds(to + VS_AT, vsb + k);
                }
            }
        } else {
            // lane j looks up key j (lanes from 32 on again); the lanes that load for it take its place from there
            const int j = j0 + (lane & 31), page = div_by(j, a.c.by_page);
            const int id = __shfl(ids, min(page - page0, 63), kWave);
            const bool in = j < end && (unsigned)id < (unsigned)a.c.pages;
            const int row_of = in ? j - page * a.c.page_size : 0, page_of = in ? id : 0;
            ok[R - 1] = (uint32_t)__ballot(in);
            const auto at = [&](int key) __attribute__((always_inline)) {
                return ((size_t)__shfl(page_of, key, kWave) * a.c.heads + head) * a.c.page_size + __shfl(row_of, key, kWave);
            };
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int g = 64 * i + lane, r = min(g / NB, 31), in_row = g - g / NB * NB;
                const size_t k = at(r), v = at((r & 16) | value_row(r & 15));
                if (g < 32 * NB) {
                    load16_lds(to + (uint32_t)i * 1024u, kq + k * RB + in_row * 16);
                    load16_lds(to + V_AT + (uint32_t)i * 1024u, vq + v * RB + in_row * 16);
                }
                if constexpr (!WORDS) {
                    if (g < 32 * NB) {
                        load1_lds(to + KS_AT + (uint32_t)i * 256u, ksb + k * NB + in_row);
                        load1_lds(to + VS_AT + (uint32_t)i * 256u, vsb + k * NB + in_row);
                    }
                }
            }
            if constexpr (WORDS && DIM == 128) {
                const size_t k = at(lane & 31);
                load4_lds(to + KS_AT, (lane < 32 ? ksb : vsb) + k * 4);
            } else if constexpr (WORDS) {
                const size_t k = at(lane >> 1) * 8 + (lane & 1) * 4;
                load4_lds(to + KS_AT, ksb + k);
                load4_lds(to + VS_AT, vsb + k);
            }
        }
    };

    // q, as products' operand: with the sign of the scale, and for none zeros, so that the largest product is the largest score
    // dims of a lane: DIM 64 16 kg .., 128 32 kg .., 256 128 i + 32 kg .. (beyond D: q is zero there, and nothing is stored)
    const auto key_dim = [&](int i) __attribute__((always_inline)) { return DIM == 64 ? 16 * kg : DIM == 128 ? 32 * kg : 128 * i + 32 * kg; };
    ma_b8 qf[QP][KW];
    const float qscale = a.scale == 0.0f ? 1.0f : fabsf(a.scale) * kLog2e;
    {
        const T* qp = static_cast<const T*>(a.q) + (size_t)(rq.token0 + token) * a.q_token + (size_t)(head * a.group + gh) * a.q_head;
        float v[KW][8];
        if (s_from < s_to) look();
#pragma unroll
        for (int i = 0; i < KW; ++i) {
            const int d = key_dim(i / 4) + 8 * (i % 4);
            load8<TYPE>(qp + d, D - d, a.wide_q, v[i]);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
            for (int u = 0; u + 1 < R; ++u) ok[u] = ok[u + 1];
            if (s_from + i < s_to) fetch(s_from + i, i);
        }
        const float sign = a.scale > 0.0f ? 1.0f : a.scale < 0.0f ? -1.0f : 0.0f;
#pragma unroll
        for (int i = 0; i < KW; ++i) {
#pragma unroll
            for (int u = 0; u < 8; ++u) v[i][u] *= sign;
            ma_b8 piece[QP];
            bf16_pieces<QP>(v[i], piece);
#pragma unroll
            for (int p = 0; p < QP; ++p) qf[p][i] = piece[p];
        }
    }

    float m = kNone, unit = 0.0f;                // the largest score when the unit last moved; the unit: m, or 0 where nothing was seen yet
    float l = 0.0f;                              // sum of this lane's p
    tk_f4 o[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) o[c] = tk_f4{0.f, 0.f, 0.f, 0.f};

    // where the lane's operands lie in a step: keys 16 t + n16; values 16 t + 4 kg + i
    constexpr int SB = WORDS ? 1 : 4;            // bytes of a scale
    const int v_dim = n16 * CB < D ? n16 * CB : 0;
    const uint32_t s_key = (uint32_t)(n16 * NB * SB), s_value = (uint32_t)((4 * kg * NB + v_dim / 32) * SB);
    uint32_t k_at[KW / 4 ? KW / 4 : 1], v_at[4];
#pragma unroll
    for (int i = 0; i < (KW / 4 ? KW / 4 : 1); ++i) k_at[i] = (uint32_t)(n16 * RB + (key_dim(i) < D ? key_dim(i) : 0) / 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) v_at[i] = (uint32_t)((4 * kg + ((i + kg) & 3)) * RB + v_dim / 2);

    int slot = 0;
    for (int s = s_from; s < s_to; ++s) {
        const int j0 = from + s * 32;
        if (s + R <= s_to) wait_loads<(R - 1) * NL>();
        else wait_loads<0>();
        // this step's operands, then its place is loaded again
        const uint8_t* const step = mine + slot * STEP;
        uint32_t kw[2][KW], ke[2][KW / 4 ? KW / 4 : 1], vw[8][VW], vs[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if constexpr (DIM == 64) {
                const uint2 w = *reinterpret_cast<const uint2*>(step + 16 * t * RB + k_at[0]);
                kw[t][0] = w.x; kw[t][1] = w.y;
                ke[t][0] = step[KS_AT + 16 * t * NB * SB + s_key + (key_dim(0) < D ? key_dim(0) : 0) / 32 * SB];
            } else {
#pragma unroll
                for (int i = 0; i < KW / 4; ++i) {
                    const uint4 w = *reinterpret_cast<const uint4*>(step + 16 * t * RB + k_at[i]);
                    kw[t][4 * i] = w.x; kw[t][4 * i + 1] = w.y; kw[t][4 * i + 2] = w.z; kw[t][4 * i + 3] = w.w;
                    ke[t][i] = step[KS_AT + 16 * t * NB * SB + s_key + (key_dim(i) < D ? key_dim(i) : 0) / 32 * SB];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int u = 4 * t + i;
                const uint8_t* const at = step + V_AT + 16 * t * RB + v_at[i];
                if constexpr (DIM == 64) vw[u][0] = *reinterpret_cast<const uint16_t*>(at);
                else if constexpr (DIM == 128) vw[u][0] = *reinterpret_cast<const uint32_t*>(at);
                else {
                    const uint2 w = *reinterpret_cast<const uint2*>(at);
                    vw[u][0] = w.x; vw[u][VW - 1] = w.y;
                }
                vs[u] = step[VS_AT + s_value + (uint32_t)((16 * t + i) * NB * SB)];
            }
        }
        const uint32_t in = ok[0];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int u = 0; u + 1 < R; ++u) ok[u] = ok[u + 1];
        if (s + R < s_to) fetch(s + R, slot);
        slot = slot + 1 == R ? 0 : slot + 1;

        float x[8], kscale[2][KW / 4 ? KW / 4 : 1];
        uint32_t largest_scale = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < (KW / 4 ? KW / 4 : 1); ++i) {
                kscale[t][i] = __uint_as_float(ke[t][i] << 23);
                largest_scale = max(largest_scale, ke[t][i]);
            }
        if (__any(largest_scale == 255u)) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < (KW / 4 ? KW / 4 : 1); ++i) kscale[t][i] = mx_power(ke[t][i]);
            rarely();
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            tk_f4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                const float scale = kscale[t][i / 4];
                const uint4 f = make_uint4(codes_bf16<0>(kw[t][i], scale), codes_bf16<1>(kw[t][i], scale), codes_bf16<2>(kw[t][i], scale), codes_bf16<3>(kw[t][i], scale));
                const ma_b8 kf = __builtin_bit_cast(ma_b8, f);
#pragma unroll
                for (int p = 0; p < QP; ++p) sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[p][i], sc, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * t + i] = sc[i];
        }
        largest_scale = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) largest_scale = max(largest_scale, vs[u]);
        if (j0 + 32 > all || in != 0xffffffffu) {            // some keys are not there, or not for all rows
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int j = 16 * (u >> 2) + 4 * kg + (u & 3);
                const bool there = ((in >> j) & 1u) != 0;
                vs[u] = there ? vs[u] : 0u;
                x[u] = there && j0 + j < limit ? x[u] : kNone;
            }
            rarely();
        }
        float top = kNone;
#pragma unroll
        for (int u = 0; u < 8; ++u) top = fmaxf(top, x[u]);
        top *= qscale;
        // Larger values take as much from p's range as they are beyond that: the unit goes by a key's score and this together (by 29 more at most with 32 keys).  By the row's own
        // keys: one that it does not see, or sees at 2^-100, leaves the others their bits.
        const bool large = __any(largest_scale > calm);
        if (large) {
            top = kNone;
#pragma unroll
            for (int u = 0; u < 8; ++u) top = fmaxf(top, __builtin_fmaf(x[u], qscale, (float)(max(dims_max(vs[u]), calm) - calm)));
            rarely();
        }
        // (bf16 holds p far above 1: the unit moves rarely)
        if (__any(top > m + 16.0f)) {
            const float largest = halves_max(rows16_max(top));
            const bool moves = largest > m + 16.0f;              // (of this row: it does not go by its neighbours')
            const float by = !moves ? 1.0f : m == kNone ? 0.0f : __builtin_amdgcn_exp2f(unit - largest);
            m = moves ? largest : m;
            unit = moves ? largest : unit;
            l *= by;
#pragma unroll
            for (int d = 0; d < CB; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[d][r] *= by;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            x[u] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u], qscale, -unit));
            l += x[u];
        }
        // Values that are not finite (some lane has a block of them) go into p of the rows that see them, and become zeros for the others.
        if (large) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const unsigned long long lanes = __ballot(vs[u] >= 253u) >> (16 * kg) & 0xffffull;
                if (lanes && x[u] != 0.0f) x[u] = NAN;
                if (lanes) vs[u] = 0u;
            }
        }
        ma_b8 pf[PP];
        bf16_pieces<PP>(x, pf);
        // values: pairs of dims of a key, then pairs of keys of a dim
        float scale[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) scale[u] = __uint_as_float(vs[u] << 23);
#pragma unroll
        for (int c2 = 0; c2 < CB / 2; ++c2) {
            uint32_t w[8], f[2][4];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t word = vw[u][c2 / 4];
                w[u] = c2 % 4 == 0 ? codes_bf16<0>(word, scale[u]) : c2 % 4 == 1 ? codes_bf16<1>(word, scale[u]) : c2 % 4 == 2 ? codes_bf16<2>(word, scale[u]) : codes_bf16<3>(word, scale[u]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                f[0][u] = __builtin_amdgcn_perm(w[2 * u + 1], w[2 * u], 0x05040100u);
                f[1][u] = __builtin_amdgcn_perm(w[2 * u + 1], w[2 * u], 0x07060302u);
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const ma_b8 vf = __builtin_bit_cast(ma_b8, make_uint4(f[c][0], f[c][1], f[c][2], f[c][3]));
#pragma unroll
                for (int p = 0; p < PP; ++p) o[2 * c2 + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[p], o[2 * c2 + c], 0, 0, 0);
            }
        }
    }
    __syncthreads();                             // (the steps' places are the sums' now)
    l = halves_sum(rows16_sum(l));
    float down;
    const float mw = normalised(-unit, &l, &down);

    // the waves' sums, in LDS: [wave][row][DIM + 4].  A lane has CB neighbouring dims of its row for each r.
    float* const sm = lds;
    float* const sl = sm + 16 * RW;
    float* const so = sl + 16 * RW;
    constexpr int PITCH = DIM + 4;
    if (kg == 0) {
        sm[wave * 16 + n16] = mw;
        sl[wave * 16 + n16] = l;
    }
    if (have) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < CB; c += 4)
                *reinterpret_cast<float4*>(so + (wave * 16 + n16) * PITCH + CB * (4 * kg + r) + c) =
                    make_float4(o[c][r] * down, o[c + 1][r] * down, o[c + 2][r] * down, o[c + 3][r] * down);
    }
    __syncthreads();
    constexpr int LR = 4 * RW, PER = DIM / LR < 4 ? 4 : DIM / LR;      // lanes per row; dims of a lane
    const int jr = (int)threadIdx.x / LR, jl = (int)threadIdx.x % LR;
    if (r0 + jr >= nrows) return;
    // An eighth of the waves' sums (the joining pass takes them so): together they may pass fp32 where their mean does not.
    constexpr float kEighth = 1.0f / kRowsPartScale;
    float mm = sm[jr], total = 0.0f, w[RW];
#pragma unroll
    for (int i = 1; i < RW; ++i) mm = fmaxf(mm, sm[16 * i + jr]);
#pragma unroll
    for (int i = 0; i < RW; ++i) {
        const float mi = sm[16 * i + jr];
        w[i] = mi == kNone ? 0.0f : __builtin_amdgcn_exp2f(mi - mm);
        total += w[i] * sl[16 * i + jr];
        w[i] *= kEighth;
    }
    const int jt = div_by(r0 + jr, a.by_group), jg = (r0 + jr) - jt * a.group;
    const size_t out_row = (size_t)(rq.token0 + jt) * heads + head * a.group + jg;
    const bool whole = a.splits == 1;
    const size_t part_row = (size_t)split * a.tokens * heads + out_row;
    const float by = whole ? per_sum(total) * kRowsPartScale : 1.0f;
    if (jl == 0) {
        if (whole) {
            if (a.lse) a.lse[out_row] = log_of_sum(mm, total);
        } else {
            a.part_ml[2 * part_row] = mm;
            a.part_ml[2 * part_row + 1] = total;
        }
    }
#pragma unroll
    for (int c = 0; c < PER; c += 4) {
        const int d = jl * PER + c;
        if (d >= D) break;
        tk_f4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < RW; ++i) {
            const tk_f4 t = *reinterpret_cast<const tk_f4*>(so + (16 * i + jr) * PITCH + d);
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] += w[i] * t[u];
        }
        typedef T V __attribute__((ext_vector_type(4)));
        V r;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            v[u] *= by;
            r[u] = (T)v[u];
        }
        if (whole) *reinterpret_cast<V*>(static_cast<T*>(a.out) + out_row * D + d) = r;
        else *reinterpret_cast<tk_f4*>(a.part_o + part_row * D + d) = v;
    }
}

template <int TYPE, int DIM, bool UNI, bool WORDS, int RW>
hipError_t rows_dim(const AttendArgs& a, hipStream_t st) {
    constexpr int LDS = rows_lds(DIM, WORDS, RW);
    static std::atomic<unsigned long long> done{0};
    const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(&mx_attend_rows_kernel<TYPE, DIM, UNI, WORDS, RW>), LDS, done);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((long long)a.tokens * a.group / 16 + a.requests), (unsigned)a.c.heads, (unsigned)a.splits);
    KernelTimer kt(KID_MX_ATTEND, st);
    launch_timed(kt, (mx_attend_rows_kernel<TYPE, DIM, UNI, WORDS, RW>), grid, dim3(64 * RW), LDS, st, a);
    return hipGetLastError();
}
template <int TYPE, int DIM, int RW>
hipError_t rows_of(const AttendArgs& a, hipStream_t st) {
    const int blocks = mx_blocks(a.c.dim);
    if (blocks == DIM / 32 && a.c.page_size % 16 == 0) return rows_dim<TYPE, DIM, true, (DIM > 64), RW>(a, st);
    if (DIM > 64 && blocks == DIM / 32) return rows_dim<TYPE, DIM, false, (DIM > 64), RW>(a, st);
    return rows_dim<TYPE, DIM, false, false, RW>(a, st);
}
template <int TYPE, int RW>
hipError_t rows_any(const AttendArgs& a, hipStream_t st) {
    return a.c.dim <= 64 ? rows_of<TYPE, 64, RW>(a, st) : a.c.dim <= 128 ? rows_of<TYPE, 128, RW>(a, st) : rows_of<TYPE, 256, RW>(a, st);
}
template <int TYPE>
hipError_t rows_type(const AttendArgs& a, hipStream_t st) { return a.waves == 8 ? rows_any<TYPE, 8>(a, st) : rows_any<TYPE, 4>(a, st); }

}  // namespace

hipError_t launch_mx_attend_rows(const AttendArgs& a, hipStream_t st) {
    if (a.type == kF32) return rows_type<kF32>(a, st);
    if (a.type == kBF16) return rows_type<kBF16>(a, st);
    return rows_type<kF16>(a, st);
}

}  // namespace int8t
