// Attention of many new tokens of a request (chunks of a prompt) over the paged cache: the formulas and the joining of shares of
// token_attend.hip.
//
// A block has 32 NW rows (tokens times heads of a group, in order) of one request and head of the cache, a wave 32 of them; the keys pass
// by in tiles of 64.  While one tile is multiplied, the next one's codes, which were loaded a tile ahead, become fp16 (exactly) in LDS,
// once for all waves, and the one after it is loaded.
//   scores   S^T[key][row] = K Q^T in products of 32 x 32 x 16: a lane's 16 scores of 32 keys belong to one row, so its unit (RowUnit) needs
//            one exchange between the halves of the wave;
//   values   O^T[dim][row] = V^T P^T: the scores' layout is P^T's operand layout with the keys in the order that the transposing LDS read
//            of V (rows of keys, as they came) delivers: p never leaves its lane.
// Bound by vector and matrix units together: a score costs 9 to 10 vector operations, of which the exponential counts for four, and 256 multiply-adds
// (DIM 128), and arithmetic of one wave and products of another overlap by half only (fma 295 us, products 322, together 466).  Two chunks of 2048 tokens over 8192 keys, 32 heads of 128 on 8, bf16:
// 603 to 615 us (478 GFLOP: 0.8 PFLOP/s; a large library product in fp16 1.18), in 55 % of whose cycles a SIMD issues vector instructions and in 32 % has a product: 88 %
// together; LDS 12 %.
#include "mx4.h"
#include "token_attend.h"

namespace int8t {
namespace {

typedef short tc_s4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) tc_s4* tc_lds;
constexpr int TK = 64;          // keys of a tile

// granule (16 bytes, eight dims) g of key `key` in a tile of rows of DIM fp16.  Keys' operand: 16 neighbouring keys, one granule; values':
// four neighbouring keys, four granules: either way 16 different granules modulo 16.
template <int DIM>
__device__ __forceinline__ int k_slot(int key, int g) { return DIM == 64 ? key * 8 + (g ^ ((key >> 1) & 7)) : key * (DIM / 8) + (g ^ (key & 15)); }
template <int DIM>
__device__ __forceinline__ int v_slot(int key, int g) { return DIM == 64 ? key * 8 + (g ^ ((key & 2) << 1)) : key * (DIM / 8) + (g ^ ((key & 3) << 2)); }

// Tiles in LDS of keys, of values (multiplied a step after their keys) and of scales, see the steps below; and how far ahead tiles are written.
constexpr bool takes_turns(int NW) { return NW == 8; }
constexpr int key_tiles(int NW) { return takes_turns(NW) ? 3 : 2; }
constexpr int value_tiles(int DIM, int NW) { return takes_turns(NW) ? 4 : DIM == 256 ? 2 : 3; }
constexpr int chunk_lds(int DIM, int NW) { return (key_tiles(NW) + value_tiles(DIM, NW)) * TK * DIM * 2 + 3 * 3 * TK * 4; }

// MX: keys and values are microscaled 4-bit codes (mx4.h).  A block's codes become fp16 times a power of two relative to its row's largest scale, which is then
// the row's: what is above stays as it is.  Blocks 2^36 below the row's largest lose bits, 2^41 below they are zeros.  Two chunks of 2048 tokens over 8192 keys, 32 heads on 8 of
// 128, bf16: 578 us, 0.83 PFLOP/s; vector instructions are issued in 50 % of the cycles and products run in 33 %, hardly at once, and waves wait in 40 % of their time.
template <bool MX> struct Piece { typedef uint4 codes; typedef float scale; };
template <> struct Piece<true> { typedef uint2 codes; typedef uint32_t scale; };
constexpr int kMxUp = 13;       // 6 2^13 is in fp16's range
// The largest of the DIM / 16 neighbouring lanes that have a key
template <int DIM>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
    v = max(v, (uint32_t)dpp_word<kDppSwap1>((int)v));
    v = max(v, (uint32_t)dpp_word<kDppSwap2>((int)v));
    if (DIM == 128) v = max(v, (uint32_t)dpp_word<0x141>((int)v));      // (row_half_mirror: the quads of eight lanes)
    return v;
}

// bf16 tensors' keys keep their scales -- bf16 has the range, and q is exact in it --, so that scores need no factor of a key (two chunks of 2048 tokens over 8192 keys
// 600 -> 579 us); values, whose weights need more bits than bf16's, are fp16 in either case.
constexpr bool whole_keys(int type, bool mx) { return mx && type == kBF16; }
typedef __bf16 tc_b8 __attribute__((ext_vector_type(8)));

// UNI: the keys whose pieces a wave loads at a time lie on one page (its size is a multiple of 1024 / DIM): addresses are scalar.
template <int TYPE, int DIM, int NW, bool UNI, bool MX>
__global__ __launch_bounds__(64 * NW, NW == 4 && (DIM == 256 || (DIM == 128 && TYPE == kF32)) ? 1 : 2) void attend_chunk_kernel(const AttendArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int PARTS = TYPE == kF32 ? 2 : 1, NT = 64 * NW, ROWS = 32 * NW;
    constexpr bool WHOLE = whole_keys(TYPE, MX);               // keys in LDS are bf16 with their scales, and q as it is
    constexpr int QS = DIM / 16, DT = DIM / 32;                // steps of the scores' products; tiles of dims
    constexpr int CH = 4 * DIM;                                // 16-byte pieces of a tile of codes
    constexpr int NP = CH / NT;                                // pieces of either tensor per thread
    static_assert(CH % NT == 0, "whole rounds of pieces");
    extern __shared__ __attribute__((aligned(1024))) uint4 lds[];
    constexpr bool TURNS = takes_turns(NW);                    // two waves on each SIMD that take turns, see below
    constexpr int KT = key_tiles(NW), VT = value_tiles(DIM, NW), TILE = TK * DIM / 8, AHEAD = TURNS ? 2 : 1;
    uint4* const sk = lds;                                     // [KT][TK][DIM] fp16
    uint4* const sv = lds + KT * TILE;                         // [VT][TK][DIM]
    float* const sc = reinterpret_cast<float*>(lds + (KT + VT) * TILE);      // [3][3][TK]: key scales, value scales, 0 or -infinity

    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n32 = lane & 31, half = lane >> 5;
    // Heads first, so that an XCD has as few heads' keys in its L2 as can be, and each request's last rows, which see the most keys, before its others, so that
    // the chip runs out of short blocks (tiles first, in order: 9 % more time for two chunks of 2048 tokens over 8192 keys).
    const bool close = MX && a.close;                          // (4 bits: blocks that have rows come first where requests are few)
    const int place = (int)((close ? blockIdx.z * gridDim.y * gridDim.x : 0u) + blockIdx.y * gridDim.x + blockIdx.x), group_of = div_by(place, a.by_heads);
    const int head = place - group_of * a.c.heads, block = (int)gridDim.x - 1 - group_of;
    const int D = a.c.dim;

    Unit job{};
    if (close && !unit_of(a, group_of, ROWS, false, lane, &job)) return;
    const int split = close ? job.share : (int)blockIdx.z;
    const int b = close ? 0 : tile_request(a, block, ROWS);
    const Request rq = close ? job.rq : request_of(a, b);
    const int nrows = rq.tokens * a.group;
    const long long tile = close ? job.tile : (long long)block - ((long long)a.starts[b] * a.group / ROWS + b);
    if (tile < 0 || tile * ROWS >= nrows) return;
    const int r0 = (int)tile * ROWS;
    const int row = r0 + 32 * wave + n32;
    const bool have = row < nrows;
    const int token = div_by(have ? row : r0, a.by_group), gh = (have ? row : r0) - token * a.group;
    const int behind = rq.length - rq.new_tokens;               // keys before the new tokens
    const int limit = a.causal ? min(rq.length, behind + token + 1) : rq.length;
    // keys that the block's last row sees, and those that all of its rows see
    const int last_token = div_by(min(r0 + ROWS - 1, nrows - 1), a.by_group);
    const int end = max(0, a.causal ? min(rq.length, behind + last_token + 1) : rq.length);
    const int all = max(0, a.causal ? min(rq.length, behind + div_by(r0, a.by_group) + 1) : rq.length);
    const int tiles = (end + TK - 1) / TK;
    const int t_from = (int)((long long)tiles * split / a.splits), t_to = (int)((long long)tiles * (split + 1) / a.splits);

    // q as the scores' right operand
    tk_h8 qf[PARTS][QS];
    float qscale;
    {
        const T* qp = static_cast<const T*>(a.q) + (size_t)(rq.token0 + token) * a.q_token + (size_t)(head * a.group + gh) * a.q_head;
        float v[QS][8];
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < QS; ++i) {
            const int d = i * 16 + half * 8;
            load8<TYPE>(qp + d, D - d, a.wide_q, v[i]);
#pragma unroll
            for (int u = 0; u < 8; ++u) m = fmaxf(m, fabsf(v[i][u]));
        }
        m = halves_max(m);
        float back = 1.0f;
        float up = WHOLE ? 1.0f : row_scale(m, &back);
        qscale = score_scale(a.scale, back, &up);
#pragma unroll
        for (int i = 0; i < QS; ++i)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float t = v[i][u] * up;
                if constexpr (WHOLE) {           // (bf16's bits, in the same registers)
                    qf[0][i][u] = __builtin_bit_cast(_Float16, (__bf16)t);
                    continue;
                }
                _Float16 first = (_Float16)t, rest;
                if (PARTS == 2) {
                    two_pieces(t, &first, &rest);
                    qf[PARTS - 1][i][u] = rest;
                }
                qf[0][i][u] = first;
            }
    }

    // ---- loader: this thread's pieces, piece p is 16 dims of a key; a wave's are those of KW neighbouring keys
    constexpr int KW = 1024 / DIM;
    typename Piece<MX>::codes rk[NP], rv[NP];
    typename Piece<MX>::scale rks[NP], rvs[NP];
    bool rok[NP];
    int ids[NP], ins[NP];                                      // pages, and places on them, of the keys that are loaded next
    const int d16 = (tid % (DIM / 16)) * 16, dc = d16 < D ? d16 : 0;              // (beyond D: q is zero there, and nothing is stored)
    const int key0 = tid / (DIM / 16), wkey0 = __builtin_amdgcn_readfirstlane(key0);
    auto key_of = [&](int p) __attribute__((always_inline)) { return key0 + p * (NT / (DIM / 16)); };
    auto page_ids = [&](int t) __attribute__((always_inline)) {                               // of tile t's keys
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int j = t * TK + (UNI ? wkey0 + p * (NT / (DIM / 16)) : key_of(p)), page = div_by(j, a.c.by_page);
            ids[p] = j < end ? rq.pages[page] : -1;
            ins[p] = j - page * a.c.page_size;
        }
    };
    const size_t page_rows = (size_t)a.c.heads * a.c.page_size, head_rows = (size_t)head * a.c.page_size;
    const int row_scales = MX ? mx_blocks(D) : 1, row_bytes = MX ? 16 * row_scales : D;      // of a key
    const uint32_t code_at = (uint32_t)(MX ? dc / 2 : dc) + (UNI ? (uint32_t)((key0 - wkey0) * row_bytes) : 0u);                  // from a wave's (a key's) place on
    const uint32_t scale_at = (uint32_t)(MX ? dc / 32 : 0) + (UNI ? (uint32_t)((key0 - wkey0) * row_scales) : 0u);
    typedef typename Piece<MX>::codes Codes;
    auto fetch = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const bool ok = (unsigned)ids[p] < (unsigned)a.c.pages;
            int id = ok ? ids[p] : 0, in = ok ? ins[p] : 0;
            if (UNI) {
                id = __builtin_amdgcn_readfirstlane(id);
                in = __builtin_amdgcn_readfirstlane(in);
            }
            const size_t place = (size_t)id * page_rows + (head_rows + in), codes = place * row_bytes;
            rok[p] = ok && t * TK + key_of(p) < end;
            rk[p] = *reinterpret_cast<const Codes*>(a.c.kq + codes + code_at);
            rv[p] = *reinterpret_cast<const Codes*>(a.c.vq + codes + code_at);
            if constexpr (MX) {
                rks[p] = (reinterpret_cast<const uint8_t*>(a.c.ks) + place * row_scales)[scale_at];
                rvs[p] = (reinterpret_cast<const uint8_t*>(a.c.vs) + place * row_scales)[scale_at];
            } else {
                rks[p] = (a.c.ks + place)[scale_at];
                rvs[p] = (a.c.vs + place)[scale_at];
            }
        }
    };
    // 16 codes as fp16; 4 bits: their block's scale becomes the row's factor (in place: handed out through a pointer of its own, the 8-bit form spilled)
    auto expand = [](const auto& c, auto& scale, uint4* lo, uint4* hi) __attribute__((always_inline)) {
        if constexpr (MX) {
            const uint32_t top = lanes_max<DIM>(scale);
            const int base = max((int)top - kMxUp, 1);       // (the row's factor is not below 2^-126: small rows keep their bits in smaller codes)
            const float up = __uint_as_float((uint32_t)max(127 + (int)scale - base, 0) << 23);
            scale = top == 255u ? 0x7fc00000u : (uint32_t)base << 23;
            const auto pair = [up](uint32_t w, auto sel) __attribute__((always_inline)) { return as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, up, decltype(sel)::value)); };
            typedef std::integral_constant<int, 0> B0; typedef std::integral_constant<int, 1> B1; typedef std::integral_constant<int, 2> B2; typedef std::integral_constant<int, 3> B3;
            *lo = make_uint4(pair(c.x, B0()), pair(c.x, B1()), pair(c.x, B2()), pair(c.x, B3()));
            *hi = make_uint4(pair(c.y, B0()), pair(c.y, B1()), pair(c.y, B2()), pair(c.y, B3()));
        } else {
            const uint32_t w[4] = {c.x ^ 0x80808080u, c.y ^ 0x80808080u, c.z ^ 0x80808080u, c.w ^ 0x80808080u};
            *lo = make_uint4(codes_f16<kLowPair>(w[0]), codes_f16<kHighPair>(w[0]), codes_f16<kLowPair>(w[1]), codes_f16<kHighPair>(w[1]));
            *hi = make_uint4(codes_f16<kLowPair>(w[2]), codes_f16<kHighPair>(w[2]), codes_f16<kLowPair>(w[3]), codes_f16<kHighPair>(w[3]));
        }
    };
    auto expand_key = [&](const auto& c, auto& scale, uint4* lo, uint4* hi) __attribute__((always_inline)) {
        if constexpr (WHOLE) {
            const float up = mx_power(scale);
            const auto pair = [up](uint32_t w, auto sel) __attribute__((always_inline)) {
                return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, up, decltype(sel)::value));
            };
            typedef std::integral_constant<int, 0> B0; typedef std::integral_constant<int, 1> B1; typedef std::integral_constant<int, 2> B2; typedef std::integral_constant<int, 3> B3;
            *lo = make_uint4(pair(c.x, B0()), pair(c.x, B1()), pair(c.x, B2()), pair(c.x, B3()));
            *hi = make_uint4(pair(c.y, B0()), pair(c.y, B1()), pair(c.y, B2()), pair(c.y, B3()));
        } else {
            expand(c, scale, lo, hi);
        }
    };
    const auto as_scale = [](auto s) __attribute__((always_inline)) { return __builtin_bit_cast(float, s); };
    auto stage = [&](int kslot, int vslot, int sslot) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int key = key_of(p), g = d16 >> 3;
            uint4 lo, hi;
            float* const s = sc + sslot * 3 * TK;
            expand_key(rk[p], rks[p], &lo, &hi);
            sk[kslot * TILE + k_slot<DIM>(key, g)] = lo;
            sk[kslot * TILE + k_slot<DIM>(key, g + 1)] = hi;
            expand(rv[p], rvs[p], &lo, &hi);
            sv[vslot * TILE + v_slot<DIM>(key, g)] = lo;
            sv[vslot * TILE + v_slot<DIM>(key, g + 1)] = hi;
            if (g == 0) {
                if (!WHOLE) s[key] = rok[p] ? as_scale(rks[p]) : 0.0f;
                s[TK + key] = rok[p] ? as_scale(rvs[p]) : 0.0f;
                s[2 * TK + key] = rok[p] ? 0.0f : kNone;
            }
        }
    };

    RowUnit unit;
    float l = 0.0f;                              // sum of this lane's p
    tk_f16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[d][v] = 0.0f;

    // What is the same for every tile: where a lane finds its operands.  Values: slot 8 half + i of a product of 16 keys is key 4 half + i
    // (i < 4) or 8 + 4 half + i - 4; a group of 16 lanes reads four keys by 16 dims: lane j points at key j / 4, dims 4 (j % 4) .. + 3, and gets
    // dim j of the four.
    const int vg = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), vkey = 4 * half + ((lane & 15) >> 2);
    const auto keys_at = [&](int kslot, int kt, int i) __attribute__((always_inline)) { return __builtin_bit_cast(tk_h8, sk[kslot * TILE + k_slot<DIM>(kt * 32 + n32, 2 * i + half)]); };
    const auto values_at = [&](uint32_t tv, int kt, int u, int d) __attribute__((always_inline)) {
        typedef short tc_s8 __attribute__((ext_vector_type(8)));
        const uint32_t at = tv + 16 * v_slot<DIM>(vkey, d * 4 + vg), row = (kt * 32 + u * 16) * DIM * 2;
        const tc_s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tc_lds)(uintptr_t)(at + row));
        const tc_s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tc_lds)(uintptr_t)(at + row + 8 * DIM * 2));
        return __builtin_bit_cast(tk_h8, tc_s8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    };
    tk_f16 x[2];                 // scores of a tile
    tk_h8 pf[2][PARTS][2];       // p of the tile before
    // values of the tile before
    tk_h8 vf[DT];
    const auto first_values = [&](int vslot) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < DT; ++d) vf[d] = values_at((uint32_t)(size_t)(sv + vslot * TILE) + 8 * (lane & 1), 0, 0, d);
    };
    const auto add_values = [&](int vslot) __attribute__((always_inline)) {      // (the first operands are there)
        const uint32_t tv = (uint32_t)(size_t)(sv + vslot * TILE) + 8 * (lane & 1);
#pragma unroll
        for (int ku = 0; ku < 4; ++ku) {
#pragma unroll
            for (int d = 0; d < DT; ++d) {
#pragma unroll
                for (int p = 0; p < PARTS; ++p) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[d], pf[ku >> 1][p][ku & 1], o[d], 0, 0, 0);
                if (ku < 3) vf[d] = values_at(tv, (ku + 1) >> 1, (ku + 1) & 1, d);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // scores.  A half tile's operands are requested together, ahead of its products: read one by one, each product would wait for LDS.  The
    // values' first ones follow (fp32: there are no registers for them yet).
    const auto scores = [&](int kslot, int vslot) __attribute__((always_inline)) {
        tk_h8 kf[QS];
#pragma unroll
        for (int i = 0; i < QS; ++i) kf[i] = keys_at(kslot, 0, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
            for (int v = 0; v < 16; ++v) x[kt][v] = 0.0f;
#pragma unroll
            for (int i = 0; i < QS; ++i) {
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    if constexpr (WHOLE) x[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(tc_b8, kf[i]), __builtin_bit_cast(tc_b8, qf[p][i]), x[kt], 0, 0, 0);
                    else x[kt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[i], qf[p][i], x[kt], 0, 0, 0);
                }
                if (kt == 0) kf[i] = keys_at(kslot, 1, i);
            }
            if (kt == 0 && PARTS == 1) first_values(vslot);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // (dims up to 256 leave no registers for operands that are read ahead: without 13 of them are spilled, and chunks take 4 % longer)
    const auto packed = []() __attribute__((always_inline)) {
        if constexpr (DIM == 256) __builtin_amdgcn_sched_barrier(0);
    };
    const auto softmax = [&](int t, int sslot) __attribute__((always_inline)) {
        const float* const s = sc + sslot * 3 * TK;
        // times the keys' scales; the tile's last keys and those behind a row's own
        const bool masked = (t + 1) * TK > all || __any(s[2 * TK + lane] != 0.0f);
        if constexpr (!WHOLE) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const tk_f4 ks = *reinterpret_cast<const tk_f4*>(s + kt * 32 + 8 * q + 4 * half);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[kt][4 * q + i] *= ks[i];
                }
        }
        if (masked) {
            const int left = limit - t * TK - 4 * half;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const tk_f4 none = *reinterpret_cast<const tk_f4*>(s + 2 * TK + kt * 32 + 8 * q + 4 * half);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (none[i] != 0.0f || kt * 32 + 8 * q + i >= left) x[kt][4 * q + i] = kNone;
                }
        }
        float top = kNone;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int v = 0; v < 16; ++v) top = fmaxf(top, x[kt][v]);
        top *= qscale;
        const float scale = s[TK + lane];
        if (__any(top > unit.room || fabsf(scale) > unit.vs) && unit.unknown(top = halves_max(top), scale)) {
            float weight = kNone;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const tk_f4 vs = *reinterpret_cast<const tk_f4*>(s + TK + kt * 32 + 8 * q + 4 * half);
#pragma unroll
                    for (int i = 0; i < 4; ++i) weight = fmaxf(weight, x[kt][4 * q + i] * qscale + RowUnit::log_of(vs[i]));
                    packed();
                }
            const float by = unit.set(top, halves_max(weight));
            l *= by;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[d][v] *= by;
        }
        packed();
        float largest = 0.0f;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const tk_f4 vs = *reinterpret_cast<const tk_f4*>(s + TK + kt * 32 + 8 * q + 4 * half);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[kt][4 * q + i], qscale, unit.c));
                    l += p;
                    x[kt][4 * q + i] = weight_of(p, vs[i]);
                    if (DIM < 256) largest = fmaxf(largest, fabsf(x[kt][4 * q + i]));
                }
                if (q & 1) packed();
            }
        if (DIM == 256) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int v = 0; v < 16; ++v) largest = fmaxf(largest, fabsf(x[kt][v]));
        }
        if (RowUnit::large(largest, l)) {
            const float by = unit.lower(halves_max(largest), halves_max(l));
            l *= by;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int v = 0; v < 16; ++v) x[kt][v] *= by;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[d][v] *= by;
        }
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                _Float16 first = (_Float16)x[kt][v], rest;
                if (PARTS == 2) {
                    two_pieces(x[kt][v], &first, &rest);
                    pf[kt][PARTS - 1][v >> 3][v & 7] = rest;
                }
                pf[kt][0][v >> 3][v & 7] = first;
            }
    };

    // Steps: products (scores of tile t, values of tile t - 1), then arithmetic (softmax of tile t, tile t + AHEAD to LDS).  With eight waves the
    // two of a SIMD take turns, a barrier between: the first has the products of tile t in turn 2 t and its arithmetic in turn 2 t + 1, the
    // second in turns 2 t + 1 and 2 t + 2.  Tile t + 2 is then written in turns 2 t + 1 and 2 t + 2 and read from turn 2 t + 4 on; in its place
    // were (three tiles of keys, four of values, three of scales) the keys of tile t - 1, last read in turn 2 t - 1, the values of
    // tile t - 2, last read in turn 2 t - 1, the scales of tile t - 1, last read in turn 2 t.  With four waves there is one barrier a step (two
    // where only two tiles of values fit): tile t + 1 takes the place of keys of tile t - 1 and values of tile t - 2, last read before it.
    const auto turn = []() __attribute__((always_inline)) { __syncthreads(); };
    if (t_from < t_to) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            page_ids(t_from + i);
            fetch(t_from + i);
            stage(i, i, i);
        }
        page_ids(t_from + AHEAD);
        turn();
        if (TURNS && wave >= 4) turn();
        int kcur = 0, knext = AHEAD % KT, vlast = 0, vcur = 0, vnext = AHEAD % VT, scur = 0, snext = AHEAD % 3;
        const auto after = [](int slot, int n) { return slot + 1 == n ? 0 : slot + 1; };
        for (int t = t_from; t < t_to; ++t) {
            if (t + AHEAD < t_to) {
                fetch(t + AHEAD);
                page_ids(t + AHEAD + 1);
            }
            scores(kcur, vlast);
            if (t > t_from) {
                if (PARTS == 2) first_values(vlast);
                add_values(vlast);
            }
            if (TURNS || VT == 2) turn();
            // (the arithmetic goes first where both waves have something to issue: without 2 % slower)
            if (TURNS) __builtin_amdgcn_s_setprio(2);
            softmax(t, scur);
            if (t + AHEAD < t_to) stage(knext, vnext, snext);
            if (TURNS) __builtin_amdgcn_s_setprio(0);
            turn();
            vlast = vcur;
            kcur = after(kcur, KT);
            knext = after(knext, KT);
            vcur = after(vcur, VT);
            vnext = after(vnext, VT);
            scur = after(scur, 3);
            snext = after(snext, 3);
        }
        first_values(vlast);
        add_values(vlast);
        if (TURNS && wave < 4) turn();
    }

    l = halves_sum(l);
    if (!have) return;
    const int heads = a.c.heads * a.group;
    const size_t out_row = (size_t)(rq.token0 + token) * heads + head * a.group + gh;
    if (a.splits == 1) {
        const float by = per_sum(l);
        if (a.lse && half == 0) a.lse[out_row] = log_of_sum(-unit.c, l);
        T* const out = static_cast<T*>(a.out) + out_row * D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int at = 32 * d + 8 * q + 4 * half;
                if (at < D) {
                    typedef T V4 __attribute__((ext_vector_type(4)));
                    V4 r;
#pragma unroll
                    for (int i = 0; i < 4; ++i) r[i] = (T)(o[d][4 * q + i] * by);
                    *reinterpret_cast<V4*>(out + at) = r;
                }
            }
    } else {
        const size_t part_row = (size_t)split * a.tokens * heads + out_row;
        float down;
        const float m = normalised(unit.c, &l, &down);
        if (half == 0) {
            a.part_ml[2 * part_row] = m;
            a.part_ml[2 * part_row + 1] = l;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int at = 32 * d + 8 * q + 4 * half;
                if (at < D)
                    *reinterpret_cast<float4*>(a.part_o + part_row * D + at) =
                        make_float4(o[d][4 * q] * down, o[d][4 * q + 1] * down, o[d][4 * q + 2] * down, o[d][4 * q + 3] * down);
            }
    }
}

template <int TYPE, int DIM, int NW, bool UNI, bool MX>
hipError_t chunk_pages(const AttendArgs& a, hipStream_t st) {
    static std::atomic<unsigned long long> done{0};
    const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(&attend_chunk_kernel<TYPE, DIM, NW, UNI, MX>), chunk_lds(DIM, NW), done);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((long long)a.tokens * a.group / (32 * NW) + a.requests), (unsigned)a.c.heads, (unsigned)a.splits);
    KernelTimer kt(MX ? KID_MX_ATTEND : KID_ATTEND, st);
    launch_timed(kt, (attend_chunk_kernel<TYPE, DIM, NW, UNI, MX>), grid, dim3(64 * NW), chunk_lds(DIM, NW), st, a);
    return hipGetLastError();
}
template <int TYPE, int DIM, int NW, bool MX>
hipError_t chunk_of(const AttendArgs& a, hipStream_t st) {
    return a.c.page_size % (1024 / DIM) == 0 ? chunk_pages<TYPE, DIM, NW, true, MX>(a, st) : chunk_pages<TYPE, DIM, NW, false, MX>(a, st);
}
template <int TYPE, bool MX>
hipError_t chunk_type(const AttendArgs& a, hipStream_t st) {
    if (a.c.dim <= 64) return chunk_of<TYPE, 64, 4, MX>(a, st);
    if constexpr (MX) {          // (others have blocks of 16 rows: attend_plan())
        if constexpr (TYPE != kF32) return chunk_of<TYPE, 128, 8, MX>(a, st);
        return hipErrorInvalidValue;
    } else {
        if (a.c.dim <= 128) return chunk_of<TYPE, 128, TYPE == kF32 ? 4 : 8, MX>(a, st);
        return chunk_of<TYPE, 256, 4, MX>(a, st);
    }
}
template <bool MX>
hipError_t chunk_any(const AttendArgs& a, hipStream_t st) {
    if (a.type == kF32) return chunk_type<kF32, MX>(a, st);
    if (a.type == kBF16) return chunk_type<kBF16, MX>(a, st);
    return chunk_type<kF16, MX>(a, st);
}

}  // namespace

hipError_t launch_attend_chunk(const AttendArgs& a, hipStream_t st) { return a.mx ? chunk_any<true>(a, st) : chunk_any<false>(a, st); }

}  // namespace int8t
