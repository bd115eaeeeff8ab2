// Attention of many new tokens of a request (chunks of a prompt) over the paged cache: the formulas and the joining of shares of
// token_attend.hip.
//
// A block has 32 NW rows (tokens times heads of a group, in order) of one request and head of the cache, a wave 32 of them; the keys pass
// by in tiles of 64.  While one tile is multiplied, the next one's codes, which were loaded a tile ahead, become fp16 (exactly) in LDS,
// once for all waves, and the one after it is loaded.
//   scores   S^T[key][row] = K Q^T in products of 32 x 32 x 16: a lane's 16 scores of 32 keys belong to one row, so maximum and sum need
//            one exchange between the halves of the wave;
//   values   O^T[dim][row] = V^T P^T: the scores' layout is P^T's operand layout with the keys in the order that the transposing LDS read
//            of V (rows of keys, as they came) delivers: p never leaves its lane.
// Bound by the vector units: 9 to 10 operations per score, of which the exponential counts for four, against 256 multiply-adds of the
// matrix units (DIM 128).
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

constexpr int chunk_lds(int DIM) { return 2 * (2 * TK * DIM * 2 + 3 * TK * 4); }

template <int TYPE, int DIM, int NW>
__global__ __launch_bounds__(64 * NW, DIM == 256 ? 1 : 2) void attend_chunk_kernel(const AttendArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int PARTS = TYPE == kF32 ? 2 : 1, NT = 64 * NW, ROWS = 32 * NW;
    constexpr int QS = DIM / 16, DT = DIM / 32;                // steps of the scores' products; tiles of dims
    constexpr int CH = 4 * DIM;                                // 16-byte pieces of a tile of codes
    constexpr bool APART = CH < NT;                            // keys' and values' pieces to different threads
    constexpr int NP = APART ? 1 : CH / NT;                    // pieces of either tensor per thread
    extern __shared__ __attribute__((aligned(1024))) uint4 lds[];
    uint4* const sk = lds;                                     // [2][TK][DIM] fp16
    uint4* const sv = lds + 2 * TK * DIM / 8;
    float* const sc = reinterpret_cast<float*>(lds + 4 * TK * DIM / 8);      // [2][3][TK]: key scales, value scales, 0 or -infinity

    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n32 = lane & 31, half = lane >> 5;
    const int head = (int)blockIdx.y, split = (int)blockIdx.z;
    const int D = a.c.dim;

    const int b = tile_request(a, (int)blockIdx.x, ROWS);
    const Request rq = request_of(a, b);
    const int nrows = rq.tokens * a.group;
    const long long tile = (long long)blockIdx.x - ((long long)a.starts[b] * a.group / ROWS + b);
    if (tile < 0 || tile * ROWS >= nrows) return;
    const int r0 = (int)tile * ROWS;
    const int row = r0 + 32 * wave + n32;
    const bool have = row < nrows;
    const int token = (have ? row : r0) / a.group, gh = (have ? row : r0) - token * a.group;
    const int behind = rq.length - rq.new_tokens;               // keys before the new tokens
    const int limit = !have ? 0 : a.causal ? min(rq.length, behind + token + 1) : rq.length;
    // keys that the block's last row sees, and those that all of its rows see
    const int last_token = min(r0 + ROWS - 1, nrows - 1) / a.group;
    const int end = max(0, a.causal ? min(rq.length, behind + last_token + 1) : rq.length);
    const int all = max(0, a.causal ? min(rq.length, behind + r0 / a.group + 1) : rq.length);
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
        m = fmaxf(m, __shfl_xor(m, 32, kWave));
        float back;
        float up = row_scale(m, &back);
        // the scores' factor is kept positive (the maximum is taken before it): a negative scale goes into q, and for none q is zero
        qscale = fmaxf(back * (fabsf(a.scale) * kLog2e), 1e-37f);
        if (a.scale < 0.0f) up = -up;
        if (a.scale == 0.0f) up = 0.0f;
#pragma unroll
        for (int i = 0; i < QS; ++i)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float t = v[i][u] * up;
                _Float16 first = (_Float16)t, rest;
                if (PARTS == 2) {
                    two_pieces(t, &first, &rest);
                    qf[PARTS - 1][i][u] = rest;
                }
                qf[0][i][u] = first;
            }
    }

    // ---- loader: this thread's pieces, piece p is 16 dims of a key
    const bool loads_k = !APART || tid < CH, loads_v = !APART || (tid >= CH && tid < 2 * CH);
    const int pt = APART ? tid % CH : tid;
    uint4 rk[NP], rv[NP];
    float rks[NP], rvs[NP];
    bool rok[NP];
    int ids[NP];
    auto key_of = [&](int p) { return (pt + p * NT) / (DIM / 16); };
    auto page_ids = [&](int t) {                               // pages of tile t's keys
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int j = t * TK + key_of(p);
            ids[p] = j < end ? rq.pages[div_by(j, a.c.by_page)] : -1;
        }
    };
    auto fetch = [&](int t) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int j = t * TK + key_of(p), d = ((pt + p * NT) % (DIM / 16)) * 16;
            rok[p] = (unsigned)ids[p] < (unsigned)a.c.pages;
            const size_t place = rok[p] ? ((size_t)ids[p] * a.c.heads + head) * a.c.page_size + (j - div_by(j, a.c.by_page) * a.c.page_size) : 0;
            const size_t at = place * D + (d < D ? d : 0);      // (beyond D: q is zero there, and nothing is stored)
            if (loads_k) {
                rk[p] = *reinterpret_cast<const uint4*>(a.c.kq + at);
                rks[p] = a.c.ks[place];
            }
            if (loads_v) {
                rv[p] = *reinterpret_cast<const uint4*>(a.c.vq + at);
                rvs[p] = a.c.vs[place];
            }
        }
    };
    auto expand = [](const uint4& c, uint4* lo, uint4* hi) {
        const uint32_t w[4] = {c.x ^ 0x80808080u, c.y ^ 0x80808080u, c.z ^ 0x80808080u, c.w ^ 0x80808080u};
        *lo = make_uint4(codes_f16<kLowPair>(w[0]), codes_f16<kHighPair>(w[0]), codes_f16<kLowPair>(w[1]), codes_f16<kHighPair>(w[1]));
        *hi = make_uint4(codes_f16<kLowPair>(w[2]), codes_f16<kHighPair>(w[2]), codes_f16<kLowPair>(w[3]), codes_f16<kHighPair>(w[3]));
    };
    auto stage = [&](int buf) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int key = key_of(p), g = ((pt + p * NT) % (DIM / 16)) * 2;
            uint4 lo, hi;
            float* const s = sc + buf * 3 * TK;
            if (loads_k) {
                expand(rk[p], &lo, &hi);
                sk[buf * (TK * DIM / 8) + k_slot<DIM>(key, g)] = lo;
                sk[buf * (TK * DIM / 8) + k_slot<DIM>(key, g + 1)] = hi;
                if (g == 0) {
                    s[key] = rok[p] ? rks[p] : 0.0f;
                    s[2 * TK + key] = rok[p] ? 0.0f : kNone;
                }
            }
            if (loads_v) {
                expand(rv[p], &lo, &hi);
                sv[buf * (TK * DIM / 8) + v_slot<DIM>(key, g)] = lo;
                sv[buf * (TK * DIM / 8) + v_slot<DIM>(key, g + 1)] = hi;
                if (g == 0) s[TK + key] = rok[p] ? rvs[p] : 0.0f;
            }
        }
    };

    float m = kNone, l = 0.0f, ref = 0.0f, unit = 0.0f;       // maximum (times qscale); sum of this lane's p; largest value scale so far, 2^15 / it
    tk_f16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[d][v] = 0.0f;

    if (t_from < t_to) {
        page_ids(t_from);
        fetch(t_from);
        page_ids(t_from + 1);
        stage(t_from & 1);
        fetch(t_from + 1);
        page_ids(t_from + 2);
    }
    for (int t = t_from; t < t_to; ++t) {
        const int buf = t & 1;
        __syncthreads();                          // the tile is in LDS; the other buffer has been read by all
        if (t + 1 < t_to) {
            stage(buf ^ 1);
            fetch(t + 2);
            page_ids(t + 3);
        }
        const float* const s = sc + buf * 3 * TK;
        // scores
        tk_f16 x[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
            for (int v = 0; v < 16; ++v) x[kt][v] = 0.0f;
#pragma unroll
            for (int i = 0; i < QS; ++i) {
                const tk_h8 kf = __builtin_bit_cast(tk_h8, sk[buf * (TK * DIM / 8) + k_slot<DIM>(kt * 32 + n32, 2 * i + half)]);
#pragma unroll
                for (int p = 0; p < PARTS; ++p) x[kt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[p][i], x[kt], 0, 0, 0);
            }
        }
        // times the keys' scales; the tile's last keys and those behind a row's own
        const bool masked = (t + 1) * TK > all || __any(s[2 * TK + lane] != 0.0f);
        float top = kNone;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const tk_f4 ks = *reinterpret_cast<const tk_f4*>(s + kt * 32 + 8 * q + 4 * half);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[kt][4 * q + i] *= ks[i];
            }
        if (masked) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const tk_f4 none = *reinterpret_cast<const tk_f4*>(s + 2 * TK + kt * 32 + 8 * q + 4 * half);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (none[i] != 0.0f || t * TK + kt * 32 + 8 * q + 4 * half + i >= limit) x[kt][4 * q + i] = kNone;
                }
        }
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int v = 0; v < 16; ++v) top = fmaxf(top, x[kt][v]);
        top = fmaxf(top, __shfl_xor(top, 32, kWave)) * qscale;
        const float vmax = wave_max(s[TK + lane]);
        if (vmax > ref || __any(top > m)) {
            const float m1 = fmaxf(m, top), ref1 = fmaxf(fmaxf(vmax, ref), 1e-30f);
            const float keep = m == kNone ? 0.0f : __builtin_amdgcn_exp2f(m - m1);
            const float by = keep * (ref / ref1);
            l *= keep;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[d][v] *= by;
            m = m1;
            ref = ref1;
            unit = 32768.0f / ref1;
        }
        // p, times the values' scales in units of 2^-15 of the largest
        const float base = m == kNone ? 0.0f : -m;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            tk_h8 pf[PARTS][2];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const tk_f4 vs = *reinterpret_cast<const tk_f4*>(s + TK + kt * 32 + 8 * q + 4 * half);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[kt][4 * q + i], qscale, base));
                    l += p;
                    const float w = p * (vs[i] * unit);
                    _Float16 first = (_Float16)w, rest;
                    if (PARTS == 2) {
                        two_pieces(w, &first, &rest);
                        pf[PARTS - 1][q >> 1][4 * (q & 1) + i] = rest;
                    }
                    pf[0][q >> 1][4 * (q & 1) + i] = first;
                }
            }
            // values: 16 keys at a time; slot 8 half + i of the product is key 4 half + i (i < 4) or 8 + 4 half + i - 4
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    // a group of 16 lanes reads four keys by 16 dims: lane j points at key j / 4, dims 4 (j % 4) .. + 3, and gets dim j of the four
                    const int g4 = (lane >> 4) & 1, j = lane & 15;
                    const int key = kt * 32 + u * 16 + 4 * half + (j >> 2), gran = d * 4 + g4 * 2 + ((j & 3) >> 1);
                    const uint4* const at = sv + buf * (TK * DIM / 8);
                    const uintptr_t p0 = (uintptr_t)(uint32_t)(size_t)(at + v_slot<DIM>(key, gran)) + 8 * (j & 1);
                    const uintptr_t p1 = (uintptr_t)(uint32_t)(size_t)(at + v_slot<DIM>(key + 8, gran)) + 8 * (j & 1);
                    const tc_s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tc_lds)p0), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tc_lds)p1);
                    typedef short tc_s8 __attribute__((ext_vector_type(8)));
                    const tk_h8 vf = __builtin_bit_cast(tk_h8, tc_s8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pf[p][u], o[d], 0, 0, 0);
                }
        }
    }

    l += __shfl_xor(l, 32, kWave);
    if (!have) return;
    const int heads = a.c.heads * a.group;
    const size_t out_row = (size_t)(rq.token0 + token) * heads + head * a.group + gh;
    const float out_unit = ref * (1.0f / 32768.0f);
    if (a.splits == 1) {
        const float by = l > 0.0f ? out_unit / l : 0.0f;
        if (a.lse && half == 0) a.lse[out_row] = l > 0.0f ? (m + __log2f(l)) * (1.0f / kLog2e) : kNone;
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
                        make_float4(o[d][4 * q] * out_unit, o[d][4 * q + 1] * out_unit, o[d][4 * q + 2] * out_unit, o[d][4 * q + 3] * out_unit);
            }
    }
}

template <int TYPE, int DIM, int NW>
hipError_t chunk_of(const AttendArgs& a, hipStream_t st) {
    static std::atomic<unsigned long long> done{0};
    const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(&attend_chunk_kernel<TYPE, DIM, NW>), chunk_lds(DIM), done);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((long long)a.tokens * a.group / (32 * NW) + a.requests), (unsigned)a.c.heads, (unsigned)a.splits);
    KernelTimer kt(KID_ATTEND, st);
    launch_timed(kt, (attend_chunk_kernel<TYPE, DIM, NW>), grid, dim3(64 * NW), chunk_lds(DIM), st, a);
    return hipGetLastError();
}
template <int TYPE>
hipError_t chunk_type(const AttendArgs& a, hipStream_t st) {
    const bool many = a.rows == 256;
    if (a.c.dim <= 64) return many ? chunk_of<TYPE, 64, 8>(a, st) : chunk_of<TYPE, 64, 4>(a, st);
    if (a.c.dim <= 128) return many ? chunk_of<TYPE, 128, 8>(a, st) : chunk_of<TYPE, 128, 4>(a, st);
    return chunk_of<TYPE, 256, 4>(a, st);
}

}  // namespace

hipError_t launch_attend_chunk(const AttendArgs& a, hipStream_t st) {
    if (a.type == kF32) return chunk_type<kF32>(a, st);
    if (a.type == kBF16) return chunk_type<kBF16>(a, st);
    return chunk_type<kF16>(a, st);
}

}  // namespace int8t
