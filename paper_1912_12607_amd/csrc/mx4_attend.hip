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
// x in pieces of bf16, each the nearest to what the ones before leave: 8 bits of x each
template <int PARTS>
__device__ __forceinline__ void bf16_pieces(float x, __bf16 out[PARTS]) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        out[p] = (__bf16)x;
        x -= (float)out[p];
    }
}

// ------------------------------------------------------------------------------------------------
// Sixteen rows (tokens times heads of a group, in order) of one request and one head of the cache per block.  The request's keys are dealt
// out in shares of `share` to blocks and in each to RW waves, which run on their own, 32 keys at a time, the next 32 on their way
// meanwhile, and join their sums in LDS.
//   scores   S^T[key][row] = K Q^T (16 x 16 x 32 products): a lane has a quarter of a key's dims, its codes become bf16 with their block's power of two, exactly;
//   softmax  a lane's eight scores belong to one row; its unit m (p = 2^(s - m)) is shared by the row's four lanes and moves up when some lane's scores pass it far;
//   values   O^T[dim][row] = V^T P^T: S^T's layout is P^T's operand layout if the keys of a 32 are numbered (lane group, tile, i), so
//            nothing is exchanged; a lane loads DIM / 16 dims of eight keys and turns them in registers.
// bf16 has fp32's range, so that no scale leaves the codes; q and p are held in pieces of it: q exactly (bf16 1, fp16 2, fp32 3 pieces), p to 16 bits for bf16 and fp16
// tensors and to 24 for fp32 ones.
// UNI: the page size is a multiple of 16, whole tiles of 16 keys lie on a page and their address is scalar.
// ------------------------------------------------------------------------------------------------
template <int TYPE, int DIM, bool UNI, int RW>
__global__ __launch_bounds__(64 * RW, 2) void mx_attend_rows_kernel(const AttendArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int QP = TYPE == kF32 ? 3 : TYPE == kF16 ? 2 : 1, PP = TYPE == kF32 ? 3 : 2;      // pieces
    constexpr int CB = DIM / 16, KW = DIM / 32, VW = DIM == 256 ? 2 : 1;       // a lane's dims of a value; words of a key, of a value
    extern __shared__ __attribute__((aligned(1024))) float lds[];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n16 = lane & 15, kg = lane >> 4;
    // Heads first: an XCD has as few heads' keys in its L2 as can be, and blocks without rows, a few for each request, lie together.
    const int place = (int)(blockIdx.y * gridDim.x + blockIdx.x), group_of = div_by(place, a.by_heads);
    const int head = place - group_of * a.c.heads, split = (int)blockIdx.z, block = (int)gridDim.x - 1 - group_of;
    const int D = a.c.dim, NB = mx_blocks(D), RB = 16 * NB;

    const int b = tile_request(a, block, 16);
    const Request rq = request_of(a, b);
    const int nrows = rq.tokens * a.group;
    const long long tile = (long long)block - ((long long)a.starts[b] * a.group / 16 + b);
    if (tile < 0 || tile * 16 >= nrows) return;
    const int r0 = (int)tile * 16;
    const int heads = a.c.heads * a.group;

    // the block's keys: of those that its last row sees
    const int last_token = div_by(min(r0 + 15, nrows - 1), a.by_group);
    const int behind = rq.length - rq.new_tokens;               // keys before the new tokens
    const int seen_end = max(0, a.causal ? min(rq.length, behind + last_token + 1) : rq.length);
    const int all = max(0, a.causal ? min(rq.length, behind + div_by(r0, a.by_group) + 1) : rq.length);      // keys that all of its rows see
    const int from = (int)min((long long)split * a.share, (long long)seen_end), end = split + 1 == a.splits ? seen_end : min(from + a.share, seen_end);
    if (a.splits > 1 && from >= end && !(split == 0)) {              // nothing here: the joining pass looks at m alone
        if ((int)threadIdx.x < 16 && r0 + (int)threadIdx.x < nrows) {
            const int r = r0 + (int)threadIdx.x, t = div_by(r, a.by_group);
            a.part_ml[2 * ((size_t)split * a.tokens * heads + (size_t)(rq.token0 + t) * heads + head * a.group + (r - t * a.group))] = kNone;
        }
        return;
    }

    // this lane's row
    const int row = r0 + n16;
    const bool have = row < nrows;
    const int token = div_by(have ? row : r0, a.by_group), gh = (have ? row : r0) - token * a.group;
    const int limit = a.causal ? min(rq.length, behind + token + 1) : rq.length;

    // this wave's keys: whole 32s of the block's share
    const int steps = (end - from + 31) >> 5;
    const int s_from = steps * wave / RW, s_to = steps * (wave + 1) / RW;

    // ---- loader: a step's codes and scales as they are
    const uint8_t *const kq = reinterpret_cast<const uint8_t*>(a.c.kq), *const vq = reinterpret_cast<const uint8_t*>(a.c.vq);
    const uint8_t *const ksb = reinterpret_cast<const uint8_t*>(a.c.ks), *const vsb = reinterpret_cast<const uint8_t*>(a.c.vs);
    uint32_t kw[2][KW];                  // keys of the scores' operand: 16 t + n16
    uint32_t ke[2][DIM == 256 ? 2 : 1];  // their scales
    uint32_t vw[8][VW], ve[8];           // slot u = 4 t + i is key 16 t + 4 kg + i, of this lane's scores and values
    uint32_t okl;                        // bit u: the slot's key is in the cache, and before `end`
    int ids[2];
    // dims of a lane: DIM 64 16 kg .., 128 32 kg .., 256 128 i + 32 kg .. (beyond D: q is zero there, and nothing is stored)
    const auto key_dim = [&](int i) __attribute__((always_inline)) { return DIM == 64 ? 16 * kg : DIM == 128 ? 32 * kg : 128 * i + 32 * kg; };
    const int v_dim = n16 * CB < D ? n16 * CB : 0;
    const uint32_t v_at = (uint32_t)v_dim / 2, v_block = (uint32_t)v_dim / 32;
    auto page_ids = [&](int s) __attribute__((always_inline)) {
        if (!UNI) return;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int j = from + s * 32 + 16 * t;
            ids[t] = j < end ? rq.pages[div_by(j, a.c.by_page)] : -1;
        }
    };
    const auto fetch_key = [&](int t, const uint8_t* codes, const uint8_t* scales) __attribute__((always_inline)) {
        if constexpr (DIM == 64) {
            const int d = key_dim(0) < D ? key_dim(0) : 0;
            const uint2 w = *reinterpret_cast<const uint2*>(codes + d / 2);
            kw[t][0] = w.x; kw[t][1] = w.y;
            ke[t][0] = scales[d / 32];
        } else {
#pragma unroll
            for (int i = 0; i < KW / 4; ++i) {
                const int d = key_dim(i) < D ? key_dim(i) : 0;
                const uint4 w = *reinterpret_cast<const uint4*>(codes + d / 2);
                kw[t][4 * i] = w.x; kw[t][4 * i + 1] = w.y; kw[t][4 * i + 2] = w.z; kw[t][4 * i + 3] = w.w;
                ke[t][i] = scales[d / 32];
            }
        }
    };
    const auto fetch_value = [&](int u, const uint8_t* codes, const uint8_t* scales) __attribute__((always_inline)) {
        if constexpr (DIM == 64) vw[u][0] = *reinterpret_cast<const uint16_t*>(codes + v_at);
        else if constexpr (DIM == 128) vw[u][0] = *reinterpret_cast<const uint32_t*>(codes + v_at);
        else {
            const uint2 w = *reinterpret_cast<const uint2*>(codes + v_at);
            vw[u][0] = w.x; vw[u][VW - 1] = w.y;
        }
        ve[u] = scales[v_block];
    };
    auto fetch = [&](int s) __attribute__((always_inline)) {
        const int j0 = from + s * 32;
        okl = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int j = j0 + 16 * t;
            if (UNI) {
                const bool ok = (unsigned)ids[t] < (unsigned)a.c.pages;
                const int id = __builtin_amdgcn_readfirstlane(ok ? ids[t] : 0), in = ok ? j - div_by(j, a.c.by_page) * a.c.page_size : 0;
                const size_t place = ((size_t)id * a.c.heads + head) * a.c.page_size + in;
                fetch_key(t, kq + place * RB + (uint32_t)(n16 * RB), ksb + place * NB + (uint32_t)(n16 * NB));
#pragma unroll
                for (int i = 0; i < 4; ++i) fetch_value(4 * t + i, vq + place * RB + (uint32_t)((4 * kg + i) * RB), vsb + place * NB + (uint32_t)((4 * kg + i) * NB));
                if (ok) okl |= (j + 16 <= end ? 15u : (1u << min(4, max(0, end - j - 4 * kg))) - 1u) << (4 * t);
            } else {
                size_t place;
                key_place(a, rq, head, j + n16, end, &place);
                fetch_key(t, kq + place * RB, ksb + place * NB);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (key_place(a, rq, head, j + 4 * kg + i, end, &place)) okl |= 1u << (4 * t + i);
                    fetch_value(4 * t + i, vq + place * RB, vsb + place * NB);
                }
            }
        }
    };
    // q is requested first: its place is known before the keys' pages are
    ma_b8 qf[QP][KW];
    const float qscale = a.scale * kLog2e;
    {
        const T* qp = static_cast<const T*>(a.q) + (size_t)(rq.token0 + token) * a.q_token + (size_t)(head * a.group + gh) * a.q_head;
        float v[KW][8];
#pragma unroll
        for (int i = 0; i < KW; ++i) {
            const int d = key_dim(i / 4) + 8 * (i % 4);
            load8<TYPE>(qp + d, D - d, a.wide_q, v[i]);
        }
        if (s_from < s_to) {
            page_ids(s_from);
            fetch(s_from);
            page_ids(s_from + 1);
        }
#pragma unroll
        for (int i = 0; i < KW; ++i)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                __bf16 piece[QP];
                bf16_pieces<QP>(v[i][u], piece);
#pragma unroll
                for (int p = 0; p < QP; ++p) qf[p][i][u] = piece[p];
            }
    }

    float m = kNone, unit = 0.0f;                // the largest score when the unit last moved; the unit: m, or 0 where nothing was seen yet
    float l = 0.0f;                              // sum of this lane's p
    tk_f4 o[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) o[c] = tk_f4{0.f, 0.f, 0.f, 0.f};

    for (int s = s_from; s < s_to; ++s) {
        const int j0 = from + s * 32;
        // this step's operands leave the loader's registers (scores: at once; values: as they are), then the next step's are requested
        float x[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            tk_f4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                const float scale = mx_power(ke[t][DIM == 256 ? i / 4 : 0]);
                const uint4 f = make_uint4(codes_bf16<0>(kw[t][i], scale), codes_bf16<1>(kw[t][i], scale), codes_bf16<2>(kw[t][i], scale), codes_bf16<3>(kw[t][i], scale));
                const ma_b8 kf = __builtin_bit_cast(ma_b8, f);
#pragma unroll
                for (int p = 0; p < QP; ++p) sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[p][i], sc, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * t + i] = sc[i] * qscale;
        }
        uint32_t vc[8][VW], vs[8];
        const uint32_t in = okl;
        bool bad = false;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            vs[u] = ve[u];
            bad = bad || vs[u] >= 253u;
#pragma unroll
            for (int c = 0; c < VW; ++c) vc[u][c] = vw[u][c];
        }
        if (s + 1 < s_to) {
            fetch(s + 1);
            page_ids(s + 2);
        }
        if (j0 + 32 > all || __any(in != 255u)) {            // some keys are not there, or not for all rows
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const bool there = ((in >> u) & 1u) != 0;
                vs[u] = there ? vs[u] : 0u;
                x[u] = there && j0 + 16 * (u >> 2) + 4 * kg + (u & 3) < limit ? x[u] : kNone;
            }
        }
        float top = kNone;
#pragma unroll
        for (int u = 0; u < 8; ++u) top = fmaxf(top, x[u]);
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
            x[u] = __builtin_amdgcn_exp2f(x[u] - unit);
            l += x[u];
        }
        // Values that are not finite (some lane has a block of them) go into p of the rows that see them, and become zeros for the others.
        if (__any(bad)) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const unsigned long long lanes = __ballot(vs[u] >= 253u) >> (16 * kg) & 0xffffull;
                if (lanes && x[u] != 0.0f) x[u] = NAN;
                if (lanes) vs[u] = 0u;
            }
        }
        ma_b8 pf[PP];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            __bf16 piece[PP];
            bf16_pieces<PP>(x[u], piece);
#pragma unroll
            for (int p = 0; p < PP; ++p) pf[p][u] = piece[p];
        }
        // values: pairs of dims of a key, then pairs of keys of a dim
        float scale[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) scale[u] = __uint_as_float(vs[u] << 23);
#pragma unroll
        for (int c2 = 0; c2 < CB / 2; ++c2) {
            uint32_t w[8], f[2][4];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t word = vc[u][c2 / 4];
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
    float mm = sm[jr], total = 0.0f, w[RW];
#pragma unroll
    for (int i = 1; i < RW; ++i) mm = fmaxf(mm, sm[16 * i + jr]);
#pragma unroll
    for (int i = 0; i < RW; ++i) {
        const float mi = sm[16 * i + jr];
        w[i] = mi == kNone ? 0.0f : __builtin_amdgcn_exp2f(mi - mm);
        total += w[i] * sl[16 * i + jr];
    }
    const int jt = div_by(r0 + jr, a.by_group), jg = (r0 + jr) - jt * a.group;
    const size_t out_row = (size_t)(rq.token0 + jt) * heads + head * a.group + jg;
    const bool whole = a.splits == 1;
    const size_t part_row = (size_t)split * a.tokens * heads + out_row;
    const float by = whole ? per_sum(total) : 1.0f;
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

template <int TYPE, int DIM, bool UNI, int RW>
hipError_t rows_dim(const AttendArgs& a, hipStream_t st) {
    constexpr int LDS = RW * 16 * (DIM + 4 + 2) * 4;
    static std::atomic<unsigned long long> done{0};
    const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(&mx_attend_rows_kernel<TYPE, DIM, UNI, RW>), LDS, done);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((long long)a.tokens * a.group / 16 + a.requests), (unsigned)a.c.heads, (unsigned)a.splits);
    KernelTimer kt(KID_MX_ATTEND, st);
    launch_timed(kt, (mx_attend_rows_kernel<TYPE, DIM, UNI, RW>), grid, dim3(64 * RW), LDS, st, a);
    return hipGetLastError();
}
template <int TYPE, bool UNI, int RW>
hipError_t rows_of(const AttendArgs& a, hipStream_t st) {
    return a.c.dim <= 64 ? rows_dim<TYPE, 64, UNI, RW>(a, st) : a.c.dim <= 128 ? rows_dim<TYPE, 128, UNI, RW>(a, st) : rows_dim<TYPE, 256, UNI, RW>(a, st);
}
template <int TYPE>
hipError_t rows_type(const AttendArgs& a, hipStream_t st) {
    const bool uni = a.c.page_size % 16 == 0;
    return a.waves == 8 ? (uni ? rows_of<TYPE, true, 8>(a, st) : rows_of<TYPE, false, 8>(a, st)) : (uni ? rows_of<TYPE, true, 4>(a, st) : rows_of<TYPE, false, 4>(a, st));
}

}  // namespace

hipError_t launch_mx_attend_rows(const AttendArgs& a, hipStream_t st) {
    if (a.type == kF32) return rows_type<kF32>(a, st);
    if (a.type == kBF16) return rows_type<kBF16>(a, st);
    return rows_type<kF16>(a, st);
}

}  // namespace int8t
