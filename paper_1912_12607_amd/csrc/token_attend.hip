// Attention of new tokens over a paged cache in 8 bits:
//   o_i = sum_j p_ij vs_j vq_j / sum_j p_ij,   p_ij = exp(scale ks_j (q_i . kq_j)),   j < length (causal: up to the token's own place).
#include "token_attend.h"

namespace int8t {
namespace {

// ------------------------------------------------------------------------------------------------
// Sixteen rows (tokens times heads of a group, in order) of one request and one head of the cache per block.  The request's keys are dealt
// out in shares of `share` to blocks and in each to RW waves, which run on their own, 32 keys at a time, the next 32 on their way
// meanwhile, and join their sums in LDS.
//   scores   S^T[key][row] = K Q^T (16 x 16 x 32 products): a lane loads 16 bytes of a key, codes become fp16 exactly;
//   softmax  a lane's eight scores belong to one row; its unit (RowUnit) is shared by the row's four lanes and changes when some lane needs it;
//   values   O^T[dim][row] = V^T P^T: S^T's layout is P^T's operand layout if the keys of a 32 are numbered (lane group, tile, i), so
//            nothing is exchanged; a lane loads DIM / 16 bytes of eight keys and turns them in registers.
// PARTS = 2 (fp32): q and p in two fp16 pieces each.  UNI: the page size is a multiple of 16, whole tiles of 16 keys lie on a page and their
// address is scalar.  Bound by memory, codes and scales read once: the next token of 64 requests over 1 to 8192 keys, 8 heads of 128, 139 us with the
// joining pass (640 MB: 4.8 TB/s, a large copy 5.1).  A request alone, by its few blocks' arithmetic: 1021 keys 12 us, 5.8 and 1.7 for each 32 keys of a wave.
// ------------------------------------------------------------------------------------------------
// RW waves: four (two blocks on a compute unit, one at work while the other starts or ends), or eight where there are few blocks.
template <int TYPE, int DIM, bool UNI, int RW>
__global__ __launch_bounds__(64 * RW, 2) void attend_rows_kernel(const AttendArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int PARTS = TYPE == kF32 ? 2 : 1, KL = DIM / 64, CB = DIM / 16;      // 16-byte loads of a key; bytes of a value row per lane
    extern __shared__ __attribute__((aligned(1024))) float lds[];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n16 = lane & 15, kg = lane >> 4;
    // Heads first: an XCD has as few heads' keys in its L2 as can be, and blocks without rows, a few for each request, lie together.  (Tiles first: 16
    // requests of 16 tokens over 2048 keys, 8 heads of 256, 152 us, not 84; the next token of 64 requests over 4096 keys, 8 of 128, 121, not 107.)
    const int place = (int)(blockIdx.y * gridDim.x + blockIdx.x), group_of = div_by(place, a.by_heads);
    const int head = place - group_of * a.c.heads, split = (int)blockIdx.z, block = (int)gridDim.x - 1 - group_of;
    const int D = a.c.dim;

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
    uint4 kw[2][KL];                     // keys of the scores' operand: 16 t + n16
    uint32_t vw[8][CB / 4];              // slot u = 4 t + i is key 16 t + 4 kg + i, of this lane's scores and values
    float ks[8], vs[8];
    uint32_t okl;                        // bit u: the slot's key is in the cache, and before `end`
    int ids[2];
    uint32_t k_at[KL];                   // (beyond D: q is zero there, and nothing is stored)
#pragma unroll
    for (int i = 0; i < KL; ++i) k_at[i] = (uint32_t)(i * 64 + kg * 16 < D ? i * 64 + kg * 16 : 0);
    const uint32_t v_at = (uint32_t)(n16 * CB < D ? n16 * CB : 0), key_row = (uint32_t)(n16 * D), value_row = (uint32_t)(4 * kg * D) + v_at;
    const bool quads = a.c.page_size % 4 == 0;
    auto page_ids = [&](int s) __attribute__((always_inline)) {
        if (!UNI) return;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int j = from + s * 32 + 16 * t;
            ids[t] = j < end ? rq.pages[div_by(j, a.c.by_page)] : -1;
        }
    };
    auto fetch = [&](int s) __attribute__((always_inline)) {
        const int j0 = from + s * 32;
        okl = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (UNI) {
                const int j = j0 + 16 * t;
                const bool ok = (unsigned)ids[t] < (unsigned)a.c.pages;
                const int id = __builtin_amdgcn_readfirstlane(ok ? ids[t] : 0), in = ok ? j - div_by(j, a.c.by_page) * a.c.page_size : 0;
                const size_t place = ((size_t)id * a.c.heads + head) * a.c.page_size + in;
                const int8_t *kq = a.c.kq + place * D, *vq = a.c.vq + place * D;
#pragma unroll
                for (int i = 0; i < KL; ++i) kw[t][i] = *reinterpret_cast<const uint4*>(kq + (key_row + k_at[i]));
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < CB / 4; ++c) vw[4 * t + i][c] = reinterpret_cast<const uint32_t*>(vq + (value_row + (uint32_t)(i * D)))[c];
                const float4 k4 = *reinterpret_cast<const float4*>(a.c.ks + place + 4u * kg), v4 = *reinterpret_cast<const float4*>(a.c.vs + place + 4u * kg);
                ks[4 * t] = k4.x; ks[4 * t + 1] = k4.y; ks[4 * t + 2] = k4.z; ks[4 * t + 3] = k4.w;
                vs[4 * t] = v4.x; vs[4 * t + 1] = v4.y; vs[4 * t + 2] = v4.z; vs[4 * t + 3] = v4.w;
                if (ok) okl |= (j + 16 <= end ? 15u : (1u << min(4, max(0, end - j - 4 * kg))) - 1u) << (4 * t);
            } else {
                size_t place;
                key_place(a, rq, head, j0 + 16 * t + n16, end, &place);
#pragma unroll
                for (int i = 0; i < KL; ++i) kw[t][i] = *reinterpret_cast<const uint4*>(a.c.kq + place * D + k_at[i]);
                const int j = j0 + 16 * t + 4 * kg;
                if (quads) {                     // four neighbouring keys lie on a page: one look at the table for them
                    const bool ok = key_place(a, rq, head, j, end, &place);
                    if (ok) okl |= ((1u << min(4, end - j)) - 1u) << (4 * t);
                    const float4 k4 = *reinterpret_cast<const float4*>(a.c.ks + place), v4 = *reinterpret_cast<const float4*>(a.c.vs + place);
                    ks[4 * t] = k4.x; ks[4 * t + 1] = k4.y; ks[4 * t + 2] = k4.z; ks[4 * t + 3] = k4.w;
                    vs[4 * t] = v4.x; vs[4 * t + 1] = v4.y; vs[4 * t + 2] = v4.z; vs[4 * t + 3] = v4.w;
                    const int8_t* const vq = a.c.vq + place * D + v_at;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int c = 0; c < CB / 4; ++c) vw[4 * t + i][c] = reinterpret_cast<const uint32_t*>(vq + i * D)[c];
                    continue;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (key_place(a, rq, head, j + i, end, &place)) okl |= 1u << (4 * t + i);
                    ks[4 * t + i] = a.c.ks[place];
                    vs[4 * t + i] = a.c.vs[place];
#pragma unroll
                    for (int c = 0; c < CB / 4; ++c) vw[4 * t + i][c] = reinterpret_cast<const uint32_t*>(a.c.vq + place * D + v_at)[c];
                }
            }
        }
    };
    // q is requested first: its place is known before the keys' pages are
    tk_h8 qf[PARTS][2 * KL];
    float qscale;
    {
        const T* qp = static_cast<const T*>(a.q) + (size_t)(rq.token0 + token) * a.q_token + (size_t)(head * a.group + gh) * a.q_head;
        float v[2 * KL][8];
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * KL; ++i) {
            const int d = (i >> 1) * 64 + kg * 16 + (i & 1) * 8;
            load8<TYPE>(qp + d, D - d, a.wide_q, v[i]);
        }
        if (s_from < s_to) {
            page_ids(s_from);
            fetch(s_from);
            page_ids(s_from + 1);
        }
#pragma unroll
        for (int i = 0; i < 2 * KL; ++i)
#pragma unroll
            for (int u = 0; u < 8; ++u) m = fmaxf(m, fabsf(v[i][u]));
        m = halves_max(rows16_max(m));
        float back;
        float up = row_scale(m, &back);
        qscale = score_scale(a.scale, back, &up);
#pragma unroll
        for (int i = 0; i < 2 * KL; ++i)
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

    RowUnit unit;
    float l = 0.0f;                              // sum of this lane's p
    tk_f4 o[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) o[c] = tk_f4{0.f, 0.f, 0.f, 0.f};

    for (int s = s_from; s < s_to; ++s) {
        const int j0 = from + s * 32;
        // this step's operands leave the loader's registers as fp16 (scores: at once; values: as they are), then the next step's are requested
        tk_f4 sc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            sc[t] = tk_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KL; ++i) {
                const uint32_t w[4] = {kw[t][i].x ^ 0x80808080u, kw[t][i].y ^ 0x80808080u, kw[t][i].z ^ 0x80808080u, kw[t][i].w ^ 0x80808080u};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 f = make_uint4(codes_f16<kLowPair>(w[2 * h]), codes_f16<kHighPair>(w[2 * h]), codes_f16<kLowPair>(w[2 * h + 1]),
                                               codes_f16<kHighPair>(w[2 * h + 1]));
                    const tk_h8 kf = __builtin_bit_cast(tk_h8, f);
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[p][2 * i + h], sc[t], 0, 0, 0);
                }
            }
        }
        uint32_t vc[8][CB / 4];
        float kc[8], vsc[8];
        const uint32_t in = okl;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            kc[u] = ks[u];
            vsc[u] = vs[u];
#pragma unroll
            for (int c = 0; c < CB / 4; ++c) vc[u][c] = vw[u][c] ^ 0x80808080u;
        }
        if (s + 1 < s_to) {
            fetch(s + 1);
            page_ids(s + 2);
        }
        float x[8], top = kNone, scale = 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = sc[u >> 2][u & 3] * kc[u];
        if (j0 + 32 > all || __any(in != 255u)) {            // some keys are not there, or not for all rows
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const bool there = ((in >> u) & 1u) != 0;
                vsc[u] = there ? vsc[u] : 0.0f;
                x[u] = there && j0 + 16 * (u >> 2) + 4 * kg + (u & 3) < limit ? x[u] : kNone;
            }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            top = fmaxf(top, x[u]);
            scale = fmaxf(scale, fabsf(vsc[u]));
        }
        top *= qscale;
        if (__any(top > unit.room || scale > unit.vs)) {
            top = halves_max(rows16_max(top));
            if (unit.unknown(top, scale)) {
                float weight = kNone;
#pragma unroll
                for (int u = 0; u < 8; ++u) weight = fmaxf(weight, x[u] * qscale + RowUnit::log_of(vsc[u]));
                const float by = unit.set(top, halves_max(rows16_max(weight)));
                l *= by;
#pragma unroll
                for (int d = 0; d < CB; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[d][r] *= by;
            }
        }
        float largest = 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u], qscale, unit.c));
            l += p;
            x[u] = weight_of(p, vsc[u]);
            largest = fmaxf(largest, fabsf(x[u]));
        }
        if (RowUnit::large(largest, l)) {
            const float by = unit.lower(halves_max(rows16_max(largest)), halves_max(rows16_max(l)));
            l *= by;
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] *= by;
#pragma unroll
            for (int d = 0; d < CB; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[d][r] *= by;
        }
        tk_h8 pf[PARTS];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            _Float16 first = (_Float16)x[u], rest;
            if (PARTS == 2) {
                two_pieces(x[u], &first, &rest);
                pf[PARTS - 1][u] = rest;
            }
            pf[0][u] = first;
        }
        // values: pairs of keys interleaved, two bytes of a dim at a time under 0x64
#pragma unroll
        for (int c4 = 0; c4 < CB / 4; ++c4) {
            uint32_t f[4][4];        // [byte of the word][pair of keys]
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t lo = __builtin_amdgcn_perm(vc[2 * u + 1][c4], vc[2 * u][c4], 0x05010400u), hi = __builtin_amdgcn_perm(vc[2 * u + 1][c4], vc[2 * u][c4], 0x07030602u);
                f[0][u] = codes_f16<kLowPair>(lo);
                f[1][u] = codes_f16<kHighPair>(lo);
                f[2][u] = codes_f16<kLowPair>(hi);
                f[3][u] = codes_f16<kHighPair>(hi);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const tk_h8 vf = __builtin_bit_cast(tk_h8, make_uint4(f[c][0], f[c][1], f[c][2], f[c][3]));
#pragma unroll
                for (int p = 0; p < PARTS; ++p) o[c4 * 4 + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[p], o[c4 * 4 + c], 0, 0, 0);
            }
        }
    }
    l = halves_sum(rows16_sum(l));
    float down;
    const float m = normalised(unit.c, &l, &down);

    // the waves' sums, in LDS: [wave][row][DIM + 4], in units of the values.  A lane has CB neighbouring dims of its row for each r.
    float* const sm = lds;
    float* const sl = sm + 16 * RW;
    float* const so = sl + 16 * RW;
    constexpr int PITCH = DIM + 4;
    if (kg == 0) {
        sm[wave * 16 + n16] = m;
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

// Joins the shares of a row: 16 lanes each, which look at 16 shares' maxima and sums at a time.
template <int TYPE>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    const size_t rows = (size_t)a.tokens * a.c.heads * a.group;
    const size_t row = ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 16 + ((int)threadIdx.x >> 4);      // (y: a launch has fewer than 2^32 threads a dimension)
    const int l = (int)threadIdx.x & 15, D = a.c.dim;
    const bool have = row < rows;                       // (all lanes stay for the exchanges)
    const size_t r = have ? row : 0;
    float m = kNone, total = 0.0f;
    int end = 0;                                        // behind the last share that saw keys
    for (int s = l; s < a.splits; s += 16) {
        const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * (s * rows + r));
        if (ml.x == kNone) continue;
        end = s + 1;
        const float m1 = fmaxf(m, ml.x);
        total = total * __builtin_amdgcn_exp2f(m - m1) + __builtin_amdgcn_exp2f(ml.x - m1) * ml.y;      // (m = -infinity: total is 0)
        m = m1;
    }
#pragma unroll
    for (int o = 1; o < 16; o *= 2) {
        const float m2 = __shfl_xor(m, o, kWave), t2 = __shfl_xor(total, o, kWave), m1 = fmaxf(m, m2);
        if (m1 != kNone) total = total * __builtin_amdgcn_exp2f(m - m1) + t2 * __builtin_amdgcn_exp2f(m2 - m1);
        else total += t2;                        // (nothing, or NaN)
        m = m1;
        end = max(end, __shfl_xor(end, o, kWave));
    }
    if (!have) return;
    const float by = per_sum(total);
    if (l == 0 && a.lse) a.lse[row] = log_of_sum(m, total);
    for (int d = l * 8; d < D; d += 128) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = 0; s < end; ++s) {
            const float ms = a.part_ml[2 * (s * rows + row)];
            // (a share between others of which nothing was seen may have written no sums: they are read -- the memory is there -- and not used)
            float p[8];
            load8<kF32>(a.part_o + (s * rows + row) * D + d, 8, true, p);
            const float w = __builtin_amdgcn_exp2f(ms - m) * by;
            if (ms != kNone) {
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] += w * p[u];
            }
        }
        store8<TYPE>(static_cast<T*>(a.out) + row * D + d, 8, true, v);
    }
}

template <int TYPE, int DIM, bool UNI, int RW>
hipError_t rows_dim(const AttendArgs& a, hipStream_t st) {
    constexpr int LDS = RW * 16 * (DIM + 4 + 2) * 4;
    static std::atomic<unsigned long long> done{0};
    const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(&attend_rows_kernel<TYPE, DIM, UNI, RW>), LDS, done);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((long long)a.tokens * a.group / 16 + a.requests), (unsigned)a.c.heads, (unsigned)a.splits);
    KernelTimer kt(KID_ATTEND, st);
    launch_timed(kt, (attend_rows_kernel<TYPE, DIM, UNI, RW>), grid, dim3(64 * RW), LDS, st, a);
    return hipGetLastError();
}
template <int TYPE, bool UNI, int RW>
hipError_t rows_of(const AttendArgs& a, hipStream_t st) {
    return a.c.dim <= 64 ? rows_dim<TYPE, 64, UNI, RW>(a, st) : a.c.dim <= 128 ? rows_dim<TYPE, 128, UNI, RW>(a, st) : rows_dim<TYPE, 256, UNI, RW>(a, st);
}

template <int TYPE>
hipError_t attend_type(const AttendArgs& a, hipStream_t st) {
    if (a.rows > 16) {
        const hipError_t e = launch_attend_chunk(a, st);
        if (e != hipSuccess) return e;
    } else {
        const bool uni = a.c.page_size % 16 == 0;
        const hipError_t e = a.waves == 8 ? (uni ? rows_of<TYPE, true, 8>(a, st) : rows_of<TYPE, false, 8>(a, st))
                                          : (uni ? rows_of<TYPE, true, 4>(a, st) : rows_of<TYPE, false, 4>(a, st));
        if (e != hipSuccess) return e;
    }
    if (a.splits > 1) {
        const size_t rows = (size_t)a.tokens * a.c.heads * a.group;
        const size_t blocks = (rows + 15) / 16, x = blocks < (1u << 22) ? blocks : (1u << 22);
        KernelTimer kt(KID_ATTEND_JOIN, st);
        launch_timed(kt, attend_join_kernel<TYPE>, dim3((unsigned)x, (unsigned)((blocks + x - 1) / x)), dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

}  // namespace

// Rows of a block and shares of the keys.  Blocks of 16 rows stream the cache; the larger ones of token_attend_chunk.hip multiply it.  These are faster from so many rows
// of a request on average that their rows are filled, and from so many of all requests and heads that a block is there for a third of the compute units at least
// (us with 16 rows / with 128, dim 128 in bf16: 256; equal requests, all keys seen:
//   rows, requests, heads, keys    66,9,12,1500  200,2,32,6000  264,8,8,2048  256,4,8,2048  400,4,8,3000  2048,1,8,8192  64,64,8,1024  400,64,4,1024  512,2,4,2000  384,1,2,16000  96,4,2,700
//   pages of 16, dim  64 bf16     27/39          95/68         50/50         33/37         56/44          145/88        46/68          125/83        24/27          34/59        10/20
//   pages of 16, dim  64 fp32     31/45          114/84        62/61         38/44         64/53         174/110        55/85         154/107        26/31          36/63        10/23
//   pages of 16, dim 128 bf16     42/68          169/85        82/62         35/60         92/82         253/109        80/98         234/158        26/92          47/68        11/35
//   pages of 16, dim 128 fp32     48/92         186/200        95/140        42/81        107/114        296/256        93/192        280/267        30/40          55/91        14/34
//   pages of 16, dim 256 bf16    112/130        386/276       200/192        80/110       201/156        582/356       213/271        530/368        53/53         104/145       20/45
//   pages of 16, dim 256 fp32    171/220        636/516       321/335       123/181       311/271        948/617       332/528        902/703        74/80         147/205       29/71
//   pages of 24, dim  64 bf16     38/39          126/68        64/50         41/38         66/44          183/88        60/67          166/84        27/26          38/58        10/20
//   pages of 24, dim  64 fp32     41/45          137/85        72/62         46/44         74/54         204/111        66/84         184/107        30/31          42/63        11/23
//   pages of 24, dim 128 bf16     49/68          200/85        104/63        58/60         103/83        289/108        96/99         259/157        38/92          49/68        13/36
//   pages of 24, dim 128 fp32     74/92         255/199       131/140        53/81        141/114        384/257       125/192        367/267        36/40          69/90        16/34
//   pages of 24, dim 256 bf16     97/129        342/277       172/193        73/111       187/156        517/356       185/270        478/368        49/53          95/144       19/46
//   pages of 24, dim 256 fp32    130/220        494/545       243/337       101/181       258/270        744/615       259/528        705/732        63/81         125/204       28/71
//   pages of  7, dim  64 bf16     62/38          210/68        104/50        60/38         98/44          291/88        93/68          265/85        36/26          48/58        13/20
//   pages of  7, dim  64 fp32     64/45          219/85        114/62        64/44         108/54        307/112        99/84         281/109        39/31          51/63        14/23
//   pages of  7, dim 128 bf16     75/70          311/88        163/63        79/62         156/84        420/111       144/101        393/161        48/94          65/70        17/35
//   pages of  7, dim 128 fp32     127/92        417/197       218/138        75/81        214/113        576/253       197/189        579/264        45/40          103/91       19/33
//   pages of  7, dim 256 bf16    152/129        498/271       265/189       105/111       255/154        718/349       280/271        681/360        63/53         127/145       22/45
//   pages of  7, dim 256 fp32    181/258        666/674       325/390       130/208       316/311        946/722       350/677        914/890        78/92         151/226       31/76).
// Over 1210 calls (those and drawn ones: ragged and equal, causal and not, dims from 48 to 256, pages from 1 to 64) the rule costs 2.6 % over the faster of the two, the
// best pair of limits for each dim, type and kind of page 2.0, rows of a request alone 7.9.
// Shares of the keys of larger blocks: up to a block for each compute unit (two of 128 rows), of 256 keys at least (us with 256, 512, 1024 keys at
// least: 256 rows of 5 requests and 8 heads over 1500 keys, dim 64 bf16 30, 33, 48, fp32 36, 39, 60, dim 128 59, 53, 74 and 66, 62, 95, dim 256 86, 82, 132 and
// 144, 138, 232; 300 rows of 4 and 12 over 1000: 31, 34, 34 | 36, 42, 42 | 44, 55, 56 | 67, 69, 69 | 92, 94, 94 | 155, 165, 166; 256 rows of 12 and 4 over 2500: 36, 37, 57 |
// 42, 46, 70 | 82, 88, 74 | 86, 98, 89 | 120, 137, 123 | 226, 251, 238).
void attend_plan(AttendArgs* a, int longest) {
    const long long rows = (long long)a->tokens * a->group, each = rows / a->requests;
    const bool fp32 = a->type == kF32;
    const int dim = a->c.dim <= 64 ? 64 : a->c.dim <= 128 ? 128 : 256;
    int many = dim == 128 && fp32 ? 300 : 160, all = 10000;
    // smaller pages: blocks of 16 rows look the table up for four keys at a time, or for each; larger ones look less often
    if (a->c.page_size % 4 != 0) {
        many = dim <= 128 ? 24 : fp32 ? 300 : 64;
        all = dim == 64 ? 2500 : dim == 128 ? 5000 : 8000;
    } else if (a->c.page_size % 16 != 0) {
        many = dim == 64 || (dim == 128 && !fp32) ? 72 : dim == 256 && fp32 ? 600 : 160;
        all = dim == 256 ? 10000 : 8000;
    }
    a->rows = each < many || rows * a->c.heads < all ? 16 : dim == 128 && !fp32 ? 256 : 128;
    const long long tiles = (rows / a->rows + a->requests) * a->c.heads;
    if (a->rows == 16) {
        // Shares of a fixed number of keys, so that long requests among short ones have more blocks: 2048, or 1024 where those are too few (below 128), or
        // too many for one block of eight waves on each compute unit and too few for two of four (us, shares of 1024 / 2048: single tokens of 1 request over
        // 2048 keys 16/19, over 8192 19/24, over 32768 39/33, 4 requests over 8192 29/25, 16 over 2000 25/20, 8 over 1 to 8192 29/30, 64 over 4096 113/107;
        // 20 tokens of 9 over 1 to 4000 27/31).  Eight waves where blocks are few (4 requests over 8192, four / eight waves: 29/25, 16 50/55, 64 over 4096
        // 107/116).
        const long long blocks = tiles * ((longest + 2047) / 2048);
        a->share = blocks >= 512 || (blocks >= 128 && blocks <= 256) ? 2048 : 1024;
        a->splits = (longest + a->share - 1) / a->share;
        a->waves = tiles * a->splits <= 256 ? 8 : 4;
        // At most 256 of them, and at most 2^14 blocks with theirs (a block leaves 16 rows of sums in the scratch, 2^20 times dim bytes together): the length may be
        // a table's, many times the requests'.
        const long long most = (1 << 14) / tiles < 1 ? 1 : (1 << 14) / tiles < 256 ? (1 << 14) / tiles : 256;
        if (a->splits > most) {
            a->splits = (int)most;
            a->share = (int)((longest + most - 1) / most + 31) & ~31;
        }
        if (a->splits < 1) a->splits = 1;
        return;
    }
    a->waves = a->rows / 32;
    const long long blocks = (each + a->rows - 1) / a->rows * a->requests * a->c.heads;
    long long s = (a->rows == 128 ? 512 : 256) / blocks;
    if (s > longest / 256) s = longest / 256;
    a->splits = s < 1 ? 1 : (int)s;
}

hipError_t launch_attend(const AttendArgs& a, hipStream_t st) {
    if (a.type == kF32) return attend_type<kF32>(a, st);
    if (a.type == kBF16) return attend_type<kBF16>(a, st);
    return attend_type<kF16>(a, st);
}

}  // namespace int8t
