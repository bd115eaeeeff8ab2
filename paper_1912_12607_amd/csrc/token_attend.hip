// Attention of new tokens over a paged cache in 8 bits:
//   o_i = sum_j p_ij vs_j vq_j / sum_j p_ij,   p_ij = exp(scale ks_j (q_i . kq_j)),   j < length (causal: up to the token's own place).
#include "token_attend.h"

namespace int8t {
namespace {

// ------------------------------------------------------------------------------------------------
// Sixteen rows (tokens times heads of a group, in order) of one request and one head of the cache per block; the request's keys are dealt
// to `splits` blocks and in each to four waves, which run on their own, 32 keys at a time, and join their sums in LDS.
//   scores   S^T[key][row] = K Q^T (16 x 16 x 32 products): a lane loads 16 bytes of a key, codes become fp16 exactly;
//   softmax  a lane's eight scores belong to one row; running maximum shared by a row's four lanes, raised when some lane needs it;
//   values   O^T[dim][row] = V^T P^T: S^T's layout is P^T's operand layout if the keys of a 32 are numbered (lane group, tile, i), so
//            nothing is exchanged; a lane loads DIM / 16 bytes of eight keys and turns them in registers.
// PARTS = 2 (fp32): q and p in two fp16 pieces each.
// ------------------------------------------------------------------------------------------------
template <int TYPE, int DIM>
__global__ __launch_bounds__(256) void attend_rows_kernel(const AttendArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    constexpr int PARTS = TYPE == kF32 ? 2 : 1, KL = DIM / 64, CB = DIM / 16;      // 16-byte loads of a key; bytes of a value row per lane
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n16 = lane & 15, kg = lane >> 4;
    const int head = (int)blockIdx.y, split = (int)blockIdx.z;
    const int D = a.c.dim;

    const int b = tile_request(a, (int)blockIdx.x, 16);
    const Request rq = request_of(a, b);
    const int nrows = rq.tokens * a.group;
    const long long tile = (long long)blockIdx.x - ((long long)a.starts[b] * a.group / 16 + b);
    if (tile < 0 || tile * 16 >= nrows) return;
    const int r0 = (int)tile * 16;

    // this lane's row
    const int row = r0 + n16;
    const bool have = row < nrows;
    const int token = (have ? row : r0) / a.group, gh = (have ? row : r0) - token * a.group;
    const int limit = !have ? 0 : a.causal ? min(rq.length, rq.length - rq.new_tokens + token + 1) : rq.length;
    // the block's keys: those that its last row sees
    const int last_token = min(r0 + 15, nrows - 1) / a.group;
    const int end = max(0, a.causal ? min(rq.length, rq.length - rq.new_tokens + last_token + 1) : rq.length);

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
#pragma unroll
            for (int u = 0; u < 8; ++u) m = fmaxf(m, fabsf(v[i][u]));
        }
        m = fmaxf(m, __shfl_xor(m, 16, kWave));
        m = fmaxf(m, __shfl_xor(m, 32, kWave));
        float back;
        const float up = row_scale(m, &back);
        qscale = back * (a.scale * kLog2e);
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

    // this wave's keys: whole 32s of the block's share
    const int steps = (end + 31) >> 5;
    const int s_from = (int)((long long)steps * split / a.splits), s_to = (int)((long long)steps * (split + 1) / a.splits);
    const int w_from = s_from + (int)((long long)(s_to - s_from) * wave / 4), w_to = s_from + (int)((long long)(s_to - s_from) * (wave + 1) / 4);

    float m = kNone, l = 0.0f, ref = 0.0f, inv_ref = 0.0f;      // maximum; sum of this lane's p; largest value scale so far, 2^15 / it
    tk_f4 o[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) o[c] = tk_f4{0.f, 0.f, 0.f, 0.f};

    for (int s = w_from; s < w_to; ++s) {
        const int j0 = s * 32;
        // keys of the scores' operand: 16 t + n16
        uint4 kw[2][KL];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            size_t place;
            key_place(a, rq, head, j0 + 16 * t + n16, end, &place);
#pragma unroll
            for (int i = 0; i < KL; ++i) {
                const int d = i * 64 + kg * 16;
                kw[t][i] = *reinterpret_cast<const uint4*>(a.c.kq + place * D + (d < D ? d : 0));      // (beyond D: q is zero there)
            }
        }
        // keys of this lane's scores and values: slot u = 4 t + i is key 16 t + 4 kg + i
        uint32_t vw[8][CB / 4];
        float ks[8], vs[8];
        bool seen[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int j = j0 + 16 * (u >> 2) + 4 * kg + (u & 3);
            size_t place;
            const bool ok = key_place(a, rq, head, j, end, &place);
            seen[u] = ok && j < limit;
            ks[u] = a.c.ks[place];
            const float s0 = a.c.vs[place];
            vs[u] = ok ? s0 : 0.0f;
            const int d = n16 * CB;
            const uint32_t* p = reinterpret_cast<const uint32_t*>(a.c.vq + place * D + (d < D ? d : 0));
#pragma unroll
            for (int c = 0; c < CB / 4; ++c) vw[u][c] = p[c];
        }
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
        float x[8], top = kNone, vmax = 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float t = sc[u >> 2][u & 3] * (ks[u] * qscale);
            x[u] = seen[u] ? t : kNone;
            top = fmaxf(top, x[u]);
            vmax = fmaxf(vmax, vs[u]);
        }
        if (__any(top > m || vmax > ref)) {
            top = fmaxf(top, __shfl_xor(top, 16, kWave));
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            const float m1 = fmaxf(m, top);
            vmax = fmaxf(wave_max(vmax), fmaxf(ref, 1e-30f));
            const float keep = m == kNone ? 0.0f : __builtin_amdgcn_exp2f(m - m1);
            l *= keep;
            const float by = keep * (ref / vmax);
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[c][r] *= by;
            m = m1;
            ref = vmax;
            inv_ref = 32768.0f / vmax;
        }
        const float base = m == kNone ? 0.0f : m;
        tk_h8 pf[PARTS];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float p = __builtin_amdgcn_exp2f(x[u] - base);
            l += p;
            const float w = p * (vs[u] * inv_ref);
            _Float16 first = (_Float16)w, rest;
            if (PARTS == 2) {
                two_pieces(w, &first, &rest);
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
                const uint32_t x0 = vw[2 * u][c4] ^ 0x80808080u, x1 = vw[2 * u + 1][c4] ^ 0x80808080u;
                const uint32_t lo = __builtin_amdgcn_perm(x1, x0, 0x05010400u), hi = __builtin_amdgcn_perm(x1, x0, 0x07030602u);
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
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    const float unit = ref * (1.0f / 32768.0f);

    // the four waves' sums, in LDS: [wave][row][DIM + 1], in units of the values
    __shared__ float sm[4][16], sl[4][16];
    __shared__ float so[4][16][DIM + 4];
    if (kg == 0) {
        sm[wave][n16] = m;
        sl[wave][n16] = l;
    }
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) so[wave][n16][CB * (4 * kg + r) + c] = o[c][r] * unit;
    __syncthreads();
    // 16 lanes per row
    const int jr = (int)threadIdx.x >> 4, jl = (int)threadIdx.x & 15;
    if (r0 + jr >= nrows) return;
    const float mm = fmaxf(fmaxf(sm[0][jr], sm[1][jr]), fmaxf(sm[2][jr], sm[3][jr]));
    float w[4], total = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = sm[i][jr] == kNone ? 0.0f : __builtin_amdgcn_exp2f(sm[i][jr] - mm);
        total += w[i] * sl[i][jr];
    }
    const int jt = (r0 + jr) / a.group, jg = (r0 + jr) - jt * a.group;
    const int heads = a.c.heads * a.group;
    const size_t out_row = (size_t)(rq.token0 + jt) * heads + head * a.group + jg;
    const bool whole = a.splits == 1;
    const float by = !whole ? 1.0f : total > 0.0f ? 1.0f / total : 0.0f;
    const size_t part_row = (size_t)split * a.tokens * heads + out_row;
    if (jl == 0) {
        if (whole) {
            if (a.lse) a.lse[out_row] = total > 0.0f ? (mm + __log2f(total)) * (1.0f / kLog2e) : kNone;
        } else {
            a.part_ml[2 * part_row] = mm;
            a.part_ml[2 * part_row + 1] = total;
        }
    }
#pragma unroll
    for (int d = jl * 8; d < DIM; d += 128) {
        if (d >= D) break;
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            v[u] = (w[0] * so[0][jr][d + u] + w[1] * so[1][jr][d + u] + w[2] * so[2][jr][d + u] + w[3] * so[3][jr][d + u]) * by;
        if (whole) store8<TYPE>(static_cast<T*>(a.out) + out_row * D + d, 8, true, v);
        else store8<kF32>(a.part_o + part_row * D + d, 8, true, v);
    }
}

// Joins the shares of a row: 16 lanes each.
template <int TYPE>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    const size_t rows = (size_t)a.tokens * a.c.heads * a.group;
    const size_t row = (size_t)blockIdx.x * 16 + ((int)threadIdx.x >> 4);
    const int l = (int)threadIdx.x & 15, D = a.c.dim;
    if (row >= rows) return;
    float m = kNone;
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.part_ml[2 * (s * rows + row)]);
    float total = 0.0f;
    for (int s = 0; s < a.splits; ++s) {
        const float ms = a.part_ml[2 * (s * rows + row)];
        if (ms != kNone) total += __builtin_amdgcn_exp2f(ms - m) * a.part_ml[2 * (s * rows + row) + 1];
    }
    const float by = total > 0.0f ? 1.0f / total : 0.0f;
    if (l == 0 && a.lse) a.lse[row] = total > 0.0f ? (m + __log2f(total)) * (1.0f / kLog2e) : kNone;
    for (int d = l * 8; d < D; d += 128) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < a.splits; ++s) {
            const float ms = a.part_ml[2 * (s * rows + row)];
            if (ms == kNone) continue;
            const float w = __builtin_amdgcn_exp2f(ms - m) * by;
            float p[8];
            load8<kF32>(a.part_o + (s * rows + row) * D + d, 8, true, p);
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] += w * p[u];
        }
        store8<TYPE>(static_cast<T*>(a.out) + row * D + d, 8, true, v);
    }
}

template <int TYPE>
hipError_t attend_type(const AttendArgs& a, hipStream_t st) {
    if (a.rows > 16) {
        const hipError_t e = launch_attend_chunk(a, st);
        if (e != hipSuccess) return e;
    } else {
        const dim3 grid((unsigned)((long long)a.tokens * a.group / 16 + a.requests), (unsigned)a.c.heads, (unsigned)a.splits);
        KernelTimer kt(KID_ATTEND, st);
        if (a.c.dim <= 64) launch_timed(kt, (attend_rows_kernel<TYPE, 64>), grid, dim3(256), 0, st, a);
        else if (a.c.dim <= 128) launch_timed(kt, (attend_rows_kernel<TYPE, 128>), grid, dim3(256), 0, st, a);
        else launch_timed(kt, (attend_rows_kernel<TYPE, 256>), grid, dim3(256), 0, st, a);
    }
    if (a.splits > 1) {
        const size_t rows = (size_t)a.tokens * a.c.heads * a.group;
        KernelTimer kt(KID_ATTEND_JOIN, st);
        launch_timed(kt, attend_join_kernel<TYPE>, dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

}  // namespace

// Rows of a block by the average of a request, and shares of the keys: enough blocks to fill the chip, and at least 256 keys in a share where
// all requests are as long as the longest
void attend_plan(AttendArgs* a, int longest) {
    const long long rows = (long long)a->tokens * a->group, each = rows / a->requests;
    a->rows = each <= 32 ? 16 : each < 256 || a->c.dim > 128 ? 128 : 256;
    const long long tiles = (rows / a->rows + a->requests) * a->c.heads;
    const long long fill = a->rows == 16 ? 1024 : a->rows == 128 ? 512 : 256;
    long long s = fill / (tiles > 0 ? tiles : 1);
    const long long most = (longest + 255) / 256;
    if (s > most) s = most;
    if (s > 64) s = 64;
    a->splits = s < 1 ? 1 : (int)s;
}

hipError_t launch_attend(const AttendArgs& a, hipStream_t st) {
    if (a.type == kF32) return attend_type<kF32>(a, st);
    if (a.type == kBF16) return attend_type<kBF16>(a, st);
    return attend_type<kF16>(a, st);
}

}  // namespace int8t
