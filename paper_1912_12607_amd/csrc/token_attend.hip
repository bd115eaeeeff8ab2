// Attention of new tokens over a paged cache in 8 bits:
//   o_i = sum_j p_ij vs_j vq_j / sum_j p_ij,   p_ij = exp(scale ks_j (q_i . kq_j)),   j < length (causal: up to the token's own place).
#include "device_common.h"
#include "tokens.h"

namespace int8t {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNone = -INFINITY;

__device__ __forceinline__ tk_h2 as_h2(uint32_t w) { return __builtin_bit_cast(tk_h2, w); }
__device__ __forceinline__ uint32_t as_u32(tk_h2 h) { return __builtin_bit_cast(uint32_t, h); }

// Two codes as fp16, exactly: u = code + 128 placed in the low bits of 0x6400 is 1024 + u; minus 1152.  `w` holds codes xor 0x80, the
// selector puts two of its bytes under 0x64.
template <uint32_t SEL>
__device__ __forceinline__ uint32_t codes_f16(uint32_t w) {
    const tk_h2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    return as_u32(as_h2(__builtin_amdgcn_perm(0x64646464u, w, SEL)) + off);
}
constexpr uint32_t kLowPair = 0x04010400u, kHighPair = 0x04030402u;

// The request that owns tile `t` of `per` rows: request b's tiles start at floor(starts[b] * group / per) + b, which leaves each request
// at least the tiles it needs.  Returns the last b with start <= t.
__device__ __forceinline__ int tile_request(const AttendArgs& a, int t, int per) {
    int lo = 0, hi = a.requests - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        const long long s = (long long)a.starts[mid] * a.group / per + mid;
        if (s <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// What a block knows of its request: rows (token, head of the group) and keys
struct Request {
    int token0, tokens;      // first token of q, how many (within q)
    int length;              // keys
    int new_tokens;          // (as the starts say: the causal limit goes by it)
    const int* pages;
};
__device__ __forceinline__ Request request_of(const AttendArgs& a, int b) {
    Request r;
    const int s0 = a.starts[b], s1 = a.starts[b + 1];
    r.new_tokens = s1 - s0;
    r.token0 = s0 < 0 ? 0 : s0;
    const int end = s1 < a.tokens ? s1 : a.tokens;
    r.tokens = end > r.token0 && s0 >= 0 ? end - r.token0 : 0;
    const long long most = (long long)a.width * a.c.page_size;
    const int len = a.lengths[b];
    r.length = len < 0 ? 0 : (long long)len < most ? len : (int)most;
    r.pages = a.table + (size_t)b * a.table_pitch;
    return r;
}

// Where key j of a request lies (its row of the cache's codes and scales); false: nowhere -- beyond `end`, or on a page that there is not.
__device__ __forceinline__ bool key_place(const AttendArgs& a, const Request& r, int head, int j, int end, size_t* place) {
    *place = 0;
    if (j >= end) return false;
    const int p = div_by(j, a.c.by_page);
    const int id = r.pages[p];
    if ((unsigned)id >= (unsigned)a.c.pages) return false;
    *place = ((size_t)id * a.c.heads + head) * a.c.page_size + (j - p * a.c.page_size);
    return true;
}

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

    // q: scaled by a power of two that brings the row's largest into [2^14, 2^15), which fp16 holds with room below
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
        const int e = max((int)((__float_as_uint(m) >> 23) & 255u), 30);         // (biased)
        const float up = __uint_as_float((uint32_t)min(127 + 14 + 127 - e, 254) << 23);
        qscale = __uint_as_float((uint32_t)max(e - 14, 1) << 23) * (a.scale * kLog2e);
#pragma unroll
        for (int i = 0; i < 2 * KL; ++i)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float t = v[i][u] * up;
                const _Float16 h = (_Float16)t;
                qf[0][i][u] = h;
                if (PARTS == 2) qf[PARTS - 1][i][u] = (_Float16)(t - (float)h);
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
            const float t = p * (vs[u] * inv_ref);
            const _Float16 h = (_Float16)t;
            pf[0][u] = h;
            if (PARTS == 2) pf[PARTS - 1][u] = (_Float16)(t - (float)h);
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
    const dim3 grid((unsigned)((long long)a.tokens * a.group / 16 + a.requests), (unsigned)a.c.heads, (unsigned)a.splits);
    {
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

// Shares of the keys: enough blocks to fill the chip, at least 256 keys (64 a wave) in a share where all requests are as long as the longest
int attend_splits(const AttendArgs& a, int longest) {
    const long long tiles = ((long long)a.tokens * a.group / 16 + a.requests) * a.c.heads;
    long long s = (1024 + tiles - 1) / tiles;
    const long long most = (longest + 255) / 256;
    if (s > most) s = most;
    if (s > 64) s = 64;
    return s < 1 ? 1 : (int)s;
}

hipError_t launch_attend(const AttendArgs& a, hipStream_t st) {
    if (a.type == kF32) return attend_type<kF32>(a, st);
    if (a.type == kBF16) return attend_type<kBF16>(a, st);
    return attend_type<kF16>(a, st);
}

}  // namespace int8t
