// Shared by the attention kernels: codes as fp16, whose rows and keys a block has.
#pragma once
#include "device_common.h"
#include "tokens.h"

namespace int8t {

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
__device__ __forceinline__ Request request_of(const AttendArgs& a, int b, int s0, int s1, int len) {
    Request r;
    r.new_tokens = s1 - s0;
    r.token0 = s0 < 0 ? 0 : s0;
    const int end = s1 < a.tokens ? s1 : a.tokens;
    r.tokens = end > r.token0 && s0 >= 0 ? end - r.token0 : 0;
    const long long most = (long long)a.width * a.c.page_size;
    r.length = len < 0 ? 0 : (long long)len < most ? len : (int)most;
    r.pages = a.table + (size_t)b * a.table_pitch;
    return r;
}
__device__ __forceinline__ Request request_of(const AttendArgs& a, int b) { return request_of(a, b, a.starts[b], a.starts[b + 1], a.lengths[b]); }

// Inclusive sums over a wave's lanes
__device__ __forceinline__ int wave_sums(int n) {
    n += __builtin_amdgcn_update_dpp(0, n, 0x111, 0xf, 0xf, false);      // (row_shr: rows of 16 lanes)
    n += __builtin_amdgcn_update_dpp(0, n, 0x112, 0xf, 0xf, false);
    n += __builtin_amdgcn_update_dpp(0, n, 0x114, 0xf, 0xf, false);
    n += __builtin_amdgcn_update_dpp(0, n, 0x118, 0xf, 0xf, false);
    n += __builtin_amdgcn_update_dpp(0, n, 0x142, 0xa, 0xf, false);      // (the last lane of the row before)
    n += __builtin_amdgcn_update_dpp(0, n, 0x143, 0xc, 0xf, false);      // (of the half before)
    return n;
}
// The shares that a request of `length` keys is dealt out in: as many of `share` keys as it has, `splits` at most
__device__ __forceinline__ int shares_of(const AttendArgs& a, int length) { return a.splits == 1 || length <= a.share ? 1 : min(a.splits, div_by(length - 1, a.by_share) + 1); }

// What request, which tile of `rows` rows of it and which share the u-th block (of a head) has, counted over those that there are: false behind the last one.  A request's last rows,
// which see the most keys, come first.  Workgroups are dealt out to an XCD's groups of compute units in turn, whatever these have to do: where every other one ends
// at once, half of the chip has two rounds of work and the other none (256 blocks of 256 rows with 500 keys 69 us, not 34).
struct Unit { Request rq; int tile, share, shares; };
__device__ __forceinline__ bool unit_of(const AttendArgs& a, int u, int rows, bool by_length, int lane, Unit* out) {
    const long long most = (long long)a.width * a.c.page_size;
    int before = 0;
    for (int r0 = 0; r0 < a.requests; r0 += 64) {
        const int r = min(r0 + lane, a.requests - 1), s0 = a.starts[r], s1 = a.starts[r + 1], len = a.lengths[r], end = min(s1, a.tokens);
        const int n = r0 + lane < a.requests && s0 >= 0 && end > s0 ? end - s0 : 0;
        const int tiles = (int)(((long long)n * a.group + rows - 1) / rows), shares = by_length ? shares_of(a, (int)min((long long)max(0, len), most)) : a.splits;
        const int units = tiles * shares, upto = before + wave_sums(units);
        const unsigned long long behind = __ballot(upto > u);
        if (behind) {
            const int l = __builtin_ctzll(behind);
            const int all = __builtin_amdgcn_readlane(tiles, l), in = u - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(units, l));
            out->rq = request_of(a, r0 + l, __builtin_amdgcn_readlane(s0, l), __builtin_amdgcn_readlane(s1, l), __builtin_amdgcn_readlane(len, l));
            out->shares = __builtin_amdgcn_readlane(shares, l);
            out->share = (int)((uint32_t)in / (uint32_t)max(all, 1));
            out->tile = all - 1 - (in - out->share * all);
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
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

// Query rows in fp16: scaled by a power of two that brings the row's largest value (m, over all of its lanes) into [2^14, 2^15), which
// fp16 holds with room below; *back undoes it.
__device__ __forceinline__ float row_scale(float m, float* back) {
    const int e = max((int)((__float_as_uint(m) >> 23) & 255u), 30);         // (biased)
    *back = __uint_as_float((uint32_t)max(e - 14, 1) << 23);
    return __uint_as_float((uint32_t)min(127 + 14 + 127 - e, 254) << 23);
}

// The scores' factor, kept positive (maxima are taken before it): a negative scale goes into q through *up, and for none q becomes zero.
__device__ __forceinline__ float score_scale(float scale, float back, float* up) {
    if (scale < 0.0f) *up = -*up;
    if (scale == 0.0f) *up = 0.0f;
    return fmaxf(back * (fabsf(scale) * kLog2e), 1e-37f);
}

// Exchanges between the halves of a wave and between neighbouring rows of 16 lanes, in registers: both sides of a pair get both values.
struct Pair { float a, b; };
__device__ __forceinline__ Pair halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return Pair{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ Pair rows16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return Pair{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float halves_max(float x) { const Pair p = halves(x); return fmaxf(p.a, p.b); }
__device__ __forceinline__ float halves_sum(float x) { const Pair p = halves(x); return p.a + p.b; }
__device__ __forceinline__ float rows16_max(float x) { const Pair p = rows16(x); return fmaxf(p.a, p.b); }
__device__ __forceinline__ float rows16_sum(float x) { const Pair p = rows16(x); return p.a + p.b; }

// What a row's p carries, as a power of two: p_j = 2^(s_j + c), s_j its scores times log2(e), so that l = sum p and the weights w_j = p_j vs_j that the
// products take in fp16 share it.  c brings the largest weight that the row has seen to 2^14 .. 2^15, where fp16 has 11 bits down to 2^-28 of it and steps
// of 2^-38 below; a larger weight lowers c.  It goes by the row's own weights: by the tile's largest scale and score, a key that the row does not see, or
// sees at 2^-40, would take the bits of the others.
// bf16 and fp16 tensors have a weight in one piece, off by 2^-12 of itself at most and to either side: errors against 64 bits are 1.6e-3 to 1.7e-3 of bf16 results, as
// with weights in fp32, and 2.8e-4 to 2.9e-4 of fp16 ones (over 8-bit caches and over 4-bit ones), where those have 2.1e-4.  A second piece costs a chunk 60 % more time (two of 2048 tokens over 8192 keys 610 -> 994 us,
// dim 64 477 -> 570, dim 256 583 -> 659), single tokens 1 to 6 %.
struct RowUnit {
    static constexpr float kMostWeight = 63000.0f, kMostSum = 0x1p120f;     // (p alone stays in range where the scales are tiny or zero)
    float c = 0.0f;
    float room = kNone;          // p and p vs are finite up to this score; -infinity: nothing seen yet
    float vs = 0.0f;             // the largest value scale so far, of all rows of the wave
    static __device__ __forceinline__ float log_of(float scale) { return fminf(__builtin_amdgcn_logf(fabsf(scale)), 128.0f); }
    // Before p of a tile is formed, where a score may pass `room` or a value scale (each in some lane) vs: whether the size of some row's weights has to be
    // found out; `top`: its largest score.
    __device__ __forceinline__ bool unknown(float top, float scale) {
        vs = fmaxf(vs, wave_max(fabsf(scale)));
        if (room != kNone) room = limit();
        return __any(top > room);
    }
    // then, 2^weight the row's largest: what to multiply l and o with.  (Rows that have seen keys: only as far as p and p vs are finite, so that c
    // does not depend on what made the wave look.)
    __device__ __forceinline__ float set(float top, float weight) {
        if (!(top > room)) return 1.0f;
        const float before = c;
        const bool first = room == kNone;
        c = first ? floorf(fminf(15.0f - weight, 110.0f - top)) : fminf(c, floorf(fminf(100.0f - weight, 110.0f - top)));
        room = limit();
        return first ? 0.0f : __builtin_amdgcn_exp2f(c - before);
    }
    // after: whether weights are too large for fp16 (or l for fp32), and by how much (l, o, this tile's weights); `largest`, `sum` of the row
    static __device__ __forceinline__ bool large(float largest, float sum) { return __any(largest > kMostWeight || sum > kMostSum); }
    __device__ __forceinline__ float lower(float largest, float sum) {
        const int d = max(max(largest > kMostWeight ? __builtin_amdgcn_frexp_expf(largest) - 15 : 0, sum > kMostSum ? __builtin_amdgcn_frexp_expf(sum) - 105 : 0), 0);
        c -= (float)d;
        room += (float)d;
        return __builtin_ldexpf(1.0f, -d);
    }
   private:
    __device__ __forceinline__ float limit() const { return fminf(112.0f, 126.0f - log_of(vs)) - c; }
};
// p vs, and 0 where p is, whatever the scale: the place of a key that a row does not see may not have been written yet.
extern "C" __device__ __attribute__((const)) float multiply_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");       // 0 times anything is 0
__device__ __forceinline__ float weight_of(float p, float vs) { return multiply_legacy(p, vs); }
// What o of a row is multiplied with, and the row's natural logarithm, from its sum l in units of 2^m.  Only a sum of zero is one of no keys: NaN shows.
__device__ __forceinline__ float per_sum(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ float log_of_sum(float m, float l) { return l == 0.0f ? kNone : (m + __log2f(l)) * (1.0f / kLog2e); }
// Blocks of 16 rows over 4-bit caches leave this part of their sums of values for the joining pass (their l is whole): a power of two, as many as a block has waves
constexpr float kRowsPartScale = 8.0f;
// l to 1/2 .. 1: the shares of a row are joined by m = log2 of what l and o are in units of, and l;  *down: what o is to be multiplied with
__device__ __forceinline__ float normalised(float c, float* l, float* down) {
    const int e = __builtin_amdgcn_frexp_expf(*l);
    *down = __builtin_ldexpf(1.0f, -e);
    const float m = *l == 0.0f ? kNone : (float)e - c;
    *l *= *down;
    return m;
}

// w in two fp16 pieces.  The product that w is must be rounded to fp32 before it is split: left to itself the compiler forms the first
// piece from the unrounded product and the rest from the rounded one, which differ by a step of the first now and then.
__device__ __forceinline__ void two_pieces(float w, _Float16* first, _Float16* rest) {
    asm("" : "+v"(w));
    *first = (_Float16)w;
    *rest = (_Float16)(w - (float)*first);
}

}  // namespace int8t
