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

// The power of two that p carries: p times a value scale is held in fp16, and 2^up times the largest scale seen so far lies between 2^14 and
// 2^15, so that it fits, with room below (p may pass 1 by a factor below 2).
struct ValueUnit {
    float up = 0.0f, ref = -1.0f;            // ref: the largest scale that up allows
    // `largest`, of all of the wave's rows: the change of up
    __device__ __forceinline__ float raise(float largest) {
        if (!(largest > ref)) return 0.0f;
        const int e = max((int)((__float_as_uint(largest) >> 23) & 255u), 27);
        const float before = up;
        up = (float)(14 + 127 - e);
        ref = __uint_as_float(((uint32_t)(e + 1) << 23) - 1u);
        return up - before;
    }
};

// w in two fp16 pieces.  The product that w is must be rounded to fp32 before it is split: left to itself the compiler forms the first
// piece from the unrounded product and the rest from the rounded one, which differ by a step of the first now and then.
__device__ __forceinline__ void two_pieces(float w, _Float16* first, _Float16* rest) {
    asm("" : "+v"(w));
    *first = (_Float16)w;
    *rest = (_Float16)(w - (float)*first);
}

}  // namespace int8t
