// Keys and values on their way into and out of a paged cache of microscaled 4-bit codes: blocks of 32 dims of a head.
#include "mx4.h"

namespace int8t {
namespace {

// place of a slot, counted in rows of a head's page; false: no such place
__device__ __forceinline__ bool place_of(const CacheArgs& c, long long slot, int head, size_t* place) {
    if (slot < 0 || slot >= c.places) return false;
    const int s = (int)slot;                     // (below 2^31: checked on the host)
    const int p = div_by(s, c.by_page);
    *place = ((size_t)p * c.heads + head) * c.page_size + (s - p * c.page_size);
    return true;
}

// LANES neighbouring lanes have a row of up to 8 LANES values, of the keys and of the values; a block has 256 / LANES rows (y: a launch has fewer than 2^32 threads a
// dimension, and there may be more rows than that).  A block of 32 is four lanes' values: its largest goes round by lane exchanges, nothing goes through LDS.  Bound by
// memory: 16384 tokens of 8 heads of 128, fp16, written in 17 to 18 us (85 MB, 4.7 to 5 TB/s) and read in 20 (4.2 TB/s).
template <int TYPE, int LANES>
__global__ __launch_bounds__(256) void mx_cache_write_kernel(const CacheMoveArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    const int l = (int)threadIdx.x % LANES;
    const long long row = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * (256 / LANES) + (int)threadIdx.x / LANES;
    const long long token = row / a.c.heads;
    const int head = (int)(row - token * a.c.heads), blocks = mx_blocks(a.c.dim);
    const long long slot = token < a.tokens ? a.slots[token] : -1;
    float v[2][8], m[2];
    {
        const int left = token < a.tokens ? a.c.dim - 8 * l : 0;
        load8<TYPE>(static_cast<const T*>(a.k) + (size_t)token * a.k_token + (size_t)head * a.k_head + 8 * l, left, a.wide, v[0]);
        load8<TYPE>(static_cast<const T*>(a.v) + (size_t)token * a.v_token + (size_t)head * a.v_head + 8 * l, left, a.wide, v[1]);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        m[t] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m[t] = most(m[t], fabsf(v[t][i]));
        m[t] = most(m[t], dpp_of<kDppSwap1>(m[t]));
        m[t] = most(m[t], dpp_of<kDppSwap2>(m[t]));
    }
    size_t place = 0;
    if (!place_of(a.c, slot, head, &place) || l >= 4 * blocks) return;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint32_t byte = mx_byte_of(m[t]);
        if ((l & 3) == 0) reinterpret_cast<uint8_t*>(t ? a.c.vs : a.c.ks)[place * blocks + (l >> 2)] = (uint8_t)byte;
        *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(t ? a.c.vq : a.c.kq) + place * (16 * blocks) + 4 * l) = byte < 255u ? mx_codes8(v[t], mx_power(byte)) : 0u;
    }
}

template <int TYPE, int LANES>
__global__ __launch_bounds__(256) void mx_cache_read_kernel(const CacheMoveArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    const int l = (int)threadIdx.x % LANES;
    const long long row = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * (256 / LANES) + (int)threadIdx.x / LANES;
    const long long token = row / a.c.heads;
    const int head = (int)(row - token * a.c.heads), blocks = mx_blocks(a.c.dim);
    if (token >= a.tokens || 8 * l >= a.c.dim) return;
    size_t place = 0;
    uint32_t w[2] = {0u, 0u}, byte[2] = {0u, 0u};
    if (place_of(a.c, a.slots[token], head, &place)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            byte[t] = reinterpret_cast<const uint8_t*>(t ? a.c.vs : a.c.ks)[place * blocks + (l >> 2)];
            w[t] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(t ? a.c.vq : a.c.kq) + place * (16 * blocks) + 4 * l);
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        float v[8];
        mx_values8(w[t], v);
        const float s = mx_power(byte[t]);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], s);
        T* x = t ? static_cast<T*>(a.v) + (size_t)token * a.v_token + (size_t)head * a.v_head : static_cast<T*>(a.k) + (size_t)token * a.k_token + (size_t)head * a.k_head;
        store8<TYPE>(x + 8 * l, 8, a.wide, v);
    }
}

constexpr long long kMostBlocks = 1 << 22;
template <int TYPE, int LANES>
void move_of(const CacheMoveArgs& a, bool write, hipStream_t st) {
    const long long blocks = ((long long)a.tokens * a.c.heads + 256 / LANES - 1) / (256 / LANES), x = blocks < kMostBlocks ? blocks : kMostBlocks;
    const dim3 grid((unsigned)x, (unsigned)((blocks + x - 1) / x));
    KernelTimer kt(write ? KID_MX_CACHE_WRITE : KID_MX_CACHE_READ, st);
    if (write) launch_timed(kt, (mx_cache_write_kernel<TYPE, LANES>), grid, dim3(256), 0, st, a);
    else launch_timed(kt, (mx_cache_read_kernel<TYPE, LANES>), grid, dim3(256), 0, st, a);
}
template <int TYPE>
void move_type(const CacheMoveArgs& a, bool write, hipStream_t st) {
    if (a.c.dim <= 64) move_of<TYPE, 8>(a, write, st);
    else if (a.c.dim <= 128) move_of<TYPE, 16>(a, write, st);
    else move_of<TYPE, 32>(a, write, st);
}
hipError_t move(const CacheMoveArgs& a, bool write, hipStream_t st) {
    if (a.type == kF32) move_type<kF32>(a, write, st);
    else if (a.type == kBF16) move_type<kBF16>(a, write, st);
    else move_type<kF16>(a, write, st);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_cache_write(const CacheMoveArgs& a, hipStream_t st) { return move(a, true, st); }
hipError_t launch_mx_cache_read(const CacheMoveArgs& a, hipStream_t st) { return move(a, false, st); }

}  // namespace int8t
