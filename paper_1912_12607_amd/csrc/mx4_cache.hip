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

// LANES neighbouring lanes have a row of up to 8 LANES values; a block has 256 / LANES rows, keys in blocks with y = 0 and values in those with y = 1 (z: a
// launch has fewer than 2^32 threads a dimension, and there may be more rows than that).
template <int TYPE, int LANES>
__global__ __launch_bounds__(256) void mx_cache_write_kernel(const CacheMoveArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    const int l = (int)threadIdx.x % LANES;
    const long long row = ((long long)blockIdx.z * gridDim.x + blockIdx.x) * (256 / LANES) + (int)threadIdx.x / LANES;
    const long long token = row / a.c.heads;
    const int head = (int)(row - token * a.c.heads), blocks = mx_blocks(a.c.dim);
    const bool values = blockIdx.y != 0;
    size_t place = 0;
    const bool live = token < a.tokens && place_of(a.c, a.slots[token < a.tokens ? token : 0], head, &place);
    float v[8];
    {
        const T* x = values ? static_cast<const T*>(a.v) + (size_t)token * a.v_token + (size_t)head * a.v_head
                            : static_cast<const T*>(a.k) + (size_t)token * a.k_token + (size_t)head * a.k_head;
        load8<TYPE>(x + 8 * l, live ? a.c.dim - 8 * l : 0, a.wide, v);
    }
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = most(m, fabsf(v[i]));
    m = most(m, dpp_of<kDppSwap1>(m));
    m = most(m, dpp_of<kDppSwap2>(m));
    if (!live || l >= 4 * blocks) return;
    const uint32_t byte = mx_byte_of(m);
    if ((l & 3) == 0) reinterpret_cast<uint8_t*>(values ? a.c.vs : a.c.ks)[place * blocks + (l >> 2)] = (uint8_t)byte;
    *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(values ? a.c.vq : a.c.kq) + place * (16 * blocks) + 4 * l) = byte < 255u ? mx_codes8(v, mx_power(byte)) : 0u;
}

template <int TYPE, int LANES>
__global__ __launch_bounds__(256) void mx_cache_read_kernel(const CacheMoveArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    const int l = (int)threadIdx.x % LANES;
    const long long row = ((long long)blockIdx.z * gridDim.x + blockIdx.x) * (256 / LANES) + (int)threadIdx.x / LANES;
    const long long token = row / a.c.heads;
    const int head = (int)(row - token * a.c.heads), blocks = mx_blocks(a.c.dim);
    if (token >= a.tokens || 8 * l >= a.c.dim) return;
    const bool values = blockIdx.y != 0;
    size_t place = 0;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (place_of(a.c, a.slots[token], head, &place)) {
        const float s = mx_power(reinterpret_cast<const uint8_t*>(values ? a.c.vs : a.c.ks)[place * blocks + (l >> 2)]);
        const uint32_t w = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(values ? a.c.vq : a.c.kq) + place * (16 * blocks) + 4 * l);
        mx_values8(w, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], s);
    }
    T* x = values ? static_cast<T*>(a.v) + (size_t)token * a.v_token + (size_t)head * a.v_head
                  : static_cast<T*>(a.k) + (size_t)token * a.k_token + (size_t)head * a.k_head;
    store8<TYPE>(x + 8 * l, 8, a.wide, v);
}

constexpr long long kMostBlocks = 1 << 22;
template <int TYPE, int LANES>
void move_of(const CacheMoveArgs& a, bool write, hipStream_t st) {
    const long long blocks = ((long long)a.tokens * a.c.heads + 256 / LANES - 1) / (256 / LANES), x = blocks < kMostBlocks ? blocks : kMostBlocks;
    const dim3 grid((unsigned)x, 2, (unsigned)((blocks + x - 1) / x));
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
