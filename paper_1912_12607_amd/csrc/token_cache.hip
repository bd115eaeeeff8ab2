// Keys and values on their way into and out of a paged cache in 8 bits: a scale for each token and head, found and applied as a row is
// written (Eq.1, c the row's maximum), and applied again where rows are read back.
#include "device_common.h"
#include "tokens.h"

namespace int8t {
namespace {

// place of a slot: page and row in it; false: no such place
__device__ __forceinline__ bool place_of(const CacheArgs& c, long long slot, size_t* page, int* at) {
    if (slot < 0 || slot >= c.places) return false;
    const int s = (int)slot;                     // (below 2^31: checked on the host)
    const int p = div_by(s, c.by_page);
    *page = (size_t)p;
    *at = s - p * c.page_size;
    return true;
}

// LANES neighbouring lanes have a row of up to 8 LANES values; a block has 256 / LANES rows, keys in blocks with y = 0 and values in
// those with y = 1 (z: a launch has fewer than 2^32 threads a dimension, and there may be more rows than that).  Bound by memory: 16384 tokens of 8 heads of 128 values, fp16, are written in 24.5 us and read back in 20.3 (102 MB each way: 4.2 and
// 5.0 TB/s, a large copy 5.1; writes leave scattered lines of 128 bytes and single scales); 64 tokens take the 3 us of a launch.
template <int TYPE, int LANES>
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheMoveArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    const int l = (int)threadIdx.x % LANES;
    const long long row = ((long long)blockIdx.z * gridDim.x + blockIdx.x) * (256 / LANES) + (int)threadIdx.x / LANES;
    const long long token = row / a.c.heads;
    const int head = (int)(row - token * a.c.heads);
    const bool values = blockIdx.y != 0;
    size_t page = 0;
    int at = 0;
    const bool live = token < a.tokens && place_of(a.c, a.slots[token < a.tokens ? token : 0], &page, &at);
    float v[8];
    {
        const T* x = values ? static_cast<const T*>(a.v) + (size_t)token * a.v_token + (size_t)head * a.v_head
                            : static_cast<const T*>(a.k) + (size_t)token * a.k_token + (size_t)head * a.k_head;
        load8<TYPE>(x + 8 * l, live ? a.c.dim - 8 * l : 0, a.wide, v);
    }
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = most(m, fabsf(v[i]));
#pragma unroll
    for (int o = 1; o < LANES; o *= 2) m = most(m, __shfl_xor(m, o, kWave));
    if (!live) return;
    const float inv = inv_scale_of(m);
    const size_t place = (page * a.c.heads + head) * a.c.page_size + at;
    if (l == 0) (values ? a.c.vs : a.c.ks)[place] = token_scale_of(m);
    if (8 * l < a.c.dim) {
        int c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = quantize_one<false>(v[i], inv, 0u, 0u, 0u);
        *reinterpret_cast<uint2*>((values ? a.c.vq : a.c.kq) + place * a.c.dim + 8 * l) = make_uint2(pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7]));
    }
}

template <int TYPE, int LANES>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheMoveArgs a) {
    typedef typename ElemOf<TYPE>::type T;
    const int l = (int)threadIdx.x % LANES;
    const long long row = ((long long)blockIdx.z * gridDim.x + blockIdx.x) * (256 / LANES) + (int)threadIdx.x / LANES;
    const long long token = row / a.c.heads;
    const int head = (int)(row - token * a.c.heads);
    if (token >= a.tokens || 8 * l >= a.c.dim) return;
    const bool values = blockIdx.y != 0;
    size_t page = 0;
    int at = 0;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (place_of(a.c, a.slots[token], &page, &at)) {
        const size_t place = (page * a.c.heads + head) * a.c.page_size + at;
        const float s = (values ? a.c.vs : a.c.ks)[place];
        const uint2 w = *reinterpret_cast<const uint2*>((values ? a.c.vq : a.c.kq) + place * a.c.dim + 8 * l);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fmul_rn((float)(int)(int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3))), s);
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
    KernelTimer kt(write ? KID_CACHE_WRITE : KID_CACHE_READ, st);
    if (write) launch_timed(kt, (cache_write_kernel<TYPE, LANES>), grid, dim3(256), 0, st, a);
    else launch_timed(kt, (cache_read_kernel<TYPE, LANES>), grid, dim3(256), 0, st, a);
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

hipError_t launch_cache_write(const CacheMoveArgs& a, hipStream_t st) { return move(a, true, st); }
hipError_t launch_cache_read(const CacheMoveArgs& a, hipStream_t st) { return move(a, false, st); }

}  // namespace int8t
