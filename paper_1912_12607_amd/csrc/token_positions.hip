// What stands between a layer and the cache: queries and keys turned by their positions, and the pages, slots and positions of new tokens.
#include "device_common.h"
#include "positions.h"

namespace int8t {
namespace {

// ------------------------------------------------------------------------------------------------
// Rotary positions: pair i of a head at position p is turned by the angle 2 pi p turns[i].  The product is formed in 64 bits and its whole turns taken off
// before anything is rounded to 32 (at position 2^20 a fp32 angle would be off by 0.06); what rounding the rest to 32 bits loses comes back as a first-order
// term.  A lane has eight pairs of a token, finds their sines and cosines once and goes through heads with them; what is not turned is copied 16 values a lane.
// ------------------------------------------------------------------------------------------------
struct RotatePlan {
    int chunks, turned;      // lanes of a head, those of them whose values are turned
    int stride;              // lanes that share a token's heads: lane g has heads g, g + stride, ..
    FastDiv by_chunks, by_stride;
};
template <int TYPE>
__global__ __launch_bounds__(256) void rotate_kernel(const RotateArgs a, const RotatePlan p) {
    typedef typename ElemOf<TYPE>::type T;
    const int at = (int)(blockIdx.x * 256 + threadIdx.x);
    const int lane = div_by(at, p.by_chunks), c = at - lane * p.chunks;
    const int token = div_by(lane, p.by_stride), first = lane - token * p.stride;
    if (token >= a.tokens) return;
    const int heads = a.t[0].heads + a.t[1].heads, pairs = a.rot >> 1;
    const bool turned = c < p.turned;
    float cs[8], sn[8];
    if (turned) {
        const double position = (double)a.positions[token];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double turn = position * a.turns[min(8 * c + i, pairs - 1)], rest = turn - __builtin_rint(turn);
            const float high = (float)rest, low = (float)(rest - (double)high) * 6.28318530717958647692f;
            float s, k;
            sincospif(2.0f * high, &s, &k);
            cs[i] = __builtin_fmaf(-low, s, k) * a.amplitude;
            sn[i] = __builtin_fmaf(low, k, s) * a.amplitude;
            if (a.back) sn[i] = -sn[i];
        }
    }
    // the two runs of eight values of a lane, how many of them there are
    int at0, at1, left0, left1;
    if (!turned) {
        at0 = a.rot + 16 * (c - p.turned);
        at1 = at0 + 8;
        left0 = a.dim - at0;
        left1 = a.dim - at1;
    } else if (a.interleaved) {
        at0 = 16 * c;
        at1 = at0 + 8;
        left0 = a.rot - at0;
        left1 = a.rot - at1;
    } else {
        at0 = 8 * c;
        at1 = pairs + at0;
        left0 = left1 = pairs - at0;
    }
    const bool even0 = at0 * (int)sizeof(T) % 16 == 0, even1 = at1 * (int)sizeof(T) % 16 == 0;
    for (int h = first; h < heads; h += p.stride) {
        const bool second = h >= a.t[0].heads;
        const RotateTensor& t = second ? a.t[1] : a.t[0];
        const int head = second ? h - a.t[0].heads : h;
        const T* const x = static_cast<const T*>(t.x) + (size_t)token * t.x_token + (size_t)head * t.x_head;
        T* const y = static_cast<T*>(t.y) + (size_t)token * t.y_token + (size_t)head * t.y_head;
        if (!turned && t.x == t.y) continue;
        float u[8], v[8];
        load8<TYPE>(x + at0, left0, t.wide_x && even0, u);
        load8<TYPE>(x + at1, left1, t.wide_x && even1, v);
        if (turned) {
            float ru[8], rv[8];
            if (a.interleaved) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ru[2 * i] = __builtin_fmaf(u[2 * i], cs[i], -__fmul_rn(u[2 * i + 1], sn[i]));
                    ru[2 * i + 1] = __builtin_fmaf(u[2 * i], sn[i], __fmul_rn(u[2 * i + 1], cs[i]));
                    rv[2 * i] = __builtin_fmaf(v[2 * i], cs[4 + i], -__fmul_rn(v[2 * i + 1], sn[4 + i]));
                    rv[2 * i + 1] = __builtin_fmaf(v[2 * i], sn[4 + i], __fmul_rn(v[2 * i + 1], cs[4 + i]));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    ru[i] = __builtin_fmaf(u[i], cs[i], -__fmul_rn(v[i], sn[i]));
                    rv[i] = __builtin_fmaf(u[i], sn[i], __fmul_rn(v[i], cs[i]));
                }
            }
            store8<TYPE>(y + at0, left0, t.wide_y && even0, ru);
            store8<TYPE>(y + at1, left1, t.wide_y && even1, rv);
        } else {
            store8<TYPE>(y + at0, left0, t.wide_y && even0, u);
            store8<TYPE>(y + at1, left1, t.wide_y && even1, v);
        }
    }
}

template <int TYPE>
void rotate_of(const RotateArgs& a, hipStream_t st) {
    RotatePlan p;
    p.turned = (a.rot + 15) / 16;
    p.chunks = p.turned + (a.dim - a.rot + 15) / 16;
    const int heads = a.t[0].heads + a.t[1].heads;
    // heads of a lane: as many as leave lanes for the chip, eight at most
    const long long lanes = (long long)a.tokens * p.chunks * heads;
    int each = 1;
    while (each < 8 && lanes / (2 * each) >= 131072) each *= 2;
    p.stride = (heads + each - 1) / each;
    p.by_chunks = fast_div((unsigned)p.chunks);
    p.by_stride = fast_div((unsigned)p.stride);
    KernelTimer kt(KID_ROTATE, st);
    launch_timed(kt, rotate_kernel<TYPE>, dim3((unsigned)(((long long)a.tokens * p.stride * p.chunks + 255) / 256)), dim3(256), 0, st, a, p);
}

// ------------------------------------------------------------------------------------------------
// Pages of new tokens.  Every block goes through the requests, 256 at a time: inclusive sums of their new tokens and of the pages that these need beside the
// requests' own; a request whose pages the stack does not reach, whose table does not, or whose tokens pass the batch gets none.  The first block leaves the
// requests' results; each block marks in LDS which requests begin among its own tokens, and a running maximum over them gives every token its request.  A
// token's page is in the table already, or comes from the stack at a place known from the sums; the first token on a new page enters it in the table.
// ------------------------------------------------------------------------------------------------
constexpr int PT = 256, PE = 4, TILE = PT * PE;

// inclusive sums over the block's lanes of two values
struct Two { long long n; int pages; };
__device__ __forceinline__ Two block_sums(long long n, int pages, Two* waves) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const long long tn = __shfl_up(n, o, kWave);
        const int tp = __shfl_up(pages, o, kWave);
        if (lane >= o) {
            n += tn;
            pages += tp;
        }
    }
    __syncthreads();
    if (lane == 63) waves[wave] = Two{n, pages};
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        n += waves[w].n;
        pages += waves[w].pages;
    }
    return Two{n, pages};
}
__device__ __forceinline__ int pages_of(long long n, const FastDiv& by) { return div_by((int)(n - 1), by) + 1; }      // n > 0

__global__ __launch_bounds__(PT) void pages_extend_kernel(const PagesArgs a) {
    __shared__ Two sums[PT / 64];
    __shared__ int owner[TILE], have_of[TILE], first_of[TILE], count[2], tops[PT / 64];
    __shared__ long long start_of[TILE];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long t0 = (long long)blockIdx.x * TILE;
    for (int i = tid; i < TILE; i += PT) owner[i] = -1;
    if (tid < 2) count[tid] = 0;
    const int there = max(0, min(*a.available, a.pages));
    const long long most = (long long)a.width * a.page_size;
    Two before = {0, 0};
    int taken = 0, without = 0;
    for (int r0 = 0; r0 < a.requests; r0 += PT) {
        const int r = r0 + tid;
        const bool is = r < a.requests;
        const int n = is ? max(0, a.add[r]) : 0, have = is ? max(0, a.have[r]) : 0;
        Two s = block_sums(n, 0, sums);
        const long long end = before.n + s.n, start = end - n, want = (long long)have + n;
        const bool fits = is && want <= most && end <= a.tokens;
        const int held = have ? pages_of(min((long long)have, most), a.by_page) : 0, need = fits && want > 0 ? pages_of(want, a.by_page) - held : 0;
        s.pages = block_sums(0, need, sums).pages;
        const int upto = before.pages + s.pages;
        const bool placed = fits && (need == 0 || upto <= there);
        if (placed && need > 0) taken = max(taken, upto);
        if (is && !placed) ++without;
        if (blockIdx.x == 0 && is) {
            a.starts[r + 1] = (int)min(end, 0x7fffffffll);
            a.lengths[r] = placed ? (int)want : a.have[r];
        }
        if (n > 0 && start < t0 + TILE && end > t0) {
            const int i = (int)max(0ll, start - t0);
            owner[i] = placed ? r : -2 - r;
            have_of[i] = have;
            first_of[i] = upto - need - held;          // (page k of the request, k from `held` on: the stack's first_of + k from the top)
            start_of[i] = start;
        }
        // what the last lane has goes on
        __syncthreads();
        if (tid == PT - 1) sums[0] = Two{end, upto};
        __syncthreads();
        before = sums[0];
    }
    if (blockIdx.x == 0) {
        if (taken > 0) atomicMax(&count[0], taken);
        if (without > 0) atomicAdd(&count[1], without);
    }
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        a.starts[0] = 0;
        *a.left = there - count[0];
        *a.without = count[1];
    }
    // the last marked place at or before each of the lane's tokens
    int at[PE], last = -1;
#pragma unroll
    for (int u = 0; u < PE; ++u) {
        const int i = tid * PE + u;
        if (owner[i] != -1) last = i;
        at[u] = last;
    }
    int run = last;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int t = __shfl_up(run, o, kWave);
        if (lane >= o) run = max(run, t);
    }
    if (lane == 63) tops[wave] = run;
    __syncthreads();
    int earlier = __shfl_up(run, 1, kWave);
    if (lane == 0) earlier = -1;
    for (int w = 0; w < wave; ++w) earlier = max(earlier, tops[w]);
#pragma unroll
    for (int u = 0; u < PE; ++u) {
        const long long t = t0 + tid * PE + u;
        if (t >= a.tokens) break;
        const int i = max(at[u], earlier);
        long long slot = -1;
        int position = 0;
        const int r = i >= 0 ? owner[i] : -1;
        if (r >= 0) {
            const int n = max(0, a.add[r]);
            const long long in = t - start_of[i];
            if (in < n) {
                position = have_of[i] + (int)in;
                const int k = div_by(position, a.by_page), row = position - k * a.page_size, held = have_of[i] ? pages_of(have_of[i], a.by_page) : 0;
                int* const entry = a.table + (size_t)r * a.table_pitch + k;
                int id;
                if (k < held) {
                    id = *entry;
                } else {
                    id = a.free[there - 1 - (first_of[i] + k)];
                    if (row == 0) *entry = id;
                }
                if (id >= 0) slot = (long long)id * a.page_size + row;
            }
        }
        a.slots[t] = slot;
        a.positions[t] = position;
    }
}

// Pages behind the tokens that stay go back onto the stack, in the order of the requests; one block.
__global__ __launch_bounds__(PT) void pages_shrink_kernel(const PagesArgs a) {
    __shared__ Two sums[PT / 64];
    const int tid = (int)threadIdx.x;
    const int there = max(0, min(*a.available, a.pages));
    const long long most = (long long)a.width * a.page_size;
    int before = 0;
    for (int r0 = 0; r0 < a.requests; r0 += PT) {
        const int r = r0 + tid;
        const bool is = r < a.requests;
        const int have = is ? max(0, a.have[r]) : 0, stay = is ? max(0, min(a.add[r], have)) : 0;
        const int from = stay ? pages_of(min((long long)stay, most), a.by_page) : 0, to = have ? pages_of(min((long long)have, most), a.by_page) : 0;
        const int upto = before + block_sums(0, to - from, sums).pages, at = there + upto - (to - from);
        for (int k = from; k < to; ++k)
            if (at + k - from < a.pages) const_cast<int*>(a.free)[at + k - from] = a.table[(size_t)r * a.table_pitch + k];
        if (is) a.lengths[r] = stay;
        __syncthreads();
        if (tid == PT - 1) sums[0].pages = upto;
        __syncthreads();
        before = sums[0].pages;
    }
    if (tid == 0) *a.left = min(there + before, a.pages);
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, hipStream_t st) {
    if (a.type == kF32) rotate_of<kF32>(a, st);
    else if (a.type == kBF16) rotate_of<kBF16>(a, st);
    else rotate_of<kF16>(a, st);
    return hipGetLastError();
}
hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t st) {
    const int blocks = a.tokens > 0 ? (int)(((long long)a.tokens + TILE - 1) / TILE) : 1;
    KernelTimer kt(KID_PAGES, st);
    launch_timed(kt, pages_extend_kernel, dim3((unsigned)blocks), dim3(PT), 0, st, a);
    return hipGetLastError();
}
hipError_t launch_pages_shrink(const PagesArgs& a, hipStream_t st) {
    KernelTimer kt(KID_PAGES, st);
    launch_timed(kt, pages_shrink_kernel, dim3(1), dim3(PT), 0, st, a);
    return hipGetLastError();
}

}  // namespace int8t
