// What stands between a layer and the cache: queries and keys turned by their positions, and the pages, slots and positions of new tokens.
#include "device_common.h"
#include "positions.h"

namespace int8t {
namespace {

// ------------------------------------------------------------------------------------------------
// Rotary positions: pair i of a head at position p is turned by the angle 2 pi p turns[i].  The product is formed in 64 bits and its whole turns taken off
// before anything is rounded to 32 (at position 2^20 a fp32 angle would be off by 0.06); what rounding the rest to 32 bits loses comes back as a first-order
// term.  A lane has two runs of eight values of a head that hold eight pairs -- or that are copied --, neighbouring lanes neighbouring runs; it finds its sines and cosines
// once and goes through heads with them, the next head's values on their way.  Bound by memory: 8192 tokens of 32 and 8 heads of 128, fp16, 39 to 41 us (168 MB, 4.1 to 4.3
// TB/s); with a lane's two runs next to each other about 65.  64 tokens: 4.3 us, the launch and three loads in sequence.
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
    // the two runs: where they begin, how many values of them there are
    int at0, at1, left0, left1;
    if (!turned) {
        const int copies = p.chunks - p.turned;
        at0 = a.rot + 8 * (c - p.turned);
        at1 = at0 + 8 * copies;
        left0 = a.dim - at0;
        left1 = a.dim - at1;
    } else if (a.interleaved) {
        at0 = 8 * c;
        at1 = at0 + 8 * p.turned;
        left0 = a.rot - at0;
        left1 = a.rot - at1;
    } else {
        at0 = 8 * c;
        at1 = pairs + at0;
        left0 = left1 = pairs - at0;
    }
    const bool even0 = at0 * (int)sizeof(T) % 16 == 0, even1 = at1 * (int)sizeof(T) % 16 == 0;
    float u[8], v[8];
    const auto load = [&](int h) __attribute__((always_inline)) {
        const bool second = h >= a.t[0].heads;
        const RotateTensor& t = second ? a.t[1] : a.t[0];
        const T* const x = static_cast<const T*>(t.x) + (size_t)token * t.x_token + (size_t)(second ? h - a.t[0].heads : h) * t.x_head;
        load8<TYPE>(x + at0, left0, t.wide_x && even0, u);
        load8<TYPE>(x + at1, left1, t.wide_x && even1, v);
    };
    load(first);
    float cs[8], sn[8];
    if (turned) {
        const double position = (double)a.positions[token];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int pair = a.interleaved ? (i < 4 ? at0 / 2 + i : at1 / 2 + i - 4) : at0 + i;
            const double turn = position * a.turns[min(pair, pairs - 1)], rest = turn - __builtin_rint(turn);
            const float high = (float)rest, low = (float)(rest - (double)high) * 6.28318530717958647692f;
            float s, k;
            sincospif(2.0f * high, &s, &k);
            cs[i] = __builtin_fmaf(-low, s, k) * a.amplitude;
            sn[i] = __builtin_fmaf(low, k, s) * a.amplitude;
            if (a.back) sn[i] = -sn[i];
        }
    }
    for (int h = first; h < heads;) {
        const bool second = h >= a.t[0].heads;
        const RotateTensor& t = second ? a.t[1] : a.t[0];
        T* const y = static_cast<T*>(t.y) + (size_t)token * t.y_token + (size_t)(second ? h - a.t[0].heads : h) * t.y_head;
        float ru[8], rv[8];
        if (!turned) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                ru[i] = u[i];
                rv[i] = v[i];
            }
        } else if (a.interleaved) {
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
        h += p.stride;
        if (h < heads) load(h);                  // (a head's values are its lanes' alone, in place too)
        if (turned || t.x != t.y) {
            store8<TYPE>(y + at0, left0, t.wide_y && even0, ru);
            store8<TYPE>(y + at1, left1, t.wide_y && even1, rv);
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
// One launch: blocks find the sums again rather than wait for each other.  Bound by its steps in sequence: 64 requests with a token each 4.3 us, 300 prompts of up to 4096
// tokens 9 us (8 MB written).
// ------------------------------------------------------------------------------------------------
constexpr int PT = 256, PE = 4, TILE = PT * PE;

// What the lane some places before has, or 0: places of a row of 16 lanes (row_shr), the last lane of the row before (row_bcast15), of the half before (row_bcast31)
template <int CTRL, int ROWS>
__device__ __forceinline__ int before_of(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ long long before_of(long long v) {
    const uint32_t lo = (uint32_t)before_of<CTRL, ROWS>((int)(uint32_t)v), hi = (uint32_t)before_of<CTRL, ROWS>((int)(uint32_t)(v >> 32));
    return (long long)((uint64_t)hi << 32 | lo);
}
// Inclusive sums over the block's lanes; `all`: the block's
template <typename N, int LANES = PT>
__device__ __forceinline__ N block_sums(N n, N* waves, N* all) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    n += before_of<0x111, 0xf>(n);
    n += before_of<0x112, 0xf>(n);
    n += before_of<0x114, 0xf>(n);
    n += before_of<0x118, 0xf>(n);
    n += before_of<0x142, 0xa>(n);
    n += before_of<0x143, 0xc>(n);
    __syncthreads();
    if (lane == 63) waves[wave] = n;
    __syncthreads();
    N total = 0;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) {
        if (w < wave) n += waves[w];
        total += waves[w];
    }
    *all = total;
    return n;
}
__device__ __forceinline__ int pages_of(long long n, const FastDiv& by) { return div_by((int)(n - 1), by) + 1; }      // n > 0

__global__ __launch_bounds__(PT) void pages_extend_kernel(const PagesArgs a, const int wide) {
    __shared__ long long token_sums[PT / 64];
    __shared__ int page_sums[PT / 64], tops[PT / 64], count[2];
    __shared__ __attribute__((aligned(16))) int owner[TILE];
    __shared__ int have_of[TILE], new_of[TILE], first_of[TILE];
    __shared__ long long start_of[TILE];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long t0 = (long long)blockIdx.x * TILE;
    const bool first_block = blockIdx.x == 0;
    *reinterpret_cast<int4*>(owner + 4 * tid) = make_int4(-1, -1, -1, -1);
    if (tid < 2) count[tid] = 0;
    const int there = max(0, min(*a.available, a.pages));
    const long long most = (long long)a.width * a.page_size;
    long long tokens_before = 0;
    int pages_before = 0, taken = 0, without = 0;
    for (int r0 = 0; r0 < a.requests; r0 += PT) {
        const int r = r0 + tid;
        const bool is = r < a.requests;
        const int n = is ? max(0, a.add[r]) : 0, raw = is ? a.have[r] : 0, have = max(0, raw);
        long long tokens;
        const long long end = tokens_before + block_sums<long long>(n, token_sums, &tokens), start = end - n, want = (long long)have + n;
        const bool fits = is && want <= most && end <= a.tokens;
        const int held = have ? pages_of(min((long long)have, most), a.by_page) : 0, need = fits && want > 0 ? pages_of(want, a.by_page) - held : 0;
        int pages;
        const int upto = pages_before + block_sums<int>(need, page_sums, &pages);
        const bool placed = fits && (need == 0 || upto <= there);
        if (placed && need > 0) taken = max(taken, upto);
        if (is && !placed) ++without;
        if (first_block && is) {
            a.starts[r + 1] = (int)min(end, 0x7fffffffll);
            a.lengths[r] = placed ? (int)want : raw;
        }
        if (n > 0 && start < t0 + TILE && end > t0) {
            const int i = (int)max(0ll, start - t0);
            owner[i] = placed ? r : -2 - r;
            have_of[i] = have;
            new_of[i] = n;
            first_of[i] = upto - need - held;          // (page k of the request, k from `held` on: the stack's first_of + k from the top)
            start_of[i] = start;
        }
        tokens_before += tokens;
        pages_before += pages;
    }
    if (first_block) {
        if (taken > 0) atomicMax(&count[0], taken);
        if (without > 0) atomicAdd(&count[1], without);
    }
    __syncthreads();
    if (first_block && tid == 0) {
        a.starts[0] = 0;
        *a.left = there - count[0];
        *a.without = count[1];
    }
    // the last marked place at or before each of the lane's tokens
    int at[PE], last = -1;
    const int4 marks = *reinterpret_cast<const int4*>(owner + 4 * tid);
    const int mark[PE] = {marks.x, marks.y, marks.z, marks.w};
#pragma unroll
    for (int u = 0; u < PE; ++u) {
        if (mark[u] != -1) last = tid * PE + u;
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
    long long slot[PE];
    int position[PE];
#pragma unroll
    for (int u = 0; u < PE; ++u) {
        const long long t = t0 + tid * PE + u;
        const int i = max(at[u], earlier);
        slot[u] = -1;
        position[u] = 0;
        const int r = i >= 0 ? owner[i] : -1;
        if (r < 0 || t >= a.tokens) continue;
        const long long in = t - start_of[i];
        if (in >= new_of[i]) continue;
        const int p = position[u] = have_of[i] + (int)in;
        const int k = div_by(p, a.by_page), row = p - k * a.page_size, held = have_of[i] ? pages_of(have_of[i], a.by_page) : 0;
        int* const entry = a.table + (size_t)r * a.table_pitch + k;
        int id;
        if (k < held) {
            id = *entry;
        } else {
            id = a.free[there - 1 - (first_of[i] + k)];
            if (row == 0) *entry = id;
        }
        if (id >= 0) slot[u] = (long long)id * a.page_size + row;
    }
    const long long t = t0 + tid * PE;
    if (wide && t + PE <= a.tokens) {
        *reinterpret_cast<longlong2*>(a.slots + t) = make_longlong2(slot[0], slot[1]);
        *reinterpret_cast<longlong2*>(a.slots + t + 2) = make_longlong2(slot[2], slot[3]);
        *reinterpret_cast<int4*>(a.positions + t) = make_int4(position[0], position[1], position[2], position[3]);
    } else {
#pragma unroll
        for (int u = 0; u < PE; ++u)
            if (t + u < a.tokens) {
                a.slots[t + u] = slot[u];
                a.positions[t + u] = position[u];
            }
    }
}

// Pages behind the tokens that stay go back onto the stack, in the order of the requests; one block, since lengths and the stack's height change under it.  A request's
// pages are a wave's, four loads of each lane at a time; neighbouring requests, which end together more often, are different waves'.  64 requests of 8192 tokens that end, pages of 16: 14 us, one of
// them 7 (a lane for each request took 141 and 56).
constexpr int PS = 1024;
__global__ __launch_bounds__(PS) void pages_shrink_kernel(const PagesArgs a) {
    constexpr int NW = PS / 64;
    __shared__ long long sums[NW];
    __shared__ int from_of[PS], count_of[PS], at_of[PS];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int there = max(0, min(*a.available, a.pages));
    const long long most = (long long)a.width * a.page_size;
    long long before = 0;                        // (lengths that nobody keeps in order may count more pages than an int)
    for (int r0 = 0; r0 < a.requests; r0 += PS) {
        const int r = r0 + tid;
        const bool is = r < a.requests;
        const int have = is ? max(0, a.have[r]) : 0, stay = is ? max(0, min(a.add[r], have)) : 0;
        const int from = stay ? pages_of(min((long long)stay, most), a.by_page) : 0, to = have ? pages_of(min((long long)have, most), a.by_page) : 0;
        long long all;
        const long long at = there + before + block_sums<long long, PS>(max(0, to - from), sums, &all) - max(0, to - from);
        from_of[tid] = from;
        count_of[tid] = (int)max(0ll, min((long long)(to - from), a.pages - at));
        at_of[tid] = (int)min(at, (long long)a.pages);
        if (is) a.lengths[r] = stay;
        before += all;
        __syncthreads();
        for (unsigned long long left = __ballot(count_of[lane * NW + wave] > 0); left; left &= left - 1) {
            const int i = __builtin_ctzll(left) * NW + wave, n = count_of[i];
            const int* const row = a.table + (size_t)(r0 + i) * a.table_pitch + from_of[i];
            int* const to_free = const_cast<int*>(a.free) + at_of[i];
            for (int k = lane; k < n; k += 256) {
                int id[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) id[u] = k + 64 * u < n ? row[k + 64 * u] : 0;
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (k + 64 * u < n) to_free[k + 64 * u] = id[u];
            }
        }
    }
    __syncthreads();                             // (everyone has read what is there)
    if (tid == 0) *a.left = (int)min(there + before, (long long)a.pages);
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
    launch_timed(kt, pages_extend_kernel, dim3((unsigned)blocks), dim3(PT), 0, st, a, (((uintptr_t)a.slots | (uintptr_t)a.positions) & 15) == 0);
    return hipGetLastError();
}
hipError_t launch_pages_shrink(const PagesArgs& a, hipStream_t st) {
    KernelTimer kt(KID_PAGES, st);
    launch_timed(kt, pages_shrink_kernel, dim3(1), dim3(PS), 0, st, a);
    return hipGetLastError();
}

}  // namespace int8t
