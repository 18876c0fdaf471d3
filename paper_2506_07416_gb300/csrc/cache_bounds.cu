// The ranges of the keys of a page: for each key head and channel the largest and the
// smallest value of the page's tokens, outwards as whole numbers of a power of two that
// the head's channels share.
//
// x = e2m1 * e4m3 (exact in f16, NaN counts as 0); m = max |x| over the page's tokens and the head's channels
// = f * 2^p, f in [1/2, 1). With e = p - 7 the codes ceil(max x / 2^e) and floor(min x / 2^e)
// lie in [-126, 126]: x has at most six significant bits, so f <= 63/64. A page costs its codes and
// scales once (page * d * 9/16 bytes a head) and 2 d + 1 bytes written.
// A warp takes key heads of a page: four lanes a row, 16 bytes of codes each, eight rows
// at a time, the largest and smallest of 32 channels in half pairs; the eight rows' lanes then
// halve the channels they hold as they exchange them. The next 32 rows, or the next head's, are on their way
// meanwhile.
// What bounds it: the extremes, an instruction of the integer pipe each for two channels of a row (64 of the 110 that eight
// rows take, two clocks each). 128 prompts of 1100 tokens, 32 heads, pages of 64 (343 MB): 98 us; without the
// loads ahead 124, as 5 CTAs an SM take 102, 4 105 and 6, which spill, 116. A token of each of these requests, whose last page
// it renews: 9 us.

#include <algorithm>

#include "cache.cuh"

namespace lvs {

namespace {

constexpr int kBoundsThreads = 128;

// Two blocks' scales; NaN counts as 0.
__device__ __forceinline__ __half2 block_scales(uint32_t s)
{
    const uint32_t nan = ((s & 0x7F7Fu) + 0x0101u) & 0x8080u;
    if (nan) s &= ~((nan >> 7) * 0xFFu);
    return e4m3x2_value(s);
}

// Of N half pairs that the lanes d apart (16 down to LAST) hold of the same channels, each keeps the extremes of its own
// ones: the upper lane the upper half. Returns the first pair that the lane keeps. (Values are picked by copies: picked by
// index they would live in memory.)
template <int N, int d, int LAST, int A>
__device__ __forceinline__ int halve(__half2 (&top)[A], __half2 (&low)[A], int lane)
{
    if constexpr (d < LAST) {
        return 0;
    } else {
        constexpr int n = N / 2;
        const bool up = lane & d;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const __half2 t0 = top[i], t1 = top[i + n], l0 = low[i], l1 = low[i + n];
            const uint32_t tg = up ? h2_bits(t0) : h2_bits(t1), tk = up ? h2_bits(t1) : h2_bits(t0);
            const uint32_t lg = up ? h2_bits(l0) : h2_bits(l1), lk = up ? h2_bits(l1) : h2_bits(l0);
            top[i] = __hmax2(bits_h2(tk), bits_h2(__shfl_xor_sync(0xffffffffu, tg, d)));
            low[i] = __hmin2(bits_h2(lk), bits_h2(__shfl_xor_sync(0xffffffffu, lg, d)));
        }
        return (up ? n : 0) + halve<n, d / 2, LAST>(top, low, lane);
    }
}

template <int D>
__global__ void __launch_bounds__(kBoundsThreads, 5) bounds_kernel(const __grid_constant__ BoundsArgs a, int heads)
{
    constexpr int LANES = D / 32;     // lanes of a row
    constexpr int ROWS = 32 / LANES;  // rows of a warp at a time
    constexpr int PAIRS = 16;         // half pairs of a lane's 32 channels
    const int lane = threadIdx.x & 31;
    const int64_t unit = ((int64_t)blockIdx.x * kBoundsThreads + threadIdx.x) >> 5;
    const int parts = (a.cache.hkv + heads - 1) / heads;
    const int64_t place = unit / parts;
    const int h0 = (int)(unit - place * parts) * heads, h1 = min(a.cache.hkv, h0 + heads);
    griddep_wait();
    griddep_launch_dependents();
    if (place >= a.places) return;
    const int lo =  // the request
        last_before(a.batch, [&](int x) { return page_at(__ldg(a.off + x), x, a.cache.page_shift) <= place; });
    const int q0 = __ldg(a.off + lo), t = __ldg(a.off + lo + 1) - q0;
    bool bad;
    const int len = cache_len(__ldg(a.lens + lo), a.limit, bad);
    if (t <= 0) return;
    if (bad && lane == 0) atomicOr(a.err, kErrBounds);
    const int64_t o = (max(len - t, 0) >> a.cache.page_shift) + (place - page_at(q0, lo, a.cache.page_shift));
    const int64_t first = o << a.cache.page_shift;
    if (first >= len) return;
    const int32_t page = cache_page(a.cache.table, a.cache.width, a.cache.num_pages, a.cache.page_shift, lo, first);
    if (page < 0) {
        if (lane == 0) atomicOr(a.err, kErrBounds);
        return;
    }
    const int rows = min(1 << a.cache.page_shift, len - (int)first);
    const int c = lane % LANES, g = lane / LANES;
    // the rows of one head after the other's, U groups of ROWS at a time, the next ones' on their way
    constexpr int U = 4;
    const int per_head = (rows + ROWS * U - 1) / (ROWS * U), n = per_head * (h1 - h0);
    uint4 next_w[U];
    uint32_t next_s[U];
    auto load = [&](int x) {
        const int h = h0 + x / per_head, r0 = x % per_head * (ROWS * U);
        const int64_t at = cache_row(page, a.cache.hkv, h, a.cache.page_shift, 0);
        const uint4* codes = reinterpret_cast<const uint4*>(a.cache.codes[0] + at * (D / 2)) + c;
        const uint16_t* scales = reinterpret_cast<const uint16_t*>(a.cache.scales[0] + at * (D / 16)) + c;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = min(r0 + u * ROWS + g, rows - 1);  // (the last row again changes nothing)
            next_w[u] = __ldg(codes + r * LANES);
            next_s[u] = __ldg(scales + r * LANES);
        }
    };
    load(0);
    __half2 top[PAIRS], low[PAIRS];
    const __half2 inf = bits_h2(0x7C007C00u), ninf = bits_h2(0xFC00FC00u);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) top[i] = ninf, low[i] = inf;
#pragma unroll 1
    for (int x = 0; x < n; ++x) {
        uint4 w[U];
        uint32_t s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = next_w[u], s[u] = next_s[u];
        if (x + 1 < n) load(x + 1);
        const int h = h0 + x / per_head, r0 = x % per_head * (ROWS * U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r0 + u * ROWS >= rows) break;
            const uint32_t words[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
            const __half2 both = block_scales(s[u]), sc[2] = {__low2half2(both), __high2half2(both)};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                __half2 v[4];
                e2m1x8_value(words[k], v);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __half2 y = __hmul2(v[i], sc[k / 2]);
                    top[4 * k + i] = __hmax2(top[4 * k + i], y);
                    low[4 * k + i] = __hmin2(low[4 * k + i], y);
                }
            }
        }
        if (r0 + ROWS * U < rows) continue;
        // lanes of the same channels exchange halves of what they hold, until each has its own 32 / ROWS
        const int mine = halve<PAIRS, 16, LANES>(top, low, lane);
        constexpr int KEPT = PAIRS / ROWS;  // pairs of a lane now
        float m = 0.f;
        float hi_v[2 * KEPT], lo_v[2 * KEPT];
#pragma unroll
        for (int i = 0; i < KEPT; ++i) {
            const float2 x = __half22float2(top[i]), y = __half22float2(low[i]);
            hi_v[2 * i] = x.x, hi_v[2 * i + 1] = x.y;
            lo_v[2 * i] = y.x, lo_v[2 * i + 1] = y.y;
            m = fmaxf(m, fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(y.x), fabsf(y.y))));
        }
        m = warp_max_f32(m);
        // m = f * 2^p, p = exponent field - 126 (values are normal in fp32); the unit is 2^(p - 7)
        const int e = m > 0.f ? (int)(__float_as_uint(m) >> 23) - 126 - 7 : 0;
        const float per = __uint_as_float((uint32_t)(127 - e) << 23);
        int8_t* to = a.codes + ((int64_t)page * a.cache.hkv + h) * 2 * D + c * 32 + mine * 2;
        static_assert(KEPT == 1 || KEPT == 2, "two or four channels a lane");
        uint32_t ch = 0, cl = 0;
#pragma unroll
        for (int i = 0; i < 2 * KEPT; ++i) {
            ch |= ((uint32_t)(int)ceilf(hi_v[i] * per) & 0xFFu) << (8 * i);
            cl |= ((uint32_t)(int)floorf(lo_v[i] * per) & 0xFFu) << (8 * i);
        }
        if constexpr (KEPT == 2) {
            *reinterpret_cast<uint32_t*>(to) = ch;
            *reinterpret_cast<uint32_t*>(to + D) = cl;
        } else {
            *reinterpret_cast<uint16_t*>(to) = (uint16_t)ch;
            *reinterpret_cast<uint16_t*>(to + D) = (uint16_t)cl;
        }
        if (lane == 0) a.exps[(int64_t)page * a.cache.hkv + h] = (int8_t)e;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) top[i] = ninf, low[i] = inf;
    }
}

}  // namespace

cudaError_t launch_cache_bounds(const BoundsArgs& a, int head_dim, int num_sms, cudaStream_t stream)
{
    if (a.places <= 0) return cudaSuccess;
    // heads of a warp, which finds its page once for them: more where the pages alone fill the GPU
    int heads = 1;
    while (heads < a.cache.hkv && a.places * a.cache.hkv / (2 * heads) >= (int64_t)num_sms * 128) heads *= 2;
    const int64_t warps = a.places * ((a.cache.hkv + heads - 1) / heads);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((warps * 32 + kBoundsThreads - 1) / kBoundsThreads), 1, 1);
    cfg.blockDim = dim3(kBoundsThreads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, head_dim == 128 ? bounds_kernel<128> : bounds_kernel<64>, a, heads);
}

}  // namespace lvs
