// What the kernels that score a cache's pages share: the queries' whole numbers, the order of the scores, what a CTA scores.
#pragma once

#include "cache.cuh"

namespace lvs {

// Columns of a query: its heads padded to 1, 2, 4 or a multiple of 8.
__host__ __device__ __forceinline__ int padded_group(int group)
{
    return group <= 2 ? group : (group <= 4 ? 4 : (group + 7) & ~7);
}
// Order of the scores as whole numbers, above 1 (0: a page that the query does not see, 1: one that the pool has not).
// Scores are below 2^7 * 2^14 * 2^100, so keys are below 0xFC000000.
__device__ __forceinline__ uint32_t score_key(float s)
{
    const uint32_t u = __float_as_uint(s);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The four signed bytes of w as f16 (bytes 0, 1 and 2, 3): 1024 + (x + 128) has x's bits as its last ones
__device__ __forceinline__ void s8x4_value(uint32_t w, uint32_t& a, uint32_t& b)
{
    const uint32_t u = w ^ 0x80808080u;
    const __half2 off = bits_h2(0x64806480u);  // 1152
    a = h2_bits(__hsub2(bits_h2(__byte_perm(u, 0x64646464u, 0x4140)), off));
    b = h2_bits(__hsub2(bits_h2(__byte_perm(u, 0x64646464u, 0x4342)), off));
}

// A query's elements as they are in memory, sixteen bytes at a time: NaN as 0 and infinities as the largest value (clean),
// the largest magnitude's bits, and pairs of values.
template <bool FP8>
struct QueryBytes {
    static constexpr uint32_t kBad = FP8 ? 0x7Fu : 0x7F80u;  // magnitudes from here on are not finite
    __device__ static __forceinline__ uint32_t top(const uint4& v, uint32_t t)  // in both halves
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (FP8) t = __vmaxu2(t, __vmaxu2(w[i] & 0x007F007Fu, w[i] >> 8 & 0x007F007Fu));
            else t = __vmaxu2(t, w[i] & 0x7FFF7FFFu);
        }
        return t;
    }
    __device__ static __forceinline__ uint32_t clean_word(uint32_t w)
    {
        constexpr int BITS = FP8 ? 8 : 16;
        uint32_t r = 0u;
#pragma unroll
        for (int i = 0; i < 32; i += BITS) {
            uint32_t x = w >> i & ((1u << BITS) - 1u);
            const uint32_t m = x & ((1u << (BITS - 1)) - 1u);
            if (FP8 ? m == 0x7Fu : m > 0x7F80u) x = 0u;
            else if (!FP8 && m == 0x7F80u) --x;
            r |= x << i;
        }
        return r;
    }
    __device__ static __forceinline__ uint4 clean(const uint4& v)
    {
        return make_uint4(clean_word(v.x), clean_word(v.y), clean_word(v.z), clean_word(v.w));
    }
    // p of the magnitude with these bits: in [2^(p - 1), 2^p)
    __device__ static __forceinline__ int exponent(uint32_t bits)
    {
        if constexpr (FP8) return (int)(__float_as_uint(__low2float(e4m3x2_value(bits))) >> 23) - 126;
        else return (int)(bits >> 7) - 126;
    }
};

// The whole numbers of a query (of key head h) for the columns from col0 on, by a warp; zeros where !real.
// store(column, channel, r0, r1): r of four neighbouring channels from this one on, as f16.
template <int D, bool FP8, typename F>
__device__ __forceinline__ void stage_query(const PickArgs& a, int64_t row, int h, bool real, int padded, int col0, F store)
{
    using Q = QueryBytes<FP8>;
    constexpr int PARTS = D * (FP8 ? 1 : 2) / 16, PER = 32 / PARTS, E = FP8 ? 16 : 8, U = 4;
    const int lane = threadIdx.x & 31, sub = lane % PARTS, first = lane / PARTS, step = PER;
    const uint8_t* from =
        static_cast<const uint8_t*>(a.q) + (row * a.q_stride + (int64_t)h * a.group * D) * (FP8 ? 1 : 2);
    auto load = [&](int y) { return __ldg(reinterpret_cast<const uint4*>(from + (int64_t)y * D * (FP8 ? 1 : 2)) + sub); };
    if (!real) {
        const __half2 zero = bits_h2(0u);
        for (int y = first; y < padded; y += step)
#pragma unroll
            for (int e = 0; e < E; e += 4) store(col0 + y, sub * E + e, zero, zero);
        return;
    }
    uint4 kept[U];  // the first rows stay in registers between the two passes
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u * step < padded) kept[u] = load(min(first + u * step, a.group - 1));
    bool dirty = false;
    uint32_t top = 0u;
    for (;;) {  // (a second time where something is not finite)
        uint32_t t = 0u;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * step < padded) {
                if (dirty) kept[u] = Q::clean(kept[u]);
                t = Q::top(kept[u], t);
            }
        for (int y = first + U * step; y < a.group; y += step) t = Q::top(dirty ? Q::clean(load(y)) : load(y), t);
        top = __reduce_max_sync(0xffffffffu, max(t & 0xFFFFu, t >> 16));
        if (dirty || top < Q::kBad) break;
        dirty = true;
    }
    // the largest is f * 2^p, f in [1/2, 1); the unit is 2^(p - 7)
    const int p = max(Q::exponent(top), -119);
    const float up = __uint_as_float((uint32_t)(127 + 7 - p) << 23);
    const float2 up2 = make_float2(up, up), round2 = make_float2(0x1.8p23f, 0x1.8p23f), back2 = make_float2(-0x1.8p23f, -0x1.8p23f);
    const __half2 most = bits_h2(0x57F057F0u), least = bits_h2(0xD7F0D7F0u);  // 127, -127
    // the product is exact and below 2^22: added to 1.5 * 2^23 it is rounded to a whole number, a tie to the even one
    auto whole = [&](float2 x) {
        const float2 r = fadd2(ffma2(x, up2, round2), back2);
        return __hmin2(__hmax2(__floats2half2_rn(r.x, r.y), least), most);
    };
    auto put = [&](const uint4& v, int y) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; i += FP8 ? 1 : 2) {
            __half2 r[2];
            if constexpr (FP8) {
                __half2 x[2];
                e4m3x4_value(w[i], x);
#pragma unroll
                for (int k = 0; k < 2; ++k) r[k] = whole(__half22float2(x[k]));
            } else {
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    r[k] = whole(make_float2(__uint_as_float(w[i + k] << 16), __uint_as_float(w[i + k] & 0xFFFF0000u)));
            }
            store(col0 + y, sub * E + i * (FP8 ? 4 : 2), r[0], r[1]);
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (first + u * step < padded) put(kept[u], first + u * step);  // (behind the last head: that one again)
    for (int y = first + U * step; y < padded; y += step) {
        const uint4 v = load(min(y, a.group - 1));
        put(dirty ? Q::clean(v) : v, y);
    }
}

// What a CTA scores: queries [i0, i0 + queries) of its request, over the pages that the last of them sees (none: nothing to
// do, also where the select kernel reads no scores because all pages may be picked).
struct ScoreTile {
    int q0, i0, queries, pages;
};
__device__ __forceinline__ ScoreTile score_tile(const PickArgs& a, int b, int part, int per)
{
    ScoreTile s;
    s.q0 = __ldg(a.off + b);
    const int t = __ldg(a.off + b + 1) - s.q0;
    bool bad;
    const int len = cache_len(__ldg(a.lens + b), a.limit, bad);
    s.i0 = part * per;
    s.queries = min(per, t - s.i0);
    if (bad && s.queries > 0 && threadIdx.x == 0) atomicOr(a.err, kErrBounds);
    const int last = len - t + s.i0 + s.queries - 1;
    s.pages = s.queries <= 0 || last < 0 ? 0 : (last >> a.page_shift) + 1;
    if (s.pages <= a.budget) s.pages = 0;
    return s;
}

// The launch of cache_pick_tile.cu, for many columns (query x head) a request.
cudaError_t launch_pick_tiles(const PickArgs& a, int head_dim, bool fp8, int max_t, int max_pages, int num_sms,
                              cudaStream_t stream);
int pick_tile_queries(int group);  // queries of a CTA there

}  // namespace lvs
