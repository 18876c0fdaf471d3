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
__device__ __forceinline__ uint32_t score_key(float s)
{
    const uint32_t u = __float_as_uint(s);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Element x of a row's 16-byte parts as a finite number (NaN: 0, an infinity: the largest).
template <bool FP8>
__device__ __forceinline__ void query_values(const uint4& v, float (&x)[FP8 ? 16 : 8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (FP8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __half2 h[2];
            e4m3x4_value(w[i], h);
            const float2 a = __half22float2(h[0]), b = __half22float2(h[1]);
            x[4 * i] = a.x, x[4 * i + 1] = a.y, x[4 * i + 2] = b.x, x[4 * i + 3] = b.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
#pragma unroll
    for (int i = 0; i < (FP8 ? 16 : 8); ++i) {
        if (x[i] != x[i]) x[i] = 0.f;
        if constexpr (!FP8) x[i] = fminf(fmaxf(x[i], -0x1.FEp127f), 0x1.FEp127f);
    }
}

// The four signed bytes of w as f16 (bytes 0, 1 and 2, 3): 1024 + (x + 128) has x's bits as its last ones
__device__ __forceinline__ void s8x4_value(uint32_t w, uint32_t& a, uint32_t& b)
{
    const uint32_t u = w ^ 0x80808080u;
    const __half2 off = bits_h2(0x64806480u);  // 1152
    a = h2_bits(__hsub2(bits_h2(__byte_perm(u, 0x64646464u, 0x4140)), off));
    b = h2_bits(__hsub2(bits_h2(__byte_perm(u, 0x64646464u, 0x4342)), off));
}

// The whole numbers of a query (of key head h) into the columns' tiles, by a warp; zeros where !real.
// store(column, channel, r): four neighbouring channels from this one on.
template <int D, bool FP8, typename F>
__device__ __forceinline__ void stage_query(const PickArgs& a, int64_t row, int h, bool real, int padded, int col0, F store)
{
    constexpr int PARTS = D * (FP8 ? 1 : 2) / 16, PER = 32 / PARTS, E = FP8 ? 16 : 8, U = 4;
    const int lane = threadIdx.x & 31, sub = lane % PARTS, first = lane / PARTS, step = PER;
    const uint8_t* from =
        static_cast<const uint8_t*>(a.q) + (row * a.q_stride + (int64_t)h * a.group * D) * (FP8 ? 1 : 2);
    auto load = [&](int y) { return __ldg(reinterpret_cast<const uint4*>(from + (int64_t)y * D * (FP8 ? 1 : 2)) + sub); };
    if (!real) {
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
        for (int y = first; y < padded; y += step)
#pragma unroll
            for (int e = 0; e < E; e += 4) store(col0 + y, sub * E + e, zero);
        return;
    }
    uint4 kept[U];  // the first rows stay in registers between the two passes
    float top = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u * step < padded) kept[u] = load(min(first + u * step, a.group - 1));
    auto reach = [&](const uint4& w) {
        float v[E];
        query_values<FP8>(w, v);
#pragma unroll
        for (int e = 0; e < E; ++e) top = fmaxf(top, fabsf(v[e]));
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u * step < padded) reach(kept[u]);
    for (int y = first + U * step; y < a.group; y += step) reach(load(y));
    top = warp_max_f32(top);
    // top = f * 2^p, f in [1/2, 1); the unit is 2^(p - 7)
    const int p = max((int)(__float_as_uint(top) >> 23) - 126, -119);
    const float up = __uint_as_float((uint32_t)(127 + 7 - p) << 23);
    auto put = [&](const uint4& w, int y) {
        float v[E];
        query_values<FP8>(w, v);
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            float r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = fminf(fmaxf(rintf(v[e + i] * up), -127.f), 127.f);
            store(col0 + y, sub * E + e, r);
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (first + u * step < padded) put(kept[u], first + u * step);  // (behind the last head: that one again)
    for (int y = first + U * step; y < padded; y += step)
        put(load(min(y, a.group - 1)), y);
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
