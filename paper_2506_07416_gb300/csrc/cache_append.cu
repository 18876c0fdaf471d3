// Rows quantised into the 4-bit cache.
//
// For every 16 channels of a new K or V row, in fp32: y = x * in_scale / scale,
// s = e4m3(max |y| / 6) (nearest, at most 448), code = e2m1(y / s) (nearest, ties
// to the even code, at most 6 in magnitude). A code stands for code * s * scale.
// One thread makes one block: it reads 32 bytes (bf16) or 16 (e4m3) and writes 8
// bytes of codes and one scale. A warp takes neighbouring rows of one head, as
// many as fill the 32 bytes of a sector of scales, so no two warps write to one
// sector of a full page.
// Bound by memory: 128 prompts of 1100 bf16 rows of 32 heads (5.27 GB read and written)
// take 824 us, 6.4 TB/s, 0.94 of a plain copy's rate. With picked e4m3 rows and the values
// written back (13 Ki rows, 388 MB) 78 us: 4.2 TB/s at 70% of the issue slots.

#include <type_traits>

#include "cache.cuh"

namespace lvs {

namespace {

constexpr int kAppendThreads = 256;

// x / d correctly rounded, with inv = 1 / d rounded: the product's remainder is exact
// under FMA, and one correction by it gives the nearest quotient (Markstein's theorem),
// for products in f32's range. Without it a quotient that lies on a boundary between two
// codes, as many of bf16 rows do, could fall to either side. The remainder is taken as
// z d - x, not x - z d, so that a zero keeps its sign.
__device__ __forceinline__ float quotient(float x, float d, float inv)
{
    const float z = x * inv;
    return fmaf(-fmaf(z, d, -x), inv, z);
}

// the largest of three magnitudes, NaN where one is
__device__ __forceinline__ float top3(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
    return r;
}

// e2m1 codes of eight values, the first in the lowest four bits
__device__ __forceinline__ uint32_t e2m1x8_codes(const float* v)
{
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// A block's 16 elements as they are read: 16 bytes of e4m3 codes, or 32 of bf16.
template <bool FP8>
struct Block {
    uint4 v[FP8 ? 1 : 2];
};
template <bool FP8>
__device__ __forceinline__ Block<FP8> load_block(const void* src, int64_t at)
{
    Block<FP8> b;
    const uint4* s = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(src) + at * (FP8 ? 1 : 2));
#pragma unroll
    for (int i = 0; i < (FP8 ? 1 : 2); ++i) b.v[i] = __ldcs(s + i);
    return b;
}

// GRANTED: with a.granted (asked in every call, 128 prompts of 1100 rows took 831 us and not 826).
template <int D, bool FP8, bool GRANTED>
__global__ void __launch_bounds__(kAppendThreads, 5) append_kernel(const __grid_constant__ AppendArgs a, int heads_per_warp)
{
    constexpr int BLOCKS = D / 16;        // of a row of one head
    constexpr int ROWS = 32 / BLOCKS;     // rows of a warp
    const int lane = threadIdx.x & 31;
    const int64_t warp = ((int64_t)blockIdx.x * kAppendThreads + threadIdx.x) >> 5;
    const int head_parts = (a.cache.hkv + heads_per_warp - 1) / heads_per_warp;
    griddep_wait();
    griddep_launch_dependents();
    for (int64_t b = (int64_t)blockIdx.x * kAppendThreads + threadIdx.x; b < a.batch;
         b += (int64_t)gridDim.x * kAppendThreads) {
        bool bad;
        const int64_t len = cache_len(a.lens[b], a.limit, bad);
        int64_t n = len + a.off[b + 1] - a.off[b];
        if (GRANTED) n = appended_len(len, n, a.granted[b]);
        if (bad || n > a.limit) atomicOr(a.err, kErrBounds);
        a.new_lens[b] = (int32_t)(n < a.limit ? n : a.limit);
    }
    const int64_t r = warp / head_parts * ROWS + lane / BLOCKS;
    const int blk = lane % BLOCKS;
    if (r >= a.rows) return;
    // the request of row r: the last whose first row is not behind it
    int lo = 0, hi = a.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(a.off + mid) <= r) lo = mid;
        else hi = mid;
    }
    bool bad;
    const int64_t pos = (int64_t)cache_len(a.lens[lo], a.limit, bad) + r - a.off[lo];
    if (GRANTED && pos >= a.granted[lo]) return;
    const int32_t page =
        pos < a.limit ? cache_page(a.cache.table, a.cache.width, a.cache.num_pages, a.cache.page_shift, lo, pos) : -1;
    const int64_t src_row = a.row_idx ? (int64_t)__ldg(a.row_idx + r) : r;
    if (page < 0 || src_row < 0 || src_row >= a.src_rows) {
        if (blk == 0) atomicOr(a.err, kErrBounds);
        return;
    }
    const int64_t slot = pos & ((1 << a.cache.page_shift) - 1);
    const int part = (int)(warp % head_parts);
    const int h0 = part * heads_per_warp, h1 = min(a.cache.hkv, h0 + heads_per_warp);
    if (a.weights && part == 0 && blk == 0) a.weights[((int64_t)page << a.cache.page_shift) + slot] = 0.f;
    // K and V of head after head, the next one's elements on their way while one is made into codes
    const int64_t at[2] = {src_row * a.stride[0] + blk * 16, src_row * a.stride[1] + blk * 16};
    Block<FP8> next = load_block<FP8>(a.src[0], at[0] + h0 * D);
#pragma unroll 1
    for (int hv = 2 * h0; hv < 2 * h1; ++hv) {
        const int h = hv >> 1, t = hv & 1;
        const Block<FP8> now = next;
        if (hv + 1 < 2 * h1) next = load_block<FP8>(a.src[t ^ 1], at[t ^ 1] + ((hv + 1) >> 1) * D);
        float y[16];
        const float scale = t ? a.cache.scale[1] : a.cache.scale[0], inv = t ? a.inv_scale[1] : a.inv_scale[0];
        const float in_scale = t ? a.in_scale[1] : a.in_scale[0];
        if constexpr (FP8) {
            const uint32_t w[4] = {now.v[0].x, now.v[0].y, now.v[0].z, now.v[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                __half2 v[2];
                e4m3x4_value(w[i], v);
                const float2 f = __half22float2(v[0]), g = __half22float2(v[1]);
                y[4 * i] = f.x, y[4 * i + 1] = f.y;
                y[4 * i + 2] = g.x, y[4 * i + 3] = g.y;
            }
        } else {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t w[4] = {now.v[q].x, now.v[q].y, now.v[q].z, now.v[q].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y[8 * q + 2 * i] = __uint_as_float(w[i] << 16);
                    y[8 * q + 2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
                }
            }
        }
        // x * in_scale / scale; a power of two divides exactly by its reciprocal, and the two
        // factors are one
        if ((__float_as_uint(scale) & 0x7FFFFFu) == 0u) {
            const float f = in_scale * inv;
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] *= f;
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x = FP8 ? y[i] * in_scale : y[i];
                y[i] = fabsf(x * inv) < 0x1p120f ? quotient(x, scale, inv) : x * inv;
            }
        }
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) top = top3(top, y[i], y[i + 1]);
        if (!(top < 0x1p100f)) {  // infinite, NaN or nearly: any magnitude from here on has the code 6
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = fminf(fmaxf(y[i], -0x1p100f), 0x1p100f);
        }
        const bool nan = top != top;
        const uint8_t code_s =
            nan ? (uint8_t)0x7F : (uint8_t)__nv_cvt_float_to_fp8(__fdiv_rn(top, 6.f), __NV_SATFINITE, __NV_E4M3);
        const __half2 s2 = __low2half2(e4m3x2_value(code_s));
        const float s = nan ? 0.f : __low2float(s2);
        const float s_inv = s > 0.f ? __frcp_rn(s) : 0.f;  // (a scale of 0: every code 0, the signs kept)
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = quotient(y[i], s, s_inv);
        uint32_t w[2] = {e2m1x8_codes(y), e2m1x8_codes(y + 8)};
        if (nan) w[0] = w[1] = 0u;
        const int64_t row = cache_row(page, a.cache.hkv, h, a.cache.page_shift, slot);
        *reinterpret_cast<uint2*>(a.cache.codes[t] + row * (D / 2) + blk * 8) = make_uint2(w[0], w[1]);
        a.cache.scales[t][row * BLOCKS + blk] = code_s;
        if (a.stored[t]) {
            uint4* dst = reinterpret_cast<uint4*>(a.stored[t] + (r * a.cache.hkv + h) * D + blk * 16);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                __half2 v[4];
                e2m1x8_value(w[q], v);
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = __half22float2(__hmul2(v[i], s2));  // (exact)
                    const __nv_bfloat162 p = __floats2bfloat162_rn(f.x * scale, f.y * scale);
                    o[i] = *reinterpret_cast<const uint32_t*>(&p);
                }
                __stcs(dst + q, make_uint4(o[0], o[1], o[2], o[3]));
            }
        }
    }
}

}  // namespace

cudaError_t launch_cache_append(const AppendArgs& a, int head_dim, bool fp8, int num_sms, cudaStream_t stream)
{
    const int rows_per_warp = 32 / (head_dim / 16);
    const int64_t row_groups = (a.rows + rows_per_warp - 1) / rows_per_warp;
    // heads of a warp: all of them once the rows alone fill the GPU
    int per_warp = 1;
    while (per_warp < a.cache.hkv && row_groups * a.cache.hkv / (2 * per_warp) >= (int64_t)num_sms * 128) per_warp *= 2;
    const int64_t parts = (a.cache.hkv + per_warp - 1) / per_warp;
    const int64_t warps = row_groups * parts;
    int64_t blocks = (warps * 32 + kAppendThreads - 1) / kAppendThreads;
    if (blocks < 1) blocks = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks, 1, 1);
    cfg.blockDim = dim3(kAppendThreads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    auto pick = [&](auto granted) {
        constexpr bool G = decltype(granted)::value;
        return fp8 ? append_kernel<128, true, G> : (head_dim == 128 ? append_kernel<128, false, G> : append_kernel<64, false, G>);
    };
    return cudaLaunchKernelEx(&cfg, a.granted ? pick(std::true_type{}) : pick(std::false_type{}), a, per_warp);
}

}  // namespace lvs
