// Rows quantised into the 4-bit cache.
//
// For every 16 channels of a new K or V row, in fp32: y = x * in_scale / scale,
// s = e4m3(max |y| / 6) (nearest, at most 448), code = e2m1(y / s) (nearest, ties
// to the even code, at most 6 in magnitude). A code stands for code * s * scale.
// One thread makes one block: it reads 32 bytes (bf16) or 16 (e4m3) and writes 8
// bytes of codes and one scale. A warp takes neighbouring rows of one head, as
// many as fill the 32 bytes of a sector of scales, so no two warps write to one
// sector of a full page.

#include "cache.cuh"

namespace lvs {

namespace {

constexpr int kAppendThreads = 256;

// x / d correctly rounded, with inv = 1 / d rounded: the product's remainder is
// exact under FMA, and one correction by it gives the nearest quotient
// (Markstein's theorem). Without it a quotient that lies on a boundary between
// two codes, as many of bf16 rows do, could fall to either side. Products that
// are 0 (their sign is kept) or beyond 2^120 (the theorem asks for a product in
// range) stay as they are.
__device__ __forceinline__ float quotient(float x, float d, float inv)
{
    const float z = x * inv;
    return z != 0.f && fabsf(z) < 0x1p120f ? fmaf(fmaf(-z, d, x), inv, z) : z;
}

template <int D, bool FP8>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ AppendArgs a, int heads_per_warp)
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
        const int64_t n = (int64_t)cache_len(a.lens[b], a.limit, bad) + a.off[b + 1] - a.off[b];
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
#pragma unroll 1
    for (int hv = 2 * h0; hv < 2 * h1; ++hv) {
        const int h = hv >> 1, t = hv & 1;
        float y[16];
        const float scale = a.cache.scale[t], inv = a.inv_scale[t], in_scale = a.in_scale[t];
        if constexpr (FP8) {
            const uint8_t* s = static_cast<const uint8_t*>(a.src[t]) + src_row * a.stride[t] + h * D + blk * 16;
            const uint4 v = __ldcs(reinterpret_cast<const uint4*>(s));
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 f = __half22float2(e4m3x2_value(w[i / 2] >> (16 * (i & 1))));
                y[2 * i] = f.x * in_scale;
                y[2 * i + 1] = f.y * in_scale;
            }
        } else {
            const __nv_bfloat16* s =
                static_cast<const __nv_bfloat16*>(a.src[t]) + src_row * a.stride[t] + h * D + blk * 16;
            const uint4 v0 = __ldcs(reinterpret_cast<const uint4*>(s));
            const uint4 v1 = __ldcs(reinterpret_cast<const uint4*>(s) + 1);
            const uint32_t w[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[2 * i] = __uint_as_float(w[i] << 16);
                y[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
        float top = 0.f;
        bool nan = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            y[i] = quotient(y[i], scale, inv);
            nan |= y[i] != y[i];
            top = fmaxf(top, fabsf(y[i]));
        }
        const uint8_t code_s =
            nan ? (uint8_t)0x7F : (uint8_t)__nv_cvt_float_to_fp8(__fdiv_rn(top, 6.f), __NV_SATFINITE, __NV_E4M3);
        const float s = __half2float(__low2half(e4m3x2_value(code_s)));
        const float s_inv = s > 0.f ? __frcp_rn(s) : 0.f;  // (a scale of 0: every code 0, the signs kept)
        uint64_t codes = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 z = make_float2(quotient(y[2 * i], s, s_inv), quotient(y[2 * i + 1], s, s_inv));
            codes |= (uint64_t)(uint8_t)__nv_cvt_float2_to_fp4x2(z, __NV_E2M1, cudaRoundNearest) << (8 * i);
        }
        if (nan) codes = 0;
        const int64_t row = cache_row(page, a.cache.hkv, h, a.cache.page_shift, slot);
        *reinterpret_cast<uint64_t*>(a.cache.codes[t] + row * (D / 2) + blk * 8) = codes;
        a.cache.scales[t][row * BLOCKS + blk] = code_s;
        if (a.stored[t]) {
            const uint32_t w[2] = {(uint32_t)codes, (uint32_t)(codes >> 32)};
            uint32_t o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 f = __half22float2(e2m1x2_value(w[i / 4] >> (8 * (i & 3))));
                const __nv_bfloat162 p = __floats2bfloat162_rn(f.x * s * scale, f.y * s * scale);
                o[i] = *reinterpret_cast<const uint32_t*>(&p);
            }
            uint4* dst = reinterpret_cast<uint4*>(a.stored[t] + (r * a.cache.hkv + h) * D + blk * 16);
            __stcs(dst, make_uint4(o[0], o[1], o[2], o[3]));
            __stcs(dst + 1, make_uint4(o[4], o[5], o[6], o[7]));
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
    while (per_warp < a.cache.hkv && row_groups * a.cache.hkv / (2 * per_warp) >= (int64_t)num_sms * 64) per_warp *= 2;
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
    auto kern = fp8 ? append_kernel<128, true> : (head_dim == 128 ? append_kernel<128, false> : append_kernel<64, false>);
    return cudaLaunchKernelEx(&cfg, kern, a, per_warp);
}

}  // namespace lvs
