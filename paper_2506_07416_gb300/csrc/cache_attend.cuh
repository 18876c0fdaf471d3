// What the attention kernels of the 4-bit cache share: the split of the keys, the rows of
// a CTA, and the units of their sums.
#pragma once

#include "cache.cuh"

namespace lvs {

constexpr float kNoRef = -3.0e38f;   // reference of a row without keys so far
// A row's reference is put this much below its largest score so far and moves when a score passes it by kRefSlack: a
// probability in f16, 2^(score - reference), then lies between 2^7 and 2^15 at the largest score and is off by at most
// 2^-32 of it where it falls below f16's normal range. (With the reference at the largest score 2^-25: a million keys
// of 2^-25 of the largest, 3% of a row's sum, were lost.)
constexpr float kRefBelow = 7.f, kRefSlack = 15.f;

// What turns a row's products into scores in log2 units (`back` undoes the scaling of its query). Not 0, where the
// factors' product is below 32 bits, as for a query of zeros, whose back is 2^-126: masked keys have a score of
// -inf, which 0 would make NaN, and at the smallest normal value every 2^s is 1 too. And at most 2^90, so that no
// score leaves fp32 (products are below 2^30): two sums that differ at all, by 2^-34 or more, are then 2^56
// apart, and the softmax is as with any larger factor.
__device__ __forceinline__ float row_factor(float c_log2, float back)
{
    return fminf(fmaxf(c_log2 * back, 0x1p-126f), 0x1p90f);
}
// Up to this factor a score stays below 2^22, and the rounding of a reference or an lse, by which the kernels with
// a fused multiplication and subtraction move a whole row, is at most 2^-3. Beyond it they round each score as
// its row's reference was rounded and subtract then: a reference of 2^33 is rounded by up to 2^9, and 2^512
// is no number.
constexpr float kFusedFactor = 0x1p-8f;

__device__ __forceinline__ uint32_t pack_h2(float lo, float hi) { return h2_bits(__floats2half2_rn(lo, hi)); }

// How the keys are split, where the plan gives them slots (below three rounds of whole requests, see
// plan_cache_attend), found by a warp from the lengths on the device: equal chunks, as short as they may be while all
// requests together have at most a.slots of them (the CTAs that run at once), so that neither lengths that differ
// nor a max_len far above them leave SMs without work. Of 32 candidate lengths from the mean on, in steps of an
// eighth of it, the first that fits is taken. Requests without queries take no part.
__device__ __forceinline__ int keys_of(const AttendArgs& a, int b)
{
    bool bad;
    const int n = cache_len(__ldg(a.lens + b), a.limit, bad);
    return __ldg(a.q_off + b + 1) > __ldg(a.q_off + b) ? n : 0;
}
__device__ __forceinline__ int chunks_of(int keys, int chunk)
{
    return (int)(((unsigned)keys + chunk - 1) / (unsigned)chunk);
}
__device__ __forceinline__ int chunk_keys(const AttendArgs& a)
{
    if (a.batch == 1) return max(64, (chunks_of(keys_of(a, 0), a.slots) + 63) & ~63);
    const int lane = threadIdx.x & 31;
    long long total = 0;
    for (int b = lane; b < a.batch; b += 32) total += keys_of(a, b);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    const long long mean = (total + a.slots - 1) / a.slots;
    const int c = max(64, (int)min((long long)kMostKeys, (mean + mean * lane / 8 + 63) & ~63ll));
    // ceil(n / c) as that of (n - 1/2) / c: below 2^21 keys the product's error cannot reach a
    // whole number; longer requests count with a margin (never fewer chunks than there are)
    const float inv = 1.f / (float)c;
    float count = 0.f;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
        float mine = b0 + lane < a.batch ? (float)keys_of(a, b0 + lane) : 0.f;
        mine = mine < 2097152.f ? fmaxf(mine - 0.5f, 0.f) : mine * 1.000001f;
        for (int x = 0; x < min(32, a.batch - b0); ++x) count += ceilf(__shfl_sync(0xffffffffu, mine, x) * inv);
    }
    const uint32_t fits = __ballot_sync(0xffffffffu, count <= (float)a.slots);
    return fits ? __shfl_sync(0xffffffffu, c, __ffs(fits) - 1) : (a.limit + 63) & ~63;
}
// The request that a slot is of (a.batch: none), and the slot's first key.
__device__ __forceinline__ void find_slot(const AttendArgs& a, int slot, int chunk, int& b, int& k0)
{
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
        const int n = b0 + lane < a.batch ? chunks_of(keys_of(a, b0 + lane), chunk) : 0;
        int sum = n;  // inclusive
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += y;
        }
        const uint32_t hit = __ballot_sync(0xffffffffu, slot < before + sum);
        if (hit) {
            const int x = __ffs(hit) - 1;
            b = b0 + x;
            k0 = (slot - before - __shfl_sync(0xffffffffu, sum - n, x)) * chunk;
            return;
        }
        before += __shfl_sync(0xffffffffu, sum, 31);
    }
    b = a.batch;
    k0 = 0;
}

// The n-th request with queries, by a warp.
__device__ __forceinline__ int find_active(const AttendArgs& a, int n)
{
    const int lane = threadIdx.x & 31;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
        const int b = min(b0 + lane, a.batch - 1);
        const bool there = b0 + lane < a.batch && __ldg(a.q_off + b + 1) > __ldg(a.q_off + b);
        const uint32_t mask = __ballot_sync(0xffffffffu, there);
        const uint32_t hit = __ballot_sync(0xffffffffu, there && __popc(mask & ((1u << lane) - 1u)) == n);
        if (hit) return b0 + __ffs(hit) - 1;
        n -= __popc(mask);
    }
    return a.batch;
}

// What every CTA of a request's tile needs to know of its rows.
struct RowTile {
    int len, t, row0, rows, last0;  // last0: position of the first query
    int group;
    // query of a row (a row's head is its key head's first plus the rest)
    __device__ __forceinline__ int query(int row) const { return t == 1 ? 0 : row / group; }
};

__device__ __forceinline__ RowTile row_tile(const AttendArgs& a, int b, int tile, int per)
{
    RowTile r;
    bool bad;
    r.len = cache_len(a.lens[b], a.limit, bad);
    if (bad && threadIdx.x == 0) atomicOr(a.err, kErrBounds);
    r.t = a.q_off[b + 1] - a.q_off[b];
    r.row0 = tile * per;
    r.rows = min(per, r.t * a.group - r.row0);
    r.last0 = r.len - r.t;
    r.group = a.group;
    return r;
}

// The launch of cache_tile.cu: `tiles` tiles of 128 or 256 rows for the longest request.
cudaError_t launch_attend_tiles(const AttendArgs& a, int head_dim, bool fp8, int row_tile, int tiles, cudaStream_t stream);

// The weights of a call of many rows, from their lse.
cudaError_t launch_attend_weights(const AttendArgs& a, int head_dim, bool fp8, int max_len, cudaStream_t stream);

}  // namespace lvs
