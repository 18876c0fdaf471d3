// Pages given to requests and taken back, and the slots of their new tokens.
//
// With hp = ceil(held / page), wp = ceil(want / page): a request takes wp - hp pages from
// the front of the ring of free ones, or puts hp - wp behind its end; both in the order of
// the requests, so a request's place in the ring is a prefix sum of the others'. Every CTA
// finds the sums for itself, which leaves its rows of the table, of the ring and of the slots
// without a word to the other CTAs: a page's number is read from the ring also where another CTA puts
// it into the table. Pages that are taken lie in the ring's first `count` places and pages that
// come back go behind them, so no CTA writes what another reads.
// What bounds it: for a decoding step the launch and a chain of four loads; for prompts the 8 bytes
// written for every slot.

#include <algorithm>

#include "cache_index.h"
#include "internal.h"
#include "ptx.cuh"

namespace lvs {

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;

// Sums before this thread's of x and of y, over the CTA; `all` receives the totals.
__device__ __forceinline__ longlong2 scan2(long long x, long long y, longlong2* warp_s, longlong2& all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long sx = x, sy = y;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, sx, d), b = __shfl_up_sync(0xffffffffu, sy, d);
        if (lane >= d) sx += a, sy += b;
    }
    if (lane == 31) warp_s[warp] = make_longlong2(sx, sy);
    __syncthreads();
    longlong2 before = make_longlong2(0, 0);
    all = before;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) {
        const longlong2 v = warp_s[w];
        if (w < warp) before.x += v.x, before.y += v.y;
        all.x += v.x, all.y += v.y;
    }
    return make_longlong2(before.x + sx - x, before.y + sy - y);
}

__global__ void __launch_bounds__(kThreads) reserve_kernel(const __grid_constant__ ReserveArgs a)
{
    // of the requests in hand, one a thread
    __shared__ int32_t off_s[kThreads + 1], want_s[kThreads], has_s[kThreads], need_s[kThreads];
    __shared__ int64_t from_s[kThreads];  // place in the ring, from its head on, of the first page taken or given back
    __shared__ longlong2 warp_s[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x;
    griddep_wait();
    griddep_launch_dependents();
    const int64_t total = a.num_pages;
    int64_t head = __ldg(a.state), count = __ldg(a.state + 1);
    if (head < 0 || head >= total || count < 0 || count > total) {  // a ring that is none: nothing is taken or given
        if (blockIdx.x == 0 && tid == 0) atomicOr(a.err, kErrBounds);
        head = 0, count = -1;
    }
    long long taken = 0, given = 0;  // by the requests before
    int64_t used = 0;
    for (int b0 = 0; b0 < a.batch; b0 += threads) {
        const int n = min(threads, a.batch - b0);
        int held = 0, want = 0, has = 0, need = 0;
        if (tid < n) {
            bool bad, bad2;
            held = cache_len(__ldg(a.held + b0 + tid), a.limit, bad);
            want = cache_len(__ldg(a.want + b0 + tid), a.limit, bad2);
            if ((bad || bad2) && blockIdx.x == 0) atomicOr(a.err, kErrBounds);
            off_s[tid] = __ldg(a.off + b0 + tid);
            if (tid == n - 1) off_s[n] = __ldg(a.off + b0 + n);
            const int64_t round = (1 << a.page_shift) - 1;
            has = (int)((held + round) >> a.page_shift);
            need = (int)((want + round) >> a.page_shift);
        }
        longlong2 all;
        const longlong2 before = scan2(max(need - has, 0), max(has - need, 0), warp_s, all);
        // (the sum only grows: behind the first request that finds too few none takes a page)
        const bool served = need <= has || taken + before.x + need - has <= count;
        if (tid < n) {
            want_s[tid] = want;
            has_s[tid] = has;
            need_s[tid] = served ? need : -1;
            from_s[tid] = need > has ? taken + before.x : count + given + before.y;
            if (blockIdx.x == 0) a.granted[b0 + tid] = served ? want : held;
        }
        if (count >= 0) {
            // pages taken by the requests that are served: the largest end of theirs
            long long mine = tid < n && served && need > has ? taken + before.x + need - has : 0;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) mine = max(mine, __shfl_xor_sync(0xffffffffu, mine, d));
            __syncthreads();
            if (lane == 0) warp_s[tid >> 5].x = mine;
            __syncthreads();
            for (int w = 0; w < threads >> 5; ++w) used = max(used, (int64_t)warp_s[w].x);
        }
        taken += all.x, given += all.y;
        __syncthreads();
        // ---- pages, a request a warp
        const int step = (threads >> 5) * gridDim.x;
        for (int x = (tid >> 5) * gridDim.x + blockIdx.x; x < n; x += step) {
            const int hp = has_s[x], np = need_s[x];
            int32_t* row = a.table + (int64_t)(b0 + x) * a.width;
            if (np > hp) {
                for (int o = hp + lane; o < np; o += 32) {
                    const int32_t p = __ldg(a.free + (head + from_s[x] + o - hp) % total);
                    if (p < 0 || p >= total) atomicOr(a.err, kErrBounds);
                    row[o] = p;
                }
            } else if (np >= 0 && count >= 0) {
                for (int o = np + lane; o < hp; o += 32) {
                    const int64_t to = from_s[x] + o - np;
                    const int32_t p = row[o];
                    if (p < 0 || p >= total || to >= total) atomicOr(a.err, kErrBounds);
                    if (to < total) a.free[(head + to) % total] = p;
                }
            }
        }
        // ---- slots, four neighbouring tokens a thread
        const int64_t r0 = max(off_s[0], 0), r1 = min((int64_t)off_s[n], a.rows);
        const int64_t q0 = (r0 & ~3ll) + 4 * ((int64_t)blockIdx.x * threads + tid), q_step = 4ll * gridDim.x * threads;
        for (int64_t q = q0; q < r1; q += q_step) {
            int lo = 0, hi = n;
            const int64_t first = q > r0 ? q : r0;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (off_s[mid] <= first) lo = mid;
                else hi = mid;
            }
            long long s[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t r = q + e;
                s[e] = -1;
                if (r < r0 || r >= r1) continue;
                while (off_s[lo + 1] <= r) ++lo;
                if (need_s[lo] < 0) continue;
                const int64_t pos = (int64_t)want_s[lo] - off_s[lo + 1] + r;
                int32_t p = -1;
                if (pos >= 0) {
                    const int o = (int)(pos >> a.page_shift);
                    p = o < has_s[lo] ? __ldg(a.table + (int64_t)(b0 + lo) * a.width + o)
                                      : __ldg(a.free + (head + from_s[lo] + o - has_s[lo]) % total);
                }
                if (p >= 0 && p < total) s[e] = ((int64_t)p << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
                else atomicOr(a.err, kErrBounds);
            }
            if (q >= r0 && q + 4 <= r1 && a.vec) {
                reinterpret_cast<longlong2*>(a.slots + q)[0] = make_longlong2(s[0], s[1]);
                reinterpret_cast<longlong2*>(a.slots + q)[1] = make_longlong2(s[2], s[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (q + e >= r0 && q + e < r1) a.slots[q + e] = s[e];
            }
        }
        __syncthreads();
    }
    if (blockIdx.x == 0 && tid == 0) {
        if (count < 0) {
            a.new_state[0] = __ldg(a.state), a.new_state[1] = __ldg(a.state + 1);
        } else {
            a.new_state[0] = (int32_t)((head + used) % total);
            a.new_state[1] = (int32_t)(count - used + min((long long)(total - count), given));
        }
    }
}

}  // namespace

cudaError_t launch_cache_reserve(const ReserveArgs& a, int num_sms, cudaStream_t stream)
{
    // a CTA for every 2048 slots or 128 requests, no more than one an SM; small batches in small CTAs, whose scan is short
    const int threads = a.batch <= 128 ? 128 : (a.batch <= 256 ? 256 : kThreads);
    const int64_t ctas = std::max<int64_t>((a.rows + 2047) / 2048, (a.batch + 127) / 128);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min<int64_t>(ctas, num_sms), 1, 1);
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, reserve_kernel, a);
}

}  // namespace lvs
