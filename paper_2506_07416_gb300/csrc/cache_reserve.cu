// Pages given to requests and taken back, and the slots of their new tokens.
//
// With hp = ceil(held / page), wp = ceil(want / page): a request takes wp - hp pages from
// the front of the ring of free ones, or puts hp - wp behind its end; both in the order of
// the requests, so a request's place in the ring is a prefix sum of the others'. Every CTA
// finds the sums for itself, which leaves its rows of the table, of the ring and of the slots
// without a word to the other CTAs: a page's number is read from the ring also where another CTA puts
// it into the table. Pages that are taken lie in the ring's first `count` places and pages that
// come back go behind them, so no CTA writes what another reads.
// What bounds it: the launch and a chain of loads, ring behind state behind lengths: 10 us for a decoding step of 128
// requests; 14 where 1024 requests come, go and grow and 1.6 million slots (13 MB) are written, which take 2 of it.

#include <algorithm>

#include "cache.cuh"

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
    // the warps' sums, by every warp
    longlong2 v = lane < (int)(blockDim.x >> 5) ? warp_s[lane] : make_longlong2(0, 0);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, v.x, d), b = __shfl_up_sync(0xffffffffu, v.y, d);
        if (lane >= d) v.x += a, v.y += b;
    }
    all.x = __shfl_sync(0xffffffffu, v.x, 31), all.y = __shfl_sync(0xffffffffu, v.y, 31);
    const long long bx = __shfl_sync(0xffffffffu, v.x, max(warp - 1, 0)), by = __shfl_sync(0xffffffffu, v.y, max(warp - 1, 0));
    return make_longlong2((warp ? bx : 0) + sx - x, (warp ? by : 0) + sy - y);
}

__global__ void __launch_bounds__(kThreads) reserve_kernel(const __grid_constant__ ReserveArgs a)
{
    // of the requests in hand, one a thread
    __shared__ int32_t off_s[kThreads + 1], want_s[kThreads], has_s[kThreads], need_s[kThreads];  // (need_s: ~need: refused)
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
    // place x from the head on, x < total (a 64-bit remainder took 3 us of a decoding step's call)
    auto ring = [&](int64_t x) { return head + x < total ? head + x : head + x - total; };
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
        // (the sum only grows: behind the first request that finds too few none takes a page; a ring that is none takes
        // nothing back either, and who wanted to give still holds what it held)
        const bool served = need == has || (need < has ? count >= 0 : taken + before.x + need - has <= count);
        if (tid < n) {
            want_s[tid] = want;
            has_s[tid] = has;
            need_s[tid] = served ? need : ~need;
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
            long long most = lane < threads >> 5 ? warp_s[lane].x : 0;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
            used = max(used, (int64_t)most);
        }
        taken += all.x, given += all.y;
        __syncthreads();
        // ---- pages: the few that most requests of a step take or give by the request's thread, more by a warp. Of a request
        // that is not served the entries of the pages that it wanted become -1: they may name pages that it gave back
        // and another request has by now
        const int64_t step = (int64_t)(threads >> 5) * gridDim.x;
        auto move = [&](int x, int o0, int by) {
            const int hp = has_s[x], np = need_s[x];
            int32_t* row = a.table + (int64_t)(b0 + x) * a.width;
            if (np < 0) {
                for (int o = hp + o0; o < ~np; o += by) row[o] = -1;
            } else if (np > hp) {
                for (int o = hp + o0; o < np; o += by) {
                    const int32_t p = __ldg(a.free + ring(from_s[x] + o - hp));
                    if (p < 0 || p >= total) atomicOr(a.err, kErrBounds);
                    row[o] = p;
                }
            } else {
                for (int o = np + o0; o < hp; o += by) {
                    const int64_t to = from_s[x] + o - np;
                    const int32_t p = row[o];
                    if (p < 0 || p >= total || to >= total) atomicOr(a.err, kErrBounds);
                    if (to < total) a.free[ring(to)] = p;
                }
            }
        };
        constexpr int kFewPages = 2;
        auto few = [&](int x) { return abs((need_s[x] < 0 ? ~need_s[x] : need_s[x]) - has_s[x]) <= kFewPages; };
        if (tid < n && tid % gridDim.x == blockIdx.x && few(tid)) move(tid, 0, 1);
        for (int x = (tid >> 5) * gridDim.x + blockIdx.x; x < n; x += (int)step)
            if (!few(x)) move(x, lane, 32);
        // ---- slots: a warp takes 256 neighbouring tokens, whose pages' numbers are all on their way at once
        const int64_t r0 = max(off_s[0], 0), r1 = min((int64_t)off_s[n], a.rows);
        constexpr int U = 8;
        for (int64_t q = r0 + 32 * U * ((int64_t)(tid >> 5) * gridDim.x + blockIdx.x); q < r1; q += 32 * U * step) {
            int x = last_before(n, [&](int y) { return off_s[y] <= q; });  // the request of the first token
            int32_t p[U], in[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t r = q + u * 32 + lane;
                p[u] = -1, in[u] = -1;
                if (r >= r1) continue;
                while (off_s[x + 1] <= r) ++x;
                if (need_s[x] < 0) continue;
                const int64_t pos = (int64_t)want_s[x] - off_s[x + 1] + r;
                in[u] = (int)(pos & ((1 << a.page_shift) - 1));
                if (pos < 0) continue;
                const int o = (int)(pos >> a.page_shift);
                p[u] = o < has_s[x] ? __ldg(a.table + (int64_t)(b0 + x) * a.width + o)
                                    : __ldg(a.free + ring(from_s[x] + o - has_s[x]));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t r = q + u * 32 + lane;
                if (r >= r1) continue;
                const bool there = p[u] >= 0 && p[u] < total;
                if (!there && in[u] >= 0) atomicOr(a.err, kErrBounds);
                a.slots[r] = there ? ((int64_t)p[u] << a.page_shift) + in[u] : -1;
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
    const int64_t ctas = std::max<int64_t>({1, (a.rows + 2047) / 2048, (a.batch + 127) / 128});
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
