// Eviction from the 4-bit cache by accumulated attention weight.
//
// Of a request of n > budget tokens stay: the first `sink`, the last `recent`,
// and of the rest those with the largest weight (NaN below every number, -0 equal
// to +0, ties to the lower position) until `budget` are kept; their rows move, in
// order, to the front of the request's pages or to pages of their own.
//
// evict_select_kernel: a cluster per request. Weights become order-preserving
// 32-bit keys in shared memory (protected tokens above all others); a radix select
// of 4 passes of 8 bits adds up the CTAs' histograms through distributed shared
// memory, one cluster barrier a pass; two counts in index order give every kept
// token its place. evict_move_kernel: a CTA moves rows of some heads, 16 bytes a
// thread. In place a CTA moves all of a head's rows, a batch of rows at a time:
// every load of a batch ends before its first store, and since the kept rows
// ascend (row i comes from a position >= i), no store touches a row of a later
// batch.
// 64 requests of up to 8162 tokens cut to 2048, 8 heads (300 MB): 79 us, 16 of selecting (cluster
// barriers) and 61 of moving at 5.6 TB/s of DRAM traffic: a picked row's scales are 8 of a sector's 32
// bytes. A request of 560 tokens: 10 us, latency. The same 64 requests in place: 190 us, one of 8191 tokens and 4 heads
// 150: a CTA's 128 threads move a head's rows 32 at a time, one round trip to memory after another.

#include <type_traits>

#include "cache.cuh"

namespace lvs {

namespace {

constexpr int kSelThreads = 512;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelMaxCluster = 8;
constexpr int kSelSmemKeys = 48 * 1024;  // keys of a CTA in shared memory (192 KB); the rest is read again

__device__ __forceinline__ uint32_t weight_key(float f)
{
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0u;  // NaN ranks below everything
    if (u == 0x80000000u) u = 0u;                    // -0 equals +0
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ int ld_cluster_i32(uint32_t addr)
{
    int v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const __grid_constant__ EvictArgs a, int smem_keys)
{
    extern __shared__ uint32_t keys_s[];
    __shared__ uint32_t hist[2][256];
    __shared__ uint32_t tot[256];
    __shared__ int warp_gt[kSelWarps], warp_eq[kSelWarps];
    __shared__ int cta_count[2];
    __shared__ uint32_t s_digit, s_above;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.y;
    const int rank = (int)cluster_ctarank(), ctas = (int)cluster_nctarank();
    griddep_wait();
    griddep_launch_dependents();
    bool bad_len;
    const int n = cache_len(a.lens[b], a.limit, bad_len);
    const int k = n < a.budget ? n : a.budget;
    int32_t* kept = a.kept + (int64_t)b * a.budget;
    if (rank == 0 && tid == 0) {
        a.new_lens[b] = k;
        if (bad_len) atomicOr(a.err, kErrBounds);
    }
    for (int i = k + rank * kSelThreads + tid; i < a.budget; i += ctas * kSelThreads) kept[i] = -1;
    if (n <= a.budget) {
        for (int i = rank * kSelThreads + tid; i < n; i += ctas * kSelThreads) kept[i] = i;
        return;
    }
    const int per = ((n + ctas - 1) / ctas + 31) & ~31;
    const int j0 = min(n, rank * per), j1 = min(n, j0 + per);
    auto read_key = [&](int j) -> uint32_t {
        if (j < a.sink || j >= n - a.recent) return 0xFFFFFFFFu;
        const int32_t page = cache_page(a.cache.table, a.cache.width, a.cache.num_pages, a.cache.page_shift, b, j);
        if (page < 0) {
            atomicOr(a.err, kErrBounds);
            return 0u;
        }
        return weight_key(
            a.weights[((int64_t)page << a.cache.page_shift) + (j & ((1 << a.cache.page_shift) - 1))]);
    };
    const bool in_smem = per <= smem_keys;
    if (in_smem) {
        for (int j = j0 + tid; j < j1; j += kSelThreads) keys_s[j - j0] = read_key(j);
    }
    for (int i = tid; i < 512; i += kSelThreads) (&hist[0][0])[i] = 0u;
    __syncthreads();
    auto key_at = [&](int j) -> uint32_t { return in_smem ? keys_s[j - j0] : read_key(j); };

    // ---- the k-th largest key: the digits from the highest on
    uint32_t prefix = 0u, mask = 0u;
    int remaining = k;
    for (int pass = 0; pass < 4; ++pass) {
        const int shift = 24 - 8 * pass;
        uint32_t* h = hist[pass & 1];
        if (pass >= 2) {  // last read two passes ago, before the barrier of the pass between
            if (tid < 256) h[tid] = 0u;
            __syncthreads();
        }
        for (int base = j0 + warp * 32; base < j1; base += kSelThreads) {
            const int j = base + lane;
            uint32_t bin = 256u;
            if (j < j1) {
                const uint32_t u = key_at(j);
                if ((u & mask) == prefix) bin = (u >> shift) & 0xFFu;
            }
            const uint32_t peers = __match_any_sync(0xffffffffu, bin);
            if (bin < 256u && lane == __ffs(peers) - 1) atomicAdd(&h[bin], (uint32_t)__popc(peers));
        }
        cluster_sync_all();
        if (tid < 256) {
            uint32_t s = 0;
            const uint32_t addr = smem_u32(&h[tid]);
            for (int r = 0; r < ctas; ++r) s += (uint32_t)ld_cluster_i32(mapa_shared(addr, (uint32_t)r));
            tot[tid] = s;
        }
        __syncthreads();
        if (warp == 0) {
            uint32_t c[8], sum = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                c[e] = tot[lane * 8 + e];
                sum += c[e];
            }
            uint32_t suf = sum;  // over the lanes from this one on
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y = __shfl_down_sync(0xffffffffu, suf, o);
                if (lane + o < 32) suf += y;
            }
            uint32_t above = suf - sum;
            if (above < (uint32_t)remaining && (uint32_t)remaining <= suf) {
#pragma unroll
                for (int e = 7; e >= 0; --e) {
                    if (above + c[e] >= (uint32_t)remaining) {
                        s_digit = (uint32_t)(lane * 8 + e);
                        s_above = above;
                        break;
                    }
                    above += c[e];
                }
            }
        }
        __syncthreads();
        prefix |= s_digit << shift;
        mask |= 0xFFu << shift;
        remaining -= (int)s_above;
    }

    // ---- places: keys above prefix, and the first `remaining` equal to it, in index order
    const int seg = ((j1 - j0 + kSelWarps - 1) / kSelWarps + 31) & ~31;
    const int w0 = min(j1, j0 + warp * seg), w1 = min(j1, w0 + seg);
    int n_gt = 0, n_eq = 0;
    for (int base = w0; base < w1; base += 32) {
        const int j = base + lane;
        const uint32_t u = j < w1 ? key_at(j) : 0u;
        n_gt += __popc(__ballot_sync(0xffffffffu, j < w1 && u > prefix));
        n_eq += __popc(__ballot_sync(0xffffffffu, j < w1 && u == prefix));
    }
    if (lane == 0) {
        warp_gt[warp] = n_gt;
        warp_eq[warp] = n_eq;
    }
    __syncthreads();
    if (tid < 2) {
        int s = 0;
        for (int w = 0; w < kSelWarps; ++w) s += tid == 0 ? warp_gt[w] : warp_eq[w];
        cta_count[tid] = s;
    }
    cluster_sync_all();
    int gt = 0, eq = 0;
    for (int r = 0; r < rank; ++r) {
        const uint32_t addr = mapa_shared(smem_u32(cta_count), (uint32_t)r);
        gt += ld_cluster_i32(addr);
        eq += ld_cluster_i32(addr + 4);
    }
    for (int w = 0; w < warp; ++w) {
        gt += warp_gt[w];
        eq += warp_eq[w];
    }
    const uint32_t below = (1u << lane) - 1u;
    for (int base = w0; base < w1; base += 32) {
        const int j = base + lane;
        const uint32_t u = j < w1 ? key_at(j) : 0u;
        const uint32_t m_gt = __ballot_sync(0xffffffffu, j < w1 && u > prefix);
        const uint32_t m_eq = __ballot_sync(0xffffffffu, j < w1 && u == prefix);
        const int my_eq = eq + __popc(m_eq & below);
        const bool keep = ((m_gt >> lane) & 1u) || (((m_eq >> lane) & 1u) && my_eq < remaining);
        if (keep) kept[gt + __popc(m_gt & below) + min(my_eq, remaining)] = j;
        gt += __popc(m_gt);
        eq += __popc(m_eq);
    }
    cluster_sync_all();  // every CTA stays until its counts have been read
}

constexpr int kMoveThreads = 128;
constexpr int kMoveRows = 2;  // rows of a thread in flight

// Rows [first, first + rows_per_cta) of the heads [h0, h0 + heads_per_cta). Where a row comes
// from and goes to is the same for every head, so a CTA finds that once and then moves head
// after head.
template <int D, bool INPLACE>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ EvictArgs a, int rows_per_cta,
                                                                  int heads_per_cta)
{
    constexpr int VECS = D / 32;      // 16-byte vectors of a row's codes
    constexpr int LANES = 2 * VECS;   // threads of a row: the vectors of K, then those of V
    constexpr int BATCH = kMoveThreads / LANES * kMoveRows;
    using Scales = typename std::conditional<D == 128, uint2, uint32_t>::type;  // of a row of one head
    const int e = threadIdx.x % LANES, t = e / VECS, vec = e % VECS;
    const int b = blockIdx.z, h0 = blockIdx.y * heads_per_cta, h1 = min(a.cache.hkv, h0 + heads_per_cta);
    const int shift = a.cache.page_shift, smask = (1 << shift) - 1;
    griddep_wait();
    griddep_launch_dependents();
    const int k = a.new_lens[b];
    const int32_t* kept = a.kept + (int64_t)b * a.budget;
    const int first = blockIdx.x * rows_per_cta, end = min(k, first + rows_per_cta);
    uint8_t* const codes = a.cache.codes[t] + vec * 16;
    uint8_t* const scales = a.cache.scales[t];
    for (int base = first; base < end; base += BATCH) {
        int64_t from[kMoveRows], to[kMoveRows];  // rows of head 0; -1: nothing to move
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u) {
            const int i = base + u * (BATCH / kMoveRows) + threadIdx.x / LANES;
            from[u] = to[u] = -1;
            if (i >= end) continue;
            const int j = __ldcg(kept + i);
            if (INPLACE && j == i) continue;
            const int32_t from_page =
                j < 0 ? -1 : cache_page(a.cache.table, a.cache.width, a.cache.num_pages, shift, b, j);
            const int32_t to_page = cache_page(a.to_table, a.to_width, a.cache.num_pages, shift, b, i);
            if (from_page < 0 || to_page < 0) {
                if (e == 0) atomicOr(a.err, kErrBounds);
                continue;
            }
            from[u] = cache_row(from_page, a.cache.hkv, 0, shift, j & smask);
            to[u] = cache_row(to_page, a.cache.hkv, 0, shift, i & smask);
        }
        if (h0 == 0) {
            float w[kMoveRows];
            // (slots of the weights: a page has one row of them where it has hkv rows of each head)
            auto slot = [&](int64_t row) { return ((row >> shift) / a.cache.hkv << shift) + (row & smask); };
            if (e == 0)
#pragma unroll
                for (int u = 0; u < kMoveRows; ++u) w[u] = to[u] >= 0 ? a.weights[slot(from[u])] : 0.f;
            if constexpr (INPLACE) __syncthreads();
            if (e == 0)
#pragma unroll
                for (int u = 0; u < kMoveRows; ++u)
                    if (to[u] >= 0) a.weights[slot(to[u])] = w[u];
        }
#pragma unroll 1
        for (int h = h0; h < h1; ++h) {
            uint4 code[kMoveRows];
            Scales scale[kMoveRows];
            const int64_t head = (int64_t)h << shift;
#pragma unroll
            for (int u = 0; u < kMoveRows; ++u) {
                if (to[u] < 0) continue;
                code[u] = __ldcg(reinterpret_cast<const uint4*>(codes + (from[u] + head) * (D / 2)));
                if (vec == 0) scale[u] = *reinterpret_cast<const Scales*>(scales + (from[u] + head) * (D / 16));
            }
            if constexpr (INPLACE) __syncthreads();
#pragma unroll
            for (int u = 0; u < kMoveRows; ++u) {
                if (to[u] < 0) continue;
                *reinterpret_cast<uint4*>(codes + (to[u] + head) * (D / 2)) = code[u];
                if (vec == 0) *reinterpret_cast<Scales*>(scales + (to[u] + head) * (D / 16)) = scale[u];
            }
        }
    }
}

}  // namespace

cudaError_t launch_cache_evict(const EvictArgs& a, int head_dim, int num_sms, cudaStream_t stream, int32_t* launches)
{
    *launches = 0;
    if (a.batch <= 0) return cudaSuccess;
    // a CTA for every 2048 tokens of a request, while the batch leaves SMs free
    int ctas = 1;
    while (ctas < kSelMaxCluster && a.limit > 2048 * ctas && 2 * ctas * a.batch <= 2 * num_sms) ctas *= 2;
    const int per = ((a.limit + ctas - 1) / ctas + 31) & ~31;
    const int keys = per < kSelSmemKeys ? per : kSelSmemKeys;
    cudaError_t e = cudaSuccess;
    if (keys * 4 > 40 * 1024)  // more than a launch has without asking, beside the static arrays
        e = cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelSmemKeys * 4);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas, (unsigned)a.batch, 1);
    cfg.blockDim = dim3(kSelThreads, 1, 1);
    cfg.dynamicSmemBytes = (size_t)keys * 4;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2] = {pdl_attribute(), {}};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ctas;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, evict_select_kernel, a, keys);
    if (e != cudaSuccess) return e;
    *launches = 1;

    const bool inplace = a.to_table == a.cache.table;
    const int most = a.limit < a.budget ? a.limit : a.budget;
    const int batch_rows = kMoveThreads / (head_dim / 16) * kMoveRows;
    const int rows = inplace ? most : batch_rows;
    if (most <= 0) return cudaSuccess;
    const int64_t chunks = (most + rows - 1) / rows * (int64_t)a.batch;
    // heads of a CTA: eight, fewer while that leaves SMs without work
    int heads = inplace ? 1 : 8;
    while (heads > 1 && chunks * ((a.cache.hkv + heads - 1) / heads) < 4 * (int64_t)num_sms) heads /= 2;
    cudaLaunchConfig_t mv = {};
    mv.gridDim = dim3((unsigned)((most + rows - 1) / rows), (unsigned)((a.cache.hkv + heads - 1) / heads),
                      (unsigned)a.batch);
    mv.blockDim = dim3(kMoveThreads, 1, 1);
    mv.stream = stream;
    mv.attrs = attr;
    mv.numAttrs = 1;
    auto kern = head_dim == 128 ? (inplace ? evict_move_kernel<128, true> : evict_move_kernel<128, false>)
                                : (inplace ? evict_move_kernel<64, true> : evict_move_kernel<64, false>);
    e = cudaLaunchKernelEx(&mv, kern, a, rows, heads);
    if (e == cudaSuccess) *launches = 2;
    return e;
}

}  // namespace lvs
