// Verification of drafted tokens against the target's probabilities.
//
// Request b has T_b drafted tokens x_t with the draft model's probabilities q_t
// and the target's p_t (one row more: the token behind the last draft). Token t
// is taken while u_t * q_t[x_t] < p_t[x_t]. At the first refusal (or behind the
// last draft) one more token is sampled from w = max(p - q, 0) (w = p behind the
// last draft, or where no entry of p - q is above 0): the lowest index i with
// w_i > 0 and w_0 + .. + w_i > u * (w_0 + .. + w_V-1); where no sum passes (u >= 1),
// the last index with w_i > 0; -1 where there is none. NaN counts as 0.
//
// A cluster works on a request: each CTA adds up its part of the row, the CTAs
// exchange their sums, and the warp whose part holds the index reads its few
// hundred entries again. Only the one row of p and of q that is sampled is read.
//   Sums: fp64 is scarce here (2 additions a clock and SM: the largest batch
// would spend longer adding than reading), and fp32 sums would put the index one
// entry off in one draw of some dozens (V entries, each with its border). So
// p - q and the threads' sums are kept as unevaluated pairs of floats, about 48
// bits, by error-free transformations (Dekker's difference for p >= q >= 0,
// Knuth's two-sum); warps, CTAs and the search add in fp64.

#include "cache.cuh"

namespace lvs {

namespace {

constexpr int kVerifyThreads = 512;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyMaxCluster = 8;

__device__ __forceinline__ float prob(const float* p, int64_t i) { return __ldg(p + i); }
__device__ __forceinline__ float prob(const __nv_bfloat16* p, int64_t i) { return __bfloat162float(p[i]); }

// entry of w and its rounding error; an infinite entry has none
__device__ __forceinline__ float2 residual(float p, float q)
{
    const float w = p - q;
    if (!(w > 0.f)) return make_float2(0.f, 0.f);
    return make_float2(w, w <= 3.4028234e38f ? (p - w) - q : 0.f);
}

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

struct VerifyPart {
    double sum;
    int32_t last;  // last index with w > 0, or -1
    int32_t pad;
};

// What drafts of the row leave: MODE 0: p - q, 1: p with the entry x struck out, 2: p
template <int MODE, typename T>
__device__ __forceinline__ float2 entry(const T* p, const T* q, int32_t x, int i)
{
    if constexpr (MODE == 0) return residual(prob(p, i), prob(q, i));
    const float v = prob(p, i);
    return make_float2(v > 0.f && !(MODE == 1 && i == x) ? v : 0.f, 0.f);
}

// Sum and last positive index of the entries [i0, i1) of a warp's part
template <int MODE, typename T>
__device__ VerifyPart part_sum(const T* p, const T* q, int32_t x, int i0, int i1)
{
    const int lane = threadIdx.x & 31;
    float hi = 0.f, lo = 0.f;
    int last = -1;
    constexpr int U = 8;
    for (int i = i0 + lane; i < i1; i += 32 * U) {
        float2 w[U];
#pragma unroll
        for (int k = 0; k < U; ++k)
            w[k] = i + 32 * k < i1 ? entry<MODE>(p, q, x, i + 32 * k) : make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const float s = hi + w[k].x, t = s - hi;
            const float e = (hi - (s - t)) + (w[k].x - t);
            hi = s;
            if (s <= 3.4028234e38f) lo += e + w[k].y;
            if (w[k].x > 0.f) last = i + 32 * k;
        }
    }
    VerifyPart r;
    r.sum = warp_sum((double)hi + (double)lo);
    r.last = __reduce_max_sync(0xffffffffu, last);
    r.pad = 0;
    return r;
}

// The lowest index of [i0, i1) with w > 0 whose running sum (from `before` on)
// passes `bar`; the last one with w > 0 where rounding lets none pass.
template <int MODE, typename T>
__device__ int find(const T* p, const T* q, int32_t x, int i0, int i1, double before, double bar)
{
    const int lane = threadIdx.x & 31;
    int last = -1;
    for (int base = i0; base < i1; base += 32) {
        const int i = base + lane;
        const float2 w = i < i1 ? entry<MODE>(p, q, x, i) : make_float2(0.f, 0.f);
        double c = (double)w.x + (double)w.y;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(0xffffffffu, c, o);
            if (lane >= o) c += y;
        }
        c += before;
        const uint32_t pos = __ballot_sync(0xffffffffu, w.x > 0.f);
        const uint32_t hit = __ballot_sync(0xffffffffu, w.x > 0.f && c > bar);
        if (hit) return base + __ffs(hit) - 1;
        if (pos) last = base + 31 - __clz(pos);
        before = __shfl_sync(0xffffffffu, c, 31);
    }
    return last;
}

// Samples the token of one row; returns whether any entry was above 0. Called by
// the whole cluster; `slot`: this CTA's part in shared memory.
template <int MODE, typename T>
__device__ bool sample(const T* p, const T* q, int32_t x, int vocab, float u, VerifyPart* parts, VerifyPart* slot,
                       int32_t* out)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_ctarank(), ctas = (int)cluster_nctarank();
    // parts of a whole number of 32 entries for the cluster's warps
    const int nw = ctas * kVerifyWarps;
    const int per = ((vocab + nw - 1) / nw + 31) & ~31;
    const int64_t at = (int64_t)(rank * kVerifyWarps + warp) * per;
    const int i0 = (int)(at < vocab ? at : vocab), i1 = (int)(at + per < vocab ? at + per : vocab);
    const VerifyPart mine = part_sum<MODE>(p, q, x, i0, i1);
    if (lane == 0) parts[warp] = mine;
    __syncthreads();
    if (tid == 0) {
        VerifyPart c{0.0, -1, 0};
        for (int w = 0; w < kVerifyWarps; ++w) {
            c.sum += parts[w].sum;
            c.last = max(c.last, parts[w].last);
        }
        *slot = c;
    }
    cluster_sync_all();
    double total = 0.0, before = 0.0;
    int last = -1;
    {
        double sums[kVerifyMaxCluster];
        const uint32_t addr = smem_u32(slot);
        for (int r = 0; r < ctas; ++r) {
            const uint32_t a = mapa_shared(addr, (uint32_t)r);
            int l;
            asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(sums[r]) : "r"(a) : "memory");
            asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(l) : "r"(a + 8) : "memory");
            last = max(last, l);
            total += sums[r];
        }
        const double bar = (double)u * total;
        // the first CTA, then the first of its warps, whose running sum passes the bar
        double c = 0.0;
        int cta = -1;
        for (int r = 0; r < ctas && cta < 0; ++r) {
            before = c;
            c += sums[r];
            if (sums[r] > 0.0 && c > bar) cta = r;
        }
        if (last >= 0) {
            if (cta < 0) {
                if (rank == 0 && tid == 0) *out = last;
            } else if (cta == rank) {
                int w = -1;
                double cw = before, start = before;
                for (int k = 0; k < kVerifyWarps; ++k) {
                    start = w < 0 ? cw : start;
                    cw += parts[k].sum;
                    if (w < 0 && parts[k].sum > 0.0 && cw > bar) w = k;
                }
                if (w < 0) {  // the two orders of addition differ by a last bit: the CTA's last entry
                    if (tid == 0) *out = slot->last;
                } else if (w == warp) {
                    const int f = find<MODE>(p, q, x, i0, i1, start, bar);
                    if (lane == 0) *out = f;
                }
            }
        }
    }
    cluster_sync_all();  // the slots are free, and every CTA stays until its part has been read
    return last >= 0;
}

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) verify_kernel(const __grid_constant__ VerifyArgs a)
{
    __shared__ VerifyPart parts[kVerifyWarps];
    __shared__ VerifyPart slot;
    __shared__ int s_first;
    const int tid = threadIdx.x;
    const int b = blockIdx.y;
    const bool lead = cluster_ctarank() == 0;
    if (tid == 0) s_first = 0x7FFFFFFF;
    __syncthreads();
    griddep_wait();
    griddep_launch_dependents();
    const int t0 = a.off[b], n = a.off[b + 1] - t0;
    const T* P = static_cast<const T*>(a.p);
    const T* Q = static_cast<const T*>(a.q);
    // the first refused draft
    for (int t = tid; t < n; t += kVerifyThreads) {
        const int32_t x = a.tokens[t0 + t];
        bool take = false;
        if (x >= 0 && x < a.vocab) {
            const float px = prob(P, ((int64_t)t0 + b + t) * a.vocab + x);
            const float qx = Q ? prob(Q, ((int64_t)t0 + t) * a.vocab + x) : 1.f;
            take = (double)a.u[t0 + t] * (double)qx < (double)px;  // (an exact product)
        } else if (lead) {
            atomicOr(a.err, kErrBounds);
        }
        if (!take) atomicMin(&s_first, t);
    }
    __syncthreads();
    const int acc = min(s_first, n);
    int32_t* out = a.out + t0 + b;
    if (lead) {
        if (tid == 0) a.accepted[b] = acc;
        for (int t = tid; t <= n; t += kVerifyThreads) out[t] = t < acc ? a.tokens[t0 + t] : -1;
    }
    __syncthreads();
    const T* p = P + ((int64_t)t0 + b + acc) * a.vocab;
    const T* q = Q ? Q + ((int64_t)t0 + (acc < n ? acc : 0)) * a.vocab : nullptr;
    const float u = a.u_last[b];
    bool any = false;
    // (every CTA of the cluster takes the same branches; the token is written behind the
    // first cluster barrier, so after the lead CTA's -1)
    if (acc < n && Q) any = sample<0>(p, q, 0, a.vocab, u, parts, &slot, out + acc);
    else if (acc < n) any = sample<1>(p, q, a.tokens[t0 + acc], a.vocab, u, parts, &slot, out + acc);
    if (!any) sample<2>(p, q, 0, a.vocab, u, parts, &slot, out + acc);
}

}  // namespace

cudaError_t launch_verify(const VerifyArgs& a, bool bf16, cudaStream_t stream)
{
    if (a.batch <= 0) return cudaSuccess;
    // a CTA for every 2048 entries, up to a cluster of eight
    int ctas = 1;
    while (ctas < kVerifyMaxCluster && a.vocab > 2048 * ctas) ctas *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas, (unsigned)a.batch, 1);
    cfg.blockDim = dim3(kVerifyThreads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2] = {pdl_attribute(), {}};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ctas;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, bf16 ? verify_kernel<__nv_bfloat16> : verify_kernel<float>, a);
}

}  // namespace lvs
