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
// A cluster works on a request: each CTA adds up its part of the row, a sixteenth of it a
// warp, and the CTAs exchange their sums; the CTA whose part holds the index splits the
// warp's part that holds it over its sixteen warps again, and one warp searches the
// hundred entries that are left. Only the one row of p and of q that is sampled is read.
//   Sums: fp64 is scarce here (2 additions a clock and SM: the largest batch would spend
// longer adding than reading), and fp32 sums would put the index one entry off in one draw
// of some dozens (V entries, each with its border). So p - q and the sums of threads and
// warps are unevaluated pairs of floats, about 48 bits, by error-free transformations
// (Dekker's difference for p >= q >= 0, Knuth's two-sum); one warp adds the warps' and
// CTAs' sums in fp64. With every thread adding those, fp64 took 60 of 93 us.
//   64 requests of 0 to 8 drafts, 128003 floats a row (61 MB): 18 us, 9 of which are memory's; the
// rest is latency, tokens, their probabilities, two rounds of sums and a search one behind the other. In bf16 20 us: half
// the bytes, as many instructions and loads. Drafts that were certain (one row to read) 16, in bf16 17.
// One request of 32000 entries: 7 us.

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
    return make_float2(w > 0.f ? w : 0.f, w > 0.f && w <= 3.4028234e38f ? (p - w) - q : 0.f);
}

// (hi, lo) += (w, e)
__device__ __forceinline__ void add_pair(float& hi, float& lo, float w, float e)
{
    const float s = hi + w, t = s - hi;
    const float err = (hi - (s - t)) + (w - t) + e;
    hi = s;
    lo += s <= 3.4028234e38f ? err : 0.f;  // (an infinite sum has no error)
}

// What drafts of the row leave of its entry i: MODE 0: p - q, 1: p with the entry x struck out, 2: p
template <int MODE>
__device__ __forceinline__ float2 entry(float p, float q, int32_t x, int i)
{
    if constexpr (MODE == 0) return residual(p, q);
    return make_float2(p > 0.f && !(MODE == 1 && i == x) ? p : 0.f, 0.f);
}

struct VerifyShared {
    float2 sum[kVerifyWarps];   // the warps' sums
    int last[kVerifyWarps];     // their last indices with w > 0, or -1
    double cta_sum;             // read by the cluster
    int cta_last;
    int row_last;               // the last index of the whole row
    int part;                   // the warp whose part holds the index; -1: settled, or another CTA's
    double before, bar;         // sum before that part, and what the running sum has to pass
};

// The sixteen parts of [i0, i1): a whole number of 32 entries each.
__device__ __forceinline__ void part_of(int i0, int i1, int w, int& a, int& b)
{
    const int per = ((i1 - i0 + kVerifyWarps - 1) / kVerifyWarps + 31) & ~31;
    const long long at = (long long)i0 + (long long)w * per;
    a = (int)(at < i1 ? at : i1);
    b = i1 - a < per ? i1 : a + per;
}

// Sums and last positive indices of the warps' parts of [i0, i1), into shared memory.
template <int MODE, typename T>
__device__ void part_sums(const T* p, const T* q, int32_t x, int i0, int i1, VerifyShared& sh)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int a, b;
    part_of(i0, i1, warp, a, b);
    float hi = 0.f, lo = 0.f;
    int last = -1;
    constexpr int U = 8;  // entries of a lane on their way, and as many being added
    float pn[U], qn[U];
    auto load = [&](int i) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            pn[k] = i + 32 * k < b ? prob(p, i + 32 * k) : 0.f;
            qn[k] = MODE == 0 && i + 32 * k < b ? prob(q, i + 32 * k) : 0.f;
        }
    };
    load(a + lane);
#pragma unroll 1
    for (int i = a + lane; i < b; i += 32 * U) {
        float pc[U], qc[U];
#pragma unroll
        for (int k = 0; k < U; ++k) pc[k] = pn[k], qc[k] = qn[k];
        load(i + 32 * U);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const float2 w = entry<MODE>(pc[k], qc[k], x, i + 32 * k);
            add_pair(hi, lo, w.x, w.y);
            if (w.x > 0.f) last = i + 32 * k;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float h2 = __shfl_xor_sync(0xffffffffu, hi, o), l2 = __shfl_xor_sync(0xffffffffu, lo, o);
        add_pair(hi, lo, h2, l2);
    }
    last = __reduce_max_sync(0xffffffffu, last);
    if (lane == 0) {
        sh.sum[warp] = make_float2(hi, lo);
        sh.last[warp] = last;
    }
}

// Inclusive sums over the lanes.
__device__ __forceinline__ double scan(double v, int lanes)
{
    const int lane = threadIdx.x & 31;
    for (int o = 1; o < lanes; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += y;
    }
    return v;
}

// By warp 0: the part of the warps' sums whose running sum from `before` on passes sh.bar (the
// last with an entry above 0 where rounding lets none pass).
__device__ __forceinline__ void pick_part(double before, VerifyShared& sh)
{
    const int lane = threadIdx.x & 31;
    const float2 s = lane < kVerifyWarps ? sh.sum[lane] : make_float2(0.f, 0.f);
    const double v = (double)s.x + (double)s.y, c = before + scan(v, kVerifyWarps);
    const uint32_t some = __ballot_sync(0xffffffffu, v > 0.0), hit = __ballot_sync(0xffffffffu, v > 0.0 && c > sh.bar);
    const int w = hit ? __ffs(hit) - 1 : 31 - __clz(some | 1u);
    if (lane == w) {
        sh.part = w;
        sh.before = c - v;
    }
}

// Samples the token of one row; returns whether any entry was above 0. Called by the whole
// cluster.
template <int MODE, typename T>
__device__ bool sample(const T* p, const T* q, int32_t x, int vocab, float u, VerifyShared& sh, int32_t* out)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = (int)cluster_ctarank(), ctas = (int)cluster_nctarank();
    const int per = ((vocab + ctas - 1) / ctas + 31) & ~31;
    const long long at = (long long)rank * per;
    const int i0 = (int)(at < vocab ? at : vocab), i1 = vocab - i0 < per ? vocab : i0 + per;
    part_sums<MODE>(p, q, x, i0, i1, sh);
    __syncthreads();
    if (warp == 0) {
        const float2 s = lane < kVerifyWarps ? sh.sum[lane] : make_float2(0.f, 0.f);
        const double sum = scan((double)s.x + (double)s.y, kVerifyWarps);
        const int last = __reduce_max_sync(0xffffffffu, lane < kVerifyWarps ? sh.last[lane] : -1);
        if (lane == kVerifyWarps - 1) {
            sh.cta_sum = sum;
            sh.cta_last = last;
            sh.part = -1;
        }
    }
    cluster_sync_all();
    if (warp == 0) {
        double v = 0.0;
        int last = -1;
        if (lane < ctas) {
            const uint32_t r = (uint32_t)lane;
            asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(mapa_shared(smem_u32(&sh.cta_sum), r)) : "memory");
            asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(last) : "r"(mapa_shared(smem_u32(&sh.cta_last), r)) : "memory");
        }
        const double c = scan(v, kVerifyMaxCluster);
        const double bar = (double)u * __shfl_sync(0xffffffffu, c, ctas - 1);
        const uint32_t hit = __ballot_sync(0xffffffffu, lane < ctas && v > 0.0 && c > bar);
        last = __reduce_max_sync(0xffffffffu, last);
        const double before = __shfl_sync(0xffffffffu, c - v, rank);
        if (lane == 0) {
            sh.row_last = last;
            sh.bar = bar;
        }
        __syncwarp();
        if (hit && __ffs(hit) - 1 == rank) pick_part(before, sh);
        else if (!hit && last >= 0 && rank == 0 && lane == 0) *out = last;
    }
    __syncthreads();
    const int part = sh.part;
    const double first = sh.before, bar = sh.bar;
    if (part >= 0) {
        int a, b;
        part_of(i0, i1, part, a, b);
        __syncthreads();  // (everyone has read what the second round overwrites)
        part_sums<MODE>(p, q, x, a, b, sh);
        __syncthreads();
        if (warp == 0) pick_part(first, sh);
        __syncthreads();
        if (warp == sh.part) {
            int s0, s1;
            part_of(a, b, warp, s0, s1);
            double before = sh.before;
            int found = -1;
            for (int base = s0; base < s1; base += 32) {
                const int i = base + lane;
                const float2 w = i < s1 ? entry<MODE>(prob(p, i), MODE == 0 ? prob(q, i) : 0.f, x, i) : make_float2(0.f, 0.f);
                const double c = before + scan((double)w.x + (double)w.y, 32);
                const uint32_t pos = __ballot_sync(0xffffffffu, w.x > 0.f);
                const uint32_t hit = __ballot_sync(0xffffffffu, w.x > 0.f && c > bar);
                if (pos) found = base + 31 - __clz(pos);
                if (hit) {
                    found = base + __ffs(hit) - 1;
                    break;
                }
                before = __shfl_sync(0xffffffffu, c, 31);
            }
            if (lane == 0) *out = found;
        }
    }
    cluster_sync_all();  // every CTA stays until its sums have been read
    return sh.row_last >= 0;
}

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) verify_kernel(const __grid_constant__ VerifyArgs a)
{
    __shared__ VerifyShared sh;
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
    if (acc < n && Q) any = sample<0>(p, q, 0, a.vocab, u, sh, out + acc);
    else if (acc < n) any = sample<1>(p, q, a.tokens[t0 + acc], a.vocab, u, sh, out + acc);
    if (!any) sample<2>(p, q, 0, a.vocab, u, sh, out + acc);
}

}  // namespace

cudaError_t launch_verify(const VerifyArgs& a, bool bf16, int num_sms, cudaStream_t stream)
{
    if (a.batch <= 0) return cudaSuccess;
    // a CTA for every 2048 entries, up to a cluster of eight, while the batch's CTAs run at once
    // (two on an SM)
    int ctas = 1;
    while (ctas < kVerifyMaxCluster && a.vocab > 2048 * ctas && 2 * ctas * a.batch <= 2 * num_sms) ctas *= 2;
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
