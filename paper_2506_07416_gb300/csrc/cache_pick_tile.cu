// Scores of a cache's pages for many queries (chunks of a prompt), on the fifth-generation tensor cores.
//
// The product is that of cache_pick.cu, [pages, 2 d] x [2 d, columns] with a column for each query head of a query,
// in f16 whole numbers with fp32 sums (exact). Pages are the M rows, so that a thread reads its page's columns from
// tensor memory and finds the largest of a query's heads without another lane's help. A CTA takes a key head of a request,
// 128 columns (16 queries of eight padded heads) and all pages that they see, 128 at a time. Its warps:
//   all lay out the queries once, K-major and swizzled;
//   eight make f16 of the codes of the next 128 pages (two stages), their bytes on the way one tile ahead;
//   one issues the contraction into one of two places in tensor memory;
//   eight turn the last one's columns into keys and write them, neighbouring pages by neighbouring lanes.
// What bounds it: the chain codes - contraction - keys, and a CTA's start, two fifths of its time. A chunk of a prompt, 777
// and 1024 queries of 28 / 4 heads over up to 512 pages of 64: 27 us, 38 with the picking (45 with four warps making the
// codes and the pages of a tile found when it is due); 64 columns a CTA and two CTAs an SM took a microsecond more.

#include <algorithm>

#include "cache_pick.cuh"
#include "pipe.cuh"

namespace lvs {

namespace {

constexpr int kCols = 128, kTilePages = 128;
constexpr int kOutWarps = 8, kCodeWarps = 8, kMmaWarp = kOutWarps + kCodeWarps;
constexpr int kPickThreads = 32 * (kMmaWarp + 1);
constexpr int kAtom = 128 * 128;  // 128 rows of 64 f16
enum { P_A_FULL = 0, P_A_FREE = 2, P_D_FULL = 4, P_D_FREE = 6, P_DRAIN = 8, P_COUNT };

template <int D>
struct PickLayout {
    static constexpr int ROWS = 2 * D / 64 * kAtom;
    static constexpr int Q = 0, A = ROWS;  // two stages of pages
    static constexpr int BAR = 3 * ROWS;
    static constexpr int MISC = BAR + 8 * P_COUNT;
    static constexpr int ALLOC = MISC + 16 + 1024;
};

__device__ __forceinline__ void st_shared16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

template <int D, bool FP8>
__global__ void __launch_bounds__(kPickThreads, 1) pick_tile_kernel(const __grid_constant__ PickArgs a, int blocks)
{
    using L = PickLayout<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - raw);
    auto BAR = [&](int i) { return base + L::BAR + 8 * i; };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::MISC);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::MISC + 4);
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = uniform(tid >> 5);
    const int h = blockIdx.y % a.hkv, part = blockIdx.y / a.hkv, b = blockIdx.z;
    griddep_wait();
    griddep_launch_dependents();
    const int padded = padded_group(a.group);
    const ScoreTile st = score_tile(a, b, part, max(1, kCols / padded));
    const int n_tiles = uniform((st.pages + kTilePages - 1) / kTilePages);  // of which this CTA takes every `blocks`-th
    const int mine = uniform(n_tiles > (int)blockIdx.x ? (n_tiles - 1 - (int)blockIdx.x) / blocks + 1 : 0);
    if (mine == 0) return;
    auto first_page = [&](int n) { return ((int)blockIdx.x + n * blocks) * kTilePages; };

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(BAR(P_A_FULL + i), kCodeWarps);
            mbar_init(BAR(P_A_FREE + i), 1);
            mbar_init(BAR(P_D_FULL + i), 1);
            mbar_init(BAR(P_D_FREE + i), kOutWarps);
        }
        mbar_init(BAR(P_DRAIN), 1);
        *abort_flag = 0;
        fence_mbar_init_cluster();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(tmem_slot), 256);
        tmem_relinquish();
    }
    const Ctl ctl{abort_flag, a.err, a.wait_budget};
    auto find = [&](int64_t o) -> int32_t {
        return o < st.pages ? cache_page(a.table, a.width, a.num_pages, a.page_shift, b, o << a.page_shift) : -1;
    };
    // ---- of the code warps w the pages [16 w, 16 w + 16) of a tile: a load takes whole pages, 16 channels of largest or
    // smallest a lane; the first tile's are on their way while the queries are laid out
    constexpr int LANES = 2 * D / 16, PER = 32 / LANES, LOADS = 16 / PER;  // lanes of a page, pages a load
    const int w = warp - kOutWarps, sub = lane % LANES, at = lane / LANES;
    uint4 next[LOADS];
    int32_t found = -1;  // page of row lane % 16
    auto load = [&]() {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int32_t p = __shfl_sync(0xffffffffu, found, i * PER + at);
            next[i] = __ldg(reinterpret_cast<const uint4*>(a.codes + ((int64_t)max(p, 0) * a.hkv + h) * 2 * D) + sub);
        }
    };
    if (warp >= kOutWarps && warp < kMmaWarp) {
        found = find(first_page(0) + w * 16 + (lane & 15));
        load();
        if (mine > 1) found = find(first_page(1) + w * 16 + (lane & 15));
    }
    // ---- the queries: column n of the operand is row n, channel ch its K index (and D + ch)
    if (warp < kMmaWarp) {
        for (int x = warp; x < kCols / padded; x += kMmaWarp)  // (zeros behind the last query)
            stage_query<D, FP8>(a, st.q0 + st.i0 + min(x, st.queries - 1), h, x < st.queries, padded, x * padded,
                                [&](int col, int ch, __half2 r0, __half2 r1) {
                                    const auto put = [&](int k, __half2 v0, __half2 v1) {
                                        uint2* to = reinterpret_cast<uint2*>(smem + L::Q + (k >> 6) * kAtom + col * 128 +
                                                                             ((((k >> 3) & 7) ^ (col & 7)) << 4) + (k & 7) * 2);
                                        *to = make_uint2(h2_bits(v0), h2_bits(v1));
                                    };
                                    const __half2 zero = bits_h2(0u);
                                    put(ch, __hmax2(r0, zero), __hmax2(r1, zero));
                                    put(D + ch, __hmin2(r0, zero), __hmin2(r1, zero));
                                });
        fence_proxy_async_shared();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(*tmem_slot);

    if (warp < kOutWarps) {
        // ---------------------------------------------------------------- keys: a page a thread
        // (two warps share the 32 pages that their lanes may read, and the columns where a query has one half's alone)
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const bool halves = kCols / 2 % padded == 0;
        const int row = tid & 127, col0 = halves ? (warp >> 2) * (kCols / 2) : 0;
        const int cols = halves ? min(kCols / 2, st.queries * padded - col0) : (warp < 4 ? st.queries * padded : 0);
        // the page and its unit are found a tile ahead
        auto exps_of = [&](int32_t page) { return (int)__ldg(a.exps + (int64_t)max(page, 0) * a.hkv + h); };
        int32_t next_page = find(first_page(0) + row);
        int next_exp = exps_of(next_page);
        for (int n = 0; n < mine; ++n) {
            const int o = first_page(n) + row;
            const int32_t page = next_page;
            const float unit = __uint_as_float((uint32_t)(127 + min(max(next_exp, -100), 100)) << 23);
            if (n + 1 < mine) {
                next_page = find(first_page(n + 1) + row);
                next_exp = exps_of(next_page);
            }
            if (page < 0 && o < st.pages && warp < 4) atomicOr(a.err, kErrBounds);
            uint32_t* out = a.keys + ((int64_t)(st.q0 + st.i0 + col0 / padded) * a.hkv + h) * a.key_stride + o;
            const int64_t step = (int64_t)a.hkv * a.key_stride;
            auto put = [&](float s) {  // of the next query
                if (o < st.pages) *out = page >= 0 ? score_key(s * unit) : 1u;
                out += step;
            };
            if (!poll_phase_warp(BAR(P_D_FULL + (n & 1)), (uint32_t)(n >> 1) & 1u, ctl)) break;
            tc_fence_after();
            float best = -INFINITY;
            int left = padded;  // columns of the query in hand
#pragma unroll 1
            for (int c0 = 0; c0 < cols; c0 += 32) {
                float v[32];
                tmem_ld32(tmem + lanes + (n & 1) * kCols + col0 + c0, v);
                tmem_wait_ld();
                if (padded == 8) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (c0 + 8 * q < cols)
                            put(fmax3(fmax3(v[8 * q], v[8 * q + 1], v[8 * q + 2]), fmax3(v[8 * q + 3], v[8 * q + 4], v[8 * q + 5]),
                                      fmaxf(v[8 * q + 6], v[8 * q + 7])));
                } else if (padded == 4) {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (c0 + 4 * q < cols) put(fmaxf(fmax3(v[4 * q], v[4 * q + 1], v[4 * q + 2]), v[4 * q + 3]));
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        if (c0 + i >= cols) break;
                        best = fmaxf(best, v[i]);
                        if (--left == 0) {
                            put(best);
                            best = -INFINITY, left = padded;
                        }
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(P_D_FREE + (n & 1)));
        }
    } else if (warp < kMmaWarp) {
        // ---------------------------------------------------------------- codes to f16
        // (of eight neighbouring lanes the first four write their first 16 bytes first, the others their second, so that
        // they cover all banks)
        const int k0 = sub * 16, unit0 = (k0 >> 3) & 7, swap = (sub >> 2) & 1;
        for (int n = 0; n < mine; ++n) {
            const int stage = n & 1;
            if (a.stall && n == min(1, mine - 1)) break;
            if (n >= 2 && !poll_phase_warp(BAR(P_A_FREE + stage), (uint32_t)(n / 2 - 1) & 1u, ctl)) break;
            const uint32_t to = base + L::A + stage * L::ROWS + (k0 >> 6) * kAtom;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int row = w * 16 + i * PER + at;
                uint32_t f[8];
                s8x4_value(next[i].x, f[0], f[1]);
                s8x4_value(next[i].y, f[2], f[3]);
                s8x4_value(next[i].z, f[4], f[5]);
                s8x4_value(next[i].w, f[6], f[7]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const bool second = e != swap;
                    st_shared16(to + row * 128 + (((unit0 + second) ^ (row & 7)) << 4), second ? f[4] : f[0],
                                second ? f[5] : f[1], second ? f[6] : f[2], second ? f[7] : f[3]);
                }
            }
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(P_A_FULL + stage));
            if (n + 1 < mine) load();
            if (n + 2 < mine) found = find(first_page(n + 2) + w * 16 + (lane & 15));
        }
    } else {
        // ---------------------------------------------------------------- contractions
        const uint32_t idesc = idesc_make(kTilePages, kCols, 0u);
        for (int n = 0; n < mine; ++n) {
            const int stage = n & 1;
            if (!poll_phase_warp(BAR(P_A_FULL + stage), (uint32_t)(n >> 1) & 1u, ctl)) break;
            if (n >= 2 && !poll_phase_warp(BAR(P_D_FREE + stage), (uint32_t)(n / 2 - 1) & 1u, ctl)) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int x = 0; x < 2 * D / 16; ++x) {
                    const uint32_t off = (x >> 2) * kAtom + (x & 3) * 32;
                    mma_f16(tmem + stage * kCols, sdesc_k_sw128(base + L::A + stage * L::ROWS + off),
                            sdesc_k_sw128(base + L::Q + off), idesc, x > 0);
                }
                mma_commit(BAR(P_D_FULL + stage));
                mma_commit(BAR(P_A_FREE + stage));
            }
            __syncwarp();
        }
        // every contraction issued has ended before tensor memory is released, also where a wait gave up
        if (elect_one()) mma_commit(BAR(P_DRAIN));
        __syncwarp();
        volatile int no_abort = 0;
        const Ctl drain{&no_abort, a.err, kWaitBudgetCycles};
        wait_phase(BAR(P_DRAIN), 0u, drain);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 256);
    }
}

template <int D, bool FP8>
cudaError_t launch(const PickArgs& a, int max_t, int max_pages, int num_sms, cudaStream_t stream)
{
    const int per = pick_tile_queries(a.group), parts = (max_t + per - 1) / per;
    auto kern = pick_tile_kernel<D, FP8>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, PickLayout<D>::ALLOC);
    if (e != cudaSuccess) return e;
    // a CTA an SM; the pages are shared out where the columns alone leave SMs empty
    const int64_t others = (int64_t)parts * a.hkv * a.batch, steps = (max_pages + kTilePages - 1) / kTilePages;
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(steps, num_sms / others));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks, (unsigned)(parts * a.hkv), (unsigned)a.batch);
    cfg.blockDim = dim3(kPickThreads, 1, 1);
    cfg.dynamicSmemBytes = PickLayout<D>::ALLOC;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, a, (int)blocks);
}

}  // namespace

int pick_tile_queries(int group) { return std::max(1, kCols / padded_group(group)); }

cudaError_t launch_pick_tiles(const PickArgs& a, int head_dim, bool fp8, int max_t, int max_pages, int num_sms,
                              cudaStream_t stream)
{
    if (fp8) return launch<128, true>(a, max_t, max_pages, num_sms, stream);
    return head_dim == 128 ? launch<128, false>(a, max_t, max_pages, num_sms, stream)
                           : launch<64, false>(a, max_t, max_pages, num_sms, stream);
}

}  // namespace lvs
