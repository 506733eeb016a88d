// The 8-bit linear layer for many tokens: CTA pairs, 256 tokens x 256 output features per tile.
//
// Bound: the tensor cores.  One tcgen05.mma (cta_group::2, e4m3) of a pair takes 256 tokens (128 of each CTA, the M dimension: a
// tensor-memory lane is a token) times 256 rows of W (half from each CTA's shared memory) over 32 columns.  The scales change every 128
// columns, so the four MMAs of a block start a new accumulator and its sums go, while the next block's MMAs fill the other
// half of tensor memory, into fp32 registers under the block's scale:  acc += d * (sx[token] * sw[128 features]).  A thread owns
// one token and 128 features, so both scales are one number per thread and block, and the step costs 64 packed multiply-adds
// per thread, 2 x 64 of 512 issue slots that the block's MMAs take on an SM.
//
// Warps of a CTA (10): 0 TMA of its 128 tokens and 128 rows of W per block into a ring of 32 KB slots; 1 in the leader the
// MMAs, in the other CTA the relay that tells the leader its half has landed; 2 to 9 sums and output.  Persistent pairs; every wait is bounded and
// reports through the workspace status word.
#include "slim_fp8.cuh"

#include <atomic>

namespace slim {

constexpr int kFgThreads = 320;
constexpr int kFgTok = 256, kFgFeat = 256;         // of a pair's tile; each CTA: 128 tokens, and brings 128 rows of W
constexpr int kFgStages = 6;
constexpr int kFgSlot = 2 * 128 * 128;
constexpr int kFgOffBar = kFgStages * kFgSlot;
constexpr int kFgSmem = kFgOffBar + 256 + 1024;

struct FgParams {
    const float* x_scales;       // [G][Mp]
    const float* scales;         // [ceil(N / 128)][G]
    void* y;
    long long ldy;
    unsigned int* status;
    int y_type, M, N, G, Mp;
    int tok_tiles, tiles;
};

namespace fg {
__device__ __forceinline__ uint32_t map_to_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void arrive_cluster(uint32_t cluster_bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory"); }
// Tensor memory of the pair: one warp of each CTA executes these together.
__device__ __forceinline__ void alloc(uint32_t smem_dst, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
}
__device__ __forceinline__ void relinquish() { asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void dealloc(uint32_t taddr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
// When the pair's MMAs issued so far have completed, arrive on the barrier at this offset in both CTAs.
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
}
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
}  // namespace fg

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kFgThreads, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map, const FgParams p) {
    extern __shared__ unsigned char fg_raw[];
    unsigned char* smem = fg_raw + ((1024u - (smem_u32(fg_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem), bars = base + kFgOffBar;
    auto full = [&](int s) { return bars + 8u * s; };                         // this CTA's slot has landed
    auto peer = [&](int s) { return bars + 8u * (kFgStages + s); };           // leader's: the other CTA's has
    auto empty = [&](int s) { return bars + 8u * (2 * kFgStages + s); };
    auto d_full = [&](int b) { return bars + 8u * (3 * kFgStages + b); };
    auto d_empty = [&](int b) { return bars + 8u * (3 * kFgStages + 2 + b); };    // leader's: the sums' warps of both CTAs
    static_assert(8 * (3 * kFgStages + 4) <= 240, "room for the barriers");
    volatile int* abort = reinterpret_cast<volatile int*>(smem + kFgOffBar + 240);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + kFgOffBar + 244);

    const int tid = threadIdx.x, lane = tid & 31, warp = static_cast<int>(tc::uniform(tid >> 5));
    const int rank = static_cast<int>(cluster_ctarank());
    const int pair = static_cast<int>(blockIdx.x >> 1), pairs = static_cast<int>(gridDim.x >> 1);
    const int G = p.G;

    if (tid == 0) {
        *abort = 0;
        for (int s = 0; s < kFgStages; ++s) { sb::init(full(s), 1); sb::init(peer(s), 1); sb::init(empty(s), 1); }
        for (int b = 0; b < 2; ++b) { sb::init(d_full(b), 1); sb::init(d_empty(b), 16); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        fg::alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
        fg::relinquish();
    }
    tc::fence_before();
    __syncthreads();
    cluster_sync_all();                                // both CTAs' barriers exist
    tc::fence_after();
    const uint32_t tmem = tc::uniform(*tmem_slot);
    pdl_launch_dependents();
    pdl_wait();

    int issued = 0;                                    // blocks this role has begun
    if (warp == 0) {
        for (int tile = pair; tile < p.tiles; tile += pairs) {
            const int m0 = tile % p.tok_tiles * kFgTok + 128 * rank, n0 = tile / p.tok_tiles * kFgFeat + 128 * rank;
            int g = 0;
            for (; g < G; ++g, ++issued) {
                const int s = issued % kFgStages;
                if (!tc::warp_wait(empty(s), ((issued / kFgStages) & 1u) ^ 1u, abort)) break;
                if (tc::elect()) {
                    sb::expect_tx(full(s), kFgSlot);
                    tc::tma_load_2d(base + s * kFgSlot, &x_map, 128 * g, m0, full(s));
                    tc::tma_load_2d(base + s * kFgSlot + kFgSlot / 2, &w_map, 128 * g, n0, full(s));
                }
                __syncwarp();
            }
            if (g < G) break;
        }
    } else if (warp == 1) {
        for (int tile = pair; tile < p.tiles; tile += pairs) {
            int g = 0;
            for (; g < G; ++g, ++issued) {
                const int s = issued % kFgStages, b = issued & 1;
                const uint32_t ph = (issued / kFgStages) & 1u;
                if (!tc::warp_wait(full(s), ph, abort)) break;
                if (rank != 0) {
                    if (tc::elect()) fg::arrive_cluster(fg::map_to_cta(peer(s), 0));
                    __syncwarp();
                    continue;
                }
                if (!tc::warp_wait(peer(s), ph, abort)) break;
                if (!tc::warp_wait(d_empty(b), ((issued >> 1) & 1u) ^ 1u, abort)) break;
                tc::fence_after();
                const uint64_t a = tc::desc_k128(base + s * kFgSlot), w = tc::desc_k128(base + s * kFgSlot + kFgSlot / 2);
                if (tc::elect()) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) fg::mma_ss(tmem + b * kFgFeat, a + 2 * k, w + 2 * k, f8::idesc(kFgTok, kFgFeat), k > 0 ? 1u : 0u);
                    fg::commit(empty(s));
                    fg::commit(d_full(b));
                }
                __syncwarp();
            }
            if (g < G) break;
        }
    } else {
        const int half = (warp - 2) >> 2, q = warp & 3;
        const uint32_t d_t = tmem + 128u * half + (static_cast<uint32_t>(32 * q) << 16);
        const uint32_t d_empty_leader = fg::map_to_cta(d_empty(0), 0);
        const int n_blocks = (p.N + 127) / 128;
        for (int tile = pair; tile < p.tiles; tile += pairs) {
            const int token = tile % p.tok_tiles * kFgTok + 128 * rank + 32 * q + lane;
            const int n0 = tile / p.tok_tiles * kFgFeat + 128 * half;
            const float* sx = p.x_scales + min(token, p.M - 1);
            const float* sw = p.scales + static_cast<size_t>(min(n0 / 128, n_blocks - 1)) * G;
            uint64_t acc[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = 0ull;
            float x_next = __ldcg(sx), w_next = __ldg(sw);
            int g = 0;
            for (; g < G; ++g, ++issued) {
                const int b = issued & 1;
                const float sc = x_next * w_next;
                if (g + 1 < G) { x_next = __ldcg(sx + static_cast<size_t>(g + 1) * p.Mp); w_next = __ldg(sw + g + 1); }
                const uint64_t sc2 = f8::pack2(__float_as_uint(sc), __float_as_uint(sc));
                if (!tc::warp_wait(d_full(b), (issued >> 1) & 1u, abort)) break;
                tc::fence_after();
#pragma unroll
                for (int c = 0; c < 128; c += 16) {
                    uint32_t d[16];
                    f8::ld16(d_t + b * kFgFeat + c, d);
                    tc::wait_ld();
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[c / 2 + i] = f8::fma2(f8::pack2(d[2 * i], d[2 * i + 1]), sc2, acc[c / 2 + i]);
                }
                tc::fence_before();
                __syncwarp();
                if (lane == 0) fg::arrive_cluster(d_empty_leader + 8u * b);
            }
            if (g < G) break;
            if (token < p.M && n0 < p.N) {
                const size_t at = static_cast<size_t>(token) * p.ldy + n0;
                const int n = min(128, p.N - n0);
                const bool whole = n == 128 && p.ldy % 8 == 0;          // y is 16-byte aligned
                if (whole && p.y_type == SLIM_F32) {
#pragma unroll
                    for (int i = 0; i < 64; i += 2) {
                        const float2 u = f8::unpack2(acc[i]), v = f8::unpack2(acc[i + 1]);
                        *reinterpret_cast<float4*>(static_cast<float*>(p.y) + at + 2 * i) = make_float4(u.x, u.y, v.x, v.y);
                    }
                } else if (whole) {
#pragma unroll
                    for (int i = 0; i < 64; i += 4) {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 u = f8::unpack2(acc[i + j]);
                            if (p.y_type == SLIM_F16) { const __half2 h = __floats2half2_rn(u.x, u.y); w[j] = *reinterpret_cast<const uint32_t*>(&h); }
                            else { const __nv_bfloat162 h = __floats2bfloat162_rn(u.x, u.y); w[j] = *reinterpret_cast<const uint32_t*>(&h); }
                        }
                        *reinterpret_cast<uint4*>(static_cast<__half*>(p.y) + at + 2 * i) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 64; ++i) {
                        const float2 u = f8::unpack2(acc[i]);
                        if (2 * i < n) f8::store_y(p.y, p.y_type, at + 2 * i, u.x);
                        if (2 * i + 1 < n) f8::store_y(p.y, p.y_type, at + 2 * i + 1, u.y);
                    }
                }
            }
        }
    }

    // ---- after a wait that gave up: what was issued has landed before the shared and tensor memory goes
    if (warp == 0 && *abort != 0)
        for (int i = max(0, issued - kFgStages); i < issued; ++i) {
            if (tc::elect()) f8::drain(full(i % kFgStages), (i / kFgStages) & 1u);
            __syncwarp();
        }
    if (warp == 1 && rank == 0 && *abort != 0)
        for (int i = max(0, issued - 2); i < issued; ++i) {
            if (tc::elect()) f8::drain(d_full(i & 1), (i >> 1) & 1u);
            __syncwarp();
        }
    tc::fence_before();
    __syncthreads();
    cluster_sync_all();                                // nobody leaves while the other may signal it or its MMAs read from here
    tc::fence_after();
    if (warp == 1) fg::dealloc(tmem, 512);
    if (tid == 0 && *abort != 0) report_timeout(p.status, false);
}

// ------------------------------------------------------------------------------------------ host side
cudaError_t fp8_gemm(const Fp8Args& a) {
    static std::atomic<bool> attr_set[64];    // zero-initialised; set-up is idempotent, so a race repeats it harmlessly
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = cudaFuncSetAttribute(fp8_gemm_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFgSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    FgParams p;
    memset(&p, 0, sizeof p);
    p.x_scales = a.x_scales; p.scales = a.scales; p.y = a.y; p.ldy = a.ldy;
    p.status = reinterpret_cast<unsigned int*>(a.workspace);
    p.y_type = a.y_type; p.M = a.M; p.N = a.N; p.G = (a.K + f8::kBlock - 1) / f8::kBlock; p.Mp = a.Mp;
    p.tok_tiles = (a.M + kFgTok - 1) / kFgTok;
    p.tiles = p.tok_tiles * ((a.N + kFgFeat - 1) / kFgFeat);
    CUtensorMap x_map, w_map;
    if (!make_byte_map(&x_map, a.x_codes, a.M, a.K, 128) || !make_byte_map(&w_map, a.codes, a.N, a.K, 128)) return cudaErrorUnknown;
    const int pairs = device_sm_count() / 2;
    PdlLaunch l(static_cast<unsigned>(2 * (p.tiles < pairs ? p.tiles : pairs)), kFgThreads, kFgSmem, a.stream);      // clusters of 2: see the kernel
    return cudaLaunchKernelEx(&l.cfg, fp8_gemm_kernel, x_map, w_map, p);
}
bool fp8_use_gemm(int M, int N, int K) {
    (void)N; (void)K;
    return M > 128;
}

}  // namespace slim
