// The 8-bit linear layer for many tokens: CTA pairs, 256 tokens x up to 256 output features per tile.
//
// Bound: the tensor cores.  One tcgen05.mma (cta_group::2, e4m3) of a pair takes 256 tokens (128 of each CTA, the M dimension: a
// tensor-memory lane is a token) times up to 256 rows of W (half from each CTA's shared memory) over 32 columns.  All scales are powers of two, so the
// block-scaled form (kind::mxf8f6f4, E8M0 scales of 32 columns each) applies them inside the MMA: the four MMAs of a block of 128 columns name the
// same byte of a row's scale word, and a tile's sum over all of K stays in tensor memory.  Plain MMAs with a pass over D per block (into
// registers, under the block's scale) took 139 us at 2048 x 13824 x 5120 in the best of four forms where this takes 122 (both in short runs): reading D
// competes with the MMAs' own accumulation (430 to 550 cycles per block beside them, 150 alone, of 512 that its MMAs take).
//
// Scale words (four blocks' bytes) go to tensor memory by tcgen05.st: row r's word at lane r % 32 of column r / 32, the same in all four lane
// quarters; two buffers.  A CTA has the words of its own tokens and of all features.
//
// Warps of a CTA (16): 0 TMA of its 128 tokens and its half of the rows of W per block into a ring of 32 KB slots; 1 in the leader the
// MMAs, in the other CTA the relay that tells the leader its half has landed; 4 to 7 scale words; 8 to 15 output: they take D into
// registers at once, so that the next tile's MMAs wait for the reading alone, and convert and store beside them.
// Measured, call after call at the power cap, the quantizer of x among it: 2048 x 13824 x 5120 139 us (2.1 PFLOP/s at 1.25 GHz), 512 x 5120 x 13824 46,
// 1000 x 4096 x 32000 137.
// Persistent pairs; every wait is bounded and reports through the workspace status word.  Compiled for 128 registers, as before the split, 100 bytes a thread
// are spilled (the output warps alone hold 128 sums each, once a tile).
#include "slim_fp8.cuh"

#include <atomic>

namespace slim {

constexpr int kFgThreads = 512;
// Registers after the split: 256 x 80 + 256 x 176 = 512 x 128, what the block is launched with.
constexpr int kFgRegsFew = 80, kFgRegsMany = 176;
constexpr int kFgTok = 256, kFgFeat = 256;         // of a pair's tile, at most; each CTA: 128 tokens, and brings half of the rows of W
constexpr int kFgStages = 6;
constexpr int kFgSlot = 2 * 128 * 128;
constexpr int kFgOffBar = kFgStages * kFgSlot;
constexpr int kFgSmem = kFgOffBar + 256 + 1024;
constexpr int kFgColScales = 480;                  // tensor memory: D (twice, where it has at most 224 columns), then two buffers of 4 + 8 columns of
constexpr int kFgScaleCols = 16;                   // scale words
constexpr int kFgFeatTwice = 224;

struct FgParams {
    const uint32_t* x_scales;    // [ceil(G / 4)][Mp]
    const float* scales;         // [ceil(N / 128)][G]
    void* y;
    long long ldy;
    unsigned int* status;
    int y_type, M, N, G, Mp;
    int feat;                    // features of a tile, a multiple of 32
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
// D (+)= A B^T over the pair, e4m3, the products of every row of A and of B times the row's scale.
__device__ __forceinline__ void mma_scaled(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
}
// Instruction descriptor: e4m3 operands, both K-major, E8M0 scales from byte `id` of their words, m x n.
__device__ __forceinline__ uint32_t idesc_scaled(int m, int n, int id) {
    return (static_cast<uint32_t>(id) << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) | (static_cast<uint32_t>(m >> 7) << 27) |
           (static_cast<uint32_t>(id) << 29);
}
__device__ __forceinline__ void st4(uint32_t taddr, const uint32_t* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
}  // namespace fg

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kFgThreads, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map, const FgParams p) {
    extern __shared__ unsigned char fg_raw[];
    unsigned char* smem = fg_raw + ((1024u - (smem_u32(fg_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem), bars = base + kFgOffBar;
    auto full = [&](int s) { return bars + 8u * s; };                         // this CTA's slot has landed; the leader's: and the other CTA's
    auto empty = [&](int s) { return bars + 8u * (kFgStages + s); };
    auto sf_full = [&](int b) { return bars + 8u * (2 * kFgStages + b); };    // leader's: the scale warps of both CTAs
    auto sf_empty = [&](int b) { return bars + 8u * (2 * kFgStages + 2 + b); };
    auto d_full = [&](int b) { return bars + 8u * (2 * kFgStages + 4 + b); };
    auto d_empty = [&](int b) { return bars + 8u * (2 * kFgStages + 6 + b); };           // leader's, the output warps of both CTAs
    static_assert(8 * (2 * kFgStages + 8) <= 240, "room for the barriers");
    volatile int* abort = reinterpret_cast<volatile int*>(smem + kFgOffBar + 240);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + kFgOffBar + 244);

    const int tid = threadIdx.x, lane = tid & 31, warp = static_cast<int>(tc::uniform(tid >> 5));
    const int rank = static_cast<int>(cluster_ctarank());
    const int pair = static_cast<int>(blockIdx.x >> 1), pairs = static_cast<int>(gridDim.x >> 1);
    const int G = p.G, feat = p.feat, bufs = feat <= kFgFeatTwice ? 2 : 1;      // of D

    if (tid == 0) {
        *abort = 0;
        for (int s = 0; s < kFgStages; ++s) { sb::init(full(s), rank == 0 ? 2 : 1); sb::init(empty(s), 1); }
        for (int b = 0; b < 2; ++b) { sb::init(sf_full(b), 8); sb::init(sf_empty(b), 1); }
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
    // The kernel ahead is the quantizer of x, which lets this one start only when all before it has completed: W is there, and requested at once.
    const uint32_t bytes = (128u + static_cast<uint32_t>(feat) / 2u) * 128u;
    int first = 0;                                     // blocks of W requested ahead
    if (warp == 0) {
        first = min(G, kFgStages);
        if (tc::elect())
            for (int i = 0; i < first; ++i) {
                sb::expect_tx(full(i), bytes);
                tc::tma_load_2d(base + i * kFgSlot + kFgSlot / 2, &w_map, 128 * i, pair / p.tok_tiles * feat + feat / 2 * rank, full(i));
            }
        __syncwarp();
    }
    pdl_wait();

    int issued = 0;                                    // blocks this role has begun
    if (warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFgRegsFew));
        if (warp == 0) {
            for (int tile = pair; tile < p.tiles; tile += pairs) {
                const int m0 = tile % p.tok_tiles * kFgTok + 128 * rank, n0 = tile / p.tok_tiles * feat + feat / 2 * rank;
                int g = 0;
                for (; g < G; ++g, ++issued) {
                    const int s = issued % kFgStages;
                    if (!tc::warp_wait(empty(s), ((issued / kFgStages) & 1u) ^ 1u, abort)) break;
                    if (tc::elect()) {
                        if (issued >= first) {
                            sb::expect_tx(full(s), bytes);
                            tc::tma_load_2d(base + s * kFgSlot + kFgSlot / 2, &w_map, 128 * g, n0, full(s));
                        }
                        tc::tma_load_2d(base + s * kFgSlot, &x_map, 128 * g, m0, full(s));
                    }
                    __syncwarp();
                }
                if (g < G) break;
            }
        } else if (warp == 1 && rank == 0) {
            // The MMAs of a block take 512 cycles (256 features) and a turn of this loop must not: a wait for a barrier that is ready costs some
            // 110 cycles, so a slot has one barrier for both CTAs' halves, and the scale words one per four blocks.
            int words = 0, s = 0;                      // groups of four blocks begun; slot
            uint32_t ph = 0, phd = 0;
            int buf = 0;
            bool ok = true;
            for (int tile = pair; tile < p.tiles && ok; tile += pairs) {
                const uint32_t d = tmem + static_cast<uint32_t>(feat * buf);
                ok = tc::warp_wait(d_empty(buf), phd ^ 1u, abort);
                for (int g = 0; g < G && ok; ++g, ++issued) {
                    const int b = words & 1;
                    if ((g & 3) == 0 && !tc::warp_wait(sf_full(b), (words >> 1) & 1u, abort)) { ok = false; break; }
                    if (!tc::warp_wait(full(s), ph, abort)) { ok = false; break; }
                    tc::fence_after();
                    const uint64_t a = tc::desc_k128(base + s * kFgSlot), w = tc::desc_k128(base + s * kFgSlot + kFgSlot / 2);
                    const uint32_t idesc = fg::idesc_scaled(kFgTok, feat, g & 3), sa = tmem + kFgColScales + kFgScaleCols * b;
                    const bool last = (g & 3) == 3 || g + 1 == G;
                    if (tc::elect()) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) fg::mma_scaled(d, a + 2 * k, w + 2 * k, idesc, sa, sa + 4, g > 0 || k > 0 ? 1u : 0u);
                        fg::commit(empty(s));
                        if (last) fg::commit(sf_empty(b));
                        if (g + 1 == G) fg::commit(d_full(buf));
                    }
                    __syncwarp();
                    if (last) ++words;
                    if (++s == kFgStages) { s = 0; ph ^= 1u; }
                }
                if (++buf == bufs) { buf = 0; phd ^= 1u; }
            }
        } else if (warp == 1) {
            // tells the leader that this CTA's half of a slot has landed
            int s = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int tile = pair; tile < p.tiles && ok; tile += pairs)
                for (int g = 0; g < G; ++g) {
                    ok = tc::warp_wait(full(s), ph, abort);
                    if (!ok) break;
                    if (tc::elect()) fg::arrive_cluster(fg::map_to_cta(full(s), 0));
                    __syncwarp();
                    if (++s == kFgStages) { s = 0; ph ^= 1u; }
                }
        } else if (warp >= 4) {
            // ---- scale words: this warp's quarter of the lanes, of all of the CTA's tokens and the tile's features.  A group's are fetched while
            // the one before is written: lane l reads W's scale of column l / 4 (32 features, which lie in one block of 128), block g + l % 4.
            const int q = warp & 3;
            const uint32_t sf_t = tmem + kFgColScales + (static_cast<uint32_t>(32 * q) << 16);
            const uint32_t sf_full_leader = fg::map_to_cta(sf_full(0), 0);
            const int n_blocks = (p.N + 127) / 128;
            struct Words { uint32_t x[4], w; };
            auto fetch = [&](int tile, int g, Words& v) {
                const int m0 = min(tile % p.tok_tiles * kFgTok + 128 * rank, p.Mp - 128), n = tile / p.tok_tiles * feat + 32 * (lane >> 2);
#pragma unroll
                for (int c = 0; c < 4; ++c) v.x[c] = __ldcg(p.x_scales + static_cast<size_t>(g >> 2) * p.Mp + m0 + 32 * c + lane);
                v.w = __float_as_uint(__ldg(p.scales + static_cast<size_t>(min(n >> 7, n_blocks - 1)) * G + min(g + (lane & 3), G - 1)));
            };
            auto put = [&](const Words& v) {
                const int b = issued & 1;
                uint32_t own = f8::e8m0(v.w) << (8 * (lane & 3)), ww[8];
                own |= __shfl_xor_sync(0xffffffffu, own, 1);
                own |= __shfl_xor_sync(0xffffffffu, own, 2);
#pragma unroll
                for (int c = 0; c < 8; ++c) ww[c] = __shfl_sync(0xffffffffu, own, 4 * c);
                if (!tc::warp_wait(sf_empty(b), ((issued >> 1) & 1u) ^ 1u, abort)) return false;
                tc::fence_after();
                fg::st4(sf_t + kFgScaleCols * b, v.x);
                tc::st8(sf_t + kFgScaleCols * b + 4, ww);
                tc::wait_st();
                tc::fence_before();
                __syncwarp();
                if (lane == 0) fg::arrive_cluster(sf_full_leader + 8u * b);
                ++issued;
                return true;
            };
            int tile = pair, g = 0;                    // of the group fetched last
            auto next = [&] {
                g += 4;
                if (g >= G) { g = 0; tile += pairs; }
                return tile < p.tiles;
            };
            Words even, odd;
            bool more = tile < p.tiles;
            if (more) fetch(tile, g, even);
            while (more) {
                more = next();
                if (more) fetch(tile, g, odd);
                if (!put(even) || !more) break;
                more = next();
                if (more) fetch(tile, g, even);
                if (!put(odd)) break;
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kFgRegsMany));
        const int half = (warp - 8) >> 2, q = warp & 3, cols = feat / 2;
        const uint32_t d_t = tmem + static_cast<uint32_t>(cols * half) + (static_cast<uint32_t>(32 * q) << 16);
        const uint32_t d_empty_leader = fg::map_to_cta(d_empty(0), 0);
        uint32_t ph = 0;
        int buf = 0;
        for (int tile = pair; tile < p.tiles; tile += pairs) {
            const int token = tile % p.tok_tiles * kFgTok + 128 * rank + 32 * q + lane;
            const int n0 = tile / p.tok_tiles * feat + cols * half;
            uint32_t d[8][16];
            if (!tc::warp_wait(d_full(buf), ph, abort)) break;
            tc::fence_after();
            const uint32_t d_b = d_t + static_cast<uint32_t>(feat * buf);
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (16 * c < cols) f8::ld16(d_b + 16 * c, d[c]);
            tc::wait_ld();
            tc::fence_before();
            __syncwarp();
            if (lane == 0) fg::arrive_cluster(d_empty_leader + 8u * buf);
            if (++buf == bufs) { buf = 0; ph ^= 1u; }
            if (token < p.M) {
                const size_t at = static_cast<size_t>(token) * p.ldy + n0;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const int n = min(16, min(cols, p.N - n0) - 16 * c);
                    if (n <= 0) break;
                    const float* v = reinterpret_cast<const float*>(d[c]);
                    if (n == 16 && p.ldy % 8 == 0) {   // y is 16-byte aligned, and so is n0
                        if (p.y_type == SLIM_F32) {
#pragma unroll
                            for (int i = 0; i < 16; i += 4)
                                *reinterpret_cast<float4*>(static_cast<float*>(p.y) + at + 16 * c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                        } else {
                            uint32_t w[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                if (p.y_type == SLIM_F16) { const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
                                else { const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
                            }
                            uint4* o = reinterpret_cast<uint4*>(static_cast<__half*>(p.y) + at + 16 * c);
                            o[0] = make_uint4(w[0], w[1], w[2], w[3]);
                            o[1] = make_uint4(w[4], w[5], w[6], w[7]);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (i < n) f8::store_y(p.y, p.y_type, at + 16 * c + i, v[i]);
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
        for (int i = max(0, issued - kFgStages); i < issued; ++i) {
            if (tc::elect()) f8::drain(empty(i % kFgStages), (i / kFgStages) & 1u);
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
// Features of a tile: a multiple of 32.  Measured in cycles of the issuing warp: a block takes its MMAs' time, 2.05 per feature, or 390 however few
// features (that warp's turn), and a tile 2400 beside its blocks (reading D slows the next tile's MMAs), 3100 where there is one D (256 features).
// 2048 x 13824 x 5120 comes to 145000 at 256, 224 and 192 alike (138, 137 and 139 us); 512 x 5120 x 13824 at 256 / 192 / 160 took 49.5 / 45.1 / 44.3 us, 1024 x 11008 x
// 4096 at 256 / 224 / 160 53.6 / 50.3 / 51.9.  Equal, wider tiles read less.
static int fg_features(int tok_tiles, int N, int G, int pairs, double* cycles) {
    int best = kFgFeat;
    double least = 1e30;
    for (int feat = kFgFeat; feat >= 160; feat -= 32) {
        const long long tiles = static_cast<long long>(tok_tiles) * ((N + feat - 1) / feat), waves = (tiles + pairs - 1) / pairs;
        const double t = static_cast<double>(waves) * (G * (feat > 190 ? 2.05 * feat : 390.0) + (feat > kFgFeatTwice ? 3100.0 : 2400.0));
        if (t < 0.995 * least) { least = t; best = feat; }
    }
    *cycles = least;
    return best;
}

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
    const int pairs = device_sm_count() / 2;
    double cycles = 0.0;
    p.feat = fg_features(p.tok_tiles, a.N, p.G, pairs, &cycles);
    p.tiles = p.tok_tiles * ((a.N + p.feat - 1) / p.feat);
    CUtensorMap x_map, w_map;
    if (!make_byte_map(&x_map, a.x_codes, a.M, a.K, 128) || !make_byte_map(&w_map, a.codes, a.N, a.K, p.feat / 2)) return cudaErrorUnknown;
    PdlLaunch l(static_cast<unsigned>(2 * (p.tiles < pairs ? p.tiles : pairs)), kFgThreads, kFgSmem, a.stream);      // clusters of 2: see the kernel
    return cudaLaunchKernelEx(&l.cfg, fp8_gemm_kernel, x_map, w_map, p);
}
// Up to 128 tokens the other kernel, which cuts K; beyond, whichever is expected to end first: that one also at 129 to 256 tokens of narrow and deep layers,
// whose few tiles walk all of K here.  (us, that one / this one: 4096 x 11008 at 65, 128, 256 and 300 tokens 16.4 / 25.9, 18.9 / 27.2, 24.2 / 28.5, 35.3 / 30.6;
// 11008 x 4096 17.2 / 17.1, 20.0 / 20.0, 34.7 / 20.7; 32000 x 4096 28.7 / 34.6, 29.7 / 36.3, 52.7 / 38.6.)
bool fp8_use_gemm(int M, int N, int K) {
    if (M <= 128) return false;
    double cycles = 0.0;
    fg_features((M + kFgTok - 1) / kFgTok, N, (K + f8::kBlock - 1) / f8::kBlock, device_sm_count() / 2, &cycles);
    return cycles + 4000.0 <= fp8_few_cycles(M, N, K);
}

}  // namespace slim
