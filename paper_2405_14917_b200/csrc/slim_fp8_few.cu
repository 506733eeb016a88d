// The 8-bit linear layer for few tokens: W is the M dimension of the MMA (128 rows per CTA), up to 128 tokens its N dimension.
//
// Bound: HBM, the codes of W (one byte per weight).  A tile of 128 rows is cut along K over the CTAs of a cluster, so that
// narrow layers too have about two CTAs per SM and everything a CTA reads is in flight at once: TMA brings 128 x 128 bytes per block of
// 128 columns into a ring of 128-byte-swizzled slots, four K = 32 MMAs per block leave its sums in one of two buffers of tensor memory,
// and four warps take them from there into fp32 registers under the block's scale.  The CTAs of a cluster then add their sums
// through distributed shared memory, every CTA a share of the tokens, in rank order: no workspace, no second kernel, one result.
//
// Up to 32 tokens x is quantised here (kTakesX), by four warps ahead of the MMAs, from x itself: every CTA does it for its part of K,
// which costs L2 reads of 2 T bytes per 128 bytes of W and saves the launch of the quantizer.  Beyond, the codes come
// by TMA from the workspace (slim_fp8.cu).
//
// Warps: 0 loads of W (and of staged x); 1 MMAs, tensor memory; 2, 3, 8, 9 quantisation of x, or the scales of staged x;
// 4 to 7 sums (tensor-memory lanes 32 (w % 4) on).  Every wait is bounded and reports through the workspace status word.
#include "slim_fp8.cuh"

#include <atomic>

namespace slim {

constexpr int kFewThreads = 320;
constexpr int kFewXWarps = 4;
constexpr int kFewMaxCluster = 8;

template <int T> struct FewCfg {
    static constexpr bool TAKES_X = T <= 32;
    static constexpr int PER_SM = T <= 64 ? 2 : 1;
    static constexpr int W_BYTES = 128 * 128, X_BYTES = T * 128;
    static constexpr int STAGES = T <= 16 ? 5 : T <= 32 ? 5 : T <= 64 ? 4 : 6;
    static constexpr int TMEM = 2 * T < 32 ? 32 : 2 * T;
    static constexpr int OFF_SX = STAGES * (W_BYTES + X_BYTES);           // [STAGES][T] fp32
    static constexpr int OFF_BAR = OFF_SX + STAGES * T * 4;
    static constexpr int SMEM = OFF_BAR + 256 + 1024;                     // + alignment of the slots
};

struct FewParams {
    const void* x;
    long long ldx;
    const uint8_t* x_scales;     // staged: exponents, byte g % 4 of word [g / 4][token]
    const float* scales;
    void* y;
    long long ldy;
    unsigned int* status;
    int y_type, M, N, K, G, Mp, ranks;
};

template <int T, typename X>
__global__ void __launch_bounds__(kFewThreads, FewCfg<T>::PER_SM)
fp8_few_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map, const FewParams p) {
    using C = FewCfg<T>;
    extern __shared__ unsigned char few_raw[];
    unsigned char* smem = few_raw + ((1024u - (smem_u32(few_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const uint32_t s_x = base + C::STAGES * C::W_BYTES, s_sx = base + C::OFF_SX, bars = base + C::OFF_BAR;
    auto w_full = [&](int s) { return bars + 8u * s; };
    auto w_empty = [&](int s) { return bars + 8u * (C::STAGES + s); };
    auto x_full = [&](int s) { return bars + 8u * (2 * C::STAGES + s); };
    auto x_empty = [&](int s) { return bars + 8u * (3 * C::STAGES + s); };
    auto d_full = [&](int b) { return bars + 8u * (4 * C::STAGES + b); };
    auto d_empty = [&](int b) { return bars + 8u * (4 * C::STAGES + 2 + b); };
    static_assert(8 * (4 * C::STAGES + 4) <= 240, "room for the barriers");
    volatile int* abort = reinterpret_cast<volatile int*>(smem + C::OFF_BAR + 240);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + C::OFF_BAR + 244);

    const int tid = threadIdx.x, lane = tid & 31, warp = static_cast<int>(tc::uniform(tid >> 5));
    const int rank = static_cast<int>(blockIdx.x) % p.ranks, tile = static_cast<int>(blockIdx.x) / p.ranks;
    const int row_tiles = (p.N + 127) / 128;
    const int nb = tile % row_tiles, n0 = 128 * nb, m0 = tile / row_tiles * T;
    const int tokens = min(T, p.M - m0);
    const int g0 = static_cast<int>(static_cast<long long>(p.G) * rank / p.ranks), g1 = static_cast<int>(static_cast<long long>(p.G) * (rank + 1) / p.ranks);
    const int steps = g1 - g0;

    if (tid == 0) {
        *abort = 0;
        for (int s = 0; s < C::STAGES; ++s) {
            sb::init(w_full(s), 1);
            sb::init(w_empty(s), 1);
            sb::init(x_full(s), C::TAKES_X ? kFewXWarps : 2);      // quantising warps, or the codes' TMA and the warp with their scales
            sb::init(x_empty(s), 1 + 4);                           // MMAs, and the warps that read the scales
        }
        for (int b = 0; b < 2; ++b) { sb::init(d_full(b), 1); sb::init(d_empty(b), 4); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        tc::alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), C::TMEM);
        tc::relinquish();
    }
    if (C::TAKES_X) {                                  // tokens past the last stay zero
        for (int i = tid; i < C::STAGES * C::X_BYTES / 16; i += kFewThreads)
            *reinterpret_cast<uint4*>(smem + C::STAGES * C::W_BYTES + 16 * i) = make_uint4(0, 0, 0, 0);
        for (int i = tid; i < C::STAGES * T; i += kFewThreads) *reinterpret_cast<float*>(smem + C::OFF_SX + 4 * i) = 0.f;
        tc::fence_proxy_async();
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tc::uniform(*tmem_slot);
    pdl_launch_dependents();
    pdl_wait();

    float acc[T];                                      // this thread's row, all tokens (warps 4 to 7)
    if (warp == 0) {
        // ---- W, and the codes of staged x
        for (int i = 0; i < steps; ++i) {
            const int s = i % C::STAGES;
            const uint32_t ph = (i / C::STAGES) & 1u;
            if (!tc::warp_wait(w_empty(s), ph ^ 1u, abort)) break;
            if (!C::TAKES_X && !tc::warp_wait(x_empty(s), ph ^ 1u, abort)) break;
            if (tc::elect()) {
                sb::expect_tx(w_full(s), C::W_BYTES);
                tc::tma_load_2d(base + s * C::W_BYTES, &w_map, 128 * (g0 + i), n0, w_full(s));
                if (!C::TAKES_X) {
                    sb::expect_tx(x_full(s), C::X_BYTES);
                    tc::tma_load_2d(s_x + s * C::X_BYTES, &x_map, 128 * (g0 + i), m0, x_full(s));
                }
            }
            __syncwarp();
        }
    } else if (warp == 1) {
        // ---- MMAs
        for (int i = 0; i < steps; ++i) {
            const int s = i % C::STAGES, b = i & 1;
            const uint32_t ph = (i / C::STAGES) & 1u;
            if (!tc::warp_wait(d_empty(b), ((i >> 1) & 1u) ^ 1u, abort)) break;
            if (!tc::warp_wait(x_full(s), ph, abort)) break;
            if (!tc::warp_wait(w_full(s), ph, abort)) break;
            tc::fence_after();
            const uint64_t a = tc::desc_k128(base + s * C::W_BYTES), x = tc::desc_k128(s_x + s * C::X_BYTES);
            if (tc::elect()) {
#pragma unroll
                for (int k = 0; k < 4; ++k) f8::mma_ss(tmem + b * T, a + 2 * k, x + 2 * k, f8::idesc(128, T), k > 0 ? 1u : 0u);
                tc::commit(w_empty(s));
                tc::commit(x_empty(s));
                tc::commit(d_full(b));
            }
            __syncwarp();
        }
    } else if (warp < 4 || warp >= 8) {
        const int xw = warp < 4 ? warp - 2 : warp - 6;
        if (C::TAKES_X) {
            // ---- x into codes: half a warp per token and block, two tokens of a warp at a time
            constexpr int PAIRS = T / 2 / kFewXWarps;               // pairs of tokens of a warp
            const int half = lane >> 4, c = lane & 15;
            const X* x = static_cast<const X*>(p.x);
            uint4 v[PAIRS];
            auto fetch = [&](int i) {
#pragma unroll
                for (int u = 0; u < PAIRS; ++u) {
                    const int t = 2 * (xw + kFewXWarps * u) + half, k = 128 * (g0 + i) + 8 * c;
                    v[u] = t < tokens && k < p.K ? __ldg(reinterpret_cast<const uint4*>(x + static_cast<size_t>(m0 + t) * p.ldx + k)) : make_uint4(0, 0, 0, 0);
                }
            };
            if (steps > 0) fetch(0);
            for (int i = 0; i < steps; ++i) {
                const int s = i % C::STAGES;
                const uint32_t ph = (i / C::STAGES) & 1u;
                if (!tc::warp_wait(x_empty(s), ph ^ 1u, abort)) break;
                uint4 now[PAIRS];
#pragma unroll
                for (int u = 0; u < PAIRS; ++u) now[u] = v[u];
                if (i + 1 < steps) fetch(i + 1);
#pragma unroll
                for (int u = 0; u < PAIRS; ++u) {
                    const int t = 2 * (xw + kFewXWarps * u) + half;
                    if (2 * (xw + kFewXWarps * u) >= tokens) continue;
                    float f[8];
                    f8::unpack8<X>(now[u], f);
                    uint32_t mx = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) mx = max(mx, f8::magnitude(f[e]));
#pragma unroll
                    for (int o = 8; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                    const uint32_t sbits = f8::scale_bits(mx);
                    const float inv = f8::inverse_scale(sbits);
                    // row t of a swizzled tile: its 16-byte chunks stand at chunk ^ (t & 7)
                    const uint32_t at = s_x + s * C::X_BYTES + t * 128 + ((((c >> 1) ^ (t & 7)) << 4) | ((c & 1) << 3));
                    asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(at), "r"(f8::codes4(f, inv)), "r"(f8::codes4(f + 4, inv)) : "memory");
                    if (c == 0) *reinterpret_cast<float*>(smem + C::OFF_SX + 4 * (s * T + t)) = __uint_as_float(sbits);
                }
                tc::fence_proxy_async();
                __syncwarp();
                if (lane == 0) sb::arrive(x_full(s));
            }
        } else if (xw == 0) {
            // ---- the scales of staged x
            for (int i = 0; i < steps; ++i) {
                const int s = i % C::STAGES;
                const uint32_t ph = (i / C::STAGES) & 1u;
                if (!tc::warp_wait(x_empty(s), ph ^ 1u, abort)) break;
#pragma unroll
                for (int t = lane; t < T; t += 32)
                    *reinterpret_cast<float*>(smem + C::OFF_SX + 4 * (s * T + t)) = t < tokens ? __uint_as_float(static_cast<uint32_t>(__ldcg(p.x_scales + (static_cast<size_t>((g0 + i) >> 2) * p.Mp + m0 + t) * 4 + ((g0 + i) & 3))) << 23) : 0.f;
                __syncwarp();
                if (lane == 0) sb::arrive(x_full(s));
            }
        }
    } else {
        // ---- sums: D of every block under its scales
#pragma unroll
        for (int t = 0; t < T; ++t) acc[t] = 0.f;
        const float* sw = p.scales + static_cast<size_t>(nb) * p.G + g0;
        float w_next = steps > 0 ? __ldg(sw) : 0.f;
        for (int i = 0; i < steps; ++i) {
            const int s = i % C::STAGES, b = i & 1;
            const float w = w_next;
            if (i + 1 < steps) w_next = __ldg(sw + i + 1);
            // the scales were written by other warps, ahead of the barrier that the MMAs waited for: this warp waits for it too
            if (!tc::warp_wait(x_full(s), (i / C::STAGES) & 1u, abort)) break;
            if (!tc::warp_wait(d_full(b), (i >> 1) & 1u, abort)) break;
            tc::fence_after();
            const uint32_t d_t = tmem + b * T + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
#pragma unroll
            for (int t0 = 0; t0 < T; t0 += 16) {
                uint32_t d[16];
                f8::ld16(d_t + t0, d);
                tc::wait_ld();
#pragma unroll
                for (int t = 0; t < 16; t += 4) {
                    const float4 sx = *reinterpret_cast<const float4*>(smem + C::OFF_SX + 4 * (s * T + t0 + t));
                    acc[t0 + t] = fmaf(__uint_as_float(d[t]), w * sx.x, acc[t0 + t]);
                    acc[t0 + t + 1] = fmaf(__uint_as_float(d[t + 1]), w * sx.y, acc[t0 + t + 1]);
                    acc[t0 + t + 2] = fmaf(__uint_as_float(d[t + 2]), w * sx.z, acc[t0 + t + 2]);
                    acc[t0 + t + 3] = fmaf(__uint_as_float(d[t + 3]), w * sx.w, acc[t0 + t + 3]);
                }
            }
            tc::fence_before();
            __syncwarp();
            if (lane == 0) { sb::arrive(d_empty(b)); sb::arrive(x_empty(s)); }
        }
    }

    // ---- everything in flight has landed, also after a wait that gave up; then the ring holds the sums of the cluster
    if (warp == 0)
        for (int i = max(0, steps - C::STAGES); i < steps && *abort != 0; ++i) {
            if (tc::elect()) {
                f8::drain(w_full(i % C::STAGES), (i / C::STAGES) & 1u);
                if (!C::TAKES_X) f8::drain(x_full(i % C::STAGES), (i / C::STAGES) & 1u);
            }
            __syncwarp();
        }
    if (warp == 1 && *abort != 0) {
        for (int i = max(0, steps - 2); i < steps; ++i) {
            if (tc::elect()) f8::drain(d_full(i & 1), (i >> 1) & 1u);
            __syncwarp();
        }
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == 1) tc::dealloc(tmem, C::TMEM);
    const int row = 32 * (warp & 3) + lane;            // warps 4 to 7
    const bool sums = warp >= 4 && warp < 8;
    if (p.ranks == 1) {
        if (sums && n0 + row < p.N) {
#pragma unroll
            for (int t = 0; t < T; ++t)
                if (t < tokens) f8::store_y(p.y, p.y_type, static_cast<size_t>(m0 + t) * p.ldy + n0 + row, acc[t]);
        }
    } else {
        float* part = reinterpret_cast<float*>(smem);  // [T][128]
        if (sums) {
#pragma unroll
            for (int t = 0; t < T; ++t) part[t * 128 + row] = acc[t];
        }
        cluster_sync_all();
        if (sums && n0 + row < p.N) {
            for (int t = rank; t < tokens; t += p.ranks) {
                const uint32_t at = base + 4u * (t * 128 + row);
                float v[kFewMaxCluster];
#pragma unroll
                for (int r = 0; r < kFewMaxCluster; ++r) {
                    uint32_t remote;
                    v[r] = 0.f;
                    if (r < p.ranks) {
                        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(at), "r"(r));
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[r]) : "r"(remote) : "memory");
                    }
                }
                float y = v[0];
#pragma unroll
                for (int r = 1; r < kFewMaxCluster; ++r) y += v[r];
                f8::store_y(p.y, p.y_type, static_cast<size_t>(m0 + t) * p.ldy + n0 + row, y);
            }
        }
        cluster_sync_all();                            // the others may still read this CTA's sums
    }
    if (tid == 0 && *abort != 0) report_timeout(p.status, false);
}

// ------------------------------------------------------------------------------------------ host side
// Cut of a tile's K over c CTAs: time in blocks of 128 columns, of which a CTA's start and end cost about four.
static int few_cluster(long long tiles, int G, int slots) {
    int best = 1;
    double least = 1e30;
    for (int c = 1; c <= kFewMaxCluster && c <= G; ++c) {
        const long long waves = (tiles * c + slots - 1) / slots;
        const double t = static_cast<double>(waves) * ((G + c - 1) / c + 4);
        if (t < least) { least = t; best = c; }
    }
    return best;
}

template <int T, typename X>
static cudaError_t few_launch(const Fp8Args& a) {
    using C = FewCfg<T>;
    static std::atomic<bool> attr_set[64];    // zero-initialised; set-up is idempotent, so a race repeats it harmlessly
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = cudaFuncSetAttribute(fp8_few_kernel<T, X>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    FewParams p;
    memset(&p, 0, sizeof p);
    p.x = a.x; p.ldx = a.ldx; p.x_scales = reinterpret_cast<const uint8_t*>(a.x_scales); p.scales = a.scales; p.y = a.y; p.ldy = a.ldy;
    p.status = reinterpret_cast<unsigned int*>(a.workspace);
    p.y_type = a.y_type; p.M = a.M; p.N = a.N; p.K = a.K; p.G = (a.K + f8::kBlock - 1) / f8::kBlock; p.Mp = a.Mp;
    CUtensorMap w_map, x_map;
    if (!make_byte_map(&w_map, a.codes, a.N, a.K, 128)) return cudaErrorUnknown;
    if (C::TAKES_X) x_map = w_map;                    // not used
    else if (!make_byte_map(&x_map, a.x_codes, a.M, a.K, T)) return cudaErrorUnknown;
    const long long tiles = static_cast<long long>((a.N + 127) / 128) * ((a.M + T - 1) / T);
    p.ranks = few_cluster(tiles, p.G, C::PER_SM * device_sm_count());
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(static_cast<unsigned>(tiles * p.ranks), 1, 1);
    cfg.blockDim = dim3(kFewThreads, 1, 1);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = a.stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(p.ranks); attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, fp8_few_kernel<T, X>, w_map, x_map, p);
}
template <typename X>
static cudaError_t few_by_tokens(const Fp8Args& a) {
    if (a.M <= 16) return few_launch<16, X>(a);
    if (a.M <= 32) return few_launch<32, X>(a);
    if (a.M <= 64) return few_launch<64, X>(a);
    return few_launch<128, X>(a);
}
bool fp8_few_takes_x(int M) { return M <= 32; }
cudaError_t fp8_few(const Fp8Args& a) { return a.x_type == SLIM_F16 ? few_by_tokens<__half>(a) : few_by_tokens<__nv_bfloat16>(a); }

}  // namespace slim
