// The 8-bit linear layer for few tokens: W is the M dimension of the MMA (128 rows per CTA), up to 128 tokens its N dimension.
//
// Bound: HBM, the codes of W (one byte per weight).  A tile of 128 rows is cut along K over the CTAs of a cluster, so that
// narrow layers too have about two CTAs per SM and most of what a CTA reads is in flight at once: TMA brings 128 x 128 bytes per block of
// 128 columns into a ring of 128-byte-swizzled slots, and four K = 32 MMAs per block (block-scaled, E8M0: see slim_fp8_gemm.cu) add it to D in
// tensor memory.  Both operands' scales of a block are one byte per row, written to tensor memory by tcgen05.st (row r's at lane r % 32 of column
// r / 32, the same in all lane quarters) into a buffer per slot.  At the end the CTAs of a cluster add their sums through
// distributed shared memory, every CTA a share of the tokens, in rank order: no workspace, no second kernel, one result.
//
// Up to 16 tokens x is quantised here (TAKES_X), by four warps that take the blocks in turn, from x itself: every CTA does it for its part of K,
// which costs L2 reads of 2 T bytes per 128 bytes of W and saves the launch of the quantizer (us, here / by the quantizer: 4096 x 4096 at 1 and 16
// tokens 6.2 / 7.3 and 7.7 / 8.1, 32000 x 4096 24.2 / 25.9 and 24.3 / 25.8; at 32 tokens 9.5 / 8.7 and 31.8 / 26.1).  Beyond, the codes come
// by TMA from the workspace (slim_fp8.cu); W is then requested while the quantizer still runs.
//
// Measured, call after call (the bytes at the copy rate in brackets): 1 x 4096 x 4096 5.7 us (2.6), 16 x 11008 x 4096 11.6 (7.1), 33 x 11008 x 4096 13.9
// (7.3), 77 x 32003 x 4112 38 (22).  W streams at 5.5 to 7 TB/s once it runs; the rest is set-up, the first block's way, and the meeting at the end.
//
// Warps: 0 loads of W (and of staged x); 1 MMAs, tensor memory; 4 to 7 scales, then the output (tensor-memory lanes 32 (w % 4) on); 2, 3, 8, 9
// quantisation of x.  Every wait is bounded and reports through the workspace status word.
#include "slim_fp8.cuh"

#include <atomic>

namespace slim {

constexpr int kFewXWarps = 4;
constexpr int kFewMaxCluster = 8;

template <int T> struct FewCfg {
    static constexpr bool TAKES_X = T <= 16;
    static constexpr int THREADS = TAKES_X ? 320 : 256;
    static constexpr int W_BYTES = 128 * 128, X_BYTES = T * 128;
    static constexpr int STAGES = T <= 16 ? 5 : T <= 32 ? 4 : 3;
    static constexpr bool OWN_RECV = T <= 64;                             // the others' sums have a place of their own, not the ring's
    static constexpr int COL_SF = T;                                      // tensor memory: D, then per slot 4 columns of W's scales and T / 32 of x's
    static constexpr int TMEM_USED = T + 8 * STAGES;
    static constexpr int TMEM = TMEM_USED <= 64 ? 64 : TMEM_USED <= 128 ? 128 : 256;
    static constexpr int OFF_SX = STAGES * (W_BYTES + X_BYTES);           // TAKES_X: [STAGES][T] scale exponents
    static constexpr int OFF_RECV = OWN_RECV ? OFF_SX + STAGES * T : 0;   // [ranks][share of the tokens][128] fp32
    static constexpr int RECV = (T + 8) * 512;
    static constexpr int OFF_BAR = OFF_SX + STAGES * T + (OWN_RECV ? RECV : 0);
    static constexpr int SMEM = OFF_BAR + 256 + 1024;                     // + alignment of the slots
};

struct FewParams {
    const void* x;
    long long ldx;
    const uint32_t* x_scales;    // staged: exponents of four blocks in a word, [ceil(G / 4)][Mp]
    const float* scales;
    void* y;
    long long ldy;
    unsigned int* status;
    int y_type, M, N, K, G, Mp, ranks;
};

namespace few {
__device__ __forceinline__ void mma_scaled(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
}
}  // namespace few

template <int T, typename X>
__global__ void __launch_bounds__(FewCfg<T>::THREADS, 2)
fp8_few_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map, const FewParams p) {
    using C = FewCfg<T>;
    extern __shared__ unsigned char few_raw[];
    unsigned char* smem = few_raw + ((1024u - (smem_u32(few_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const uint32_t s_x = base + C::STAGES * C::W_BYTES, bars = base + C::OFF_BAR;
    auto w_full = [&](int s) { return bars + 8u * s; };                   // W's block, and staged x's, has landed
    auto x_full = [&](int s) { return bars + 8u * (C::STAGES + s); };     // TAKES_X: x's codes and exponents are written
    auto sf_full = [&](int s) { return bars + 8u * (2 * C::STAGES + s); };
    auto empty = [&](int s) { return bars + 8u * (3 * C::STAGES + s); };
    const uint32_t d_full = bars + 8u * (4 * C::STAGES);
    static_assert(8 * (4 * C::STAGES + 1) <= 240, "room for the barriers");
    volatile int* abort = reinterpret_cast<volatile int*>(smem + C::OFF_BAR + 240);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + C::OFF_BAR + 244);

    const int tid = threadIdx.x, lane = tid & 31, warp = static_cast<int>(tc::uniform(tid >> 5));
    const int rank = static_cast<int>(blockIdx.x) % p.ranks, tile = static_cast<int>(blockIdx.x) / p.ranks;
    const int row_tiles = (p.N + 127) / 128;
    const int nb = tile % row_tiles, n0 = 128 * nb, m0 = tile / row_tiles * T;
    const int tokens = min(T, p.M - m0);
    const int g0 = static_cast<int>(static_cast<long long>(p.G) * rank / p.ranks), g1 = static_cast<int>(static_cast<long long>(p.G) * (rank + 1) / p.ranks);
    const int steps = g1 - g0;                         // at least 1: there are no more ranks than blocks

    if (tid == 0) {
        *abort = 0;
        for (int s = 0; s < C::STAGES; ++s) {
            sb::init(w_full(s), 1);
            sb::init(x_full(s), 1);
            sb::init(sf_full(s), 4);
            sb::init(empty(s), 1);
        }
        sb::init(d_full, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&w_map)) : "memory");
        if (!C::TAKES_X) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&x_map)) : "memory");
    }
    if (warp == 1) {
        tc::alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), C::TMEM);
        tc::relinquish();
    }
    if (C::TAKES_X) {                                  // tokens past the last stay zero
        for (int i = tid; i < C::STAGES * C::X_BYTES / 16; i += C::THREADS)
            *reinterpret_cast<uint4*>(smem + C::STAGES * C::W_BYTES + 16 * i) = make_uint4(0, 0, 0, 0);
        for (int i = tid; i < C::STAGES * T; i += C::THREADS) smem[C::OFF_SX + i] = 127;
        tc::fence_proxy_async();
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tc::uniform(*tmem_slot);
    const bool meet = C::OWN_RECV && p.ranks > 1;
    if (meet) cluster_arrive_relaxed();                // a CTA is written to only when it is known to have started
    pdl_launch_dependents();
    // The kernel ahead of staged x is its quantizer, which lets this one start only when all before it has completed: W is there.
    int first = 0;                                     // blocks of W requested ahead
    if (!C::TAKES_X && warp == 0) {
        first = min(steps, C::STAGES);
        if (tc::elect())
            for (int i = 0; i < first; ++i) {
                sb::expect_tx(w_full(i), C::W_BYTES + C::X_BYTES);
                tc::tma_load_2d(base + i * C::W_BYTES, &w_map, 128 * (g0 + i), n0, w_full(i));
            }
        __syncwarp();
    }
    pdl_wait();

    if (warp == 0) {
        // ---- W, and the codes of staged x
        int s = 0;
        uint32_t ph = 0;
        for (int i = 0; i < steps; ++i) {
            if (!tc::warp_wait(empty(s), ph ^ 1u, abort)) break;
            if (tc::elect()) {
                if (i >= first) {
                    sb::expect_tx(w_full(s), C::TAKES_X ? C::W_BYTES : C::W_BYTES + C::X_BYTES);
                    tc::tma_load_2d(base + s * C::W_BYTES, &w_map, 128 * (g0 + i), n0, w_full(s));
                }
                if (!C::TAKES_X) tc::tma_load_2d(s_x + s * C::X_BYTES, &x_map, 128 * (g0 + i), m0, w_full(s));
            }
            __syncwarp();
            if (++s == C::STAGES) { s = 0; ph ^= 1u; }
        }
    } else if (warp == 1) {
        // ---- MMAs
        // e4m3 operands, both K-major, E8M0 scales (the lowest byte of their words), 128 x T
        constexpr uint32_t idesc = (static_cast<uint32_t>(T >> 3) << 17) | (1u << 23) | (1u << 27);
        int s = 0;
        uint32_t ph = 0;
        for (int i = 0; i < steps; ++i) {
            if (!tc::warp_wait(sf_full(s), ph, abort)) break;             // behind x_full, where x is quantised here
            if (!tc::warp_wait(w_full(s), ph, abort)) break;
            tc::fence_after();
            const uint64_t a = tc::desc_k128(base + s * C::W_BYTES), x = tc::desc_k128(s_x + s * C::X_BYTES);
            const uint32_t sf = tmem + C::COL_SF + 8u * s;
            if (tc::elect()) {
#pragma unroll
                for (int k = 0; k < 4; ++k) few::mma_scaled(tmem, a + 2 * k, x + 2 * k, idesc, sf, sf + 4, i > 0 || k > 0 ? 1u : 0u);
                tc::commit(empty(s));
                if (i + 1 == steps) tc::commit(d_full);
            }
            __syncwarp();
            if (++s == C::STAGES) { s = 0; ph ^= 1u; }
        }
    } else if (warp >= 4 && warp < 8) {
        // ---- scales: this warp's quarter of the lanes, of the 128 rows (one scale) and of all tokens
        const uint32_t sf_t = tmem + C::COL_SF + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
        const float* sw = p.scales + static_cast<size_t>(nb) * p.G + g0;
        uint32_t w_now = 0, w_next = lane < steps ? __float_as_uint(__ldg(sw + lane)) : 0u;      // a lane holds one of 32 blocks'
        constexpr int XC = (T + 31) / 32;
        uint32_t x_now[XC], x_next[XC];
        auto x_words = [&](int g, uint32_t* v) {
#pragma unroll
            for (int c = 0; c < XC; ++c) v[c] = g < g1 ? __ldcg(p.x_scales + static_cast<size_t>(g >> 2) * p.Mp + min(m0 + 32 * c + lane, p.Mp - 1)) : 0u;
        };
        if (!C::TAKES_X) x_words(g0, x_next);
        int s = 0;
        uint32_t ph = 0;
        for (int i = 0; i < steps; ++i) {
            if ((i & 31) == 0) {
                w_now = w_next;
                w_next = i + 32 + lane < steps ? __float_as_uint(__ldg(sw + i + 32 + lane)) : 0u;
            }
            const uint32_t w = f8::e8m0(__shfl_sync(0xffffffffu, w_now, i & 31));
            uint32_t v[8] = {w, w, w, w, 0, 0, 0, 0};
            if (C::TAKES_X) {
                if (!tc::warp_wait(x_full(s), ph, abort)) break;
                tc::fence_after();
                v[4] = lane < T ? smem[C::OFF_SX + s * T + lane] : 127;
            } else {
                const int g = g0 + i;
                if (i == 0 || (g & 3) == 0) {
#pragma unroll
                    for (int c = 0; c < XC; ++c) x_now[c] = x_next[c];
                    x_words((g & ~3) + 4, x_next);
                }
                if (!tc::warp_wait(empty(s), ph ^ 1u, abort)) break;
                tc::fence_after();
#pragma unroll
                for (int c = 0; c < XC; ++c) v[4 + c] = x_now[c] >> (8 * (g & 3)) & 0xffu;
            }
            tc::st8(sf_t + 8u * s, v);
            tc::wait_st();
            tc::fence_before();
            __syncwarp();
            if (lane == 0) sb::arrive(sf_full(s));
            if (++s == C::STAGES) { s = 0; ph ^= 1u; }
        }
    } else if (C::TAKES_X) {
        // ---- x into codes: half a warp per token and block, two tokens of a warp at a time, one block in four
        const int xw = warp < 4 ? warp - 2 : warp - 6;
        constexpr int TURNS = kFewXWarps;
        static_assert(!C::TAKES_X || TURNS <= C::STAGES, "the first blocks of the warps have slots of their own");
        const int half = lane >> 4, c = lane & 15;
        const X* x = static_cast<const X*>(p.x) + static_cast<size_t>(m0) * p.ldx;
        uint4 v[8];
        auto fetch = [&](int i) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int t = 2 * u + half, k = 128 * (g0 + i) + 8 * c;
                v[u] = i < steps && t < tokens && k < p.K ? __ldg(reinterpret_cast<const uint4*>(x + static_cast<size_t>(t) * p.ldx + k)) : make_uint4(0, 0, 0, 0);
            }
        };
        int s = xw;
        uint32_t ph = 0;
        fetch(s);
        for (int i = s; i < steps; i += TURNS) {
            if (!tc::warp_wait(empty(s), ph ^ 1u, abort)) break;
            // tokens past the last are zeros, with codes of zeros
            uint2 codes[8];
            uint32_t e[8];
            auto put = [&](int u) {
                // row t of a swizzled tile: its 16-byte chunks stand at chunk ^ (t & 7)
                const int t = 2 * u + half;
                const uint32_t at = s_x + s * C::X_BYTES + t * 128 + ((((c >> 1) ^ (t & 7)) << 4) | ((c & 1) << 3));
                asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(at), "r"(codes[u].x), "r"(codes[u].y) : "memory");
                if (c == 0) smem[C::OFF_SX + s * T + t] = static_cast<uint8_t>(e[u]);
            };
            if (tokens <= 2) {                         // one pair: the others' slots are zero from the start
                uint4 one[1] = {v[0]};
                uint2 q[1];
                uint32_t x1[1];
                f8::quantise8<X>(one, q, x1);
                codes[0] = q[0];
                e[0] = x1[0];
                put(0);
            } else {
                f8::quantise8<X>(v, codes, e);
#pragma unroll
                for (int u = 0; u < 8; ++u) put(u);
            }
            fetch(i + TURNS);
            tc::fence_proxy_async();
            __syncwarp();
            if (lane == 0) sb::arrive(x_full(s));
            s += TURNS;
            if (s >= C::STAGES) { s -= C::STAGES; ph ^= 1u; }
        }
    }

    // ---- D is complete; after a wait that gave up, what is in flight has landed before the shared memory is used again
    bool done = true;
    if (warp >= 4 && warp < 8) done = tc::warp_wait(d_full, 0, abort);
    if (warp == 0 && *abort != 0)
        for (int s = 0; s < C::STAGES; ++s) {
            if (tc::elect()) { f8::drain(w_full(s), 0); f8::drain(w_full(s), 1); }
            __syncwarp();
        }
    if (warp == 1 && *abort != 0)
        for (int s = 0; s < C::STAGES; ++s) {
            if (tc::elect()) { f8::drain(empty(s), 0); f8::drain(empty(s), 1); }
            __syncwarp();
        }
    if (meet) cluster_wait();
    if (!C::OWN_RECV && p.ranks > 1) cluster_sync_all();      // everyone's ring is free
    else __syncthreads();
    tc::fence_after();
    if (warp >= 4 && warp < 8 && done) {
        const int row = 32 * (warp & 3) + lane;
        const uint32_t d_t = tmem + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
        int owner = 0, u = 0;                          // of the token: its CTA, its place there
        const int share = (tokens + p.ranks - 1) / p.ranks;
#pragma unroll 1
        for (int t0 = 0; t0 < tokens; t0 += 16) {
            uint32_t d[16];
            f8::ld16(d_t + t0, d);
            tc::wait_ld();
            if (p.ranks > 1) {
#pragma unroll
                for (int t = 0; t < 16; ++t) {
                    if (t0 + t < tokens) {
                        uint32_t remote;
                        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(base + C::OFF_RECV + 4u * ((rank * share + u) * 128 + row)), "r"(owner));
                        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote), "r"(d[t]) : "memory");
                    }
                    if (++owner == p.ranks) { owner = 0; ++u; }
                }
            } else if (n0 + row < p.N) {
                const size_t at = static_cast<size_t>(m0 + t0) * p.ldy + n0 + row;
                const int n = min(16, tokens - t0);
                f8::store_column(p.y, p.y_type, at, p.ldy, d, n);
            }
        }
    }
    if (p.ranks > 1) {
        cluster_sync_all();
        // every CTA adds its share of the tokens, 128 rows of one per four warps
        constexpr int turns = C::THREADS / 128;
        const int turn = tid >> 7, row = tid & 127, share = (tokens + p.ranks - 1) / p.ranks;
        if (turn < turns && n0 + row < p.N) {
            const float* recv = reinterpret_cast<const float*>(smem + C::OFF_RECV) + row;
            for (int u = turn; rank + p.ranks * u < tokens; u += turns) {
                float y = recv[u * 128];
#pragma unroll
                for (int r = 1; r < kFewMaxCluster; ++r)
                    if (r < p.ranks) y += recv[(r * share + u) * 128];
                f8::store_y(p.y, p.y_type, static_cast<size_t>(m0 + rank + p.ranks * u) * p.ldy + n0 + row, y);
            }
        }
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == 1) tc::dealloc(tmem, C::TMEM);
    if (tid == 0 && *abort != 0) report_timeout(p.status, false);
}

// ------------------------------------------------------------------------------------------ host side
// Cut of a tile's K over c CTAs: time in blocks of 128 columns, of which a CTA's start and end cost about four.  It compares cuts of one call; what is the same
// in all of them (launches, quantizer) does not count here, but does in fp8_few_cycles, which stands against another kernel's time.
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
    p.x = a.x; p.ldx = a.ldx; p.x_scales = a.x_scales; p.scales = a.scales; p.y = a.y; p.ldy = a.ldy;
    p.status = reinterpret_cast<unsigned int*>(a.workspace);
    p.y_type = a.y_type; p.M = a.M; p.N = a.N; p.K = a.K; p.G = (a.K + f8::kBlock - 1) / f8::kBlock; p.Mp = a.Mp;
    CUtensorMap w_map, x_map;
    if (!make_byte_map(&w_map, a.codes, a.N, a.K, 128)) return cudaErrorUnknown;
    if (C::TAKES_X) x_map = w_map;                    // not used
    else if (!make_byte_map(&x_map, a.x_codes, a.M, a.K, T)) return cudaErrorUnknown;
    const long long tiles = static_cast<long long>((a.N + 127) / 128) * ((a.M + T - 1) / T);
    p.ranks = few_cluster(tiles, p.G, 2 * device_sm_count());
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(static_cast<unsigned>(tiles * p.ranks), 1, 1);
    cfg.blockDim = dim3(C::THREADS, 1, 1);
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
bool fp8_few_takes_x(int M) { return M <= 16; }
// Cycles from 65 tokens on: a block of a CTA takes 1300 (its W, two CTAs per SM, at HBM's rate), a CTA 9000 beside its blocks.
double fp8_few_cycles(int M, int N, int K) {
    const long long tiles = static_cast<long long>((N + 127) / 128) * ((M + 127) / 128);
    const int G = (K + f8::kBlock - 1) / f8::kBlock, slots = 2 * device_sm_count(), c = few_cluster(tiles, G, slots);
    return static_cast<double>((tiles * c + slots - 1) / slots) * ((G + c - 1) / c * 1300.0 + 9000.0);
}
cudaError_t fp8_few(const Fp8Args& a) { return a.x_type == SLIM_F16 ? few_by_tokens<__half>(a) : few_by_tokens<__nv_bfloat16>(a); }

}  // namespace slim
