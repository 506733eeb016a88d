// slim_fp8_quantize, slim_fp8_linear: a linear layer in 8-bit floats (e4m3), the group-wise layer's counterpart for the weights that
// one to four bits do not do: W in blocks of 128 x 128 with one fp32 scale each, x quantised inside the call in blocks of 128 columns of a token,
//     y[m][n] = sum_g sx[m][g] * sw[n / 128][g] * sum_{k in block g} xq[m][k] * wq[n][k]
// on the tensor cores (tcgen05, e4m3 in, fp32 accumulator), which apply the scales too: they are powers of two.
// This file: the two quantizers, which kernel a call goes to, and the entry points.
#include "slim_fp8.cuh"

#include <atomic>

namespace slim {

// ------------------------------------------------------------------------------------------ W
// A block of 256 threads per 128 x 128 block of W; thread (r, c): row r + 16 i, columns 8c .. 8c + 7.  Bound: HBM, one read and
// one write; the block stays in registers between its maximum and its codes (23 us at 11008 x 4096 bf16, 5.8 TB/s).
// Eight elements of W as they lie in memory, their largest magnitude (as fp32 bits; anything from infinity's on is not finite), their codes.
template <typename T> struct W8 {
    uint4 v;
    __device__ __forceinline__ void load(const T* p) { v = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void unpack(float* f) const { f8::Half16<T>::unpack(v, f); }
    // over several: halves of 16 bits, joined at the end
    __device__ __forceinline__ void top(uint32_t& m) const { m = __vmaxu2(m, f8::top2(v)); }
    static __device__ __forceinline__ uint32_t join(uint32_t m) {
        m = max(m & 0xffffu, m >> 16);
        return __float_as_uint(f8::Half16<T>::one(m));
    }
};
template <> struct W8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = __ldcs(reinterpret_cast<const float4*>(p)); b = __ldcs(reinterpret_cast<const float4*>(p) + 1); }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void unpack(float* f) const { f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w; }
    __device__ __forceinline__ void top(uint32_t& m) const {
        float f[8];
        unpack(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(f[e]) & 0x7fffffffu);
    }
    static __device__ __forceinline__ uint32_t join(uint32_t m) { return m; }
};
template <typename T>
__global__ void __launch_bounds__(256) fp8_quantize_kernel(const T* __restrict__ W, long long ld, uint8_t* __restrict__ codes,
                                                           float* __restrict__ scales, int N, int K) {
    __shared__ uint32_t s_max[8];
    const int tid = threadIdx.x, c = tid & 15, r = tid >> 4;
    const int n0 = blockIdx.y * f8::kBlock, k = blockIdx.x * f8::kBlock + 8 * c;
    W8<T> v[8];
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int n = n0 + r + 16 * i;
        if (n < N && k < K) v[i].load(W + static_cast<size_t>(n) * ld + k);
        else v[i].zero();
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i].top(mx);
    mx = __reduce_max_sync(0xffffffffu, W8<T>::join(mx));
    if ((tid & 31) == 0) s_max[tid >> 5] = mx;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) mx = max(mx, s_max[w]);
    const bool finite = mx < 0x7f800000u;
    if (!finite) {                                     // the whole block of threads: once more, of what is finite
        mx = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float f[8];
            v[i].unpack(f);
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = max(mx, f8::magnitude(f[e]));
        }
        mx = __reduce_max_sync(0xffffffffu, mx);
        __syncthreads();
        if ((tid & 31) == 0) s_max[tid >> 5] = mx;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) mx = max(mx, s_max[w]);
    }
    const uint32_t sb = f8::scale_bits(mx);
    const float inv = f8::inverse_scale(sb);
    if (tid == 0) scales[static_cast<size_t>(blockIdx.y) * gridDim.x + blockIdx.x] = __uint_as_float(sb);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int n = n0 + r + 16 * i;
        if (n < N && k < K) {
            float f[8];
            v[i].unpack(f);
            *reinterpret_cast<uint2*>(codes + static_cast<size_t>(n) * K + k) =
                finite ? make_uint2(f8::codes4<false>(f, inv), f8::codes4<false>(f + 4, inv)) : make_uint2(f8::codes4<true>(f, inv), f8::codes4<true>(f + 4, inv));
        }
    }
}

// ------------------------------------------------------------------------------------------ x
// Half a warp per four blocks of 128 columns of a token, 8 columns of each per lane: four loads in flight per thread and one word of
// scale exponents (1280 blocks of threads at 2048 x 5120, one wave; 7.6 us, 16 at 1000 x 32000, 6 TB/s).  The kernel that reads the codes may be set up meanwhile.
template <typename T>
__global__ void __launch_bounds__(256) fp8_stage_kernel(const T* __restrict__ x, long long ld, uint8_t* __restrict__ codes,
                                                        uint32_t* __restrict__ scales, int M, int K, int words, int Mp) {
    pdl_wait();
    pdl_launch_dependents();                           // in this order: the kernel behind may read W at once
    const long long unit = (static_cast<long long>(blockIdx.x) * 256 + threadIdx.x) >> 4;
    const int c = threadIdx.x & 15;
    const int m = static_cast<int>(unit / words), j = static_cast<int>(unit - static_cast<long long>(m) * words);
    const T* row = x + static_cast<size_t>(m) * ld;
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = (4 * j + i) * f8::kBlock + 8 * c;
        v[i] = m < M && k < K ? __ldg(reinterpret_cast<const uint4*>(row + k)) : make_uint4(0, 0, 0, 0);
    }
    uint2 q[4];
    uint32_t e[4];
    f8::quantise8<T>(v, q, e);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = (4 * j + i) * f8::kBlock + 8 * c;
        if (m < M && k < K) *reinterpret_cast<uint2*>(codes + static_cast<size_t>(m) * K + k) = q[i];
    }
    const uint32_t word = e[0] | e[1] << 8 | e[2] << 16 | e[3] << 24;
    if (c == 0 && m < M) scales[static_cast<size_t>(j) * Mp + m] = word;
}

static cudaError_t fp8_stage(const Fp8Args& a, uint8_t* codes, uint32_t* scales, int Mp) {
    const int words = (a.K + 4 * f8::kBlock - 1) / (4 * f8::kBlock);
    const long long units = static_cast<long long>(a.M) * words;
    PdlLaunch l(static_cast<unsigned>((units + 15) / 16), 256, 0, a.stream);
    if (a.x_type == SLIM_F16)
        return cudaLaunchKernelEx(&l.cfg, fp8_stage_kernel<__half>, static_cast<const __half*>(a.x), a.ldx, codes, scales, a.M, a.K, words, Mp);
    return cudaLaunchKernelEx(&l.cfg, fp8_stage_kernel<__nv_bfloat16>, static_cast<const __nv_bfloat16*>(a.x), a.ldx, codes, scales, a.M, a.K, words, Mp);
}

// ------------------------------------------------------------------------------------------ tensor maps
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool make_byte_map(CUtensorMap* map, const void* p, int rows, int cols, int box_rows) {
    static std::atomic<EncodeTiledFn> found{nullptr};
    EncodeTiledFn enc = found.load();
    if (enc == nullptr) {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess) return false;
        enc = reinterpret_cast<EncodeTiledFn>(sym);
        found.store(enc);
    }
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(cols)};
    const cuuint32_t box[2] = {128u, static_cast<cuuint32_t>(box_rows)};
    const cuuint32_t estr[2] = {1u, 1u};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int fp8_shape(int M, int N, int K) {
    if (M < 0 || N < 0 || K < 0) return SLIM_ERR_INVALID_ARG;
    if (K % 16 != 0 || K > SLIM_FP8_MAX_K || M > SLIM_FP8_MAX_M || N > SLIM_FP8_MAX_N) return SLIM_ERR_UNSUPPORTED;
    return SLIM_OK;
}

}  // namespace slim

extern "C" int slim_fp8_quantize(const void* W, int type, long long ld, void* codes, float* scales, int N, int K, void* stream) {
    const int st = slim::fp8_shape(0, N, K);
    if (st != SLIM_OK) return st;
    if ((type != SLIM_F32 && type != SLIM_F16 && type != SLIM_BF16) || ld < K) return SLIM_ERR_INVALID_ARG;
    if (N == 0 || K == 0) return SLIM_OK;
    if (W == nullptr || codes == nullptr || scales == nullptr) return SLIM_ERR_INVALID_ARG;
    if (!slim::aligned16(W) || !slim::aligned16(codes) || !slim::aligned16(scales) || ld % (type == SLIM_F32 ? 4 : 8) != 0) return SLIM_ERR_ALIGNMENT;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid((K + 127) / 128, (N + 127) / 128);
    uint8_t* c = static_cast<uint8_t*>(codes);
    if (type == SLIM_F32) slim::fp8_quantize_kernel<float><<<grid, 256, 0, s>>>(static_cast<const float*>(W), ld, c, scales, N, K);
    else if (type == SLIM_F16) slim::fp8_quantize_kernel<__half><<<grid, 256, 0, s>>>(static_cast<const __half*>(W), ld, c, scales, N, K);
    else slim::fp8_quantize_kernel<__nv_bfloat16><<<grid, 256, 0, s>>>(static_cast<const __nv_bfloat16*>(W), ld, c, scales, N, K);
    SLIM_CUDA_TRY(cudaGetLastError());
    return SLIM_OK;
}

extern "C" int slim_fp8_workspace_bytes(int M, int N, int K, size_t* out_bytes) {
    if (out_bytes == nullptr) return SLIM_ERR_INVALID_ARG;
    const int st = slim::fp8_shape(M, N, K);
    if (st != SLIM_OK) return st;
    *out_bytes = M == 0 || slim::fp8_few_takes_x(M) ? slim::kWsFlagsOffset + slim::kWsFlagsBytes : slim::fp8_staging(M, K).bytes;
    return SLIM_OK;
}

extern "C" int slim_fp8_linear(const void* x, int x_type, long long ldx, const void* codes, const float* scales, void* y, int y_type, long long ldy,
                               int M, int N, int K, void* workspace, size_t workspace_bytes, void* stream) {
    const int st = slim::fp8_shape(M, N, K);
    if (st != SLIM_OK) return st;
    if ((x_type != SLIM_F16 && x_type != SLIM_BF16) || (y_type != x_type && y_type != SLIM_F32) || ldx < K || ldy < N) return SLIM_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return SLIM_OK;
    if (y == nullptr) return SLIM_ERR_INVALID_ARG;
    if (!slim::aligned16(y)) return SLIM_ERR_ALIGNMENT;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (K == 0) {                                      // an empty sum
        const size_t es = y_type == SLIM_F32 ? 4 : 2;
        SLIM_CUDA_TRY(cudaMemset2DAsync(y, static_cast<size_t>(ldy) * es, 0, static_cast<size_t>(N) * es, static_cast<size_t>(M), s));
        return SLIM_OK;
    }
    if (x == nullptr || codes == nullptr || scales == nullptr) return SLIM_ERR_INVALID_ARG;
    if (!slim::aligned16(x) || !slim::aligned16(codes) || !slim::aligned16(scales) || ldx % 8 != 0) return SLIM_ERR_ALIGNMENT;
    size_t need = 0;
    slim_fp8_workspace_bytes(M, N, K, &need);
    if (workspace == nullptr || workspace_bytes < need) return SLIM_ERR_WORKSPACE;
    if (!slim::aligned16(workspace)) return SLIM_ERR_ALIGNMENT;
    const long long ys = y_type == SLIM_F32 ? 4 : 2;
    if (slim::fp8_few_takes_x(M) && slim::rows_share(x, 2 * ldx, 2ll * K, y, ys * ldy, ys * N, M)) return SLIM_ERR_INVALID_ARG;
    slim::Fp8Args a;
    memset(&a, 0, sizeof a);
    a.x = x; a.x_type = x_type; a.ldx = ldx;
    a.codes = static_cast<const uint8_t*>(codes); a.scales = scales;
    a.y = y; a.y_type = y_type; a.ldy = ldy;
    a.M = M; a.N = N; a.K = K;
    a.workspace = static_cast<uint8_t*>(workspace);
    a.stream = s;
    if (!slim::fp8_few_takes_x(M)) {
        const slim::Fp8Staging sg = slim::fp8_staging(M, K);
        SLIM_CUDA_TRY(slim::fp8_stage(a, a.workspace + sg.codes, reinterpret_cast<uint32_t*>(a.workspace + sg.scales), sg.Mp));
        a.x_codes = a.workspace + sg.codes;
        a.x_scales = reinterpret_cast<const uint32_t*>(a.workspace + sg.scales);
        a.Mp = sg.Mp;
    }
    SLIM_CUDA_TRY(slim::fp8_use_gemm(M, N, K) ? slim::fp8_gemm(a) : slim::fp8_few(a));
    return SLIM_OK;
}
