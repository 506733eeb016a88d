// Shared by the kernels of the 8-bit linear layer: the block scale, the codes of 8 elements, element types.
#pragma once

#include "slim_tc.cuh"

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp8.h>

namespace slim {
namespace f8 {

constexpr int kBlock = 128;                        // columns, and rows of W, that share a scale

// The smallest power of two s >= amax / 448 (448 = 1.75 * 2^8 is e4m3's largest value), at least 2^-126; 1 for a block of zeros.
// A power of two, so that v / s is exact and the code's is the only rounding: a block's codes do not depend on how the division is done,
// and e4m3 being a floating-point type nothing is lost by it but at most one bit of the exponent's range.
// `amax` as bits of a finite fp32 value >= 0.
__device__ __forceinline__ uint32_t scale_bits(uint32_t amax) {
    if (amax == 0) return 127u << 23;
    if (amax < (1u << 23)) return 1u << 23;        // a subnormal maximum: the scale's lower bound
    const int e = static_cast<int>(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return static_cast<uint32_t>(max(e, 1)) << 23;
}
// 1 / s for s of scale_bits (2^-126 .. 2^120): exact.
__device__ __forceinline__ float inverse_scale(uint32_t bits) { return __uint_as_float((254u << 23) - bits); }

// E8M0 of a scale of W: its exponent if it is a power of two from 2^-126 to 2^127, else 255, NaN, so that no other scale passes for the power of two below it.
__device__ __forceinline__ uint32_t e8m0(uint32_t bits) {
    const uint32_t e = bits >> 23;                 // 256 and more with a sign
    return (bits & 0x7fffffu) == 0 && e - 1u < 254u ? e : 255u;
}

// Four codes of v * inv.  NaN gives NaN (0x7f or 0xff); `checked` makes NaN of infinities too (e4m3 has none, and 448 would pass for a value).
template <bool checked>
__device__ __forceinline__ uint32_t codes4(const float* v, float inv) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(v[1] * inv), "f"(v[0] * inv));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(v[3] * inv), "f"(v[2] * inv));
    uint32_t r = static_cast<uint32_t>(lo) | static_cast<uint32_t>(hi) << 16;
    if (checked) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (!(fabsf(v[i]) <= 3.402823466e38f)) r |= 0x7fu << (8 * i);
    }
    return r;
}
// Magnitude for the block's maximum: what is not finite does not count.
__device__ __forceinline__ uint32_t magnitude(float v) {
    const uint32_t m = __float_as_uint(v) & 0x7fffffffu;
    return m < 0x7f800000u ? m : 0u;
}

// Eight elements of a 16-bit type as floats, the bits of its infinity, and one from its bits.
template <typename T> struct Half16;
template <> struct Half16<__half> {
    static constexpr uint32_t INF = 0x7c00u;
    static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = t.x; f[2 * i + 1] = t.y;
        }
    }
    static __device__ __forceinline__ float one(uint32_t bits) { return __half2float(__ushort_as_half(static_cast<unsigned short>(bits))); }
};
template <> struct Half16<__nv_bfloat16> {
    static constexpr uint32_t INF = 0x7f80u;
    static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ float one(uint32_t bits) { return __uint_as_float(bits << 16); }
};
// Largest magnitudes of eight elements, as bits, in two halves: without their signs the bits are in the order of the values.
__device__ __forceinline__ uint32_t top2(const uint4& v) {
    return __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
}
// Blocks of 128 that half a warp holds, eight elements a lane and block: this lane's codes, and the scales' exponents.  All lanes of the warp take
// part.  What is not finite is looked for once for all U blocks, so that their chains run side by side.
template <typename T, int U>
__device__ __forceinline__ void quantise8(const uint4 (&v)[U], uint2 (&codes)[U], uint32_t (&exponent)[U]) {
    uint32_t m[U], most = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = top2(v[u]);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
#pragma unroll
        for (int u = 0; u < U; ++u) m[u] = __vmaxu2(m[u], __shfl_xor_sync(0xffffffffu, m[u], o));
#pragma unroll
    for (int u = 0; u < U; ++u) {
        m[u] = max(m[u] & 0xffffu, m[u] >> 16);
        most = max(most, m[u]);
    }
    if (__any_sync(0xffffffffu, most >= Half16<T>::INF)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[8];
            Half16<T>::unpack(v[u], f);
            uint32_t mx = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = max(mx, magnitude(f[e]));
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const uint32_t sb = scale_bits(mx);
            const float inv = inverse_scale(sb);
            exponent[u] = sb >> 23;
            codes[u] = make_uint2(codes4<true>(f, inv), codes4<true>(f + 4, inv));
        }
        return;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[8];
        Half16<T>::unpack(v[u], f);
        const uint32_t sb = scale_bits(__float_as_uint(Half16<T>::one(m[u])));
        const float inv = inverse_scale(sb);
        exponent[u] = sb >> 23;
        codes[u] = make_uint2(codes4<false>(f, inv), codes4<false>(f + 4, inv));
    }
}

// y element: `type` is SLIM_F32, SLIM_F16 or SLIM_BF16; one rounding of the fp32 sum.
__device__ __forceinline__ void store_y(void* y, int type, size_t at, float v) {
    if (type == SLIM_F32) static_cast<float*>(y)[at] = v;
    else if (type == SLIM_F16) static_cast<__half*>(y)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(y)[at] = __float2bfloat16_rn(v);
}

// n <= 16 of them, a row stride apart.
__device__ __forceinline__ void store_column(void* y, int type, size_t at, long long ld, const uint32_t* d, int n) {
    if (type == SLIM_F32) {
        float* o = static_cast<float*>(y) + at;
#pragma unroll
        for (int t = 0; t < 16; ++t, o += ld)
            if (t < n) *o = __uint_as_float(d[t]);
    } else if (type == SLIM_F16) {
        __half* o = static_cast<__half*>(y) + at;
#pragma unroll
        for (int t = 0; t < 16; ++t, o += ld)
            if (t < n) *o = __float2half_rn(__uint_as_float(d[t]));
    } else {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(y) + at;
#pragma unroll
        for (int t = 0; t < 16; ++t, o += ld)
            if (t < n) *o = __float2bfloat16_rn(__uint_as_float(d[t]));
    }
}
// 32 lanes x 16 columns of 32 bits
__device__ __forceinline__ void ld16(uint32_t taddr, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr) : "memory");
}
// Waits, for a millisecond at most and whatever the other roles do, until a barrier's phase completes: what is in flight when a call
// gives up has landed before its shared memory goes.
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) {
    const unsigned long long t0 = sb::timer_ns();
    while (!sb::try_wait(bar, parity) && sb::timer_ns() - t0 < 1000000ull) { }
}

}  // namespace f8

// Where the quantised activations of a call lie in its workspace: behind the header and the flags of the other calls, which
// are left alone, the codes [M][K], then the scales' exponents, a word of four groups per token, [groups / 4][Mp], Mp = M rounded up to 128.
struct Fp8Staging {
    size_t codes, scales, bytes;
    int Mp;
};
inline Fp8Staging fp8_staging(int M, int K) {
    Fp8Staging s;
    s.Mp = (M + 127) / 128 * 128;
    s.codes = kWsFlagsOffset + kWsFlagsBytes;
    s.scales = (s.codes + static_cast<size_t>(M) * K + 255) / 256 * 256;
    s.bytes = s.scales + static_cast<size_t>((K + 4 * f8::kBlock - 1) / (4 * f8::kBlock)) * s.Mp * sizeof(uint32_t);
    return s;
}

struct Fp8Args {
    const void* x;            // [M][K], row stride ldx, or null when staged
    int x_type;
    long long ldx;
    const uint8_t* codes;     // [N][K]
    const float* scales;      // [ceil(N / 128)][ceil(K / 128)]
    void* y;
    int y_type;
    long long ldy;
    int M, N, K;
    uint8_t* workspace;
    const uint8_t* x_codes;   // staged
    const uint32_t* x_scales;
    int Mp;
    cudaStream_t stream;
};

// Tensor map of a matrix of bytes [rows][cols]: boxes of 128 bytes x `box_rows`, 128-byte swizzle, zeros past the ends.
bool make_byte_map(CUtensorMap* map, const void* p, int rows, int cols, int box_rows);
// The kernels for few tokens (slim_fp8_few.cu) and for many (slim_fp8_gemm.cu).
bool fp8_few_takes_x(int M);                       // quantises x itself
cudaError_t fp8_few(const Fp8Args& a);
cudaError_t fp8_gemm(const Fp8Args& a);
bool fp8_use_gemm(int M, int N, int K);
double fp8_few_cycles(int M, int N, int K);

}  // namespace slim
