// slim_distill_loss / _grad / _step: distillation from a teacher's top logits, the KL of func SBA's error measure
// (softmax over the output features of each token, Sec. 3.2.2) with a teacher of which only the k largest logits are kept, and its
// gradient with respect to the student's logits.
//
// With p = softmax(s / T) over all V logits of a row, entries (i_j, u_j) and q_j the teacher's probabilities,
//     loss   = sum_j q_j (log q_j - log p_{i_j})   [ + q' (log q' - log p') ],   q' = 1 - sum_j q_j, p' = 1 - sum of p over the set
//     dloss/ds_v = (p_v * c - sum_{j: i_j = v} q_j) / T
// without the rest q_j is the softmax over the entries and c = sum_j q_j; with it q_j = exp(u_j / T - lse), and c is
// sum_j q_j + q' for the listed columns, that less q' / p' for all others.  So a row needs its sum of exponentials (with the rest, that outside the listed
// columns, relative to the largest logit there, however far below the listed ones that lies) and k logits; then its gradient is one
// multiplication per element and k corrections.
//
// Bound: HBM (a row is read once, its gradient written once), with two ex2 per element next to it.  Two kernels: a CTA or cluster per row, and
// one that takes row after row (below).  A row belongs to 1 to 8 CTAs of 512 threads, each with a slice of its columns; a thread takes eight 16-byte
// vectors of it at a time and, in the one call for both, keeps them in registers between the statistics and the gradient; a longer row is read a second
// time, from L2.  The slices' statistics meet through distributed shared memory; every sum has a fixed order.  Sums over the columns are fp32, what is
// computed of the entries, and the loss, is fp64, because a small loss is the difference of large terms.
// Measured: loss of 512 x 152064 bf16 45 us, its gradient 55 (5.7 TB/s), both in one call 88; 777 x 50257 fp32 in one call 74, 4096 x 32000 bf16 126;
// loss of 16 x 32000 8.1, all of it latency.  Registers are held to two CTAs per SM (64 a thread, 56 in the many-rows kernel); what does not fit, up to 48 bytes a
// thread of a row's terms and addresses, is read back a few times per row.
#include "slim_exp.cuh"
#include "slim_gemv_i8.cuh"

#include <cuda_bf16.h>

#include <atomic>
#include <cmath>

namespace slim {

constexpr int kDsThreads = 512;
constexpr int kDsWarps = kDsThreads / 32;
constexpr int kDsVecs = 8;                    // vectors of 16 bytes that a thread holds
constexpr int kDsMaxCluster = 8;

enum { kDsLoss = 0, kDsGrad = 1, kDsStep = 2 };

struct DistillParams {
    const void* logits;
    const void* index;       // int32 or int64 [M][k]
    const void* value;       // [M][k]
    const float* lse;        // [M], or null: the teacher is renormalised over its entries
    const float* dloss;      // [M]
    float* loss;             // [M]
    float* saved;            // [M][4]: the largest logit outside the set, the row's sum of exponentials, that outside the set relative to the first, 0
    void* grad;
    long long ld, ldg;       // row strides in elements
    float c;                 // log2(e) / T
    double inv_t;
    int M, V, k;
    int index64, value_type;
    int ranks;               // CTAs of a row, a cluster
    int slice;               // columns of a CTA
    int mark_bytes;          // bytes of the set's marks (a byte per vector of the slice)
};

// ------------------------------------------------------------------------------------------ element types
template <uint32_t NINF2>
__device__ __forceinline__ void ds_hide16(uint4& v, uint32_t b) {
    uint32_t* w[4] = {&v.x, &v.y, &v.z, &v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {                      // bit 2i as the sign of a byte 0, bit 2i + 1 of a byte 1, spread over a half each
        uint32_t m;
        asm("prmt.b32 %0, %1, %2, 0xdd88;" : "=r"(m) : "r"(b << (7 - 2 * i)), "r"(b << (14 - 2 * i)));
        *w[i] = (*w[i] & ~m) | (NINF2 & m);
    }
}
template <typename T> struct DsType;
template <> struct DsType<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    // elements whose bit is set become minus infinity
    static __device__ __forceinline__ void hide(uint4& v, uint32_t b) {
        constexpr uint32_t NINF = 0xff800000u;
        v.x = b & 1u ? NINF : v.x; v.y = b & 2u ? NINF : v.y; v.z = b & 4u ? NINF : v.z; v.w = b & 8u ? NINF : v.w;
    }
    static __device__ __forceinline__ float one(float v) { return v; }
    static __device__ __forceinline__ float round(float v) { return v; }
};
template <> struct DsType<__half> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = t.x; f[2 * i + 1] = t.y;
        }
    }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ void hide(uint4& v, uint32_t b) { ds_hide16<0xfc00fc00u>(v, b); }
    static __device__ __forceinline__ float one(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half round(float v) { return __float2half_rn(v); }
};
template <> struct DsType<__nv_bfloat16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ void hide(uint4& v, uint32_t b) { ds_hide16<0xff80ff80u>(v, b); }
    static __device__ __forceinline__ float one(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 round(float v) { return __float2bfloat16_rn(v); }
};

// Largest of n of a thread's vectors, two elements at a time where they are 16 bits wide (a NaN loses: it shows in the sum).
template <int n>
__device__ __forceinline__ float vec_max(const uint4* x, const float*) {
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < n; ++u)
        m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(x[u].x), __uint_as_float(x[u].y)), fmaxf(__uint_as_float(x[u].z), __uint_as_float(x[u].w))));
    return m;
}
template <int n, typename H2, typename T>
__device__ __forceinline__ float vec_max2(const uint4* x, T) {
    auto h = [](const uint32_t& w) { return *reinterpret_cast<const H2*>(&w); };
    H2 m = h(x[0].x);
#pragma unroll
    for (int u = 0; u < n; ++u) m = __hmax2(m, __hmax2(__hmax2(h(x[u].x), h(x[u].y)), __hmax2(h(x[u].z), h(x[u].w))));
    const float a = DsType<T>::one(m.x), b = DsType<T>::one(m.y);
    return fmaxf(fmaxf(a, b), -INFINITY);
}
template <int n> __device__ __forceinline__ float vec_max(const uint4* x, const __half*) { return vec_max2<n, __half2>(x, __half()); }
template <int n> __device__ __forceinline__ float vec_max(const uint4* x, const __nv_bfloat16*) { return vec_max2<n, __nv_bfloat162>(x, __nv_bfloat16()); }

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pair2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// The vectors again, as values that the compiler takes for new: it would otherwise keep all of them unpacked from one pass to the next.
__device__ __forceinline__ void forget(uint4& v) { asm volatile("" : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w)); }

__device__ __forceinline__ float ex2(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float rcp(float v) {      // within an ulp
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// What a row's sums come to: R outside the set, relative to m, the largest logit there (all of the row without the rest), and z of the set's columns,
// relative to `top`, the largest of them; and the teacher's listed mass, that of the rest (0 without it) and both together.  R has a maximum of its own
// because the student may leave the rest next to nothing: relative to the row's maximum it would be nothing from a distance of 87 T on.
struct RowTerms {
    float ref, Z;            // the row's maximum (0 if that is minus infinity), the sum of all columns relative to it
    float m, R;
    float inv_z;
    float out, factor;       // of 2^((s - out) c) in the gradient of the columns outside the set, but for the row's weight; out is m, or 0 for minus infinity
};
template <bool REST>
__device__ __forceinline__ RowTerms row_terms(float c, float m, float R, float top, float z, float q_sum, float q_rest, float mass) {
    RowTerms t;
    const float most = REST ? fmaxf(m, top) : m;
    t.ref = most == -INFINITY ? 0.f : most;
    t.m = m;
    t.R = R;
    t.out = m == -INFINITY ? 0.f : m;
    float a = 1.f, r = R;                              // of the two parts the one with the smaller maximum is brought to the other's
    if (REST) {
        const float d = ex2((fminf(m, top) - t.ref) * c);
        const bool set_leads = top > m;
        a = set_leads ? d : 1.f;
        r = R * a;
        z *= set_leads ? 1.f : d;
    } else z = 0.f;
    t.Z = r + z;
    const float over = rcp(t.Z);
    t.inv_z = t.Z == 0.f ? 0.f : over;
    const float p_in = z * t.inv_z;                  // the set's mass
    t.factor = mass * a * t.inv_z;
    // p (1 - q'/p') = 2^.. (p' - q') / R, where p' is what the set leaves of 1, or r / Z where that would cancel.  R is at least 1, or 0 where there is nothing
    // outside (a NaN in the set goes through): no factor exceeds 1, whatever p' is.
    if (REST && !(q_rest == 0.f))
        t.factor = R == 0.f && t.Z == t.Z ? 0.f : (p_in < 0.5f ? q_sum - p_in : r * over - q_rest) * rcp(R);
    return t;
}
// What the entries leave of the teacher's mass.  Its log-sum-exp is fp32 and moves log q by its error: 2^-24 of the largest logit / T from the division, of the
// result from the last addition, and a few 2^-24 from the sum and its logarithm.  What is within twice that (2^-22 (1 + |lse|)) is that error and counts as
// nothing; it would otherwise be weighed against a p' that may be 0.  NaN stays NaN.
__device__ __forceinline__ double rest_mass(double q_sum, float lse) {
    const double rest = 1.0 - q_sum;
    return rest <= static_cast<double>(fminf(0x1p-22f * (1.f + fabsf(lse)), 0.5f)) ? 0.0 : rest;
}
__device__ __forceinline__ float redux_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double warp_max(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// A row's loss, in 64 bits, by a warp.  The set's mass is taken from the same log p as the entries' terms, so that an error in Z, which is fp32, shows in
// the difference of the set's two masses alone: with little in the set the loss is as small as that difference.
template <bool REST>
__device__ __forceinline__ double row_loss(const RowTerms& t, double q_rest, int k, float c, const double* s_q, const double* s_lq, const int* s_idx,
                                           const float* s_s, const uint8_t* s_first, int lane) {
    const double ln2 = 0.69314718055994530942, cd = c;
    // logarithms by a lane each
    const double v = log(lane == 0 ? static_cast<double>(t.Z) : lane == 1 ? q_rest : static_cast<double>(t.R));
    const double lz = __shfl_sync(0xffffffffu, v, 0);
    double l = 0.0, p_in = 0.0;
#pragma unroll 2
    for (int j = lane; j < k; j += 32) {
        const bool in = s_idx[j] >= 0;
        const double q = s_q[j], lp = t.Z == 0.f ? -INFINITY : (static_cast<double>(s_s[j]) - static_cast<double>(t.ref)) * cd * ln2 - lz;
        l += !in || q == 0.0 ? 0.0 : q * (s_lq[j] - lp);
        if (REST) p_in += in && s_first[j] ? exp_log(lp) : 0.0;
    }
    l = warp_sum(l);
    if (REST && !(q_rest == 0.0)) {
        p_in = warp_sum(p_in);
        const double lr = (static_cast<double>(t.m) - static_cast<double>(t.ref)) * cd * ln2 + __shfl_sync(0xffffffffu, v, 2) - lz;
        l += q_rest * (__shfl_sync(0xffffffffu, v, 1) - (t.Z == 0.f || (t.R == 0.f && t.Z == t.Z) ? -INFINITY : p_in < 0.5 ? log(1.0 - p_in) : lr));
    }
    return l;
}

// A slice of a row: its first column sits `shift` elements behind a 16-byte boundary, and vector j holds the columns
// v0 - shift + j * E on; only the first and the last may reach past the slice, and are read and written by element.
template <typename T>
struct Slice {
    const T* base;           // the 16-byte boundary
    int shift, end, nv;      // elements [shift, end) from base belong to the slice
    __device__ __forceinline__ Slice(const T* first, int n) {
        constexpr int E = DsType<T>::E;
        shift = static_cast<int>((reinterpret_cast<uintptr_t>(first) & 15u) / sizeof(T));
        base = first - shift;
        end = shift + n;
        nv = n > 0 ? (end + E - 1) / E : 0;
    }
    __device__ __forceinline__ bool whole(int j) const {
        constexpr int E = DsType<T>::E;
        return j * E >= shift && (j + 1) * E <= end;
    }
    // Columns outside the slice read as minus infinity: they take no part in the maximum or the sum.
    // `again`: they will be read once more, so L2 should keep them.
    __device__ __forceinline__ uint4 load(int j, bool again = false) const {
        constexpr int E = DsType<T>::E;
        if (j < nv && whole(j)) {
            const uint4* at = reinterpret_cast<const uint4*>(base) + j;
            return again ? __ldcg(at) : __ldcs(at);
        }
        float f[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = j * E + e;
            f[e] = j < nv && i >= shift && i < end ? DsType<T>::one(base[i]) : -INFINITY;
        }
        return DsType<T>::pack(f);
    }
};

// An entry as it lies in memory, and what it says: its column (-1: absent) and the teacher's logit.
__device__ __forceinline__ int2 raw_index(const DistillParams& p, size_t at) {
    if (p.index64) return static_cast<const int2*>(p.index)[at];
    return make_int2(static_cast<const int*>(p.index)[at], 0);
}
__device__ __forceinline__ int column_of(const DistillParams& p, int2 raw) {
    const bool in = (!p.index64 || raw.y == 0) && raw.x >= 0 && raw.x < p.V;
    return in ? raw.x : -1;
}
__device__ __forceinline__ uint32_t raw_value(const DistillParams& p, size_t at) {
    if (p.value_type == SLIM_F32) return static_cast<const uint32_t*>(p.value)[at];
    return static_cast<const unsigned short*>(p.value)[at];
}
__device__ __forceinline__ float teacher_logit(const DistillParams& p, uint32_t raw) {
    if (p.value_type == SLIM_F32) return __uint_as_float(raw);
    if (p.value_type == SLIM_F16) return __half2float(__ushort_as_half(static_cast<unsigned short>(raw)));
    return __uint_as_float(raw << 16);
}

// Shared memory of k entries (a multiple of 16 bytes).
__host__ __device__ __forceinline__ int entry_bytes(int k) { return (25 * k + 16 + 15) & ~15; }

template <typename T, bool REST, int MODE>
__global__ void __launch_bounds__(kDsThreads, 2) distill_kernel(const DistillParams p) {
    constexpr int E = DsType<T>::E;
    extern __shared__ __align__(16) unsigned char ds_smem[];
    double* s_q = reinterpret_cast<double*>(ds_smem);                  // [k] teacher's probability
    double* s_lq = s_q + p.k;                                          // [k] its logarithm
    int* s_idx = reinterpret_cast<int*>(s_lq + p.k);                   // [k + 4] column, -1 where the entry is absent
    float* s_s = reinterpret_cast<float*>(s_idx + p.k + 4);            // [k] student's logit
    uint8_t* s_first = reinterpret_cast<uint8_t*>(s_s + p.k);          // [k] no entry before it has this column
    uint32_t* s_mark = reinterpret_cast<uint32_t*>(ds_smem + entry_bytes(p.k));    // REST: bit e of byte j: element e of vector j is listed
    __shared__ float2 s_part[kDsWarps];                                // maximum and sum of every warp's columns
    __shared__ float4 s_set[kDsWarps];                                 // REST: of every warp's entries the largest logit, the sum of exponentials relative to it, the columns
    __shared__ float2 s_slice;                                         // maximum and sum of this slice, for the cluster
    __shared__ double s_row[2];                                         // the teacher's listed mass; whether there is any

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ranks = p.ranks;
    const int row = static_cast<int>(blockIdx.x) / ranks, rank = static_cast<int>(blockIdx.x) - row * ranks;
    const int v0 = min(p.V, rank * p.slice), v1 = min(p.V, v0 + p.slice);
    const T* r_logits = static_cast<const T*>(p.logits) + static_cast<long long>(row) * p.ld;
    const Slice<T> sl(r_logits + v0, v1 - v0);
    pdl_launch_dependents();
    pdl_wait();

    // ---- the entries: columns, the teacher's values, the student's logits at them (wanted last, and fetched meanwhile).  The first 512
    // are asked for before the row, behind which they would wait.
    const size_t entry0 = static_cast<size_t>(row) * p.k;
    int2 own_index = make_int2(-1, -1);
    uint32_t own_value = 0;
    if (tid < p.k) {
        own_index = raw_index(p, entry0 + tid);
        own_value = raw_value(p, entry0 + tid);
    }
    const float lse = REST ? p.lse[row] : 0.f;
    uint4 x[kDsVecs];
#pragma unroll
    for (int u = 0; u < kDsVecs; ++u) x[u] = sl.load(tid + u * kDsThreads, MODE == kDsStep && sl.nv > kDsVecs * kDsThreads);
    float early = 0.f;
    if (tid < p.k) {
        const int i = column_of(p, own_index);
        s_idx[tid] = i;
        s_lq[tid] = static_cast<double>(teacher_logit(p, own_value)) * p.inv_t;
        if (i >= 0) early = DsType<T>::one(r_logits[i]);
    }
#pragma unroll 1
    for (int j = tid + kDsThreads; j < p.k; j += kDsThreads) {
        const int i = column_of(p, raw_index(p, entry0 + j));
        s_idx[j] = i;
        s_lq[j] = static_cast<double>(teacher_logit(p, raw_value(p, entry0 + j))) * p.inv_t;
        s_s[j] = i >= 0 ? DsType<T>::one(r_logits[i]) : 0.f;
    }
    if (tid < 4) s_idx[p.k + tid] = -1;              // the search below reads whole quadruples
    if (REST)
        for (int j = tid; j < p.mark_bytes / 4; j += kDsThreads) s_mark[j] = 0u;
    __syncthreads();
    int twice = 0;                                   // an entry of this thread has the column of one before it
    for (int j = tid; j < p.k; j += kDsThreads) {
        const int i = s_idx[j];
        bool again = false;
        for (int o = 0; o < j; o += 4) {
            const int4 c = *reinterpret_cast<const int4*>(s_idx + o);
            again = again || (c.x == i) || (o + 1 < j && c.y == i) || (o + 2 < j && c.z == i) || (o + 3 < j && c.w == i);
        }
        s_first[j] = i >= 0 && !again;
        twice |= i >= 0 && again;
        if (REST && i >= v0 && i < v1) {
            const int e = i - v0 + sl.shift;
            atomicOr(s_mark + (e / E >> 2), 1u << ((e / E & 3) * 8 + e % E));
        }
    }
    if (warp == kDsWarps - 1) {
        // the teacher's probabilities; a row has something to learn from if an entry is present (and, without the rest, not all of them are minus infinity)
        double top = -INFINITY;
        int any = 0, finite = 0;
        for (int j = lane; j < p.k; j += 32)
            if (s_idx[j] >= 0) { top = fmax(top, s_lq[j]); any = 1; finite |= !(s_lq[j] == -INFINITY); }
        any = __any_sync(0xffffffffu, any);
        double norm;
        if (REST) norm = lse;
        else {
            any = __any_sync(0xffffffffu, finite);
            top = warp_max(top);
            double sum = 0.0;
            for (int j = lane; j < p.k; j += 32)
                if (s_idx[j] >= 0) sum += exp_log(s_lq[j] - top);
            norm = top + log(warp_sum(sum));
        }
        double q_sum = 0.0;
        for (int j = lane; j < p.k; j += 32) {
            const double lq = s_lq[j] - norm;
            const double q = s_idx[j] >= 0 && any ? exp_log(lq) : 0.0;
            s_lq[j] = lq;
            s_q[j] = q;
            q_sum += q;
        }
        q_sum = warp_sum(q_sum);
        if (lane == 0) { s_row[0] = q_sum; s_row[1] = any; }
    }
    twice = __syncthreads_or(twice);

    // A warp's entries' part of the set's columns: every column once, by its first entry.
    auto set_part = [&] {
        float top = -INFINITY, z = 0.f;
        int columns = 0;
        if (tid < p.k && s_first[tid]) { top = early; ++columns; }
#pragma unroll 1
        for (int j = tid + kDsThreads; j < p.k; j += kDsThreads)
            if (s_first[j]) { top = fmaxf(top, s_s[j]); ++columns; }
        top = redux_max(top);
        const float ref = top == -INFINITY ? 0.f : top;
        if (tid < p.k && s_first[tid]) z = ex2((early - ref) * p.c);
#pragma unroll 1
        for (int j = tid + kDsThreads; j < p.k; j += kDsThreads)
            if (s_first[j]) z += ex2((s_s[j] - ref) * p.c);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        columns = static_cast<int>(__reduce_add_sync(0xffffffffu, columns));
        if (lane == 0) s_set[warp] = make_float4(top, z, __int_as_float(columns), 0.f);
    };

    // ---- the row's maximum and sum of exponentials, of the columns outside the set with REST
    float m;
    double R;                                        // sum over the columns (outside the set) of 2^((s - m) c)
    const uint8_t* mark = reinterpret_cast<const uint8_t*>(s_mark);
    const uint64_t c2 = pair2(p.c, p.c);
    if (MODE != kDsGrad) {
        float tm = -INFINITY, ts = 0.f;
        // Half of the vectors at a time; where the row has more, theirs are asked for as soon as these are done with.
        constexpr int HALF = kDsVecs / 2;
        for (int j0 = 0; j0 < sl.nv; j0 += kDsVecs * kDsThreads) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint4* xh = x + HALF * h;
                if (REST) {                            // the listed columns take no part; their gradient is written apart
                    uint32_t b[HALF], some = 0;
#pragma unroll
                    for (int u = 0; u < HALF; ++u) {
                        const int j = j0 + tid + (HALF * h + u) * kDsThreads;
                        b[u] = j < sl.nv ? mark[j] : 0u;
                        some |= b[u];
                    }
                    if (some != 0) {
#pragma unroll
                        for (int u = 0; u < HALF; ++u) DsType<T>::hide(xh[u], b[u]);
                    }
                }
                const float cm = vec_max<HALF>(xh, static_cast<const T*>(nullptr));
                if (cm > tm) { ts *= tm == -INFINITY ? 0.f : ex2((tm - cm) * p.c); tm = cm; }
                const float neg = tm == -INFINITY ? 0.f : -tm;
                const uint64_t neg2 = pair2(neg, neg);
                uint64_t acc = pair2(ts, 0.f);
#pragma unroll
                for (int u = 0; u < HALF; ++u) {
                    forget(xh[u]);
                    const int j = j0 + tid + (HALF * h + u) * kDsThreads;
                    if (j < sl.nv) {
                        float f[E];
                        DsType<T>::unpack(xh[u], f);
#pragma unroll
                        for (int e = 0; e < E; e += 2) {
                            float a, b;
                            unpair2(mul2(add2(pair2(f[e], f[e + 1]), neg2), c2), a, b);
                            acc = add2(acc, pair2(ex2(a), ex2(b)));
                        }
                    }
                }
                float a, b;
                unpair2(acc, a, b);
                ts = a + b;
                if (j0 + kDsVecs * kDsThreads < sl.nv) {
#pragma unroll
                    for (int u = 0; u < HALF; ++u) xh[u] = sl.load(j0 + tid + (kDsVecs + HALF * h + u) * kDsThreads, MODE == kDsStep);
                }
            }
        }
        // a warp's, then the slice's, then the row's
        float wm = tm;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) wm = fmaxf(wm, __shfl_xor_sync(0xffffffffu, wm, o));
        float ws = tm == -INFINITY ? ts : ts * ex2((tm - wm) * p.c);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
        if (lane == 0) s_part[warp] = make_float2(wm, ws);
        if (tid < p.k) s_s[tid] = early;
        if (REST) set_part();
        __syncthreads();
        auto join = [&](float2 part, bool in) {
            m = in ? part.x : -INFINITY;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            R = warp_sum(!in ? 0.0 : part.x == -INFINITY ? static_cast<double>(part.y) : static_cast<double>(part.y) * static_cast<double>(ex2((part.x - m) * p.c)));
        };
        join(s_part[lane % kDsWarps], lane < kDsWarps);
        if (ranks > 1) {
            if (tid == 0) s_slice = make_float2(m, static_cast<float>(R));
            cluster_sync_all();
            join(ld_cluster_f32x2(smem_u32(&s_slice), lane % ranks), lane < ranks);
        }
    } else {
        const float4 sv = *reinterpret_cast<const float4*>(p.saved + 4 * static_cast<size_t>(row));
        m = sv.x;
        R = REST ? sv.z : sv.y;
        if (tid < p.k) s_s[tid] = early;
        if (REST) set_part();
        __syncthreads();
        if (ranks > 1) cluster_sync_all();           // grad may be logits: every CTA of the row has its entries' logits
    }

    // ---- what the row comes to, by every warp for itself
    const double q_sum = s_row[0];
    const bool any = s_row[1] != 0.0;
    double q_rest = 0.0;
    float z = 0.f, top = -INFINITY;
    if (REST) {
        // the warps' parts of the set
        const float4 part = s_set[lane % kDsWarps];
        top = redux_max(part.x);
        z = part.x == -INFINITY ? part.y : part.y * ex2((part.x - top) * p.c);
#pragma unroll
        for (int o = kDsWarps / 2; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        const int columns = static_cast<int>(__reduce_add_sync(0xffffffffu, lane < kDsWarps ? __float_as_int(part.z) : 0));
        if (columns < p.V) q_rest = rest_mass(q_sum, lse);
    }
    const double mass = q_sum + q_rest;
    const RowTerms t = row_terms<REST>(p.c, m, static_cast<float>(R), top, z, static_cast<float>(q_sum), static_cast<float>(q_rest), static_cast<float>(mass));
    // loss, in 64 bits, by the warp that is given it (below, beside the gradient)
    auto write_loss = [&] {
        const double l = row_loss<REST>(t, q_rest, p.k, p.c, s_q, s_lq, s_idx, s_s, s_first, lane);
        if (lane == 0) {
            p.loss[row] = any ? static_cast<float>(l) : 0.f;
            if (MODE == kDsLoss && p.saved != nullptr)
                *reinterpret_cast<float4*>(p.saved + 4 * static_cast<size_t>(row)) = make_float4(m, t.Z, t.R, 0.f);
        }
    };
    if (MODE == kDsLoss) {
        if (rank == 0 && warp == 0) write_loss();
        if (ranks > 1) cluster_sync_all();           // the others may still read this CTA's slice statistics
        return;
    }

    // ---- the gradient: one factor for the whole row, then the listed columns
    const double d = static_cast<double>(p.dloss[row]) * p.inv_t;
    const float factor = any ? t.factor * static_cast<float>(d) : 0.f;
    T* r_grad = static_cast<T*>(p.grad) + static_cast<long long>(row) * p.ldg;
    T* g_base = r_grad + v0 - sl.shift;
    const bool vectors = (reinterpret_cast<uintptr_t>(g_base) & 15u) == 0;
    const uint64_t neg2 = pair2(-t.out, -t.out), factor2 = pair2(factor, factor);
    for (int j0 = 0; j0 < sl.nv; j0 += kDsVecs * kDsThreads) {
        if (MODE == kDsStep && sl.nv > kDsVecs * kDsThreads) {          // more than the registers hold: read again
#pragma unroll
            for (int u = 0; u < kDsVecs; ++u) x[u] = sl.load(j0 + tid + u * kDsThreads);
        }
        if (MODE == kDsGrad && j0 > 0) {
#pragma unroll
            for (int u = 0; u < kDsVecs; ++u) x[u] = sl.load(j0 + tid + u * kDsThreads);
        }
#pragma unroll
        for (int u = 0; u < kDsVecs; ++u) {
            forget(x[u]);
            const int j = j0 + tid + u * kDsThreads;
            if (j < sl.nv) {
                float f[E];
                DsType<T>::unpack(x[u], f);
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    float a, b;
                    unpair2(mul2(add2(pair2(f[e], f[e + 1]), neg2), c2), a, b);
                    unpair2(mul2(pair2(ex2(a), ex2(b)), factor2), f[e], f[e + 1]);
                }
                if (!any) {
#pragma unroll
                    for (int e = 0; e < E; ++e) f[e] = 0.f;
                }
                if (vectors && sl.whole(j)) __stcs(reinterpret_cast<uint4*>(g_base) + j, DsType<T>::pack(f));
                else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int i = j * E + e;
                        if (i >= sl.shift && i < sl.end) g_base[i] = DsType<T>::round(f[e]);
                    }
                }
            }
        }
    }
    __syncthreads();                                 // the listed columns are written over
    if (any) {
        for (int j = tid; j < p.k; j += kDsThreads) {
            const int i = s_idx[j];
            if (!s_first[j] || i < v0 || i >= v1) continue;
            double q = s_q[j];
            if (twice)
                for (int o = j + 1; o < p.k; ++o) q += s_idx[o] == i ? s_q[o] : 0.0;
            r_grad[i] = DsType<T>::round(static_cast<float>((static_cast<double>(ex2((s_s[j] - t.ref) * p.c) * t.inv_z) * mass - q) * d));
        }
    }
    if (MODE == kDsStep) {
        if (rank == 0 && warp == kDsWarps - 1) write_loss();
        if (ranks > 1) cluster_sync_all();
    }
}

// ------------------------------------------------------------------------------------------ the one pass over many rows
// With more rows than CTAs at once, a CTA (or cluster) takes row after row, and what a row waits for is done for later ones meanwhile, by two warps beside
// the sixteen that take the rows in turn: they have a row brought into shared memory (one bulk copy), read its entries and the logits at them two
// rows ahead, work out the teacher's probabilities, and when the sixteen have the row's statistics compute its loss beside their
// gradient.  (One such warp was what all waited for: it runs some 700 instructions per row, alone in its code and at an instruction in 20 cycles.)
// The sixteen take the row from shared memory into registers at once, which frees the buffer for the next.  4096 x 32000 bf16 took 173 us with
// a CTA per row (of 22000 cycles 9000 went until the entries were there and 4000 into the row's own terms), two per SM.
// Statistics meet in a cluster by asynchronous stores that count on the receiver's barrier.  Every wait is bounded; rows left
// undone by one that gives up have NaN for a loss.
constexpr int kDsRowsThreads = kDsThreads + 64;

struct RowTeacher {          // what its entries come to
    double mass, q_rest, d;  // the teacher's whole mass, that outside the set; the row's weight over the temperature
    float q_sum;             // the teacher's listed mass
    float top, z;            // the student's largest logit of the set, its sum of 2^((s - top) c) over the set's columns
    int any, twice;          // something to learn from; a column in two entries
};
constexpr int kDsFilterBytes = 8192;     // a bit per column modulo 65536: has it been seen in this row?
constexpr int kDsEntryBufs = 4;

template <typename T>
struct RowsSmem {            // byte offsets
    int row, filter, entries, entry_stride, total;
    __host__ __device__ RowsSmem(int slice, int k) {
        row = 0;
        filter = (slice / DsType<T>::E + 1) * 16;
        entries = filter + 2 * kDsFilterBytes;         // one for each of the two warps
        entry_stride = entry_bytes(k);
        total = entries + kDsEntryBufs * entry_stride;
    }
};

__device__ __forceinline__ void st_async_f32x2(uint32_t cluster_addr, float2 v, uint32_t cluster_bar) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
                 ::"r"(cluster_addr), "f"(v.x), "f"(v.y), "r"(cluster_bar) : "memory");
}
__device__ __forceinline__ uint32_t map_cluster(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

template <typename T, bool REST, int MODE>
__global__ void __launch_bounds__(kDsRowsThreads, 2) distill_rows_kernel(const DistillParams p) {
    constexpr int E = DsType<T>::E;
    extern __shared__ __align__(16) unsigned char ds_smem[];
    const RowsSmem<T> lay(p.slice, p.k);
    __shared__ __align__(8) uint64_t s_bar[2 + 3 * kDsEntryBufs + 2];
    __shared__ float2 s_part[2][kDsWarps];
    __shared__ float2 s_slice[2][kDsMaxCluster];
    __shared__ RowTeacher s_teacher[kDsEntryBufs];
    __shared__ RowTerms s_terms[kDsEntryBufs];
    __shared__ int s_abort;
    volatile int* abort = &s_abort;
    const uint32_t bar0 = smem_u32(s_bar);
    const uint32_t row_full = bar0, row_empty = bar0 + 8;
    auto ent_full = [&](int b) { return bar0 + 16u + 8u * b; };
    auto ent_empty = [&](int b) { return bar0 + 16u + 8u * (kDsEntryBufs + b); };
    auto terms_full = [&](int b) { return bar0 + 16u + 8u * (2 * kDsEntryBufs + b); };
    auto slice_full = [&](int b) { return bar0 + 16u + 8u * (3 * kDsEntryBufs + b); };

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ranks = p.ranks, rank = ranks > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int first = static_cast<int>(blockIdx.x) / ranks, stride = static_cast<int>(gridDim.x) / ranks;
    const int v0 = min(p.V, rank * p.slice), v1 = min(p.V, v0 + p.slice);
    if (tid == 0) {
        s_abort = 0;
        sb::init(row_full, 1);
        sb::init(row_empty, kDsWarps);
        for (int b = 0; b < kDsEntryBufs; ++b) {
            sb::init(ent_full(b), 1);
            sb::init(ent_empty(b), kDsWarps);
            sb::init(terms_full(b), 1);
        }
        for (int b = 0; b < 2; ++b) sb::init(slice_full(b), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < (lay.entries - lay.filter) / 16; i += kDsRowsThreads)    // the filters are zero between rows
        reinterpret_cast<uint4*>(ds_smem + lay.filter)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    if (ranks > 1) cluster_sync_all();                 // the others' barriers exist
    pdl_launch_dependents();
    pdl_wait();
    const T* logits = static_cast<const T*>(p.logits);
    auto slice_of = [&](int row) { return Slice<T>(logits + static_cast<long long>(row) * p.ld + v0, v1 - v0); };

    if (warp >= kDsWarps) {
        // ------------------------------------------------------------------ the two beside them: even rows and odd rows of this CTA
        // The columns and values of a row's first 64 entries, its log-sum-exp and its weight are on their way while the row before is prepared, as
        // they lie in memory: a load takes some 5000 cycles beside the rows' traffic, and a conversion here would wait for it.
        const int turn = warp - kDsWarps;
        constexpr int AHEAD = 2;
        int2 f_idx[AHEAD];
        uint32_t f_val[AHEAD];
        float f_lse = 0.f, f_weight = 0.f;
        uint32_t* filter = reinterpret_cast<uint32_t*>(ds_smem + lay.filter + turn * kDsFilterBytes);
        auto fetch = [&](int row) {
            if (row >= p.M) return;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (32 * u >= p.k) break;
                const int j = lane + 32 * u;
                const size_t at = static_cast<size_t>(row) * p.k + j;
                if (j < p.k) {
                    f_idx[u] = raw_index(p, at);
                    f_val[u] = raw_value(p, at);
                }
            }
            if (REST) f_lse = p.lse[row];
            if (MODE == kDsStep) f_weight = p.dloss[row];
        };
        auto entries = [&](int row, int n) {           // of the n-th row of this CTA; its buffer is free, its first entries fetched
            const int b = n % kDsEntryBufs;
            unsigned char* e0 = ds_smem + lay.entries + b * lay.entry_stride;
            double* s_q = reinterpret_cast<double*>(e0);
            double* s_lq = s_q + p.k;
            int* s_idx = reinterpret_cast<int*>(s_lq + p.k);
            float* s_s = reinterpret_cast<float*>(s_idx + p.k + 4);
            uint8_t* s_first = reinterpret_cast<uint8_t*>(s_s + p.k);
            const T* r_logits = logits + static_cast<long long>(row) * p.ld;
            // the first 64 entries in registers, two of a lane side by side; the others after them
            T g[AHEAD];
            int idx[AHEAD];
            double u_t[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                idx[u] = lane + 32 * u < p.k ? column_of(p, f_idx[u]) : -1;
                if (idx[u] >= 0) g[u] = r_logits[idx[u]];
            }
            int seen = 0, columns = 0;
            auto enter = [&](int j, int i) {
                s_idx[j] = i;
                s_first[j] = i >= 0;
                if (i >= 0) {
                    ++columns;
                    seen |= atomicOr(filter + (i >> 5 & (kDsFilterBytes / 4 - 1)), 1u << (i & 31)) >> (i & 31) & 1u;
                }
            };
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (lane + 32 * u < p.k) enter(lane + 32 * u, idx[u]);
                u_t[u] = idx[u] >= 0 ? static_cast<double>(teacher_logit(p, f_val[u])) * p.inv_t : -INFINITY;
            }
            const float lse = f_lse, weight = f_weight;
            fetch(row + 2 * stride);
            double top = fmax(u_t[0], u_t[1]);
            bool bad = u_t[0] != u_t[0] || u_t[1] != u_t[1];
#pragma unroll 1
            for (int j = lane + 32 * AHEAD; j < p.k; j += 32) {
                const size_t at = static_cast<size_t>(row) * p.k + j;
                const int i = column_of(p, raw_index(p, at));
                const double u = i >= 0 ? static_cast<double>(teacher_logit(p, raw_value(p, at))) * p.inv_t : -INFINITY;
                enter(j, i);
                s_s[j] = i >= 0 ? DsType<T>::one(r_logits[i]) : 0.f;
                s_lq[j] = u;
                top = fmax(top, u);
                bad = bad || u != u;
            }
            __syncwarp();
            columns = static_cast<int>(__reduce_add_sync(0xffffffffu, columns));
            int any = columns, twice = 0;
            if (__any_sync(0xffffffffu, seen)) {       // perhaps a column twice (certainly so up to 65536 columns): which entry is its column's first
                for (int j = lane; j < p.k; j += 32) {
                    const int i = s_idx[j];
                    bool again = false;
                    for (int o = 0; o < j; ++o) again = again || s_idx[o] == i;
                    s_first[j] = i >= 0 && !again;
                    twice += i >= 0 && again;
                }
                twice = static_cast<int>(__reduce_add_sync(0xffffffffu, twice));
                columns -= twice;
            }
#pragma unroll 2
            for (int j = lane; j < p.k; j += 32) {     // the filter is zero again
                const int i = s_idx[j];
                if (i >= 0) filter[i >> 5 & (kDsFilterBytes / 4 - 1)] = 0u;
            }
            // the teacher's probabilities
            double norm = lse;
            if (!REST) {
                any = __any_sync(0xffffffffu, top > -INFINITY || bad);       // not all of them minus infinity
                top = warp_max(top);
                if (top == -INFINITY) top = 0.0;
                double sum = exp_log(u_t[0] - top) + exp_log(u_t[1] - top);
#pragma unroll 1
                for (int j = lane + 32 * AHEAD; j < p.k; j += 32) sum += exp_log(s_lq[j] - top);
                norm = top + log(warp_sum(sum));
            }
            double q_sum = 0.0;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int j = lane + 32 * u;
                const double lq = u_t[u] - norm, q = idx[u] >= 0 && any ? exp_log(lq) : 0.0;
                if (j < p.k) { s_lq[j] = lq; s_q[j] = q; }
                q_sum += q;
            }
#pragma unroll 1
            for (int j = lane + 32 * AHEAD; j < p.k; j += 32) {
                const double lq = s_lq[j] - norm, q = s_idx[j] >= 0 && any ? exp_log(lq) : 0.0;
                s_lq[j] = lq;
                s_q[j] = q;
                q_sum += q;
            }
            q_sum = warp_sum(q_sum);
            // the student's logits
            float sv[AHEAD], s_top = -INFINITY, z = 0.f;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                sv[u] = idx[u] >= 0 ? DsType<T>::one(g[u]) : -INFINITY;
                if (lane + 32 * u < p.k) s_s[lane + 32 * u] = sv[u];
            }
            if (REST) {
                s_top = fmaxf(sv[0], sv[1]);
#pragma unroll 1
                for (int j = lane + 32 * AHEAD; j < p.k; j += 32)
                    if (s_idx[j] >= 0) s_top = fmaxf(s_top, s_s[j]);
                s_top = redux_max(s_top);
                const float r = s_top == -INFINITY ? 0.f : s_top;
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
                    if (idx[u] >= 0 && (twice == 0 || s_first[lane + 32 * u])) z += ex2((sv[u] - r) * p.c);
#pragma unroll 1
                for (int j = lane + 32 * AHEAD; j < p.k; j += 32)
                    if (s_first[j]) z += ex2((s_s[j] - r) * p.c);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
            }
            if (lane == 0) {
                RowTeacher t;
                t.q_rest = REST && columns < p.V ? rest_mass(q_sum, lse) : 0.0;
                t.mass = q_sum + t.q_rest;
                t.d = static_cast<double>(weight) * p.inv_t;
                t.q_sum = static_cast<float>(q_sum);
                t.top = s_top; t.z = z; t.any = any; t.twice = twice;
                s_teacher[b] = t;
            }
            __syncwarp();
            if (lane == 0) sb::arrive(ent_full(b));
        };
        // The slice into shared memory, whose buffer is free: the whole vectors by a bulk copy, the ends as they are, minus infinity beside them.
        auto bring = [&](int row) {
            const Slice<T> sl = slice_of(row);
            const int j = lane < E ? 0 : sl.nv - 1, i = j * E + lane % E;
            if (lane < 2 * E && sl.nv > 0 && !sl.whole(j))
                reinterpret_cast<T*>(ds_smem + lay.row)[i] = i >= sl.shift && i < sl.end ? sl.base[i] : DsType<T>::round(-INFINITY);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the buffer was read, and its ends are written, by ordinary accesses
            __syncwarp();
            const int from = sl.shift > 0 ? 1 : 0, to = sl.end / E;
            const uint32_t bytes = to > from ? 16u * static_cast<uint32_t>(to - from) : 0u;
            if (lane == 0) {
                sb::expect_tx(row_full, bytes);
                if (bytes > 0) sb::bulk_g2s(smem_u32(ds_smem) + lay.row + 16u * from, reinterpret_cast<const uint4*>(sl.base) + from, bytes, row_full);
            }
            __syncwarp();
        };
        int n = turn;
        int row = first + turn * stride;
        if (row < p.M) {
            if (n == 0) bring(row);
            fetch(row);
            entries(row, n);
        }
        for (; row < p.M; row += 2 * stride, n += 2) {
            const int b = n % kDsEntryBufs;
            bool ok = true;
            if (n > 0) {                               // the buffer is free when the sixteen have taken the row before
                ok = __all_sync(0xffffffffu, sb::wait(row_empty, (n - 1) & 1u, abort));
                if (ok) bring(row);
            }
            if (ok && row + 2 * stride < p.M) {
                if (n >= 2) ok = __all_sync(0xffffffffu, sb::wait(ent_empty((n + 2) % kDsEntryBufs), ((n - 2) / kDsEntryBufs) & 1u, abort));
                if (ok) entries(row + 2 * stride, n + 2);
            }
            ok = ok && __all_sync(0xffffffffu, sb::wait(terms_full(b), (n / kDsEntryBufs) & 1u, abort));
            if (!ok) {
                for (int r = row; r < p.M && rank == 0 && lane == 0; r += 2 * stride) p.loss[r] = NAN;
                break;
            }
            if (rank == 0) {
                const RowTerms t = s_terms[b];
                const RowTeacher te = s_teacher[b];
                const double* s_q = reinterpret_cast<const double*>(ds_smem + lay.entries + b * lay.entry_stride);
                const double* s_lq = s_q + p.k;
                const int* s_idx = reinterpret_cast<const int*>(s_lq + p.k);
                const float* s_s = reinterpret_cast<const float*>(s_idx + p.k + 4);
                const uint8_t* s_first = reinterpret_cast<const uint8_t*>(s_s + p.k);
                const double l = row_loss<REST>(t, te.q_rest, p.k, p.c, s_q, s_lq, s_idx, s_s, s_first, lane);
                if (lane == 0) {
                    p.loss[row] = te.any ? static_cast<float>(l) : 0.f;
                    if (MODE == kDsLoss && p.saved != nullptr) *reinterpret_cast<float4*>(p.saved + 4 * static_cast<size_t>(row)) = make_float4(t.m, t.Z, t.R, 0.f);
                }
            }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------------ the sixteen
        const uint64_t c2 = pair2(p.c, p.c);
        auto meet = [] { asm volatile("bar.sync 1, %0;" ::"n"(kDsThreads) : "memory"); };
        int n = 0;
        for (int row = first; row < p.M; row += stride, ++n) {
            const int b = n & 1, eb = n % kDsEntryBufs;
            const uint32_t ph = (n >> 1) & 1u, eph = (n / kDsEntryBufs) & 1u;
            const unsigned char* e0 = ds_smem + lay.entries + eb * lay.entry_stride;
            const double* s_q = reinterpret_cast<const double*>(e0);
            const int* s_idx = reinterpret_cast<const int*>(s_q + 2 * p.k);
            const float* s_s = reinterpret_cast<const float*>(s_idx + p.k + 4);
            const uint8_t* s_first = reinterpret_cast<const uint8_t*>(s_s + p.k);
            const Slice<T> sl = slice_of(row);
            // a warp that gives up says so to the others at the next meeting; all leave there
            bool ok = sb::wait(ent_full(eb), eph, abort);
            ok = sb::wait(row_full, n & 1u, abort) && ok;
            __syncwarp();
            if (REST) {
                // The listed columns take no part in the statistics (their gradient is written apart): each warp makes minus infinity of those in its own vectors.
#pragma unroll 1
                for (int j = lane; j < p.k; j += 32) {
                    const int i = s_idx[j], at = i - v0 + sl.shift;
                    if (i >= v0 && i < v1 && (at / E / 32) % kDsWarps == warp) reinterpret_cast<T*>(ds_smem + lay.row)[at] = DsType<T>::round(-INFINITY);
                }
                __syncwarp();
            }
            const uint4* buf = reinterpret_cast<const uint4*>(ds_smem + lay.row) + tid;
            const float ninf = -INFINITY;
            uint4 x[kDsVecs];
#pragma unroll
            for (int u = 0; u < kDsVecs; ++u) {
                if (tid + u * kDsThreads < sl.nv) x[u] = buf[u * kDsThreads];
                else {
                    float f[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) f[e] = ninf;
                    x[u] = DsType<T>::pack(f);
                }
            }
            __syncwarp();
            if (lane == 0) sb::arrive(row_empty);

            // ---- maximum and sum of exponentials (outside the set with REST) of a warp, the slice, the row
            const float tm = redux_max(vec_max<kDsVecs>(x, static_cast<const T*>(nullptr)));
            float ws;
            {
                const float neg = tm == -INFINITY ? 0.f : -tm;
                const uint64_t neg2 = pair2(neg, neg);
                uint64_t acc = pair2(0.f, 0.f);
#pragma unroll
                for (int u = 0; u < kDsVecs; ++u) {
                    forget(x[u]);
                    const int j = tid + u * kDsThreads;
                    if (j < sl.nv) {
                        float f[E];
                        DsType<T>::unpack(x[u], f);
#pragma unroll
                        for (int e = 0; e < E; e += 2) {
                            float v, w;
                            unpair2(mul2(add2(pair2(f[e], f[e + 1]), neg2), c2), v, w);
                            acc = add2(acc, pair2(ex2(v), ex2(w)));
                        }
                    }
                }
                float v, w;
                unpair2(acc, v, w);
                ws = v + w;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
            if (lane == 0) s_part[b][warp] = make_float2(tm, ws);
            meet();
            float m, R;
            auto join = [&](float2 part, bool in) {    // sixteen at most, in the low and the high half of the warp alike
                m = redux_max(in ? part.x : -INFINITY);
                R = !in ? 0.f : part.x == -INFINITY ? part.y : part.y * ex2((part.x - m) * p.c);
#pragma unroll
                for (int o = kDsWarps / 2; o > 0; o >>= 1) R += __shfl_xor_sync(0xffffffffu, R, o);
            };
            join(s_part[b][lane % kDsWarps], true);
            if (ranks > 1) {
                if (tid == 0) sb::expect_tx(slice_full(b), 8u * ranks);
                if (tid < ranks)
                    st_async_f32x2(map_cluster(smem_u32(&s_slice[b][rank]), tid), make_float2(m, R), map_cluster(slice_full(b), tid));
                ok = sb::wait(slice_full(b), ph, abort) && ok;
                __syncwarp();
                join(s_slice[b][lane % ranks], lane % kDsWarps < ranks);
            }

            // ---- what the row comes to, by every thread for itself
            const RowTeacher te = s_teacher[eb];
            const RowTerms t = row_terms<REST>(p.c, m, R, te.top, te.z, te.q_sum, static_cast<float>(te.q_rest), static_cast<float>(te.mass));
            if (tid == 0) {
                s_terms[eb] = t;
                sb::arrive(terms_full(eb));
            }
            const bool any = te.any != 0;
            const float factor = any ? t.factor * static_cast<float>(te.d) : 0.f;

            // ---- the gradient: one factor for the whole row, then the listed columns
            T* r_grad = MODE == kDsStep ? static_cast<T*>(p.grad) + static_cast<long long>(row) * p.ldg : nullptr;
            if (MODE == kDsStep) {
                T* g_base = r_grad + v0 - sl.shift;
                const bool vectors = (reinterpret_cast<uintptr_t>(g_base) & 15u) == 0;
                const uint64_t neg2 = pair2(-t.out, -t.out), factor2 = pair2(factor, factor);
#pragma unroll
                for (int u = 0; u < kDsVecs; ++u) {
                    forget(x[u]);
                    const int j = tid + u * kDsThreads;
                    if (j < sl.nv) {
                        float f[E];
                        DsType<T>::unpack(x[u], f);
#pragma unroll
                        for (int e = 0; e < E; e += 2) {
                            float v, w;
                            unpair2(mul2(add2(pair2(f[e], f[e + 1]), neg2), c2), v, w);
                            unpair2(mul2(pair2(ex2(v), ex2(w)), factor2), f[e], f[e + 1]);
                        }
                        if (!any) {
#pragma unroll
                            for (int e = 0; e < E; ++e) f[e] = 0.f;
                        }
                        if (vectors && sl.whole(j)) __stcs(reinterpret_cast<uint4*>(g_base) + j, DsType<T>::pack(f));
                        else {
#pragma unroll
                            for (int e = 0; e < E; ++e) {
                                const int i = j * E + e;
                                if (i >= sl.shift && i < sl.end) g_base[i] = DsType<T>::round(f[e]);
                            }
                        }
                    }
                }
            }
            uint32_t gave_up;                          // the listed columns are written over; and who has given up says so
            asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.or.pred p, 1, %2, q;\n selp.u32 %0, 1, 0, p;\n}\n"
                         : "=r"(gave_up) : "r"(ok ? 0u : 1u), "n"(kDsThreads) : "memory");
            if (MODE == kDsStep && any) {
                for (int j = tid; j < p.k; j += kDsThreads) {
                    const int i = s_idx[j];
                    if (!s_first[j] || i < v0 || i >= v1) continue;
                    double q = s_q[j];
                    if (te.twice)
                        for (int o = j + 1; o < p.k; ++o) q += s_idx[o] == i ? s_q[o] : 0.0;
                    r_grad[i] = DsType<T>::round(static_cast<float>((static_cast<double>(ex2((s_s[j] - t.ref) * p.c) * t.inv_z) * te.mass - q) * te.d));
                }
            }
            __syncwarp();
            if (lane == 0) sb::arrive(ent_empty(eb));
            if (gave_up) break;
        }
    }
    // after a wait that gave up a copy may still be on its way to this CTA's shared memory, or the others' statistics
    if (*abort != 0 && tid == kDsThreads) {
        const unsigned long long t0 = sb::timer_ns();
        while (!(sb::try_wait(row_full, 0) && sb::try_wait(row_full, 1)) && sb::timer_ns() - t0 < 1000000ull) { }
    }
    __syncthreads();
    if (ranks > 1) cluster_sync_all();
}

// ------------------------------------------------------------------------------------------ host side
template <typename T, bool REST, int MODE>
static cudaError_t distill_launch_as(const DistillParams& p, int cluster, size_t smem, cudaStream_t s) {
    static std::atomic<bool> attr_set[64];    // zero-initialised; set-up is idempotent, so a race repeats it harmlessly
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = cudaFuncSetAttribute(distill_kernel<T, REST, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, 104 * 1024);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(static_cast<unsigned>(p.M) * cluster, 1, 1);
    cfg.blockDim = dim3(kDsThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(cluster); attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;       // set up beside the kernel ahead, which it waits for
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, distill_kernel<T, REST, MODE>, p);
}
// Clusters of the many-rows kernel that are resident at once.
template <typename T, bool REST, int MODE>
static int rows_resident(int cluster, size_t smem) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    static std::atomic<bool> attr_set[64];    // zero-initialised; set-up is idempotent, so a race repeats it harmlessly
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        if (cudaFuncSetAttribute(distill_rows_kernel<T, REST, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, 110 * 1024) != cudaSuccess) {
            (void)cudaGetLastError();
            return 0;
        }
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    return smem <= 110 * 1024 ? 2 * device_sm_count() / cluster : 0;
}
template <typename T, bool REST, int MODE>
static cudaError_t rows_launch(const DistillParams& p, int cluster, int clusters, size_t smem, cudaStream_t s) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(static_cast<unsigned>(clusters) * cluster, 1, 1);
    cfg.blockDim = dim3(kDsRowsThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(cluster); attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;       // set up beside the kernel ahead, which it waits for
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, distill_rows_kernel<T, REST, MODE>, p);
}
// The many-rows kernel, where a row fits a cluster's registers and there are more rows than clusters at once (1 if not taken).
template <typename T, bool REST, int MODE>
static int rows_try_as(const DistillParams& p, int cluster, cudaStream_t s) {
    if (p.slice / DsType<T>::E + 1 > kDsThreads * kDsVecs) return 1;
    const RowsSmem<T> lay(p.slice, p.k);
    const int clusters = rows_resident<T, REST, MODE>(cluster, static_cast<size_t>(lay.total));
    if (clusters < 1 || p.M <= clusters) return 1;
    SLIM_CUDA_TRY((rows_launch<T, REST, MODE>(p, cluster, clusters, static_cast<size_t>(lay.total), s)));
    return SLIM_OK;
}
template <typename T, int MODE>
static int rows_try_rest(const DistillParams& p, int cluster, cudaStream_t s) {
    return p.lse != nullptr ? rows_try_as<T, true, MODE>(p, cluster, s) : rows_try_as<T, false, MODE>(p, cluster, s);
}
template <int MODE>
static int rows_try(const DistillParams& p, int type, int cluster, cudaStream_t s) {
    switch (type) {
        case SLIM_F32: return rows_try_rest<float, MODE>(p, cluster, s);
        case SLIM_F16: return rows_try_rest<__half, MODE>(p, cluster, s);
        default: return rows_try_rest<__nv_bfloat16, MODE>(p, cluster, s);
    }
}

template <typename T, int MODE>
static cudaError_t distill_launch_rest(const DistillParams& p, int cluster, size_t smem, cudaStream_t s) {
    return p.lse != nullptr ? distill_launch_as<T, true, MODE>(p, cluster, smem, s) : distill_launch_as<T, false, MODE>(p, cluster, smem, s);
}
template <int MODE>
static cudaError_t distill_launch(const DistillParams& p, int type, int cluster, size_t smem, cudaStream_t s) {
    switch (type) {
        case SLIM_F32: return distill_launch_rest<float, MODE>(p, cluster, smem, s);
        case SLIM_F16: return distill_launch_rest<__half, MODE>(p, cluster, smem, s);
        default: return distill_launch_rest<__nv_bfloat16, MODE>(p, cluster, smem, s);
    }
}

static bool known_type(int t) { return t == SLIM_F32 || t == SLIM_F16 || t == SLIM_BF16; }
static bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

static int distill(int mode, const void* logits, int type, long long ld, const void* index, int index_bytes, const void* value, int value_type,
                   const float* lse, double temperature, int M, int V, int k, float* loss, float* saved, const float* dloss, void* grad,
                   long long ldg, void* stream) {
    if (M < 0 || V < 1 || k < 1 || !known_type(type) || !known_type(value_type) || (index_bytes != 4 && index_bytes != 8)) return SLIM_ERR_INVALID_ARG;
    if (!(temperature > 0.0) || !(temperature <= 1e30) || !(temperature >= 1e-30) || ld < V || (mode != kDsLoss && ldg < V)) return SLIM_ERR_INVALID_ARG;
    if (V > SLIM_DISTILL_MAX_V || k > SLIM_DISTILL_MAX_K || M > (1 << 27)) return SLIM_ERR_UNSUPPORTED;
    if (M == 0) return SLIM_OK;
    if (logits == nullptr || index == nullptr || value == nullptr) return SLIM_ERR_INVALID_ARG;
    if (mode != kDsGrad && loss == nullptr) return SLIM_ERR_INVALID_ARG;
    if (mode != kDsLoss && (dloss == nullptr || grad == nullptr)) return SLIM_ERR_INVALID_ARG;
    if (mode == kDsGrad && saved == nullptr) return SLIM_ERR_INVALID_ARG;
    const int es = type == SLIM_F32 ? 4 : 2;
    if (!aligned_to(logits, es) || !aligned_to(grad, es) || !aligned_to(index, index_bytes) || !aligned_to(value, value_type == SLIM_F32 ? 4 : 2) ||
        !aligned_to(lse, 4) || !aligned_to(dloss, 4) || !aligned_to(loss, 4) || !aligned16(saved))
        return SLIM_ERR_ALIGNMENT;
    if (mode != kDsLoss && !(grad == logits && (ldg == ld || M == 1)) &&
        rows_share(logits, ld * es, static_cast<long long>(V) * es, grad, ldg * es, static_cast<long long>(V) * es, M))
        return SLIM_ERR_INVALID_ARG;
    const int E = 16 / es, held = kDsThreads * kDsVecs;            // vectors that a CTA's registers hold
    DistillParams p;
    memset(&p, 0, sizeof p);
    p.logits = logits; p.index = index; p.value = value; p.lse = lse; p.dloss = dloss; p.loss = loss; p.saved = saved; p.grad = grad;
    p.ld = ld; p.ldg = ldg;
    p.c = static_cast<float>(1.44269504088896340736 / temperature);
    p.inv_t = 1.0 / temperature;
    p.M = M; p.V = V; p.k = k;
    p.index64 = index_bytes == 8;
    p.value_type = value_type;
    auto cut = [&](int cluster) {
        p.ranks = cluster;
        p.slice = ((V + cluster - 1) / cluster + E - 1) / E * E;
        p.mark_bytes = lse != nullptr ? (p.slice / E + 1 + 3) / 4 * 4 : 0;
    };
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int vecs = V / E + 2;
    // Many rows that one CTA's registers hold, or for the step two CTAs': the kernel that takes row after row.  (us, that one / a CTA per
    // row, with the rest: step of 4096 x 32000 bf16 125 / 178, of 2000 x 40000 by two 99 / 140; loss of 4096 x 32000 70 / 117, of 4096 x 8000 51 / 103.  By three and
    // more the CTAs of a row wait for each other longer than the second reading, from L2, takes: 1024 x 65536 128 / 81, 512 x 152064 121 / 89, 777 x 50257 fp32 95 / 74.)
    // Both CTAs of a pair prepare all entries, which is what the row waits for when there are many: 2000 x 32000 fp32 with 128, 200 and 310 113 / 132, 149 / 145, 196 / 165,
    // 2000 x 60000 bf16 with 256 and 310 170 / 183, 200 / 196.
    if (mode != kDsGrad && vecs <= (mode == kDsStep ? 2 : 1) * (held - 1)) {
        cut(vecs <= held - 1 ? 1 : 2);
        const int taken = p.ranks > 1 && k > 40 * E ? 1 : mode == kDsStep ? rows_try<kDsStep>(p, type, p.ranks, s) : rows_try<kDsLoss>(p, type, p.ranks, s);
        if (taken <= 0) return taken;
    }
    // Otherwise the cluster that ends soonest: a CTA has its part of a row to read, and what a row costs besides takes as long as some 6500 vectors.
    int cluster = 1;
    double least = 1e30;
    for (int c = 1; c <= kDsMaxCluster; ++c) {
        const long long waves = (static_cast<long long>(M) * c + 2 * device_sm_count() - 1) / (2 * device_sm_count());
        const double t = static_cast<double>(waves) * (static_cast<double>(vecs) / c + 6500.0);
        if (vecs <= c * 65538 && t < 0.98 * least) { least = t; cluster = c; }       // a byte of marks per vector has to fit
    }
    cut(cluster);
    const size_t smem = static_cast<size_t>(entry_bytes(k)) + p.mark_bytes;
    SLIM_CUDA_TRY(mode == kDsLoss ? distill_launch<kDsLoss>(p, type, cluster, smem, s)
                  : mode == kDsGrad ? distill_launch<kDsGrad>(p, type, cluster, smem, s) : distill_launch<kDsStep>(p, type, cluster, smem, s));
    return SLIM_OK;
}

}  // namespace slim

extern "C" int slim_distill_loss(const void* logits, int type, long long ld, const void* index, int index_bytes, const void* value, int value_type,
                                 const float* teacher_lse, double temperature, int M, int V, int k, float* loss, float* saved, void* stream) {
    return slim::distill(slim::kDsLoss, logits, type, ld, index, index_bytes, value, value_type, teacher_lse, temperature, M, V, k, loss, saved,
                         nullptr, nullptr, 0, stream);
}
extern "C" int slim_distill_grad(const void* logits, int type, long long ld, const void* index, int index_bytes, const void* value, int value_type,
                                 const float* teacher_lse, double temperature, int M, int V, int k, const float* saved, const float* dloss, void* grad,
                                 long long ldg, void* stream) {
    return slim::distill(slim::kDsGrad, logits, type, ld, index, index_bytes, value, value_type, teacher_lse, temperature, M, V, k, nullptr,
                         const_cast<float*>(saved), dloss, grad, ldg, stream);
}
extern "C" int slim_distill_step(const void* logits, int type, long long ld, const void* index, int index_bytes, const void* value, int value_type,
                                 const float* teacher_lse, double temperature, int M, int V, int k, const float* dloss, float* loss, void* grad,
                                 long long ldg, void* stream) {
    return slim::distill(slim::kDsStep, logits, type, ld, index, index_bytes, value, value_type, teacher_lse, temperature, M, V, k, loss, nullptr,
                         dloss, grad, ldg, stream);
}
