// What the kernels that take softmax statistics of logits rows share: rows of float32 or bf16 that start anywhere, read as 16-byte
// vectors; a thread-block cluster per row; maxima that keep a NaN; sums in a fixed order.  Device code, and the launch shape.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "s4c_common.cuh"

namespace s4c {
namespace rows {

constexpr float kLog2E = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;

__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float d;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(x));
    return d;
}
// ln x, x > 0 and finite: x = 2^k f with f in [3/4, 3/2), ln f = 2 artanh t = 2 (t + t^3/3 + t^5/5 + ...) with t = (f - 1) / (f + 1), |t| <= 1/5 (the
// next term is below 2^-28 of the sum).  f - 1 is exact, so that the result keeps its relative accuracy where x is near 1.
__device__ __forceinline__ float ln_series(float x) {
    int k = (int)(__float_as_uint(x) >> 23) - 127;
    float f = __uint_as_float((__float_as_uint(x) & 0x7fffffu) | 0x3f800000u);
    if (f >= 1.5f) f *= 0.5f, ++k;
    const float t = __fdividef(f - 1.0f, f + 1.0f), q = t * t;
    const float p = fmaf(q, fmaf(q, fmaf(q, fmaf(q, fmaf(q, 1.0f / 11, 1.0f / 9), 1.0f / 7), 1.0f / 5), 1.0f / 3), 1.0f);
    return fmaf((float)k, (float)kLn2, 2.0f * t * p);
}
// A row maximum that a softmax can be taken against: not NaN, not +Inf, not -Inf.
__device__ __forceinline__ bool usable(float m) { return m > -INFINITY && m < INFINITY; }

// Two float32 in one 64-bit register: one instruction's issue for two additions or multiplications.
using F2 = uint64_t;
__device__ __forceinline__ F2 f2(float a, float b) {
    F2 d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float lo(F2 v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float hi(F2 v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ F2 exp2_2(F2 y) { return f2(exp2_fast(lo(y)), exp2_fast(hi(y))); }

// ----------------------------------------------------------------------------- 16-byte vectors of a row
// Not through L1 (nothing is read twice there), and not through the read-only path: a gradient may be written over its logits.
__device__ __forceinline__ uint4 load16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// 16 bytes into shared memory, in the background
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int E = 4;
    static constexpr uint32_t kNone = 0xff800000u;  // -inf
    __device__ __forceinline__ static void unpack(const uint4& v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
    }
    __device__ __forceinline__ static uint4 pack(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    template <int N>
    __device__ __forceinline__ static float max(const uint4 (&v)[N]) {
        float m[N];
#pragma unroll
        for (int k = 0; k < N; ++k)
            m[k] = max_nan(max_nan(__uint_as_float(v[k].x), __uint_as_float(v[k].y)), max_nan(__uint_as_float(v[k].z), __uint_as_float(v[k].w)));
#pragma unroll
        for (int k = 1; k < N; ++k) m[0] = max_nan(m[0], m[k]);
        return m[0];
    }
    // the elements in pairs, no lower than `low` (which keeps a NaN)
    __device__ __forceinline__ static void pairs(const uint4& v, uint32_t low, F2 (&x)[2]) {
        const float l = __uint_as_float(low);
        x[0] = f2(max_nan(__uint_as_float(v.x), l), max_nan(__uint_as_float(v.y), l)), x[1] = f2(max_nan(__uint_as_float(v.z), l), max_nan(__uint_as_float(v.w), l));
    }
    __device__ __forceinline__ static uint32_t low(float x) { return __float_as_uint(x); }
    __device__ __forceinline__ static void pairs(const uint4& v, F2 (&x)[2]) {
        x[0] = f2(__uint_as_float(v.x), __uint_as_float(v.y)), x[1] = f2(__uint_as_float(v.z), __uint_as_float(v.w));
    }
    __device__ __forceinline__ static uint4 pack(const F2 (&x)[2]) {
        return make_uint4(__float_as_uint(lo(x[0])), __float_as_uint(hi(x[0])), __float_as_uint(lo(x[1])), __float_as_uint(hi(x[1])));
    }
    __device__ __forceinline__ static float get(const float* p) { return *p; }
    __device__ __forceinline__ static void put(float x, float* p) { *p = x; }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int E = 8;
    static constexpr uint32_t kNone = 0xff80ff80u;  // two of -inf
    __device__ __forceinline__ static void unpack(const uint4& v, float (&x)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    __device__ __forceinline__ static uint32_t two(float lo, float hi) {
        uint32_t d;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
        return d;
    }
    __device__ __forceinline__ static uint4 pack(const float (&x)[8]) {
        return make_uint4(two(x[0], x[1]), two(x[2], x[3]), two(x[4], x[5]), two(x[6], x[7]));
    }
    __device__ __forceinline__ static uint32_t two_max(uint32_t a, uint32_t b) {
        uint32_t d;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    }
    template <int N>
    __device__ __forceinline__ static float max(const uint4 (&v)[N]) {
        uint32_t m[N];
#pragma unroll
        for (int k = 0; k < N; ++k) m[k] = two_max(two_max(v[k].x, v[k].y), two_max(v[k].z, v[k].w));
#pragma unroll
        for (int k = 1; k < N; ++k) m[0] = two_max(m[0], m[k]);
        const uint32_t d = m[0];
        return max_nan(__uint_as_float(d << 16), __uint_as_float(d & 0xffff0000u));
    }
    __device__ __forceinline__ static void pairs(const uint4& v, uint32_t low, F2 (&x)[4]) {
        pairs(make_uint4(two_max(v.x, low), two_max(v.y, low), two_max(v.z, low), two_max(v.w, low)), x);
    }
    __device__ __forceinline__ static void pairs(const uint4& v, F2 (&x)[4]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    // twice the greatest bf16 not above x (x finite, in bf16's range)
    __device__ __forceinline__ static uint32_t low(float x) {
        const uint32_t b = __float_as_uint(x), h = ((b >> 31) ? b + 0xffffu : b) >> 16;
        return h | h << 16;
    }
    __device__ __forceinline__ static uint4 pack(const F2 (&x)[4]) {
        return make_uint4(two(lo(x[0]), hi(x[0])), two(lo(x[1]), hi(x[1])), two(lo(x[2]), hi(x[2])), two(lo(x[3]), hi(x[3])));
    }
    __device__ __forceinline__ static float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    __device__ __forceinline__ static void put(float x, __nv_bfloat16* p) { *p = __float2bfloat16_rn(x); }
};

// A row of V elements at any element's address.  Vector i covers elements i E - lead ... + E - 1, so that vectors are aligned.  All but the
// first and the last one are whole; those two may stick out of the row and are read and written element by element there.
template <typename T>
struct Row {
    T* x;
    int V, lead, n;  // n vectors
    __device__ __forceinline__ Row(T* row, int V_) : x(row), V(V_) {
        constexpr int E = Vec<T>::E;
        lead = (int)(reinterpret_cast<uintptr_t>(row) & 15u) / (int)sizeof(T);
        n = (int)(((long long)V + lead + E - 1) / E);
    }
    __device__ __forceinline__ int first(int i) const { return (int)((unsigned)i * Vec<T>::E - lead); }  // of a vector i < n
    __device__ __forceinline__ const uint4* vectors() const { return reinterpret_cast<const uint4*>(x - lead); }
    // vector i < n, -inf where it is out of the row
    __device__ __forceinline__ uint4 load(int i) const {
        constexpr int E = Vec<T>::E;
        const int e0 = first(i);
        if (e0 >= 0 && e0 <= V - E) return load16(x + e0);
        float f[E];
#pragma unroll
        for (int j = 0; j < E; ++j) f[j] = e0 + j >= 0 && e0 + j < V ? Vec<T>::get(x + e0 + j) : -INFINITY;
        return Vec<T>::pack(f);  // (exact: these are T's values)
    }
};

// A block's share of a row: whole vectors b .. e - 1, and the row's first and last vector where they fall to it.
struct Share {
    int begin, end;  // all of its vectors
    int b, e;
    // `per` vectors for each block: `blocks` of them cover the longest row, wherever it starts
    __device__ __forceinline__ Share(int n, int rank, int per) {
        begin = min(n, rank * per), end = min(n, begin + per);
        b = max(begin, 1), e = min(end, n - 1);
    }
    // the row's first or last vector, if it is this thread's; else -1
    __device__ __forceinline__ int edge(int n, int tid) const {
        return tid == 0 && begin == 0 && end > 0 ? 0 : tid == 1 && end == n && n > 1 && begin < end ? n - 1 : -1;
    }
};
template <typename T>
__device__ __forceinline__ uint4 none() {
    return make_uint4(Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone);
}
// Batch by batch f(i, v): v[k] of N is vector i + k threads, -inf from `e` on; the edges come last, as f(-1, v) with the thread's edge as the
// only vector, from the block's first warp.  `at(i)` gives whole vector i, `edge(i)` one of the row's ends.
template <typename T, int N, typename At, typename Edge, typename F>
__device__ __forceinline__ void batches(const Share& s, int n, int threads, At at, Edge edge, F f) {
    const int tid = threadIdx.x;
    for (int i = s.b + tid; i < s.e; i += N * threads) {
        uint4 v[N];
        if (i + (N - 1) * threads < s.e) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = at(i + k * threads);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                v[k] = none<T>();
                if (i + k * threads < s.e) v[k] = at(i + k * threads);
            }
        }
        f(i, v);
    }
    if (tid < 32 && (s.begin == 0 || s.end == n)) {
        const int i = s.edge(n, tid);
        uint4 v[1] = {none<T>()};
        if (i >= 0) v[0] = edge(i);
        f(-1, v);
    }
}

// ----------------------------------------------------------------------------- clusters
// One cluster of blocks per row, a slice of the row's vectors each.  A block arrives when it has started and waits for the others before
// it writes to a peer's shared memory; they meet once more before what was written is read.  Nothing of a peer is touched behind that.
__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
// the same where nothing that was written has to be seen behind it (a block that says it has started)
__device__ __forceinline__ void cluster_arrive_relaxed() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_address(const void* p, int rank) {
    uint32_t d;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return d;
}
__device__ __forceinline__ void peer_store(uint32_t at, uint64_t v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(v) : "memory"); }
__device__ __forceinline__ void peer_store(uint32_t at, int v) { asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ void peer_store(uint32_t at, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

__device__ __forceinline__ int cluster_rank() {
    uint32_t d;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(d));
    return (int)d;
}
__device__ __forceinline__ int cluster_index() {
    uint32_t d;
    asm("mov.u32 %0, %%clusterid.x;" : "=r"(d));
    return (int)d;
}
// maxima over a warp
__device__ __forceinline__ float warp_max_nan(float v) {
    float d;
    asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(d) : "f"(v));
    return d;
}
__device__ __forceinline__ float warp_max(float v) {
    float d;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(d) : "f"(v));
    return d;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

constexpr int kMaxCluster = 8;
constexpr long long kSMs = 148;  // of a B200
constexpr size_t kMaxRowSmem = 200 * 1024;  // dynamic shared memory of a block at most

// `cluster` blocks for each row, as a cluster where they exchange anything
template <typename Kernel, typename Params>
static s4c_status row_launch(Kernel kernel, const Params& p, long long rows, int cluster, int per, int threads, size_t smem, cudaStream_t stream, bool exchange = true) {
    // (always the same limit: the attribute is the kernel's, and another thread's call of another size may come between this line and the launch)
    if (smem > 32 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxRowSmem) != cudaSuccess) {
        cudaGetLastError();
        return S4C_ERR_CUDA;
    }
    if (rows * cluster > INT_MAX) return S4C_ERR_SHAPE;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = exchange ? cluster : 1, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * cluster), 1, 1), cfg.blockDim = dim3(threads, 1, 1), cfg.dynamicSmemBytes = smem, cfg.stream = stream;
    cfg.attrs = attr, cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kernel, p, cluster, per) != cudaSuccess) {
        cudaGetLastError();
        return S4C_ERR_CUDA;
    }
    return S4C_OK;
}

}  // namespace rows
}  // namespace s4c
