// Shared by the dense operators (alcs_norm.cu, alcs_mx4.cu, alcs_mx4_product.cu): checks of buffers, element types.
#ifndef ALCS_DENSE_H_
#define ALCS_DENSE_H_

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "alcs_internal.h"

namespace alcs {
void set_cuda_error_text(const char* s);

namespace {

#define ALCS_CUDA(call)                                        \
    do {                                                       \
        cudaError_t e_ = (call);                               \
        if (e_ != cudaSuccess) {                               \
            alcs::set_cuda_error_text(cudaGetErrorString(e_)); \
            (void)cudaGetLastError();                          \
            return ALCS_ERR_CUDA;                              \
        }                                                      \
    } while (0)

inline size_t elt_bytes(alcs_dtype dt) { return dt == ALCS_F32 ? 4 : 2; }
inline bool known_type(alcs_dtype dt) { return dt == ALCS_F32 || dt == ALCS_F16 || dt == ALCS_BF16; }
inline long long up_div(long long a, long long b) { return (a + b - 1) / b; }

// A buffer of a call.
struct Buffer {
    const void* p;
    size_t bytes, align;
    bool written;
    bool optional;       // may be null
    unsigned may_be;     // bit i: may start where buffer i does; any other overlap of a written buffer with another is refused
};

// Null, misaligned or overlapping buffers; then memory that is not the current device's.
template <int N>
int check_buffers(const Buffer (&b)[N], int* device)
{
    for (int i = 0; i < N; ++i) {
        if (!b[i].p) {
            if (!b[i].optional && b[i].bytes) return ALCS_ERR_INVALID_ARG;
            continue;
        }
        if ((uintptr_t)b[i].p % b[i].align) return ALCS_ERR_INVALID_ARG;
    }
    for (int i = 0; i < N; ++i)
        for (int j = 0; j < N; ++j) {
            if (i == j || !b[i].written || !b[i].p || !b[j].p || !b[i].bytes || !b[j].bytes) continue;
            if ((b[i].may_be >> j & 1u) && b[i].p == b[j].p) continue;
            if (b[j].written && (b[j].may_be >> i & 1u) && b[i].p == b[j].p) continue;
            const uintptr_t s = (uintptr_t)b[i].p, t = (uintptr_t)b[j].p;
            if (s < t + b[j].bytes && t < s + b[i].bytes) return ALCS_ERR_INVALID_ARG;
        }
    ALCS_CUDA(cudaGetDevice(device));
    for (int i = 0; i < N; ++i) {
        if (!b[i].p || !b[i].bytes) continue;
        cudaPointerAttributes at;
        ALCS_CUDA(cudaPointerGetAttributes(&at, b[i].p));
        if (at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged) return ALCS_ERR_INVALID_ARG;
        if (at.type == cudaMemoryTypeDevice && at.device != *device) return ALCS_ERR_STATE;
    }
    return ALCS_OK;
}

// Eight (16-bit types) or four (fp32) elements of 16 bytes as fp32, and back.
template <typename T> struct Pack;
template <> struct Pack<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void get(const uint4& r, float* v)
    {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 put(const float* v)
    {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
__device__ __forceinline__ unsigned pack2(float lo, float hi, __half) 
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return reinterpret_cast<const unsigned&>(h);
}
__device__ __forceinline__ unsigned pack2(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return reinterpret_cast<const unsigned&>(h);
}
__device__ __forceinline__ void unpack2(unsigned r, float* v, __half)
{
    const float2 f = __half22float2(reinterpret_cast<const __half2&>(r));
    v[0] = f.x; v[1] = f.y;
}
__device__ __forceinline__ void unpack2(unsigned r, float* v, __nv_bfloat16)
{
    v[0] = __uint_as_float(r << 16); v[1] = __uint_as_float(r & 0xffff0000u);
}
template <typename T> struct Pack16 {
    static constexpr int n = 8;
    static __device__ __forceinline__ void get(const uint4& r, float* v)
    {
        unpack2(r.x, v, T()); unpack2(r.y, v + 2, T()); unpack2(r.z, v + 4, T()); unpack2(r.w, v + 6, T());
    }
    static __device__ __forceinline__ uint4 put(const float* v)
    {
        return make_uint4(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()), pack2(v[4], v[5], T()), pack2(v[6], v[7], T()));
    }
};
template <> struct Pack<__half> : Pack16<__half> {};
template <> struct Pack<__nv_bfloat16> : Pack16<__nv_bfloat16> {};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void from_f32(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void from_f32(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// max(v, 0) of packed values, NaN to 0 (of rounded values: the rounding keeps their sign)
__device__ __forceinline__ unsigned positive(unsigned v, __half)
{
    const __half2 z = __hmax2(reinterpret_cast<const __half2&>(v), __float2half2_rn(0.0f));
    return reinterpret_cast<const unsigned&>(z);
}
__device__ __forceinline__ unsigned positive(unsigned v, __nv_bfloat16)
{
    const __nv_bfloat162 z = __hmax2(reinterpret_cast<const __nv_bfloat162&>(v), __float2bfloat162_rn(0.0f));
    return reinterpret_cast<const unsigned&>(z);
}
__device__ __forceinline__ unsigned positive(unsigned v, float) { return __float_as_uint(fmaxf(__uint_as_float(v), 0.0f)); }
template <typename T>
__device__ __forceinline__ uint4 positive(const uint4& v, T t) { return make_uint4(positive(v.x, t), positive(v.y, t), positive(v.z, t), positive(v.w, t)); }

// d = a + b, a - b, a * b, a * b + c on E elements, two per instruction.
#define ALCS_PAIRS(name, op)                                                                                                                            \
    template <int E>                                                                                                                                    \
    __device__ __forceinline__ void name(float (&d)[E], const float (&a)[E], const float (&b)[E])                                                       \
    {                                                                                                                                                   \
        if constexpr (E == 1) asm(op ".f32 %0, %1, %2;" : "=f"(d[0]) : "f"(a[0]), "f"(b[0]));                                                           \
        else                                                                                                                                            \
            _Pragma("unroll") for (int i = 0; i < E; i += 2)                                                                                            \
                asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t" op ".f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"            \
                    : "=f"(d[i]), "=f"(d[i + 1]) : "f"(a[i]), "f"(a[i + 1]), "f"(b[i]), "f"(b[i + 1]));                                                 \
    }
ALCS_PAIRS(add, "add.rn")
ALCS_PAIRS(sub, "sub.rn")
ALCS_PAIRS(mul, "mul.rn")
template <int E>
__device__ __forceinline__ void fma(float (&d)[E], const float (&a)[E], const float (&b)[E], const float (&c)[E])
{
    if constexpr (E == 1) d[0] = fmaf(a[0], b[0], c[0]);
    else
#pragma unroll
        for (int i = 0; i < E; i += 2)
            asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
                : "=f"(d[i]), "=f"(d[i + 1]) : "f"(a[i]), "f"(a[i + 1]), "f"(b[i]), "f"(b[i + 1]), "f"(c[i]), "f"(c[i + 1]));
}
// Programmatic dependent launch: the next kernel on the stream may set up, this one waits for what the one before it wrote.  A kernel thus runs while its
// inputs, parameters too, may still be written: it reads them by ordinary loads behind the wait.  The read-only path wants memory that nobody writes during the kernel.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The two halves of a barrier of the cluster's blocks.  A warp's lanes have to come to an .aligned instruction together, whatever branch they were in before.
__device__ __forceinline__ void cluster_arrive()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait()
{
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <typename... P, typename... A>
cudaError_t launch_pdl(void (*fn)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, const A&... a)
{
    cudaLaunchConfig_t lc = {};
    lc.gridDim = grid;
    lc.blockDim = dim3((unsigned)threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&lc, fn, a...);
}

}  // namespace
}  // namespace alcs

#endif  // ALCS_DENSE_H_
