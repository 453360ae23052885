// Microscaled 4-bit floating point (E2M1 values, one E8M0 scale per 32 of a row): quantisation and its inverse, sm_100a.
//
// Both are bound by memory: 2 (fp32: 4) bytes per value on one side, 17/32 on the other.  Four lanes take a block of 32 values, 8
// each; a warp takes 8 rows x 4 blocks, one block of its 8 rows at a time: it reads 8 runs of 64 (128) bytes and writes 128 contiguous
// bytes, since 8 rows of a block lie together in the storage format.  The largest magnitude goes round the four
// lanes by shuffles; the rounding is the hardware's conversion to E2M1 (to nearest, ties to even, saturating).
#include <algorithm>

#include "alcs_dense.h"

namespace alcs {
namespace {

constexpr int kThreads = 256;

struct Args {
    const void* x;
    void* y;
    unsigned char *data, *scales;
    long long ld;
    int rows, cols, blocks, quads;      // blocks of a row as stored (even), groups of four
    long long units;                    // 8 rows x 4 blocks
};

// Two values as a byte of two codes, the first in the low half.
__device__ __forceinline__ unsigned encode4(const float* v)      // four values, 16 bits
{
    unsigned r;
    asm("{\n\t.reg .b8 a, b, z;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "mov.b32 %0, {a, b, a, b};\n\t}" : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]));
    return r & 0xffffu;
}

// Values of four codes (16 bits).
__device__ __forceinline__ void decode4(unsigned r, float* v)
{
    unsigned lo, hi;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %2;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(r));
    unpack2(lo, v, __half());
    unpack2(hi, v + 2, __half());
}

// A lane's 8 values of a row, from column c on; zeros behind the last column.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int c, int cols, float (&v)[8])
{
    if (VEC) {      // (cols is a multiple of 16 bytes' elements)
#pragma unroll
        for (int i = 0; i < 8; i += Pack<T>::n) {
            uint4 r = make_uint4(0, 0, 0, 0);
            if (c + i < cols) asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(row + c + i));
            Pack<T>::get(r, v + i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? to_f32(row[c + i]) : 0.0f;
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) quantize_kernel(const Args a)
{
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, q = lane & 3;
    const long long warps = (long long)gridDim.x * (kThreads / 32);
#pragma unroll 1
    for (long long u = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); u < a.units; u += warps) {
        const int quad = (int)(u % a.quads), r = (int)(u / a.quads) * 8 + (lane >> 2);
        const bool mine = r < a.rows;
        const T* row = static_cast<const T*>(a.x) + (size_t)r * a.ld;
        float v[4][8];
#pragma unroll
        for (int b = 0; b < 4; ++b) load8<T, VEC>(row, (quad * 4 + b) * 32 + q * 8, mine ? a.cols : 0, v[b]);
        unsigned char* to = a.data + ((size_t)(r >> 7) * a.blocks + quad * 4) * 2048 + (r & 127) * 16 + q * 4;
        unsigned scales = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            unsigned top = 0;      // of magnitudes, as integers: their order is that of the numbers, NaN above infinity
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[b][i]) & 0x7fffffffu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = (int)(top >> 23);             // floor(log2) + 127; 0 for subnormal numbers, whose scale is 2^-127, too
            const bool finite = e < 255;
            const int s = finite ? max(e - 2, 0) : 255;
            const float inv = __uint_as_float((unsigned)(254 - (finite ? s : 127)) << 23);      // 2^(127 - s)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[b][i] = finite ? v[b][i] * inv : 0.0f;
            scales |= (unsigned)s << (8 * b);
            const unsigned code = encode4(v[b]) | encode4(v[b] + 4) << 16;
            if (mine && quad * 4 + b < a.blocks) *reinterpret_cast<unsigned*>(to + b * 2048) = code;
        }
        if (mine && q == 0)
            *reinterpret_cast<unsigned*>(a.scales + ((size_t)(r >> 7) * a.quads + quad) * 512 + (r & 31) * 16 + (r >> 5 & 3) * 4) = scales;
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const Args a)
{
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, q = lane & 3;
    const long long warps = (long long)gridDim.x * (kThreads / 32);
#pragma unroll 1
    for (long long u = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); u < a.units; u += warps) {
        const int quad = (int)(u % a.quads), r = (int)(u / a.quads) * 8 + (lane >> 2);
        if (r >= a.rows) continue;
        const unsigned char* from = a.data + ((size_t)(r >> 7) * a.blocks + quad * 4) * 2048 + (r & 127) * 16 + q * 4;
        const unsigned scales = __ldg(reinterpret_cast<const unsigned*>(a.scales + ((size_t)(r >> 7) * a.quads + quad) * 512 + (r & 31) * 16 + (r >> 5 & 3) * 4));
        unsigned code[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) code[b] = quad * 4 + b < a.blocks ? __ldg(reinterpret_cast<const unsigned*>(from + b * 2048)) : 0u;
        T* row = static_cast<T*>(a.y) + (size_t)r * a.ld;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const unsigned s = scales >> (8 * b) & 255u;
            // 2^(s - 127): a subnormal number for s = 0; 255 is the exponent of NaN
            const float scale = __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7fffffffu : s << 23);
            float v[8];
            decode4(code[b], v);
            decode4(code[b] >> 16, v + 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= scale;
            const int c = (quad * 4 + b) * 32 + q * 8;
            if (VEC) {
#pragma unroll
                for (int i = 0; i < 8; i += Pack<T>::n)
                    if (c + i < a.cols) *reinterpret_cast<uint4*>(row + c + i) = Pack<T>::put(v + i);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < a.cols) from_f32(row + c + i, v[i]);
            }
        }
    }
}

template <typename T>
cudaError_t launch(bool quantize, bool vec, const Args& a, int blocks, cudaStream_t st)
{
    auto* fn = quantize ? (vec ? quantize_kernel<T, true> : quantize_kernel<T, false>) : (vec ? dequantize_kernel<T, true> : dequantize_kernel<T, false>);
    return launch_pdl(fn, dim3((unsigned)blocks), kThreads, 0, 1, st, a);
}

int convert(bool quantize, void* data, void* scales, int rows, int cols, void* m, long long ld, alcs_dtype dt, void* cuda_stream)
{
    size_t db = 0, sb = 0;
    if (!known_type(dt) || ld < cols) return ALCS_ERR_INVALID_ARG;
    int rc = alcs_mx4_bytes(rows, cols, &db, &sb);
    if (rc) return rc;
    if (!db) return ALCS_OK;
    const size_t elt = elt_bytes(dt);
    if (ld > (1ll << 40) / rows) return ALCS_ERR_SHAPE;
    const Buffer buffers[3] = {{m, ((size_t)(rows - 1) * ld + cols) * elt, elt, !quantize, false, 0},
                               {data, db, 16, quantize, false, 0}, {scales, sb, 16, quantize, false, 0}};
    int dev = 0, sms = 0, smem = 0;
    rc = check_buffers(buffers, &dev);
    if (!rc) rc = device_limits(dev, &sms, &smem);
    if (rc) return rc;
    Args a;
    a.x = m; a.y = m; a.data = static_cast<unsigned char*>(data); a.scales = static_cast<unsigned char*>(scales);
    a.ld = ld; a.rows = rows; a.cols = cols;
    a.blocks = 2 * ((cols + 63) / 64);
    a.quads = (cols + 127) / 128;
    a.units = up_div(rows, 8) * a.quads;
    const bool vec = (uintptr_t)m % 16 == 0 && (size_t)ld * elt % 16 == 0 && (size_t)cols * elt % 16 == 0;
    const int blocks = (int)std::min<long long>(up_div(a.units, kThreads / 32), (long long)sms * 8);
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    ALCS_CUDA(dt == ALCS_F32 ? launch<float>(quantize, vec, a, blocks, st) : dt == ALCS_F16 ? launch<__half>(quantize, vec, a, blocks, st)
                                                                                            : launch<__nv_bfloat16>(quantize, vec, a, blocks, st));
    return ALCS_OK;
}

}  // namespace
}  // namespace alcs

extern "C" {

ALCS_API int alcs_mx4_bytes(int rows, int cols, size_t* data_bytes, size_t* scale_bytes)
{
    if (!data_bytes || !scale_bytes || rows < 0 || cols < 0) return ALCS_ERR_INVALID_ARG;
    if (rows > (1 << 30) || cols > (1 << 24)) return ALCS_ERR_SHAPE;
    const size_t tiles = cols ? ((size_t)rows + 127) / 128 : 0;
    *data_bytes = tiles * (2 * (((size_t)cols + 63) / 64)) * 2048;
    *scale_bytes = tiles * (((size_t)cols + 127) / 128) * 512;
    return ALCS_OK;
}

ALCS_API int alcs_mx4_quantize(const void* x, int rows, int cols, long long ldx, alcs_dtype dt, void* data, void* scales, void* cuda_stream)
{
    return alcs::convert(true, data, scales, rows, cols, const_cast<void*>(x), ldx, dt, cuda_stream);
}

ALCS_API int alcs_mx4_dequantize(const void* data, const void* scales, int rows, int cols, void* y, long long ldy, alcs_dtype dt,
                                 void* cuda_stream)
{
    return alcs::convert(false, const_cast<void*>(data), const_cast<void*>(scales), rows, cols, y, ldy, dt, cuda_stream);
}

}  // extern "C"
