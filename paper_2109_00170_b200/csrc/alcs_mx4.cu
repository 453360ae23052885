// Microscaled 4-bit floating point (E2M1 values, one E8M0 scale per 32 of a row): quantisation and its inverse, sm_100a.
//
// Both are bound by memory: 2 (fp32: 4) bytes per value on one side, 17/32 on the other.  Four lanes take a block of 32 values, 8
// each; a warp takes 8 rows x 4 blocks, one block of its 8 rows at a time: it reads 8 runs of 64 (128) bytes and writes 128 contiguous
// bytes, since 8 rows of a block lie together in the storage format.  The largest magnitude goes round the four
// lanes by shuffles; the rounding is the hardware's conversion to E2M1 (to nearest, ties to even, saturating).
#include <algorithm>

#include "alcs_dense.h"
#include "alcs_tc.h"

namespace alcs {
namespace {

constexpr int kThreads = 256;

struct Args {
    const void* x;
    void* y;
    unsigned char *data, *scales;
    long long ld;
    int rows, cols, blocks;             // blocks of a row as stored (even)
    TcDiv quads;                        // groups of four
    long long units;                    // 8 rows x 4 blocks
};

// u / quads: a multiplication where u has 31 bits
__device__ __forceinline__ int band_of(const Args& a, long long u)
{
    if (a.units < 0x7fffffffll) return (int)((unsigned long long)(unsigned)u * a.quads.mul >> a.quads.shift);
    return (int)(u / a.quads.d);
}

// Eight values as codes, the first in the lowest four bits.
__device__ __forceinline__ unsigned encode8(const float* v)
{
    unsigned r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// Values of eight codes.
__device__ __forceinline__ void decode8(unsigned r, float* v)
{
    unsigned h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}" : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(r));
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(h[i], v + 2 * i, __half());
}

// A lane's 8 values of a row as they lie in memory, from column c on; zeros behind the last column.
template <typename T> struct Eight { uint4 r[8 * sizeof(T) / 16]; };
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int c, int cols, Eight<T>& v)
{
    constexpr int n = Pack<T>::n;
    if (VEC) {      // (cols is a multiple of 16 bytes' elements)
#pragma unroll
        for (int i = 0; i < 8 / n; ++i) {
            v.r[i] = make_uint4(0, 0, 0, 0);
            if (c + i * n < cols)
                asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.r[i].x), "=r"(v.r[i].y), "=r"(v.r[i].z), "=r"(v.r[i].w) : "l"(row + c + i * n));
        }
    } else {
        T* const e = reinterpret_cast<T*>(&v);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = c + i < cols ? row[c + i] : T(0.0f);
    }
}

__device__ __forceinline__ unsigned max_halves(unsigned a, unsigned b)      // of 16 bits each
{
    unsigned r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// The largest magnitude of a block, of which four lanes have 8 values each, as fp32 bits: as integers magnitudes have the numbers' order, NaN above infinity.  16-bit
// types are compared two at a time, as they are.
__device__ __forceinline__ unsigned largest(const Eight<float>& v)
{
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) top = max(max(top, max(v.r[i].x & 0x7fffffffu, v.r[i].y & 0x7fffffffu)), max(v.r[i].z & 0x7fffffffu, v.r[i].w & 0x7fffffffu));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    return max(top, __shfl_xor_sync(0xffffffffu, top, 2));
}
template <typename T>
__device__ __forceinline__ unsigned largest(const Eight<T>& v)
{
    const uint4& r = v.r[0];
    unsigned top = max_halves(max_halves(r.x & 0x7fff7fffu, r.y & 0x7fff7fffu), max_halves(r.z & 0x7fff7fffu, r.w & 0x7fff7fffu));
    top = max_halves(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max_halves(top, __shfl_xor_sync(0xffffffffu, top, 2));
    float f[2];
    unpack2(max(top & 0xffffu, top >> 16), f, T());
    return __float_as_uint(f[0]) & 0x7fffffffu;
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
        const int band = band_of(a, u), quad = (int)(u - (long long)band * a.quads.d), r = band * 8 + (lane >> 2);
        const bool mine = r < a.rows;
        const T* row = static_cast<const T*>(a.x) + (size_t)r * a.ld;
        Eight<T> v[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) load8<T, VEC>(row, (quad * 4 + b) * 32 + q * 8, mine ? a.cols : 0, v[b]);
        unsigned char* to = a.data + ((size_t)(r >> 7) * a.blocks + quad * 4) * 2048 + (r & 127) * 16 + q * 4;
        unsigned scales = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int e = (int)(largest(v[b]) >> 23);   // floor(log2) + 127; 0 for subnormal numbers, whose scale is 2^-127, too
            const bool finite = e < 255;
            const int s = finite ? max(e - 2, 0) : 255;
            const float inv = __uint_as_float((unsigned)(254 - (finite ? s : 127)) << 23);      // 2^(127 - s)
            float f[8], k[8];
#pragma unroll
            for (int i = 0; i < 8; i += Pack<T>::n) Pack<T>::get(v[b].r[i / Pack<T>::n], f + i);
#pragma unroll
            for (int i = 0; i < 8; ++i) k[i] = inv;
            mul<8>(f, f, k);
            scales |= (unsigned)s << (8 * b);
            const unsigned code = finite ? encode8(f) : 0u;
            if (mine && quad * 4 + b < a.blocks) *reinterpret_cast<unsigned*>(to + b * 2048) = code;
        }
        if (mine && q == 0)
            *reinterpret_cast<unsigned*>(a.scales + ((size_t)(r >> 7) * a.quads.d + quad) * 512 + (r & 31) * 16 + (r >> 5 & 3) * 4) = scales;
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
        const int band = band_of(a, u), quad = (int)(u - (long long)band * a.quads.d), r = band * 8 + (lane >> 2);
        if (r >= a.rows) continue;
        const unsigned char* from = a.data + ((size_t)(r >> 7) * a.blocks + quad * 4) * 2048 + (r & 127) * 16 + q * 4;
        const unsigned scales = *reinterpret_cast<const unsigned*>(a.scales + ((size_t)(r >> 7) * a.quads.d + quad) * 512 + (r & 31) * 16 + (r >> 5 & 3) * 4);
        unsigned code[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) code[b] = quad * 4 + b < a.blocks ? *reinterpret_cast<const unsigned*>(from + b * 2048) : 0u;
        T* row = static_cast<T*>(a.y) + (size_t)r * a.ld;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const unsigned s = scales >> (8 * b) & 255u;
            // 2^(s - 127): a subnormal number for s = 0; 255 is the exponent of NaN
            const float scale = __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7fffffffu : s << 23);
            float v[8], k[8];
            decode8(code[b], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) k[i] = scale;
            mul<8>(v, v, k);
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
    a.quads = tc_div((cols + 127) / 128);
    a.units = up_div(rows, 8) * a.quads.d;
    const bool vec = (uintptr_t)m % 16 == 0 && (size_t)ld * elt % 16 == 0 && (size_t)cols * elt % 16 == 0;
    const int blocks = (int)std::min<long long>(up_div(a.units, kThreads / 32), (long long)sms * 64);      // (short blocks: the scheduler balances them)
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
