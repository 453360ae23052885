// Group norm with an activation on channels-last activations, forward and backward, sm_100a.
//
//     mu, var over a group's pixels and channels;  xh = (x - mu) rstd;  z = gamma xh + beta;  y = act(z)
//     dz = dy act'(z), t = gamma dz:  dbeta = sum dz, dgamma = sum dz xh, dx = rstd (t - mean t - xh mean(t xh))
//
// Bound by memory: x has to be read and y written once (backward: x, dy and dx), and a group's statistics need all of its values before
// the first output.  So a group's part of an image is kept on chip between the two: a work item is a span of neighbouring groups
// (their channels are 64 to 128 bytes of a pixel where that is possible: whole sectors of memory) of one image, its pixels are
// shared out to the blocks of a cluster, and a block holds its share in registers, 16 bytes per load and up to 16 loads per thread in flight.
// A thread keeps to its channels, whose parameters stay in registers.  The sums go through shared memory, in a fixed order, and
// between the cluster's blocks through distributed shared memory.
// Where a span's pixels do not fit a cluster, three passes: statistics of chunks of pixels, their union, and the outputs from a second reading of x.
//
// The variance is that of values with a mean taken off: every block subtracts the mean of its own share, and shares are united by
// M2 = sum M2_k + sum n_k (mean_k - mean)^2, which has no cancellation where the mean is large.  All of it in fp32.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "alcs_dense.h"

namespace alcs {
namespace {

constexpr int kSplitThreads = 256;
constexpr int kMaxThreads = 512;
constexpr int kMaxSpanGroups = 64;          // groups of a span
constexpr int kBatch = 8;                   // loads in flight of the three-pass kernels
enum { kNone = 0, kRelu = 1, kSilu = 2 };

struct Args {
    const void *x, *dy;
    void* out;                   // y, dx
    const float *gamma, *beta;
    float *mean, *rstd;          // stored by the forward, read by the backward pass
    float *part, *sums, *means;  // workspace: see Workspace
    int n, hw, c, groups, cg;    // cg: channels per group
    int gs, spans;               // groups per span
    int chunk, chunks;           // pixels per block, blocks per (span, image)
    float eps;
    int act;
};

// E neighbouring elements as they lie in memory.
template <int B> struct Raw;
template <> struct Raw<16> { using type = uint4; };
template <> struct Raw<8> { using type = uint2; };
template <> struct Raw<4> { using type = unsigned; };
template <> struct Raw<2> { using type = unsigned short; };
template <typename T, int E> using raw_t = typename Raw<E * (int)sizeof(T)>::type;

template <typename T, int E>
__device__ __forceinline__ raw_t<T, E> load(const T* p)
{
    return *reinterpret_cast<const raw_t<T, E>*>(p);
}
template <typename T, int E>
__device__ __forceinline__ void get(const raw_t<T, E>& r, float (&v)[E])
{
    if constexpr (E == 1) {
        T t;
        memcpy(&t, &r, sizeof(T));
        v[0] = to_f32(t);
    } else if constexpr (E * sizeof(T) == 16) {
        Pack<T>::get(r, v);
    } else {
        unpack2(r.x, v, T());
        unpack2(r.y, v + 2, T());
    }
}
template <typename T, int E>
__device__ __forceinline__ void store(T* p, const float (&v)[E])
{
    if constexpr (E == 1) from_f32(p, v[0]);
    else if constexpr (E * sizeof(T) == 16) *reinterpret_cast<uint4*>(p) = Pack<T>::put(v);
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()));
}

__device__ __forceinline__ float activate(float z, int act)
{
    if (act == kRelu) return fmaxf(z, 0.0f);
    if (act == kSilu) return __fdividef(z, 1.0f + __expf(-z));      // (a few units in the last place of fp32)
    return z;
}
// dy * act'(z)
__device__ __forceinline__ float activate_back(float z, float dy, int act)
{
    if (act == kRelu) return z > 0.0f ? dy : 0.0f;
    if (act == kSilu) {
        const float s = __fdividef(1.0f, 1.0f + __expf(-z));
        return dy * (s * fmaf(z, 1.0f - s, 1.0f));
    }
    return dy;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float ld_rank(const float* p, int rank)      // the same place in another block's shared memory
{
    unsigned at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((unsigned)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Where a thread stands: its channels and pixels.
template <int E>
struct Place {
    int img, span, rank;
    int ch0, ng, nch, nv;        // span: first channel, groups, channels, vectors of E channels
    int rows, v, r;              // pixels side by side in the block; the thread's vector, pixel
    bool active;
    int p0, p1;                  // the block's pixels
    __device__ __forceinline__ explicit Place(const Args& a)
    {
        const int unit = blockIdx.x / a.chunks;
        rank = blockIdx.x - unit * a.chunks;
        img = unit / a.spans;
        span = unit - img * a.spans;
        ch0 = span * a.gs * a.cg;
        ng = min(a.gs, a.groups - span * a.gs);
        nch = ng * a.cg;
        nv = nch / E;
        rows = max(1, (int)blockDim.x / nv);
        r = nv <= (int)blockDim.x ? threadIdx.x / nv : 0;
        v = threadIdx.x - r * nv;
        active = r < rows && v < nv;
        p0 = min(a.hw, rank * a.chunk);
        p1 = min(a.hw, p0 + a.chunk);
    }
};

// Sums over the block's threads of values that belong to a thread's E channels, per group of the span: out[group].  `red`: E floats per thread.
// WIDE spans (more vectors than threads) have one group.
template <int E>
__device__ __forceinline__ void sum_groups(const Place<E>& at, int cg, float (&acc)[E], float* red, float* out)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const bool whole = cg % E == 0;                          // a vector lies in one group
    const int nv = min(at.nv, (int)blockDim.x);
    const bool lanes = nv < 32 && (nv & (nv - 1)) == 0;       // lanes nv apart have the same vector
    if (whole)
#pragma unroll
        for (int j = 1; j < E; ++j) acc[0] += acc[j];
    if (lanes)
        for (int o = nv; o < 32; o <<= 1)
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (j == 0 || !whole) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], o);
    const int per = whole ? nv : nv * E;                      // values of a row of `red`
    const int rows = lanes ? warps : at.nv > nv ? 1 : at.rows;
    if (lanes ? lane < nv : at.active) {
        const int row = lanes ? warp : at.r, v = lanes ? lane : at.v;
        if (whole) red[row * per + v] = acc[0];
        else
#pragma unroll
            for (int j = 0; j < E; ++j) red[row * per + v * E + j] = acc[j];
    }
    __syncthreads();
    const int m = at.nv > nv ? per : whole ? cg / E : cg;      // values of a group in a row
    for (int g = warp; g < at.ng; g += warps) {
        float s = 0.0f;
        for (int e = lane; e < rows * m; e += 32) {
            const int row = e / m;
            s += red[row * per + g * m + e - row * m];
        }
        s = warp_sum(s);
        if (lane == 0) out[g] = s;
    }
    __syncthreads();
}

// Sums over the block's pixels of two values per channel: out[0 .. nch) and out[nch .. 2 nch).  `red`: 2 E floats per thread.
template <int E>
__device__ __forceinline__ void sum_channels(const Place<E>& at, float (&u)[E], float (&w)[E], float* red, float* out)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, nv = at.nv;
    const bool lanes = nv < 32 && (nv & (nv - 1)) == 0;
    if (lanes)
        for (int o = nv; o < 32; o <<= 1)
#pragma unroll
            for (int j = 0; j < E; ++j) {
                u[j] += __shfl_xor_sync(0xffffffffu, u[j], o);
                w[j] += __shfl_xor_sync(0xffffffffu, w[j], o);
            }
    const int rows = lanes ? warps : at.rows;
    if (lanes ? lane < nv : at.active) {
        float* to = red + ((lanes ? warp : at.r) * nv + (lanes ? lane : at.v)) * E;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            to[j] = u[j];
            to[rows * at.nch + j] = w[j];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * at.nch; i += blockDim.x) {
        const int k = i >= at.nch, ch = i - k * at.nch;
        float s = 0.0f;
        for (int row = 0; row < rows; ++row) s += red[(k * rows + row) * at.nch + ch];
        out[i] = s;
    }
    __syncthreads();
}

// gamma, beta, mean and rstd of a thread's channels.
template <int E>
struct Channels {
    float gamma[E], beta[E], mean[E], rstd[E];
    __device__ __forceinline__ void params(const Args& a, int ch)
    {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            gamma[j] = a.gamma ? __ldg(a.gamma + ch + j) : 1.0f;
            beta[j] = a.beta ? __ldg(a.beta + ch + j) : 0.0f;
        }
    }
    // from arrays of groups, the first of which is that of channel 0 of `ch`
    __device__ __forceinline__ void stats(const float* m, const float* s, int ch, int cg)
    {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int g = (ch + j) / cg;
            mean[j] = m[g];
            rstd[j] = s[g];
        }
    }
};

template <typename T, int E>
__device__ __forceinline__ void normalise(const raw_t<T, E>& raw, T* to, const Channels<E>& ch, int act)
{
    float v[E];
    get<T, E>(raw, v);
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = activate(fmaf((v[j] - ch.mean[j]) * ch.rstd[j], ch.gamma[j], ch.beta[j]), act);
    store<T, E>(to, v);
}

// ---------------------------------------------------------------------------------------------
// One pass: a block holds its pixels of a span in registers, V loads per thread.

template <typename T, int E, int V>
__global__ void __launch_bounds__(kMaxThreads, V <= 4 ? 2 : 1) norm_kernel(const Args a)
{
    extern __shared__ __align__(16) float red[];
    __shared__ float own_mean[kMaxSpanGroups], own_m2[kMaxSpanGroups], mean[kMaxSpanGroups], rstd[kMaxSpanGroups];
    const Place<E> at(a);
    const int ch = at.v * E;
    let_next_start();
    wait_for_previous();
    Channels<E> par;
    if (at.active) par.params(a, at.ch0 + ch);
    const size_t first = ((size_t)at.img * a.hw + at.p0 + at.r) * a.c + at.ch0 + ch, step = (size_t)at.rows * a.c;
    const T* const x = static_cast<const T*>(a.x) + first;
    const int mine = at.active ? at.p1 - at.p0 - at.r : 0;      // pixels from the thread's first on
    raw_t<T, E> raw[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i * at.rows < mine) raw[i] = load<T, E>(x + i * step);
    float acc[E] = {};
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i * at.rows < mine) {
            float v[E];
            get<T, E>(raw[i], v);
#pragma unroll
            for (int j = 0; j < E; ++j) acc[j] += v[j];
        }
    sum_groups<E>(at, a.cg, acc, red, own_mean);
    const float own = (float)(at.p1 - at.p0) * a.cg, inv = own > 0.0f ? 1.0f / own : 0.0f;
    if (threadIdx.x < at.ng) own_mean[threadIdx.x] *= inv;
    __syncthreads();
    if (at.active) par.stats(own_mean, own_mean, ch, a.cg);
#pragma unroll
    for (int j = 0; j < E; ++j) acc[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i * at.rows < mine) {
            float v[E];
            get<T, E>(raw[i], v);
#pragma unroll
            for (int j = 0; j < E; ++j) acc[j] = fmaf(v[j] - par.mean[j], v[j] - par.mean[j], acc[j]);
        }
    sum_groups<E>(at, a.cg, acc, red, own_m2);
    if (a.chunks > 1) cluster_sync();
    if (threadIdx.x < at.ng) {
        const int g = threadIdx.x;
        float m = 0.0f, m2 = 0.0f;
        const float total = (float)a.hw * a.cg;
        if (a.chunks == 1) {
            m = own_mean[g];
            m2 = own_m2[g];
        } else {
            float sum = 0.0f;
#pragma unroll 1
            for (int k = 0; k < a.chunks; ++k) {
                const int px = max(0, min(a.hw, (k + 1) * a.chunk) - k * a.chunk);
                sum = fmaf(ld_rank(own_mean + g, k), (float)px * a.cg, sum);
            }
            m = sum / total;
#pragma unroll 1
            for (int k = 0; k < a.chunks; ++k) {
                const int px = max(0, min(a.hw, (k + 1) * a.chunk) - k * a.chunk);
                const float d = ld_rank(own_mean + g, k) - m;
                m2 += ld_rank(own_m2 + g, k);
                if (px > 0) m2 = fmaf(d * d, (float)px * a.cg, m2);
            }
        }
        const float s = 1.0f / sqrtf(m2 / total + a.eps);
        mean[g] = m;
        rstd[g] = s;
        if (at.rank == 0 && a.mean) a.mean[(size_t)at.img * a.groups + at.span * a.gs + g] = m;
        if (at.rank == 0 && a.rstd) a.rstd[(size_t)at.img * a.groups + at.span * a.gs + g] = s;
    }
    __syncthreads();
    if (a.chunks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // done with the others' shared memory
    if (at.active) par.stats(mean, rstd, ch, a.cg);
    T* const y = static_cast<T*>(a.out) + first;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i * at.rows < mine) normalise<T, E>(raw[i], y + i * step, par, a.act);
    __syncwarp();
    if (a.chunks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <typename T, int E, int V>
__global__ void __launch_bounds__(kMaxThreads, V <= 2 ? 2 : 1) norm_back_kernel(const Args a)
{
    extern __shared__ __align__(16) float red[];      // 2 E floats per thread; sums per channel: the block's, the image's
    __shared__ float k1[kMaxSpanGroups], k2[kMaxSpanGroups];
    const Place<E> at(a);
    const int ch = at.v * E, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float* const own = red + 2 * E * blockDim.x;
    float* const all = own + 2 * at.nch;
    let_next_start();
    wait_for_previous();
    const size_t first = ((size_t)at.img * a.hw + at.p0 + at.r) * a.c + at.ch0 + ch, step = (size_t)at.rows * a.c;
    const int mine = at.active ? at.p1 - at.p0 - at.r : 0;
    const T* const x = static_cast<const T*>(a.x) + first;
    const T* const dy = static_cast<const T*>(a.dy) + first;
    raw_t<T, E> raw[V], draw[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i * at.rows < mine) {
            raw[i] = load<T, E>(x + i * step);
            draw[i] = load<T, E>(dy + i * step);
        }
    Channels<E> par;
    if (at.active) {
        const size_t g0 = (size_t)at.img * a.groups + at.span * a.gs;
        par.params(a, at.ch0 + ch);
        par.stats(a.mean + g0, a.rstd + g0, ch, a.cg);
    }
    float u[E] = {}, w[E] = {};
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i * at.rows < mine) {
            float v[E], d[E];
            get<T, E>(raw[i], v);
            get<T, E>(draw[i], d);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float xh = (v[j] - par.mean[j]) * par.rstd[j];
                const float dz = activate_back(fmaf(xh, par.gamma[j], par.beta[j]), d[j], a.act);
                u[j] += dz;
                w[j] = fmaf(dz, xh, w[j]);
            }
        }
    sum_channels<E>(at, u, w, red, own);
    if (a.chunks > 1) cluster_sync();
    for (int i = threadIdx.x; i < 2 * at.nch; i += blockDim.x) {
        float s = 0.0f;
        if (a.chunks == 1) s = own[i];
        else
#pragma unroll 1
            for (int k = 0; k < a.chunks; ++k) s += ld_rank(own + i, k);
        all[i] = s;
        if (at.rank == 0 && a.sums) {
            const int k = i >= at.nch, c = at.ch0 + i - k * at.nch;
            a.sums[((size_t)at.img * 2 + k) * a.c + c] = s;
        }
    }
    __syncthreads();
    if (a.chunks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    const float inv = 1.0f / ((float)a.hw * a.cg);
    for (int g = warp; g < at.ng; g += blockDim.x >> 5) {
        float s1 = 0.0f, s2 = 0.0f;
        for (int j = lane; j < a.cg; j += 32) {
            const int c = g * a.cg + j;
            const float gm = a.gamma ? __ldg(a.gamma + at.ch0 + c) : 1.0f;
            s1 = fmaf(gm, all[c], s1);
            s2 = fmaf(gm, all[at.nch + c], s2);
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if (lane == 0) { k1[g] = s1 * inv; k2[g] = s2 * inv; }
    }
    __syncthreads();
    T* const dx = static_cast<T*>(a.out) + first;
    if (at.active) {
#pragma unroll
        for (int j = 0; j < E; ++j) { u[j] = k1[(ch + j) / a.cg]; w[j] = k2[(ch + j) / a.cg]; }
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i * at.rows < mine) {
            float v[E], d[E];
            get<T, E>(raw[i], v);
            get<T, E>(draw[i], d);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float xh = (v[j] - par.mean[j]) * par.rstd[j];
                const float dz = activate_back(fmaf(xh, par.gamma[j], par.beta[j]), d[j], a.act);
                v[j] = par.rstd[j] * (fmaf(par.gamma[j], dz, -u[j]) - xh * w[j]);
            }
            store<T, E>(dx + i * step, v);
        }
    __syncwarp();
    if (a.chunks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---------------------------------------------------------------------------------------------
// Three passes, for spans that do not fit.

// Mean and sum of squared distances from it of a chunk, per group: part[image][chunk][group][2].
template <typename T, int E>
__global__ void __launch_bounds__(kSplitThreads) stats_kernel(const Args a)
{
    extern __shared__ __align__(16) float red[];
    __shared__ float mean[kMaxSpanGroups], m2[kMaxSpanGroups];
    const Place<E> at(a);
    let_next_start();
    wait_for_previous();
    float m[E] = {}, q[E] = {}, count = 0.0f;      // of the thread's values, per channel (or, of a wide span, all of one group)
    for (int v = at.v; at.active && v < at.nv; v += kSplitThreads) {
        const T* const x = static_cast<const T*>(a.x) + (size_t)at.img * a.hw * a.c + at.ch0 + v * E;
        for (int p = at.p0 + at.r; p < at.p1; p += kBatch * at.rows) {
            raw_t<T, E> raw[kBatch];
            int k = 0;
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (p + i * at.rows < at.p1) { raw[i] = load<T, E>(x + (size_t)(p + i * at.rows) * a.c); ++k; }
            float s[E] = {}, b[E] = {};
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (i < k) {
                    float f[E];
                    get<T, E>(raw[i], f);
#pragma unroll
                    for (int j = 0; j < E; ++j) s[j] += f[j];
                }
            const float kf = (float)k, inv = 1.0f / kf, total = count + kf;
#pragma unroll
            for (int j = 0; j < E; ++j) s[j] *= inv;
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (i < k) {
                    float f[E];
                    get<T, E>(raw[i], f);
#pragma unroll
                    for (int j = 0; j < E; ++j) b[j] = fmaf(f[j] - s[j], f[j] - s[j], b[j]);
                }
            const float share = kf / total, both = count * share;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float d = s[j] - m[j];
                m[j] = fmaf(d, share, m[j]);
                q[j] += fmaf(d * d, both, b[j]);
            }
            count = total;
        }
    }
    float acc[E];
#pragma unroll
    for (int j = 0; j < E; ++j) acc[j] = m[j] * count;
    sum_groups<E>(at, a.cg, acc, red, mean);
    const float inv = at.p1 > at.p0 ? 1.0f / ((float)(at.p1 - at.p0) * a.cg) : 0.0f;
    if (threadIdx.x < at.ng) mean[threadIdx.x] *= inv;
    __syncthreads();
    if (at.active)
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float d = m[j] - mean[at.nv > kSplitThreads ? 0 : (at.v * E + j) / a.cg];
            acc[j] = fmaf(d * d, count, q[j]);
        }
    else
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] = 0.0f;
    sum_groups<E>(at, a.cg, acc, red, m2);
    if (threadIdx.x < at.ng) {
        float* to = a.part + (((size_t)at.img * a.chunks + at.rank) * a.groups + at.span * a.gs + threadIdx.x) * 2;
        to[0] = mean[threadIdx.x];
        to[1] = m2[threadIdx.x];
    }
}

// The union of the chunks' statistics, by every block for its groups, and the outputs.
template <typename T, int E>
__global__ void __launch_bounds__(kSplitThreads) apply_kernel(const Args a)
{
    __shared__ float mean[kMaxSpanGroups], rstd[kMaxSpanGroups];
    const Place<E> at(a);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    let_next_start();
    wait_for_previous();
    for (int g = warp; g < at.ng; g += kSplitThreads / 32) {
        const float* const from = a.part + ((size_t)at.img * a.chunks * a.groups + at.span * a.gs + g) * 2;
        const float total = (float)a.hw * a.cg;
        float s = 0.0f, m2 = 0.0f;
        for (int k = lane; k < a.chunks; k += 32) s = fmaf(from[(size_t)k * a.groups * 2], (float)(min(a.hw, (k + 1) * a.chunk) - k * a.chunk) * a.cg, s);
        const float m = warp_sum(s) / total;
        for (int k = lane; k < a.chunks; k += 32) {
            const float d = from[(size_t)k * a.groups * 2] - m;
            m2 += fmaf(d * d, (float)(min(a.hw, (k + 1) * a.chunk) - k * a.chunk) * a.cg, from[(size_t)k * a.groups * 2 + 1]);
        }
        m2 = warp_sum(m2);
        const float r = 1.0f / sqrtf(m2 / total + a.eps);
        if (lane == 0) {
            mean[g] = m;
            rstd[g] = r;
            const size_t o = (size_t)at.img * a.groups + at.span * a.gs + g;
            if (at.rank == 0 && a.mean) a.mean[o] = m;
            if (at.rank == 0 && a.rstd) a.rstd[o] = r;
        }
    }
    __syncthreads();
    for (int v = at.v; at.active && v < at.nv; v += kSplitThreads) {
        Channels<E> par;
        par.params(a, at.ch0 + v * E);
        par.stats(mean, rstd, v * E, a.cg);
        const size_t first = (size_t)at.img * a.hw * a.c + at.ch0 + v * E;
        const T* const x = static_cast<const T*>(a.x) + first;
        T* const y = static_cast<T*>(a.out) + first;
        for (int p = at.p0 + at.r; p < at.p1; p += kBatch * at.rows) {
            raw_t<T, E> raw[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (p + i * at.rows < at.p1) raw[i] = load<T, E>(x + (size_t)(p + i * at.rows) * a.c);
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (p + i * at.rows < at.p1) normalise<T, E>(raw[i], y + (size_t)(p + i * at.rows) * a.c, par, a.act);
        }
    }
}

// sum dz and sum dz xh of a chunk, per channel: part[image][chunk][2][channel].
template <typename T, int E>
__global__ void __launch_bounds__(kSplitThreads) back_stats_kernel(const Args a)
{
    extern __shared__ __align__(16) float red[];
    const Place<E> at(a);
    let_next_start();
    wait_for_previous();
    const size_t g0 = (size_t)at.img * a.groups + at.span * a.gs;
    float* const to = a.part + ((size_t)at.img * a.chunks + at.rank) * 2 * a.c + at.ch0;
    float u[E] = {}, w[E] = {};
    for (int v = at.v; at.active && v < at.nv; v += kSplitThreads) {
        Channels<E> par;
        par.params(a, at.ch0 + v * E);
        par.stats(a.mean + g0, a.rstd + g0, v * E, a.cg);
        const size_t first = (size_t)at.img * a.hw * a.c + at.ch0 + v * E;
        const T* const x = static_cast<const T*>(a.x) + first;
        const T* const dy = static_cast<const T*>(a.dy) + first;
#pragma unroll
        for (int j = 0; j < E; ++j) u[j] = w[j] = 0.0f;
        for (int p = at.p0 + at.r; p < at.p1; p += kBatch / 2 * at.rows) {
            raw_t<T, E> raw[kBatch / 2], draw[kBatch / 2];
#pragma unroll
            for (int i = 0; i < kBatch / 2; ++i)
                if (p + i * at.rows < at.p1) {
                    raw[i] = load<T, E>(x + (size_t)(p + i * at.rows) * a.c);
                    draw[i] = load<T, E>(dy + (size_t)(p + i * at.rows) * a.c);
                }
#pragma unroll
            for (int i = 0; i < kBatch / 2; ++i)
                if (p + i * at.rows < at.p1) {
                    float f[E], d[E];
                    get<T, E>(raw[i], f);
                    get<T, E>(draw[i], d);
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const float xh = (f[j] - par.mean[j]) * par.rstd[j];
                        const float dz = activate_back(fmaf(xh, par.gamma[j], par.beta[j]), d[j], a.act);
                        u[j] += dz;
                        w[j] = fmaf(dz, xh, w[j]);
                    }
                }
        }
        if (at.nv > kSplitThreads)      // a wide span: the thread has all of the chunk's pixels
#pragma unroll
            for (int j = 0; j < E; ++j) {
                to[v * E + j] = u[j];
                to[a.c + v * E + j] = w[j];
            }
    }
    if (at.nv > kSplitThreads) return;
    float* const sums = red + 2 * E * kSplitThreads;
    sum_channels<E>(at, u, w, red, sums);
    for (int i = threadIdx.x; i < at.nch; i += kSplitThreads) {
        to[i] = sums[i];
        to[a.c + i] = sums[at.nch + i];
    }
}

// The chunks' sums of an image's group: sums[image][2][channel], means[image][group][2].  One block per (image, group).
__global__ void __launch_bounds__(128) back_unite_kernel(const Args a)
{
    __shared__ float s1[4], s2[4];
    let_next_start();
    wait_for_previous();
    const int img = blockIdx.x / a.groups, g = blockIdx.x - img * a.groups, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float t1 = 0.0f, t2 = 0.0f;
    for (int j = threadIdx.x; j < a.cg; j += 128) {
        const int c = g * a.cg + j;
        const float* const from = a.part + (size_t)img * a.chunks * 2 * a.c + c;
        float u = 0.0f, w = 0.0f;
#pragma unroll 4
        for (int k = 0; k < a.chunks; ++k) {
            u += from[(size_t)k * 2 * a.c];
            w += from[(size_t)k * 2 * a.c + a.c];
        }
        a.sums[(size_t)img * 2 * a.c + c] = u;
        a.sums[((size_t)img * 2 + 1) * a.c + c] = w;
        const float gm = a.gamma ? __ldg(a.gamma + c) : 1.0f;
        t1 = fmaf(gm, u, t1);
        t2 = fmaf(gm, w, t2);
    }
    t1 = warp_sum(t1);
    t2 = warp_sum(t2);
    if (lane == 0) { s1[warp] = t1; s2[warp] = t2; }
    __syncthreads();
    if (threadIdx.x == 0) {
        const float inv = 1.0f / ((float)a.hw * a.cg);
        float* const to = a.means + ((size_t)img * a.groups + g) * 2;
        to[0] = (s1[0] + s1[1] + s1[2] + s1[3]) * inv;
        to[1] = (s2[0] + s2[1] + s2[2] + s2[3]) * inv;
    }
}

template <typename T, int E>
__global__ void __launch_bounds__(kSplitThreads) back_apply_kernel(const Args a)
{
    const Place<E> at(a);
    let_next_start();
    wait_for_previous();
    const size_t g0 = (size_t)at.img * a.groups + at.span * a.gs;
    for (int v = at.v; at.active && v < at.nv; v += kSplitThreads) {
        Channels<E> par;
        par.params(a, at.ch0 + v * E);
        par.stats(a.mean + g0, a.rstd + g0, v * E, a.cg);
        float k1[E], k2[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            k1[j] = a.means[(g0 + (v * E + j) / a.cg) * 2];
            k2[j] = a.means[(g0 + (v * E + j) / a.cg) * 2 + 1];
        }
        const size_t first = (size_t)at.img * a.hw * a.c + at.ch0 + v * E;
        const T* const x = static_cast<const T*>(a.x) + first;
        const T* const dy = static_cast<const T*>(a.dy) + first;
        T* const dx = static_cast<T*>(a.out) + first;
        for (int p = at.p0 + at.r; p < at.p1; p += kBatch / 2 * at.rows) {
            raw_t<T, E> raw[kBatch / 2], draw[kBatch / 2];
#pragma unroll
            for (int i = 0; i < kBatch / 2; ++i)
                if (p + i * at.rows < at.p1) {
                    raw[i] = load<T, E>(x + (size_t)(p + i * at.rows) * a.c);
                    draw[i] = load<T, E>(dy + (size_t)(p + i * at.rows) * a.c);
                }
#pragma unroll
            for (int i = 0; i < kBatch / 2; ++i)
                if (p + i * at.rows < at.p1) {
                    float f[E], d[E];
                    get<T, E>(raw[i], f);
                    get<T, E>(draw[i], d);
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const float xh = (f[j] - par.mean[j]) * par.rstd[j];
                        const float dz = activate_back(fmaf(xh, par.gamma[j], par.beta[j]), d[j], a.act);
                        f[j] = par.rstd[j] * (fmaf(par.gamma[j], dz, -k1[j]) - xh * k2[j]);
                    }
                    store<T, E>(dx + (size_t)(p + i * at.rows) * a.c, f);
                }
        }
    }
}

// dbeta and dgamma: sums[image][2][channel] over the images, 32 channels per block, eight lanes of images.
__global__ void __launch_bounds__(256) params_kernel(const float* sums, float* dgamma, float* dbeta, int n, int c)
{
    __shared__ float s[2][8][32];
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, ch = blockIdx.x * 32 + lane;
    float u = 0.0f, w = 0.0f;
    if (ch < c)
#pragma unroll 4
        for (int i = warp; i < n; i += 8) {
            u += sums[(size_t)i * 2 * c + ch];
            w += sums[((size_t)i * 2 + 1) * c + ch];
        }
    s[0][warp][lane] = u;
    s[1][warp][lane] = w;
    __syncthreads();
    if (warp >= 2 || ch >= c) return;
    float t = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) t += s[warp][k][lane];
    float* const to = warp ? dgamma : dbeta;
    if (to) to[ch] = t;
}

// ---------------------------------------------------------------------------------------------
// Host

struct NormPlan {
    int e;                     // elements per load
    int gs, threads, loads, cluster, chunk;
    bool one_pass;
    int chunks;                // three passes
    size_t smem;
};

// The loads a one-pass kernel may hold per thread.
constexpr int kLoads[2][4] = {{2, 4, 8, 16}, {1, 2, 4, 8}};

int plan_loads(bool back, long long need)
{
    for (int v : kLoads[back])
        if (v >= need) return v;
    return 0;
}

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

NormPlan make_plan(int n, int hw, int c, int groups, int elt, int align, bool back, int sms)
{
    NormPlan p = {};
    const int cg = c / groups;
    p.e = c * elt % 16 == 0 && align % 16 == 0 ? 16 / elt : elt == 2 && c % 4 == 0 && align % 8 == 0 ? 4 : 1;
    int gs0 = p.e / gcd(p.e, cg);                       // groups whose channels are whole loads
    const int most = kLoads[back][3];
    auto fits = [&](int gs, int threads, int cluster) {
        const long long nv = (long long)gs * cg / p.e;
        return gs <= kMaxSpanGroups && nv <= threads && up_div(up_div(hw, cluster), threads / nv) <= most;
    };
    for (int want : {128, 64, 32, 1}) {
        int gs = gs0;
        while (gs * 2 <= std::min(kMaxSpanGroups, groups) && gs * cg * elt < want) gs *= 2;
        gs = std::min(gs, std::max(gs0, groups));
        for (int threads : {256, 512})
            for (int cluster = 1; cluster <= 8; cluster *= 2) {
                if (!fits(gs, threads, cluster)) continue;
                const long long units = (long long)n * up_div(groups, gs);
                const int rows = threads / (gs * cg / p.e);
                while (cluster < 8 && units * cluster * 2 <= 2 * sms && up_div(hw, cluster * 2) >= 2 * rows) cluster *= 2;
                p.gs = gs; p.threads = threads; p.cluster = cluster;
                p.chunk = (int)up_div(hw, cluster);
                p.loads = plan_loads(back, up_div(p.chunk, rows));
                p.one_pass = true;
                const size_t nch = (size_t)gs * cg;
                p.smem = (size_t)threads * p.e * 4 * (back ? 2 : 1) + (back ? 4 * nch * 4 : 0);
                if (p.smem <= 47 * 1024) return p;
                p.one_pass = false;
            }
    }
    // Three passes.  A span of more loads than threads has to be one group.
    p.threads = kSplitThreads;
    if ((long long)gs0 * cg / p.e > kSplitThreads && gs0 > 1) { p.e = 1; gs0 = 1; }
    p.gs = gs0;
    while (p.gs * 2 <= std::min(kMaxSpanGroups, groups) && (long long)p.gs * 2 * cg / p.e <= kSplitThreads && p.gs * cg * elt < 512) p.gs *= 2;
    const long long units = (long long)n * up_div(groups, p.gs);
    const long long nv = (long long)p.gs * cg / p.e, rows = std::max<long long>(1, kSplitThreads / nv);
    // enough blocks for four per SM, of at least two batches
    long long chunks = std::min(up_div(4ll * sms, units), up_div(hw, 2 * kBatch * rows));
    chunks = std::max(1ll, std::min(chunks, 256ll));
    p.chunk = (int)up_div(hw, chunks);
    p.chunks = (int)up_div(hw, p.chunk);
    p.smem = (size_t)kSplitThreads * p.e * 4 * 2 + (nv <= kSplitThreads ? (size_t)2 * p.gs * cg * 4 : 0);
    return p;
}

// Of the caller's workspace, in floats: sums [n][2][c]; three passes: means [n][groups][2], part.
struct Workspace {
    size_t sums, means, part;
    size_t bytes() const { return (sums + means + part) * 4; }
};
Workspace workspace_of(const NormPlan& p, bool back, int n, int c, int groups)
{
    Workspace w = {};
    if (back) w.sums = (size_t)n * 2 * c;
    if (!p.one_pass) {
        if (back) w.means = (size_t)n * groups * 2;
        w.part = (size_t)n * p.chunks * 2 * (back ? c : groups);
    }
    return w;
}

int check_shape(int n, int h, int wd, int c, int groups)
{
    if (n < 0 || h < 0 || wd < 0 || c < 0 || groups < 1) return ALCS_ERR_INVALID_ARG;
    if (c % groups || c > 65536 || (long long)h * wd >= (1ll << 30) || (long long)n * c >= (1ll << 30)) return ALCS_ERR_SHAPE;
    return ALCS_OK;
}

using Kernel = void (*)(const Args);
template <typename T, int E>
Kernel one_pass_kernel(bool back, int loads)
{
    if (back) return loads == 1 ? norm_back_kernel<T, E, 1> : loads == 2 ? norm_back_kernel<T, E, 2> : loads == 4 ? norm_back_kernel<T, E, 4> : norm_back_kernel<T, E, 8>;
    return loads == 2 ? norm_kernel<T, E, 2> : loads == 4 ? norm_kernel<T, E, 4> : loads == 8 ? norm_kernel<T, E, 8> : norm_kernel<T, E, 16>;
}
// which: 0 one pass, 1 statistics, 2 outputs
template <typename T, int E>
Kernel kernel_of(bool back, int which, int loads)
{
    if (which == 0) return one_pass_kernel<T, E>(back, loads);
    if (which == 1) return back ? back_stats_kernel<T, E> : stats_kernel<T, E>;
    return back ? back_apply_kernel<T, E> : apply_kernel<T, E>;
}
template <typename T>
Kernel kernel_of(int e, bool back, int which, int loads)
{
    if (e == 1) return kernel_of<T, 1>(back, which, loads);
    if constexpr (sizeof(T) == 2) {
        if (e == 4) return kernel_of<T, 4>(back, which, loads);
        return kernel_of<T, 8>(back, which, loads);
    } else {
        return kernel_of<T, 4>(back, which, loads);
    }
}
Kernel kernel_of(alcs_dtype dt, const NormPlan& p, bool back, int which)
{
    return dt == ALCS_F32 ? kernel_of<float>(p.e, back, which, p.loads) : dt == ALCS_F16 ? kernel_of<__half>(p.e, back, which, p.loads)
                                                                                        : kernel_of<__nv_bfloat16>(p.e, back, which, p.loads);
}

int align_of(std::initializer_list<const void*> ps)
{
    int align = 16;
    for (const void* p : ps)
        while ((uintptr_t)p % align) align /= 2;
    return align;
}

int run(Args& a, bool back, alcs_dtype dt, int dev, const NormPlan& p, void* workspace, cudaStream_t st)
{
    const Workspace w = workspace_of(p, back, a.n, a.c, a.groups);
    a.sums = static_cast<float*>(workspace);
    a.means = a.sums + w.sums;
    a.part = a.means + w.means;
    a.gs = p.gs;
    a.spans = (int)up_div(a.groups, p.gs);
    a.chunk = p.chunk;
    a.chunks = p.one_pass ? p.cluster : p.chunks;
    const long long blocks = (long long)a.n * a.spans * a.chunks;
    if (blocks > 0x7fffffffll) return ALCS_ERR_SHAPE;
    const dim3 grid((unsigned)blocks);
    if (p.one_pass) {
        ALCS_CUDA(launch_pdl(kernel_of(dt, p, back, 0), grid, p.threads, p.smem, p.cluster, st, a));
    } else {
        ALCS_CUDA(launch_pdl(kernel_of(dt, p, back, 1), grid, p.threads, p.smem, 1, st, a));
        if (back) ALCS_CUDA(launch_pdl(back_unite_kernel, dim3((unsigned)(a.n * a.groups)), 128, 0, 1, st, a));
        ALCS_CUDA(launch_pdl(kernel_of(dt, p, back, 2), grid, p.threads, p.smem, 1, st, a));
    }
    return ALCS_OK;
}

}  // namespace
}  // namespace alcs

extern "C" {

ALCS_API size_t alcs_group_norm_workspace(int n, int h, int wd, int c, int groups, alcs_dtype dt)
{
    using namespace alcs;
    if (!known_type(dt) || check_shape(n, h, wd, c, groups) || n == 0 || c == 0 || (long long)h * wd == 0) return 0;
    size_t most = 0;
    // (whatever the alignment of the buffers and the number of SMs)
    for (int align : {16, 8, 4})
        for (bool back : {false, true}) {
            const NormPlan p = make_plan(n, h * wd, c, groups, (int)elt_bytes(dt), align, back, 148);
            most = std::max(most, workspace_of(p, back, n, c, groups).bytes());
        }
    return most;
}

ALCS_API int alcs_group_norm(const void* x, void* y, int n, int h, int wd, int c, int groups, const float* gamma, const float* beta,
                             float eps, unsigned flags, alcs_dtype dt, float* mean, float* rstd, void* workspace,
                             size_t workspace_bytes, void* cuda_stream)
{
    using namespace alcs;
    if (!known_type(dt) || (flags & ~(ALCS_RELU | ALCS_SILU)) || flags == (ALCS_RELU | ALCS_SILU) || !(eps >= 0.0f) || !std::isfinite(eps))
        return ALCS_ERR_INVALID_ARG;
    int rc = check_shape(n, h, wd, c, groups);
    if (rc) return rc;
    const int hw = h * wd;
    if (n == 0 || hw == 0 || c == 0) return ALCS_OK;
    const size_t elt = elt_bytes(dt), bytes = (size_t)n * hw * c * elt, sb = (size_t)n * groups * 4;
    const NormPlan p = make_plan(n, hw, c, groups, (int)elt, align_of({x, y}), false, 148);
    const size_t need = workspace_of(p, false, n, c, groups).bytes();
    if (workspace_bytes < need) return ALCS_ERR_INVALID_ARG;
    const Buffer buffers[7] = {{y, bytes, elt, true, false, 1u << 1}, {x, bytes, elt, false, false, 0}, {gamma, (size_t)c * 4, 4, false, true, 0},
                               {beta, (size_t)c * 4, 4, false, true, 0}, {mean, sb, 4, true, true, 0}, {rstd, sb, 4, true, true, 0},
                               {need ? workspace : nullptr, need, 16, true, need == 0, 0}};
    int dev = 0;
    rc = check_buffers(buffers, &dev);
    if (rc) return rc;
    Args a = {};
    a.x = x; a.out = y; a.gamma = gamma; a.beta = beta; a.mean = mean; a.rstd = rstd;
    a.n = n; a.hw = hw; a.c = c; a.groups = groups; a.cg = c / groups; a.eps = eps;
    a.act = flags & ALCS_RELU ? kRelu : flags & ALCS_SILU ? kSilu : kNone;
    return run(a, false, dt, dev, p, workspace, static_cast<cudaStream_t>(cuda_stream));
}

ALCS_API int alcs_group_norm_backward(const void* x, const void* dy, void* dx, int n, int h, int wd, int c, int groups,
                                      const float* mean, const float* rstd, const float* gamma, const float* beta, float* dgamma,
                                      float* dbeta, unsigned flags, alcs_dtype dt, void* workspace, size_t workspace_bytes,
                                      void* cuda_stream)
{
    using namespace alcs;
    if (!known_type(dt) || (flags & ~(ALCS_RELU | ALCS_SILU)) || flags == (ALCS_RELU | ALCS_SILU)) return ALCS_ERR_INVALID_ARG;
    int rc = check_shape(n, h, wd, c, groups);
    if (rc) return rc;
    const int hw = h * wd;
    if (c == 0) return ALCS_OK;
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t elt = elt_bytes(dt), bytes = (size_t)n * hw * c * elt, sb = (size_t)n * groups * 4;
    const bool none = bytes == 0;
    NormPlan p = {};
    size_t need = 0;
    if (!none) {
        p = make_plan(n, hw, c, groups, (int)elt, align_of({x, dy, dx}), true, 148);
        need = workspace_of(p, true, n, c, groups).bytes();
        if (workspace_bytes < need) return ALCS_ERR_INVALID_ARG;
    }
    const Buffer buffers[10] = {{dx, bytes, elt, true, false, 1u << 1 | 1u << 2}, {x, bytes, elt, false, false, 0}, {dy, bytes, elt, false, false, 0},
                                {mean, none ? 0 : sb, 4, false, false, 0}, {rstd, none ? 0 : sb, 4, false, false, 0},
                                {gamma, (size_t)c * 4, 4, false, true, 0}, {beta, (size_t)c * 4, 4, false, true, 0},
                                {dgamma, (size_t)c * 4, 4, true, true, 0}, {dbeta, (size_t)c * 4, 4, true, true, 0},
                                {need ? workspace : nullptr, need, 16, true, need == 0, 0}};
    int dev = 0;
    rc = check_buffers(buffers, &dev);
    if (rc) return rc;
    if (!none) {
        Args a = {};
        a.x = x; a.dy = dy; a.out = dx; a.gamma = gamma; a.beta = beta; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
        a.n = n; a.hw = hw; a.c = c; a.groups = groups; a.cg = c / groups;
        a.act = flags & ALCS_RELU ? kRelu : flags & ALCS_SILU ? kSilu : kNone;
        rc = run(a, true, dt, dev, p, workspace, st);
        if (rc) return rc;
    }
    if (dgamma || dbeta)
        ALCS_CUDA(launch_pdl(params_kernel, dim3((unsigned)up_div(c, 32)), 256, 0, 1, st, static_cast<const float*>(workspace), dgamma, dbeta, none ? 0 : n, c));
    return ALCS_OK;
}

}  // extern "C"
