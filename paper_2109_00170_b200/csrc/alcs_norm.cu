// Group norm with an activation on channels-last activations, forward and backward, sm_100a.
//
//     mu, var over a group's pixels and channels;  xh = (x - mu) rstd;  z = gamma xh + beta;  y = act(z)
//     dz = dy act'(z), t = gamma dz:  dbeta = sum dz, dgamma = sum dz xh, dx = rstd (t - mean t - xh mean(t xh))
//
// Bound by memory: x has to be read and y written once (backward: x, dy and dx), and a group's statistics need all of its values before
// the first output.
//
// One pass: a group's part of an image is kept on chip between the two.  A work item is a span of neighbouring groups (their channels are 64 to 128 bytes
// of a pixel where that is possible: whole sectors of memory) of one image; its pixels are shared out to the blocks of a cluster, and a block holds its
// share in shared memory, which cp.async fills without holding registers.  A thread keeps to its channels.  Sums go through shared memory, in a fixed
// order, and between the cluster's blocks through distributed shared memory.  What it costs over a copy is the sums: all blocks of an SM tend to be at them
// at the same time, with memory idle (64 images of 56x56x128, bf16: 29.7 us among other calls; a copy of them 22.5; the same
// kernel without the sums 24.6; floor 15.7 at 6.5 TB/s).
//
// Two passes: sums of chunks of pixels, then the outputs from a second reading, which L2 serves as far as it holds x (and dy).  For spans that do
// not fit a cluster, and for large calls of the backward pass.  Every thread keeps 8 loads (4 of x and dy each) on their way to slots of its own in
// shared memory: with as many registers instead, a third of the bytes were in flight (backward of 64 images of 56x56x256, SiLU: 143 us, then 105;
// 95 now, 47 and 52 us for the passes by themselves, with cold caches).
//
// The variance has no cancellation: a thread takes its values one by one into a running mean and sum of squared distances, and these are united by
// M2 = M2_a + M2_b + n_a n_b / n (mean_a - mean_b)^2.  A mean of means is a sum of each one's share, so that no sum is larger than the values.  All of it is held in fp32.
#include <algorithm>
#include <cmath>
#include <mutex>
#include <set>

#include "alcs_dense.h"
#include "alcs_tc.h"

namespace alcs {
namespace {

constexpr int kThreads = 128, kSplitThreads = 256;      // one pass; two passes
constexpr int kMaxCluster = 16, kMostThreads = 1024;      // one pass, forward: threads per SM (64 registers each)
constexpr int kMaxGroupChannels = 8192;     // (their sums stand in shared memory)
constexpr int kMaxSpanGroups = 64;          // groups of a span

struct Args {
    const void *x, *dy;
    void* out;                   // y, dx
    const float *gamma, *beta;
    float *mean, *rstd;          // stored by the forward, read by the backward pass
    float *part, *sums;          // workspace: see Workspace
    int n, hw, c, groups, cg;    // cg: channels per group
    int gs, spans;               // groups per span
    int chunk, chunks;           // pixels per block, blocks per (span, image)
    int loads;                   // one pass: loads per thread
    int span_ch;                 // channels per span, rounded up to a multiple of 4
    int whole;                   // a load's channels lie in one group
    TcDiv cdiv, vdiv;            // by cg; by the loads of a group
    TcDiv chdiv, spdiv;          // by chunks, spans
    TcDiv nvdiv, rowdiv;         // of a span of gs groups: by its loads per pixel, by the pixels side by side in a block
    float eps;
    int relu, silu;
    float *dgamma, *dbeta;
    int first;                   // blocks in front of those that the kernel's own work is for (see back_apply_kernel)
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
    } else if constexpr (sizeof(T) == 4) {
        v[0] = __uint_as_float(r.x);
        v[1] = __uint_as_float(r.y);
    } else if constexpr (E == 2) {
        unpack2(r, v, T());
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
    else if constexpr (sizeof(T) == 4) *reinterpret_cast<uint2*>(p) = make_uint2(__float_as_uint(v[0]), __float_as_uint(v[1]));
    else if constexpr (E == 2) *reinterpret_cast<unsigned*>(p) = pack2(v[0], v[1], T());
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()));
}

template <int E>
__device__ __forceinline__ void set(float (&d)[E], float v)
{
#pragma unroll
    for (int j = 0; j < E; ++j) d[j] = v;
}
// E floats of shared memory, 4 E bytes aligned to their size up to 16
template <int E>
__device__ __forceinline__ void load_shared(float (&d)[E], const float* p)
{
    if constexpr (E == 1) {
        d[0] = p[0];
    } else if constexpr (E == 2) {
        const float2 f = *reinterpret_cast<const float2*>(p);
        d[0] = f.x; d[1] = f.y;
    } else
#pragma unroll
        for (int j = 0; j < E; j += 4) {
            const float4 f = *reinterpret_cast<const float4*>(p + j);
            d[j] = f.x; d[j + 1] = f.y; d[j + 2] = f.z; d[j + 3] = f.w;
        }
}
template <int E>
__device__ __forceinline__ void store_shared(float* p, const float (&d)[E])
{
    if constexpr (E == 1) p[0] = d[0];
    else if constexpr (E == 2) *reinterpret_cast<float2*>(p) = make_float2(d[0], d[1]);
    else
#pragma unroll
        for (int j = 0; j < E; j += 4) *reinterpret_cast<float4*>(p + j) = make_float4(d[j], d[j + 1], d[j + 2], d[j + 3]);
}

// s = 1 / (1 + exp(-z)).  What bounds SiLU is the special function unit: two neighbours share a reciprocal (r = 1 / (a b), 1 / a = r b), so that an
// element takes it one and a half times.  exp(-z) is held below 2^62 for that, and z, whose product with s is wanted, above -43, where that is: SiLU and its slope stay
// what they are there, -9.3e-18, however low z is (1 to 2 % of a SiLU pass; an exact branch for what lies below cost 3 to 10).  Each instruction is good to 2^-22
// or so, and the exponent to z 2^-24.
template <int E>
__device__ __forceinline__ void sigmoid(float (&s)[E], float (&z)[E])
{
    float k[E], one[E];
    set<E>(k, -1.4426950408889634f);
    set<E>(one, 1.0f);
    mul<E>(s, z, k);
#pragma unroll
    for (int j = 0; j < E; ++j) {
        s[j] = fminf(s[j], 62.0f);      // (NaN, too, which its own z brings back, so that a neighbour's stays its own)
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(s[j]));
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(z[j]) : "f"(-43.0f));      // (a NaN stays)
    }
    add<E>(s, s, one);
    if constexpr (E == 1) {
        asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(s[0]));
    } else {
#pragma unroll
        for (int j = 0; j < E; j += 2) {
            float r = s[j] * s[j + 1];
            asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r));
            const float first = r * s[j + 1];
            s[j + 1] = r * s[j];
            s[j] = first;
        }
    }
}

template <bool SILU, int E>
__device__ __forceinline__ void activate(float (&z)[E], bool relu)
{
    if (SILU) {
        float s[E];
        sigmoid<E>(s, z);
        mul<E>(z, z, s);
    } else if (relu) {
#pragma unroll
        for (int j = 0; j < E; ++j) z[j] = fmaxf(z[j], 0.0f);
    }
}
// y = act(z).  ReLU of 16-bit types takes two values at a time, behind their rounding, which keeps the sign.
template <typename T, int E, bool SILU>
__device__ __forceinline__ void store_activated(T* y, float (&z)[E], bool relu)
{
    if constexpr (!SILU && sizeof(T) == 2 && E == 8) {
        uint4 r = Pack<T>::put(z);
        if (relu) r = positive(r, T());
        *reinterpret_cast<uint4*>(y) = r;
    } else {
        activate<SILU, E>(z, relu);
        store<T, E>(y, z);
    }
}
// d = dy * act'(z)
template <bool SILU, int E>
__device__ __forceinline__ void activate_back(float (&d)[E], float (&z)[E], bool relu)
{
    if (SILU) {      // s (1 + z (1 - s)) = s + (z s) (1 - s)
        float s[E], one[E];
        set<E>(one, 1.0f);
        sigmoid<E>(s, z);
        mul<E>(z, z, s);
        sub<E>(one, one, s);
        fma<E>(s, z, one, s);
        mul<E>(d, d, s);
    } else if (relu) {
#pragma unroll
        for (int j = 0; j < E; ++j) d[j] = z[j] > 0.0f ? d[j] : 0.0f;
    }
}

__device__ __forceinline__ void cluster_sync()
{
    cluster_arrive();
    cluster_wait();
}
__device__ __forceinline__ float2 ld_rank(const float2* p, int rank)      // the same place in another block's shared memory
{
    unsigned at;
    float2 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((unsigned)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}
// Sum over the neighbouring `n` lanes (a power of two)
__device__ __forceinline__ float lanes_sum(float v, int n)
{
    for (int o = n >> 1; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// E floats in two places of E elements of T (fp32: in the first alone)
template <typename T, int E>
__device__ __forceinline__ void put_dz(raw_t<T, E>* a, raw_t<T, E>* b, const float (&d)[E])
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (E == 1) *a = __float_as_uint(d[0]);
        else if constexpr (E == 2) *a = make_uint2(__float_as_uint(d[0]), __float_as_uint(d[1]));
        else *a = Pack<float>::put(d);
    } else if constexpr (E == 8) {
        *a = Pack<float>::put(d);
        *b = Pack<float>::put(d + 4);
    } else if constexpr (E == 4) {
        *a = make_uint2(__float_as_uint(d[0]), __float_as_uint(d[1]));
        *b = make_uint2(__float_as_uint(d[2]), __float_as_uint(d[3]));
    } else if constexpr (E == 2) {
        *a = __float_as_uint(d[0]);
        *b = __float_as_uint(d[1]);
    } else {
        *a = (unsigned short)(__float_as_uint(d[0]) & 0xffffu);
        *b = (unsigned short)(__float_as_uint(d[0]) >> 16);
    }
}
template <typename T, int E>
__device__ __forceinline__ void get_dz(const raw_t<T, E>* a, const raw_t<T, E>* b, float (&d)[E])
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (E == 1) d[0] = __uint_as_float(*a);
        else if constexpr (E == 2) get<T, E>(*a, d);
        else Pack<float>::get(*a, d);
    } else if constexpr (E == 8) {
        Pack<float>::get(*a, d);
        Pack<float>::get(*b, d + 4);
    } else if constexpr (E == 4) {
        const uint2 x = *a, y = *b;
        d[0] = __uint_as_float(x.x); d[1] = __uint_as_float(x.y); d[2] = __uint_as_float(y.x); d[3] = __uint_as_float(y.y);
    } else if constexpr (E == 2) {
        d[0] = __uint_as_float(*a);
        d[1] = __uint_as_float(*b);
    } else {
        d[0] = __uint_as_float((unsigned)*a | (unsigned)*b << 16);
    }
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// n / d as a multiplication (an integer division is 30 instructions, and there are ten per thread)
__device__ __forceinline__ int over(int n, const TcDiv& d) { return (int)((unsigned long long)(unsigned)n * d.mul >> d.shift); }

// Where a thread stands: its channels and pixels.
template <int E, int N>
struct Place {
    int img, span, rank;
    int ch0, ng, nch, nv;        // span: first channel, groups, channels, vectors of E channels
    int rows, v, r;              // pixels side by side in the block; the thread's vector, pixel
    bool active;
    int p0, p1;                  // the block's pixels
    int loads;                   // the thread's, of a column of loads
    __device__ __forceinline__ explicit Place(const Args& a)
    {
        const int block = (int)blockIdx.x - a.first, unit = over(block, a.chdiv);
        rank = block - unit * a.chunks;
        img = over(unit, a.spdiv);
        span = unit - img * a.spans;
        ch0 = span * a.gs * a.cg;
        ng = min(a.gs, a.groups - span * a.gs);
        nch = ng * a.cg;
        p0 = min(a.hw, rank * a.chunk);
        p1 = min(a.hw, p0 + a.chunk);
        const bool whole = ng == a.gs;      // (the last span may have fewer)
        nv = whole ? a.nvdiv.d : nch / E;
        rows = whole ? a.rowdiv.d : max(1, N / nv);
        r = nv > N ? 0 : whole ? over(threadIdx.x, a.nvdiv) : threadIdx.x / nv;
        v = threadIdx.x - r * nv;
        active = r < rows && v < nv;
        const int mine = active ? max(0, p1 - p0 - r + rows - 1) : 0;
        loads = whole ? over(mine, a.rowdiv) : mine / rows;
    }
};

// Threads that share a group's values in the sums below: 2^k neighbouring lanes, as many as there are threads for.
template <int N>
__device__ __forceinline__ int lanes_of(int groups) { return min(5, 31 - __clz(max(1, N / groups))); }

// Mean and sum of squared distances from it, value by value (Welford's recurrence, E channels side by side): one operation more per value than sums of values
// less one of them, and no loss where that one is far from the others.
template <int E>
struct Running {
    float m[E], q[E], n = 0.0f;
    __device__ __forceinline__ Running()
    {
        set<E>(m, 0.0f);
        set<E>(q, 0.0f);
    }
    __device__ __forceinline__ void take(float (&v)[E])
    {
        n += 1.0f;
        float r, d[E], k[E];
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(n));      // (the mean's steps need no more)
        set<E>(k, r);
        sub<E>(d, v, m);
        fma<E>(m, d, k, m);
        sub<E>(v, v, m);
        fma<E>(q, d, v, q);
    }
};

// n values of mean m and sum of squared distances q, united with as many again as `other` says.  Either may be none (m = q = 0): the distance of the means then
// is the size of a value, whose square, or n times which, may not be a number of fp32 (0 times which is NaN), and is multiplied by 0 before it is squared.
struct Union {
    float to, w;      // share of the other's; weight of the squared distance of the means
    __device__ __forceinline__ Union(float n, float other) : to(n + other > 0.0f ? other / (n + other) : 0.0f), w(n * to) {}
    __device__ __forceinline__ void operator()(float& m, float& q, float om, float oq) const
    {
        const float d = om - m;
        m = fmaf(d, to, m);
        q += fmaf(d * w, d, oq);
    }
};

// Mean and sum of squared distances from it of the block's values of every group of the span: out[group].  A thread has n values of mean m and
// squared distances q per channel.  `red`: 2 E floats per thread, `count`: one per thread.
template <int N, int E>
__device__ __forceinline__ void unite(const Place<E, N>& at, const Args& a, float n, float (&m)[E], float (&q)[E], float* red, float* count, float2* out)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool lanes = at.nv < 32 && (at.nv & (at.nv - 1)) == 0;       // lanes nv apart have the same vector
    float k = n;
    if (a.whole && E > 1) {      // the thread's channels are one group's
        float s = 0.0f, t = 0.0f;
#pragma unroll
        for (int j = 0; j < E; ++j) s = fmaf(m[j], 1.0f / E, s);
#pragma unroll
        for (int j = 0; j < E; ++j) t += fmaf((m[j] - s) * k, m[j] - s, q[j]);
        m[0] = s;
        q[0] = t;
        k *= E;
    }
    if (lanes)
        for (int o = at.nv; o < 32; o <<= 1) {
            const float other = __shfl_xor_sync(0xffffffffu, k, o);
            const Union u(k, other);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (j == 0 || !a.whole) u(m[j], q[j], __shfl_xor_sync(0xffffffffu, m[j], o), __shfl_xor_sync(0xffffffffu, q[j], o));
            k += other;
        }
    const int per = a.whole ? at.nv : at.nch, rows = lanes ? N / 32 : at.rows;
    const int row = lanes ? warp : at.r, v = lanes ? lane : at.v;
    if (lanes ? lane < at.nv : at.active) {
        if (v == 0) count[row] = k;
        float* const to = red + row * per;
        if (a.whole) {
            to[v] = m[0];
            to[rows * per + v] = q[0];
        } else {
            store_shared<E>(to + v * E, m);
            store_shared<E>(to + rows * per + v * E, q);
        }
    }
    __syncthreads();
    const int w = a.whole ? a.cg / E : a.cg;      // entries of a group in a row
    const float inv = at.p1 > at.p0 ? 1.0f / ((float)(at.p1 - at.p0) * a.cg) : 0.0f;
    const int lk = lanes_of<N>(at.ng), l = 1 << lk, sub = threadIdx.x & (l - 1), mine = threadIdx.x >> lk;
    for (int g0 = mine; g0 - mine < at.ng; g0 += N >> lk) {      // (all threads: their lanes exchange sums)
        const int g = min(g0, at.ng - 1);
        const float* const from = red + g * w;
        float s = 0.0f, t = 0.0f;
        for (int e = sub; e < rows * w; e += l) {
            const int r = over(e, a.whole ? a.vdiv : a.cdiv);
            s = fmaf(from[r * per + e - r * w], count[r] * inv, s);
        }
        s = lanes_sum(s, l);
        for (int e = sub; e < rows * w; e += l) {
            const int r = over(e, a.whole ? a.vdiv : a.cdiv), i = r * per + e - r * w;
            const float d = from[i] - s;
            t += count[r] > 0.0f ? fmaf(d * d, count[r], from[rows * per + i]) : 0.0f;
        }
        t = lanes_sum(t, l);
        if (sub == 0 && g == g0) out[g] = make_float2(s, t);
    }
}

// rstd times a sum of dz (x - mean): 0 where rstd is, even if the distances that it is 0 for have no sum.
__device__ __forceinline__ float times_rstd(float sum, float rstd) { return rstd == 0.0f ? 0.0f : sum * rstd; }

// gamma-weighted sums of the groups from the sums per channel: out[group].
template <int N, int E>
__device__ __forceinline__ void weigh(const Place<E, N>& at, const Args& a, const float* gamma, const float* rstd, const float* sums, float2* out)
{
    const int lk = lanes_of<N>(at.ng), l = 1 << lk, sub = threadIdx.x & (l - 1), mine = threadIdx.x >> lk;
    for (int g0 = mine; g0 - mine < at.ng; g0 += N >> lk) {
        const int g = min(g0, at.ng - 1);
        float s1 = 0.0f, s2 = 0.0f;
        for (int j = sub; j < a.cg; j += l) {
            const int c = g * a.cg + j;
            s1 = fmaf(gamma[c], sums[c], s1);
            s2 = fmaf(gamma[c], sums[at.nch + c], s2);
        }
        s1 = lanes_sum(s1, l);
        s2 = lanes_sum(s2, l);
        if (sub == 0 && g == g0) out[g] = make_float2(s1, times_rstd(s2, rstd[g * a.cg]));
    }
}

// Sums over the block's pixels of two values per channel: out[0 .. nch) and out[nch .. 2 nch).  `red`: 2 E floats per thread.
template <int N, int E>
__device__ __forceinline__ void sum_channels(const Place<E, N>& at, float (&u)[E], float (&w)[E], float* red, float* out)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = N / 32, nv = at.nv;
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
        store_shared<E>(to, u);
        store_shared<E>(to + rows * at.nch, w);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * at.nch; i += N) {
        const float* from = red + (i >= at.nch ? (rows - 1) * at.nch : 0) + i;
        float s = 0.0f;
#pragma unroll 4
        for (int row = 0; row < rows; ++row) s += from[row * at.nch];
        out[i] = s;
    }
    __syncthreads();
}

// ---------------------------------------------------------------------------------------------
// One pass: a block holds its pixels of a span in shared memory, slot [i][thread] the thread's i-th load.  A thread reads only what it has
// fetched itself, so that no barrier stands between.

template <int B>
__device__ __forceinline__ void fetch_async(void* to, const void* from)
{
    const unsigned at = (unsigned)__cvta_generic_to_shared(to);
    if constexpr (B == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(B) : "memory");
}
// The thread's n loads, `step` elements apart, on their way to its slots.
template <typename T, int E, int N>
__device__ __forceinline__ void fetch(raw_t<T, E>* slot, const T* x, size_t step, int n)
{
#pragma unroll 4
    for (int i = 0; i < n; ++i, x += step) {
        if constexpr (E * sizeof(T) >= 4) fetch_async<E * (int)sizeof(T)>(slot + i * N, x);
        else slot[i * N] = load<T, E>(x);
    }
}
__device__ __forceinline__ void fetched() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ int pixels_of(const Args& a, int k) { return max(0, min(a.hw, (k + 1) * a.chunk) - k * a.chunk); }      // of block k of a cluster

template <typename T, int E, bool SILU, int N>
__global__ void __launch_bounds__(N, kMostThreads / N) norm_kernel(const Args a)
{
    extern __shared__ __align__(16) float red[];      // 2 E floats per thread; per channel; slots
    __shared__ float count[N];
    __shared__ float2 own[kMaxSpanGroups];             // of the block's pixels: mean, squared distances from it
    const Place<E, N> at(a);
    float* const mean = red + 2 * E * N;        // of the image, per channel
    float* const scale = mean + a.span_ch;             // rstd * gamma, beta
    float* const shift = scale + a.span_ch;
    raw_t<T, E>* const slot = reinterpret_cast<raw_t<T, E>*>(shift + a.span_ch) + threadIdx.x;
    const int ch = at.v * E;
    let_next_start();
    wait_for_previous();
    const size_t first = ((size_t)at.img * a.hw + at.p0 + at.r) * a.c + at.ch0 + ch, step = (size_t)at.rows * a.c;
    const int n = at.loads;
    fetch<T, E, N>(slot, static_cast<const T*>(a.x) + first, step, n);
    for (int i = threadIdx.x; i < at.nch; i += N) {
        scale[i] = a.gamma ? a.gamma[at.ch0 + i] : 1.0f;
        shift[i] = a.beta ? a.beta[at.ch0 + i] : 0.0f;
    }
    fetched();
    Running<E> stat;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        float v[E];
        get<T, E>(slot[i * N], v);
        stat.take(v);
    }
    unite<N, E>(at, a, stat.n, stat.m, stat.q, red, count, own);
    if (a.chunks > 1) cluster_sync();
    else __syncthreads();
    // Every block unites the cluster's, a lane per (group, block), and spreads a group's result over its channels.
    const float total = 1.0f / ((float)a.hw * a.cg);
    const int lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i - lane < at.ng * a.chunks; i += N) {
        const int g = min(over(i, a.chdiv), at.ng - 1), r = i & (a.chunks - 1);      // (chunks: a power of two, at most 16)
        const float w = (float)pixels_of(a, r) * a.cg;
        const float2 o = a.chunks > 1 ? ld_rank(own + g, r) : own[g];
        const float mu = lanes_sum(w > 0.0f ? o.x * (w * total) : 0.0f, a.chunks);      // (a block without pixels adds nothing, but its lanes take part)
        const float d = o.x - mu;
        const float var = lanes_sum(w > 0.0f ? fmaf(d * d, w * total, o.y * total) : 0.0f, a.chunks);      // (each part's share: less than their sum)
        const float rs = 1.0f / sqrtf(var + a.eps);
        if (i < at.ng * a.chunks) {
            for (int j = r; j < a.cg; j += a.chunks) {
                mean[g * a.cg + j] = mu;
                scale[g * a.cg + j] *= rs;
            }
            if (at.rank == 0 && r == 0) {
                const size_t to = (size_t)at.img * a.groups + at.span * a.gs + g;
                if (a.mean) a.mean[to] = mu;
                if (a.rstd) a.rstd[to] = rs;
            }
        }
    }
    __syncthreads();
    if (a.chunks > 1) cluster_arrive();      // done with the others' shared memory
    if (n) {
        T* y = static_cast<T*>(a.out) + first;
        float m[E], s[E], b[E];
        load_shared<E>(m, mean + ch);
        load_shared<E>(s, scale + ch);
        load_shared<E>(b, shift + ch);
#pragma unroll 2
        for (int i = 0; i < n; ++i, y += step) {
            float v[E];
            get<T, E>(slot[i * N], v);
            sub<E>(v, v, m);
            fma<E>(v, v, s, b);
            store_activated<T, E, SILU>(y, v, a.relu);
        }
    }
    if (a.chunks > 1) cluster_wait();
}

// With SiLU, dz of the first pass is kept for the second, in the place of dy (and, of 16 bits, in as much again): to compute it again would
// take the special function unit longer than memory takes for the rest.
template <typename T, int E, bool SILU>
__global__ void __launch_bounds__(kThreads, 6) norm_back_kernel(const Args a)
{
    extern __shared__ __align__(16) float red[];      // 2 E floats per thread; per channel; slots of x, of dy or dz
    __shared__ float2 own[kMaxSpanGroups];             // the block's sums of gamma dz and gamma dz xh
    const Place<E, kThreads> at(a);
    float* const mean = red + 2 * E * kThreads;
    float* const rstd = mean + a.span_ch;
    float* const gamma = rstd + a.span_ch;
    float* const beta = gamma + a.span_ch;
    float* const sums = beta + a.span_ch;              // the block's, two per channel
    raw_t<T, E>* const slot = reinterpret_cast<raw_t<T, E>*>(sums + 2 * a.span_ch) + threadIdx.x;
    raw_t<T, E>* const dslot = slot + a.loads * kThreads;
    // dz: E floats, the first half where dy is (16 bits)
    raw_t<T, E>* const dslot2 = dslot + a.loads * kThreads;
    const int ch = at.v * E, lane = threadIdx.x & 31;
    let_next_start();
    wait_for_previous();
    const size_t first = ((size_t)at.img * a.hw + at.p0 + at.r) * a.c + at.ch0 + ch, step = (size_t)at.rows * a.c;
    const int n = at.loads;
    fetch<T, E, kThreads>(slot, static_cast<const T*>(a.x) + first, step, n);
    fetch<T, E, kThreads>(dslot, static_cast<const T*>(a.dy) + first, step, n);
    for (int i = threadIdx.x; i < at.nch; i += kThreads) {
        const size_t g = (size_t)at.img * a.groups + at.span * a.gs + over(i, a.cdiv);
        mean[i] = a.mean[g];
        rstd[i] = a.rstd[g];
        gamma[i] = a.gamma ? a.gamma[at.ch0 + i] : 1.0f;
        beta[i] = a.beta ? a.beta[at.ch0 + i] : 0.0f;
    }
    __syncthreads();
    float m[E], g[E], b[E], u[E], w[E];
    if (n) {
        load_shared<E>(m, mean + ch);
        load_shared<E>(g, gamma + ch);
        load_shared<E>(u, rstd + ch);
        load_shared<E>(b, beta + ch);
        mul<E>(g, g, u);
    }
    set<E>(u, 0.0f);
    set<E>(w, 0.0f);
    fetched();
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        float v[E], d[E], z[E];
        get<T, E>(slot[i * kThreads], v);
        get<T, E>(dslot[i * kThreads], d);
        sub<E>(v, v, m);
        fma<E>(z, v, g, b);
        activate_back<SILU, E>(d, z, a.relu);
        add<E>(u, u, d);
        fma<E>(w, d, v, w);      // (times rstd below)
        if constexpr (SILU) put_dz<T, E>(dslot + i * kThreads, dslot2 + i * kThreads, d);
    }
    sum_channels<kThreads, E>(at, u, w, red, sums);
    for (int i = threadIdx.x; i < at.nch; i += kThreads) {
        float* const to = a.sums + ((size_t)at.img * a.chunks + at.rank) * 2 * a.c + at.ch0 + i;
        to[0] = sums[i];
        to[a.c] = times_rstd(sums[at.nch + i], rstd[i]);
    }
    weigh<kThreads, E>(at, a, gamma, rstd, sums, own);
    if (a.chunks > 1) cluster_sync();
    else __syncthreads();
    const float inv = 1.0f / ((float)a.hw * a.cg);
    for (int i = threadIdx.x; i - lane < at.ng * a.chunks; i += kThreads) {
        const int q = min(over(i, a.chdiv), at.ng - 1), k = i & (a.chunks - 1);
        const float2 o = a.chunks > 1 ? ld_rank(own + q, k) : own[q];
        const float r = rstd[q * a.cg];
        const float s1 = lanes_sum(o.x, a.chunks) * inv * -r, s2 = lanes_sum(o.y, a.chunks) * inv * -r * r;
        if (i < at.ng * a.chunks)
            for (int j = k; j < a.cg; j += a.chunks) { red[q * a.cg + j] = s1; red[at.nch + q * a.cg + j] = s2; }
    }
    __syncthreads();
    if (a.chunks > 1) cluster_arrive();
    if (n) {      // dx = (rstd gamma) dz - rstd k1 - (rstd^2 k2) (x - mean)
        T* dx = static_cast<T*>(a.out) + first;
        load_shared<E>(u, red + ch);
        load_shared<E>(w, red + at.nch + ch);
#pragma unroll 2
        for (int i = 0; i < n; ++i, dx += step) {
            float v[E], d[E];
            get<T, E>(slot[i * kThreads], v);
            sub<E>(v, v, m);
            if constexpr (SILU) {
                get_dz<T, E>(dslot + i * kThreads, dslot2 + i * kThreads, d);
            } else {
                get<T, E>(dslot[i * kThreads], d);
                if (a.relu) {
                    float z[E];
                    fma<E>(z, v, g, b);
                    activate_back<false, E>(d, z, true);
                }
            }
            fma<E>(v, v, w, u);
            fma<E>(v, d, g, v);
            store<T, E>(dx, v);
        }
    }
    if (a.chunks > 1) cluster_wait();
}

// ---------------------------------------------------------------------------------------------
// Two passes: the sums of chunks of pixels, and the outputs from a second reading.  A block has a chunk of pixels and a span of as many groups as it
// has threads for (a thread has all pixels of a column of loads, or every rows-th).

// gamma, beta, mean and rstd of a thread's channels, of a span's first channel on
template <int E>
__device__ __forceinline__ void channels(const Args& a, int ch0, int ch, const float* mean, const float* rstd, float (&m)[E], float (&r)[E], float (&g)[E], float (&b)[E])
{
    int q = over(ch, a.cdiv), next = (q + 1) * a.cg - ch;      // the group, and the channels left in it
#pragma unroll
    for (int j = 0; j < E; ++j) {
        if (j == next) { ++q; next += a.cg; }
        m[j] = mean[q];
        r[j] = rstd[q];
        g[j] = a.gamma ? a.gamma[ch0 + ch + j] : 1.0f;
        b[j] = a.beta ? a.beta[ch0 + ch + j] : 0.0f;
    }
}

// A thread's column of n loads, D of them on their way to its slots of shared memory [D][thread]: for a kernel that keeps no more of what it reads, registers
// would hold too few loads in flight.  Loops are unrolled D times, so that a slot's place is known.
template <typename T, int E, int D>
struct Column {
    raw_t<T, E>* slot;
    const T* next;
    size_t step;
    __device__ __forceinline__ Column(void* ring, const T* x, size_t step_) : slot(static_cast<raw_t<T, E>*>(ring) + threadIdx.x), next(x), step(step_) {}
    __device__ __forceinline__ void ask(int j, bool any)      // the next load, for slot j
    {
        if (any) {
            if constexpr (E * sizeof(T) >= 4) fetch_async<E * (int)sizeof(T)>(slot + j * kSplitThreads, next);
            else slot[j * kSplitThreads] = load<T, E>(next);
        }
        next += step;
    }
    __device__ __forceinline__ const raw_t<T, E>& at(int j) const { return slot[j * kSplitThreads]; }
};
__device__ __forceinline__ void asked() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int D>
__device__ __forceinline__ void wait_oldest() { asm volatile("cp.async.wait_group %0;" ::"n"(D - 1) : "memory"); }
constexpr int kDeep = 8, kDeepBack = 4;      // of one tensor; of x and dy each

// Mean and sum of squared distances from it of a chunk, per group: part[image][chunk][group][2].  A wide span is one group and one chunk's column
// of loads after the other; its threads then unite theirs as if they were channels' of one load.
template <typename T, int E>
__global__ void __launch_bounds__(kSplitThreads, 4) stats_kernel(const Args a)
{
    extern __shared__ __align__(16) float red[];      // 2 E floats per thread; ring
    __shared__ float count[kSplitThreads];
    void* const ring = red + 2 * E * kSplitThreads;
    const Place<E, kSplitThreads> at(a);
    let_next_start();
    wait_for_previous();
    Running<E> stat;
    const bool wide = at.nv > kSplitThreads;
    for (int v = at.v; at.active && v < at.nv; v += kSplitThreads) {
        const T* x = static_cast<const T*>(a.x) + ((size_t)at.img * a.hw + at.p0 + at.r) * a.c + at.ch0 + v * E;
        const size_t step = (size_t)at.rows * a.c;
        const int loads = at.loads;
        Column<T, E, kDeep> col(ring, x, step);
#pragma unroll
        for (int j = 0; j < kDeep; ++j) { col.ask(j, j < loads); asked(); }
        for (int i = 0; i < loads; i += kDeep)
#pragma unroll
            for (int j = 0; j < kDeep; ++j)
                if (i + j < loads) {
                    wait_oldest<kDeep>();
                    float d[E];
                    get<T, E>(col.at(j), d);
                    stat.take(d);
                    col.ask(j, i + j + kDeep < loads);
                    asked();
                }
    }
    float2* const to = reinterpret_cast<float2*>(a.part) + ((size_t)at.img * a.chunks + at.rank) * a.groups + at.span * a.gs;
    if (!wide) {
        unite<kSplitThreads, E>(at, a, stat.n, stat.m, stat.q, red, count, to);
        return;
    }
    // one group: all of the block's values
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float c = stat.n;
#pragma unroll
    for (int j = 1; j < E; ++j) {
        const Union both(c, stat.n);
        both(stat.m[0], stat.q[0], stat.m[j], stat.q[j]);
        c += stat.n;
    }
    for (int o = 1; o < 32; o <<= 1) {
        const float other = __shfl_xor_sync(0xffffffffu, c, o);
        const Union both(c, other);
        both(stat.m[0], stat.q[0], __shfl_xor_sync(0xffffffffu, stat.m[0], o), __shfl_xor_sync(0xffffffffu, stat.q[0], o));
        c += other;
    }
    if (lane == 0) { red[warp] = stat.m[0]; red[32 + warp] = stat.q[0]; count[warp] = c; }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kSplitThreads / 32; ++i) {
            const Union both(c, count[i]);
            both(stat.m[0], stat.q[0], red[i], red[32 + i]);
            c += count[i];
        }
        *to = make_float2(stat.m[0], stat.q[0]);
    }
}

// The union of the chunks' statistics, by every block for its groups, and the outputs.
template <typename T, int E, bool SILU>
__global__ void __launch_bounds__(kSplitThreads, 4) apply_kernel(const Args a)
{
    extern __shared__ __align__(16) float ring[];
    __shared__ float mean[kMaxSpanGroups], rstd[kMaxSpanGroups];
    const Place<E, kSplitThreads> at(a);
    let_next_start();
    wait_for_previous();
    const int lk = lanes_of<kSplitThreads>(at.ng), l = 1 << lk, sub_ = threadIdx.x & (l - 1), mine = threadIdx.x >> lk;
    const float total = (float)a.hw * a.cg;
    for (int g0 = mine; g0 - mine < at.ng; g0 += kSplitThreads >> lk) {
        const int g = min(g0, at.ng - 1);
        const float2* const from = reinterpret_cast<const float2*>(a.part) + (size_t)at.img * a.chunks * a.groups + at.span * a.gs + g;
        float s = 0.0f, var = 0.0f;
        for (int k = sub_; k < a.chunks; k += l) s = fmaf(from[(size_t)k * a.groups].x, (float)pixels_of(a, k) * a.cg / total, s);
        const float m = lanes_sum(s, l);
        for (int k = sub_; k < a.chunks; k += l) {
            const float2 o = from[(size_t)k * a.groups];
            var += fmaf((o.x - m) * (o.x - m), (float)pixels_of(a, k) * a.cg / total, o.y / total);      // (each chunk's share: less than their sum)
        }
        var = lanes_sum(var, l);
        if (sub_ == 0 && g == g0) {
            const float r = 1.0f / sqrtf(var + a.eps);
            mean[g] = m;
            rstd[g] = r;
            const size_t o = (size_t)at.img * a.groups + at.span * a.gs + g;
            if (at.rank == 0 && a.mean) a.mean[o] = m;
            if (at.rank == 0 && a.rstd) a.rstd[o] = r;
        }
    }
    __syncthreads();
    for (int v = at.v; at.active && v < at.nv; v += kSplitThreads) {
        float m[E], r[E], g[E], b[E];
        channels<E>(a, at.ch0, v * E, mean, rstd, m, r, g, b);
        mul<E>(r, r, g);
        size_t first = ((size_t)at.img * a.hw + at.p0 + at.r) * a.c + at.ch0 + v * E;
        const size_t step = (size_t)at.rows * a.c;
        const T* x = static_cast<const T*>(a.x) + first;
        T* y = static_cast<T*>(a.out) + first;
        const int loads = at.loads;
        Column<T, E, kDeep> col(ring, x, step);
#pragma unroll
        for (int j = 0; j < kDeep; ++j) { col.ask(j, j < loads); asked(); }
        for (int i = 0; i < loads; i += kDeep)
#pragma unroll
            for (int j = 0; j < kDeep; ++j)
                if (i + j < loads) {
                    wait_oldest<kDeep>();
                    float f[E];
                    get<T, E>(col.at(j), f);
                    sub<E>(f, f, m);
                    fma<E>(f, f, r, b);
                    store_activated<T, E, SILU>(y, f, a.relu);
                    y += step;
                    col.ask(j, i + j + kDeep < loads);
                    asked();
                }
    }
}

// sum dz and sum dz xh of a chunk, per channel: sums[image][chunk][2][channel]; times gamma, per group: part[image][chunk][group][2].
template <typename T, int E, bool SILU>
__global__ void __launch_bounds__(kSplitThreads, 3) back_stats_kernel(const Args a)
{
    extern __shared__ __align__(16) float red[];      // 2 E floats per thread; rings; per channel: gamma, rstd, two sums
    const Place<E, kSplitThreads> at(a);
    void* const ring = red + 2 * E * kSplitThreads;
    void* const dring = static_cast<raw_t<T, E>*>(ring) + kDeepBack * kSplitThreads;
    float* const gamma = reinterpret_cast<float*>(static_cast<raw_t<T, E>*>(dring) + kDeepBack * kSplitThreads);
    float* const rstd = gamma + a.span_ch;
    float* const sums = rstd + a.span_ch;
    let_next_start();
    wait_for_previous();
    const size_t q0 = (size_t)at.img * a.groups + at.span * a.gs;
    for (int i = threadIdx.x; i < at.nch; i += kSplitThreads) {
        gamma[i] = a.gamma ? a.gamma[at.ch0 + i] : 1.0f;
        rstd[i] = a.rstd[q0 + over(i, a.cdiv)];
    }
    float u[E], w[E];
    set<E>(u, 0.0f);
    set<E>(w, 0.0f);
    const bool wide = at.nv > kSplitThreads;
    for (int v = at.v; at.active && v < at.nv; v += kSplitThreads) {
        float m[E], g[E], b[E];
        channels<E>(a, at.ch0, v * E, a.mean + q0, a.rstd + q0, m, u, g, b);
        mul<E>(g, g, u);
        set<E>(u, 0.0f);
        set<E>(w, 0.0f);
        const size_t first = ((size_t)at.img * a.hw + at.p0 + at.r) * a.c + at.ch0 + v * E, step = (size_t)at.rows * a.c;
        const T* x = static_cast<const T*>(a.x) + first;
        const T* dy = static_cast<const T*>(a.dy) + first;
        const int loads = at.loads;
        Column<T, E, kDeepBack> col(ring, x, step), dcol(dring, dy, step);
#pragma unroll
        for (int j = 0; j < kDeepBack; ++j) { col.ask(j, j < loads); dcol.ask(j, j < loads); asked(); }
        for (int i = 0; i < loads; i += kDeepBack)
#pragma unroll
            for (int j = 0; j < kDeepBack; ++j)
                if (i + j < loads) {
                    wait_oldest<kDeepBack>();
                    float f[E], d[E], z[E];
                    get<T, E>(col.at(j), f);
                    get<T, E>(dcol.at(j), d);
                    sub<E>(f, f, m);
                    if (SILU || a.relu) {
                        fma<E>(z, f, g, b);
                        activate_back<SILU, E>(d, z, a.relu);
                    }
                    add<E>(u, u, d);
                    fma<E>(w, d, f, w);
                    col.ask(j, i + j + kDeepBack < loads);
                    dcol.ask(j, i + j + kDeepBack < loads);
                    asked();
                }
        if (wide) {      // the thread has all of the chunk's pixels
            store_shared<E>(sums + v * E, u);
            store_shared<E>(sums + at.nch + v * E, w);
        }
    }
    if (wide) __syncthreads();
    else sum_channels<kSplitThreads, E>(at, u, w, red, sums);
    float* const to = a.sums + ((size_t)at.img * a.chunks + at.rank) * 2 * a.c + at.ch0;
    for (int i = threadIdx.x; i < at.nch; i += kSplitThreads) {
        to[i] = sums[i];
        to[a.c + i] = times_rstd(sums[at.nch + i], rstd[i]);
    }
    weigh<kSplitThreads, E>(at, a, gamma, rstd, sums, reinterpret_cast<float2*>(a.part) + ((size_t)at.img * a.chunks + at.rank) * a.groups + at.span * a.gs);
}

// dbeta and dgamma: sums[part][2][channel] over the n parts (blocks of images), channels 8 k to 8 k + 7 (32 bytes of a part), N / 8 parts side by side.
template <int N>
__device__ __forceinline__ void sum_params(float* s, const float* sums, float* dgamma, float* dbeta, int n, int c, int k8)
{
    constexpr int kRows = N / 8;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = threadIdx.x & 7, row = threadIdx.x >> 3, ch = k8 * 8 + k;
    float u = 0.0f, w = 0.0f;
    if (ch < c)
#pragma unroll 8
        for (int i = row; i < n; i += kRows) {
            u += sums[(size_t)i * 2 * c + ch];
            w += sums[((size_t)i * 2 + 1) * c + ch];
        }
    s[k * (kRows + 1) + row] = u;
    s[(8 + k) * (kRows + 1) + row] = w;
    __syncthreads();
    for (int j = warp; j < 16; j += N / 32) {
        float t = 0.0f;
#pragma unroll
        for (int r = 0; r < kRows; r += 32) t += s[j * (kRows + 1) + r + lane];
        t = warp_sum(t);
        float* const to = j >> 3 ? dgamma : dbeta;
        const int out = k8 * 8 + (j & 7);
        if (lane == 0 && out < c && to) to[out] = t;
    }
}

// The first blocks sum dgamma and dbeta meanwhile.
template <typename T, int E, bool SILU>
__global__ void __launch_bounds__(kSplitThreads, 3) back_apply_kernel(const Args a)
{
    extern __shared__ __align__(16) float ring[];
    __shared__ float k1[kMaxSpanGroups], k2[kMaxSpanGroups];
    void* const dring = reinterpret_cast<raw_t<T, E>*>(ring) + kDeepBack * kSplitThreads;
    let_next_start();
    wait_for_previous();
    if ((int)blockIdx.x < a.first) {
        sum_params<kSplitThreads>(ring, a.sums, a.dgamma, a.dbeta, a.n * a.chunks, a.c, blockIdx.x);
        return;
    }
    const Place<E, kSplitThreads> at(a);
    const size_t q0 = (size_t)at.img * a.groups + at.span * a.gs;
    const int lk = lanes_of<kSplitThreads>(at.ng), l = 1 << lk, sub_ = threadIdx.x & (l - 1), mine = threadIdx.x >> lk;
    const float inv = 1.0f / ((float)a.hw * a.cg);
    for (int g0 = mine; g0 - mine < at.ng; g0 += kSplitThreads >> lk) {
        const int g = min(g0, at.ng - 1);
        const float2* const from = reinterpret_cast<const float2*>(a.part) + (size_t)at.img * a.chunks * a.groups + at.span * a.gs + g;
        float s1 = 0.0f, s2 = 0.0f;
        for (int k = sub_; k < a.chunks; k += l) {
            const float2 o = from[(size_t)k * a.groups];
            s1 += o.x;
            s2 += o.y;
        }
        s1 = lanes_sum(s1, l);
        s2 = lanes_sum(s2, l);
        if (sub_ == 0 && g == g0) {
            const float r = a.rstd[q0 + g];
            k1[g] = s1 * inv * -r;
            k2[g] = s2 * inv * -r * r;
        }
    }
    __syncthreads();
    for (int v = at.v; at.active && v < at.nv; v += kSplitThreads) {
        float m[E], g[E], b[E], u[E], w[E];
        channels<E>(a, at.ch0, v * E, a.mean + q0, a.rstd + q0, m, u, g, b);
        mul<E>(g, g, u);
        int q = over(v * E, a.cdiv), next = (q + 1) * a.cg - v * E;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (j == next) { ++q; next += a.cg; }
            u[j] = k1[q];
            w[j] = k2[q];
        }
        const size_t first = ((size_t)at.img * a.hw + at.p0 + at.r) * a.c + at.ch0 + v * E, step = (size_t)at.rows * a.c;
        const T* x = static_cast<const T*>(a.x) + first;
        const T* dy = static_cast<const T*>(a.dy) + first;
        T* dx = static_cast<T*>(a.out) + first;
        const int loads = at.loads;
        Column<T, E, kDeepBack> col(ring, x, step), dcol(dring, dy, step);
#pragma unroll
        for (int j = 0; j < kDeepBack; ++j) { col.ask(j, j < loads); dcol.ask(j, j < loads); asked(); }
        for (int i = 0; i < loads; i += kDeepBack)
#pragma unroll
            for (int j = 0; j < kDeepBack; ++j)
                if (i + j < loads) {
                    wait_oldest<kDeepBack>();
                    float f[E], d[E], z[E];
                    get<T, E>(col.at(j), f);
                    get<T, E>(dcol.at(j), d);
                    sub<E>(f, f, m);
                    if (SILU || a.relu) {
                        fma<E>(z, f, g, b);
                        activate_back<SILU, E>(d, z, a.relu);
                    }
                    fma<E>(f, f, w, u);
                    fma<E>(f, d, g, f);
                    store<T, E>(dx, f);
                    dx += step;
                    col.ask(j, i + j + kDeepBack < loads);
                    dcol.ask(j, i + j + kDeepBack < loads);
                    asked();
                }
    }
}

__global__ void __launch_bounds__(1024) params_kernel(const float* sums, float* dgamma, float* dbeta, int n, int c)
{
    __shared__ float s[2 * 8 * (1024 / 8 + 1)];
    let_next_start();
    wait_for_previous();
    sum_params<1024>(s, sums, dgamma, dbeta, n, c, blockIdx.x);
}

// ---------------------------------------------------------------------------------------------
// Host

struct NormPlan {
    int e;                     // elements per load
    int gs, chunk, loads;
    int threads;               // of a block
    int cluster;               // one pass: blocks of a cluster; 0: two passes
    int chunks;                // blocks per (span, image)
    size_t smem, ring;         // shared memory of the (first) kernel; two passes: of the second
};

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

// One pass with blocks of `threads`: the span and cluster of the smallest estimate, in microseconds.  A block's loads and sums take an SM's issue slots (the more
// warps are there, the better they are filled), but no less than their latencies; memory is idle meanwhile as far as all blocks are at the same; spans that
// are parts of sectors cost memory time.  Fitted to sweeps of six shapes, from 4x14x14x512 (8 to 12 us) to 32x112x112x64 (55 to 75): within 15 % of the
// best of each.
struct OnePass {
    NormPlan plan;
    int resident;              // blocks an SM has room for
    double per_sm;             // blocks of the call per SM
    double us = 0;             // 0: no span fits
};
OnePass one_pass(int threads, NormPlan p, int n, int hw, int c, int groups, int gs0, int elt, bool back, bool silu, int sms)
{
    OnePass best = {};
    const int cg = c / groups;
    p.threads = threads;
    for (int gs = gs0;; gs *= 2) {
        const long long nv = (long long)gs * cg / p.e, nch = up_div((long long)gs * cg, 4) * 4;
        if (gs > kMaxSpanGroups || gs > std::max(gs0, groups) || nv > kThreads) break;
        const int rows = (int)(threads / nv), bytes = gs * cg * elt;
        for (int cluster = 1; cluster <= kMaxCluster; cluster *= 2) {
            const int chunk = (int)up_div(hw, cluster), loads = (int)up_div(chunk, rows);
            if (cluster > 1 && up_div(hw, chunk) <= cluster / 2) break;
            const int slots = !back ? 1 : silu && elt == 2 ? 3 : 2;
            const size_t smem = (size_t)threads * p.e * 8 + (back ? 6 : 3) * nch * 4 + (size_t)loads * slots * threads * p.e * elt;
            if (smem > 200 * 1024) continue;
            const int resident = std::min<int>(back ? 6 : kMostThreads / threads, (int)(225 * 1024 / (smem + 1024)));
            const double per_sm = (double)n * up_div(groups, gs) * cluster / sms, at_once = std::min((double)resident, std::max(1.0, per_sm));
            const double per_load = 0.015 + p.e * (back ? (silu ? 0.017 : 0.010) : silu ? 0.0085 : 0.0065);
            const double latency = 2.5 + 0.1 * loads + (cluster > 1 ? 1.5 : 0) + (cluster > 8 ? 1.5 : 0);
            const double times = (double)threads / kThreads, warps = at_once * times;      // (in units of kThreads)
            const double slots_time = per_sm * (1 + loads * per_load) * times * (warps >= 6 ? 1 : warps >= 4 ? 1.15 : 1.4);
            const double memory = (double)n * hw * c * elt * (back ? 3 : 2) / 6.2e6 * (bytes >= 64 ? 1 : bytes >= 32 ? 1.25 : 2) * (per_sm > 2 * at_once ? 0.6 : 1);
            const double us = std::max(slots_time, std::ceil(per_sm / at_once) * latency) + memory;
            if (best.us == 0 || us < best.us) {
                p.gs = gs; p.cluster = p.chunks = cluster; p.chunk = chunk; p.loads = loads; p.smem = smem;
                best = {p, resident, per_sm, us};
            }
        }
    }
    return best;
}

NormPlan make_plan(int n, int hw, int c, int groups, int elt, int align, bool back, bool silu, int sms)
{
    NormPlan p = {};
    const int cg = c / groups;
    for (p.e = 16 / elt; p.e > 1 && (c % p.e || align % (p.e * elt)); p.e /= 2) {}      // elements of a load
    int gs0 = p.e / gcd(p.e, cg);                       // groups whose channels are whole loads
    // The backward pass holds x, dy and, with SiLU, dz: few blocks per SM.  Large calls, which keep the memory busy either way, are faster in two passes
    // (64 images of 56x56x256, SiLU: 162 us in one pass, 106 in two; 32 of 28x28x256: 18 and 25).
    if (!back || (long long)n * hw * c * elt <= (32 << 20)) {
        const OnePass one = one_pass(kThreads, p, n, hw, c, groups, gs0, elt, back, silu, sms);
        // Blocks of twice the threads have the same shared memory and more warps: where an SM has room for three blocks or fewer and there are several rounds of
        // them (64x56x56x256 bf16 with SiLU: 66 us, so 58; 128x28x28x512: 59 and 51; 64x28x28x256 fp32: 29 and 24), or not a block for every SM
        // (1x224x224x64: 20 and 12).  With more blocks per SM, or one round, their sums cost more than that gives (16x56x56x256 fp32: 27 and 29;
        // 16x112x112x64 bf16: 20 and 24).
        if (one.us > 0 && !back && ((one.resident <= 3 && one.per_sm > 2 * one.resident) || (one.per_sm <= 1 && one.plan.loads > 16))) {
            const OnePass two = one_pass(2 * kThreads, p, n, hw, c, groups, gs0, elt, back, silu, sms);
            if (two.us > 0) return two.plan;
        }
        if (one.us > 0) return one.plan;
    }
    // Two passes.  A span of more loads than threads has to be one group.
    p.threads = kSplitThreads;
    if ((long long)gs0 * cg / p.e > kSplitThreads && gs0 > 1) { p.e = 1; gs0 = 1; }
    p.gs = gs0;
    while (p.gs * 2 <= std::min(kMaxSpanGroups, groups) && (long long)p.gs * 2 * cg / p.e <= kSplitThreads) p.gs *= 2;
    const long long units = (long long)n * up_div(groups, p.gs);
    const long long nv = (long long)p.gs * cg / p.e, rows = std::max<long long>(1, kSplitThreads / nv);
    // Long columns of a thread's loads, as far as every SM has work.
    const long long loads = std::max(4ll, std::min(32ll, up_div(up_div(hw, rows) * units, 4ll * sms)));
    p.chunks = (int)std::min(up_div(hw, rows * loads), 4096ll);
    p.chunk = (int)up_div(hw, p.chunks);
    p.chunks = (int)up_div(hw, p.chunk);
    p.ring = (size_t)kSplitThreads * p.e * elt * (back ? 2 * kDeepBack : kDeep);
    p.smem = ((size_t)kSplitThreads * p.e * 2 + (back ? 4 * up_div((long long)p.gs * cg, 4) * 4 : 0)) * 4 + p.ring;
    return p;
}

// Of the caller's workspace, in floats: sums [n][blocks of an image][2][c] (backward); two passes: part [n][blocks of an image][groups][2].
struct Workspace {
    size_t sums, part;
    size_t bytes() const { return (sums + part) * 4; }
};
Workspace workspace_of(const NormPlan& p, bool back, int n, int c, int groups)
{
    Workspace w = {};
    if (back) w.sums = (size_t)n * p.chunks * 2 * c;
    if (!p.cluster) w.part = (size_t)n * p.chunks * 2 * groups;
    return w;
}

int check_shape(int n, int h, int wd, int c, int groups)
{
    if (n < 0 || h < 0 || wd < 0 || c < 0 || groups < 1) return ALCS_ERR_INVALID_ARG;
    if (c % groups || c > 65536 || (long long)h * wd >= (1ll << 30) || (long long)n * c >= (1ll << 30)) return ALCS_ERR_SHAPE;
    return c / groups > kMaxGroupChannels ? ALCS_ERR_UNSUPPORTED : ALCS_OK;
}

using Kernel = void (*)(const Args);
// which: 0 one pass, 1 statistics, 2 outputs
template <typename T, int E>
Kernel kernel_of(bool back, int which, bool silu, int threads)
{
    if (which == 0 && !back && threads > kThreads) return silu ? norm_kernel<T, E, true, 2 * kThreads> : norm_kernel<T, E, false, 2 * kThreads>;
    if (which == 0) return back ? (silu ? norm_back_kernel<T, E, true> : norm_back_kernel<T, E, false>) : silu ? norm_kernel<T, E, true, kThreads> : norm_kernel<T, E, false, kThreads>;
    if (which == 1) return back ? (silu ? back_stats_kernel<T, E, true> : back_stats_kernel<T, E, false>) : stats_kernel<T, E>;
    return back ? (silu ? back_apply_kernel<T, E, true> : back_apply_kernel<T, E, false>) : silu ? apply_kernel<T, E, true> : apply_kernel<T, E, false>;
}
template <typename T>
Kernel kernel_of(int e, bool back, int which, bool silu, int threads)
{
    if (e == 1) return kernel_of<T, 1>(back, which, silu, threads);
    if (e == 2) return kernel_of<T, 2>(back, which, silu, threads);
    if constexpr (sizeof(T) == 2) {
        if (e == 4) return kernel_of<T, 4>(back, which, silu, threads);
        return kernel_of<T, 8>(back, which, silu, threads);
    } else {
        return kernel_of<T, 4>(back, which, silu, threads);
    }
}
Kernel kernel_of(alcs_dtype dt, const NormPlan& p, bool back, int which, bool silu)
{
    return dt == ALCS_F32 ? kernel_of<float>(p.e, back, which, silu, p.threads) : dt == ALCS_F16 ? kernel_of<__half>(p.e, back, which, silu, p.threads)
                                                                                        : kernel_of<__nv_bfloat16>(p.e, back, which, silu, p.threads);
}

int align_of(std::initializer_list<const void*> ps)
{
    int align = 16;
    for (const void* p : ps)
        while ((uintptr_t)p % align) align /= 2;
    return align;
}

// Shared memory beyond 48 KB (with a kernel's own) and clusters of 16, allowed once per kernel and device.
int allow(const void* fn, size_t smem, int cluster, int dev)
try {
    static std::mutex mu;
    static std::set<std::pair<const void*, int>> allowed;
    if (smem <= 40 * 1024 && cluster <= 8) return ALCS_OK;
    std::lock_guard<std::mutex> lk(mu);
    if (allowed.count({fn, dev})) return ALCS_OK;
    ALCS_CUDA(cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024));
    ALCS_CUDA(cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    allowed.insert({fn, dev});
    return ALCS_OK;
} catch (const std::exception&) {      // no memory for an entry
    return ALCS_ERR_ALLOC;
}

int run(Args& a, bool back, alcs_dtype dt, int dev, const NormPlan& p, void* workspace, cudaStream_t st)
{
    const Workspace w = workspace_of(p, back, a.n, a.c, a.groups);
    a.sums = static_cast<float*>(workspace);
    a.part = a.sums + w.sums;
    a.gs = p.gs;
    a.spans = (int)up_div(a.groups, p.gs);
    a.chunk = p.chunk;
    a.chunks = p.chunks;
    a.loads = p.loads;
    const long long blocks = (long long)a.n * a.spans * a.chunks;
    if (blocks > 0x7fffffffll) return ALCS_ERR_SHAPE;
    a.span_ch = (int)up_div((long long)a.gs * a.cg, 4) * 4;
    a.whole = a.cg % p.e == 0;
    a.cdiv = tc_div(a.cg);
    a.vdiv = tc_div(std::max(1, a.cg / p.e));
    a.chdiv = tc_div(a.chunks);
    a.spdiv = tc_div(a.spans);
    const int nv = a.gs * a.cg / p.e;
    a.nvdiv = tc_div(nv);
    a.rowdiv = tc_div(std::max(1, p.threads / nv));
    const dim3 grid((unsigned)blocks);
    const Kernel first = kernel_of(dt, p, back, p.cluster ? 0 : 1, a.silu);
    const int rc = allow((const void*)first, p.smem, p.cluster, dev);
    if (rc) return rc;
    ALCS_CUDA(launch_pdl(first, grid, p.threads, p.smem, std::max(1, p.cluster), st, a));
    if (p.cluster) return ALCS_OK;
    if (back && (a.dgamma || a.dbeta)) a.first = (int)up_div(a.c, 8);
    if (blocks + a.first > 0x7fffffffll) return ALCS_ERR_SHAPE;
    ALCS_CUDA(launch_pdl(kernel_of(dt, p, back, 2, a.silu), dim3((unsigned)(blocks + a.first)), kSplitThreads, std::max(p.ring, (size_t)(back ? 16 * (kSplitThreads / 8 + 1) * 4 : 0)),
                         1, st, a));
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
    // (whatever the alignment of the buffers and the activation)
    for (int align : {16, 8, 4, 2})
        for (bool back : {false, true})
            for (bool silu : {false, true}) {
                const NormPlan p = make_plan(n, h * wd, c, groups, (int)elt_bytes(dt), align, back, silu, 148);
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
    const NormPlan p = make_plan(n, hw, c, groups, (int)elt, align_of({x, y}), false, flags & ALCS_SILU, 148);
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
    a.relu = (flags & ALCS_RELU) != 0; a.silu = (flags & ALCS_SILU) != 0;
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
        p = make_plan(n, hw, c, groups, (int)elt, align_of({x, dy, dx}), true, flags & ALCS_SILU, 148);
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
        a.relu = (flags & ALCS_RELU) != 0; a.silu = (flags & ALCS_SILU) != 0;
        a.dgamma = dgamma; a.dbeta = dbeta;
        rc = run(a, true, dt, dev, p, workspace, st);
        if (rc) return rc;
    }
    if ((dgamma || dbeta) && (none || p.cluster))
        ALCS_CUDA(launch_pdl(params_kernel, dim3((unsigned)up_div(c, 8)), 1024, 0, 1, st, static_cast<const float*>(workspace), dgamma, dbeta, none ? 0 : n * p.chunks, c));
    return ALCS_OK;
}

}  // extern "C"
