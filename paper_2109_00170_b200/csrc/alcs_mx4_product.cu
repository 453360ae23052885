// Product of two microscaled 4-bit matrices on the fifth-generation tensor cores, sm_100a:
//     y[r][o] = act( sum_c x[r][c] w[o][c] + bias[o] + residual[r][o] ).
//
// tcgen05.mma of kind::mxf4 multiplies 64 columns of E2M1 values at a time and applies the scales (one E8M0 byte per 32
// columns and row, in tensor memory) to the products before it adds them in fp32.  The storage format (include/alcs.h) is the
// order in which shared memory has to hold the operands: a block of 32 columns is 16 bytes per row, rows one after
// the other (K-major, no swizzle: 8 rows x 16 bytes are a core matrix), so that a stage is fetched by a few bulk copies of whole
// runs; 128 rows x 4 blocks of scales are the 512 bytes that one tcgen05.cp spreads over the four lane quarters.
//
// One operand's 128 rows are the rows of a tile (M), `n` rows of the other its columns (N).  Usually pixels are M and output
// channels N, and a lane of the epilogue has a pixel.  With few pixels the roles are swapped: a tile of 128 channels times 16 pixels
// costs the tensor cores an eighth of one of 128 pixels.
// A block of 320 threads: eight warps for the epilogue (two per lane quarter, which take the columns by turns of 32), one that copies, one that
// multiplies.  Blocks stay and walk over the tiles; the accumulator's 384 columns hold as many tiles as fit, and the epilogue takes a tile into
// registers before it works on it, so that the next one can start.
// Where the tiles are fewer than SMs and rows are long, a cluster shares a tile: each block multiplies a part of the columns, leaves its
// partial sums in its shared memory, and adds up, in a fixed order, a share of the outputs over all of them.
#include <algorithm>
#include <atomic>

#include "alcs_dense.h"
#include "alcs_tc.cuh"

namespace alcs {
namespace {

constexpr int kEpiWarps = 8, kLoadWarp = 8, kMmaWarp = 9;
constexpr int kThreads = 320;
constexpr int kStageBlocks = 4;                         // blocks of 32 columns per stage: one group of scales
constexpr int kMaxN = 256, kAccCols = 384;              // tensor memory: accumulators, then 12 columns of scales per stage
constexpr int kMaxStages = 8;
constexpr int kHeader = 1024, kStaging = 32 * 128;      // shared memory: barriers; a 32 x 32 piece of the output per epilogue warp
constexpr int kMaxSplit = 8;
constexpr int kScaleBytes = 512;
static_assert(kAccCols + 12 * kMaxStages <= 512, "tensor memory");

__device__ int g_error;      // see alcs_dense_status

struct Operand {
    const unsigned char *data, *scales;
    int rows, tiles;            // tiles of 128 rows
};

struct Args {
    Operand a, b;               // rows and columns of a tile
    int blocks, quads;          // blocks of 32 columns as stored (even), groups of four
    int n;                      // columns of a tile: 64, 128, 192, 256, or the only tile's, a multiple of 16
    int tiles_b;
    long long tiles;
    int split, stages, stage_bytes;
    int cout;                   // of y's row
    int swapped;                // a is the weights
    int relu, vec;              // vec: rows of y (and the residual) are whole 16 bytes
    const float* bias;
    const void* res;
    void* y;
};

__device__ __forceinline__ void mma_mx4(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned sa, unsigned sb, unsigned acc)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
}
__device__ __forceinline__ void scales_to_tmem(unsigned d, unsigned long long desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(d), "l"(desc) : "memory");
}
// The address field of a matrix descriptor: 14 bits (in a cluster an address carries the block's rank above them).
__device__ __forceinline__ unsigned field(unsigned addr) { return addr >> 4 & 0x3fffu; }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ unsigned cluster_rank()
{
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ float ld_rank(unsigned addr, unsigned rank)      // of another block's shared memory
{
    unsigned at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

template <typename T>
__device__ __forceinline__ void store_one(const Args& a, size_t at, float v, float bias)
{
    v += bias;
    if (a.res) v += to_f32(static_cast<const T*>(a.res)[at]);
    if (a.relu) v = fmaxf(v, 0.0f);
    from_f32(static_cast<T*>(a.y) + at, v);
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 1) mx4_kernel(const Args a)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    const unsigned base = smem_u32(smem);
    const unsigned full = base, empty = base + 8 * kMaxStages, acc_full = empty + 8 * kMaxStages, acc_empty = acc_full + 8 * 8, drained = acc_empty + 8 * 8;
    const unsigned tmem_slot = drained + 8;
    const unsigned staging0 = base + kHeader, stage0 = staging0 + kEpiWarps * kStaging;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = a.stages, n = a.n, n_acc = min(8, kAccCols / ((n + 31) / 32 * 32));
    const unsigned acc_cols = (unsigned)((n + 31) / 32 * 32);
    const unsigned rank = a.split > 1 ? cluster_rank() : 0;
    const long long first_tile = blockIdx.x / a.split, tile_step = gridDim.x / a.split;
    // this block's share of the columns, in groups of four blocks
    const int q0 = (int)((long long)a.quads * rank / a.split), q1 = (int)((long long)a.quads * (rank + 1) / a.split);

    if (threadIdx.x == 0) {
        for (int i = 0; i < kMaxStages; ++i) { bar_init(full + 8 * i, 1); bar_init(empty + 8 * i, 1); }
        for (int i = 0; i < 8; ++i) { bar_init(acc_full + 8 * i, 1); bar_init(acc_empty + 8 * i, kEpiWarps); }
        bar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tmem_slot) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_before();
    __syncthreads();
    tc_after();
    unsigned tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot));
    let_next_start();
    wait_for_previous();

    bool ok = true;
    if (warp == kLoadWarp) {
        unsigned stage = 0, ph = 1, used = 0;
        const int pitch = n * 16;      // bytes of a block's rows of b in shared memory
#pragma unroll 1
        for (long long t = first_tile; t < a.tiles && ok; t += tile_step) {
            const int ta = (int)(t / a.tiles_b), tb = (int)(t - (long long)ta * a.tiles_b);
            const int r0 = tb * n, r1 = min(r0 + n, a.b.tiles * 128);      // rows of b that exist (those behind b.rows hold anything)
            const int t0 = r0 >> 7, nt = (r1 - 1 >> 7) - t0 + 1;           // its tiles of 128 rows: 1 to 3
#pragma unroll 1
            for (int q = q0; q < q1 && ok; ++q) {
                const int nb = min(kStageBlocks, a.blocks - q * kStageBlocks);
                ok = __all_sync(0xffffffffu, bar_wait(empty + 8 * stage, ph));
                if (!ok) break;
                const unsigned bar = full + 8 * stage, at = stage0 + stage * a.stage_bytes;
                if (lane == 0)
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;"
                                 ::"r"(bar), "r"((unsigned)(nb * (2048 + (r1 - r0) * 16) + (1 + nt) * kScaleBytes)) : "memory");
                __syncwarp();
                // lanes 0 .. 11: rows of b; then the rows of a, the scales of both
                const unsigned to_b = at + 8192, to_s = to_b + kStageBlocks * pitch;
                if (lane < 12) {
                    const int b = lane & 3, i = lane >> 2;
                    const int s0 = max(r0, (t0 + i) * 128), s1 = min(r1, (t0 + i + 1) * 128);
                    if (b < nb && s0 < s1)
                        bulk_load(to_b + b * pitch + (s0 - r0) * 16, a.b.data + (((size_t)(t0 + i) * a.blocks + q * kStageBlocks + b) * 128 + (s0 & 127)) * 16,
                                  (unsigned)(s1 - s0) * 16, bar);
                } else if (lane == 12) {
                    bulk_load(at, a.a.data + ((size_t)ta * a.blocks + q * kStageBlocks) * 2048, (unsigned)nb * 2048, bar);
                } else if (lane == 13) {
                    bulk_load(to_s, a.a.scales + ((size_t)ta * a.quads + q) * kScaleBytes, kScaleBytes, bar);
                } else if (lane < 14 + nt) {
                    bulk_load(to_s + (lane - 13) * kScaleBytes, a.b.scales + ((size_t)(t0 + lane - 14) * a.quads + q) * kScaleBytes, kScaleBytes, bar);
                }
                ++used;
                if (++stage == (unsigned)S) { stage = 0; ph ^= 1u; }
            }
        }
        // whoever waits for them may have given up: see the copies in flight land before shared memory goes away
#pragma unroll 1
        for (unsigned i = 0; i < min(used, (unsigned)S); ++i) {
            const unsigned at = (stage + S - 1 - i) % S;
            (void)bar_wait(full + 8 * at, at < stage ? ph ^ 1u : ph);
        }
        if (!ok) atomicExch(&g_error, 2);
    } else if (warp == kMmaWarp) {
        if (elect_one()) {
            unsigned stage = 0, ph = 0, acc = 0, acc_ph = 1;
            // E2M1 x E2M1 (type 1 each), scales E8M0; N / 8 at bit 17, M / 128 at bit 27
            const unsigned idesc = (1u << 7) | (1u << 10) | ((unsigned)(n >> 3) << 17) | (1u << 23) | (1u << 27);
            // K-major, no swizzle: blocks of 32 columns 2048 (b: 16 n) bytes apart, groups of 8 rows 128 bytes
            const unsigned long long da = (128ull << 16) | (8ull << 32) | (1ull << 46), db = ((unsigned long long)n << 16) | (8ull << 32) | (1ull << 46);
            const unsigned long long ds = (8ull << 16) | (8ull << 32) | (1ull << 46);
#pragma unroll 1
            for (long long t = first_tile; t < a.tiles && ok; t += tile_step) {
                const int tb = (int)(t % a.tiles_b);
                const unsigned shift = (unsigned)(tb * n & 127) >> 5;      // where row 0 of the tile stands in its first 128 rows' scales
                const int nt = (min(tb * n + n, a.b.tiles * 128) - 1 >> 7) - (tb * n >> 7) + 1;
                const unsigned d = tmem + acc * acc_cols;
                ok = bar_wait(acc_empty + 8 * acc, acc_ph);
#pragma unroll 1
                for (int q = q0; q < q1 && ok; ++q) {
                    ok = bar_wait(full + 8 * stage, ph);
                    if (!ok) break;
                    tc_after();
                    const unsigned at = stage0 + stage * a.stage_bytes, to_b = at + 8192, to_s = to_b + kStageBlocks * n * 16;
                    const unsigned sa = tmem + kAccCols + 12 * stage, sb = sa + 4;
                    scales_to_tmem(sa, ds | field(to_s));
#pragma unroll 1
                    for (int i = 0; i < nt; ++i) scales_to_tmem(sb + 4 * i, ds | field(to_s + (1 + i) * kScaleBytes));
                    const int steps = min(kStageBlocks, a.blocks - q * kStageBlocks) / 2;
#pragma unroll 1
                    for (int k = 0; k < steps; ++k)      // two blocks each; bits 4 and 29: which bytes of the scales
                        mma_mx4(d, da | field(at + k * 4096), db | field(to_b + k * n * 32), idesc | (unsigned)k << 5 | (unsigned)k << 30, sa, sb + shift, q > q0 || k > 0);
                    mma_commit(empty + 8 * stage);
                    if (++stage == (unsigned)S) { stage = 0; ph ^= 1u; }
                }
                if (ok) mma_commit(acc_full + 8 * acc);
                if (++acc == (unsigned)n_acc) { acc = 0; acc_ph ^= 1u; }
            }
            if (!ok) {      // gave up: see the MMAs in flight end before tensor memory is given back
                mma_commit(drained);
                (void)bar_wait(drained, 0);
                atomicExch(&g_error, 1);
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, half = warp >> 2;
        const unsigned staging = staging0 + warp * kStaging;
        unsigned acc = 0, acc_ph = 0;
#pragma unroll 1
        for (long long t = first_tile; t < a.tiles && ok; t += tile_step) {
            const int ta = (int)(t / a.tiles_b), tb = (int)(t - (long long)ta * a.tiles_b);
            float v[4][32];
            ok = __all_sync(0xffffffffu, bar_wait(acc_full + 8 * acc, acc_ph));
            if (!ok) break;
            tc_after();
            const unsigned from = tmem + acc * acc_cols + ((unsigned)quarter << 21);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((2 * i + half) * 32 < n) tmem_ld32(from + (2 * i + half) * 32, v[i]);
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_wait_ld(v[i]);
            if (q0 == q1)      // no columns: nothing was multiplied
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[i][j] = 0.0f;
            tc_before();
            __syncwarp();
            if (lane == 0) bar_arrive(acc_empty + 8 * acc);
            if (++acc == (unsigned)n_acc) { acc = 0; acc_ph ^= 1u; }
            const int row = quarter * 32 + lane;      // of the tile
            if (a.split > 1) {
                // partial sums to shared memory, where the stages were: swapped [column][128], else [row][n + 1] (no bank twice)
                float* const part = reinterpret_cast<float*>(smem + (stage0 - base));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c0 = (2 * i + half) * 32;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (c0 + j < n) part[a.swapped ? (c0 + j) * 128 + row : row * (n + 1) + c0 + j] = v[i][j];
                }
                break;
            }
            if (a.swapped) {      // a lane has a channel: 32 neighbours of a pixel's row at a time
                const int c = ta * 128 + row;
                if (c < a.a.rows) {
                    const float bias = a.bias ? __ldg(a.bias + c) : 0.0f;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const int p = tb * n + (2 * i + half) * 32 + j;
                            if ((2 * i + half) * 32 + j < n && p < a.b.rows) store_one<T>(a, (size_t)p * a.cout + c, v[i][j], bias);
                        }
                }
                continue;
            }
            // a lane has a pixel: a piece of 32 channels goes through shared memory, so that neighbouring lanes store neighbouring bytes
            constexpr int W = Pack<T>::n, L = 32 / W;      // elements of a store, lanes of a row
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c0 = tb * n + (2 * i + half) * 32, c1 = min(min(c0 + 32, tb * n + n), a.b.rows);
                if (c0 >= c1) continue;
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(staging + lane * 128 + ((j ^ (lane & 7)) << 4)), "f"(v[i][4 * j]), "f"(v[i][4 * j + 1]),
                                 "f"(v[i][4 * j + 2]), "f"(v[i][4 * j + 3]) : "memory");
                __syncwarp();
                const int c = c0 + lane % L * W;
                if (a.vec) {
                    float bias[W];
#pragma unroll
                    for (int j = 0; j < W; ++j) bias[j] = a.bias && c + j < c1 ? __ldg(a.bias + c + j) : 0.0f;
#pragma unroll
                    for (int k = 0; k < L; ++k) {
                        const int r = k * W + lane / L;      // (32 / L = W rows at a time)
                        const int p = ta * 128 + quarter * 32 + r;
                        float o[W];
#pragma unroll
                        for (int j = 0; j < W; j += 4)
                            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(o[j]), "=f"(o[j + 1]), "=f"(o[j + 2]), "=f"(o[j + 3])
                                         : "r"(staging + r * 128 + (((lane % L * W + j) / 4 ^ (r & 7)) << 4)) : "memory");
                        if (p >= a.a.rows || c >= c1) continue;
                        const size_t at = (size_t)p * a.cout + c;
#pragma unroll
                        for (int j = 0; j < W; ++j) o[j] += bias[j];
                        if (a.res) {
                            float x[W];
                            Pack<T>::get(*reinterpret_cast<const uint4*>(static_cast<const T*>(a.res) + at), x);
#pragma unroll
                            for (int j = 0; j < W; ++j) o[j] += x[j];
                        }
                        if (a.relu)
#pragma unroll
                            for (int j = 0; j < W; ++j) o[j] = fmaxf(o[j], 0.0f);
                        *reinterpret_cast<uint4*>(static_cast<T*>(a.y) + at) = Pack<T>::put(o);
                    }
                } else {      // a row at a time, a lane per channel
                    const int cl = c0 + lane;
                    const float bias = a.bias && cl < c1 ? __ldg(a.bias + cl) : 0.0f;
#pragma unroll 4
                    for (int r = 0; r < 32; ++r) {
                        const int p = ta * 128 + quarter * 32 + r;
                        float o;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(o) : "r"(staging + r * 128 + ((lane >> 2 ^ (r & 7)) << 4) + (lane & 3) * 4) : "memory");
                        if (p < a.a.rows && cl < c1) store_one<T>(a, (size_t)p * a.cout + cl, o, bias);
                    }
                }
            }
        }
        if (!ok && lane == 0) atomicExch(&g_error, 1);
        __syncwarp();
    }
    if (a.split > 1) {
        // (every block gets here, whatever happened; a tile that a block gave up is marked in g_error)
        __syncthreads();
        cluster_arrive();
        cluster_wait();
        const int ta = (int)(first_tile / a.tiles_b), tb = (int)(first_tile % a.tiles_b);
        const unsigned part = stage0;
        const int total = 128 * n, e0 = (int)((long long)total * rank / a.split), e1 = (int)((long long)total * (rank + 1) / a.split);
#pragma unroll 1
        for (int e = e0 + (int)threadIdx.x; e < e1; e += kThreads) {
            const int row = a.swapped ? e & 127 : e / n, col = a.swapped ? e >> 7 : e - row * n;
            const unsigned at = part + 4u * (a.swapped ? col * 128 + row : row * (n + 1) + col);
            float sum = 0.0f;
#pragma unroll
            for (int s = 0; s < kMaxSplit; ++s)
                if (s < a.split) sum += ld_rank(at, s);
            const int ga = ta * 128 + row, gb = tb * n + col;
            if (ga >= a.a.rows || gb >= a.b.rows) continue;
            const int c = a.swapped ? ga : gb, p = a.swapped ? gb : ga;
            store_one<T>(a, (size_t)p * a.cout + c, sum, a.bias ? __ldg(a.bias + c) : 0.0f);
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    tc_before();
    __syncthreads();
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

struct Shape {
    bool swapped;
    int n, split;
};

// How a product is cut.
Shape choose(int rows, int cout, int quads, int sms)
{
    Shape s = {rows <= 64, 0, 1};
    const int mine = s.swapped ? cout : rows, other = s.swapped ? rows : cout;
    const long long ta = up_div(mine, 128);
    s.n = (int)std::min<long long>(kMaxN, up_div(other, 16) * 16);
    if (other > kMaxN || ta * up_div(other, s.n) < sms)
        while (s.n > 64 && ta * up_div(other, s.n) < sms) s.n = s.n > 192 ? 192 : s.n > 128 ? 128 : 64;
    const long long tiles = ta * up_div(other, s.n);
    while (s.split < kMaxSplit && tiles * s.split * 2 <= sms && quads >= s.split * 2) s.split *= 2;
    return s;
}

template <typename T>
int launch(const Args& a, int blocks, size_t smem, int device, cudaStream_t st)
{
    static std::atomic<bool> ready[64];      // (two first calls set the same attribute twice)
    if (device < 0 || device >= 64) return ALCS_ERR_INVALID_ARG;
    if (!ready[device]) {
        ALCS_CUDA(cudaFuncSetAttribute(mx4_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024));
        ready[device] = true;
    }
    ALCS_CUDA(launch_pdl(mx4_kernel<T>, dim3((unsigned)blocks), kThreads, smem, a.split, st, a));
    return ALCS_OK;
}

}  // namespace
}  // namespace alcs

extern "C" {

ALCS_API int alcs_mx4_product(const void* x, const void* x_scales, int rows, const void* w, const void* w_scales, int cout, int cin,
                              void* y, const float* bias, const void* residual, unsigned flags, alcs_dtype dt, void* cuda_stream)
{
    using namespace alcs;
    if (!known_type(dt) || (flags & ~ALCS_RELU)) return ALCS_ERR_INVALID_ARG;
    size_t xd = 0, xs = 0, wd = 0, ws = 0;
    int rc = alcs_mx4_bytes(rows, cin, &xd, &xs);
    if (!rc) rc = alcs_mx4_bytes(cout, cin, &wd, &ws);
    if (rc) return rc;
    if (cout > (1 << 24)) return ALCS_ERR_SHAPE;
    if (rows == 0 || cout == 0) return ALCS_OK;
    const size_t elt = elt_bytes(dt), yb = (size_t)rows * cout * elt;
    const Buffer buffers[7] = {{y, yb, elt, true, false, 1u << 1}, {residual, yb, elt, false, true, 0}, {bias, (size_t)cout * 4, 4, false, true, 0},
                               {x, xd, 16, false, false, 0}, {x_scales, xs, 16, false, false, 0}, {w, wd, 16, false, false, 0},
                               {w_scales, ws, 16, false, false, 0}};
    int dev = 0, sms = 0, optin = 0;
    rc = check_buffers(buffers, &dev);
    if (!rc) rc = device_limits(dev, &sms, &optin);
    if (rc) return rc;
    Args a;
    a.blocks = 2 * ((cin + 63) / 64);
    a.quads = (cin + 127) / 128;
    const Shape s = choose(rows, cout, a.quads, sms);
    const Operand ox = {static_cast<const unsigned char*>(x), static_cast<const unsigned char*>(x_scales), rows, (rows + 127) / 128};
    const Operand ow = {static_cast<const unsigned char*>(w), static_cast<const unsigned char*>(w_scales), cout, (cout + 127) / 128};
    a.a = s.swapped ? ow : ox;
    a.b = s.swapped ? ox : ow;
    a.n = s.n;
    a.swapped = s.swapped;
    a.split = s.split;
    a.tiles_b = (int)up_div(a.b.rows, a.n);
    a.tiles = (long long)a.a.tiles * a.tiles_b;
    if (a.tiles > 0x7fffffffll) return ALCS_ERR_SHAPE;
    a.stage_bytes = 8192 + kStageBlocks * a.n * 16 + 3 * kScaleBytes;
    constexpr int fixed = kHeader + kEpiWarps * kStaging;
    a.stages = std::min(kMaxStages, (227 * 1024 - fixed) / a.stage_bytes);
    const size_t part = a.split > 1 ? (size_t)128 * (a.n + 1) * 4 : 0;      // (takes the place of the stages)
    const size_t smem = fixed + std::max((size_t)a.stages * a.stage_bytes, part);
    a.cout = cout;
    a.relu = (flags & ALCS_RELU) ? 1 : 0;
    a.vec = (size_t)cout * elt % 16 == 0 && (uintptr_t)y % 16 == 0 && (uintptr_t)residual % 16 == 0;
    a.bias = bias;
    a.res = residual;
    a.y = y;
    const int blocks = (int)std::min<long long>(a.tiles * a.split, a.split > 1 ? a.tiles * a.split : sms);
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return dt == ALCS_F32 ? launch<float>(a, blocks, smem, dev, st) : dt == ALCS_F16 ? launch<__half>(a, blocks, smem, dev, st)
                                                                                     : launch<__nv_bfloat16>(a, blocks, smem, dev, st);
}

ALCS_API int alcs_dense_status(int* code)
{
    using namespace alcs;
    if (!code) return ALCS_ERR_INVALID_ARG;
    ALCS_CUDA(cudaMemcpyFromSymbol(code, g_error, sizeof(int)));
    return ALCS_OK;
}

}  // extern "C"
