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
// channels N, and a lane of the epilogue has a pixel.  With few pixels and long rows the roles are swapped (see choose).
// What bounds it, measured with 16384x4096x4096 (bf16): the number of copies, about 117 cycles each whatever their size (2 KB at a time 341 us, 8 KB 172,
// 16 KB 129); the instructions of the one thread that issues the tensor cores' (160 us before their descriptors came down to an addition); then both and
// what is in flight, three stages of 51 KB: 1070 cycles per stage, 512 of them the tensor cores'.  Tiles of 256 x 256 by pairs of blocks (cta_group::2) fetch a
// third less and were slower where one block per tile took 160 us, 177: the hand-shakes of a stage took longer than it.  Few columns: the outputs' way to memory.
// A block has sixteen warps for the epilogue (32 rows x 32 columns of an accumulator each; with eight, 200704x64x256 took 32 us and not 29), one that copies,
// one that multiplies.  Blocks stay and walk over the tiles.  An accumulator has 128 columns, a tile one or two of the three; the epilogue takes them into
// registers before it works on them, so that the next tile starts at once.
// Where the tiles are fewer than SMs and rows are long, a cluster shares a tile: each block multiplies a part of the columns, leaves its
// partial sums in its shared memory, and adds up, in a fixed order, a share of the outputs over all of them.
#include <algorithm>
#include <atomic>

#include "alcs_dense.h"
#include "alcs_tc.cuh"

namespace alcs {
namespace {

constexpr int kEpiWarps = 16, kLoadWarp = 16, kMmaWarp = 17;
constexpr int kThreads = 576;
constexpr int kQuads = 2;                               // a stage: up to so many groups of four blocks of 32 columns
constexpr int kSlots = 3, kSlotCols = 128;              // tensor memory: accumulators of 128 columns, a tile has one or two; then scales, 12 columns per group
constexpr int kMaxStages = 8;
constexpr int kBias = 1024, kHeader = kBias + kEpiWarps * 128, kStaging = 32 * 128;      // shared memory: barriers; per epilogue warp: bias, a 32 x 32 piece of the output
constexpr int kMaxSplit = 8;
constexpr int kScaleBytes = 512;
constexpr int kScaleCols = 512 - kSlots * kSlotCols;

__device__ int g_error;      // see alcs_mx4_status

struct Operand {
    const unsigned char *data, *scales;
    int rows, tiles;            // tiles of 128 rows
};

struct Args {
    Operand a, b;               // rows and columns of a tile
    int blocks, quads;          // blocks of 32 columns as stored (even), groups of four
    int n;                      // columns of a tile: 64, 128, 192, 256, or the only tile's, a multiple of 16
    int tiles;
    TcDiv tiles_b;
    int split, stages;
    int stage_quads, tile_bytes, stage_bytes;      // of a stage: groups; 128 rows of one operand; all
    int cout;                   // of y's row
    int swapped;                // a is the weights
    int relu, vec;              // vec: rows of y (and the residual) are whole 16 bytes
    const float* bias;
    const void* res;
    void* y;
};

// The upper half of all matrix descriptors: groups of 8 rows 128 bytes apart, no swizzle.  The lower half: the address, and blocks of 32 columns 2048 bytes
// apart (K-major: 8 rows x 16 bytes lie together).
constexpr unsigned kDescHigh = 8u | (1u << 14), kDescLow = 128u << 16;
__device__ __forceinline__ void mma_mx4(unsigned d, unsigned a, unsigned b, unsigned idesc, unsigned sa, unsigned sb, unsigned acc)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 a, {%1, %7};\n\tmov.b64 b, {%2, %7};\n\t"
                 "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void scales_to_tmem(unsigned d, unsigned at)
{
    asm volatile("{\n\t.reg .b64 a;\n\tmov.b64 a, {%1, %2};\n\ttcgen05.cp.cta_group::1.32x128b.warpx4 [%0], a;\n\t}" ::"r"(d), "r"(at), "r"(kDescHigh) : "memory");
}
// The address field of a matrix descriptor: 14 bits (in a cluster an address carries the block's rank above them).
__device__ __forceinline__ unsigned field(unsigned addr) { return addr >> 4 & 0x3fffu; }
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

// E2M1 x E2M1 (type 1 each), scales E8M0; N / 8 is at bit 17, M / 128 at bit 27, which two bytes of the scales at bits 4 and 29.
constexpr unsigned kIdesc = (1u << 7) | (1u << 10) | (1u << 23);
constexpr unsigned kSecond = (1u << 5) | (1u << 30);

// A stage's products: scales of `tiles` tiles of rows (0: they are there) to tensor memory, then per 64 columns one or two instructions, whose columns of the
// accumulators are d0 and d1, rows of shared memory b0 and b1, and scales those of the second operand from column `shift` and column 4 on.  One thread issues all
// of it, so what counts is how few instructions that takes: the descriptors' lower halves are all that changes.
template <int PIECES>
__device__ __forceinline__ void multiply_stage(unsigned a, unsigned b0, unsigned b1, unsigned scales, int Q, int quads, int blocks, unsigned tmem, unsigned shift, int tiles,
                                               unsigned d0, unsigned d1, unsigned id0, unsigned id1, unsigned add)
{
    a = kDescLow | field(a);
    b0 = kDescLow | field(b0);
    if (PIECES > 1) b1 = kDescLow | field(b1);
    scales = kDescLow | field(scales);
    const int pitch = Q * (kScaleBytes >> 4);
#pragma unroll
    for (int g = 0; g < kQuads; ++g) {
        if (g >= quads || g >= Q) break;
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < tiles) scales_to_tmem(tmem + 12 * g + 4 * i, scales + i * pitch + g * (kScaleBytes >> 4));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int block = 4 * g + 2 * k;
            if (block >= blocks) break;
            const unsigned step = block * 128;
            mma_mx4(d0, a + step, b0 + step, k ? id0 | kSecond : id0, tmem + 12 * g, tmem + 12 * g + 4 + shift, block > 0 || add);
            if (PIECES > 1) mma_mx4(d1, a + step, b1 + step, k ? id1 | kSecond : id1, tmem + 12 * g, tmem + 12 * g + 8, block > 0 || add);
        }
    }
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
    const unsigned full = base, empty = base + 8 * kMaxStages, acc_full = empty + 8 * kMaxStages, acc_empty = acc_full + 8 * kSlots, drained = acc_empty + 8 * kSlots;
    const unsigned tmem_slot = drained + 8;
    const unsigned staging0 = base + kHeader, stage0 = staging0 + kEpiWarps * kStaging;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = a.stages, n = a.n, Q = a.stage_quads;
    const unsigned halves = n > kSlotCols ? 2 : 1;
    const unsigned rank = a.split > 1 ? cluster_rank() : 0;
    const int first_tile = blockIdx.x / a.split, tile_step = gridDim.x / a.split;
    // this block's share of the columns, in stages
    const int steps_all = Q ? (a.quads + Q - 1) / Q : 0;
    const int q0 = (int)((long long)steps_all * rank / a.split), q1 = (int)((long long)steps_all * (rank + 1) / a.split);

    if (threadIdx.x == 0) {
        for (int i = 0; i < kMaxStages; ++i) { bar_init(full + 8 * i, 1); bar_init(empty + 8 * i, 1); }
        for (int i = 0; i < kSlots; ++i) { bar_init(acc_full + 8 * i, 1); bar_init(acc_empty + 8 * i, kEpiWarps); }
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
#pragma unroll 1
        for (int t = first_tile; t < a.tiles && ok; t += tile_step) {
            const int ta = div_of(t, a.tiles_b), tb = t - ta * a.tiles_b.d;
            // whole tiles of 128 rows of b, one or two: fewer copies are worth more than the rows of neighbours
            const int t0 = tb * a.n >> 7, nt = (min(tb * a.n + a.n, a.b.tiles * 128) - 1 >> 7) - t0 + 1;
            // lanes: the rows of a; of b's tiles; the scales of a; of b's tiles
            const int which = lane <= nt ? 0 : 1, at_tile = lane <= nt ? lane : lane - nt - 1;
            const Operand& op = at_tile == 0 ? a.a : a.b;
            const size_t tile = at_tile == 0 ? ta : t0 + at_tile - 1;
            const unsigned char* from = which ? op.scales + tile * a.quads * kScaleBytes : op.data + tile * a.blocks * 2048;
            const unsigned to = (which ? (unsigned)(a.stage_bytes - 3 * Q * kScaleBytes) + at_tile * Q * kScaleBytes : at_tile * a.tile_bytes) + stage0;
#pragma unroll 1
            for (int q = q0; q < q1 && ok; ++q) {
                const int nb = min(4 * Q, a.blocks - q * 4 * Q), nq = min(Q, a.quads - q * Q);
                ok = __all_sync(0xffffffffu, bar_wait(empty + 8 * stage, ph));
                if (!ok) break;
                const unsigned bar = full + 8 * stage;
                if (lane == 0)
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((unsigned)((1 + nt) * (nb * 2048 + nq * kScaleBytes))) : "memory");
                __syncwarp();
                if (lane < 2 + 2 * nt)
                    bulk_load(to + stage * a.stage_bytes, from + (size_t)q * (which ? Q * kScaleBytes : a.tile_bytes), which ? nq * kScaleBytes : nb * 2048, bar);
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
            unsigned stage = 0, ph = 0, acc = 0, acc_ph = 1;      // (a slot's phase turns when the ring has)
#pragma unroll 1
            for (int t = first_tile; t < a.tiles && ok; t += tile_step) {
                const int tb = t - div_of(t, a.tiles_b) * a.tiles_b.d;
                // the columns that are rows of b's first tile, and of its second
                const unsigned off = (unsigned)(tb * n & 127), n0 = min((unsigned)n, 128 - off);
                const int nt = (min(tb * n + n, a.b.tiles * 128) - 1 >> 7) - (tb * n >> 7) + 1;
                const unsigned n1 = nt > 1 ? n - n0 : 0;
                const unsigned id0 = kIdesc | (1u << 27) | (n0 >> 3) << 17, id1 = kIdesc | (1u << 27) | (n1 >> 3) << 17;
                unsigned d[2], bar[2];
                for (unsigned h = 0; h < halves; ++h) {
                    d[h] = tmem + acc * kSlotCols;
                    bar[h] = acc_full + 8 * acc;
                    ok = ok && bar_wait(acc_empty + 8 * acc, acc_ph);
                    if (++acc == kSlots) { acc = 0; acc_ph ^= 1u; }
                }
#pragma unroll 1
                for (int q = q0; q < q1 && ok; ++q) {
                    ok = bar_wait(full + 8 * stage, ph);
                    if (!ok) break;
                    tc_after();
                    const unsigned at = stage0 + stage * a.stage_bytes, b0 = at + a.tile_bytes + off * 16, to_s = at + a.stage_bytes - 3 * Q * kScaleBytes;
                    const unsigned to = tmem + kSlots * kSlotCols + 12 * stage * Q;
                    const int nq = a.quads - q * Q, nb = a.blocks - q * 4 * Q;
                    if (n1 == 0) {
                        multiply_stage<1>(at, b0, 0, to_s, Q, nq, nb, to, off >> 5, 2, d[0], 0, id0, 0, q > q0);
                    } else if (off == 0) {
                        multiply_stage<2>(at, b0, b0 + a.tile_bytes, to_s, Q, nq, nb, to, 0, 3, d[0], d[1], id0, id1, q > q0);
                    } else {
                        // A tile that starts in the middle of 128 rows: its accumulators' border is not that of the tiles of rows.  64 rows of the first, 64 and 64 of
                        // the second; the scales are there from the first call on.
                        const unsigned id = kIdesc | (1u << 27) | 8u << 17, b1 = at + 2 * a.tile_bytes;
                        multiply_stage<2>(at, b0, b1, to_s, Q, nq, nb, to, 2, 3, d[0], d[0] + 64, id, id, q > q0);
                        multiply_stage<1>(at, b1 + 64 * 16, 0, to_s, Q, nq, nb, to, 6, 0, d[1], 0, id, 0, q > q0);
                    }
                    mma_commit(empty + 8 * stage);
                    if (++stage == (unsigned)S) { stage = 0; ph ^= 1u; }
                }
                if (ok)
                    for (unsigned h = 0; h < halves; ++h) mma_commit(bar[h]);
            }
            if (!ok) {      // gave up: see the MMAs in flight end before tensor memory is given back
                mma_commit(drained);
                (void)bar_wait(drained, 0);
                atomicExch(&g_error, 1);
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, part_of = warp >> 2;      // the tile's rows, and the columns of an accumulator, that are the warp's: 32 each
        const unsigned staging = staging0 + warp * kStaging, bias_at = base + kBias + warp * 128;
        constexpr int W = Pack<T>::n, L = 32 / W;      // elements of a store; lanes of a row, and stores of a piece
        unsigned acc = 0, acc_ph = 0;
#pragma unroll 1
        for (int t = first_tile; t < a.tiles && ok; t += tile_step) {
            const int ta = div_of(t, a.tiles_b), tb = t - ta * a.tiles_b.d;
            if (a.res && a.split == 1 && ta * 128 + quarter * 32 + lane < a.a.rows)      // on its way while the tile is multiplied
                for (int c = tb * n; c < min(tb * n + n, a.cout); c += 128 / (int)sizeof(T))
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const T*>(a.res) + (size_t)(ta * 128 + quarter * 32 + lane) * a.cout + c));
#pragma unroll 1
            for (unsigned h = 0; h < halves && ok; ++h) {
                const int c0 = tb * n + (int)h * kSlotCols + part_of * 32, end = min(tb * n + n, a.b.rows);
                const float bias = a.bias && a.split == 1 && c0 + lane < end ? a.bias[c0 + lane] : 0.0f;      // of the lane's column
                float v[32];
                ok = __all_sync(0xffffffffu, bar_wait(acc_full + 8 * acc, acc_ph));
                if (!ok) break;
                tc_after();
                tmem_ld32(tmem + acc * kSlotCols + ((unsigned)quarter << 21) + part_of * 32, v);
                tmem_wait_ld(v);
                tc_before();
                __syncwarp();
                if (lane == 0) bar_arrive(acc_empty + 8 * acc);
                if (++acc == kSlots) { acc = 0; acc_ph ^= 1u; }
                if (q0 == q1)      // no columns: nothing was multiplied
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = 0.0f;
                const int row = quarter * 32 + lane;      // of the tile
                if (a.split > 1) {
                    // partial sums to shared memory, where the stages were: swapped [column][128], else [row][n + 1] (no bank twice)
                    float* const part = reinterpret_cast<float*>(smem + (stage0 - base));
                    const int col = (int)h * kSlotCols + part_of * 32;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (col + j < n) part[a.swapped ? (col + j) * 128 + row : row * (n + 1) + col + j] = v[j];
                    continue;
                }
                if (c0 >= end) continue;
                // a lane has a pixel: a piece of 32 channels goes through shared memory, so that neighbouring lanes store neighbouring bytes
                {
                    __syncwarp();
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(bias_at + lane * 4), "f"(bias) : "memory");
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(staging + lane * 128 + ((j ^ (lane & 7)) << 4)), "f"(v[4 * j]), "f"(v[4 * j + 1]),
                                     "f"(v[4 * j + 2]), "f"(v[4 * j + 3]) : "memory");
                    __syncwarp();
                    const int r0 = ta * 128 + quarter * 32;      // the piece's first pixel
                    if (a.vec) {
                        const int c = c0 + lane % L * W, most = c < end ? a.a.rows - r0 - lane / L : 0;      // rows from the lane's first on
                        const size_t at = (size_t)(r0 + lane / L) * a.cout + c, step = (size_t)W * a.cout;      // (32 / L = W rows at a time)
                        uint4 res[L];
                        if (a.res)
#pragma unroll
                            for (int k = 0; k < L; ++k)
                                if (k * W < most) res[k] = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.res) + at + k * step);
                        float b[W];
#pragma unroll
                        for (int j = 0; j < W; j += 4)
                            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(b[j]), "=f"(b[j + 1]), "=f"(b[j + 2]), "=f"(b[j + 3])
                                         : "r"(bias_at + (lane % L * W + j) * 4) : "memory");
                        T* y = static_cast<T*>(a.y) + at;
#pragma unroll
                        for (int k = 0; k < L; ++k, y += step) {
                            const int r = k * W + lane / L;
                            float o[W];
#pragma unroll
                            for (int j = 0; j < W; j += 4)
                                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(o[j]), "=f"(o[j + 1]), "=f"(o[j + 2]), "=f"(o[j + 3])
                                             : "r"(staging + r * 128 + (((lane % L * W + j) / 4 ^ (r & 7)) << 4)) : "memory");
                            add<W>(o, o, b);
                            if (a.res) {
                                float x[W];
                                Pack<T>::get(res[k], x);
                                add<W>(o, o, x);
                            }
                            uint4 out = Pack<T>::put(o);
                            if (a.relu) out = positive(out, T());
                            if (k * W < most) *reinterpret_cast<uint4*>(y) = out;
                        }
                    } else {      // a row at a time, a lane per channel
                        const int cl = c0 + lane;
#pragma unroll 4
                        for (int r = 0; r < 32; ++r) {
                            float o;
                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(o) : "r"(staging + r * 128 + ((lane >> 2 ^ (r & 7)) << 4) + (lane & 3) * 4) : "memory");
                            if (r0 + r < a.a.rows && cl < end) store_one<T>(a, (size_t)(r0 + r) * a.cout + cl, o, bias);
                        }
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
        const int ta = div_of(first_tile, a.tiles_b), tb = first_tile - ta * a.tiles_b.d;
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
            store_one<T>(a, (size_t)p * a.cout + c, sum, a.bias ? a.bias[c] : 0.0f);
        }
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

// How a product is cut, `steps` stages long.
// The width of a tile is that for which the busiest block has least to do, a tile costing its columns and about 64 more (6272x256x1024: 192 columns
// 9.7 us, 256 11.0; 1568x2048x512: 64 columns 7.7, 256 10.1).
// A cluster shares a tile, where that gives idle SMs work, if its columns are many: the exchange of partial sums costs 2 to 3 us (256x4096x256: one block per tile
// 11 us, eight 7.8; 196x512x512: 4.2 and 7).  Then up to 64 pixels are the columns of the tiles, whose partial sums are few (1x2048x512: pixels as columns, eight
// blocks per tile, 5.7 us; as rows, one block, 7.0; 1x1024x1000: 5.7 and 5.2).  Clusters of eight: no more than find room on the GPU's parts at once
// (32x2048x2048 in 16 of them: 12.1 us, in clusters of four 7.0).
int blocks_per_tile(long long tiles, int steps, int sms)
{
    for (int split = kMaxSplit; split > 1; split /= 2)
        if (split <= steps && tiles * split <= (split == 8 ? 96 : sms)) return split;
    return 1;
}
Shape choose(int rows, int cout, int steps, int sms)
{
    if (rows <= 64 && steps >= 6) {
        const int split = blocks_per_tile(up_div(cout, 128), steps, sms);
        if (split > 1) return {true, (int)up_div(rows, 16) * 16, split};
    }
    Shape s = {false, 0, 1};
    const long long ta = up_div(rows, 128);
    long long best = 0;
    for (int n : {256, 192, 128, 64}) {
        const int width = (int)std::min<long long>(n, up_div(cout, 16) * 16);      // (the only tile's may be any multiple of 16)
        const long long cost = up_div(ta * up_div(cout, width), sms) * (width + 64);
        if (!s.n || cost < best) { best = cost; s.n = width; }
    }
    if (steps >= 12) s.split = blocks_per_tile(ta * up_div(cout, s.n), steps, sms);
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
    const Shape s = choose(rows, cout, (a.quads + kQuads - 1) / kQuads, sms);
    const Operand ox = {static_cast<const unsigned char*>(x), static_cast<const unsigned char*>(x_scales), rows, (rows + 127) / 128};
    const Operand ow = {static_cast<const unsigned char*>(w), static_cast<const unsigned char*>(w_scales), cout, (cout + 127) / 128};
    a.a = s.swapped ? ow : ox;
    a.b = s.swapped ? ox : ow;
    a.n = s.n;
    a.swapped = s.swapped;
    a.split = s.split;
    const long long tiles_b = up_div(a.b.rows, a.n), tiles = a.a.tiles * tiles_b;
    if (tiles > 0x7fffffffll) return ALCS_ERR_SHAPE;
    a.tiles = (int)tiles;
    a.tiles_b = tc_div((int)tiles_b);
    // A stage: one or two groups of four blocks, the rows of one tile of a and of one or two of b, and their scales.
    a.stage_quads = std::min(kQuads, a.quads);
    a.tile_bytes = std::min(4 * a.stage_quads, a.blocks) * 2048;
    a.stage_bytes = (a.n > 128 ? 3 : 2) * a.tile_bytes + 3 * a.stage_quads * kScaleBytes;
    constexpr int fixed = kHeader + kEpiWarps * kStaging;
    a.stages = a.quads ? std::min({kMaxStages, kScaleCols / (12 * a.stage_quads), (227 * 1024 - fixed) / a.stage_bytes}) : 1;
    const size_t part = a.split > 1 ? (size_t)128 * (a.n + 1) * 4 : 0;      // (takes the place of the stages)
    const size_t smem = fixed + std::max((size_t)a.stages * a.stage_bytes, part);
    a.cout = cout;
    a.relu = (flags & ALCS_RELU) ? 1 : 0;
    a.vec = (size_t)cout * elt % 16 == 0 && (uintptr_t)y % 16 == 0 && (uintptr_t)residual % 16 == 0;
    a.bias = bias;
    a.res = residual;
    a.y = y;
    const int blocks = a.split > 1 ? a.tiles * a.split : std::min(a.tiles, sms);
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return dt == ALCS_F32 ? launch<float>(a, blocks, smem, dev, st) : dt == ALCS_F16 ? launch<__half>(a, blocks, smem, dev, st)
                                                                                     : launch<__nv_bfloat16>(a, blocks, smem, dev, st);
}

ALCS_API int alcs_mx4_status(int* code)
{
    using namespace alcs;
    if (!code) return ALCS_ERR_INVALID_ARG;
    ALCS_CUDA(cudaDeviceSynchronize());
    ALCS_CUDA(cudaMemcpyFromSymbol(code, g_error, sizeof(int)));
    return ALCS_OK;
}

}  // extern "C"
