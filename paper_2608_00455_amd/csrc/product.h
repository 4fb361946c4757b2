// Matrix products on the matrix cores (gfx950), the core of the linear
// cross entropy and of the Newton-Schulz iteration:
//
//   out[j, i] = sum_k A(i, k) * B(j, k)        (out row-major, i contiguous)
//
// with 16-bit operands (BF16 or FP16) and binary32 sums.  Either operand is
// "k-contiguous" (element (r, k) at p[r*ld + k]) or "row-contiguous" (at
// p[k*ld + r]), so a product with any transposed operand needs no copy.
//
// A block owns a tile of TI x TJ outputs and walks k in steps of 64.  Each
// step's operand tiles go straight from memory to LDS (16-byte buffer loads
// with an LDS destination), into the half of a double buffer that the waves
// are not reading.  A wave's outputs stay in registers; it reads fragments
// of 16 rows x 32 k and issues v_mfma_f32_16x16x32.  The i side is the
// instruction's row operand, so a lane ends up with four consecutive i of one
// j: 8- or 16-byte stores, and reductions over i that are nearly all within
// a lane.
//
// LDS images and bank conflicts (64 banks of 4 bytes, 16-byte chunks):
//  - k-contiguous: row r is 128 bytes, chunk c (8 k) at position c ^ (r & 7);
//    a fragment read (16 bytes per lane, ds_read_b128) takes one chunk column
//    of 16 rows, which the exclusive-or spreads over all banks.
//  - row-contiguous: k is a row of 2*TR bytes; chunk c (8 rows) of k at
//    position c ^ 2h(k), h(k) = (k & 3) | (bit 3 of k) << 2; a fragment is
//    read with the transposing ds_read_b64_tr_b16 (each group of 16 lanes
//    turns 4 k x 16 rows), whose 16 k-rows the exclusive-or spreads evenly.
// The exclusive-or is applied to the global address of the load (the LDS side
// of such a load is lane-linear).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

namespace dte {
namespace pr {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

constexpr int kStepK = 64;              // k per step
constexpr int64_t kMaxLd = 1 << 22;     // 256 rows of 2-byte elements stay within 32-bit offsets

// One operand.  rows: valid rows (tiles that reach past them read the last
// one again); kvalid: valid k of a row-contiguous operand (steps that reach
// past read the last one again: the other operand holds zeros there).  A
// k-contiguous operand is readable, and zero on one side, up to the next
// multiple of 64.  wrap > 0: after wrap steps the operand starts over at k = 0.
// stride: elements between the matrices of a batch.
struct Operand {
    const uint16_t* p;
    int64_t ld;
    int64_t stride;
    int32_t rows;
    int32_t kvalid;
    int32_t wrap;
};

struct ProductArgs {
    Operand a, b;
    int32_t ni, nj;        // extents of i and j
    int32_t steps;         // k steps of 64 in all
    int32_t split;         // blocks that share one tile's steps
    int32_t tiles_i, tiles_j;
    int32_t batch;
    int32_t symmetric;     // only tiles with ti <= tj (ni == nj, out symmetric)
};

template <bool kF16>
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c)
{
#ifdef __HIP_DEVICE_COMPILE__
    if constexpr (kF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a),
                                                      __builtin_bit_cast(half8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
#else
    return c;
#endif
}

#define DTE_LDS(T) __attribute__((address_space(3))) T

// LDS address of the launch's dynamic LDS.  Everything here lies in it and is
// addressed from it: the compiler may place arrays of its own before it.
extern __shared__ __attribute__((aligned(1024))) char s_dynamic[];
__device__ __forceinline__ uint32_t lds_base()
{
#ifdef __HIP_DEVICE_COMPILE__
    return (uint32_t)(uintptr_t)(DTE_LDS(char)*)s_dynamic;
#else
    return 0;
#endif
}

// Loads of one operand's tiles to LDS: TR rows x 64 k per step, kThreads
// threads, kLoads 16-byte loads per thread.
template <int TR, int kThreads, bool kKC>
struct TileLoader {
    static constexpr int kLoads = TR * 8 / kThreads;
    static_assert(kLoads * kThreads == TR * 8, "whole loads");
    uint32_t off[kLoads];   // byte offset of each load from `base`
    uint64_t base;          // address of (row0, current k)
    int64_t step;           // bytes per step
    int32_t left;           // steps until the operand starts over (wrap)

    __device__ __forceinline__ void init(const Operand& o, const uint16_t* p, int64_t row0,
                                         int32_t step0)
    {
        const int tid = threadIdx.x;
        const int32_t s0 = o.wrap > 0 ? step0 % o.wrap : step0;
        left = o.wrap > 0 ? o.wrap - s0 : 0x7fffffff;
        if constexpr (kKC) {
            base = (uint64_t)(p + row0 * o.ld + (int64_t)s0 * kStepK);
            step = kStepK * 2;
            const int64_t last = o.rows - 1 - row0;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int q = i * kThreads + tid, row = q >> 3, pos = q & 7;
                const int64_t r = row < last ? row : last;
                off[i] = (uint32_t)(r * o.ld * 2) + ((pos ^ (row & 7)) * 16);
            }
        } else {
            base = (uint64_t)(p + row0 + (int64_t)s0 * kStepK * o.ld);
            step = o.ld * kStepK * 2;
            offsets(o, row0, s0);
        }
    }

    // Row-contiguous: offsets of the step that begins at k = 64 s.
    __device__ __forceinline__ void offsets(const Operand& o, int64_t row0, int32_t s)
    {
        const int tid = threadIdx.x;
        constexpr int kChunks = TR / 8;
        static_assert(kKC || kChunks >= 16, "the exclusive-or needs 16 chunks per row");
        const int last = (int)((o.rows - 1 - row0) >> 3);
        const int klast = o.kvalid - 1 - s * kStepK;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int q = i * kThreads + tid, k = q / kChunks, pos = q % kChunks;
            const int c = pos ^ (2 * ((k & 3) | (((k >> 3) & 1) << 2)));
            off[i] = (uint32_t)((int64_t)(k < klast ? k : klast) * o.ld * 2) +
                     (c < last ? c : last) * 16;
        }
    }

    // Step s into the LDS image at `lds`; afterwards base is at step s + 1.
    __device__ __forceinline__ void issue(const Operand& o, int64_t row0, int32_t s, uint32_t lds,
                                          int wave)
    {
#ifdef __HIP_DEVICE_COMPILE__
        if constexpr (!kKC) {
            if ((int64_t)(s + 1) * kStepK > o.kvalid && o.wrap == 0) offsets(o, row0, s);
        }
        __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0xffffffffu, 0x00020000);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                r, (DTE_LDS(void)*)(uintptr_t)(lds + i * kThreads * 16 + wave * 1024), 16, off[i],
                0, 0, 0);
        base += step;
        if (--left == 0) {
            base -= (int64_t)o.wrap * step;
            left = o.wrap;
        }
#endif
    }
};

// A wave's fragments of one operand: kFrags x 16 rows from row w0 of the tile.
template <int TR, int kFrags, bool kKC>
struct FragReader {
    uint32_t at[kKC ? 2 : kFrags];

    __device__ __forceinline__ void init(int w0)
    {
        const int l = threadIdx.x & 63, j = l & 15, g = l >> 4;
        if constexpr (kKC) {
            at[0] = (w0 + j) * 128 + ((g ^ (l & 7)) * 16);
            at[1] = at[0] ^ 64;
        } else {
            const int h = (j >> 2) | ((g & 1) << 2);
#pragma unroll
            for (int f = 0; f < kFrags; ++f)
                at[f] = (g * 8 + (j >> 2)) * (TR * 2) +
                        (((w0 / 16 + f) ^ h) * 2 + ((j & 3) >> 1)) * 16 + (j & 1) * 8;
        }
    }

    // Fragment f of k half kk (32 k): lane l holds row l & 15, k 8 (l >> 4) + 0..7.
    __device__ __forceinline__ s16x8 read(uint32_t lds, int f, int kk) const
    {
#ifdef __HIP_DEVICE_COMPILE__
        if constexpr (kKC) {
            return *(DTE_LDS(s16x8)*)(uintptr_t)(lds + at[kk] + f * 2048);
        } else {
            const uint32_t p = lds + at[f] + kk * 32 * TR * 2;
            const s16x4 x =
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((DTE_LDS(s16x4)*)(uintptr_t)p);
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (DTE_LDS(s16x4)*)(uintptr_t)(p + 4 * TR * 2));
            return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        }
#else
        return s16x8{};
#endif
    }
};

// A block's tile: which one, and this wave's part of it.
struct TileAt {
    int32_t ti, tj, split, batch;
};

// Blocks are dealt to the eight XCDs in turn (block b to XCD b mod 8); each
// XCD has an L2 of its own.  Give every XCD a contiguous range of the tile
// sequence, and order that sequence in bands of 8 tile rows so that the tiles
// in flight on one XCD share operand rows.
__device__ __forceinline__ TileAt tile_of(const ProductArgs& p, int32_t per_matrix)
{
    const int32_t nb = gridDim.x, x = blockIdx.x & 7, q = nb >> 3, r = nb & 7;
    int32_t t = x * q + (x < r ? x : r) + (blockIdx.x >> 3);
    TileAt at;
    at.batch = t / per_matrix;
    t -= at.batch * per_matrix;
    const int32_t tiles = per_matrix / p.split;
    at.split = t / tiles;
    t -= at.split * tiles;
    if (p.symmetric) {
        int32_t j = (int32_t)((__builtin_amdgcn_sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while (j * (j + 1) / 2 > t) --j;
        while ((j + 1) * (j + 2) / 2 <= t) ++j;
        at.tj = j;
        at.ti = t - j * (j + 1) / 2;
    } else {
        constexpr int32_t kBand = 8;
        const int32_t band = t / (kBand * p.tiles_j), in = t - band * kBand * p.tiles_j;
        const int32_t rows = min(kBand, p.tiles_i - band * kBand);
        at.ti = band * kBand + in % rows;
        at.tj = in / rows;
    }
    return at;
}

// Tile shapes: kWI x kWJ waves, each with (TI / kWI) x (TJ / kWJ) outputs.
template <int kTI, int kTJ, int kWI_, int kWJ_>
struct Shape {
    static constexpr int TI = kTI, TJ = kTJ, kWI = kWI_, kWJ = kWJ_;
    static constexpr int kThreads = kWI * kWJ * 64;
    static constexpr int FI = kTI / kWI / 16, FJ = kTJ / kWJ / 16;
    static constexpr uint32_t kStageBytes = (kTI + kTJ) * kStepK * 2;
    static constexpr uint32_t kLds = 2 * kStageBytes;
};
typedef Shape<256, 256, 2, 4> Large;     // one block per CU
typedef Shape<128, 128, 2, 2> Medium;    // two blocks per CU
typedef Shape<256, 64, 4, 1> Thin64;     // few j: the i operand streams past
typedef Shape<256, 32, 4, 1> Thin32;

// The k loop.  On return the block's waves have left the loop together and no
// LDS load is in flight, so the epilogue may use all of the LDS.
template <class S, bool kF16, bool kAK, bool kBK>
__device__ __forceinline__ void tile_product(const ProductArgs& p, const TileAt& at, int wave,
                                             f32x4 (&acc)[S::FI][S::FJ])
{
    constexpr uint32_t kStage = S::kStageBytes, kB = S::TI * kStepK * 2;
    const int32_t per = (p.steps + p.split - 1) / p.split;
    const int32_t s0 = at.split * per, s1 = min(p.steps, s0 + per);
#pragma unroll
    for (int i = 0; i < S::FI; ++i)
#pragma unroll
        for (int j = 0; j < S::FJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (s0 >= s1) return;

    const int64_t i0 = (int64_t)at.ti * S::TI, j0 = (int64_t)at.tj * S::TJ;
    TileLoader<S::TI, S::kThreads, kAK> la;
    TileLoader<S::TJ, S::kThreads, kBK> lb;
    la.init(p.a, p.a.p + at.batch * p.a.stride, i0, s0);
    lb.init(p.b, p.b.p + at.batch * p.b.stride, j0, s0);
    FragReader<S::TI, S::FI, kAK> fa;
    FragReader<S::TJ, S::FJ, kBK> fb;
    fa.init(wave % S::kWI * S::FI * 16);
    fb.init(wave / S::kWI * S::FJ * 16);

    const uint32_t lds = lds_base();
    la.issue(p.a, i0, s0, lds, wave);
    lb.issue(p.b, j0, s0, lds + kB, wave);
    for (int32_t s = s0; s < s1; ++s) {
        const uint32_t odd = (s - s0) & 1;
        const uint32_t cur = lds + (odd ? kStage : 0), next = lds + (odd ? 0 : kStage);
        // this step's loads have landed for every wave, and every wave is
        // done reading the other half
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + 1 < s1) {
            la.issue(p.a, i0, s + 1, next, wave);
            lb.issue(p.b, j0, s + 1, next + kB, wave);
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            s16x8 a[S::FI], b[S::FJ];
#pragma unroll
            for (int j = 0; j < S::FJ; ++j) b[j] = fb.read(cur + kB, j, kk);
#pragma unroll
            for (int i = 0; i < S::FI; ++i) a[i] = fa.read(cur, i, kk);
#pragma unroll
            for (int i = 0; i < S::FI; ++i)
#pragma unroll
                for (int j = 0; j < S::FJ; ++j) acc[i][j] = mfma<kF16>(a[i], b[j], acc[i][j]);
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Where a lane's outputs lie: acc[fi][fj][r] is
//   i = ti TI + wave_i FI 16 + fi 16 + 4 (lane >> 4) + r
//   j = tj TJ + wave_j FJ 16 + fj 16 + (lane & 15).
template <class S>
struct LanePos {
    int64_t i, j;          // of fi = 0, fj = 0, r = 0
    int wave, lane;
    __device__ __forceinline__ LanePos(const TileAt& at, int w)
    {
        wave = w;
        lane = threadIdx.x & 63;
        i = (int64_t)at.ti * S::TI + w % S::kWI * S::FI * 16 + 4 * (lane >> 4);
        j = (int64_t)at.tj * S::TJ + w / S::kWI * S::FJ * 16 + (lane & 15);
    }
};

// Epi::run(args, product, at, pos, acc) takes the sums.
template <class S, bool kF16, bool kAK, bool kBK, class Epi>
__global__ __launch_bounds__(S::kThreads, 2) void product_kernel(ProductArgs p,
                                                                 typename Epi::Args e,
                                                                 int32_t per_matrix)
{
#ifdef __HIP_DEVICE_COMPILE__
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const TileAt at = tile_of(p, per_matrix);
    f32x4 acc[S::FI][S::FJ];
    tile_product<S, kF16, kAK, kBK>(p, at, wave, acc);
    Epi::template run<S>(e, p, at, LanePos<S>(at, wave), acc);
#endif
}

template <class S, bool kF16, bool kAK, bool kBK, class Epi>
hipError_t launch_product(ProductArgs p, const typename Epi::Args& e, hipStream_t stream)
{
    p.tiles_i = (p.ni + S::TI - 1) / S::TI;
    p.tiles_j = (p.nj + S::TJ - 1) / S::TJ;
    const int64_t tiles = p.symmetric ? (int64_t)p.tiles_i * (p.tiles_i + 1) / 2
                                      : (int64_t)p.tiles_i * p.tiles_j;
    const int64_t blocks = tiles * p.split * p.batch;
    if (blocks <= 0) return hipSuccess;
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    const void* k = (const void*)product_kernel<S, kF16, kAK, kBK, Epi>;
    if (S::kLds > 65536) {
        // more dynamic LDS than the default limit: an attribute of the
        // function, set once per device
        static std::atomic<uint64_t> done{0};
        int dev = 0;
        hipError_t err = hipGetDevice(&dev);
        if (err != hipSuccess) return err;
        const uint64_t bit = dev < 64 ? 1ull << dev : 0;
        if (!(done.load(std::memory_order_relaxed) & bit) || !bit) {
            err = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);
            if (err != hipSuccess) return err;
            done.fetch_or(bit, std::memory_order_relaxed);
        }
    }
    hipLaunchKernelGGL((product_kernel<S, kF16, kAK, kBK, Epi>), dim3((unsigned)blocks),
                       dim3(S::kThreads), S::kLds, stream, p, e, (int32_t)(tiles * p.split));
    return hipGetLastError();
}

}  // namespace pr
}  // namespace dte
