// Newton-Schulz orthogonalisation and the Muon step (include/dte_train.h).
//
//   X <- a X + (b S + c S^2) X,  S = X X^T
//
// per iteration three products on the matrix cores: S (symmetric), B = b S +
// c S S (symmetric: both factors and the result), and X B or B X.  S is taken
// on the smaller side: S = X X^T for wide matrices, X^T X for tall ones, and
// neither needs a transposed copy (product.h reads either orientation).  The
// combinations are the products' epilogues.
//
// Precision: an iteration multiplies errors of weak singular directions by up
// to a = 3.4, five of them by several hundred, so BF16 operands (8 bits) cost
// percents of the result for matrices with a few strong directions.  Operands
// are FP16 (11 bits) at the same matrix-core rate, scaled by the power of two
// that the bound on the singular values allows, and the linear term a X is
// taken from a binary32 copy of X, so a weak direction never passes through
// the rounding of a strong one.  Relative error (2-norm, against binary64, 512
// x 1024 and 1536^2, five quintic steps) of this scheme / FP16 without the
// binary32 copy / BF16: random matrices 1.6e-3 / 1.3e-3 / 1.1e-2, 32 strong
// directions over noise 2.2e-4 / 5.7e-3 / 4.6e-2, one strong direction 2e-4 /
// 1.2e-1 / 9.7e-1.
#include <hip/hip_runtime.h>

#include <cmath>

#include "abi_guard.h"
#include "product.h"
#include "train_common.h"

namespace dte {
namespace {

using namespace tr;
using pr::f32x4;

[[maybe_unused]] __device__ __forceinline__ uint16_t to_f16(float x)
{
    return __builtin_bit_cast(uint16_t, (_Float16)x);
}
[[maybe_unused]] __device__ __forceinline__ float from_f16(uint16_t x)
{
    return (float)__builtin_bit_cast(_Float16, x);
}

[[maybe_unused]] __device__ __forceinline__ uint32_t pack(uint16_t lo, uint16_t hi)
{
    return lo | (uint32_t)hi << 16;
}

// ---- the matrix to work on -----------------------------------------------------

// Where the values come from: x (F32 or BF16, any stride), or a Muon step's
// momentum and gradient (contiguous, binary32).
struct Source {
    const void* x;
    int64_t ld, stride;
    int32_t bf16;
    float* momentum;       // not null: Muon
    const float* g;
    float mu;
    int32_t nesterov;
};

__device__ __forceinline__ float muon_value(const Source& s, float m, float g)
{
    return s.nesterov ? g + s.mu * m : m;
}

constexpr int kNormBlocks = 64;    // partial sums per matrix, at most

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
    return x;
}

// Partial sums of squares in binary64 (no overflow or underflow whatever the
// matrix's scale); a Muon step's momentum is updated on the way.
__global__ __launch_bounds__(256) void norm_kernel(Source s, int32_t rows, int32_t cols,
                                                   double* part)
{
    __shared__ double s_sum[4];
    const int64_t b = blockIdx.y;
    double sum = 0.0;
    if (s.momentum) {
        const int64_t n = (int64_t)rows * cols, per = div_up(n, (int64_t)gridDim.x);
        const int64_t begin = blockIdx.x * per, end = begin + per < n ? begin + per : n;
        float* m = s.momentum + b * n;
        const float* g = s.g + b * n;
        for (int64_t i = begin + threadIdx.x; i < end; i += 256) {
            const float gi = g[i], mi = s.mu * m[i] + gi;
            m[i] = mi;
            const double u = muon_value(s, mi, gi);
            sum += u * u;
        }
    } else {
        for (int32_t r = blockIdx.x; r < rows; r += gridDim.x) {
            const int64_t at = b * s.stride + r * s.ld;
            for (int32_t c = threadIdx.x; c < cols; c += 256) {
                const double u = s.bf16 ? from_bf16(((const uint16_t*)s.x)[at + c])
                                        : ((const float*)s.x)[at + c];
                sum += u * u;
            }
        }
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        part[b * gridDim.x + blockIdx.x] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

// X_0 = x / (|x| + eps), padded with zeros to [rpad, cpad], in binary32 and in
// scaled FP16.
__global__ __launch_bounds__(256) void normalise_kernel(Source s, int32_t rows, int32_t cols,
                                                        int64_t rpad, int64_t cpad,
                                                        const double* part, int32_t parts,
                                                        double eps, float scale, float* x32,
                                                        uint16_t* x16)
{
    __shared__ float s_inv;
    const int64_t b = blockIdx.y;
    if (threadIdx.x < 64) {
        double sum = threadIdx.x < (unsigned)parts ? part[b * parts + threadIdx.x] : 0.0;
        sum = wave_sum(sum);
        if (threadIdx.x == 0) s_inv = (float)(1.0 / (sqrt(sum) + eps));
    }
    __syncthreads();
    const float inv = s_inv;
    const int64_t per = cpad / 4, n = rpad * per;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < n;
         q += (int64_t)gridDim.x * 256) {
        const int64_t r = q / per, c = (q - r * per) * 4;
        f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
        if (r < rows) {
            if (s.momentum) {
                const int64_t at = (b * rows + r) * cols + c;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < cols)
                        x[k] = muon_value(s, s.momentum[at + k], s.nesterov ? s.g[at + k] : 0.f);
            } else {
                const int64_t at = b * s.stride + r * s.ld + c;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < cols)
                        x[k] = s.bf16 ? from_bf16(((const uint16_t*)s.x)[at + k])
                                      : ((const float*)s.x)[at + k];
            }
        }
        uint16_t h[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[k] *= inv;
            h[k] = to_f16(x[k] * scale);
        }
        const int64_t o = b * rpad * cpad + r * cpad + c;
        *(f32x4*)(x32 + o) = x;
        *(uint2*)(x16 + o) =
            make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
    }
}

// ---- epilogues -----------------------------------------------------------------

// Square symmetric FP16 result [k, k]: scale * sum, or (B) lin * S + scale *
// sum with S the factor.  Tiles above the diagonal are written twice, once
// transposed.
struct SquareEpi {
    struct Args {
        uint16_t* out;
        const uint16_t* s;     // null: S itself
        int64_t ld, stride;
        float scale, lin;
    };
    template <class S>
    static __device__ __forceinline__ void run(const Args& e, const pr::ProductArgs& p,
                                               const pr::TileAt& at, const pr::LanePos<S>& pos,
                                               f32x4 (&acc)[S::FI][S::FJ])
    {
        uint16_t* out = e.out + at.batch * e.stride;
        const uint16_t* s = e.s ? e.s + at.batch * e.stride : nullptr;
        const bool mirror = p.symmetric && at.ti != at.tj;
#pragma unroll
        for (int j = 0; j < S::FJ; ++j) {
            const int64_t jj = pos.j + 16 * j;
            if (jj >= p.nj) continue;
#pragma unroll
            for (int i = 0; i < S::FI; ++i) {
                const int64_t ii = pos.i + 16 * i;
                if (ii >= p.ni) continue;
                f32x4 x = acc[i][j] * e.scale;
                if (s) {
                    const uint2 w = *(const uint2*)(s + jj * e.ld + ii);
                    x[0] += e.lin * from_f16((uint16_t)w.x);
                    x[1] += e.lin * from_f16((uint16_t)(w.x >> 16));
                    x[2] += e.lin * from_f16((uint16_t)w.y);
                    x[3] += e.lin * from_f16((uint16_t)(w.y >> 16));
                }
                uint16_t h[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) h[r] = to_f16(x[r]);
                *(uint2*)(out + jj * e.ld + ii) =
                    make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
                if (mirror)
#pragma unroll
                    for (int r = 0; r < 4; ++r) out[(ii + r) * e.ld + jj] = h[r];
            }
        }
    }
};

// X' = a X + sum, in binary32 (in place) and in FP16 for the next iteration.
struct NextEpi {
    struct Args {
        float* x32;
        uint16_t* x16;
        int64_t ld, stride;
        float a, scale, next;
    };
    template <class S>
    static __device__ __forceinline__ void run(const Args& e, const pr::ProductArgs& p,
                                               const pr::TileAt& at, const pr::LanePos<S>& pos,
                                               f32x4 (&acc)[S::FI][S::FJ])
    {
        float* x32 = e.x32 + at.batch * e.stride;
        uint16_t* x16 = e.x16 + at.batch * e.stride;
#pragma unroll
        for (int j = 0; j < S::FJ; ++j) {
            const int64_t jj = pos.j + 16 * j;
            if (jj >= p.nj) continue;
#pragma unroll
            for (int i = 0; i < S::FI; ++i) {
                const int64_t ii = pos.i + 16 * i;
                if (ii >= p.ni) continue;
                f32x4* q = (f32x4*)(x32 + jj * e.ld + ii);
                const f32x4 x = *q * e.a + acc[i][j] * e.scale;
                *q = x;
                *(uint2*)(x16 + jj * e.ld + ii) =
                    make_uint2(pack(to_f16(x[0] * e.next), to_f16(x[1] * e.next)),
                               pack(to_f16(x[2] * e.next), to_f16(x[3] * e.next)));
            }
        }
    }
};

// The last iteration: the result in BF16, and (kMuon) the weights' step.
template <bool kMuon>
struct LastEpi {
    struct Args {
        const float* x32;
        int64_t ld, stride;    // of x32
        float a, scale;
        uint16_t* out;
        int64_t out_ld, out_stride;
        int32_t rows, cols;
        int32_t vec, pvec;     // rows of out at 8-byte, of p at 16-byte addresses
        float* p;              // [batch, rows, cols]
        float decay, rate;
    };
    template <class S>
    static __device__ __forceinline__ void run(const Args& e, const pr::ProductArgs& p,
                                               const pr::TileAt& at, const pr::LanePos<S>& pos,
                                               f32x4 (&acc)[S::FI][S::FJ])
    {
        const float* x32 = e.x32 + at.batch * e.stride;
        uint16_t* out = e.out + at.batch * e.out_stride;
        float* w = kMuon ? e.p + at.batch * (int64_t)e.rows * e.cols : nullptr;
#pragma unroll
        for (int j = 0; j < S::FJ; ++j) {
            const int64_t jj = pos.j + 16 * j;
            if (jj >= e.rows) continue;
#pragma unroll
            for (int i = 0; i < S::FI; ++i) {
                const int64_t ii = pos.i + 16 * i;
                if (ii >= e.cols) continue;
                const f32x4 x = *(const f32x4*)(x32 + jj * e.ld + ii) * e.a + acc[i][j] * e.scale;
                const uint32_t lo = pack(to_bf16(x[0]), to_bf16(x[1]));
                const uint32_t hi = pack(to_bf16(x[2]), to_bf16(x[3]));
                const f32x4 o = f32x4{from_bf16((uint16_t)lo), from_bf16((uint16_t)(lo >> 16)),
                                      from_bf16((uint16_t)hi), from_bf16((uint16_t)(hi >> 16))};
                const bool whole = ii + 4 <= e.cols;
                uint16_t* q = out + jj * e.out_ld + ii;
                if (e.vec && whole) {
                    *(uint2*)q = make_uint2(lo, hi);
                } else {
                    q[0] = (uint16_t)lo;
                    if (ii + 1 < e.cols) q[1] = (uint16_t)(lo >> 16);
                    if (ii + 2 < e.cols) q[2] = (uint16_t)hi;
                    if (ii + 3 < e.cols) q[3] = (uint16_t)(hi >> 16);
                }
                if constexpr (kMuon) {
                    float* v = w + jj * e.cols + ii;
                    if (e.pvec && whole) {
                        *(f32x4*)v = *(const f32x4*)v * e.decay - o * e.rate;
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (ii + r < e.cols) v[r] = e.decay * v[r] - e.rate * o[r];
                    }
                }
            }
        }
    }
};

// ---- host ------------------------------------------------------------------------

// What the coefficients do to singular values in [0, 1]: per iteration the
// largest singular value before it, and the largest |b s^2 + c s^4|.
struct Bounds {
    double sigma[DTE_MAX_NS_STEPS + 1];
    double b[DTE_MAX_NS_STEPS];
};

bool bounds_of(const dte_newton_schulz* ns, Bounds* out)
{
    if (!ns || ns->steps < 1 || ns->steps > DTE_MAX_NS_STEPS || ns->reserved != 0) return false;
    if (!(std::isfinite(ns->eps) && ns->eps >= 0.0)) return false;
    double s = 1.0;
    out->sigma[0] = s;
    for (int k = 0; k < ns->steps; ++k) {
        const double a = ns->coefficients[k][0], b = ns->coefficients[k][1],
                     c = ns->coefficients[k][2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
        double top = 0.0, btop = 0.0;
        // the polynomials in t = s^2, at the ends and where they turn
        double at[4] = {s * s, 0.0, 0.0, 0.0};
        const double disc = 9.0 * b * b - 20.0 * a * c;
        if (c != 0.0) {
            if (disc >= 0.0) {
                at[1] = (-3.0 * b + std::sqrt(disc)) / (10.0 * c);
                at[2] = (-3.0 * b - std::sqrt(disc)) / (10.0 * c);
            }
            at[3] = -b / (2.0 * c);
        } else if (b != 0.0) {
            at[1] = -a / (3.0 * b);
        }
        for (double t : at) {
            if (!(t >= 0.0 && t <= s * s)) continue;
            top = std::fmax(top, std::fabs(std::sqrt(t) * (a + t * (b + t * c))));
            btop = std::fmax(btop, std::fabs(t * (b + t * c)));
        }
        if (!(top <= 16.0) || !(btop <= 16384.0)) return false;
        out->b[k] = btop;
        out->sigma[k + 1] = s = top;
    }
    return true;
}

// The largest power of two that keeps values up to `top` within half of
// FP16's range.
double fp16_scale(double top)
{
    if (!(top > 0.0)) return 1.0;
    const double e = std::floor(std::log2(16384.0 / top));
    return std::ldexp(1.0, (int)std::fmin(std::fmax(e, -14.0), 40.0));
}

struct OrthSizes {
    int64_t batch, rows, cols, rpad, cpad, kpad;
    bool wide;
};

bool orth_sizes(int64_t batch, int64_t rows, int64_t cols, OrthSizes* z)
{
    if (batch < 0 || batch >= 1 << 16 || rows < 0 || rows >= 1 << 16 || cols < 0 ||
        cols >= 1 << 16)
        return false;
    z->batch = batch;
    z->rows = rows;
    z->cols = cols;
    z->rpad = round_up(rows, 64);
    z->cpad = round_up(cols, 64);
    z->wide = rows <= cols;
    z->kpad = z->wide ? z->rpad : z->cpad;
    return true;
}

struct OrthBuffers {
    double* part;
    float* x32;
    uint16_t *x16[2], *s, *b;
};

int64_t carve(const OrthSizes& z, void* ws, OrthBuffers* b)
{
    Carver c(ws);
    const int64_t n = z.batch * z.rpad * z.cpad, k = z.batch * z.kpad * z.kpad;
    b->part = c.take<double>(z.batch * kNormBlocks);
    b->x32 = c.take<float>(n);
    b->x16[0] = c.take<uint16_t>(n);
    b->x16[1] = c.take<uint16_t>(n);
    b->s = c.take<uint16_t>(k);
    b->b = c.take<uint16_t>(k);
    return c.used;
}

// Tile shape by the rounds that the blocks take: a round of 256 x 256 tiles
// (one per CU) does four units of work, one of 128 x 128 tiles (two per CU)
// two units at nine tenths of the rate.
bool large_tiles(int64_t ni, int64_t nj, int64_t batch, bool symmetric, int cus)
{
    auto rounds = [&](int64_t t, int64_t slots) {
        const int64_t a = div_up(ni, t), b = div_up(nj, t);
        return div_up(batch * (symmetric ? a * (a + 1) / 2 : a * b), slots);
    };
    return rounds(256, cus) * 4.0 <= rounds(128, 2 * cus) * 2.2;
}

template <pr::Layout kA, pr::Layout kB, class Epi>
hipError_t product(pr::ProductArgs p, const typename Epi::Args& e, hipStream_t st)
{
    return large_tiles(p.ni, p.nj, p.batch, p.symmetric != 0, device_cus())
               ? pr::launch_product<pr::Large, true, kA, kB, Epi>(p, e, st)
               : pr::launch_product<pr::Medium, true, kA, kB, Epi>(p, e, st);
}

struct Muon {
    float* p;
    float decay, rate;
};

hipError_t orthogonalise(const Source& src, const OrthSizes& z, const dte_newton_schulz& ns,
                         const Bounds& bd, uint16_t* out, int64_t out_ld, int64_t out_stride,
                         const Muon* muon, const OrthBuffers& b, hipStream_t st)
{
    const int64_t n = z.rpad * z.cpad;
    int64_t parts = div_up(z.rows * z.cols, 4096);
    if (!src.momentum && parts > z.rows) parts = z.rows;
    if (parts > kNormBlocks) parts = kNormBlocks;
    norm_kernel<<<dim3((unsigned)parts, (unsigned)z.batch), dim3(256), 0, st>>>(
        src, (int32_t)z.rows, (int32_t)z.cols, b.part);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    int64_t blocks = div_up(n / 4, 256);
    const int64_t most = div_up(4096, z.batch);
    if (blocks > most) blocks = most;
    double xs = fp16_scale(bd.sigma[0]);
    normalise_kernel<<<dim3((unsigned)blocks, (unsigned)z.batch), dim3(256), 0, st>>>(
        src, (int32_t)z.rows, (int32_t)z.cols, z.rpad, z.cpad, b.part, (int32_t)parts, ns.eps,
        (float)xs, b.x32, b.x16[0]);
    err = hipGetLastError();
    if (err != hipSuccess) return err;

    for (int k = 0; k < ns.steps; ++k) {
        const uint16_t* x = b.x16[k & 1];
        const double ss = fp16_scale(bd.sigma[k] * bd.sigma[k]), bs = fp16_scale(bd.b[k]);
        const double a = ns.coefficients[k][0], bc = ns.coefficients[k][1],
                     cc = ns.coefficients[k][2];
        const int64_t kk = z.kpad * z.kpad;
        // S
        pr::ProductArgs p{};
        p.a = p.b = z.wide ? pr::Operand{x, z.cpad, n, (int32_t)z.rpad, (int32_t)z.cpad, 0}
                           : pr::Operand{x, z.cpad, n, (int32_t)z.cpad, (int32_t)z.rpad, 0};
        p.ni = p.nj = (int32_t)z.kpad;
        p.steps = (int32_t)((z.wide ? z.cpad : z.rpad) / 64);
        p.split = 1;
        p.batch = (int32_t)z.batch;
        p.symmetric = 1;
        const SquareEpi::Args es{b.s, nullptr, z.kpad, kk, (float)(ss / (xs * xs)), 0.f};
        err = z.wide ? product<pr::kK, pr::kK, SquareEpi>(p, es, st)
                     : product<pr::kR, pr::kR, SquareEpi>(p, es, st);
        if (err != hipSuccess) return err;
        // B = b S + c S S
        p.a = p.b = pr::Operand{b.s, z.kpad, kk, (int32_t)z.kpad, (int32_t)z.kpad, 0};
        p.steps = (int32_t)(z.kpad / 64);
        const SquareEpi::Args eb{b.b, b.s, z.kpad, kk, (float)(cc * bs / (ss * ss)),
                                 (float)(bc * bs / ss)};
        err = product<pr::kK, pr::kK, SquareEpi>(p, eb, st);
        if (err != hipSuccess) return err;
        // X
        const bool last = k + 1 == ns.steps;
        const double next = last ? 1.0 : fp16_scale(bd.sigma[k + 1]);
        const pr::Operand bm{b.b, z.kpad, kk, (int32_t)z.kpad, (int32_t)z.kpad, 0};
        pr::ProductArgs u{};
        u.ni = (int32_t)z.cpad;
        u.nj = (int32_t)z.rpad;
        u.steps = (int32_t)(z.kpad / 64);
        u.split = 1;
        u.batch = (int32_t)z.batch;
        if (z.wide) {      // out[j, i] = sum_k X[k, i] B[j, k]
            u.a = pr::Operand{x, z.cpad, n, (int32_t)z.cpad, (int32_t)z.rpad, 0};
            u.b = bm;
        } else {           // out[j, i] = sum_k B[i, k] X[j, k]
            u.a = bm;
            u.b = pr::Operand{x, z.cpad, n, (int32_t)z.rpad, (int32_t)z.cpad, 0};
        }
        const float scale = (float)(1.0 / (bs * xs));
        if (!last) {
            const NextEpi::Args e{b.x32, b.x16[(k + 1) & 1], z.cpad, n, (float)a, scale,
                                  (float)next};
            err = z.wide ? product<pr::kR, pr::kK, NextEpi>(u, e, st)
                         : product<pr::kK, pr::kK, NextEpi>(u, e, st);
        } else if (muon) {
            const LastEpi<true>::Args e{
                b.x32, z.cpad, n, (float)a, scale, out, out_ld, out_stride, (int32_t)z.rows,
                (int32_t)z.cols, rows_aligned(out, out_ld, 2, 8) && out_stride % 4 == 0,
                rows_aligned(muon->p, z.cols, 4, 16), muon->p, muon->decay, muon->rate};
            err = z.wide ? product<pr::kR, pr::kK, LastEpi<true>>(u, e, st)
                         : product<pr::kK, pr::kK, LastEpi<true>>(u, e, st);
        } else {
            const LastEpi<false>::Args e{
                b.x32, z.cpad, n, (float)a, scale, out, out_ld, out_stride, (int32_t)z.rows,
                (int32_t)z.cols, rows_aligned(out, out_ld, 2, 8) && out_stride % 4 == 0, 0,
                nullptr, 0.f, 0.f};
            err = z.wide ? product<pr::kR, pr::kK, LastEpi<false>>(u, e, st)
                         : product<pr::kK, pr::kK, LastEpi<false>>(u, e, st);
        }
        if (err != hipSuccess) return err;
        xs = next;
    }
    return hipSuccess;
}

}  // namespace
}  // namespace dte

extern "C" {

int64_t dte_orthogonalise_workspace_bytes(int64_t batch, int64_t rows, int64_t cols)
{
    dte::OrthSizes z;
    dte::OrthBuffers b;
    if (!dte::orth_sizes(batch, rows, cols, &z)) return -1;
    if (batch == 0 || rows == 0 || cols == 0) return 0;
    return dte::carve(z, nullptr, &b);
}

dte_status dte_orthogonalise(const void* x, int32_t x_type, int64_t batch, int64_t rows,
                             int64_t cols, int64_t x_ld, int64_t x_stride,
                             const dte_newton_schulz* ns, uint16_t* out, int64_t out_ld,
                             int64_t out_stride, void* workspace, int64_t workspace_bytes,
                             void* stream)
{
    using namespace dte::tr;
    dte::OrthSizes z;
    dte::Bounds bd;
    if (!dte::orth_sizes(batch, rows, cols, &z) || !valid_type(x_type) ||
        !dte::bounds_of(ns, &bd) || !valid_ld(x_ld, cols) || !valid_ld(out_ld, cols))
        return DTE_ERR_ARG;
    if (batch == 0 || rows == 0 || cols == 0) return DTE_OK;
    const int64_t xspan = (rows - 1) * x_ld + cols, ospan = (rows - 1) * out_ld + cols;
    if (batch > 1 && (x_stride < xspan || out_stride < ospan)) return DTE_ERR_ARG;
    if (!x || !out) return DTE_ERR_ARG;
    dte::OrthBuffers b;
    if (!workspace_ok(workspace, workspace_bytes, dte::carve(z, workspace, &b)))
        return DTE_ERR_ARG;
    const dte::Source src{x, x_ld, x_stride, x_type == DTE_TYPE_BF16, nullptr, nullptr, 0.f, 0};
    return dte::orthogonalise(src, z, *ns, bd, out, out_ld, out_stride, nullptr, b,
                              (hipStream_t)stream) == hipSuccess
               ? DTE_OK
               : DTE_ERR_HIP;
}

dte_status dte_muon_forward(float* p, float* momentum, const float* g, int64_t batch, int64_t rows,
                            int64_t cols, const dte_muon_step* hp, uint16_t* update,
                            void* workspace, int64_t workspace_bytes, void* stream)
{
    using namespace dte::tr;
    dte::OrthSizes z;
    dte::Bounds bd;
    if (!dte::orth_sizes(batch, rows, cols, &z) || !hp || hp->reserved != 0 ||
        !dte::bounds_of(&hp->ns, &bd))
        return DTE_ERR_ARG;
    const double decay = 1.0 - hp->lr * hp->weight_decay, rate = hp->lr * hp->update_scale;
    if (!(std::isfinite(hp->lr) && hp->lr >= 0.0) || !std::isfinite(hp->weight_decay) ||
        !(hp->momentum >= 0.0 && hp->momentum < 1.0) || !(decay > 0.0) || !std::isfinite(decay) ||
        !std::isfinite(rate))
        return DTE_ERR_ARG;
    if (batch == 0 || rows == 0 || cols == 0) return DTE_OK;
    if (!p || !momentum || !g || !update) return DTE_ERR_ARG;
    dte::OrthBuffers b;
    if (!workspace_ok(workspace, workspace_bytes, dte::carve(z, workspace, &b)))
        return DTE_ERR_ARG;
    const dte::Source src{nullptr, cols, rows * cols, 0, momentum, g, (float)hp->momentum,
                          hp->nesterov != 0};
    const dte::Muon muon{p, (float)decay, (float)rate};
    return dte::orthogonalise(src, z, hp->ns, bd, update, cols, rows * cols, &muon, b,
                              (hipStream_t)stream) == hipSuccess
               ? DTE_OK
               : DTE_ERR_HIP;
}

}  // extern "C"
