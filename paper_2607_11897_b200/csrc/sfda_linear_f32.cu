// Linear attention with a fixed decay for each head, fp32 precision (see sfda_linear.h for the form).
//
// One CTA of eight warps takes a block of CB value columns of one (batch, head) pair and walks its chunks of 64 tokens in
// order: P = (a b^T) o D, out = P c + e o (a S), S <- g^n S + (w o b)^T c.  The columns of a state never interact, so blocks
// of columns of a pair are independent (each repeats P); they are what keeps the SMs busy when there are few pairs.
// All products run on the warp-level tensor cores with both operands split into two tf32 parts (hi hi + hi lo + lo hi:
// 21 bits of each operand, sums in fp32).  The state stays in the accumulators of the warps that own its rows; a copy in
// shared memory is the operand of a S.
//
// A value of c that is not finite would reach earlier tokens of its chunk through 0 * NaN, since masked entries of P are
// zeros of a dense product.  Such a value is taken as zero, and its column's outputs from that token on, and its column of
// the state, are NaN instead.
#include <float.h>

#include "sfda_common.cuh"
#include "sfda_linear.h"
#include "sfda_tc_ptx.cuh"

namespace sfda {
namespace {

constexpr int kThreads = 256;
constexpr int L = 64;            // tokens per chunk
constexpr int kNever = 0x7fffffff;

__device__ __forceinline__ void split_tf32(float x, uint32_t &hi, uint32_t &lo)
{
    hi = __float_as_uint(x) & 0xffffe000u;                 // the tensor core reads 10 mantissa bits: cut, not rounded,
    lo = __float_as_uint(x - __uint_as_float(hi));         // so that the rest is exact
}
// c += A B for one 16 x 8 tile and 8 values of k, both operands in two parts.  The tensor core cuts its sums off instead of
// rounding them, always towards zero: the small products are summed by themselves, and no sum runs for longer than one
// product of a chunk before fp32 additions take it over (a state of 3000 tokens summed in its accumulators was 9e-6 off).
__device__ __forceinline__ void mma3(float (&c)[4], float (&c_lo)[4], const float (&a)[4], const float (&b)[2])
{
    uint32_t ah[4], al[4], bh[2], bl[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) split_tf32(a[i], ah[i], al[i]);
#pragma unroll
    for (int i = 0; i < 2; ++i) split_tf32(b[i], bh[i], bl[i]);
    tc::mma_tf32(c_lo, al, bh);
    tc::mma_tf32(c_lo, ah, bl);
    tc::mma_tf32(c, ah, bh);
}

struct Dev {
    const float *log_decay;
    const int *lens;
    const void *a, *b, *c;
    void *out;
    const float *s_in;
    float *s_out;
    int T, H, Ha, Hb, Hc, reverse, s_in_t, out_f32;
    float sp, se, sw;
};

template <int DA, int CB>
struct Smem {
    static constexpr int LA = DA + 4, LC = CB + 8, LP = L + 4;
    float a[L * LA], b[L * LA], c[L * LC], S[DA * LC], P[L * LP];
    float pw[L + 1];             // g^0 .. g^64
    int first[CB];               // first token (in the pass's order) whose value of this column was not finite
};

template <int DA, int DC, int CB, typename T>
__global__ void __launch_bounds__(kThreads) sfda_linear_f32_kernel(const Dev p)
{
    using Sm = Smem<DA, CB>;
    extern __shared__ __align__(16) unsigned char raw[];
    Sm &s = *reinterpret_cast<Sm *>(raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, tg = lane & 3;
    const int h = blockIdx.x % p.H;
    const size_t bh = blockIdx.x, bt = (size_t)(blockIdx.x / p.H) * p.T;
    const int c0 = blockIdx.y * CB;
    const int len = p.lens ? min(max(p.lens[blockIdx.x / p.H], 0), p.T) : p.T;
    const int chunks = (len + L - 1) / L;
    const float ld = p.log_decay[h];
    for (int i = tid; i <= L; i += kThreads) s.pw[i] = i == 0 ? 1.f : expf((float)i * ld);
    for (int i = tid; i < CB; i += kThreads) s.first[i] = kNever;

    // the warp's part of the state: rows 16 wr .., columns NS wc ..
    constexpr int WR = DA / 16, WC = 8 / WR, NS = CB / WC, TS = NS / 8;
    const int wr = warp % WR, wc = warp / WR;
    float st[TS][4];
#pragma unroll
    for (int j = 0; j < TS; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int r = 16 * wr + g + 8 * (x >> 1), col = c0 + NS * wc + 8 * j + 2 * tg + (x & 1);
            st[j][x] = !p.s_in ? 0.f : p.s_in_t ? p.s_in[(bh * DC + col) * DA + r] : p.s_in[(bh * DA + r) * DC + col];
        }

    const T *pa = static_cast<const T *>(p.a), *pb = static_cast<const T *>(p.b), *pc = static_cast<const T *>(p.c);
    const int ha = h / (p.H / p.Ha), hb = h / (p.H / p.Hb), hc = h / (p.H / p.Hc);
    for (int ci = 0; ci < chunks; ++ci) {
        const int chunk = p.reverse ? chunks - 1 - ci : ci;
        const int t0 = chunk * L, n = min(L, len - t0);
        __syncthreads();                                   // the last chunk's readers are done (and pw, first are set)
        for (int i = tid; i < L * DA; i += kThreads) {
            const int r = i / DA, d = i % DA;
            const size_t row = bt + t0 + r;
            s.a[r * Sm::LA + d] = r < n ? ld_val(pa, (row * p.Ha + ha) * DA + d) : 0.f;
            s.b[r * Sm::LA + d] = r < n ? ld_val(pb, (row * p.Hb + hb) * DA + d) : 0.f;
        }
        for (int i = tid; i < L * CB; i += kThreads) {
            const int r = i / CB, d = i % CB;
            float x = r < n ? ld_val(pc, ((bt + t0 + r) * p.Hc + hc) * DC + c0 + d) : 0.f;
            if (!(fabsf(x) <= FLT_MAX)) {
                x = 0.f;
                atomicMin(&s.first[d], p.reverse ? len - 1 - (t0 + r) : t0 + r);
            }
            s.c[r * Sm::LC + d] = x;
        }
#pragma unroll
        for (int j = 0; j < TS; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                s.S[(16 * wr + g + 8 * (x >> 1)) * Sm::LC + NS * wc + 8 * j + 2 * tg + (x & 1)] = st[j][x];
        __syncthreads();

        {   // P = (a b^T) o D: the warp's 16 rows and 32 columns
            const int r0 = 16 * (warp & 3), q0 = 32 * (warp >> 2);
            float acc[4][4] = {}, low[4][4] = {};
            for (int k0 = 0; k0 < DA; k0 += 8) {
                float av[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) av[x] = s.a[(r0 + g + 8 * (x & 1)) * Sm::LA + k0 + tg + 4 * (x >> 1)];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float bv[2] = {s.b[(q0 + 8 * j + g) * Sm::LA + k0 + tg], s.b[(q0 + 8 * j + g) * Sm::LA + k0 + tg + 4]};
                    mma3(acc[j], low[j], av, bv);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int t = r0 + g + 8 * (x >> 1), i = q0 + 8 * j + 2 * tg + (x & 1), gap = p.reverse ? i - t : t - i;
                    s.P[t * Sm::LP + i] = gap >= 0 ? (acc[j][x] + low[j][x]) * (p.sp * s.pw[gap]) : 0.f;
                }
        }
        __syncthreads();
        if (p.out) {   // out = e o (a S) + P c: 16 rows and CB / 2 columns
            constexpr int TO = CB / 16;
            const int r0 = 16 * (warp & 3), q0 = (CB / 2) * (warp >> 2);
            float acc[TO][4] = {}, low[TO][4] = {};
            for (int k0 = 0; k0 < DA; k0 += 8) {
                float av[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) av[x] = s.a[(r0 + g + 8 * (x & 1)) * Sm::LA + k0 + tg + 4 * (x >> 1)];
#pragma unroll
                for (int j = 0; j < TO; ++j) {
                    float bv[2] = {s.S[(k0 + tg) * Sm::LC + q0 + 8 * j + g], s.S[(k0 + tg + 4) * Sm::LC + q0 + 8 * j + g]};
                    mma3(acc[j], low[j], av, bv);
                }
            }
            float out[TO][4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int t = r0 + g + 8 * (x >> 1);
                const float e = p.se * s.pw[p.reverse ? max(n - 1 - t, 0) : min(t + 1, L)];
#pragma unroll
                for (int j = 0; j < TO; ++j) {
                    out[j][x] = e * (acc[j][x] + low[j][x]);
                    acc[j][x] = low[j][x] = 0.f;
                }
            }
            for (int k0 = 0; k0 < L; k0 += 8) {
                float av[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) av[x] = s.P[(r0 + g + 8 * (x & 1)) * Sm::LP + k0 + tg + 4 * (x >> 1)];
#pragma unroll
                for (int j = 0; j < TO; ++j) {
                    float bv[2] = {s.c[(k0 + tg) * Sm::LC + q0 + 8 * j + g], s.c[(k0 + tg + 4) * Sm::LC + q0 + 8 * j + g]};
                    mma3(acc[j], low[j], av, bv);
                }
            }
#pragma unroll
            for (int j = 0; j < TO; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int t = r0 + g + 8 * (x >> 1), col = q0 + 8 * j + 2 * tg + (x & 1);
                    if (t >= n) continue;
                    const int order = p.reverse ? len - 1 - (t0 + t) : t0 + t;
                    const float y = order >= s.first[col] ? __int_as_float(0x7fffffff) : out[j][x] + (acc[j][x] + low[j][x]);
                    const size_t at = ((bt + t0 + t) * p.H + h) * DC + c0 + col;
                    if (p.out_f32) static_cast<float *>(p.out)[at] = y;
                    else st_val(static_cast<T *>(p.out), at, y);
                }
        }
        {   // S <- g^n S + (w o b)^T c.  Weak decays through g^n - 1, whose rounding is not the same relative error chunk
            // after chunk.
            float acc[TS][4] = {}, low[TS][4] = {};
            const float x = (float)n * ld, gn = expf(x), gm = x > -0.5f ? expm1f(x) : gn;
            for (int k0 = 0; k0 < n; k0 += 8) {
                float av[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int i = k0 + tg + 4 * (y >> 1);
                    const float w = i < n ? p.sw * s.pw[p.reverse ? i + 1 : n - 1 - i] : 0.f;
                    av[y] = w * s.b[i * Sm::LA + 16 * wr + g + 8 * (y & 1)];
                }
#pragma unroll
                for (int j = 0; j < TS; ++j) {
                    const int col = NS * wc + 8 * j + g;
                    float bv[2] = {s.c[(k0 + tg) * Sm::LC + col], s.c[(k0 + tg + 4) * Sm::LC + col]};
                    mma3(acc[j], low[j], av, bv);
                }
            }
#pragma unroll
            for (int j = 0; j < TS; ++j)
#pragma unroll
                for (int y = 0; y < 4; ++y) st[j][y] = (x > -0.5f ? fmaf(st[j][y], gm, st[j][y]) : st[j][y] * gn) + (acc[j][y] + low[j][y]);
        }
    }
    __syncthreads();
    if (p.s_out)
#pragma unroll
        for (int j = 0; j < TS; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int r = 16 * wr + g + 8 * (x >> 1), col = NS * wc + 8 * j + 2 * tg + (x & 1);
                p.s_out[(bh * DA + r) * DC + c0 + col] = s.first[col] == kNever ? st[j][x] : __int_as_float(0x7fffffff);
            }
}

template <int DA, int DC, int CB, typename T>
cudaError_t launch_block(const LinearArgs &a, const LinearPass &p, cudaStream_t stream)
{
    const Dev d = {a.log_decay, a.lens, p.a, p.b, p.c, p.out, p.s_in, p.s_out, a.T, a.H, p.Ha, p.Hb, p.Hc, p.reverse,
                   p.s_in_t, p.out_f32, p.sp, p.se, p.sw};
    auto kernel = sfda_linear_f32_kernel<DA, DC, CB, T>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<DA, CB>));
    if (e != cudaSuccess) return e;
    kernel<<<dim3((unsigned)a.B * a.H, DC / CB), kThreads, sizeof(Smem<DA, CB>), stream>>>(d);
    return cudaGetLastError();
}

template <int DA, int DC, typename T>
cudaError_t launch_one(const LinearArgs &a, const LinearPass &p, cudaStream_t stream)
{
    const long long pairs = (long long)a.B * a.H;
    if (pairs * (DC / 16) <= 148) return launch_block<DA, DC, 16, T>(a, p, stream);
    return launch_block<DA, DC, 32, T>(a, p, stream);
}

template <typename T>
cudaError_t dispatch(const LinearArgs &a, const LinearPass &p, cudaStream_t stream)
{
    if (p.DA == 128 && p.DC == 128) return launch_one<128, 128, T>(a, p, stream);
    if (p.DA == 128 && p.DC == 64) return launch_one<128, 64, T>(a, p, stream);
    if (p.DA == 64 && p.DC == 128) return launch_one<64, 128, T>(a, p, stream);
    if (p.DA == 64 && p.DC == 64) return launch_one<64, 64, T>(a, p, stream);
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_linear_f32(const LinearArgs &a, const LinearPass &p, cudaStream_t stream, int *launches)
{
    const cudaError_t e = dispatch<float>(a, p, stream);
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}

}  // namespace sfda
