// Linear attention with a fixed decay for each head, fp32 precision (see sfda_linear.h for the form).
//
// One CTA of eight warps takes a block of CB value columns of one (batch, head) pair in one pass and walks its chunks of 64 tokens
// in order, the next chunk's tiles on their way while it works: P = (a b^T) o D, out = P c + e o (a S), S <- g^n S + (w o b)^T c.  The columns of a state never interact, so blocks
// of columns of a pair are independent (each repeats P); they are what keeps the SMs busy when there are few pairs.
// All products run on the warp-level tensor cores with both operands split into two tf32 parts (hi hi + hi lo + lo hi:
// 22 bits of each operand, sums in fp32).  The state stays in the accumulators of the warps that own its rows; a copy in
// shared memory is the operand of a S.
//
// A value of c that is not finite would reach earlier tokens of its chunk through 0 * NaN, since masked entries of P are
// zeros of a dense product.  Such a value is taken as zero, and its column's outputs from that token on, and its column of
// the state, are NaN instead.  The same holds for the largest finite values (from 2^128 - 2^116 on), whose high part rounds to infinity.
#include "sfda_common.cuh"
#include "sfda_linear.h"
#include "sfda_tc_ptx.cuh"

namespace sfda {
namespace {

constexpr int kThreads = 256;
constexpr int L = 64;            // tokens per chunk
constexpr int kNever = 0x7fffffff;
constexpr float kMost = 0x1.ffdffep127f;     // the largest value whose high part is finite

__device__ __forceinline__ void split_tf32(float x, uint32_t &hi, uint32_t &lo)
{
    // The tensor core cuts its operands off at 10 mantissa bits.  Half a step added before that makes it a rounding for the high
    // part (ties away from zero), which leaves 2^-12; the low part is cut at 2^-10 of that, either sign as often as the other.
    // (A NaN of all ones loses its exponent in the high part; the difference is a NaN still, and stays one.)
    hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
    lo = __float_as_uint(x - __uint_as_float(hi));
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2])
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
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
    mma(c_lo, al, bh);
    mma(c, ah, bh);
    mma(c_lo, ah, bl);
}

struct Pass {
    const float *a, *b, *c;
    float *out;
    const float *s_in;
    float *s_out;
    int Ha, Hb, Hc, reverse, s_in_t;
    float sp, se, sw;
};
struct Dev {
    Pass pass[3];
    const float *log_decay;
    const int *lens;
    int T, H;
};

template <int DA, int CB>
struct Smem {
    static constexpr int LA = DA + 4, LC = CB + 8, LP = L + 4;
    float a[2][L * LA], b[2][L * LA], c[2][L * LC], S[DA * LC], P[L * LP];
    float pw[L + 4];             // g^0 .. g^64
    float w[2][L];               // the chunk's weights of b; of two chunks, for one is written while the other is read
    int first[CB];               // first token (in the pass's order) whose value of this column was not finite
};

// 16 bytes to shared memory in the background; zeros where `on` is not set
__device__ __forceinline__ void copy16(float *to, const float *from, bool on)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(to)), "l"(from), "r"(on ? 16 : 0) : "memory");
}

template <int DA, int DC, int CB>
__global__ void __launch_bounds__(kThreads) sfda_linear_f32_kernel(const Dev dev)
{
    using Sm = Smem<DA, CB>;
    extern __shared__ __align__(16) unsigned char raw[];
    Sm &s = *reinterpret_cast<Sm *>(raw);
    const Pass &p = dev.pass[blockIdx.z];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, tg = lane & 3;
    const int H = dev.H, T = dev.T, h = blockIdx.x % H, rev = p.reverse;
    const size_t bh = blockIdx.x, bt = (size_t)(blockIdx.x / H) * T;
    const int c0 = blockIdx.y * CB;
    const int len = dev.lens ? min(max(dev.lens[blockIdx.x / H], 0), T) : T;
    const int chunks = (len + L - 1) / L;
    const float ld = dev.log_decay[h];
    const int ha = h / (H / p.Ha), hb = h / (H / p.Hb), hc = h / (H / p.Hc);

    // the tiles of the i-th chunk in the pass's order, in the background
    const auto fetch = [&](int i) {
        const int t0 = (rev ? chunks - 1 - i : i) * L, n = min(L, len - t0), st = i & 1;
        for (int x = tid; x < L * DA / 4; x += kThreads) {
            const int r = x / (DA / 4), d = x % (DA / 4) * 4, rr = r < n ? r : 0;
            copy16(&s.a[st][r * Sm::LA + d], p.a + ((bt + t0 + rr) * p.Ha + ha) * DA + d, r < n);
            copy16(&s.b[st][r * Sm::LA + d], p.b + ((bt + t0 + rr) * p.Hb + hb) * DA + d, r < n);
        }
        for (int x = tid; x < L * CB / 4; x += kThreads) {
            const int r = x / (CB / 4), d = x % (CB / 4) * 4, rr = r < n ? r : 0;
            copy16(&s.c[st][r * Sm::LC + d], p.c + ((bt + t0 + rr) * p.Hc + hc) * DC + c0 + d, r < n);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (chunks > 0) fetch(0);
    for (int i = tid; i <= L; i += kThreads) s.pw[i] = i == 0 ? 1.f : expf((float)i * ld);
    for (int i = tid; i < CB; i += kThreads) s.first[i] = kNever;

    // the warp's part of the state: rows 16 wr .., columns NS wc ..
    constexpr int WR = DA / 16, WC = 8 / WR, NS = CB / WC, TS = NS / 8;
    const int wr = warp % WR, wc = warp / WR;
    float st[TS][4];
    const auto keep_copy = [&] {
#pragma unroll
        for (int j = 0; j < TS; ++j)
#pragma unroll
            for (int x = 0; x < 2; ++x)
                *reinterpret_cast<float2 *>(&s.S[(16 * wr + g + 8 * x) * Sm::LC + NS * wc + 8 * j + 2 * tg]) = make_float2(st[j][2 * x], st[j][2 * x + 1]);
    };
#pragma unroll
    for (int j = 0; j < TS; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int r = 16 * wr + g + 8 * (x >> 1), col = c0 + NS * wc + 8 * j + 2 * tg + (x & 1);
            st[j][x] = !p.s_in ? 0.f : p.s_in_t ? p.s_in[(bh * DC + col) * DA + r] : p.s_in[(bh * DA + r) * DC + col];
        }
    keep_copy();
    __syncthreads();

    int decay_of = 0;                                          // the chunk length that gm is for
    float gm = 0.f;
    bool weak = false;
    for (int ci = 0; ci < chunks; ++ci) {
        const int t0 = (rev ? chunks - 1 - ci : ci) * L, n = min(L, len - t0), buf = ci & 1;
        float *sa = s.a[buf], *sb = s.b[buf], *sc = s.c[buf];
        if (n != decay_of) {
            decay_of = n;
            weak = (float)n * ld > -0.5f;
            gm = weak ? expm1f((float)n * ld) : expf((float)n * ld);
        }
        if (tid < L) s.w[buf][tid] = tid < n ? p.sw * s.pw[rev ? tid + 1 : n - 1 - tid] : 0.f;
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        for (int x = tid; x < L * CB / 4; x += kThreads) {     // the thread's own copies
            const int r = x / (CB / 4), d = x % (CB / 4) * 4;
#pragma unroll
            for (int y = 0; y < 4; ++y)
                if (!(fabsf(sc[r * Sm::LC + d + y]) <= kMost)) {
                    sc[r * Sm::LC + d + y] = 0.f;
                    atomicMin(&s.first[d + y], rev ? len - 1 - (t0 + r) : t0 + r);
                }
        }
        __syncthreads();                                       // the tiles, the state's copy; the other tiles' readers are done
        if (ci + 1 < chunks) fetch(ci + 1);

        {   // P = (a b^T) o D: the warp's 16 rows and 32 columns, unless the mask leaves none of them
            const int r0 = 16 * (warp & 3), q0 = 32 * (warp >> 2);
            if (rev ? q0 + 31 >= r0 : q0 <= r0 + 15) {
                float acc[4][4] = {}, low[4][4] = {};
#pragma unroll 2
                for (int k0 = 0; k0 < DA; k0 += 8) {
                    float av[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) av[x] = sa[(r0 + g + 8 * (x & 1)) * Sm::LA + k0 + tg + 4 * (x >> 1)];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float bv[2] = {sb[(q0 + 8 * j + g) * Sm::LA + k0 + tg], sb[(q0 + 8 * j + g) * Sm::LA + k0 + tg + 4]};
                        mma3(acc[j], low[j], av, bv);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float f[4];                                // every power is read before the mask applies: no branches
#pragma unroll
                    for (int x = 0; x < 4; ++x) f[x] = s.pw[abs(r0 + g + 8 * (x >> 1) - (q0 + 8 * j + 2 * tg + (x & 1)))];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int t = r0 + g + 8 * (x >> 1), i = q0 + 8 * j + 2 * tg + (x & 1);
                        const float v = (acc[j][x] + low[j][x]) * (p.sp * f[x]);
                        s.P[t * Sm::LP + i] = (rev ? i >= t : i <= t) ? v : 0.f;
                    }
                }
            }
        }
        // out = e o (a S) + P c: 16 rows and CB / 2 columns, a S before P is there
        constexpr int TO = CB / 16;
        const int r0 = 16 * (warp & 3), q0 = (CB / 2) * (warp >> 2);
        float out[TO][4];
        {
            float acc[TO][4] = {}, low[TO][4] = {};
#pragma unroll 2
            for (int k0 = 0; k0 < DA; k0 += 8) {
                float av[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) av[x] = sa[(r0 + g + 8 * (x & 1)) * Sm::LA + k0 + tg + 4 * (x >> 1)];
#pragma unroll
                for (int j = 0; j < TO; ++j) {
                    float bv[2] = {s.S[(k0 + tg) * Sm::LC + q0 + 8 * j + g], s.S[(k0 + tg + 4) * Sm::LC + q0 + 8 * j + g]};
                    mma3(acc[j], low[j], av, bv);
                }
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int t = r0 + g + 8 * (x >> 1);
                const float e = p.se * s.pw[rev ? max(n - 1 - t, 0) : min(t + 1, L)];
#pragma unroll
                for (int j = 0; j < TO; ++j) out[j][x] = e * (acc[j][x] + low[j][x]);
            }
        }
        __syncthreads();                                       // P; and the state's copy is read
        {
            float acc[TO][4] = {}, low[TO][4] = {};
            const int k1 = rev ? L : r0 + 16;
            for (int k0 = rev ? r0 : 0; k0 < k1; k0 += 8) {
                float av[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) av[x] = s.P[(r0 + g + 8 * (x & 1)) * Sm::LP + k0 + tg + 4 * (x >> 1)];
#pragma unroll
                for (int j = 0; j < TO; ++j) {
                    float bv[2] = {sc[(k0 + tg) * Sm::LC + q0 + 8 * j + g], sc[(k0 + tg + 4) * Sm::LC + q0 + 8 * j + g]};
                    mma3(acc[j], low[j], av, bv);
                }
            }
#pragma unroll
            for (int j = 0; j < TO; ++j)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int t = r0 + g + 8 * x, col = q0 + 8 * j + 2 * tg;
                    if (t >= n) continue;
                    const int order = rev ? len - 1 - (t0 + t) : t0 + t;
                    float2 y = make_float2(out[j][2 * x] + (acc[j][2 * x] + low[j][2 * x]), out[j][2 * x + 1] + (acc[j][2 * x + 1] + low[j][2 * x + 1]));
                    if (order >= s.first[col]) y.x = __int_as_float(0x7fffffff);
                    if (order >= s.first[col + 1]) y.y = __int_as_float(0x7fffffff);
                    *reinterpret_cast<float2 *>(p.out + ((bt + t0 + t) * H + h) * DC + c0 + col) = y;
                }
        }
        {   // S <- g^n S + (w o b)^T c.  Weak decays through g^n - 1, whose rounding is not the same relative error chunk
            // after chunk.
            float acc[TS][4] = {}, low[TS][4] = {};
#pragma unroll 2
            for (int k0 = 0; k0 < L; k0 += 8) {
                float av[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int i = k0 + tg + 4 * (y >> 1);
                    av[y] = s.w[buf][i] * sb[i * Sm::LA + 16 * wr + g + 8 * (y & 1)];
                }
#pragma unroll
                for (int j = 0; j < TS; ++j) {
                    const int col = NS * wc + 8 * j + g;
                    float bv[2] = {sc[(k0 + tg) * Sm::LC + col], sc[(k0 + tg + 4) * Sm::LC + col]};
                    mma3(acc[j], low[j], av, bv);
                }
            }
#pragma unroll
            for (int j = 0; j < TS; ++j)
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    st[j][y] = (weak ? fmaf(st[j][y], gm, st[j][y]) : st[j][y] * gm) + (acc[j][y] + low[j][y]);
            keep_copy();
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

template <int DA, int DC, int CB>
cudaError_t launch_block(const LinearArgs &a, const Dev &d, int count, cudaStream_t stream)
{
    auto kernel = sfda_linear_f32_kernel<DA, DC, CB>;
    static_assert(sizeof(Smem<DA, CB>) <= 232448, "shared memory of a CTA");
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<DA, CB>));
    if (e != cudaSuccess) return e;
    kernel<<<dim3((unsigned)a.B * a.H, DC / CB, count), kThreads, sizeof(Smem<DA, CB>), stream>>>(d);
    return cudaGetLastError();
}

template <int DA, int DC>
cudaError_t launch_one(const LinearArgs &a, const Dev &d, int count, cudaStream_t stream)
{
    // wide blocks of columns repeat P less often, narrow ones fill the SMs
    const long long chains = (long long)a.B * a.H * count;
    if (chains * (DC / 16) <= 148) return launch_block<DA, DC, 16>(a, d, count, stream);
    if (chains * (DC / 32) <= 148) return launch_block<DA, DC, 32>(a, d, count, stream);
    return launch_block<DA, DC, 64>(a, d, count, stream);
}

}  // namespace

cudaError_t launch_linear_f32(const LinearArgs &a, const LinearPass *passes, int count, cudaStream_t stream, int *launches)
{
    for (int at = 0; at < count;) {
        const int DA = passes[at].DA, DC = passes[at].DC;
        Dev d = {};
        d.log_decay = a.log_decay;
        d.lens = a.lens;
        d.T = a.T;
        d.H = a.H;
        int n = 0;
        for (; at < count && passes[at].DA == DA && passes[at].DC == DC; ++at, ++n) {
            const LinearPass &x = passes[at];
            d.pass[n] = {static_cast<const float *>(x.a), static_cast<const float *>(x.b), static_cast<const float *>(x.c),
                         static_cast<float *>(x.out), x.s_in, x.s_out, x.Ha, x.Hb, x.Hc, x.reverse, x.s_in_t, x.sp, x.se, x.sw};
        }
        const cudaError_t e = DA == 128 ? (DC == 128 ? launch_one<128, 128>(a, d, n, stream) : launch_one<128, 64>(a, d, n, stream))
                                        : (DC == 128 ? launch_one<64, 128>(a, d, n, stream) : launch_one<64, 64>(a, d, n, stream));
        if (e != cudaSuccess) return e;
        if (launches) ++*launches;
    }
    return cudaSuccess;
}

}  // namespace sfda
