// Linear attention with a fixed decay for each head, bf16, on the tensor cores (see sfda_linear.h for the form).
//
// A CTA takes one (batch, head) pair of one pass, or a stretch of its time axis, and walks its chunks of 128 tokens:
//
//   A  = a b^T                 tcgen05, both operands as TMA left them
//   P  = A o D                 registers; rounded to bf16, back into tensor memory as the operand of
//   O2 = P c                   tcgen05 (c MN-major)
//   O1 = a S                   tcgen05; S as a bf16 copy of the fp32 state
//   U  = (w o b)^T c           tcgen05; w o b in two bf16 parts, so that the state keeps 2^-17 of it
//   out = e o O1 + O2,   S <- g^n S + U      registers, fp32
//
// D, e and w are powers of one number per head, so they are tables and per-thread constants.  The state lives in the
// registers of eight warps and takes U with fp32 additions: accumulators of the tensor core cut sums off instead of rounding
// them, which over thousands of tokens would be a bias.  U does not depend on the state, so the serial chain from chunk to
// chunk is only S <- g S + U, its bf16 copy and O1.
//
// Bound by memory (a, b, c read once, out written once).  Twenty warps: TMA, MMA, two idle, four for P and the output, eight for the
// state, four for w o b.  Two stages of (a, b, c); the high part of w o b replaces b, the low part a, once the products that
// read them are done.
#include <cuda.h>

#include "sfda_common.cuh"
#include "sfda_linear.h"
#include "sfda_tc_ptx.cuh"

namespace sfda {
namespace {

using namespace tc;

constexpr int C = 128;                       // tokens per chunk
constexpr int kThreads = 640;
constexpr int kNever = 0x7fffffff;
constexpr int kPairs = 4;                    // sets of `first` in use at a time (see there)
// warps: 0 TMA, 1 MMA, 4..7 P, 8..15 state, 16..19 keys
constexpr int kWarpP = 4, kWarpS = 8, kWarpK = 16;

enum { B_FULL = 0, B_EMPTY = 2, B_A = 4, B_QS, B_KHI, B_KLO, B_P, B_O, B_OFREE, B_S, B_U, kBars };

struct Pass {
    void *out;
    const float *s_in;
    float *s_out, *seg;          // seg: [pairs][nseg - 1][DA][DC] what earlier stretches leave, from a zero state
    int ma, mb, mc;              // tensor maps of a, b, c
    int sa, sb, sc;              // query heads that share a head of a, b, c
    int reverse, s_in_t, out_f32;
    float sp, se, sw;
};

struct alignas(64) Params {
    CUtensorMap map[4];
    Pass pass[3];
    const float *log_decay;
    const int *lens;
    uint32_t *status;
    int n_pass, T, H, pairs, nseg, cps, units, clear;     // cps: chunks of a stretch; clear: the call's first launch
};

// Shared memory: two stages of a, b, c and the bf16 state, then the small things.
template <int DA, int DC>
struct Layout {
    static constexpr int kA = C * DA * 2, kC = C * DC * 2, kStage = 2 * kA + kC;
    static constexpr int kS = 2 * kStage, kMisc = kS + DA * DC * 2;
};
struct Misc {
    unsigned long long bars[kBars];
    uint32_t tmem;
    volatile int abort;
    int any[kPairs];
    alignas(16) float col[32];
    float pw[C + 1];
    int first[kPairs][128];      // by value column: the first token (in the pass's order) whose value was not finite.  Four
                                 // sets, by unit: the keys' warps are at most two units ahead of the last reader
};
template <int DA, int DC>
constexpr int kSmem = Layout<DA, DC>::kMisc + (int)sizeof(Misc);

__device__ __forceinline__ bool wait_k(Misc &mi, int bar, int k)
{
    const uint32_t addr = smem_u32(&mi.bars[bar]), parity = (uint32_t)k & 1u;
    const uint32_t t0 = (uint32_t)clock();
    do {
        uint32_t ok;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}\n"
                     : "=r"(ok)
                     : "r"(addr), "r"(parity), "r"(20000u)
                     : "memory");
        if (ok) {
            chaos(addr + 77u);
            return true;
        }
    } while (!mi.abort && (uint32_t)clock() - t0 < 0x80000000u);
    mi.abort = 1;
    return false;
}
__device__ __forceinline__ bool wait_warp(Misc &mi, int bar, int k) { return __all_sync(0xffffffffu, wait_k(mi, bar, k) ? 1 : 0) != 0; }
__device__ __forceinline__ void arrive(Misc &mi, int bar)
{
    chaos(bar);
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&mi.bars[bar])) : "memory");
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t pred;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(pred));
    return pred != 0;
}
__device__ __forceinline__ void group_sync(int id, int threads) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// MN-major, 128-byte-swizzled operand: 8 rows of K by 64 elements to an atom of 1024 bytes, `ld` bytes from one block of 64 to
// the next.
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr, uint32_t ld)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(ld >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
constexpr uint32_t kMnA = 1u << 15, kMnB = 1u << 16;

// A unit of work: a stretch of the chunks of one pair in one pass.  The two reverse passes of a pair run side by side, for they
// read the same q and d_o.
struct Unit {
    int pass, pair, seg, b, h, len, lo, hi;    // chunks lo .. hi - 1 of the sequence
    __device__ __forceinline__ Unit(const Params &p, int u, bool states)
    {
        const int segs = states ? p.nseg - 1 : p.nseg, two = p.n_pass == 3 ? 2 * p.pairs : 0;
        int x = u / segs;
        seg = u % segs;
        if (x < two) {
            pass = 1 + (x & 1);
            pair = x >> 1;
        } else {
            x -= two;
            pass = p.n_pass == 3 ? 0 : x % p.n_pass;
            pair = p.n_pass == 3 ? x : x / p.n_pass;
        }
        b = pair / p.H;
        h = pair % p.H;
        len = p.lens ? min(max(p.lens[b], 0), p.T) : p.T;
        const int n = (len + C - 1) / C, j = p.pass[pass].reverse ? p.nseg - 1 - seg : seg;
        lo = min(j * p.cps, n);
        hi = min(lo + p.cps, n);
    }
    __device__ __forceinline__ int chunk(const Params &p, int i) const { return p.pass[pass].reverse ? hi - 1 - i : lo + i; }
    // tokens of the stretch that comes s-th in the pass's order
    __device__ __forceinline__ int tokens(const Params &p, int s) const
    {
        const int j = p.pass[pass].reverse ? p.nseg - 1 - s : s;
        return min(max(len - j * p.cps * C, 0), p.cps * C);
    }
};

template <int DA, int DC, bool kStates>
__device__ __forceinline__ void run_tma(unsigned char *smem, Misc &mi, const Params &p)
{
    using Lo = Layout<DA, DC>;
    int g = 0;
    for (int u = blockIdx.x; u < p.units; u += gridDim.x) {
        const Unit un(p, u, kStates);
        const Pass &ps = p.pass[un.pass];
        for (int i = 0; i < un.hi - un.lo; ++i, ++g) {
            const int st = g & 1, t0 = un.chunk(p, i) * C;
            unsigned char *at = smem + st * Lo::kStage;
            if (g >= 2 && !wait_warp(mi, B_EMPTY + st, (g >> 1) - 1)) return;
            if (elect_one()) {
                unsigned long long *bar = &mi.bars[B_FULL + st];
                mbar_expect_tx(bar, (kStates ? Lo::kA : 2 * Lo::kA) + Lo::kC);
#pragma unroll
                for (int x = 0; x < DA / 64; ++x) tma_load_4d(at + Lo::kA + x * C * 128, &p.map[ps.mb], bar, 64 * x, un.h / ps.sb, t0, un.b);
                if (!kStates)
#pragma unroll
                    for (int x = 0; x < DA / 64; ++x) tma_load_4d(at + x * C * 128, &p.map[ps.ma], bar, 64 * x, un.h / ps.sa, t0, un.b);
#pragma unroll
                for (int x = 0; x < DC / 64; ++x) tma_load_4d(at + 2 * Lo::kA + x * C * 128, &p.map[ps.mc], bar, 64 * x, un.h / ps.sc, t0, un.b);
            }
            __syncwarp();
        }
    }
}

template <int DA, int DC, bool kStates>
__device__ __forceinline__ void run_mma(unsigned char *smem, Misc &mi, const Params &p, uint32_t tmem)
{
    using Lo = Layout<DA, DC>;
    const uint32_t tA = tmem, tU = tmem + 128, tO1 = tmem + 256, tO2 = tmem + 384;
    const uint32_t base = smem_u32(smem);
    constexpr uint32_t kIdA = idesc(C, 0), kIdQS = idesc(DC, 0) | kMnB, kIdKV = idesc(DC, 0) | kMnA | kMnB;
    // DA = 64: the second 64 rows of U repeat the first
    constexpr uint32_t kLdK = DA == 128 ? C * 128 : 0, kLdC = C * 128, kLdS = DA * 128;
    int g = 0;
    for (int u = blockIdx.x; u < p.units; u += gridDim.x) {
        const Unit un(p, u, kStates);
        for (int i = 0; i < un.hi - un.lo; ++i, ++g) {
            const int st = g & 1;
            const uint32_t sa = base + st * Lo::kStage, sb = sa + Lo::kA, sc = sb + Lo::kA, ss = base + Lo::kS;
            if (!wait_warp(mi, B_FULL + st, g >> 1)) return;
            if (!kStates) {
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < DA / 16; ++k)
                        mma_ss(tA, smem_desc(sa + (k >> 2) * C * 128 + (k & 3) * 32), smem_desc(sb + (k >> 2) * C * 128 + (k & 3) * 32), kIdA, k > 0);
                    mma_commit(&mi.bars[B_A]);
                }
                __syncwarp();
            }
            if (!wait_warp(mi, B_S, g)) return;
            if (!kStates && g > 0 && !wait_warp(mi, B_OFREE, g - 1)) return;
            tc_fence_after();
            if (!kStates) {
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < DA / 16; ++k)
                        mma_ss(tO1, smem_desc(sa + (k >> 2) * C * 128 + (k & 3) * 32), desc_mn(ss + k * 2048, kLdS), kIdQS, k > 0);
                    mma_commit(&mi.bars[B_QS]);
                }
                __syncwarp();
            }
            if (!wait_warp(mi, B_KHI, g)) return;
            tc_fence_after();
            if (elect_one())
#pragma unroll
                for (int k = 0; k < C / 16; ++k) mma_ss(tU, desc_mn(sb + k * 2048, kLdK), desc_mn(sc + k * 2048, kLdC), kIdKV, k > 0);
            __syncwarp();
            if (!kStates) {
                if (!wait_warp(mi, B_P, g)) return;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < C / 16; ++k) mma_ts(tO2, tA + 8 * k, desc_mn(sc + k * 2048, kLdC), kIdQS, k > 0);
                    mma_commit(&mi.bars[B_O]);
                }
                __syncwarp();
            }
            if (!wait_warp(mi, B_KLO, g)) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < C / 16; ++k) mma_ss(tU, desc_mn(sa + k * 2048, kLdK), desc_mn(sc + k * 2048, kLdC), kIdKV, 1);
                mma_commit(&mi.bars[B_U]);
                mma_commit(&mi.bars[B_EMPTY + st]);
            }
            __syncwarp();
        }
    }
}

// P and the output: thread t has row t of the chunk
template <int DA, int DC>
__device__ __forceinline__ void run_p(Misc &mi, const Params &p, uint32_t tmem)
{
    const int t = threadIdx.x - kWarpP * 32, w = t >> 5;
    const uint32_t lane = tmem + ((uint32_t)(w * 32) << 16), tA = lane, tO1 = lane + 256, tO2 = lane + 384;
    bool live = true;                          // after a wait that ran out a warp only keeps the group's barriers company
    int g = 0, nth = 0;                        // chunks and units with chunks so far
    for (int u = blockIdx.x; u < p.units; u += gridDim.x) {
        const Unit un(p, u, false);
        const Pass &ps = p.pass[un.pass];
        const bool rev = ps.reverse != 0;
        const float ld = p.log_decay[un.h];
        if (un.hi == un.lo) continue;
        const int set = nth++ & (kPairs - 1);
        group_sync(1, 128);                    // the tables' readers are done with the last unit's
        mi.pw[t] = t == 0 ? 1.f : expf((float)t * ld);
        if (t == 0) mi.pw[C] = expf((float)C * ld);
        group_sync(1, 128);
        if (t < 32) mi.col[t] = rev ? mi.pw[t] : mi.pw[31 - t];
        group_sync(1, 128);
        for (int i = 0; i < un.hi - un.lo; ++i, ++g) {
            const int t0 = un.chunk(p, i) * C, n = min(C, un.len - t0);
            if (!(live = live && wait_warp(mi, B_A, g))) continue;
            tc_fence_after();
#pragma unroll 1
            for (int j = 0; j < 4; ++j) {
                uint32_t y[16];
                if (rev ? j < w : j > w) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) y[x] = 0;
                } else {
                    float v[32];
                    tmem_ld<32>(tA + 32 * j, reinterpret_cast<uint32_t *>(v));
                    tc_wait_ld();
                    if (j != w) {
                        const float row = ps.sp * mi.pw[rev ? 32 * j - t : t - (32 * j + 31)];
#pragma unroll
                        for (int x = 0; x < 32; x += 4) {
                            const float4 c = *reinterpret_cast<const float4 *>(&mi.col[x]);
                            v[x] *= row * c.x; v[x + 1] *= row * c.y; v[x + 2] *= row * c.z; v[x + 3] *= row * c.w;
                        }
                    } else {
                        const int tt = t & 31;
#pragma unroll
                        for (int x = 0; x < 32; ++x) {
                            const int gap = rev ? x - tt : tt - x;
                            v[x] = gap >= 0 ? v[x] * (ps.sp * mi.pw[gap & 31]) : 0.f;
                        }
                    }
                    if (rev && 32 * j + 32 > n)
#pragma unroll
                        for (int x = 0; x < 32; ++x) v[x] = 32 * j + x < n ? v[x] : 0.f;
#pragma unroll
                    for (int x = 0; x < 16; ++x) y[x] = pack_bf16(v[2 * x], v[2 * x + 1]);
                }
                tmem_st16(tA + 16 * j, y);     // the columns under it are read already
            }
            tc_wait_st();
            tc_fence_before();
            arrive(mi, B_P);
            if (!(live = wait_warp(mi, B_O, g))) continue;
            tc_fence_after();
            const float e = ps.se * mi.pw[rev ? max(n - 1 - t, 0) : t + 1];
            const bool bad = mi.any[set] != 0;
            const int order = rev ? un.len - 1 - (t0 + t) : t0 + t;
            const size_t row = (((size_t)un.b * p.T + t0 + t) * p.H + un.h) * DC;
#pragma unroll 1
            for (int j = 0; j < DC / 32; ++j) {
                float v[32], s[32];
                tmem_ld<32>(tO1 + 32 * j, reinterpret_cast<uint32_t *>(s));
                tmem_ld<32>(tO2 + 32 * j, reinterpret_cast<uint32_t *>(v));
                tc_wait_ld();
                if (j == DC / 32 - 1) {
                    tc_fence_before();
                    arrive(mi, B_OFREE);
                }
#pragma unroll
                for (int x = 0; x < 32; ++x) v[x] = fmaf(e, s[x], v[x]);
                if (bad)
#pragma unroll
                    for (int x = 0; x < 32; ++x)
                        if (order >= mi.first[set][32 * j + x]) v[x] = __int_as_float(0x7fffffff);
                if (t >= n) continue;
                if (ps.out_f32) {
                    float4 *o = reinterpret_cast<float4 *>(static_cast<float *>(ps.out) + row + 32 * j);
#pragma unroll
                    for (int x = 0; x < 8; ++x) o[x] = make_float4(v[4 * x], v[4 * x + 1], v[4 * x + 2], v[4 * x + 3]);
                } else {
                    uint4 *o = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(ps.out) + row + 32 * j);
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        o[x] = make_uint4(pack_bf16(v[8 * x], v[8 * x + 1]), pack_bf16(v[8 * x + 2], v[8 * x + 3]),
                                          pack_bf16(v[8 * x + 4], v[8 * x + 5]), pack_bf16(v[8 * x + 6], v[8 * x + 7]));
                }
            }
        }
    }
}

// The state: a thread has row k (its tensor memory lane) and half of the columns
template <int DA, int DC, bool kStates>
__device__ __forceinline__ void run_state(unsigned char *smem, Misc &mi, const Params &p, uint32_t tmem)
{
    using Lo = Layout<DA, DC>;
    constexpr int N = DC / 2;                  // columns of a thread
    const int id = threadIdx.x - kWarpS * 32, k = id & 127, c0 = (id >> 7) * N;
    const bool mine = k < DA;
    const uint32_t tU = tmem + 128 + c0 + ((uint32_t)(k & 96) << 16);
    const uint32_t ss = smem_u32(smem) + Lo::kS;
    int g = 0, nth = 0;                        // chunks and units with chunks so far
    for (int u = blockIdx.x; u < p.units; u += gridDim.x) {
        const Unit un(p, u, kStates);
        const Pass &ps = p.pass[un.pass];
        const float ld = p.log_decay[un.h];
        float s[N];
#pragma unroll
        for (int x = 0; x < N; ++x) s[x] = 0.f;
        if (!kStates && mine) {
            if (ps.s_in) {
                const size_t at = (size_t)un.pair * DA * DC;
                if (ps.s_in_t) {
#pragma unroll
                    for (int x = 0; x < N; ++x) s[x] = ps.s_in[at + (size_t)(c0 + x) * DA + k];
                } else {
#pragma unroll
                    for (int x = 0; x < N; x += 4) {
                        const float4 v = *reinterpret_cast<const float4 *>(ps.s_in + at + (size_t)k * DC + c0 + x);
                        s[x] = v.x; s[x + 1] = v.y; s[x + 2] = v.z; s[x + 3] = v.w;
                    }
                }
            }
#pragma unroll 1
            for (int j = 0; j < un.seg; ++j) {
                const int tok = un.tokens(p, j);
                if (tok == 0) continue;
                const float gn = expf((float)tok * ld);
                const float *from = ps.seg + ((size_t)un.pair * (p.nseg - 1) + j) * DA * DC + (size_t)k * DC + c0;
#pragma unroll
                for (int x = 0; x < N; x += 4) {
                    const float4 v = __ldcg(reinterpret_cast<const float4 *>(from + x));
                    s[x] = fmaf(gn, s[x], v.x); s[x + 1] = fmaf(gn, s[x + 1], v.y);
                    s[x + 2] = fmaf(gn, s[x + 2], v.z); s[x + 3] = fmaf(gn, s[x + 3], v.w);
                }
            }
        }
        const int chunks = un.hi - un.lo;
        nth += chunks > 0;
        for (int i = 0; i <= chunks; ++i) {
            if (i > 0) {
                const int n = min(C, un.len - un.chunk(p, i - 1) * C);
                // weak decays through g^n - 1, whose rounding is not the same relative error chunk after chunk
                const float x0 = (float)n * ld;
                const bool weak = x0 > -0.5f;
                const float gm = weak ? expm1f(x0) : expf(x0);
                if (!wait_warp(mi, B_U, g)) return;
                tc_fence_after();
                ++g;
#pragma unroll
                for (int x = 0; x < N; x += 16) {
                    float v[16];
                    tmem_ld<16>(tU + x, reinterpret_cast<uint32_t *>(v));
                    tc_wait_ld();
#pragma unroll
                    for (int y = 0; y < 16; ++y) s[x + y] = weak ? fmaf(gm, s[x + y], s[x + y]) + v[y] : fmaf(gm, s[x + y], v[y]);
                }
                tc_fence_before();
            }
            if (i == chunks) break;
            if (!kStates && mine) {
#pragma unroll
                for (int x = 0; x < N; x += 8) {
                    const int col = c0 + x;
                    sts128(ss + (col >> 6) * (DA * 128) + sw_off(k, col & 63), pack_bf16(s[x], s[x + 1]), pack_bf16(s[x + 2], s[x + 3]),
                           pack_bf16(s[x + 4], s[x + 5]), pack_bf16(s[x + 6], s[x + 7]));
                }
            }
            if (!kStates) fence_async_smem();
            arrive(mi, B_S);
        }
        float *to = kStates ? ps.seg + ((size_t)un.pair * (p.nseg - 1) + un.seg) * DA * DC
                            : un.seg == p.nseg - 1 && ps.s_out ? ps.s_out + (size_t)un.pair * DA * DC : nullptr;
        if (to && mine) {
            const int set = (nth - 1) & (kPairs - 1);
            if (chunks > 0 && mi.any[set])
#pragma unroll
                for (int x = 0; x < N; ++x)
                    if (mi.first[set][c0 + x] != kNever) s[x] = __int_as_float(0x7fffffff);
#pragma unroll
            for (int x = 0; x < N; x += 4)
                *reinterpret_cast<float4 *>(to + (size_t)k * DC + c0 + x) = make_float4(s[x], s[x + 1], s[x + 2], s[x + 3]);
        }
    }
}

// w o b in two parts, and c made safe: thread r has token r of the chunk
template <int DA, int DC, bool kStates>
__device__ __forceinline__ void run_keys(unsigned char *smem, Misc &mi, const Params &p)
{
    using Lo = Layout<DA, DC>;
    const int r = threadIdx.x - kWarpK * 32;
    const uint32_t base = smem_u32(smem);
    bool live = true;                          // as in run_p
    int g = 0, nth = 0;                        // chunks and units with chunks so far
    for (int u = blockIdx.x; u < p.units; u += gridDim.x) {
        const Unit un(p, u, kStates);
        const Pass &ps = p.pass[un.pass];
        const bool rev = ps.reverse != 0;
        const float ld = p.log_decay[un.h];
        const int chunks = un.hi - un.lo;
        if (chunks == 0) continue;
        const int set = nth++ & (kPairs - 1);
        mi.first[set][r] = kNever;
        if (r == 0) mi.any[set] = 0;
        group_sync(2, 128);
        for (int i = 0; i < chunks; ++i, ++g) {
            const int st = g & 1, t0 = un.chunk(p, i) * C, n = min(C, un.len - t0);
            const uint32_t sa = base + st * Lo::kStage, sb = sa + Lo::kA, sc = sb + Lo::kA;
            if (!(live = live && wait_warp(mi, B_FULL + st, g >> 1))) continue;
            uint32_t odd = 0;
#pragma unroll
            for (int x = 0; x < DC; x += 8) {
                const uint4 v = lds128(sc + (x >> 6) * C * 128 + sw_off(r, x & 63));
                odd |= ((v.x & 0x7fff7fffu) + 0x00800080u) | ((v.y & 0x7fff7fffu) + 0x00800080u) | ((v.z & 0x7fff7fffu) + 0x00800080u) |
                       ((v.w & 0x7fff7fffu) + 0x00800080u);
            }
            if (r >= n) {                      // behind the end: whatever is there is no value
#pragma unroll 1
                for (int x = 0; x < DC; x += 8) sts128(sc + (x >> 6) * C * 128 + sw_off(r, x & 63), 0, 0, 0, 0);
            } else if (odd & 0x80008000u) {
#pragma unroll 1
                for (int x = 0; x < DC; ++x) {
                    const uint32_t at = sc + (x >> 6) * C * 128 + sw_off(r, x & 63);
                    if ((lds16(at) & 0x7f80u) == 0x7f80u) {
                        sts16(at, 0);
                        atomicMin(&mi.first[set][x], rev ? un.len - 1 - (t0 + r) : t0 + r);
                        mi.any[set] = 1;
                    }
                }
            }
            const int hops = rev ? r + 1 : n - 1 - r;
            const float w = r < n ? ps.sw * (hops == 0 ? 1.f : expf((float)hops * ld)) : 0.f;
            if (!kStates && !(live = wait_warp(mi, B_A, g))) continue;
            uint32_t lo[DA / 2];
#pragma unroll
            for (int x = 0; x < DA; x += 8) {
                const uint32_t at = sb + (x >> 6) * C * 128 + sw_off(r, x & 63);
                const uint4 v = lds128(at);
                const uint32_t in[4] = {v.x, v.y, v.z, v.w};
                uint32_t hi[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float f0 = r < n ? w * __uint_as_float(in[y] << 16) : 0.f, f1 = r < n ? w * __uint_as_float(in[y] & 0xffff0000u) : 0.f;
                    hi[y] = pack_bf16(f0, f1);
                    lo[x / 2 + y] = pack_bf16(f0 - __uint_as_float(hi[y] << 16), f1 - __uint_as_float(hi[y] & 0xffff0000u));
                }
                sts128(at, hi[0], hi[1], hi[2], hi[3]);
            }
            fence_async_smem();
            arrive(mi, B_KHI);
            if (!kStates && !(live = wait_warp(mi, B_QS, g))) continue;
#pragma unroll
            for (int x = 0; x < DA; x += 8)
                sts128(sa + (x >> 6) * C * 128 + sw_off(r, x & 63), lo[x / 2], lo[x / 2 + 1], lo[x / 2 + 2], lo[x / 2 + 3]);
            fence_async_smem();
            arrive(mi, B_KLO);
        }
    }
}

template <int DA, int DC, bool kStates>
__global__ void __launch_bounds__(kThreads, 1) sfda_linear_tc_kernel(const __grid_constant__ Params p)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    Misc &mi = *reinterpret_cast<Misc *>(smem + Layout<DA, DC>::kMisc);
    const int tid = threadIdx.x, warp = tid >> 5;
    if (tid == 0) {
        const int counts[kBars] = {1, 1, 1, 1, 1, 1, 128, 128, 128, 1, 128, 256, 1};
        for (int i = 0; i < kBars; ++i) mbar_init(&mi.bars[i], counts[i]);
        mi.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (p.clear && blockIdx.x == 0) *p.status = 0;      // what an earlier call left there; a wait runs out much later
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&mi.tmem)));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = mi.tmem;
    if (warp == 0) run_tma<DA, DC, kStates>(smem, mi, p);
    else if (warp == 1) run_mma<DA, DC, kStates>(smem, mi, p, tmem);
    else if (warp >= kWarpK) run_keys<DA, DC, kStates>(smem, mi, p);
    else if (warp >= kWarpS) run_state<DA, DC, kStates>(smem, mi, p, tmem);
    else if (warp >= kWarpP && !kStates) run_p<DA, DC>(mi, p, tmem);
    tc_fence_before();
    __syncthreads();
    if (mi.abort) {
        // a wait ran out: before shared and tensor memory are given back, the copies and products in flight get the time to end
        // (microseconds; there is nothing left to wait on, for the stages' barriers may be the ones that are stuck)
        __nanosleep(200000);
        __syncthreads();
        if (tid == 0) atomicExch(p.status, 1u);
    }
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// ---- host side -----------------------------------------------------------------------------------------------------

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeTiledFn>(f);
    }();
    return fn;
}
// [B][T][H][d] bf16, a box of 128 tokens by 64 channels of one head; tokens behind T are read as zeros
bool make_map(CUtensorMap *map, const void *base, int B, int T, int H, int d)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t row = (cuuint64_t)d * 2;
    const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)H, (cuuint64_t)T, (cuuint64_t)B};
    const cuuint64_t strides[3] = {row, (cuuint64_t)H * row, (cuuint64_t)T * H * row};
    const cuuint32_t box[4] = {64, 1, C, 1}, estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sm_count()
{
    int dev = 0, n = 148;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) n = 148;
    return n;
}

template <int DA, int DC, bool kStates>
cudaError_t launch_kernel(Params &p, cudaStream_t stream, int *launches)
{
    auto kernel = sfda_linear_tc_kernel<DA, DC, kStates>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<DA, DC>);
    if (e != cudaSuccess) return e;
    p.units = p.n_pass * p.pairs * (kStates ? p.nseg - 1 : p.nseg);
    const int n = sm_count();
    kernel<<<p.units < n ? p.units : n, kThreads, kSmem<DA, DC>, stream>>>(p);
    e = cudaGetLastError();
    if (e == cudaSuccess && launches) ++*launches;
    p.clear = 0;
    return e;
}
template <int DA, int DC>
cudaError_t launch_one(Params &p, cudaStream_t stream, int *launches)
{
    static_assert(kSmem<DA, DC> <= 232448, "shared memory of a CTA");
    if (p.nseg > 1) {
        const cudaError_t e = launch_kernel<DA, DC, true>(p, stream, launches);
        if (e != cudaSuccess) return e;
    }
    return launch_kernel<DA, DC, false>(p, stream, launches);
}

}  // namespace

// How many stretches each sequence is cut into, for `chains` of `chunks` chunks on n SMs.  In units of a chunk's share of the
// memory's time on n SMs: a CTA alone needs at least kAlone of it; a cut costs a pass over b and c, and a unit its start.
static int stretches(long long chains, int chunks, int n)
{
    constexpr double kAlone = 0.6, kStart = 1.0, kLaunch = 1.5;
    const auto waves = [n](long long units) { return (double)((units + n - 1) / n); };
    int best = 1;
    double least = 0;
    for (int s = 1; s <= chunks && s <= 64; ++s) {
        const int cps = (chunks + s - 1) / s;
        if ((chunks + cps - 1) / cps != s) continue;
        double t = waves(chains * s) * (cps * kAlone + kStart);
        const double mem = (double)chains * chunks / n;
        if (t < mem) t = mem;
        if (s > 1) {
            double a = waves(chains * (s - 1)) * (cps * 0.5 * kAlone + kStart);
            if (a < 0.5 * mem) a = 0.5 * mem;
            t += a + kLaunch;
        }
        if (s == 1 || t < least) {
            least = t;
            best = s;
        }
    }
    return best;
}

namespace {

// Passes of one launch: all of them where their widths agree, otherwise the first two (dq, dk) and the third (dv).
int group_of(const LinearPass *passes, int count)
{
    for (int i = 1; i < count; ++i)
        if (passes[i].DA != passes[0].DA || passes[i].DC != passes[0].DC) return i;
    return count;
}
size_t scratch_of(const LinearArgs &a, int passes, int d_k, int d_v, int *nseg)
{
    const long long pairs = (long long)a.B * a.H;
    *nseg = stretches(pairs * passes, (a.T + C - 1) / C, 148);
    return (size_t)passes * pairs * (*nseg - 1) * d_k * d_v * 4;
}

}  // namespace

size_t linear_tc_bytes(const LinearArgs &a, int passes, int d_k, int d_v)
{
    int nseg;
    if (passes == 1 || d_k == d_v) return 256 + scratch_of(a, passes, d_k, d_v, &nseg);
    const size_t two = scratch_of(a, 2, d_k, d_v, &nseg), one = scratch_of(a, 1, d_k, d_v, &nseg);
    return 256 + (two > one ? two : one);
}

cudaError_t launch_linear_tc(const LinearArgs &a, const LinearPass *passes, int count, void *workspace, cudaStream_t stream, int *launches)
{
    Params p;
    p.log_decay = a.log_decay;
    p.lens = a.lens;
    p.status = static_cast<uint32_t *>(workspace);
    p.T = a.T;
    p.H = a.H;
    p.pairs = a.B * a.H;
    p.clear = 1;
    float *seg = reinterpret_cast<float *>(static_cast<char *>(workspace) + 256);
    for (int at = 0; at < count;) {
        p.n_pass = group_of(passes + at, count - at);
        const int DA = passes[at].DA, DC = passes[at].DC;
        const size_t each = (size_t)p.pairs * DA * DC;
        scratch_of(a, p.n_pass, DA, DC, &p.nseg);
        const int chunks = (a.T + C - 1) / C;
        p.cps = (chunks + p.nseg - 1) / p.nseg;
        const void *seen[4] = {};
        int heads[4] = {}, maps = 0;
        auto map_of = [&](const void *x, int h, int d) {
            for (int i = 0; i < maps; ++i)
                if (seen[i] == x && heads[i] == h) return i;
            if (maps == 4 || !make_map(&p.map[maps], x, a.B, a.T, h, d)) return -1;
            seen[maps] = x;
            heads[maps] = h;
            return maps++;
        };
        for (int i = 0; i < p.n_pass; ++i) {
            const LinearPass &x = passes[at + i];
            Pass &y = p.pass[i];
            y.out = x.out; y.s_in = x.s_in; y.s_out = x.s_out;
            y.seg = seg + i * each * (p.nseg - 1);
            y.ma = map_of(x.a, x.Ha, DA); y.mb = map_of(x.b, x.Hb, DA); y.mc = map_of(x.c, x.Hc, DC);
            if (y.ma < 0 || y.mb < 0 || y.mc < 0) return cudaErrorInvalidValue;
            y.sa = a.H / x.Ha; y.sb = a.H / x.Hb; y.sc = a.H / x.Hc;
            y.reverse = x.reverse; y.s_in_t = x.s_in_t; y.out_f32 = x.out_f32;
            y.sp = x.sp; y.se = x.se; y.sw = x.sw;
        }
        const cudaError_t e = DA == 128 ? (DC == 128 ? launch_one<128, 128>(p, stream, launches) : launch_one<128, 64>(p, stream, launches))
                                        : (DC == 128 ? launch_one<64, 128>(p, stream, launches) : launch_one<64, 64>(p, stream, launches));
        if (e != cudaSuccess) return e;
        at += p.n_pass;
    }
    return cudaSuccess;
}

}  // namespace sfda
