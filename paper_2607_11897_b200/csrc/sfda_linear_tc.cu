// Linear attention with a fixed decay for each head, bf16, on the tensor cores (see sfda_linear.h for the form).
//
// A CTA takes one (batch, head) pair of one pass, or a stretch of its time axis, and walks its chunks of 128 tokens:
//
//   A = a b^T                        tcgen05, both operands as TMA left them
//   P = A o D                        registers; rounded to bf16, back into tensor memory as an operand
//   O = a S,  O += P c               tcgen05; S as a bf16 copy of the fp32 state, c MN-major
//   U = (w o b)^T c                  tcgen05; w o b in two bf16 parts, through tensor memory (run_keys)
//   out = e o O,  S <- g^n S + U     registers, fp32
//
// D, e and w are powers of one number per head, so they are tables and per-thread constants; `shares` says how e gets out of P.
// The state lives in the registers of eight warps and takes U with fp32 additions: accumulators of the tensor core cut sums off
// instead of rounding them, which over thousands of tokens would be a bias.  U does not depend on the state, so the serial chain from
// chunk to chunk is S <- g S + U, its bf16 copy and a S.
//
// Memory is the floor (a, b, c read once, out written once: B = 8, T = 8192, H = 32, d = 128 take 336 us at 6.5 TB/s).  28 warps: TMA,
// MMA, output copies, one idle, eight each for P and the output, for the state and for w o b.  Two stages of b and c; one place for a,
// loaded out of L2 as soon as a S is done with it; one for the output.  Measured 457 us (4.7 TB/s) in bursts and 538 us under
// sustained load, when the clock falls: the chain P, P c, output of a chunk (5000 cycles) and the issue of its 10500 warp
// instructions are what is left above memory, and that 256 equal chains make two waves of 148 SMs.  Before: outputs stored by the
// warps themselves 841 us (32 rows of a warp lie in 32 lines), descriptors computed per instruction 668, w o b through shared
// memory 562 (its bandwidth is what the products compete for).
#include <cuda.h>
#include <stdlib.h>

#include "sfda_common.cuh"
#include "sfda_linear.h"
#include "sfda_tc_ptx.cuh"

namespace sfda {
namespace {

using namespace tc;

constexpr int C = 128;                       // tokens per chunk
constexpr int kThreads = 896;
constexpr int kNever = 0x7fffffff;
constexpr int kSets = 3;                     // sets of `first` in use at a time (see there)
// warps: 0 TMA, 1 MMA, 2 output copies, 4..11 P, 12..19 state, 20..27 keys; registers of a thread of each group (the launch gives 72 to every
// thread, 504 to seven threads of different groups of four warps, which is what these come to)
constexpr int kWarpP = 4, kWarpS = 12, kWarpK = 20;
constexpr int kRegsLaunch = 72, kRegsCtrl = 40, kRegsP = 72, kRegsS = 96, kRegsK = 64;
static_assert(kRegsCtrl + 2 * (kRegsP + kRegsS + kRegsK) <= 7 * kRegsLaunch, "setmaxnreg draws on the launch's registers");

// tensor memory: A (and P over it), U, O, the two parts of w o b
constexpr uint32_t kColA = 0, kColU = 128, kColO = 256, kColK = 384;

enum { B_FULL = 0, B_EMPTY = 2, B_FULLA = 4, B_EMPTYA, B_EMPTYO, B_A, B_QS, B_K, B_U, B_P, B_O, B_OFREE, B_OUT, B_S, B_E, kBars };

struct Pass {
    void *out;
    const float *s_in;
    float *s_out, *seg;          // seg: [pairs][nseg][DA][DC], where sequences are cut: what the stretches but the last leave (the
                                 // first from s_in, the others from zero), and a copy of s_in: s_out may be s_in, and is
                                 // written while other stretches of the pair begin
    int ma, mb, mc;              // tensor maps of a, b, c
    int sa, sb, sc;              // query heads that share a head of a, b, c
    int reverse, s_in_t, out_f32;
    float sp, se, sw;
};

struct alignas(64) Params {
    CUtensorMap map[4], out[3];  // inputs; outputs of the passes
    Pass pass[3];
    const float *log_decay;
    const int *lens;
    uint32_t *status;
    int n_pass, T, H, pairs, nseg, cps, units, clear;     // cps: chunks of a stretch; clear: the call's first launch
#ifdef SFDA_WS_CHAOS
    int withhold;
#endif
};

// Shared memory: a, two stages of b and c, the bf16 state, the output on its way out, then the small things.
template <int DA, int DC>
struct Layout {
    static constexpr int kA = C * DA * 2, kC = C * DC * 2, kStage = kA + kC;
    static constexpr int kS = kA + 2 * kStage, kOut = kS + DA * DC * 2, kMisc = kOut + kC;
};
struct Misc {
    unsigned long long bars[kBars];
    uint32_t tmem;
    volatile int abort;
#ifdef SFDA_WS_CHAOS
    int withhold;
#endif
    int any[kSets];
    alignas(16) float pw[31 + C];// the powers of g that make P (see run_p)
    int first[kSets][128];      // by value column: the first token (in the pass's order) whose value was not finite.  Three
                                 // sets, by unit: the keys' warps are at most two units ahead of the last reader
};
template <int DA, int DC>
constexpr int kSmem = Layout<DA, DC>::kMisc + (int)sizeof(Misc);

// Wait for completion number k of a barrier, with one outcome for the warp.  try_wait parks the warp in hardware for up to 20 us
// at a time; after kTries of them (seconds), or when another wait of the CTA has given up, it gives up and says so.  A few
// instructions, for it is inlined at every wait: the loops of all roles have to stay in the SM's instruction cache together.
constexpr int kTries = 1 << 17;
#ifdef SFDA_WS_CHAOS
// Development builds only: with SFDA_WITHHOLD_LINEAR in the environment no warp arrives at the barrier of that number, and the limit is
// short (milliseconds), so that waits run out.
__device__ __forceinline__ bool withheld(const Misc &mi, int bar) { return mi.withhold == bar; }
__device__ __forceinline__ int tries(const Misc &mi) { return mi.withhold < 0 ? kTries : 1 << 9; }
#else
__device__ __forceinline__ bool withheld(const Misc &, int) { return false; }
__device__ __forceinline__ int tries(const Misc &) { return kTries; }
#endif
__device__ __forceinline__ bool wait_warp(Misc &mi, int bar, int k)
{
    const uint32_t addr = smem_u32(&mi.bars[bar]), parity = (uint32_t)k & 1u;
#pragma unroll 1
    for (int n = 0; n < tries(mi); ++n) {
        uint32_t ok;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}\n"
                     : "=r"(ok)
                     : "r"(addr), "r"(parity), "r"(20000u)
                     : "memory");
        if (__all_sync(0xffffffffu, ok)) {
            chaos(addr + 77u);
            return true;
        }
        if (__any_sync(0xffffffffu, mi.abort)) break;
    }
    mi.abort = 1;
    return false;
}
// whether it has come already
__device__ __forceinline__ bool ready(Misc &mi, int bar, int k)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok)
                 : "r"(smem_u32(&mi.bars[bar])), "r"((uint32_t)k & 1u)
                 : "memory");
    return __all_sync(0xffffffffu, ok) != 0;
}
__device__ __forceinline__ void arrive(Misc &mi, int bar)
{
    chaos(bar);
    if (withheld(mi, bar)) return;
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&mi.bars[bar])) : "memory");
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t pred;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(pred));
    return pred != 0;
}
// Four 8 x 8 blocks of 16-bit elements, transposed: lane l gives the address of row l % 8 of block l / 8; register k of thread T
// holds (column T / 4; rows 2 (T % 4), + 1) of block k.
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t saddr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(saddr)
                 : "memory");
}
// 16 lanes x 16 columns: registers 2 i, 2 i + 1 of thread T are column 4 i + T % 4 of lanes T / 4, T / 4 + 8.
__device__ __forceinline__ void tmem_st_16x128b_x4(uint32_t addr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
template <int N>
__device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// two fp32 values in one instruction
__device__ __forceinline__ uint64_t two(float x, float y)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void apart(uint64_t v, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack2(uint64_t v)
{
    float x, y;
    apart(v, x, y);
    return pack_bf16(x, y);
}
__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
// the larger magnitudes; not finite once one of them is not
__device__ __forceinline__ uint32_t max_abs_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("{\n.reg .b32 x;\nabs.bf16x2 x, %1;\nmax.NaN.bf16x2 %0, x, %2;\n}\n" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ void group_sync(int id, int threads) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// Operand descriptors as two 32-bit halves, of which only the lower one moves along K: the issuing thread spends one addition of
// a constant on an instruction.  K-major (rows of 128 swizzled bytes): 32 bytes per 16 elements of K.  MN-major (atoms of 8
// rows of K by 64 elements, `ld` bytes from one block of 64 to the next): 2048 bytes per 16.
constexpr uint32_t kDescHi = (1024u >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_k(uint32_t saddr) { return saddr >> 4 | 1u << 16; }
__device__ __forceinline__ uint32_t desc_mn(uint32_t saddr, uint32_t ld) { return saddr >> 4 | (ld >> 4) << 16; }
constexpr uint32_t kStepMn = 2048 >> 4;
__device__ __forceinline__ constexpr uint32_t step_k(int k) { return (uint32_t)((k >> 2) * (C * 128 >> 4) + (k & 3) * 2); }   // tiles of C rows
constexpr uint32_t kMnB = 1u << 16;           // instruction descriptor: B is MN-major

// out_t = e_t (a_t S + sum_i (P_ti / e_t) c_i): with P / e the two products share an accumulator, and P / e needs no power of the
// row at all, only (sp / se) g^-(i + 1) (reverse: g^(i - n + 1)) of the column.  These stay below 2^40 for g >= 0.805; for heads
// that forget faster a S is multiplied by e in the accumulator before P c is added.
__device__ __forceinline__ bool shares(float log_decay, const Pass &ps) { return log_decay >= -0.2166f && ps.se != 0.f; }

// g^n; the zeroth power of a decay that forgets all is 1 too
__device__ __forceinline__ float power(float log_decay, int n) { return n == 0 ? 1.f : expf((float)n * log_decay); }

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

// The chunks of a CTA one after another
struct Cursor {
    int u, i;
    bool states;
    Unit un;
    __device__ __forceinline__ Cursor(const Params &p, bool st) : u(blockIdx.x), i(0), states(st), un(p, min((int)blockIdx.x, p.units - 1), st) { skip(p); }
    __device__ __forceinline__ void skip(const Params &p)      // units without a chunk
    {
        while (u < p.units && i >= un.hi - un.lo) {
            u += gridDim.x;
            i = 0;
            if (u < p.units) un = Unit(p, u, states);
        }
    }
    __device__ __forceinline__ void next(const Params &p) { ++i; skip(p); }
};

__device__ __forceinline__ void prefetch_4d(const CUtensorMap *map, int c0, int c1, int c2, int c3)
{
    asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global [%0, {%1, %2, %3, %4}];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1),
                 "r"(c2), "r"(c3)
                 : "memory");
}

// b and c of a chunk are loaded a chunk ahead.  a has one place, which is free from a S on: it is loaded then, out of L2, where it
// was asked for together with b and c.
template <int DA, int DC, bool kStates>
__device__ __forceinline__ void run_tma(unsigned char *smem, Misc &mi, const Params &p)
{
    using Lo = Layout<DA, DC>;
    Cursor next(p, kStates);                   // whose b and c are loaded
    int gn = 0;
    const auto load_bc = [&]() -> bool {
        if (next.u >= p.units) return true;
        const Unit &un = next.un;
        const Pass &ps = p.pass[un.pass];
        const int st = gn & 1, t0 = un.chunk(p, next.i) * C;
        unsigned char *at = smem + Lo::kA + st * Lo::kStage;
        if (gn >= 2 && !wait_warp(mi, B_EMPTY + st, (gn >> 1) - 1)) return false;
        if (elect_one()) {
            unsigned long long *bar = &mi.bars[B_FULL + st];
            mbar_expect_tx(bar, Lo::kStage);
#pragma unroll
            for (int x = 0; x < DA / 64; ++x) tma_load_4d(at + x * C * 128, &p.map[ps.mb], bar, 64 * x, un.h / ps.sb, t0, un.b);
#pragma unroll
            for (int x = 0; x < DC / 64; ++x) tma_load_4d(at + Lo::kA + x * C * 128, &p.map[ps.mc], bar, 64 * x, un.h / ps.sc, t0, un.b);
            if (!kStates)
#pragma unroll
                for (int x = 0; x < DA / 64; ++x) prefetch_4d(&p.map[ps.ma], 64 * x, un.h / ps.sa, t0, un.b);
        }
        __syncwarp();
        next.next(p);
        ++gn;
        return true;
    };
    if (!load_bc()) return;
    int g = 0;
    for (Cursor cur(p, kStates); cur.u < p.units; cur.next(p), ++g) {
        if (!kStates) {
            const Unit &un = cur.un;
            const Pass &ps = p.pass[un.pass];
            if (g >= 1 && !wait_warp(mi, B_EMPTYA, g - 1)) return;
            if (elect_one()) {
                unsigned long long *bar = &mi.bars[B_FULLA];
                mbar_expect_tx(bar, Lo::kA);
#pragma unroll
                for (int x = 0; x < DA / 64; ++x) tma_load_4d(smem + x * C * 128, &p.map[ps.ma], bar, 64 * x, un.h / ps.sa, un.chunk(p, cur.i) * C, un.b);
            }
            __syncwarp();
        }
        if (!load_bc()) return;
    }
}

template <int DA, int DC, bool kStates>
__device__ __forceinline__ void run_mma(unsigned char *smem, Misc &mi, const Params &p, uint32_t tmem)
{
    using Lo = Layout<DA, DC>;
    const uint32_t tA = tmem + kColA, tU = tmem + kColU, tO = tmem + kColO, tK = tmem + kColK;
    const uint32_t base = smem_u32(smem);
    constexpr uint32_t kIdA = idesc(C, 0), kIdC = idesc(DC, 0) | kMnB;
    constexpr uint32_t kLdC = C * 128, kLdS = DA * 128;
    const uint32_t ss = desc_mn(base + Lo::kS, kLdS);
    int g = 0, parts = 0;                      // chunks so far, and those whose a S is multiplied by e
    for (Cursor cur(p, kStates); cur.u < p.units; cur.next(p), ++g) {
        const int st = g & 1;
        const uint32_t at = base + Lo::kA + st * Lo::kStage;
        const uint32_t a = desc_k(base), b = desc_k(at), c = desc_mn(at + Lo::kA, kLdC);
        if (!wait_warp(mi, B_FULL + st, g >> 1)) return;
        if (!kStates) {
            if (!wait_warp(mi, B_FULLA, g)) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < DA / 16; ++k) mma_ss2(tA, a + step_k(k), kDescHi, b + step_k(k), kDescHi, kIdA, k > 0);
                mma_commit(&mi.bars[B_A]);
            }
            __syncwarp();
        }
        if (!wait_warp(mi, B_S, g)) return;                      // S is there, and U is read
        if (!kStates) {
            if (g > 0 && !wait_warp(mi, B_OFREE, g - 1)) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < DA / 16; ++k) mma_ss2(tO, a + step_k(k), kDescHi, ss + k * kStepMn, kDescHi, kIdC, k > 0);
                mma_commit(&mi.bars[B_QS]);
                mma_commit(&mi.bars[B_EMPTYA]);
            }
            __syncwarp();
        }
        // U, and P c as soon as P is ready: the next a S waits for the state that takes U, and for the output to be read, which
        // takes longer.  (B_K also says that c is safe.)
        if (!wait_warp(mi, B_K, g)) return;
        const bool one = kStates || shares(p.log_decay[cur.un.h], p.pass[cur.un.pass]);
        bool u = kStates || !one || !ready(mi, B_P, g), o = kStates;
        while (true) {
            tc_fence_after();
            if (u) {
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 2 * C / 16; ++k) mma_ts2(tU, tK + 8 * k, c + (k & (C / 16 - 1)) * kStepMn, kDescHi, kIdC, k > 0);
                    mma_commit(&mi.bars[B_U]);
                }
                __syncwarp();
                if (o) break;
            }
            if (!wait_warp(mi, B_P, g) || (!one && !wait_warp(mi, B_E, parts++))) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < C / 16; ++k) mma_ts2(tO, tA + (k >> 2) * 64 + (k & 3) * 8, c + k * kStepMn, kDescHi, kIdC, 1);
                mma_commit(&mi.bars[B_O]);
            }
            __syncwarp();
            if (u) break;
            u = o = true;
        }
        if (elect_one()) mma_commit(&mi.bars[B_EMPTY + st]);
        __syncwarp();
    }
}

// Outputs leave through shared memory and a tensor copy (32 rows of a warp's own stores lie in 32 different lines, which cost
// 4000 of 7300 cycles of a chunk); not those in fp32, which have no room there, nor a sequence's last rows where other rows follow
// that have to stay as they are.
__device__ __forceinline__ bool store_directly(const Params &p, const Pass &ps, int t0, int n) { return ps.out_f32 || (n < C && t0 + n < p.T); }

// The output: a thread has row t of the chunk and one half of the columns.  False: a wait ran out.
template <int DA, int DC>
__device__ __forceinline__ bool write_out(unsigned char *smem, Misc &mi, const Params &p, uint32_t tmem, const Unit &un, int g, int t0, int n, int set, float e)
{
    const int id = threadIdx.x - kWarpP * 32, t = id & 127, half = id >> 7;
    const uint32_t tO = tmem + kColO + (DC / 2) * half + ((uint32_t)(t & 96) << 16);
    const Pass &ps = p.pass[un.pass];
    if (!wait_warp(mi, B_O, g)) return false;                // (every product of the chunk is done)
    tc_fence_after();
    const bool bad = mi.any[set] != 0, direct = store_directly(p, ps, t0, n);
    const uint32_t stage = smem_u32(smem) + Layout<DA, DC>::kOut;
    // the place is free, and the copying warp has seen the last completion of B_OUT
    if (g > 0 && !wait_warp(mi, B_EMPTYO, g - 1)) return false;
    if (!bad && !direct) {
        const uint64_t ee = two(e, e);
#pragma unroll 1
        for (int j = 0; j < DC / 2; j += 32) {
            const int col = (DC / 2) * half + j;
            const uint32_t at = stage + (col >> 6) * C * 128;
            float v[32];
            tmem_ld<32>(tO + j, reinterpret_cast<uint32_t *>(v));
            tc_wait_ld();
#pragma unroll
            for (int x = 0; x < 32; x += 8)
                sts128(at + sw_off(t, (col & 63) + x), pack2(mul2(ee, two(v[x], v[x + 1]))), pack2(mul2(ee, two(v[x + 2], v[x + 3]))),
                       pack2(mul2(ee, two(v[x + 4], v[x + 5]))), pack2(mul2(ee, two(v[x + 6], v[x + 7]))));
        }
    } else {
        const int order = ps.reverse ? un.len - 1 - (t0 + t) : t0 + t;
#pragma unroll 1
        for (int j = 0; j < DC / 2; j += 8) {
            const int col = (DC / 2) * half + j;
            float v[8];
            tmem_ld8(tO + j, reinterpret_cast<uint32_t *>(v));
            tc_wait_ld();
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                v[x] *= e;
                if (bad && order >= mi.first[set][col + x]) v[x] = __int_as_float(0x7fffffff);
            }
            const uint4 y = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
            const size_t out = (((size_t)un.b * p.T + t0 + t) * p.H + un.h) * DC + col;
            if (!direct) {
                sts128(stage + (col >> 6) * C * 128 + sw_off(t, col & 63), y.x, y.y, y.z, y.w);
            } else if (t < n && ps.out_f32) {
                float4 *o = reinterpret_cast<float4 *>(static_cast<float *>(ps.out) + out);
                o[0] = make_float4(v[0], v[1], v[2], v[3]);
                o[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else if (t < n) {
                *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(ps.out) + out) = y;
            }
        }
    }
    tc_fence_before();
    arrive(mi, B_OFREE);
    if (!direct) fence_async_smem();
    arrive(mi, B_OUT);
    return true;
}

// P and the output: a thread has row t of the chunk and one half of the columns
template <int DA, int DC>
__device__ __forceinline__ void run_p(unsigned char *smem, Misc &mi, const Params &p, uint32_t tmem)
{
    const int id = threadIdx.x - kWarpP * 32, t = id & 127, w = t >> 5, half = id >> 7;
    const uint32_t lane = tmem + ((uint32_t)(w * 32) << 16);
    // the half's P goes over the half's own part of A, which its threads have read by then
    const uint32_t tA = lane + kColA + 64 * half;
    bool live = true;                          // after a wait that ran out a warp only keeps the group's barriers company
    int g = 0, nth = 0;                        // chunks and units with chunks so far
    for (int u = blockIdx.x; u < p.units; u += gridDim.x) {
        const Unit un(p, u, false);
        const Pass &ps = p.pass[un.pass];
        const bool rev = ps.reverse != 0;
        const float ld = p.log_decay[un.h];
        if (un.hi == un.lo) continue;
        const int set = nth++ % kSets;
        const float e_full = !shares(ld, ps) ? 1.f : ps.se * power(ld, rev ? C - 1 - t : t + 1);
        group_sync(1, 256);                    // the tables' readers are done with the last unit's
        // Shared accumulator: pw[i] is the factor of column i.  Otherwise of distance m = t - i, forward at pw[31 + m] (m from -31 to
        // 127), reverse at pw[127 + m] (-127 to 31).
        const bool one = shares(ld, ps);
        if (id < 31 + C) {
            if (one) mi.pw[id] = ps.sp / ps.se * expf((float)(rev ? id - C + 1 : -(id + 1)) * ld);
            else mi.pw[id] = (rev ? id > C - 1 : id < 31) ? 0.f : ps.sp * power(ld, rev ? C - 1 - id : id - 31);
        }
        const float *pw = mi.pw + (one ? 0 : rev ? C - 1 : 31);
        group_sync(1, 256);
        for (int i = 0; i < un.hi - un.lo; ++i, ++g) {
            const int t0 = un.chunk(p, i) * C, n = min(C, un.len - t0);
            if (!(live = live && wait_warp(mi, B_A, g))) continue;
            tc_fence_after();
            // a reverse pass starts at the end of a sequence, where its distance to the chunk's end is shorter
            const float short_of = one && rev && n < C ? expf((float)(C - n) * ld) : 1.f;
#pragma unroll 1
            for (int x = 0; x < 2; ++x) {
                const int j = 2 * half + x, m = t - 32 * j;            // the block of 32 tokens; the distance to its first
                uint32_t y[16];
#pragma unroll
                for (int z = 0; z < 16; ++z) y[z] = 0;
                if (rev ? j >= w : j <= w) {
                    float v[32];
                    tmem_ld<32>(tA + 32 * x, reinterpret_cast<uint32_t *>(v));
                    tc_wait_ld();
                    if (short_of != 1.f)
#pragma unroll
                        for (int z = 0; z < 32; ++z) v[z] *= short_of;
                    if (one) {
#pragma unroll
                        for (int z = 0; z < 32; z += 4) {
                            const float4 c = *reinterpret_cast<const float4 *>(&mi.pw[32 * j + z]);
                            y[z / 2] = pack2(mul2(two(v[z], v[z + 1]), two(c.x, c.y)));
                            y[z / 2 + 1] = pack2(mul2(two(v[z + 2], v[z + 3]), two(c.z, c.w)));
                        }
                    } else {
                        const float *d = pw + m;
#pragma unroll
                        for (int z = 0; z < 32; z += 2) y[z / 2] = pack_bf16(v[z] * d[-z], v[z + 1] * d[-z - 1]);
                    }
                    if (j == w || n < C) {
                        // tokens of the block that the row reads: z <= m, or m <= z < n - 32 j
                        const int lo = rev ? max(m, 0) : 0, hi = rev ? min(n - 32 * j, 32) : min(m + 1, 32);
                        const uint32_t keep = (hi <= lo ? 0u : 0xffffffffu >> (32 - hi)) & (lo > 31 ? 0u : 0xffffffffu << lo);
#pragma unroll
                        for (int z = 0; z < 16; ++z) y[z] &= (keep >> (2 * z) & 1 ? 0xffffu : 0u) | (keep >> (2 * z) & 2 ? 0xffff0000u : 0u);
                    }
                }
                tmem_st16(tA + 16 * x, y);
            }
            tc_wait_st();
            tc_fence_before();
            arrive(mi, B_P);
            live = write_out<DA, DC>(smem, mi, p, tmem, un, g, t0, n, set, one && rev && n < C ? ps.se * power(ld, max(n - 1 - t, 0)) : e_full);
        }
    }
}

// The staged outputs' copies to memory (one warp; rows behind T are cut off by the tensor map)
template <int DA, int DC>
__device__ __forceinline__ void run_out(unsigned char *smem, Misc &mi, const Params &p)
{
    int g = 0;
    for (int u = blockIdx.x; u < p.units; u += gridDim.x) {
        const Unit un(p, u, false);
        const Pass &ps = p.pass[un.pass];
        for (int i = 0; i < un.hi - un.lo; ++i, ++g) {
            const int t0 = un.chunk(p, i) * C, n = min(C, un.len - t0);
            if (!wait_warp(mi, B_OUT, g)) return;
            if (elect_one()) {
                if (!store_directly(p, ps, t0, n)) {
#pragma unroll
                    for (int x = 0; x < DC / 64; ++x)
                        tma_store_4d(&p.out[un.pass], smem + Layout<DA, DC>::kOut + x * C * 128, 64 * x, un.h, t0, un.b);
                    tma_store_commit();
                    tma_store_wait_read();
                }
                arrive(mi, B_EMPTYO);
            }
            __syncwarp();
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
    const uint32_t tU = tmem + kColU + c0 + ((uint32_t)(k & 96) << 16), tO = tmem + kColO + c0 + ((uint32_t)(k & 96) << 16);
    const uint32_t ss = smem_u32(smem) + Lo::kS;
    int g = 0, nth = 0;                        // chunks and units with chunks so far
    for (int u = blockIdx.x; u < p.units; u += gridDim.x) {
        const Unit un(p, u, kStates);
        const Pass &ps = p.pass[un.pass];
        const float ld = p.log_decay[un.h];
        const bool rev = ps.reverse != 0, one = kStates || shares(ld, ps);
        uint64_t s[N / 2];                     // two columns each
#pragma unroll
        for (int x = 0; x < N / 2; ++x) s[x] = 0;
        if (mine) {
            float *seg = ps.seg + (size_t)un.pair * p.nseg * DA * DC + (size_t)k * DC + c0;      // the thread's part of the pair's states
            const bool copied = !kStates && p.nseg > 1;
            if (un.seg == 0 && ps.s_in) {
                const float *from = copied ? seg + (size_t)(p.nseg - 1) * DA * DC : ps.s_in + (size_t)un.pair * DA * DC + (size_t)k * DC + c0;
                if (ps.s_in_t && !copied) {
                    from = ps.s_in + (size_t)un.pair * DA * DC + (size_t)c0 * DA + k;
#pragma unroll
                    for (int x = 0; x < N; x += 2) s[x / 2] = two(from[(size_t)x * DA], from[(size_t)(x + 1) * DA]);
                } else {
#pragma unroll
                    for (int x = 0; x < N; x += 4) {
                        const float4 v = *reinterpret_cast<const float4 *>(from + x);
                        s[x / 2] = two(v.x, v.y);
                        s[x / 2 + 1] = two(v.z, v.w);
                    }
                }
                if (kStates)
#pragma unroll
                    for (int x = 0; x < N; x += 4) {
                        float4 v;
                        apart(s[x / 2], v.x, v.y);
                        apart(s[x / 2 + 1], v.z, v.w);
                        *reinterpret_cast<float4 *>(seg + (size_t)(p.nseg - 1) * DA * DC + x) = v;
                    }
            }
            if (!kStates)
#pragma unroll 1
                for (int j = 0; j < un.seg; ++j) {
                    const int tok = un.tokens(p, j);
                    if (j > 0 && tok == 0) continue;
                    const float gn = power(ld, tok);
                    const uint64_t gg = two(gn, gn);
#pragma unroll
                    for (int x = 0; x < N; x += 4) {
                        const float4 v = __ldcg(reinterpret_cast<const float4 *>(seg + (size_t)j * DA * DC + x));
                        s[x / 2] = fma2(gg, s[x / 2], two(v.x, v.y));
                        s[x / 2 + 1] = fma2(gg, s[x / 2 + 1], two(v.z, v.w));
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
                const uint64_t gg = two(gm, gm), one = weak ? two(1.f, 1.f) : 0;
                if (!wait_warp(mi, B_U, g)) return;    // (and with it a S, the reader of S's copy)
                tc_fence_after();
                ++g;
#pragma unroll
                for (int x = 0; x < N; x += 16) {
                    uint32_t v[16];
                    tmem_ld<16>(tU + x, v);
                    tc_wait_ld();
#pragma unroll
                    for (int y = 0; y < 16; y += 2) {
                        uint64_t &z = s[(x + y) / 2];
                        z = fma2(gg, z, fma2(one, z, two(__uint_as_float(v[y]), __uint_as_float(v[y + 1]))));
                    }
                }
                tc_fence_before();
            }
            if (i == chunks) break;
            if (!kStates && mine) {
#pragma unroll
                for (int x = 0; x < N; x += 8) {
                    const int col = c0 + x;
                    sts128(ss + (col >> 6) * (DA * 128) + sw_off(k, col & 63), pack2(s[x / 2]), pack2(s[x / 2 + 1]), pack2(s[x / 2 + 2]),
                           pack2(s[x / 2 + 3]));
                }
            }
            if (!kStates) fence_async_smem();
            arrive(mi, B_S);
            if (!kStates && !one) {
                // e o (a S) in the accumulator, for heads where P c cannot be added to a S as it is
                const int n = min(C, un.len - un.chunk(p, i) * C);
                const float e = ps.se * power(ld, rev ? max(n - 1 - k, 0) : k + 1);
                if (!wait_warp(mi, B_QS, g)) return;
                tc_fence_after();
#pragma unroll 1
                for (int x = 0; x < N; x += 8) {
                    uint32_t v[8];
                    tmem_ld8(tO + x, v);
                    tc_wait_ld();
#pragma unroll
                    for (int y = 0; y < 8; ++y) v[y] = __float_as_uint(e * __uint_as_float(v[y]));
                    tmem_st8(tO + x, v);
                }
                tc_wait_st();
                tc_fence_before();
                arrive(mi, B_E);
            }
        }
        float *to = kStates ? ps.seg + ((size_t)un.pair * p.nseg + un.seg) * DA * DC
                            : un.seg == p.nseg - 1 && ps.s_out ? ps.s_out + (size_t)un.pair * DA * DC : nullptr;
        if (to && mine) {
            const int set = (nth - 1) % kSets;
            const bool bad = chunks > 0 && mi.any[set];
#pragma unroll
            for (int x = 0; x < N; x += 4) {
                float4 v;
                apart(s[x / 2], v.x, v.y);
                apart(s[x / 2 + 1], v.z, v.w);
                if (bad) {
                    const float nan = __int_as_float(0x7fffffff);
                    const int *f = &mi.first[set][c0 + x];
                    v = make_float4(f[0] != kNever ? nan : v.x, f[1] != kNever ? nan : v.y, f[2] != kNever ? nan : v.z, f[3] != kNever ? nan : v.w);
                }
                *reinterpret_cast<float4 *>(to + (size_t)k * DC + c0 + x) = v;
            }
        }
    }
}

// w o b in two parts, and c made safe.  With w = w1 + w2, both bf16, the high part is bf16(w1 b), and the low one b w2 plus what the
// high one's rounding left, which a fused multiply-add gives exactly: three instructions for two elements.  A warp has 32 channels of b (its tensor memory lanes) and 64 tokens: 8 x 8 blocks come
// transposed out of shared memory in the fragment that the 16-lane stores of tensor memory take, so the product's operand never
// goes back through shared memory, whose bandwidth the other products need.
template <int DA, int DC, bool kStates>
__device__ __forceinline__ void run_keys(unsigned char *smem, Misc &mi, const Params &p, uint32_t tmem)
{
    using Lo = Layout<DA, DC>;
    constexpr int NC = DC / 2;
    const int id = threadIdx.x - kWarpK * 32, lane = id & 31, quad = (id >> 5) & 3, half = id >> 7, r = id & 127;
    const uint32_t base = smem_u32(smem);
    const uint32_t tK = tmem + kColK + 32 * half + ((uint32_t)(quad * 32) << 16);
    const bool mine = 32 * quad < DA;
    const int tok0 = 64 * half + 2 * (lane & 3);               // the thread's tokens: tok0 + 8 i, and the next
    bool live = true;                          // as in run_p
    int g = 0, nth = 0;                        // chunks and units with chunks so far
    for (int u = blockIdx.x; u < p.units; u += gridDim.x) {
        const Unit un(p, u, kStates);
        const Pass &ps = p.pass[un.pass];
        const bool rev = ps.reverse != 0;
        const float ld = p.log_decay[un.h];
        const int chunks = un.hi - un.lo;
        if (chunks == 0) continue;
        const int set = nth++ % kSets;
        if (half == 0) mi.first[set][r] = kNever;
        if (id == 0) mi.any[set] = 0;
        group_sync(2, 256);
        uint32_t w[8], wlo[8];                 // two tokens each: bf16(w) and bf16 of the rest
        int weights_of = -1;                   // the chunk length that w is for
        for (int i = 0; i < chunks; ++i, ++g) {
            const int st = g & 1, t0 = un.chunk(p, i) * C, n = min(C, un.len - t0);
            const uint32_t sb = base + Lo::kA + st * Lo::kStage, sc = sb + Lo::kA;
            if (n != weights_of) {
                weights_of = n;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    float f[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int tok = tok0 + 8 * x + y, hops = rev ? tok + 1 : n - 1 - tok;
                        f[y] = tok < n ? ps.sw * power(ld, hops) : 0.f;
                    }
                    w[x] = pack_bf16(f[0], f[1]);
                    wlo[x] = pack_bf16(f[0] - bf16_low(w[x]), f[1] - bf16_high(w[x]));
                }
            }
            const auto off = [r](int ch) { return (uint32_t)((ch >> 6) * C * 128 + sw_off(r, ch & 63)); };
            live = live && wait_warp(mi, B_FULL + st, g >> 1) && (g == 0 || wait_warp(mi, B_U, g - 1));
            if (n < C) {                       // tokens behind the end: whatever is there is no value
                if (live && r >= n) {
#pragma unroll 1
                    for (int x = 0; x < DA / 2; x += 8) sts128(sb + off(half * (DA / 2) + x), 0, 0, 0, 0);
#pragma unroll 1
                    for (int x = 0; x < NC; x += 8) sts128(sc + off(half * NC + x), 0, 0, 0, 0);
                    fence_async_smem();
                }
                group_sync(2, 256);
            }
            if (!live) continue;
            tc_fence_after();
            if (mine) {
#pragma unroll 1
                for (int rows = 0; rows < 32; rows += 16) {
                    const int ch = 32 * quad + rows + 8 * ((lane >> 3) & 1);
                    const uint32_t from = sb + (ch >> 6) * C * 128;
#pragma unroll
                    for (int x = 0; x < 8; x += 4) {           // blocks of 8 tokens
                        uint32_t hi[8], lo[8];
#pragma unroll
                        for (int z = 0; z < 4; z += 2) {
                            const int tok = 64 * half + 8 * (x + z + (lane >> 4)) + (lane & 7);
                            uint32_t v[4];
                            ldmatrix_x4_trans(v, from + sw_off(tok, ch & 63));
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                const uint32_t w1 = w[x + z + (y >> 1)], w2 = wlo[x + z + (y >> 1)], h = mul_bf16x2(v[y], w1);
                                hi[2 * z + y] = h;
                                lo[2 * z + y] = fma_bf16x2(v[y], w2, fma_bf16x2(v[y], w1, h ^ 0x80008000u));
                            }
                        }
                        tmem_st_16x128b_x4(tK + 4 * x + ((uint32_t)rows << 16), hi);
                        tmem_st_16x128b_x4(tK + 64 + 4 * x + ((uint32_t)rows << 16), lo);
                    }
                }
                tc_wait_st();
            }
            tc_fence_before();
            uint32_t odd = 0;
#pragma unroll
            for (int x = 0; x < NC; x += 8) {
                const uint4 v = lds128(sc + off(half * NC + x));
                odd = max_abs_bf16x2(v.x, max_abs_bf16x2(v.y, max_abs_bf16x2(v.z, max_abs_bf16x2(v.w, odd))));
            }
            if (((odd & 0x7fff7fffu) + 0x00800080u) & 0x80008000u) {
#pragma unroll 1
                for (int x = half * NC; x < (half + 1) * NC; ++x) {
                    const uint32_t at = sc + off(x);
                    if ((lds16(at) & 0x7f80u) == 0x7f80u) {
                        sts16(at, 0);
                        atomicMin(&mi.first[set][x], rev ? un.len - 1 - (t0 + r) : t0 + r);
                        mi.any[set] = 1;
                    }
                }
                fence_async_smem();
            }
            arrive(mi, B_K);
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
        const int counts[kBars] = {1, 1, 1, 1, 1, 1, 1, 1, 1, 256, 1, 256, 1, 256, 256, 256, 256};
        for (int i = 0; i < kBars; ++i) mbar_init(&mi.bars[i], counts[i]);
        mi.abort = 0;
#ifdef SFDA_WS_CHAOS
        mi.withhold = p.withhold;
#endif
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
    if (warp < kWarpP) {
        regs_dec<kRegsCtrl>();
        if (warp == 0) run_tma<DA, DC, kStates>(smem, mi, p);
        if (warp == 1) run_mma<DA, DC, kStates>(smem, mi, p, tmem);
        if (warp == 2 && !kStates) run_out<DA, DC>(smem, mi, p);
    } else if (warp >= kWarpK) {
        regs_dec<kRegsK>();
        run_keys<DA, DC, kStates>(smem, mi, p, tmem);
    } else if (warp >= kWarpS) {
        regs_inc<kRegsS>();
        run_state<DA, DC, kStates>(smem, mi, p, tmem);
    } else {
        if (!kStates) run_p<DA, DC>(smem, mi, p, tmem);
    }
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

// How many stretches each sequence is cut into, for `chains` of `chunks` chunks on n SMs: the least of a sum of measured times in
// microseconds.  A CTA takes kChunk for a chunk (kStates for one of the pass that only makes states) and kStart for a unit; a
// stretch reads the states of those before it, kCarry each; a second launch costs kLaunch; and memory takes kMemory for a chunk.
// (Measured at d = 128, replayed from a graph: one sequence of 131072 tokens and 16 heads 2883 us uncut, 733 in 8, 726 in 9; 4 x 4096
// and 16 heads 131 uncut, 126 in 2; 4096 and 32 heads 100 uncut, 71 in 4; 1024 and 8 heads 32 uncut, 38 in 2.  The constants are those
// of d = 128; at d = 64 the same four: 489 in 9 (473 in 18); 87 uncut, 76 in 2; 44 in 4; 23 uncut, 19 in 8.)
static int stretches(long long chains, int chunks, int n)
{
    constexpr double kChunk = 2.9, kStates = 2.6, kStart = 8.0, kCarry = 2.5, kLaunch = 4.0, kMemory = 0.026;
    const auto waves = [n](long long units) { return (double)((units + n - 1) / n); };
    int best = 1;
    double least = 0;
    for (int s = 1; s <= chunks && s <= 64; ++s) {
        const int cps = (chunks + s - 1) / s;
        if ((chunks + cps - 1) / cps != s) continue;
        const double mem = (double)chains * chunks * kMemory;
        double t = waves(chains * s) * (cps * kChunk + kStart + (s - 1) * kCarry);
        if (t < mem) t = mem;
        if (s > 1) {
            double a = waves(chains * (s - 1)) * (cps * kStates + kStart);
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
    return *nseg == 1 ? 0 : (size_t)passes * pairs * *nseg * d_k * d_v * 4;
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
#ifdef SFDA_WS_CHAOS
    p.withhold = getenv("SFDA_WITHHOLD_LINEAR") ? atoi(getenv("SFDA_WITHHOLD_LINEAR")) : -1;
#endif
    float *seg = reinterpret_cast<float *>(static_cast<char *>(workspace) + 256);
    for (int at = 0; at < count;) {
        p.n_pass = group_of(passes + at, count - at);
        const int DA = passes[at].DA, DC = passes[at].DC;
        const size_t each = (size_t)p.pairs * DA * DC;
        scratch_of(a, p.n_pass, DA, DC, &p.nseg);
        const int chunks = (a.T + C - 1) / C;
        p.cps = (chunks + p.nseg - 1) / p.nseg;
        // one map for each tensor: inputs of different widths may begin at the same address
        const void *seen[4] = {};
        int heads[4] = {}, widths[4] = {}, maps = 0;
        auto map_of = [&](const void *x, int h, int d) {
            for (int i = 0; i < maps; ++i)
                if (seen[i] == x && heads[i] == h && widths[i] == d) return i;
            if (maps == 4 || !make_map(&p.map[maps], x, a.B, a.T, h, d)) return -1;
            seen[maps] = x;
            heads[maps] = h;
            widths[maps] = d;
            return maps++;
        };
        for (int i = 0; i < p.n_pass; ++i) {
            const LinearPass &x = passes[at + i];
            Pass &y = p.pass[i];
            y.out = x.out; y.s_in = x.s_in; y.s_out = x.s_out;
            y.seg = seg + i * each * p.nseg;
            y.ma = map_of(x.a, x.Ha, DA); y.mb = map_of(x.b, x.Hb, DA); y.mc = map_of(x.c, x.Hc, DC);
            if (y.ma < 0 || y.mb < 0 || y.mc < 0 || (!x.out_f32 && !make_map(&p.out[i], x.out, a.B, a.T, a.H, DC)))
                return cudaErrorInvalidValue;
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
