// sfda_group_norm: normalisation over each group of channels of a row (channels last), affine, activated or gated:
//
//     n = (x - mean) / sqrt(var + eps),   z = n w + b,   y = act(z)   or, with a gate,   y = z act(gate),
//
// and its derivative.  Bound by memory: x (gate, dy) are read once, everything between stays in registers.  A group is
// spread over P lanes of one warp or of several, NV accesses of V channels each; the mean is taken first and the variance from the
// differences, both in fp32.  For fp32 the differences' own mean, what the first one's rounding left, is taken off as well: where a
// group's mean is large beside its deviation, n would otherwise be off by the mean's 2^-24 over the deviation.  Values of 8 bits
// that are not all equal deviate by 2^-8 of the largest, so bf16 groups held in registers do without.
//
// The derivative recomputes n from x (it reads the whole group anyway).  Its CTAs keep the same channels from row to row,
// so the sums over rows behind dw and db stay in registers; each CTA writes one row of partial sums, and a second kernel
// adds them in a fixed order.
#include "sfda_common.cuh"
#include "sfda_linear.h"
#include "sfda_vec.cuh"

namespace sfda {
namespace {

constexpr int kThreads = 256;

struct Dev {
    const void *x, *gate, *dy;
    const float *weight, *bias;
    void *y, *dx, *dgate;
    float *part;                 // [2][blocks over rows][C] partial sums of dw and db, or NULL
    long long rows;
    int C, G, D, lanes, gb, rb;  // lanes of a group; groups and rows that a CTA holds at a time
    int silu;
    float eps;
};

// Sum over a group's lanes, the same for all of them: within a warp, and through shared memory where a group has several warps
// (all threads of the CTA come here together).
__device__ __forceinline__ float sum_lanes(float x, int lanes, float *red = nullptr)
{
    for (int d = min(lanes, 32) >> 1; d >= 1; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    if (lanes > 32) {
        const int warp = threadIdx.x >> 5, warps = lanes >> 5;
        __syncthreads();
        if ((threadIdx.x & 31) == 0) red[warp] = x;
        __syncthreads();
        x = 0.f;
        for (int i = 0; i < warps; ++i) x += red[warp / warps * warps + i];
    }
    return x;
}

// sum / n, from the rounded 1 / n and what the product leaves of the sum.  The mean of n equal values is that value where their sum is
// exact; the product alone missed it (500 values of 1000 in bf16: by 6e-5, which at eps = 1e-5 is a deviation of 0.02).
__device__ __forceinline__ float mean_of(float sum, float n, float inv)
{
    const float m = sum * inv;
    return fmaf(fmaf(-m, n, sum), inv, m);
}

// 1 / (1 + 2^(-x / ln 2)) in four instructions: the approximations' results below 2^-126 are zeros, which is what both ends need (the
// forward is bound by its instructions)
__device__ __forceinline__ float sigmoid(float x)
{
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return r;
}

// The next row's accesses are in flight while a row is computed.  Which of the gate and the activation there are is known when the
// kernel is compiled: decided per element at run time, the derivative took twice as many instructions and 1.9 times as long.
template <typename T, int V, int NV, bool kBackward, bool kGate, bool kSilu>
__global__ void __launch_bounds__(kThreads) sfda_group_norm_kernel(const Dev p)
{
    __shared__ float part[kThreads / 32];
    const int tid = threadIdx.x, lane = tid % p.lanes, slot = tid / p.lanes;
    // slots beyond gb * rb hold no group (but take part in the shuffles)
    const int g0 = blockIdx.y * p.gb, grp = g0 + slot % p.gb, sub = slot / p.gb;
    const bool have = sub < p.rb && grp < p.G;
    const float width = (float)p.D, inv = 1.f / width;
    float w[NV][V], b[NV][V], aw[kBackward ? NV : 1][V], ab[kBackward ? NV : 1][V];
    bool in[NV];
    int ch[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int e = (lane + j * p.lanes) * V;
        in[j] = have && e < p.D;
        ch[j] = in[j] ? grp * p.D + e : 0;
    }
    const T *px = static_cast<const T *>(p.x), *pg = static_cast<const T *>(p.gate), *pd = static_cast<const T *>(p.dy);
    const long long step = (long long)gridDim.x * p.rb;
    Raw<T, V> rx[NV], rg[kGate ? NV : 1], rd[kBackward ? NV : 1];
    const auto fetch = [&](long long row) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (in[j] && row < p.rows) {
                const long long at = row * p.C + ch[j];
                rx[j].load(px + at);
                if constexpr (kGate) rg[j].load(pg + at);
                if constexpr (kBackward) rd[j].load(pd + at);
            } else {
                rx[j].clear();
                if constexpr (kGate) rg[j].clear();
                if constexpr (kBackward) rd[j].clear();
            }
        }
    };
    fetch((long long)blockIdx.x * p.rb + sub);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[j][i] = 1.f;
            b[j][i] = 0.f;
            if (kBackward) aw[j][i] = ab[j][i] = 0.f;
        }
        // (lanes without a channel keep 1 and 0: their zeros go into the group's sums, and 0 times a parameter that is not finite is none)
        if (p.weight && in[j]) ld_vec(p.weight + ch[j], w[j]);
        if (p.bias && in[j]) ld_vec(p.bias + ch[j], b[j]);
    }
    for (long long base = (long long)blockIdx.x * p.rb; base < p.rows; base += step) {
        const long long row = base + sub;
        const bool live = have && row < p.rows;
        float x[NV][V], gt[kGate ? NV : 1][V], dy[kBackward ? NV : 1][V];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[j][i] = rx[j].get(i);
                if constexpr (kGate) gt[j][i] = rg[j].get(i);
                if constexpr (kBackward) dy[j][i] = rd[j].get(i);
                sum += x[j][i];
            }
        fetch(row + step);
        const float mean = mean_of(sum_lanes(sum, p.lanes, part), width, inv);
        float sq = 0.f, rest = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const float m = in[j] ? mean : 0.f;            // (outside the group x is zero and stays so)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[j][i] -= m;
                if constexpr (sizeof(T) == 4) rest += x[j][i];
                sq = fmaf(x[j][i], x[j][i], sq);
            }
        }
        sq = sum_lanes(sq, p.lanes, part) * inv;
        if constexpr (sizeof(T) == 4) {
            rest = mean_of(sum_lanes(rest, p.lanes, part), width, inv);
            sq = fmaxf(fmaf(-rest, rest, sq), 0.f);        // (rounding may leave less than nothing of a variance, and eps be smaller)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const float m = in[j] ? rest : 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) x[j][i] -= m;
            }
        }
        const float rstd = rsqrtf(sq + p.eps);
        if constexpr (!kBackward) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float y[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float z = fmaf(x[j][i] * rstd, w[j][i], b[j][i]), h = kGate ? gt[kGate ? j : 0][i] : z;
                    const float a = kSilu ? h * sigmoid(h) : h;
                    y[i] = kGate ? z * a : a;
                }
                if (live && in[j]) st_vec(static_cast<T *>(p.y) + row * p.C + ch[j], y);
            }
        } else {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float dg[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float n = x[j][i] * rstd, z = fmaf(n, w[j][i], b[j][i]), h = kGate ? gt[kGate ? j : 0][i] : z;
                    const float sg = kSilu ? sigmoid(h) : 1.f;
                    const float a = kSilu ? h * sg : h, slope = kSilu ? fmaf(a, 1.f - sg, sg) : 1.f;
                    const float dz = dy[j][i] * (kGate ? a : slope);
                    if (kGate) dg[i] = dy[j][i] * z * slope;
                    aw[j][i] = fmaf(dz, n, aw[j][i]);
                    ab[j][i] += dz;
                    const float dn = dz * w[j][i];
                    s1 += dn;
                    s2 = fmaf(dn, n, s2);
                    x[j][i] = n;
                    dy[j][i] = dn;
                }
                if (kGate && live && in[j]) st_vec(static_cast<T *>(p.dgate) + row * p.C + ch[j], dg);
            }
            s1 = sum_lanes(s1, p.lanes, part) * inv * rstd;
            s2 = sum_lanes(s2, p.lanes, part) * inv * rstd;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float d[V];
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] = fmaf(-x[j][i], s2, fmaf(rstd, dy[j][i], -s1));
                if (live && in[j]) st_vec(static_cast<T *>(p.dx) + row * p.C + ch[j], d);
            }
        }
    }
    if constexpr (kBackward) {
        if (!p.part) return;
        // the rows that a CTA holds at a time end in one sum: their slots add up through shared memory, in order
        __shared__ float red[kThreads][2 * V];
        float *pw = p.part + (long long)blockIdx.x * p.C, *pb = pw + (long long)gridDim.x * p.C;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) {
                red[tid][i] = aw[j][i];
                red[tid][V + i] = ab[j][i];
            }
            __syncthreads();
            if (sub == 0 && in[j]) {
                float sw[V], sb[V];
#pragma unroll
                for (int i = 0; i < V; ++i) sw[i] = sb[i] = 0.f;
                for (int r = 0; r < p.rb; ++r)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        sw[i] += red[tid + r * p.gb * p.lanes][i];
                        sb[i] += red[tid + r * p.gb * p.lanes][V + i];
                    }
                st_vec(pw + ch[j], sw);
                st_vec(pb + ch[j], sb);
            }
        }
    }
}

// A group too wide for the registers of a CTA: one CTA per (row, group), the group read again for each step (it is in the
// caches by then).
__device__ float sum_block(float x, float *red)
{
    x = sum_lanes(x, 32);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) s += red[i];
    return s;
}
template <typename T, bool kBackward>
__global__ void __launch_bounds__(kThreads) sfda_group_norm_wide_kernel(const Dev p)
{
    __shared__ float red[kThreads / 32];
    const int grp = blockIdx.y, c0 = grp * p.D;
    const float width = (float)p.D, inv = 1.f / width;
    const T *pg = static_cast<const T *>(p.gate);
    float *pw = p.part ? p.part + (long long)blockIdx.x * p.C : nullptr, *pb = pw ? pw + (long long)gridDim.x * p.C : nullptr;
    bool first = true;
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x, first = false) {
        const T *x = static_cast<const T *>(p.x) + row * p.C;
        float s = 0.f;
        for (int c = threadIdx.x; c < p.D; c += kThreads) s += ld_val(x, c0 + c);
        const float mean = mean_of(sum_block(s, red), width, inv);
        s = 0.f;
        float rest = 0.f;
        for (int c = threadIdx.x; c < p.D; c += kThreads) {
            const float d = ld_val(x, c0 + c) - mean;
            rest += d;
            s = fmaf(d, d, s);
        }
        rest = mean_of(sum_block(rest, red), width, inv);
        const float rstd = rsqrtf(fmaxf(fmaf(-rest, rest, sum_block(s, red) * inv), 0.f) + p.eps);
        float s1 = 0.f, s2 = 0.f;
        for (int pass = 0; pass < (kBackward ? 2 : 1); ++pass) {
            for (int c = threadIdx.x; c < p.D; c += kThreads) {
                const int ch = c0 + c;
                const size_t at = (size_t)row * p.C + ch;
                const float w = p.weight ? p.weight[ch] : 1.f, b = p.bias ? p.bias[ch] : 0.f;
                const float n = (ld_val(x, ch) - mean - rest) * rstd, z = fmaf(n, w, b), h = pg ? ld_val(pg, at) : z;
                const float sg = p.silu ? sigmoid(h) : 1.f, a = p.silu ? h * sg : h;
                if (!kBackward) {
                    st_val(static_cast<T *>(p.y), at, pg ? z * a : a);
                    continue;
                }
                const float slope = p.silu ? sg * fmaf(h, 1.f - sg, 1.f) : 1.f, dy = ld_val(static_cast<const T *>(p.dy), at);
                const float dz = dy * (pg ? a : slope), dn = dz * w;
                if (pass == 0) {
                    s1 += dn;
                    s2 = fmaf(dn, n, s2);
                    if (pw) {
                        pw[ch] = first ? dz * n : pw[ch] + dz * n;
                        pb[ch] = first ? dz : pb[ch] + dz;
                    }
                } else {                                   // (both outputs here: they may lie over dy and the gate)
                    if (pg) st_val(static_cast<T *>(p.dgate), at, dy * z * slope);
                    st_val(static_cast<T *>(p.dx), at, rstd * (dn - s1 - n * s2));
                }
            }
            if (kBackward && pass == 0) {
                s1 = sum_block(s1, red) * inv;
                s2 = sum_block(s2, red) * inv;
            }
        }
    }
}

// dw, db: column sums of the partial rows, 32 columns to a CTA, eight runs of rows added in order
__global__ void __launch_bounds__(kThreads) sfda_group_norm_sum_kernel(const float *__restrict__ part, float *dw, float *db, int n, int C)
{
    __shared__ float red[kThreads / 32][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
    const float *src = part + (blockIdx.y ? (long long)n * C : 0);
    float *dst = blockIdx.y ? db : dw;
    if (!dst) return;
    float s = 0.f;
    if (c < C)
        for (int r = w; r < n; r += kThreads / 32) s += src[(long long)r * C + c];
    red[w][threadIdx.x & 31] = s;
    __syncthreads();
    if (w == 0 && c < C) {
        for (int i = 1; i < kThreads / 32; ++i) s += red[i][threadIdx.x & 31];
        dst[c] = s;
    }
}

struct Shape {
    int V, NV, lanes, gb, rb, blocks_y;
    bool wide;
};
constexpr int kMaxNV = 4;

Shape shape_of(int C, int G, int dtype)
{
    Shape s = {};
    const int D = C / G;
    s.V = dtype == 1 && D % 8 == 0 ? 8 : D % 4 == 0 ? 4 : 1;
    const int n = D / s.V;                                  // accesses of a group
    s.lanes = 1;
    while (s.lanes < 32 && s.lanes < n) s.lanes *= 2;
    while (s.lanes < kThreads && s.lanes * 2 < n) s.lanes *= 2;         // several warps where two accesses a lane do not do
    s.NV = 1;
    while (s.NV * s.lanes < n) s.NV *= 2;
    s.wide = s.NV > kMaxNV;
    if (s.wide) {
        s.gb = s.rb = 1;
        s.blocks_y = G;
        return s;
    }
    const int slots = kThreads / s.lanes;
    s.gb = G < slots ? G : slots;
    s.rb = slots / s.gb;
    s.blocks_y = (G + s.gb - 1) / s.gb;
    return s;
}
// CTAs over the rows: a few waves of the device, and at least `each` steps for a CTA, so that the backward's partial sums stay few
unsigned blocks_over_rows(const Shape &s, long long rows, int waves, int each)
{
    const long long want = (rows + (long long)s.rb * each - 1) / ((long long)s.rb * each), most = (148ll * waves + s.blocks_y - 1) / s.blocks_y;
    return (unsigned)(want < most ? want : most);
}
constexpr int kForwardWaves = 8, kBackwardWaves = 8;

template <typename T, int V, int NV, bool kBackward>
void launch_kind(const Dev &p, dim3 grid, cudaStream_t stream)
{
    if (p.gate && p.silu) sfda_group_norm_kernel<T, V, NV, kBackward, true, true><<<grid, kThreads, 0, stream>>>(p);
    else if (p.gate) sfda_group_norm_kernel<T, V, NV, kBackward, true, false><<<grid, kThreads, 0, stream>>>(p);
    else if (p.silu) sfda_group_norm_kernel<T, V, NV, kBackward, false, true><<<grid, kThreads, 0, stream>>>(p);
    else sfda_group_norm_kernel<T, V, NV, kBackward, false, false><<<grid, kThreads, 0, stream>>>(p);
}
template <typename T, int V, bool kBackward>
cudaError_t launch_nv(const Shape &s, const Dev &p, dim3 grid, cudaStream_t stream)
{
    if (s.NV == 1) launch_kind<T, V, 1, kBackward>(p, grid, stream);
    else if (s.NV == 2) launch_kind<T, V, 2, kBackward>(p, grid, stream);
    else launch_kind<T, V, 4, kBackward>(p, grid, stream);
    return cudaGetLastError();
}
template <typename T, bool kBackward>
cudaError_t launch_v(const Shape &s, const Dev &p, dim3 grid, cudaStream_t stream)
{
    if (s.wide) {
        sfda_group_norm_wide_kernel<T, kBackward><<<grid, kThreads, 0, stream>>>(p);
        return cudaGetLastError();
    }
    if constexpr (sizeof(T) == 2)
        if (s.V == 8) return launch_nv<T, 8, kBackward>(s, p, grid, stream);
    return s.V == 4 ? launch_nv<T, 4, kBackward>(s, p, grid, stream) : launch_nv<T, 1, kBackward>(s, p, grid, stream);
}
Dev dev_of(const GroupNormArgs &a, const Shape &s)
{
    return {a.x, a.gate, a.dy, a.weight, a.bias, a.y, a.dx, a.dgate, nullptr, a.rows, a.C, a.G, a.C / a.G, s.lanes, s.gb, s.rb,
            a.act, a.eps};
}

}  // namespace

bool group_norm_supported(int C, int G, int dtype) { return shape_of(C, G, dtype).blocks_y <= 65535; }

cudaError_t launch_group_norm(const GroupNormArgs &a, cudaStream_t stream, int *launches)
{
    const Shape s = shape_of(a.C, a.G, a.dtype);
    const dim3 grid(blocks_over_rows(s, a.rows, kForwardWaves, 1), s.blocks_y);
    const Dev p = dev_of(a, s);
    const cudaError_t e = a.dtype == 1 ? launch_v<__nv_bfloat16, false>(s, p, grid, stream) : launch_v<float, false>(s, p, grid, stream);
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}

// Over every number of groups and either dtype: a CTA row of partial sums covers all channels once.
size_t group_norm_backward_bytes(long long rows, int C)
{
    const long long most = 148ll * kBackwardWaves;
    return (size_t)(rows < most ? rows : most) * (size_t)C * 2 * sizeof(float);
}

cudaError_t launch_group_norm_backward(const GroupNormArgs &a, void *workspace, cudaStream_t stream, int *launches)
{
    const Shape s = shape_of(a.C, a.G, a.dtype);
    Dev p = dev_of(a, s);
    if (a.dweight || a.dbias) p.part = static_cast<float *>(workspace);
    const dim3 grid(blocks_over_rows(s, a.rows, kBackwardWaves, p.part ? 4 : 1), s.blocks_y);
    cudaError_t e = a.dtype == 1 ? launch_v<__nv_bfloat16, true>(s, p, grid, stream) : launch_v<float, true>(s, p, grid, stream);
    if (e != cudaSuccess) return e;
    if (launches) ++*launches;
    if (!p.part) return cudaSuccess;
    sfda_group_norm_sum_kernel<<<dim3((a.C + 31) / 32, 2), kThreads, 0, stream>>>(p.part, a.dweight, a.dbias, (int)grid.x, a.C);
    e = cudaGetLastError();
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}

}  // namespace sfda
