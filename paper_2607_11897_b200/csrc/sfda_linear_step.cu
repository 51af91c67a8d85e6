// sfda_linear_step: one token of linear attention with a fixed decay for each head,
//
//     S <- g_h S + k v^T,    o = scale S^T q.
//
// HBM-bound: the fp32 state of a (batch, head) pair is read once and written once.  The columns of a state never
// interact, so one CTA of 128 threads takes a block of CT value columns; a thread owns four adjacent columns (16-byte
// accesses) of DK / RG rows, all of whose loads are issued before anything waits for one.
#include "sfda_common.cuh"
#include "sfda_linear.h"
#include "sfda_vec.cuh"

namespace sfda {
namespace {

constexpr int kThreads = 128;

__device__ __forceinline__ float4 ld_state(const float *p)
{
    float4 v;
    asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
    return v;
}

template <int DK, int DV, int CT, typename T>
__global__ void __launch_bounds__(kThreads)
sfda_linear_step_kernel(const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v,
                        const float *__restrict__ log_decay, float *__restrict__ S, T *__restrict__ o, int H, int H_kv, float scale)
{
    constexpr int CG = CT / 4, RG = kThreads / CG, R = DK / RG;
    static_assert(R >= 1 && DK % RG == 0, "row groups must divide the rows");
    __shared__ float s_q[DK], s_k[DK];
    __shared__ float4 s_red[RG][CG];
    const int tid = threadIdx.x, cg = tid % CG, rg = tid / CG;
    const size_t bh = blockIdx.x;
    const int b = blockIdx.x / H, h = blockIdx.x % H, c0 = blockIdx.y * CT;
    const size_t kv = (size_t)b * H_kv + h / (H / H_kv);
    float *at = S + (bh * DK + rg * R) * DV + c0 + 4 * cg;
    float4 s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = ld_state(at + (size_t)r * DV);
    const float ld = log_decay[h];
    float vv[4];
    ld_vec(v + kv * DV + c0 + 4 * cg, vv);
    for (int i = tid; i < DK; i += kThreads) {
        s_q[i] = ld_val(q, bh * DK + i);
        s_k[i] = ld_val(k, kv * DK + i);
    }
    // A state decays by the same factor step after step: near 1 its rounding would add up, so weak decays go through
    // g - 1, which keeps its own relative precision.
    const bool weak = ld > -0.5f;
    const float gm = weak ? expm1f(ld) : expf(ld);
    __syncthreads();
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float kr = s_k[rg * R + r], qr = s_q[rg * R + r];
        float4 x = s[r];
        x.x = fmaf(kr, vv[0], weak ? fmaf(x.x, gm, x.x) : x.x * gm);
        x.y = fmaf(kr, vv[1], weak ? fmaf(x.y, gm, x.y) : x.y * gm);
        x.z = fmaf(kr, vv[2], weak ? fmaf(x.z, gm, x.z) : x.z * gm);
        x.w = fmaf(kr, vv[3], weak ? fmaf(x.w, gm, x.w) : x.w * gm);
        *reinterpret_cast<float4 *>(at + (size_t)r * DV) = x;
        acc.x = fmaf(qr, x.x, acc.x);
        acc.y = fmaf(qr, x.y, acc.y);
        acc.z = fmaf(qr, x.z, acc.z);
        acc.w = fmaf(qr, x.w, acc.w);
    }
    s_red[rg][cg] = acc;
    __syncthreads();
    if (tid < CG) {
        float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < RG; ++i) {
            const float4 x = s_red[i][tid];
            y[0] += x.x; y[1] += x.y; y[2] += x.z; y[3] += x.w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] *= scale;
        st_vec(o + bh * DV + c0 + 4 * tid, y);
    }
}

template <int DK, int DV, typename T>
cudaError_t launch_one(const LinearStepArgs &a, cudaStream_t stream)
{
    constexpr int CT = 64;
    sfda_linear_step_kernel<DK, DV, CT, T><<<dim3((unsigned)a.B * a.H, DV / CT), kThreads, 0, stream>>>(
        static_cast<const T *>(a.q), static_cast<const T *>(a.k), static_cast<const T *>(a.v), a.log_decay, a.S,
        static_cast<T *>(a.o), a.H, a.H_kv, a.scale);
    return cudaGetLastError();
}

template <typename T>
cudaError_t dispatch(const LinearStepArgs &a, cudaStream_t stream)
{
    if (a.d_k == 128 && a.d_v == 128) return launch_one<128, 128, T>(a, stream);
    if (a.d_k == 128 && a.d_v == 64) return launch_one<128, 64, T>(a, stream);
    if (a.d_k == 64 && a.d_v == 128) return launch_one<64, 128, T>(a, stream);
    if (a.d_k == 64 && a.d_v == 64) return launch_one<64, 64, T>(a, stream);
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_linear_step(const LinearStepArgs &a, cudaStream_t stream, int *launches)
{
    const cudaError_t e = a.dtype == 1 ? dispatch<__nv_bfloat16>(a, stream) : dispatch<float>(a, stream);
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}

}  // namespace sfda
