// sfda_linear_forward and sfda_linear_backward as passes of the chunk form (sfda_linear.h), and the sums over the query heads
// that share a key and value head.
#include "sfda_linear.h"
#include "sfda_tc_ptx.cuh"

namespace sfda {
namespace {

// out[r][g][d] = sum over the `share` consecutive heads of x[r][g * share + j][d], rounded once; rows behind a sequence's end are
// left as they are.  Four channels of one (row, group) per thread.
template <typename T>
__global__ void __launch_bounds__(256) sfda_linear_sum_heads_kernel(const float *__restrict__ x, T *__restrict__ out, const int *lens,
                                                                   int Tn, int share, int per_row, int d, long long total)
{
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const long long row = i / per_row;
        if (lens && (int)(row % Tn) >= lens[row / Tn]) continue;
        const int e = (int)(i % per_row) * 4, grp = e / d, c = e % d;
        const float *at = x + (row * (per_row * 4 / d) + grp) * (long long)share * d + c;
        float4 s = *reinterpret_cast<const float4 *>(at);
        for (int j = 1; j < share; ++j) {
            const float4 y = *reinterpret_cast<const float4 *>(at + (long long)j * d);
            s.x += y.x; s.y += y.y; s.z += y.z; s.w += y.w;
        }
        T *o = out + i * 4;
        if (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(o) = s;
        } else {
            uint2 w = {tc::pack_bf16(s.x, s.y), tc::pack_bf16(s.z, s.w)};
            *reinterpret_cast<uint2 *>(o) = w;
        }
    }
}

cudaError_t launch_sum_heads(const float *x, void *out, const LinearArgs &a, int H_kv, int d, cudaStream_t stream, int *launches)
{
    const int per_row = H_kv * d / 4, share = a.H / H_kv;
    const long long total = (long long)a.B * a.T * per_row, blocks = (total + 255) / 256;
    const unsigned grid = (unsigned)(blocks < 148 * 16 ? blocks : 148 * 16);
    if (a.dtype == 1)
        sfda_linear_sum_heads_kernel<<<grid, 256, 0, stream>>>(x, static_cast<__nv_bfloat16 *>(out), a.lens, a.T, share, per_row, d, total);
    else
        sfda_linear_sum_heads_kernel<<<grid, 256, 0, stream>>>(x, static_cast<float *>(out), a.lens, a.T, share, per_row, d, total);
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}
size_t round256(size_t x) { return (x + 255u) & ~(size_t)255u; }

cudaError_t run_passes(const LinearArgs &a, const LinearPass *p, int count, void *workspace, cudaStream_t stream, int *launches)
{
    return a.dtype == 1 ? launch_linear_tc(a, p, count, workspace, stream, launches) : launch_linear_f32(a, p, count, stream, launches);
}
size_t pass_bytes(const LinearArgs &a, int count, int d_k, int d_v)
{
    return a.dtype == 1 ? round256(linear_tc_bytes(a, count, d_k, d_v)) : 0;
}

}  // namespace

size_t linear_forward_bytes(const LinearArgs &a, int d_k, int d_v) { return pass_bytes(a, 1, d_k, d_v); }

cudaError_t launch_linear_forward(const LinearArgs &a, const void *q, const void *k, const void *v, const float *S0, void *o,
                                  float *S_T, int H_kv, int d_k, int d_v, float scale, void *workspace, cudaStream_t stream,
                                  int *launches)
{
    LinearPass p = {q, k, v, o, S0, S_T, a.H, H_kv, H_kv, d_k, d_v};
    p.sp = p.se = scale;
    p.sw = 1.f;
    return run_passes(a, &p, 1, workspace, stream, launches);
}

// the passes' scratch; with shared heads also the gradients of every query head in fp32, before their sums
size_t linear_backward_bytes(const LinearArgs &a, int H_kv, int d_k, int d_v)
{
    const size_t rows = (size_t)a.B * a.T * a.H;
    return pass_bytes(a, 3, d_k, d_v) + (H_kv == a.H ? 0 : round256(rows * d_k * 4) + round256(rows * d_v * 4));
}

cudaError_t launch_linear_backward(const LinearArgs &a, const void *q, const void *k, const void *v, const float *S0,
                                   const void *d_o, const float *dS_T, void *dq, void *dk, void *dv, float *dS0, int H_kv,
                                   int d_k, int d_v, float scale, void *workspace, cudaStream_t stream, int *launches)
{
    const bool shared = H_kv != a.H;
    float *dk_h = reinterpret_cast<float *>(static_cast<char *>(workspace) + pass_bytes(a, 3, d_k, d_v));
    float *dv_h = dk_h + round256((size_t)a.B * a.T * a.H * d_k * 4) / 4;
    LinearPass p[3] = {{d_o, v, k, dq, S0, nullptr, a.H, H_kv, H_kv, d_v, d_k},
                       {v, d_o, q, shared ? dk_h : dk, dS_T, nullptr, H_kv, a.H, a.H, d_v, d_k},
                       {k, q, d_o, shared ? dv_h : dv, dS_T, dS0, H_kv, a.H, a.H, d_k, d_v}};
    p[0].s_in_t = 1;
    p[0].sp = p[0].se = scale;
    p[0].sw = 1.f;
    for (int i = 1; i < 3; ++i) {
        p[i].reverse = 1;
        p[i].out_f32 = shared;
        p[i].sp = p[i].sw = scale;
        p[i].se = 1.f;
    }
    p[1].s_in_t = 1;
    cudaError_t e = run_passes(a, p, 3, workspace, stream, launches);
    if (e != cudaSuccess) return e;
    if (!shared) return cudaSuccess;
    e = launch_sum_heads(dk_h, dk, a, H_kv, d_k, stream, launches);
    return e == cudaSuccess ? launch_sum_heads(dv_h, dv, a, H_kv, d_v, stream, launches) : e;
}

}  // namespace sfda
