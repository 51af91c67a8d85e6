// Linear attention with a fixed decay for each head: what the kernels and their callers share.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sfda {

// One pass of the chunk form.  With g = exp(log_decay[h]) and n = lens[b] (or T), for t = 0 .. n - 1
//
//   out_t = sp sum_{i <= t} g^(t - i) (a_t . b_i) c_i + se g^(t + 1) S_in^T a_t
//   S_out = g^n S_in + sw sum_i g^(n - 1 - i) b_i c_i^T
//
// and with `reverse` the same on reversed time in the form that gradients take:
//
//   out_t = sp sum_{i >= t} g^(i - t) (a_t . b_i) c_i + se g^(n - 1 - t) S_in^T a_t
//   S_out = g^n S_in + sw sum_i g^(i + 1) b_i c_i^T
//
// The forward is (a, b, c) = (q, k, v).  Of the gradients, dq is the forward pass on (d_o, v, k) with the initial state
// transposed; dv and dk are reverse passes on (k, q, d_o) and (v, d_o, q), the second with a transposed state; what
// the first of them leaves at the front is dS0.
struct LinearPass {
    const void *a, *b, *c;      // [B][T][Ha][DA], [B][T][Hb][DA], [B][T][Hc][DC]; head h reads head h / (H / Hx)
    void *out;                  // [B][T][H][DC], in the dtype of the call, or float with out_f32
    const float *s_in;          // [B][H][DA][DC] ([DC][DA] with s_in_t), or NULL for zero
    float *s_out;               // [B][H][DA][DC], or NULL
    int Ha, Hb, Hc, DA, DC;
    int reverse = 0, s_in_t = 0, out_f32 = 0;
    float sp, se, sw;
};

struct LinearArgs {
    const float *log_decay;     // [H]
    const int *lens;            // [B] or NULL
    int B, T, H, dtype;
};

// fp32 passes on the warp-level tensor cores (operands split into two tf32 parts).
cudaError_t launch_linear_f32(const LinearArgs &a, const LinearPass *passes, int count, cudaStream_t stream, int *launches);

// bf16 passes on tcgen05.  The workspace begins with the status word that sfda_workspace_status reads.
size_t linear_tc_bytes(const LinearArgs &a, int passes, int d_k, int d_v);
cudaError_t launch_linear_tc(const LinearArgs &a, const LinearPass *passes, int count, void *workspace, cudaStream_t stream,
                             int *launches);

// The entry points' work: passes, and the sums of shared heads' gradients.
size_t linear_forward_bytes(const LinearArgs &a, int d_k, int d_v);
cudaError_t launch_linear_forward(const LinearArgs &a, const void *q, const void *k, const void *v, const float *S0, void *o,
                                  float *S_T, int H_kv, int d_k, int d_v, float scale, void *workspace, cudaStream_t stream,
                                  int *launches);
size_t linear_backward_bytes(const LinearArgs &a, int H_kv, int d_k, int d_v);
cudaError_t launch_linear_backward(const LinearArgs &a, const void *q, const void *k, const void *v, const float *S0,
                                   const void *d_o, const float *dS_T, void *dq, void *dk, void *dv, float *dS0, int H_kv,
                                   int d_k, int d_v, float scale, void *workspace, cudaStream_t stream, int *launches);

struct LinearStepArgs {
    const void *q, *k, *v;
    const float *log_decay;
    float *S;
    void *o;
    int B, H, H_kv, d_k, d_v, dtype;
    float scale;
};
cudaError_t launch_linear_step(const LinearStepArgs &a, cudaStream_t stream, int *launches);

struct RotaryArgs {
    const void *q, *k;          // k may be NULL
    void *q_out, *k_out;
    const int *positions;       // [B][T]
    const uint64_t *turns;      // [rot / 2]
    long long rows;             // B * T
    long long q_stride, k_stride, qo_stride, ko_stride;   // elements from one token to the next
    int H, H_kv, d, rot, layout, inverse, dtype;
    float amplitude;
};
cudaError_t launch_rotary(const RotaryArgs &a, cudaStream_t stream, int *launches);

struct GroupNormArgs {
    const void *x, *gate, *dy;
    const float *weight, *bias;
    void *y, *dx, *dgate;
    float *dweight, *dbias;
    long long rows;
    int C, G, act, dtype;
    float eps;
};
bool group_norm_supported(int C, int G, int dtype);
cudaError_t launch_group_norm(const GroupNormArgs &a, cudaStream_t stream, int *launches);
size_t group_norm_backward_bytes(long long rows, int C);
cudaError_t launch_group_norm_backward(const GroupNormArgs &a, void *workspace, cudaStream_t stream, int *launches);

}  // namespace sfda
