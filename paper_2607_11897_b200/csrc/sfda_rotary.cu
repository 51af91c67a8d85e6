// sfda_rotary: the first `rot` channels of every head of q and k, as rot / 2 pairs, turned by position * frequency.
//
// Frequencies come as 64-bit counts of 2^-64 turns.  position * count, modulo 2^64, is the exact angle within the turn
// however far the position is (the same device as the recurrence's integer phases); its top 32 bits go to sincospif.
// Bound by memory: a thread takes V pairs of one token and applies their cosines and sines, computed once, to HT heads.
#include "sfda_common.cuh"
#include "sfda_linear.h"
#include "sfda_vec.cuh"

namespace sfda {
namespace {

constexpr int kThreads = 256;
constexpr int HT = 16;           // heads per thread at most
constexpr int kBatch = 4;

struct Dev {
    const void *q, *k;
    void *q_out, *k_out;
    const int *positions;
    const uint64_t *turns;
    long long rows, q_stride, k_stride, qo_stride, ko_stride;
    int H, H_kv, d, rot, inverse, ht;
    float amplitude;
};

// One work item: V channels (pairs layout) or V channels of the first half and V of the second (halves layout) of one
// token, or V channels that are only copied.  `items` items make a token.
template <typename T, int V, bool kHalves>
__global__ void __launch_bounds__(kThreads) sfda_rotary_kernel(const Dev p, const int items)
{
    const long long at = blockIdx.x * (long long)kThreads + threadIdx.x;
    const long long row = at / items;
    if (row >= p.rows) return;
    const int it = (int)(at % items), half = p.rot / 2;
    constexpr int NP = kHalves ? V : (V > 1 ? V / 2 : 1);     // pairs of this item
    constexpr int NX = kHalves ? 2 * V : (V > 1 ? V : 2);     // channels of this item
    const bool turned = kHalves ? it < half / V : it * NX < p.rot;
    // channel of the first element, and of the second half's first
    const int c = kHalves ? (turned ? it * V : p.rot + (it - half / V) * V) : it * NX;
    float cs[NP], sn[NP];
    bool on[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) on[i] = false;
    if (turned) {
        const uint64_t pos = (uint64_t)(int64_t)p.positions[row];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int pair = kHalves ? c + i : c / 2 + i;
            on[i] = pair < half;
            const uint64_t u = pos * (on[i] ? p.turns[pair] : 0ull);
            turns_to_cos_sin((uint32_t)((u + 0x80000000ull) >> 32), &cs[i], &sn[i]);
            cs[i] *= p.amplitude;
            sn[i] *= p.inverse ? -p.amplitude : p.amplitude;
        }
    }
    const int heads = p.H + p.H_kv, h0 = blockIdx.y * p.ht, h1 = min(h0 + p.ht, heads);
    // kBatch heads are read before the first of them is written: outputs may be inputs, so the compiler has to keep the order.
    constexpr int NV = kHalves ? V : NX;                      // elements of one access
    for (int hb = h0; hb < h1; hb += kBatch) {
        Raw<T, NV> a[kBatch], b[kHalves ? kBatch : 1];
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
            const int h = hb + n;
            if (h >= h1) continue;
            const T *x = h < p.H ? static_cast<const T *>(p.q) + row * p.q_stride + (long long)h * p.d
                                 : static_cast<const T *>(p.k) + row * p.k_stride + (long long)(h - p.H) * p.d;
            a[n].load(x + c);
            if (kHalves && turned) b[n].load(x + c + half);
        }
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
            const int h = hb + n;
            if (h >= h1) continue;
            T *y = h < p.H ? static_cast<T *>(p.q_out) + row * p.qo_stride + (long long)h * p.d
                           : static_cast<T *>(p.k_out) + row * p.ko_stride + (long long)(h - p.H) * p.d;
            float re[NV], im[kHalves ? NV : 1];
            if constexpr (kHalves) {
#pragma unroll
                for (int i = 0; i < NV; ++i) re[i] = a[n].get(i);
                if (turned) {
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const float u = re[i], v = b[n].get(i);
                        re[i] = u * cs[i] - v * sn[i];
                        im[i] = u * sn[i] + v * cs[i];
                    }
                    st_vec(y + c + half, im);
                }
                st_vec(y + c, re);
            } else {
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const float u = a[n].get(2 * i), v = a[n].get(2 * i + 1);
                    const bool t = turned && on[i];
                    re[2 * i] = t ? u * cs[i] - v * sn[i] : u;
                    re[2 * i + 1] = t ? u * sn[i] + v * cs[i] : v;
                }
                st_vec(y + c, re);
            }
        }
    }
}

template <typename T, int V, bool kHalves>
cudaError_t launch_v(const RotaryArgs &a, cudaStream_t stream)
{
    const int items = kHalves ? (a.rot / 2 + (a.d - a.rot)) / V : a.d / (V > 1 ? V : 2);
    const long long blocks = (a.rows * items + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    // few tokens: fewer heads to a thread, until the device is full (256 tokens of 40 heads: 7.1 us with 8, 5 with 4)
    int ht = HT;
    while (ht > kBatch && blocks * ((a.H + a.H_kv + ht - 1) / ht) < 148 * 8) ht /= 2;
    const Dev p = {a.q, a.k, a.q_out, a.k_out, a.positions, a.turns, a.rows, a.q_stride, a.k_stride, a.qo_stride, a.ko_stride,
                   a.H, a.H_kv, a.d, a.rot, a.inverse, ht, a.amplitude};
    sfda_rotary_kernel<T, V, kHalves><<<dim3((unsigned)blocks, (a.H + a.H_kv + ht - 1) / ht), kThreads, 0, stream>>>(p, items);
    return cudaGetLastError();
}

// The widest access that channels, strides and addresses all are multiples of (in elements).
int widest(const RotaryArgs &a, int most)
{
    const size_t e = a.dtype == 1 ? 2 : 4;
    for (int v = most; v > 1; v /= 2) {
        bool ok = a.d % v == 0 && a.q_stride % v == 0 && a.qo_stride % v == 0 && (!a.k || (a.k_stride % v == 0 && a.ko_stride % v == 0));
        if (a.layout == 1) ok = ok && (a.rot / 2) % v == 0 && (a.d - a.rot) % v == 0;
        const void *ptr[] = {a.q, a.k, a.q_out, a.k_out};
        for (const void *x : ptr) ok = ok && reinterpret_cast<uintptr_t>(x) % (v * e < 16 ? v * e : 16) == 0;
        if (ok) return v;
    }
    return 1;
}

template <typename T>
cudaError_t dispatch(const RotaryArgs &a, cudaStream_t stream)
{
    constexpr int kMost = 16 / (int)sizeof(T);
    const int v = widest(a, kMost);
    if (a.layout == 1) {
        if constexpr (kMost == 8)
            if (v == 8) return launch_v<T, 8, true>(a, stream);
        return v == 4 ? launch_v<T, 4, true>(a, stream) : v == 2 ? launch_v<T, 2, true>(a, stream) : launch_v<T, 1, true>(a, stream);
    }
    if constexpr (kMost == 8)
        if (v == 8) return launch_v<T, 8, false>(a, stream);
    return v == 4 ? launch_v<T, 4, false>(a, stream) : launch_v<T, 2, false>(a, stream);
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs &a, cudaStream_t stream, int *launches)
{
    const cudaError_t e = a.dtype == 1 ? dispatch<__nv_bfloat16>(a, stream) : dispatch<float>(a, stream);
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}

}  // namespace sfda
