// switchsd_logprobs.hip -- gfx950 kernels for the log probabilities of given
// tokens, entropies, ranks and the most likely alternatives (k_logprob), and
// the gradient of the first two with respect to the logits (k_logprob_grad).
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "switchsd_device.h"
#include "switchsd_internal.h"

namespace switchsd {

namespace {

constexpr int kWaves = kThreads / 64;

template <int TYPE>
__device__ __forceinline__ float load_logit(const void *base, int64_t at) {
    if (TYPE == SWITCHSD_F32)
        return ((const float *)base)[at];
    const uint16_t v = ((const uint16_t *)base)[at];
    if (TYPE == SWITCHSD_BF16)
        return __builtin_bit_cast(float, (uint32_t)v << 16);
    return (float)__builtin_bit_cast(_Float16, v);
}

template <int TYPE>
__device__ __forceinline__ void store_logit(void *base, int64_t at, float v) {
    if (TYPE == SWITCHSD_F32)
        ((float *)base)[at] = v;
    else if (TYPE == SWITCHSD_BF16)
        ((uint16_t *)base)[at] = __builtin_bit_cast(uint16_t, (__bf16)v);
    else
        ((uint16_t *)base)[at] = __builtin_bit_cast(uint16_t, (_Float16)v);
}

// The row of entry (b, i), or -1 where there is none.
__device__ __forceinline__ int entry_row(const switchsd_logprob_args &a, int b, int i) {
    const int n = a.dn ? clampi(a.dn[b], 1, a.R) : a.R;
    if (!a.accept_node)
        return i < n ? i : -1;
    const int last = a.accept_node[b];
    if (last < 0 || last >= n)
        return -1;
    if (!a.dpar)
        return i <= last ? i : -1;
    // the path's depth, then its i-th node
    int depth = 0;
    for (int x = last; x > 0; ++depth) {
        const int up = a.dpar[(int64_t)b * a.R + x];
        if (up < 0 || up >= x)
            return -1;
        x = up;
    }
    if (i > depth)
        return -1;
    int x = last;
    for (int d = depth; d > i; --d)
        x = a.dpar[(int64_t)b * a.R + x];
    return x;
}

// Keys that order logits: larger first, then the lower index; NaN behind all
// numbers.  Never 0.
__device__ __forceinline__ unsigned long long order_key(float l, uint32_t v) {
    uint32_t s = 0;
    if (l == l) {
        const uint32_t u = __builtin_bit_cast(uint32_t, l + 0.0f);
        s = (u & 0x80000000u) ? ~u : u | 0x80000000u;
    }
    return ((unsigned long long)s << 32) | (0xFFFFFFFFu - v);
}

__device__ __forceinline__ unsigned long long block_max(unsigned long long v,
                                                        unsigned long long *sh) {
    for (int x = 32; x; x >>= 1) {
        const unsigned long long o = __shfl_xor(v, x);
        v = o > v ? o : v;
    }
    if ((threadIdx.x & 63) == 0)
        sh[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w)
        v = sh[w] > v ? sh[w] : v;
    __syncthreads();
    return v;
}

__device__ __forceinline__ double block_sum(double v, double *sh) {
    for (int x = 32; x; x >>= 1)
        v += __shfl_xor(v, x);
    if ((threadIdx.x & 63) == 0)
        sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < kWaves; ++w)
        v += sh[w];
    __syncthreads();
    return v;
}

__device__ __forceinline__ float key_logit(unsigned long long key) {
    const uint32_t s = (uint32_t)(key >> 32);
    return __builtin_bit_cast(float, s == 0 ? 0x7FC00000u : (s >> 31) ? s & 0x7FFFFFFFu : ~s);
}
__device__ __forceinline__ uint32_t key_token(unsigned long long key) {
    return 0xFFFFFFFFu - (uint32_t)key;
}

// A work-group per entry.
template <int TYPE>
__global__ void __launch_bounds__(kThreads) k_logprob(const LogprobParams p) {
    const switchsd_logprob_args &a = p.a;
    __shared__ unsigned long long sk[kWaves];
    __shared__ double sd[kWaves];
    const int64_t e = blockIdx.x;
    const int b = e / a.R, i = e % a.R, tid = threadIdx.x;
    const int r = entry_row(a, b, i);
    if (r < 0)
        return;
    const int64_t row = ((int64_t)b * a.R + r) * a.V;
    unsigned long long best = 0;
    for (int v = tid; v < a.V; v += kThreads) {
        const unsigned long long k = order_key(load_logit<TYPE>(a.logits, row + v), v);
        best = k > best ? k : best;
    }
    best = block_max(best, sk);
    const float m = key_logit(best);
    const bool flat = !(fabsf(m) < INFINITY);  // no finite maximum: one-hot
    const int tok = a.tokens ? a.tokens[e] : -1;
    const bool in = tok >= 0 && tok < a.V;
    const float lt = in ? load_logit<TYPE>(a.logits, row + tok) : 0.0f;
    const unsigned long long kt = in ? order_key(lt, tok) : 0;
    double s = 0.0, t = 0.0, ahead = 0.0;
    for (int v = tid; v < a.V; v += kThreads) {
        const float l = load_logit<TYPE>(a.logits, row + v);
        ahead += order_key(l, v) > kt ? 1.0 : 0.0;
        const float x = (l - m) * p.inv_t, w = l == l && !flat ? expf(x) : 0.0f;
        s += w;
        t += w > 0.0f ? (double)w * x : 0.0;
    }
    s = block_sum(s, sd);
    t = block_sum(t, sd);
    ahead = block_sum(ahead, sd);
    const float ls = flat ? 0.0f : (float)log(s);
    const uint32_t greedy = key_token(best);
    const auto logprob = [&](float l, uint32_t v) {
        if (flat)
            return v == greedy ? 0.0f : -INFINITY;
        return l == l ? (l - m) * p.inv_t - ls : -INFINITY;
    };
    if (tid == 0) {
        if (p.logprob)
            p.logprob[e] = in ? logprob(lt, tok) : -INFINITY;
        if (p.lse)
            p.lse[e] = m != m ? -INFINITY : flat ? m : m * p.inv_t + ls;
        if (p.entropy)
            p.entropy[e] = flat ? 0.0f : (float)(log(s) - t / s);
        if (p.rank)
            p.rank[e] = in ? (int)ahead : -1;
    }
    for (int j = 0; j < p.n_top; ++j) {
        if (j > 0) {
            unsigned long long next = 0;
            for (int v = tid; v < a.V; v += kThreads) {
                const unsigned long long k = order_key(load_logit<TYPE>(a.logits, row + v), v);
                next = k < best && k > next ? k : next;
            }
            best = block_max(next, sk);
        }
        if (tid == 0) {
            if (p.top_ids)
                p.top_ids[e * p.n_top + j] = (int)key_token(best);
            if (p.top_logprobs)
                p.top_logprobs[e * p.n_top + j] = logprob(key_logit(best), key_token(best));
        }
    }
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads) k_logprob_grad(const LogprobParams p) {
    const switchsd_logprob_args &a = p.a;
    const int64_t e = blockIdx.x;
    const int b = e / a.R, i = e % a.R;
    const int r = entry_row(a, b, i);
    if (r < 0)
        return;
    const int64_t row = ((int64_t)b * a.R + r) * a.V;
    const float lse = p.in_lse[e];
    const float g = p.g_logprob ? p.g_logprob[e] : 0.0f;
    const float ge = p.g_entropy ? p.g_entropy[e] : 0.0f;
    const float H = p.g_entropy ? p.in_entropy[e] : 0.0f;
    const int tok = p.g_logprob ? a.tokens[e] : -1;
    const bool flat = !(fabsf(lse) < INFINITY);
    for (int v = threadIdx.x; v < a.V; v += kThreads) {
        const float l = load_logit<TYPE>(a.logits, row + v);
        const float x = l * p.inv_t - lse, w = l == l ? expf(x) : 0.0f;
        const float d = w > 0.0f ? -w * (g + ge * (x + H)) : 0.0f;
        store_logit<TYPE>(p.grad, row + v, flat ? 0.0f : (d + (v == tok ? g : 0.0f)) * p.inv_t);
    }
}

int launched() { return hipGetLastError() == hipSuccess ? SWITCHSD_OK : SWITCHSD_EHIP; }

}  // namespace

int launch_logprob_kernel(const LogprobParams &p, hipStream_t stream) {
    const dim3 g((unsigned)((int64_t)p.a.B * p.a.R)), t(kThreads);
    if (p.a.logits_type == SWITCHSD_BF16)
        hipLaunchKernelGGL((k_logprob<SWITCHSD_BF16>), g, t, 0, stream, p);
    else if (p.a.logits_type == SWITCHSD_F16)
        hipLaunchKernelGGL((k_logprob<SWITCHSD_F16>), g, t, 0, stream, p);
    else
        hipLaunchKernelGGL((k_logprob<SWITCHSD_F32>), g, t, 0, stream, p);
    return launched();
}

int launch_logprob_grad_kernel(const LogprobParams &p, hipStream_t stream) {
    const dim3 g((unsigned)((int64_t)p.a.B * p.a.R)), t(kThreads);
    if (p.a.logits_type == SWITCHSD_BF16)
        hipLaunchKernelGGL((k_logprob_grad<SWITCHSD_BF16>), g, t, 0, stream, p);
    else if (p.a.logits_type == SWITCHSD_F16)
        hipLaunchKernelGGL((k_logprob_grad<SWITCHSD_F16>), g, t, 0, stream, p);
    else
        hipLaunchKernelGGL((k_logprob_grad<SWITCHSD_F32>), g, t, 0, stream, p);
    return launched();
}

}  // namespace switchsd
