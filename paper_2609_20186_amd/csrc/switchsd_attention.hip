// switchsd_attention.hip -- gfx950 kernels for the contents of a paged KV cache:
// the new tokens' keys and values written to their slots (k_store) and the
// attention of new tokens over the cache (k_attend).
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "switchsd_device.h"
#include "switchsd_internal.h"

namespace switchsd {

namespace {

// ---- elements

template <int TYPE>
__device__ __forceinline__ float to_f32(uint16_t v) {
    if (TYPE == SWITCHSD_BF16)
        return __builtin_bit_cast(float, (uint32_t)v << 16);
    return (float)__builtin_bit_cast(_Float16, v);
}

template <int TYPE>
__device__ __forceinline__ uint16_t from_f32(float v) {
    if (TYPE == SWITCHSD_BF16)
        return __builtin_bit_cast(uint16_t, (__bf16)v);
    return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// ---- keys and values of new tokens

// Two 8-bit floats in the low or high half of `old`: the conversion rounds to
// nearest even; what lies beyond the largest value (448) is set to it before,
// NaN passes both comparisons.
template <bool HIGH>
__device__ __forceinline__ int pack_e4m3(float a, float b, int old) {
    a = a > 448.0f ? 448.0f : (a < -448.0f ? -448.0f : a);
    b = b > 448.0f ? 448.0f : (b < -448.0f ? -448.0f : b);
    return __builtin_amdgcn_cvt_pk_fp8_f32(a, b, old, HIGH);
}

// A lane per 16 bytes of a row's keys or values.  Moves 4 Hkv D bytes in and as
// many (or half) out: bound by its launch for the rows of a step, by the memory
// for prompts.
template <int TYPE, bool E4M3>
__global__ void __launch_bounds__(kThreads) k_store(const StoreParams p) {
    const uint32_t vecs = (uint32_t)(p.Hkv * p.D) / 8;
    const int64_t n = p.count ? clampi(p.count[0], 0, p.n) : p.n;
    const int64_t total = n * (2 * vecs);
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total;
         i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / (2 * vecs);
        uint32_t at = (uint32_t)(i - row * (2 * vecs));
        const bool val = at >= vecs;
        at -= val ? vecs : 0;
        const char *src = (const char *)(val ? p.v : p.k) + row * (val ? p.v_stride : p.k_stride);
        const u32x4 x = *(const u32x4 *)(src + (size_t)at * 16);
        const int64_t slot = p.slots[row];
        if (slot < 0 || slot >= p.n_slots)
            continue;
        char *dst = (char *)(val ? p.v_cache : p.k_cache);
        if (!E4M3) {
            *(u32x4 *)(dst + (slot * vecs + at) * 16) = x;
            continue;
        }
        const float *scales = val ? p.v_scale : p.k_scale;
        const float scale = scales ? scales[at * 8 / (uint32_t)p.D] : 1.0f;
        int out[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float f[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                f[e] = to_f32<TYPE>((uint16_t)(x[j * 2 + e / 2] >> (e % 2 * 16))) / scale;
            out[j] = pack_e4m3<true>(f[2], f[3], pack_e4m3<false>(f[0], f[1], 0));
        }
        *(int2 *)(dst + (slot * vecs + at) * 8) = make_int2(out[0], out[1]);
    }
}

// ---- attention

// A sequence's new rows: how many, the row of the first in q and out, and its
// cache position.
struct Chunk {
    int n, row, pos;
};
__device__ __forceinline__ Chunk chunk_of(const switchsd_attention_args &a, int b) {
    Chunk c;
    if (a.cu) {
        const int lo = a.cu[b], hi = a.cu[b + 1];
        const bool ok = lo >= 0 && hi >= lo && hi <= a.rows;
        c.n = ok ? (hi - lo < a.R ? hi - lo : a.R) : 0;
        c.row = ok ? lo : 0;
        c.pos = clampi(a.begin[b], 0, a.Lmax);
    } else {
        const int L = clampi(a.lengths[b], 0, a.Lmax);
        c.n = L > 0 ? clampi(a.dn[b], 1, a.R) : 0;
        c.row = b * a.R;
        c.pos = L - 1;
    }
    return c;
}

template <int TYPE, bool E4M3>
__device__ __forceinline__ float cached(const void *base, int64_t at) {
    if (E4M3)
        return __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)base)[at], 0);
    return to_f32<TYPE>(((const uint16_t *)base)[at]);
}

// A wave per row and query head, a key per lane.
template <int TYPE, bool E4M3, int D>
__global__ void __launch_bounds__(64) k_attend(const AttnParams p) {
    const switchsd_attention_args &a = p.a;
    __shared__ float sq[D];
    const int lane = threadIdx.x;
    int64_t id = blockIdx.x;
    const int h = id % a.Hq;
    id /= a.Hq;
    const int i = id % a.R, b = id / a.R;
    const Chunk c = chunk_of(a, b);
    if (i >= c.n)
        return;
    const int hk = h / p.G;
    const int64_t row = c.row + i;
    const uint16_t *q = (const uint16_t *)p.q + row * p.q_stride + (int64_t)h * D;
    for (int d = lane; d < D; d += 64)
        sq[d] = to_f32<TYPE>(q[d]);
    __syncthreads();
    const float sk = a.scale * (p.k_scale ? p.k_scale[hk] : 1.0f);
    const int held = clampi(a.held[b], 0, a.max_pages);
    const int64_t end = (int64_t)c.pos + c.n;
    const int words = (a.R + 31) / 32;
    float m = -INFINITY, l = 0.0f, o[D / 64];
    for (int t = 0; t < D / 64; ++t)
        o[t] = 0.0f;
    for (int64_t k0 = 0; k0 < end; k0 += 64) {
        const int64_t pos = k0 + lane;
        bool seen = pos < end && pos / a.page_size < held;
        int64_t slot = 0;
        if (seen) {
            slot = (int64_t)a.table[(int64_t)b * a.max_pages + pos / a.page_size] * a.page_size +
                   pos % a.page_size;
            seen = slot >= 0 && slot < p.n_slots;
            slot = seen ? slot : 0;
        }
        const int64_t j = pos - c.pos;
        if (seen && j >= 0)
            seen = a.mask ? (a.mask[row * words + j / 32] >> (j % 32)) & 1 : j <= i;
        float s = -INFINITY;
        if (seen) {
            s = 0.0f;
            for (int d = 0; d < D; ++d)
                s = fmaf(sq[d], cached<TYPE, E4M3>(p.k_cache, (slot * a.Hkv + hk) * D + d), s);
            s *= sk;
        }
        float top = s;
        for (int x = 32; x; x >>= 1)
            top = fmaxf(top, __shfl_xor(top, x));
        const float mn = fmaxf(m, top), ms = mn == -INFINITY ? 0.0f : mn;
        const float w = seen ? expf(s - ms) : 0.0f, alpha = expf(m - ms);
        m = mn;
        float sum = w;
        for (int x = 32; x; x >>= 1)
            sum += __shfl_xor(sum, x);
        l = l * alpha + sum;
        for (int t = 0; t < D / 64; ++t)
            o[t] *= alpha;
        for (int y = 0; y < 64; ++y) {
            if (!__shfl((int)seen, y))
                continue;
            const float wy = __shfl(w, y);
            const int64_t at = (__shfl((long long)slot, y) * a.Hkv + hk) * D + lane;
            for (int t = 0; t < D / 64; ++t)
                o[t] = fmaf(wy, cached<TYPE, E4M3>(p.v_cache, at + t * 64), o[t]);
        }
    }
    const float sv = p.v_scale ? p.v_scale[hk] : 1.0f;
    uint16_t *out = (uint16_t *)p.out + (row * a.Hq + h) * D;
    for (int t = 0; t < D / 64; ++t)
        out[t * 64 + lane] = from_f32<TYPE>(l == 0.0f ? 0.0f : o[t] / l * sv);
    if (p.lse && lane == 0)
        p.lse[row * a.Hq + h] = l == 0.0f ? -INFINITY : m + logf(l);
}

int launched() { return hipGetLastError() == hipSuccess ? SWITCHSD_OK : SWITCHSD_EHIP; }

}  // namespace

int launch_store_kernel(const StoreParams &p, int32_t type, int32_t cache_type,
                        hipStream_t stream) {
    const int64_t vecs = (int64_t)p.n * (2 * p.Hkv * p.D / 8);
    const int64_t most = 1 << 20, want = (vecs + kThreads - 1) / kThreads;
    const dim3 g((unsigned)(want < most ? want : most)), t(kThreads);
    const bool e4m3 = cache_type == SWITCHSD_E4M3;
    if (type == SWITCHSD_BF16 && !e4m3)
        hipLaunchKernelGGL((k_store<SWITCHSD_BF16, false>), g, t, 0, stream, p);
    else if (type == SWITCHSD_BF16)
        hipLaunchKernelGGL((k_store<SWITCHSD_BF16, true>), g, t, 0, stream, p);
    else if (!e4m3)
        hipLaunchKernelGGL((k_store<SWITCHSD_F16, false>), g, t, 0, stream, p);
    else
        hipLaunchKernelGGL((k_store<SWITCHSD_F16, true>), g, t, 0, stream, p);
    return launched();
}

namespace {

template <int TYPE, bool E4M3>
int launch_attend(const AttnParams &p, hipStream_t stream) {
    const dim3 g((unsigned)((int64_t)p.a.B * p.a.R * p.a.Hq)), t(64);
    if (p.a.D == 64)
        hipLaunchKernelGGL((k_attend<TYPE, E4M3, 64>), g, t, 0, stream, p);
    else if (p.a.D == 128)
        hipLaunchKernelGGL((k_attend<TYPE, E4M3, 128>), g, t, 0, stream, p);
    else
        hipLaunchKernelGGL((k_attend<TYPE, E4M3, 256>), g, t, 0, stream, p);
    return launched();
}

}  // namespace

int launch_attention_kernel(const AttnParams &p, int32_t type, int32_t cache_type,
                            hipStream_t stream) {
    const bool e4m3 = cache_type == SWITCHSD_E4M3;
    if (type == SWITCHSD_BF16)
        return e4m3 ? launch_attend<SWITCHSD_BF16, true>(p, stream)
                    : launch_attend<SWITCHSD_BF16, false>(p, stream);
    return e4m3 ? launch_attend<SWITCHSD_F16, true>(p, stream)
                : launch_attend<SWITCHSD_F16, false>(p, stream);
}

}  // namespace switchsd
