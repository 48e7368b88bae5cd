// switchsd_logits.hip -- gfx950 kernels for penalties, biases and grammar masks
// on the logits of the drafted rows (k_logits), written out or verified on the
// fly.
//
// A work-group takes one chunk of the vocabulary and a group of rows of one
// sequence.  It first makes a word per token of the chunk in LDS: how often the
// history holds it, whether the prompt does, whether a draft node does, and
// which bias entry names it.  Then it streams the chunk of each of its rows:
// 16-byte vectors whose words are all zero and whose tokens are all allowed pass
// as they are, the others are computed element by element.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include <stdint.h>

#include "switchsd_device.h"
#include "switchsd_internal.h"

namespace switchsd {

namespace {

// Word of a token: occurrences in the generated part of the context (at most
// SWITCHSD_MAX_HISTORY), in the prompt, as a drafted token, bias entry + 1.
constexpr uint32_t kCount = 0x1FFFFFu;
constexpr uint32_t kPrompt = 1u << 21;
constexpr uint32_t kDrafted = 1u << 22;
constexpr int kBiasShift = 23;
static_assert(SWITCHSD_MAX_HISTORY == kCount, "the count field");
static_assert(SWITCHSD_MAX_BIAS == (1 << (32 - kBiasShift)) - 1, "the bias field");

// Loads and stores of vectors at any element's address.
typedef u32x4 u32x4_a __attribute__((aligned(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_a __attribute__((aligned(2)));

__device__ __forceinline__ uint32_t order_key(float f) {
    uint32_t u = __float_as_uint(f);
    if (u == 0x80000000u)
        u = 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

template <int kType>
struct Elem;
template <>
struct Elem<SWITCHSD_BF16> {
    typedef uint16_t type;
    static constexpr int per = 8;  // elements of a 16-byte vector
    static __device__ __forceinline__ float get(uint16_t v) {
        return __uint_as_float((uint32_t)v << 16);
    }
    static __device__ __forceinline__ uint16_t put(float f) {
        return __builtin_bit_cast(uint16_t, (__bf16)f);
    }
};
template <>
struct Elem<SWITCHSD_F16> {
    typedef uint16_t type;
    static constexpr int per = 8;
    static __device__ __forceinline__ float get(uint16_t v) {
        return (float)__builtin_bit_cast(_Float16, v);
    }
    static __device__ __forceinline__ uint16_t put(float f) {
        return __builtin_bit_cast(uint16_t, (_Float16)f);
    }
};
template <>
struct Elem<SWITCHSD_F32> {
    typedef float type;
    static constexpr int per = 4;
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float f) { return f; }
};

// LDS of a work-group, carved from one array (sizes by R and the unroll).
struct Lds {
    uint32_t *word;           // [chunk elements]
    unsigned long long *key;  // [rows] row maxima (verify)
    float *bias;              // [n_bias]
    uint32_t *entry;          // [R] drafted tokens in the chunk: offset << 10 | node
    int32_t *par;             // [R]
    uint32_t *anc;            // [rows][aw] the nodes on each row's path
};

constexpr size_t kEpiBytesPerNode = 20;

__host__ __device__ inline size_t lds_bytes(int elems, int R, int rows, int n_bias, bool verify) {
    const size_t n = (size_t)elems * 4 + (size_t)rows * 8 + (size_t)n_bias * 4 + (size_t)R * 8 +
                     (size_t)rows * ((R + 31) / 32) * 4;
    const size_t epi = verify ? R * kEpiBytesPerNode : 0;
    return n > epi ? n : epi;
}

__device__ __forceinline__ Lds lds_carve(unsigned char *m, int elems, int R, int rows,
                                         int n_bias) {
    Lds l;
    l.word = (uint32_t *)m;
    l.key = (unsigned long long *)(l.word + elems);
    l.bias = (float *)(l.key + rows);
    l.entry = (uint32_t *)(l.bias + n_bias);
    l.par = (int32_t *)(l.entry + R);
    l.anc = (uint32_t *)(l.par + R);
    return l;
}

struct Penalty {
    float rho, freq, pres;
};

// One touched token's logit l with word w, at `off` of the chunk, in the row
// whose path is `anc`.
__device__ __forceinline__ float processed(float l, uint32_t w, uint32_t off, const Penalty &pe,
                                           const Lds &s, int entries, const uint32_t *anc) {
    uint32_t c = w & kCount;
    if (w & kDrafted)
        for (int e = 0; e < entries; ++e) {
            const uint32_t en = s.entry[e];
            if ((en >> 10) == off)
                c += (anc[(en & 1023u) >> 5] >> (en & 31u)) & 1u;
        }
    float y = l;
    if (c != 0u || (w & kPrompt))
        y = l > 0.0f ? l / pe.rho : l * pe.rho;
    if (c != 0u) {
        y = y - pe.freq * (float)c;
        y = y - pe.pres;
    }
    if (w >> kBiasShift)
        y = y + s.bias[(w >> kBiasShift) - 1u];
    return y;
}

// The accept rule over the row maxima of sequence b (Sec. 3.3, Parallel
// Verification), by the whole work-group: an edge holds iff the node's token
// is its valid parent's maximum; a node is accepted iff every edge up to the
// anchor holds; the deepest accepted node wins, ties to the lowest index.
__device__ void accept(const LogitsParams &p, int b, unsigned char *mem) {
    const int R = p.a.R, tid = threadIdx.x;
    const int64_t base = (int64_t)b * R;
    const int n = clampi(p.a.dn[b], 1, R);
    int32_t *am = (int32_t *)mem, *tok = am + R, *par = tok + R;
    uint32_t *st = (uint32_t *)(par + R);  // [2][R]
    __shared__ uint32_t s_best;
    unsigned long long *keys = p.keys + (int64_t)b * p.key_stride;
    for (int i = tid; i < R; i += kThreads) {
        int a = -1;
        if (i < n) {
            const unsigned long long k = ld_u64(&keys[i]);
            st_u64(&keys[i], 0ull);
            a = k ? (int32_t)(0xFFFFFFFFu - (uint32_t)k) : 0;
        }
        am[i] = a;
        tok[i] = p.a.dtok[base + i];
        par[i] = p.a.dpar ? p.a.dpar[base + i] : i - 1;
        if (p.amax)
            p.amax[base + i] = a;
    }
    if (tid == 0)
        s_best = 0u;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
        const int q = par[i];
        const bool valid = i >= 1 && q >= 0 && q < i;
        const bool ok = i == 0 || (valid && tok[i] == am[q]);
        st[i] = (ok ? kHolds : 0u) | ((i == 0 ? 0u : 1u) << 16) | (uint32_t)(valid ? q : 0);
    }
    __syncthreads();
    int cur = 0;
    for (bool open = true; open; cur ^= 1) {
        bool more = false;
        for (int i = tid; i < n; i += kThreads) {
            const uint32_t s1 = st[cur * R + i];
            const uint32_t nv = jump_compose(s1, st[cur * R + (int)(s1 & 0xFFFFu)]);
            st[(cur ^ 1) * R + i] = nv;
            more |= (nv & 0xFFFFu) != 0u;
        }
        open = __syncthreads_or(more);
    }
    for (int i = tid; i < n; i += kThreads) {
        const uint32_t s1 = st[cur * R + i];
        if (s1 & kHolds)
            atomicMax(&s_best, (((s1 >> 16) & 0x7FFFu) << 16) | (0xFFFFu - (uint32_t)i));
    }
    __syncthreads();
    const int best = (int)(0xFFFFu - (s_best & 0xFFFFu)), depth = (int)(s_best >> 16);
    for (int i = tid; i < R; i += kThreads)
        if (i > depth)
            p.out_tokens[base + i] = -1;
    if (tid == 0) {
        int node = best;
        for (int pos = depth - 1; pos >= 0; --pos) {
            p.out_tokens[base + pos] = tok[node];
            node = par[node];
        }
        p.out_tokens[base + depth] = am[best];
        p.accept_len[b] = depth;
        p.accept_node[b] = best;
        p.bonus[b] = am[best];
        st_u32(&p.tickets[(int64_t)b * kLineU32], 0u);
    }
}

template <int kIn, int kOut, int kU, bool kVerify>
__global__ __launch_bounds__(kThreads) void k_logits(LogitsParams p) {
    typedef Elem<kIn> In;
    typedef Elem<kOut> Out;
    constexpr int kPer = In::per;
    constexpr int kElems = kThreads * kU * kPer;  // tokens of a chunk
    extern __shared__ __align__(16) unsigned char mem[];
    __shared__ int s_entries, s_last;
    const int tid = threadIdx.x;
    const int chunk = blockIdx.x % p.chunks;
    const int gb = blockIdx.x / p.chunks;
    const int group = gb % p.groups, b = gb / p.groups;
    const int R = p.a.R, V = p.a.V;
    const int n = clampi(p.a.dn[b], 1, R);
    const int r0 = group * p.rows;
    if (r0 >= n)
        return;
    const int r1 = r0 + p.rows < n ? r0 + p.rows : n;
    const int e0 = chunk * kElems;  // first token of the chunk
    const Lds s = lds_carve(mem, kElems, R, p.rows, p.a.n_bias);
    const int aw = (R + 31) / 32;

    // ---- the words
    const bool touched = p.penal || p.a.n_bias > 0;
    if (touched) {
        for (int i = tid; i < kElems / 4; i += kThreads)
            ((u32x4 *)s.word)[i] = u32x4{0u, 0u, 0u, 0u};
        if (tid == 0)
            s_entries = 0;
    }
    if (kVerify && tid < p.rows)
        s.key[tid] = 0ull;
    __syncthreads();
    if (p.a.n_bias > 0) {
        // the last entry of a token holds; entries before counts, so that the
        // maximum is over entries alone
        for (int e = tid; e < p.a.n_bias; e += kThreads) {
            const int64_t at = (int64_t)b * p.a.n_bias + e;
            const uint32_t off = (uint32_t)p.a.bias_ids[at] - (uint32_t)e0;
            s.bias[e] = p.a.bias_vals[at];
            if (off < (uint32_t)kElems)
                atomicMax(&s.word[off], (uint32_t)(e + 1) << kBiasShift);
        }
        __syncthreads();
    }
    Penalty pe = {1.0f, 0.0f, 0.0f};
    if (p.penal) {
        const int L = clampi(p.a.lengths[b], 0, p.a.Lmax);
        const int P = p.a.prompt_lens ? clampi(p.a.prompt_lens[b], 0, L) : 0;
        const int32_t *x = p.a.tokens + (int64_t)b * p.a.Lmax;
        for (int i = tid; i < L; i += kThreads) {
            const uint32_t off = (uint32_t)x[i] - (uint32_t)e0;
            if (off < (uint32_t)kElems) {
                if (i < P)
                    atomicOr(&s.word[off], kPrompt);
                else
                    atomicAdd(&s.word[off], 1u);
            }
        }
        for (int i = tid; i < n; i += kThreads) {
            const int64_t at = (int64_t)b * R + i;
            s.par[i] = p.a.dpar ? p.a.dpar[at] : i - 1;
            const uint32_t off = (uint32_t)p.a.dtok[at] - (uint32_t)e0;
            if (i >= 1 && off < (uint32_t)kElems) {
                atomicOr(&s.word[off], kDrafted);
                s.entry[atomicAdd(&s_entries, 1)] = (off << 10) | (uint32_t)i;
            }
        }
        if (p.a.repetition)
            pe.rho = p.a.repetition[b];
        if (p.a.frequency)
            pe.freq = p.a.frequency[b];
        if (p.a.presence)
            pe.pres = p.a.presence[b];
        __syncthreads();
        if (s_entries > 0) {
            if (tid < r1 - r0) {
                uint32_t *a = s.anc + tid * aw;
                for (int w = 0; w < aw; ++w)
                    a[w] = 0u;
                for (int node = r0 + tid; node > 0;) {
                    a[node >> 5] |= 1u << (node & 31);
                    const int q = s.par[node];
                    if (q < 0 || q >= node)
                        break;
                    node = q;
                }
            }
            __syncthreads();
        }
    }
    const int entries = touched ? s_entries : 0;
    uint32_t hit = 0u;  // bit u: some token of this lane's vector u has a word
    if (touched)
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            uint32_t any = 0u;
#pragma unroll
            for (int q = 0; q < kPer / 4; ++q) {
                const u32x4 w = ((const u32x4 *)s.word)[(u * kThreads + tid) * (kPer / 4) + q];
                any |= w.x | w.y | w.z | w.w;
            }
            hit |= (any ? 1u : 0u) << u;
        }
    const bool masked = p.a.allowed && (!p.a.allowed_on || p.a.allowed_on[b] != 0);
    const int64_t mstride = (int64_t)((V + 31) / 32) * 4;

    // ---- the rows
    for (int r = r0; r < r1; ++r) {
        const int64_t row = (int64_t)b * R + r;
        const typename In::type *src = (const typename In::type *)p.a.logits + row * V;
        typename Out::type *dst = (typename Out::type *)p.out + row * V;
        const uint8_t *bits = (const uint8_t *)p.a.allowed + row * mstride;
        const uint32_t *anc = s.anc + (r - r0) * aw;
        float best = -__builtin_inff();
        uint32_t at = 0xFFFFFFFFu;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int vl = u * kThreads + tid;
            const int v0 = e0 + vl * kPer;
            if (v0 >= V)
                continue;
            const bool whole = v0 + kPer <= V;
            uint32_t ok = 0xFFu;
            if (masked)
                ok = (uint32_t)bits[v0 >> 3] >> (v0 & 7);
            constexpr uint32_t kAll = (1u << kPer) - 1u;
            const bool plain = !((hit >> u) & 1u) && (ok & kAll) == kAll;
            if (p.in_place && plain)
                continue;
            typename In::type x[kPer];
            if (whole) {
                *(u32x4 *)x = *(const u32x4_a *)(src + v0);
            } else {
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    x[j] = v0 + j < V ? src[v0 + j] : (typename In::type)0;
            }
            typename Out::type y[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const bool keep = (ok >> j) & 1u;
                const uint32_t w = touched && !plain ? s.word[vl * kPer + j] : 0u;
                float f = In::get(x[j]);
                if (w)
                    f = processed(f, w, (uint32_t)(vl * kPer + j), pe, s, entries, anc);
                y[j] = Out::put(keep ? f : -__builtin_inff());
                if constexpr (kIn == kOut)  // untouched values keep their bits (NaN payloads)
                    y[j] = w == 0u && keep ? x[j] : y[j];
            }
            if (kVerify) {
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const float f = Out::get(y[j]);
                    if (v0 + j < V && (f > best || (at == 0xFFFFFFFFu && f == f))) {
                        best = f;
                        at = (uint32_t)(v0 + j);
                    }
                }
            } else if (whole) {
                if (kPer * sizeof(y[0]) == 16)
                    *(u32x4_a *)(dst + v0) = *(const u32x4 *)y;
                else
                    *(u32x2_a *)(dst + v0) = *(const u32x2 *)y;
            } else {
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (v0 + j < V)
                        dst[v0 + j] = y[j];
            }
        }
        if (kVerify) {
            unsigned long long key =
                at == 0xFFFFFFFFu
                    ? 0ull
                    : ((unsigned long long)order_key(best) << 32) | (0xFFFFFFFFu - at);
#pragma unroll
            for (int o = 32; o; o >>= 1) {
                const unsigned long long k2 = __shfl_xor(key, o);
                key = k2 > key ? k2 : key;
            }
            if ((tid & 63) == 0 && key)
                atomicMax(&s.key[r - r0], key);
        }
    }
    if (!kVerify)
        return;
    __syncthreads();
    if (tid < 64) {
        // one row per lane (at most kRowGroup = 64 rows)
        const unsigned long long key = tid < r1 - r0 ? s.key[tid] : 0ull;
        if (key)
            __hip_atomic_fetch_max(&p.keys[(int64_t)b * p.key_stride + r0 + tid], key,
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const bool last = arrive(&p.tickets[(int64_t)b * kLineU32],
                                 (uint32_t)(p.chunks * ((n + p.rows - 1) / p.rows)));
        if (tid == 0)
            s_last = last;
    }
    __syncthreads();
    if (s_last)
        accept(p, b, mem);
}

template <int kIn, int kOut, int kU, bool kVerify>
int launch(const LogitsParams &p, hipStream_t stream) {
    const int elems = kThreads * kU * Elem<kIn>::per;
    const unsigned grid = (unsigned)((int64_t)p.a.B * p.groups * p.chunks);
    const size_t lds = lds_bytes(elems, p.a.R, p.rows, p.a.n_bias, kVerify);
    hipLaunchKernelGGL((k_logits<kIn, kOut, kU, kVerify>), dim3(grid), dim3(kThreads), lds, stream,
                       p);
    return hipGetLastError() == hipSuccess ? SWITCHSD_OK : SWITCHSD_EHIP;
}

template <int kIn, int kOut, bool kVerify>
int launch_unroll(const LogitsParams &p, hipStream_t stream) {
    if (kIn == SWITCHSD_F32 && p.unroll == 8)
        return launch<kIn, kOut, kIn == SWITCHSD_F32 ? 8 : 4, kVerify>(p, stream);
    if (p.unroll == 4)
        return launch<kIn, kOut, 4, kVerify>(p, stream);
    if (p.unroll == 2)
        return launch<kIn, kOut, 2, kVerify>(p, stream);
    return launch<kIn, kOut, 1, kVerify>(p, stream);
}

}  // namespace

int launch_logits_kernel(const LogitsParams &p, int32_t out_type, hipStream_t stream) {
    constexpr int BF = SWITCHSD_BF16, HF = SWITCHSD_F16, FF = SWITCHSD_F32;
    const int in = p.a.logits_type;
    if (!p.out)  // verify
        return in == BF   ? launch_unroll<BF, BF, true>(p, stream)
               : in == HF ? launch_unroll<HF, BF, true>(p, stream)
                          : launch_unroll<FF, BF, true>(p, stream);
    if (in == BF)
        return launch_unroll<BF, BF, false>(p, stream);
    if (in == HF)
        return out_type == BF ? launch_unroll<HF, BF, false>(p, stream)
                              : launch_unroll<HF, HF, false>(p, stream);
    return out_type == BF ? launch_unroll<FF, BF, false>(p, stream)
                          : launch_unroll<FF, FF, false>(p, stream);
}

}  // namespace switchsd
