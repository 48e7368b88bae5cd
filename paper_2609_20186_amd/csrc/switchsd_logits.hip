// switchsd_logits.hip -- gfx950 kernels for penalties, biases and grammar masks
// on the logits of the drafted rows (k_logits), written out or verified on the
// fly.
//
// A work-group takes one chunk of the vocabulary and a group of rows of one
// sequence.  It first makes a word per token of the chunk in LDS (how often the
// history holds it, whether the prompt does, its first draft node, the bias
// entry that names it) and lists the tokens that have one.  Then it streams the
// chunk of each of its rows, two rows ahead: 16-byte vectors that hold a listed
// token pass through LDS, where the list's tokens are computed one per lane.
// All others pass as they are, so the work per row is the row's bytes plus the
// listed tokens, however they lie.
//
// A chunk is every chunks-th block of 64 vectors: low token ids, which are the
// frequent ones, spread over all work-groups of a row.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include <stdint.h>

#include "switchsd_device.h"
#include "switchsd_internal.h"

namespace switchsd {

namespace {

constexpr int kWaves = kThreads / 64;

// Word of a token: occurrences in the generated part of the context (at most
// SWITCHSD_MAX_HISTORY), in the prompt, drafted (then the low bits are its first
// entry in the draft's table and the count is there), bias entry + 1.
constexpr uint32_t kCount = 0x1FFFFFu;
constexpr uint32_t kPrompt = 1u << 21;
constexpr uint32_t kDrafted = 1u << 22;
constexpr int kBiasShift = 23;
static_assert(SWITCHSD_MAX_HISTORY == kCount, "the count field");
static_assert(SWITCHSD_MAX_BIAS == (1 << (32 - kBiasShift)) - 1, "the bias field");
constexpr int kNodeBits = 10;
static_assert(SWITCHSD_MAX_R == 1 << kNodeBits, "the node field");
constexpr uint32_t kNone = 0xFFFFu;

// Loads and stores of vectors at any element's address.
typedef u32x4 u32x4_a __attribute__((aligned(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_a __attribute__((aligned(2)));

// Order-preserving 16-bit key of a bf16 pattern; -0 is folded onto +0, 0: NaN.
__device__ __forceinline__ uint32_t order16(uint32_t x) {
    if ((x & 0x7FFFu) > 0x7F80u)
        return 0u;
    if (x == 0x8000u)
        x = 0u;
    return (x & 0x8000u) ? x ^ 0xFFFFu : x | 0x8000u;
}

// The key of switchsd_verify_accept's row maxima: order key of the float.
__device__ __forceinline__ uint32_t order32(uint32_t key16) {
    return (key16 << 16) | ((key16 & 0x8000u) ? 0u : 0xFFFFu);
}

typedef int16_t s16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pk_max_i16(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t,
                              __builtin_elementwise_max(__builtin_bit_cast(s16x2, a),
                                                        __builtin_bit_cast(s16x2, b)));
}
__device__ __forceinline__ uint32_t pk_min_u16(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t,
                              __builtin_elementwise_min(__builtin_bit_cast(u16x2, a),
                                                        __builtin_bit_cast(u16x2, b)));
}

// Maximum over the wave, in every lane: row shifts, then two row broadcasts.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#define SWITCHSD_STEP(ctrl, mask)                                                               \
    {                                                                                           \
        const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, mask, 0xf,    \
                                                                 false);                        \
        v = o > v ? o : v;                                                                      \
    }
    SWITCHSD_STEP(0x111, 0xf)
    SWITCHSD_STEP(0x112, 0xf)
    SWITCHSD_STEP(0x114, 0xf)
    SWITCHSD_STEP(0x118, 0xf)
    SWITCHSD_STEP(0x142, 0xa)
    SWITCHSD_STEP(0x143, 0xc)
#undef SWITCHSD_STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
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

// LDS of a work-group, carved from one array.
struct Lds {
    uint32_t *word;   // [tokens]
    void *stage;      // [tokens] of the input's type: vectors with listed tokens
    uint16_t *list;   // [tokens] the tokens that have a word
    uint32_t *key;    // [rows][kWaves] row maxima (verify)
    float *bias;      // [n_bias]
    uint32_t *entry;  // [R] drafted tokens of the chunk: token << kNodeBits | node
    uint32_t *count;  // [R] count and prompt bit of a drafted token, at its first entry
    uint32_t *anc;    // [rows][aw] the nodes on each row's path
    uint16_t *next;   // [R] the next entry of the same token
    int16_t *par;     // [R]
};

constexpr size_t kEpiBytesPerNode = 20;

__host__ __device__ inline size_t lds_bytes(int tokens, int size, int R, int rows, int n_bias,
                                            bool verify) {
    const size_t n = (size_t)tokens * (4 + size + 2) + (size_t)rows * kWaves * 4 +
                     (size_t)n_bias * 4 + (size_t)R * 12 + (size_t)rows * ((R + 31) / 32) * 4;
    const size_t epi = verify ? R * kEpiBytesPerNode : 0;
    return n > epi ? n : epi;
}

__device__ __forceinline__ Lds lds_carve(unsigned char *m, int tokens, int size, int R, int rows,
                                         int n_bias) {
    Lds l;
    l.word = (uint32_t *)m;
    l.stage = l.word + tokens;
    l.list = (uint16_t *)((unsigned char *)l.stage + tokens * size);
    l.key = (uint32_t *)(l.list + tokens);
    l.bias = (float *)(l.key + rows * kWaves);
    l.entry = (uint32_t *)(l.bias + n_bias);
    l.count = l.entry + R;
    l.anc = l.count + R;
    l.next = (uint16_t *)(l.anc + rows * ((R + 31) / 32));
    l.par = (int16_t *)(l.next + R);
    return l;
}

struct Penalty {
    float rho, freq, pres;
};

// A listed token's logit l with word w in the row whose path is `anc`.
__device__ __forceinline__ float processed(float l, uint32_t w, const Penalty &pe, const Lds &s,
                                           const uint32_t *anc) {
    uint32_t c = w;
    if (w & kDrafted) {
        uint32_t e = w & ((1u << kNodeBits) - 1u);
        c = s.count[e];
        do {
            const uint32_t node = s.entry[e] & ((1u << kNodeBits) - 1u);
            c += (anc[node >> 5] >> (node & 31u)) & 1u;
            e = s.next[e];
        } while (e != kNone);
    }
    const bool prompt = c & kPrompt;
    c &= kCount;
    float y = l;
    if (c != 0u || prompt)
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

// A 16-byte vector of 16-bit pairs with the halves of clear bits of `ok` (two
// bits per word) replaced by `fill` (the same 16 bits twice).
__device__ __forceinline__ uint32_t keep16(uint32_t x, uint32_t ok, int q, uint32_t fill) {
    const uint32_t lo = (uint32_t)((int32_t)(ok << (31 - 2 * q)) >> 31);
    const uint32_t hi = (uint32_t)((int32_t)(ok << (30 - 2 * q)) >> 31);
    const uint32_t m = (lo & 0xFFFFu) | (hi << 16);
    return (x & m) | (fill & ~m);
}

// One lane's part of a row: kU vectors and the allowed bits of their tokens.
template <int kU>
struct RowRegs {
    u32x4 x[kU];
    uint32_t ok[kU];
};

// kTiny: V below one vector's tokens (read one by one).
template <int kIn, int kOut, int kU, bool kVerify, bool kTiny>
__global__ __launch_bounds__(kThreads) void k_logits(LogitsParams p) {
    typedef Elem<kIn> In;
    typedef Elem<kOut> Out;
    constexpr int kPer = In::per;
    constexpr int kBits = 128 / kPer;                  // of an element
    constexpr int kBlk = 64 * kPer;                    // tokens of a block
    constexpr int kBlkLog = kPer == 8 ? 9 : 8;
    constexpr int kTokens = kWaves * kU * kBlk;        // of a chunk
    constexpr uint32_t kAll = (1u << kPer) - 1u;
    extern __shared__ __align__(16) unsigned char mem[];
    __shared__ int s_entries, s_last, s_sum[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t cmask = (uint32_t)p.chunks - 1u;
    const uint32_t chunk = blockIdx.x & cmask;
    const int gb = blockIdx.x >> p.chunk_log;
    const int group = gb % p.groups, b = gb / p.groups;
    const int R = p.a.R, V = p.a.V;
    const int n = clampi(p.a.dn[b], 1, R);
    const int r0 = group * p.rows;
    if (r0 >= n)
        return;
    const int r1 = r0 + p.rows < n ? r0 + p.rows : n;
    const int aw = (R + 31) / 32;
    const Lds s = lds_carve(mem, kTokens, sizeof(typename In::type), R, p.rows, p.a.n_bias);
    const bool masked = p.a.allowed && (!p.a.allowed_on || p.a.allowed_on[b] != 0);
    const int64_t mstride = (int64_t)((V + 31) / 32) * 4;

    // ---- this lane's vectors: first token, how many of its tokens exist, and
    // where it is read (the row's last whole vector where fewer exist)
    int v0[kU], at[kU];
    uint32_t own[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        const uint32_t blk = ((uint32_t)(u * kWaves + wave) << p.chunk_log) | chunk;
        v0[u] = (int)(blk * kBlk) + lane * kPer;
        const int left = V - v0[u];
        own[u] = left >= kPer ? kAll : left > 0 ? (1u << left) - 1u : 0u;
        at[u] = v0[u] < V - kPer ? v0[u] : V - kPer;
    }
    const int tail = V % kPer;  // tokens of the row's last, partial vector

    auto load_row = [&](RowRegs<kU> &g, int r) {
        const int64_t row = (int64_t)b * R + r;
        const typename In::type *src = (const typename In::type *)p.a.logits + row * V;
        const uint8_t *bits = (const uint8_t *)p.a.allowed + row * mstride;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            if constexpr (kTiny) {
                union {
                    typename In::type e[kPer];
                    u32x4 v;
                } t;
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    t.e[j] = src[v0[u] + j < V ? v0[u] + j : 0];
                g.x[u] = t.v;
            } else {
                g.x[u] = __builtin_nontemporal_load((const u32x4_a *)(src + at[u]));
            }
            g.ok[u] = kAll;
            if (masked)
                g.ok[u] = (uint32_t)bits[(v0[u] < V ? v0[u] : 0) >> 3] >> (v0[u] & 7);
        }
    };
    // in place without a mask, only the listed tokens are read and written
    const bool sparse = !kVerify && p.in_place && !masked;
    RowRegs<kU> ra, rb;
    if (!sparse) {
        load_row(ra, r0);
        if (r0 + 1 < r1)
            load_row(rb, r0 + 1);
    }

    // ---- the words
    const bool touched = p.penal || p.a.n_bias > 0;
    Penalty pe = {1.0f, 0.0f, 0.0f};
    uint32_t hit = 0u;  // bit u * kPer + j: token j of vector u is listed
    int T = 0;          // listed tokens
    if (kVerify)
        for (int i = tid; i < p.rows * kWaves; i += kThreads)
            s.key[i] = 0u;
    if (touched) {
        // a token's place in the chunk, or none
        auto place = [&](int32_t t, uint32_t &off) {
            const uint32_t blk = (uint32_t)t >> kBlkLog;
            off = ((blk >> p.chunk_log) << kBlkLog) | ((uint32_t)t & (kBlk - 1u));
            return (uint32_t)t < (uint32_t)V && (blk & cmask) == chunk;
        };
        for (int i = tid; i < kTokens / 4; i += kThreads)
            ((u32x4 *)s.word)[i] = u32x4{0u, 0u, 0u, 0u};
        if (tid == 0)
            s_entries = 0;
        __syncthreads();
        if (p.a.n_bias > 0) {
            // the last entry of a token holds; entries before counts, so that
            // the maximum is over entries alone
            for (int e = tid; e < p.a.n_bias; e += kThreads) {
                const int64_t i = (int64_t)b * p.a.n_bias + e;
                uint32_t off;
                s.bias[e] = p.a.bias_vals[i];
                if (place(p.a.bias_ids[i], off))
                    atomicMax(&s.word[off], (uint32_t)(e + 1) << kBiasShift);
            }
            __syncthreads();
        }
        if (p.penal) {
            const int L = clampi(p.a.lengths[b], 0, p.a.Lmax);
            const int P = p.a.prompt_lens ? clampi(p.a.prompt_lens[b], 0, L) : 0;
            const int32_t *x = p.a.tokens + (int64_t)b * p.a.Lmax;
            for (int i0 = tid; i0 < L; i0 += 8 * kThreads) {
                int32_t t[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int i = i0 + q * kThreads;
                    t[q] = x[i < L ? i : L - 1];
                }
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int i = i0 + q * kThreads;
                    uint32_t off;
                    if (i < L && place(t[q], off)) {
                        if (i < P)
                            atomicOr(&s.word[off], kPrompt);
                        else
                            atomicAdd(&s.word[off], 1u);
                    }
                }
            }
            for (int i = tid; i < n; i += kThreads) {
                const int64_t d = (int64_t)b * R + i;
                uint32_t off;
                s.par[i] = (int16_t)clampi(p.a.dpar ? p.a.dpar[d] : i - 1, -1, R);
                if (i >= 1 && place(p.a.dtok[d], off)) {
                    atomicOr(&s.word[off], kDrafted);
                    s.entry[atomicAdd(&s_entries, 1)] = (off << kNodeBits) | (uint32_t)i;
                }
            }
            if (p.a.repetition)
                pe.rho = p.a.repetition[b];
            if (p.a.frequency)
                pe.freq = p.a.frequency[b];
            if (p.a.presence)
                pe.pres = p.a.presence[b];
            __syncthreads();
        }
        // the list, in token order
#pragma unroll
        for (int u = 0; u < kU; ++u)
#pragma unroll
            for (int q = 0; q < kPer / 4; ++q) {
                const u32x4 w = ((const u32x4 *)s.word)[(u * kThreads + tid) * (kPer / 4) + q];
                hit |= ((w.x ? 1u : 0u) | (w.y ? 2u : 0u) | (w.z ? 4u : 0u) | (w.w ? 8u : 0u))
                       << (u * kPer + q * 4);
            }
        const int mine = __popc(hit);
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int q = __shfl_up(upto, o);
            upto += lane >= o ? q : 0;
        }
        if (lane == 63)
            s_sum[wave] = upto;
        __syncthreads();
        int k = upto - mine;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            k += w < wave ? s_sum[w] : 0;
            T += s_sum[w];
        }
        for (uint32_t h = hit; h; h &= h - 1u) {
            const int j = __ffs(h) - 1;
            s.list[k++] = (uint16_t)(((j / kPer) * kThreads + tid) * kPer + j % kPer);
        }
        const int entries = s_entries;
        if (entries > 0) {
            // the entries of one token chained, its count moved to the first
            for (int e = tid; e < entries; e += kThreads) {
                const uint32_t off = s.entry[e] >> kNodeBits;
                uint32_t nx = kNone;
                bool first = true;
                for (int f = 0; f < entries; ++f)
                    if ((s.entry[f] >> kNodeBits) == off) {
                        if (f > e && nx == kNone)
                            nx = (uint32_t)f;
                        first = first && f >= e;
                    }
                s.next[e] = (uint16_t)nx;
                if (first) {
                    const uint32_t w = s.word[off];
                    s.count[e] = w & (kCount | kPrompt);
                    s.word[off] = (w & ~(kCount | kPrompt)) | (uint32_t)e;
                }
            }
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
        }
    }
    __syncthreads();

    if (sparse) {
        if constexpr (!kVerify && kIn == kOut) {
            for (int r = r0; r < r1; ++r) {
                typename Out::type *dst =
                    (typename Out::type *)p.out + ((int64_t)b * R + r) * V;
                for (int k = tid; k < T; k += kThreads) {
                    const uint32_t off = s.list[k];
                    const uint32_t blk = ((off >> kBlkLog) << p.chunk_log) | chunk;
                    typename Out::type *d = dst + (blk * kBlk + (off & (kBlk - 1u)));
                    *d = Out::put(processed(In::get(*d), s.word[off], pe, s,
                                            s.anc + (r - r0) * aw));
                }
            }
        }
        return;
    }

    // ---- the rows
    typename In::type *stage = (typename In::type *)s.stage;
    for (int r = r0; r < r1; ++r) {
        RowRegs<kU> rc;
        if (r + 2 < r1)
            load_row(rc, r + 2);
        typename Out::type *dst = (typename Out::type *)p.out + ((int64_t)b * R + r) * V;
        const uint32_t *anc = s.anc + (r - r0) * aw;
        if constexpr (!kTiny) {
            // the row's last, partial vector was read whole: its own tokens first
#pragma unroll
            for (int u = 0; u < kU; ++u)
                if (own[u] != kAll && own[u] != 0u) {
                    const int sh = (kPer - tail) * kBits;
                    typedef unsigned __int128 u128;
                    ra.x[u] = __builtin_bit_cast(u32x4, __builtin_bit_cast(u128, ra.x[u]) >> sh);
                }
        }
        if (T > 0) {
#pragma unroll
            for (int u = 0; u < kU; ++u)
                if ((hit >> (u * kPer)) & kAll)
                    ((u32x4 *)stage)[u * kThreads + tid] = ra.x[u];
            __syncthreads();
            for (int k = tid; k < T; k += kThreads) {
                const uint32_t off = s.list[k];
                const float y = processed(In::get(stage[off]), s.word[off], pe, s, anc);
                if constexpr (sizeof(typename In::type) == 4)
                    stage[off] = y;
                else
                    stage[off] = Out::put(y);
            }
            __syncthreads();
        }
        uint32_t best = 0u;         // order key of this lane's maximum, 0: none
        uint32_t pk[kU][kPer / 2];  // 16-bit results, in pairs
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const uint32_t hu = (hit >> (u * kPer)) & kAll;
            u32x4 x = ra.x[u];
            u32x4 y = x;
            if (hu)
                y = ((const u32x4 *)stage)[u * kThreads + tid];
            uint32_t ok = ra.ok[u] & kAll;
            if constexpr (kOut == SWITCHSD_F32) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    y[j] = (ok >> j) & 1u ? y[j] : 0xFF800000u;
            } else {
                constexpr uint32_t kInf = kOut == SWITCHSD_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
#pragma unroll
                for (int q = 0; q < kPer / 2; ++q) {
                    uint32_t v;
                    if constexpr (kIn == kOut) {
                        v = y[q];
                    } else if constexpr (kIn == SWITCHSD_F32) {
                        v = (uint32_t)Out::put(__uint_as_float(y[2 * q])) |
                            (uint32_t)Out::put(__uint_as_float(y[2 * q + 1])) << 16;
                    } else {
                        v = (uint32_t)Out::put(In::get((uint16_t)x[q])) |
                            (uint32_t)Out::put(In::get((uint16_t)(x[q] >> 16))) << 16;
                        if (hu)  // listed tokens already have the output's type
                            v = keep16(v, ~hu, q, 0u) | keep16(y[q], hu, q, 0u);
                    }
                    if (ok != kAll)
                        v = keep16(v, ok, q, kInf);
                    pk[u][q] = v;
                }
            }
            if constexpr (!kVerify) {
                const bool write = !p.in_place || hu || ok != kAll;
                if (own[u] == kAll && write) {
                    if constexpr (kOut == SWITCHSD_F32)
                        *(u32x4_a *)(dst + v0[u]) = y;
                    else if constexpr (kPer == 8)
                        *(u32x4_a *)(dst + v0[u]) =
                            u32x4{pk[u][0], pk[u][1], pk[u][2], pk[u][3]};
                    else
                        *(u32x2_a *)(dst + v0[u]) = u32x2{pk[u][0], pk[u][1]};
                } else if (own[u] != 0u && write) {
#pragma unroll
                    for (int j = 0; j < kPer; ++j)
                        if ((own[u] >> j) & 1u) {
                            if constexpr (kOut == SWITCHSD_F32)
                                dst[v0[u] + j] = __uint_as_float(y[j]);
                            else
                                dst[v0[u] + j] = (uint16_t)(pk[u][j / 2] >> (16 * (j & 1)));
                        }
                }
            } else {
#pragma unroll
                for (int q = 0; q < kPer / 2; ++q)  // tokens that do not exist: NaN, negative
                    if (own[u] != kAll)
                        pk[u][q] = keep16(pk[u][q], own[u], q, 0xFFFFFFFFu);
            }
        }
        if constexpr (kVerify) {
            // Maximum of the lane's bf16 patterns: as signed integers where it
            // is not negative, as unsigned ones (the smallest) where all are
            // negative; a positive NaN takes the slow way.
            uint32_t m = pk[0][0], lo = pk[0][0];
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int q = 0; q < kPer / 2; ++q) {
                    m = pk_max_i16(m, pk[u][q]);
                    lo = pk_min_u16(lo, pk[u][q]);
                }
            const int32_t m0 = (int16_t)m, m1 = (int16_t)(m >> 16);
            const int32_t mx = m0 > m1 ? m0 : m1;
            if (mx > 0x7F80) {
#pragma unroll
                for (int u = 0; u < kU; ++u)
#pragma unroll
                    for (int q = 0; q < kPer / 2; ++q) {
                        const uint32_t k0 = order16(pk[u][q] & 0xFFFFu),
                                       k1 = order16(pk[u][q] >> 16);
                        const uint32_t k = k0 > k1 ? k0 : k1;
                        best = k > best ? k : best;
                    }
            } else if (mx >= 0) {
                best = (uint32_t)mx | 0x8000u;
            } else {
                const uint32_t l0 = lo & 0xFFFFu, l1 = lo >> 16;
                best = order16(l0 < l1 ? l0 : l1);
            }
            const uint32_t top = wave_max(best);
            if (top != 0u) {
                // the lowest token that holds it
                uint32_t first = kNone;
                if (best == top) {
#pragma unroll
                    for (int u = kU - 1; u >= 0; --u)
#pragma unroll
                        for (int q = kPer / 2 - 1; q >= 0; --q) {
                            const uint32_t o = (uint32_t)((u * kThreads + tid) * kPer + 2 * q);
                            if (order16(pk[u][q] >> 16) == top)
                                first = o + 1u;
                            if (order16(pk[u][q] & 0xFFFFu) == top)
                                first = o;
                        }
                }
                const uint32_t low = kNone - wave_max(kNone - first);
                if (lane == 0)
                    s.key[(r - r0) * kWaves + wave] = (top << 16) | (kNone - low);
            }
        }
        ra = rb;
        rb = rc;
    }
    if constexpr (kVerify) {
        __syncthreads();
        if (tid < 64) {
            // one row per lane (at most kRowGroup = 64 rows)
            uint32_t k = 0u;
            if (tid < r1 - r0)
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const uint32_t o = s.key[tid * kWaves + w];
                    k = o > k ? o : k;
                }
            if (k) {
                const uint32_t off = kNone - (k & 0xFFFFu);
                const uint32_t blk = ((off >> kBlkLog) << p.chunk_log) | chunk;
                const uint32_t t = blk * kBlk + (off & (kBlk - 1u));
                __hip_atomic_fetch_max(
                    &p.keys[(int64_t)b * p.key_stride + r0 + tid],
                    ((unsigned long long)order32(k >> 16) << 32) | (0xFFFFFFFFu - t),
                    __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            const bool last = arrive(&p.tickets[(int64_t)b * kLineU32],
                                     (uint32_t)(p.chunks * ((n + p.rows - 1) / p.rows)));
            if (tid == 0)
                s_last = last;
        }
        __syncthreads();
        if (s_last)
            accept(p, b, mem);
    }
}

template <int kIn, int kOut, int kU, bool kVerify, bool kTiny>
int launch(const LogitsParams &p, hipStream_t stream) {
    const int tokens = kThreads * kU * Elem<kIn>::per;
    const unsigned grid = (unsigned)((int64_t)p.a.B * p.groups * p.chunks);
    const size_t lds = lds_bytes(tokens, sizeof(typename Elem<kIn>::type), p.a.R, p.rows,
                                 p.a.n_bias, kVerify);
    hipLaunchKernelGGL((k_logits<kIn, kOut, kU, kVerify, kTiny>), dim3(grid), dim3(kThreads), lds,
                       stream, p);
    return hipGetLastError() == hipSuccess ? SWITCHSD_OK : SWITCHSD_EHIP;
}

template <int kIn, int kOut, bool kVerify>
int launch_unroll(const LogitsParams &p, hipStream_t stream) {
    if (p.a.V < Elem<kIn>::per)
        return launch<kIn, kOut, 1, kVerify, true>(p, stream);
    if (p.unroll == 4)
        return launch<kIn, kOut, 4, kVerify, false>(p, stream);
    if (p.unroll == 2)
        return launch<kIn, kOut, 2, kVerify, false>(p, stream);
    return launch<kIn, kOut, 1, kVerify, false>(p, stream);
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
