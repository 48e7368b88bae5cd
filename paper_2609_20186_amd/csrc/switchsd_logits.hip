// switchsd_logits.hip -- gfx950 kernels for penalties, biases and grammar masks
// on the logits of the drafted rows: written out (k_process) or verified on the
// fly (k_verify).
//
// For token v in row r, with c its occurrences behind the prompt and on the
// row's path, and s whether the history holds it at all:
//   y = s ? (l > 0 ? l / rho : l * rho) : l;  c > 0: y -= f * c, y -= p;
//   y += bias_v;  not allowed: y = -inf.
// Few tokens of a row are touched by any of it but the mask, so the work is one
// pass over the rows' bytes (the bound: HBM) plus a few tokens.
//
// A work-group takes one chunk of the vocabulary and a group of rows of one
// sequence.  It first makes a word per token of the chunk in LDS (how often the
// history holds it, whether the prompt does, the draft node that stands for
// it, the bias entry that names it) and lists the tokens that have one
// (list_tokens); what a drafted token adds on each row's path is counted into a
// table once.  Counting anew in every work-group keeps the call to one launch
// and no scratch memory: 32 histories of 4096 tokens cost the verification of
// 32 x 8 rows of 128256 6.4 us (25.0 instead of 18.6), writing them 3.7 (26.4
// instead of 22.7); 300 biases alone 1.3 and 0.8.
//   k_process: vectors that hold a listed token pass through LDS, where the
//     listed tokens are computed one per lane; all others pass as they are.
//   k_verify: the rows' maxima are taken over the vectors without their listed
//     tokens, which are computed one per lane beside them; nothing is exchanged
//     between the waves until the rows are done.
// Computing the listed tokens where their vectors lie, in the lanes that hold
// them, measured 109 instead of 32 us for 32 x 8 rows of 128256 and 17 ms
// instead of 0.6 for 32 x 201 drafted rows.
//
// A chunk is every 2^k-th block of 16 vectors (k_process: 32): low token ids,
// which are the frequent ones, spread over all work-groups of a row.  Blocks of
// 16, 32, 64 vectors measured 25.5, 28.0, 30.8 us (verify, 32 x 8 rows of
// 128256) and 301, 269, 303 us (process, 32 x 60 rows of floats).
//
// Measured (MI355X), bytes that must move over time: process 32 x 8 rows of
// 128256 bf16 26.9 us, 4.9 TB/s (a large copy reaches 5.1 to 5.2 TB/s); 32 x 60
// rows of floats to bf16 under a grammar 266 us, 5.6 TB/s (a large conversion
// of floats to bf16: 5.85); verify 32 x 8 rows 25.2 us, 2.6 TB/s; 32 x 201
// candidate rows under a grammar 206 us, 4.6 TB/s; one row of 32000 written 5.2
// us, verified 9.7.  What bounds the small ones is the chain before the first
// row (draft length, history, list) and after the last (row maxima, ticket,
// accept rule).  Vocabularies that fill the chunks worse are slower (see where
// the grid is set).
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include <stdint.h>

#include "switchsd_device.h"
#include "switchsd_internal.h"

namespace switchsd {

namespace {

constexpr int kWaves = kThreads / 64;

// Word of a token: occurrences in the generated part of the context (at most
// SWITCHSD_MAX_HISTORY), in the prompt, drafted (then the low bits are the draft
// node that stands for it and the count is kept there), bias entry + 1.
constexpr uint32_t kCount = 0x1FFFFFu;
constexpr uint32_t kPrompt = 1u << 21;
constexpr uint32_t kDrafted = 1u << 22;
constexpr int kBiasShift = 23;
static_assert(SWITCHSD_MAX_HISTORY == kCount, "the count field");
static_assert(SWITCHSD_MAX_BIAS == (1 << (32 - kBiasShift)) - 1, "the bias field");
static_assert(SWITCHSD_MAX_R <= kCount, "a node in the count field");
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
    uint32_t *word;   // [tokens], then a word of each lane's
    void *stage;      // process: [tokens] of the input's type, vectors with listed tokens;
                      // verify: [rows][split][2] the vectors with the maximum
    void *list;       // process: [tokens] uint16, the tokens that have a word; verify: the
                      // first kListed of them, uint32, << 16 the place in `held`
    uint32_t *lword;  // verify: [kListed] their words
    // in place of the words, unless more tokens have one than the list holds:
    u32x4 *gone;      // verify: [vectors] all bits set where a token is listed or does not
                      // exist
    u32x4 *held;      // verify: [kWaves][kSlots] the row's vectors with listed tokens
    uint32_t *bits;   // verify: [kWaves][tokens / 32] the row's allowed bits
    uint8_t *slot;    // verify: [vectors] a vector's slot in `held` (kNoSlot: none)
    uint8_t *inner;   // verify: [vectors] the tokens that exist and are not listed
    uint32_t *key;    // verify: [2][rows][split] maxima over vectors, over listed tokens
    float *bias;      // [n_bias]
    uint32_t *count;  // [R] count and prompt bit of a drafted token, at its node
    uint32_t *node;   // [R] parent, and << 16 the node that stands for the token (kNone:
                      // not of this chunk)
    uint8_t *path;    // [rows][R] occurrences of a drafted token on a row's path, one
                      // byte each, two for R > 256
};

constexpr size_t kEpiBytesPerNode = 20;

// Listed tokens that k_verify keeps a list of (the rest are found by their
// words), and vectors with listed tokens that a wave keeps in LDS (the tokens
// of the rest are read again).
constexpr int kListed = 512;
constexpr int kSlots = 128;
constexpr uint32_t kNoSlot = 0xFFu;

__host__ __device__ inline size_t path_bytes(int rows, int R) {
    return ((size_t)rows * R * (R > 256 ? 2 : 1) + 3) / 4 * 4;
}

// Places of the parts, and the bytes of all.  split: waves that share a row
// (0: k_process).
__host__ __device__ __forceinline__ size_t lds_carve(unsigned char *m, int tokens, int size,
                                                     int R, int rows, int n_bias, int split,
                                                     Lds &l) {
    unsigned char *const m0 = m;
    auto take = [&](size_t n) {
        unsigned char *q = m;
        m += (n + 15) / 16 * 16;
        return q;
    };
    const size_t gone = split == 1 ? (size_t)tokens * size : 0;
    const size_t held = split == 1 ? (size_t)kWaves * kSlots * 16 : 0;
    const size_t words = (size_t)(tokens + 64) * 4;
    unsigned char *w = take(words > gone + held ? words : gone + held);
    l.word = (uint32_t *)w;
    l.gone = (u32x4 *)w;
    l.held = (u32x4 *)(w + gone);
    l.stage = take(split ? (size_t)rows * split * 32 : (size_t)tokens * size);
    l.list = take(split ? kListed * 4 : tokens * 2);
    l.lword = (uint32_t *)take(split ? kListed * 4 : 0);
    l.bits = (uint32_t *)take(split ? kWaves * tokens / 8 : 0);
    l.slot = take(split == 1 ? tokens * size / 16 : 0);
    l.inner = take(split == 1 ? tokens * size / 16 : 0);
    l.key = (uint32_t *)take((size_t)rows * split * 8);
    l.bias = (float *)take((size_t)n_bias * 4);
    l.count = (uint32_t *)take((size_t)R * 4);
    l.node = (uint32_t *)take((size_t)R * 4);
    l.path = take(path_bytes(rows, R));
    const size_t epi = split ? R * kEpiBytesPerNode : 0;
    return (size_t)(m - m0) > epi ? (size_t)(m - m0) : epi;
}

struct Penalty {
    float rho, freq, pres;
};

// A listed token's logit l with word w in the row whose path counts start at
// entry `row` of s.path.
__device__ __forceinline__ float processed(float l, uint32_t w, const Penalty &pe, const Lds &s,
                                           int row, bool wide) {
    uint32_t c = w & kCount;
    bool prompt = w & kPrompt;
    if (w & kDrafted) {
        const uint32_t at = s.count[c];
        c = (at & kCount) +
            (wide ? ((const uint16_t *)s.path)[row + c] : (uint32_t)s.path[row + c]);
        prompt = at & kPrompt;
    }
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

// LDS that only the wave itself uses: its operations are done in order, and
// this keeps the compiler to that order.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Row maxima of a sequence meet in the workspace: up to 64 rows in one of 16
// copies by chunk (atomics to one line follow each other), else in one.
constexpr int kCopies = 16;
__device__ __forceinline__ unsigned long long *row_keys(const LogitsParams &p, int b, int copy) {
    return p.a.R <= 64 ? p.skeys + (int64_t)b * p.skey_stride + copy * p.a.R
                       : p.keys + (int64_t)b * p.key_stride;
}

// The accept rule over the row maxima of sequence b with n nodes (Sec. 3.3,
// Parallel Verification), by wave 0: an edge holds iff the node's token is its
// valid parent's maximum; a node is accepted iff every edge up to the anchor
// holds; the deepest accepted node wins, ties to the lowest index.  tok0 and
// par0: token and parent of node `lane`.
__device__ __forceinline__ void accept(const LogitsParams &p, int b, int n, int tok0, int par0,
                                       unsigned char *mem) {
    const int R = p.a.R, lane = threadIdx.x;
    const int64_t base = (int64_t)b * R;
    int32_t *am = (int32_t *)mem, *tok = am + R, *par = tok + R;
    uint32_t *st = (uint32_t *)(par + R);  // [2][R]
    const int copies = p.chunks < kCopies ? p.chunks : kCopies;
    for (int i = lane; i < R; i += 64) {
        unsigned long long k = 0ull;
        if (i < n) {
            if (R > 64) {
                k = ld_u64(row_keys(p, b, 0) + i);
                st_u64(row_keys(p, b, 0) + i, 0ull);
            } else {
                unsigned long long c[kCopies];
#pragma unroll
                for (int q = 0; q < kCopies; ++q)
                    c[q] = ld_u64(row_keys(p, b, q < copies ? q : 0) + i);
#pragma unroll
                for (int q = 0; q < kCopies; ++q)
                    k = c[q] > k ? c[q] : k;
                for (int q = 0; q < copies; ++q)
                    st_u64(row_keys(p, b, q) + i, 0ull);
            }
        }
        const int a = i >= n ? -1 : k ? (int32_t)(0xFFFFFFFFu - (uint32_t)k) : 0;
        am[i] = a;
        tok[i] = i == lane ? tok0 : p.a.dtok[base + i];
        par[i] = i == lane ? par0 : p.a.dpar ? p.a.dpar[base + i] : i - 1;
        if (p.amax)
            p.amax[base + i] = a;
    }
    wave_fence();
    for (int i = lane; i < n; i += 64) {
        const int q = par[i];
        const bool valid = i >= 1 && q >= 0 && q < i;
        const bool ok = i == 0 || (valid && tok[i] == am[q]);
        st[i] = (ok ? kHolds : 0u) | ((i == 0 ? 0u : 1u) << 16) | (uint32_t)(valid ? q : 0);
    }
    wave_fence();
    int cur = 0;
    for (bool open = true; open; cur ^= 1) {
        bool more = false;
        for (int i = lane; i < n; i += 64) {
            const uint32_t s1 = st[cur * R + i];
            const uint32_t nv = jump_compose(s1, st[cur * R + (int)(s1 & 0xFFFFu)]);
            st[(cur ^ 1) * R + i] = nv;
            more |= (nv & 0xFFFFu) != 0u;
        }
        wave_fence();
        open = __ballot(more) != 0ull;
    }
    uint32_t kb = 0u;
    for (int i = lane; i < n; i += 64) {
        const uint32_t s1 = st[cur * R + i];
        const uint32_t k = (((s1 >> 16) & 0x7FFFu) << 16) | (0xFFFFu - (uint32_t)i);
        kb = (s1 & kHolds) && k > kb ? k : kb;
    }
    kb = wave_max(kb);
    const int best = (int)(0xFFFFu - (kb & 0xFFFFu)), depth = (int)(kb >> 16);
    for (int i = lane; i < R; i += 64)
        if (i > depth)
            p.out_tokens[base + i] = -1;
    if (lane == 0) {
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

// Bits 2q and 2q + 1 of `bits` (16 at most), each spread over one half of a word:
// both are moved to the halves' signs at once.
__device__ __forceinline__ uint32_t halves(uint32_t bits, int q) {
    const uint32_t w = (bits | bits << 15) << (15 - 2 * q);
    return __builtin_bit_cast(uint32_t, (s16x2)(__builtin_bit_cast(s16x2, w) >> (int16_t)15));
}
__device__ __forceinline__ uint32_t select16(uint32_t m, uint32_t x, uint32_t y) {
    return (x & m) | (y & ~m);
}

// What a work-group and its lanes have to do.  kBlkVecs: vectors of a block.
template <int kIn, int kU, int kBlkVecs>
struct Tile {
    typedef Elem<kIn> In;
    static constexpr int kPer = In::per;
    static constexpr int kBits = 128 / kPer;                  // of an element
    static constexpr int kBlkLog = __builtin_ctz(kBlkVecs * kPer);  // tokens of a block
    static constexpr int kTokens = kThreads * kU * kPer;      // of a chunk
    static constexpr uint32_t kAll = (1u << kPer) - 1u;

    uint32_t chunk;
    int chunk_log, b, n, r0, r1;
    bool masked;
    // this lane's vectors: first token, which of its tokens exist, and where it
    // is read (the row's last whole vector where fewer exist)
    int v0[kU], at[kU];
    uint32_t own[kU];

    __device__ __forceinline__ void init(const LogitsParams &p) {
        chunk_log = p.chunk_log;
        // consecutive work-groups go to different XCDs: neighbouring chunks, which
        // share lines of the masks and of rows that do not start on one, are
        // given to the work-groups of one XCD
        chunk = blockIdx.x & ((uint32_t)p.chunks - 1u);
        if (chunk_log >= 3)
            chunk = (chunk & 7u) << (chunk_log - 3) | chunk >> 3;
        const int gb = blockIdx.x >> chunk_log;
        const int group = gb % p.groups;
        b = gb / p.groups;
        r0 = group * p.rows;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            v0[u] = (int)token((uint32_t)(u * kThreads + threadIdx.x) * kPer);
            const int left = p.a.V - v0[u];
            own[u] = left >= kPer ? kAll : left > 0 ? (1u << left) - 1u : 0u;
            at[u] = v0[u] < p.a.V - kPer ? v0[u] : p.a.V - kPer;
        }
    }
    // the rows, once the draft's length is needed; false: none to do
    __device__ __forceinline__ bool rows(const LogitsParams &p) {
        n = clampi(p.a.dn[b], 1, p.a.R);
        r1 = r0 + p.rows < n ? r0 + p.rows : n;
        masked = p.a.allowed && (!p.a.allowed_on || p.a.allowed_on[b] != 0);
        return r0 < n;
    }
    // the token at place `off` of the chunk (tokens ascend with the places)
    __device__ __forceinline__ uint32_t token(uint32_t off) const {
        const uint32_t blk = ((off >> kBlkLog) << chunk_log) | chunk;
        return (blk << kBlkLog) | (off & ((1u << kBlkLog) - 1u));
    }
    // a token's place in the chunk, if it has one
    __device__ __forceinline__ bool place(int32_t t, int V, uint32_t &off) const {
        const uint32_t u = (uint32_t)t, low = (1u << kBlkLog) - 1u;
        off = ((u >> chunk_log) & ~low) | (u & low);
        return u < (uint32_t)V &&
               (u & (((1u << chunk_log) - 1u) << kBlkLog)) == (uint32_t)chunk << kBlkLog;
    }
};

// One lane's part of a row: kU vectors, the bytes with the allowed bits of their
// tokens.
template <int kU>
struct RowRegs {
    u32x4 x[kU];
    uint32_t bits[kU];
};

// The rows to read, in order.  The requests are unconditional, so that a wait
// for one row's leaves the later rows' in flight: behind the last row every lane
// reads that row's first vector, and without a mask the first bytes of the
// logits.  kTiny: V below one vector's tokens (read one by one).
template <int kIn, int kU, bool kMask, bool kTiny>
struct RowStream {
    typedef Elem<kIn> In;
    typedef typename In::type E;
    const char *src;
    const uint8_t *bits;
    int64_t step, bstep;
    int left;  // rows
    uint32_t o[kU], bo[kU];

    template <typename T>
    __device__ __forceinline__ void init(const LogitsParams &p, const T &t) {
        const int V = p.a.V;
        const int64_t row = (int64_t)t.b * p.a.R + t.r0;
        step = (int64_t)V * (int)sizeof(E);
        bstep = kMask && t.masked ? (int64_t)((V + 31) / 32) * 4 : 0;
        src = (const char *)p.a.logits + row * step;
        bits = kMask && t.masked ? (const uint8_t *)p.a.allowed + row * bstep
                                 : (const uint8_t *)p.a.logits;
        left = t.r1 - t.r0;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            o[u] = (uint32_t)t.at[u] * (uint32_t)sizeof(E);
            bo[u] = kMask && t.masked && t.v0[u] < V ? (uint32_t)t.v0[u] >> 3 : 0u;
        }
    }
    template <typename T>
    __device__ __forceinline__ void next(const LogitsParams &p, const T &t, RowRegs<kU> &g) {
        const bool live = left > 0;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            if constexpr (kTiny) {
                union {
                    E e[In::per];
                    u32x4 v;
                } x;
#pragma unroll
                for (int j = 0; j < In::per; ++j)
                    x.e[j] = ((const E *)src)[t.v0[u] + j < p.a.V ? t.v0[u] + j : 0];
                g.x[u] = x.v;
            } else {
                g.x[u] = __builtin_nontemporal_load((const u32x4_a *)(src + (live ? o[u] : 0u)));
            }
            if constexpr (kMask)
                g.bits[u] = bits[bo[u]];
        }
        left -= 1;
        const bool more = left > 0;
        src += more ? step : 0;
        bits += more ? bstep : 0;
    }
};

// The allowed bits of vector u.
template <bool kMask, typename T, int kU>
__device__ __forceinline__ uint32_t allowed_of(const T &t, int u, const RowRegs<kU> &g) {
    if (!kMask || !t.masked)
        return T::kAll;
    return (g.bits[u] >> (t.v0[u] & 7)) & T::kAll;
}

// The row's last, partial vector was read as a whole one: its own tokens first.
template <bool kTiny, typename T>
__device__ __forceinline__ u32x4 own_first(int V, uint32_t own, u32x4 x) {
    typedef unsigned __int128 u128;
    if (!kTiny && own != T::kAll && own != 0u)
        x = __builtin_bit_cast(u32x4, __builtin_bit_cast(u128, x) >>
                                          ((T::kPer - V % T::kPer) * T::kBits));
    return x;
}

constexpr float kOne = 1.0f, kZero = 0.0f;
__constant__ float c_none[2] = {kOne, kZero};

// Whether some lane of the wave has such a vector.
template <typename T>
__device__ __forceinline__ bool any_partial(const T &t) {
    bool e = false;
    for (uint32_t o : t.own)
        e = e || (o != T::kAll && o != 0u);
    return __ballot(e) != 0ull;
}

// What the list is made from, requested before anything is waited for: the
// biases, the first 4096 tokens of the context, the first 256 nodes.
constexpr int kAhead = 4;  // vectors of 4 context tokens per lane requested first
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_a __attribute__((aligned(4)));

struct Ahead {
    int32_t bi[2];
    float bv[2];
    i32x4 c[kAhead];
    int32_t tok, par;
};

// Vector v of the context: its 4 tokens, from the last whole one where fewer
// exist (Lmax >= 4).
__device__ __forceinline__ int ctx_start(int v, int Lmax) {
    return 4 * v < Lmax - 4 ? 4 * v : Lmax - 4;
}

__device__ __forceinline__ void request(const LogitsParams &p, int b, Ahead &h) {
    const int tid = threadIdx.x, nb = p.a.n_bias, R = p.a.R, Lmax = p.a.Lmax;
    if (nb > 0)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int e = tid + q * kThreads;
            const int64_t i = (int64_t)b * nb + (e < nb ? e : nb - 1);
            h.bi[q] = p.a.bias_ids[i];
            h.bv[q] = p.a.bias_vals[i];
        }
    if (p.penal) {
        const int32_t *x = p.a.tokens + (int64_t)b * Lmax;
        if (Lmax >= 4)
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
                h.c[q] = *(const i32x4_a *)(x + ctx_start(tid + q * kThreads, Lmax));
        const int64_t i = (int64_t)b * R + (tid < R ? tid : R - 1);
        h.tok = p.a.dtok[i];
        h.par = p.a.dpar ? p.a.dpar[i] : tid - 1;
    }
}

// The words and the list.  `hit`: bit u * kPer + j of a lane is set where token
// j of its vector u is listed; returns the number of listed tokens.
template <int kU, int kSplit, typename T>
__device__ __forceinline__ int list_tokens(const LogitsParams &p, const T &t, const Lds &s,
                                           const Ahead &h, Penalty &pe, uint32_t &hit) {
    constexpr int kPer = T::kPer;
    __shared__ int s_low, s_sum[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = t.b, R = p.a.R, V = p.a.V, nb = p.a.n_bias, Lmax = p.a.Lmax;
    const int32_t *x = p.a.tokens + (int64_t)b * Lmax;
    const int32_t *dt = p.a.dtok + (int64_t)b * R;
    const int32_t *dp = p.a.dpar ? p.a.dpar + (int64_t)b * R : nullptr;
    hit = 0u;
    pe = {1.0f, 0.0f, 0.0f};
    if (!p.penal && nb == 0)
        return 0;
    int L = 0, P = 0;
    if (p.penal) {
        // one entry for every sequence where an array is not given
        const float *rho = p.a.repetition ? p.a.repetition + b : &c_none[0];
        const float *freq = p.a.frequency ? p.a.frequency + b : &c_none[1];
        const float *pres = p.a.presence ? p.a.presence + b : &c_none[1];
        pe = {*rho, *freq, *pres};
        L = clampi(p.a.lengths[b], 0, Lmax);
        if (p.a.prompt_lens)
            P = clampi(p.a.prompt_lens[b], 0, L);
    }
    for (int i = tid; i < T::kTokens / 4; i += kThreads)
        ((u32x4 *)s.word)[i] = u32x4{0u, 0u, 0u, 0u};
    if (tid == 0)
        s_low = R;
    __syncthreads();
    if (nb > 0) {
        // the last entry of a token holds; entries before counts, so that the
        // maximum is over entries alone
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int e = tid + q * kThreads;
            uint32_t off;
            if (e < nb) {
                s.bias[e] = h.bv[q];
                if (t.place(h.bi[q], V, off))
                    atomicMax(&s.word[off], (uint32_t)(e + 1) << kBiasShift);
            }
        }
        __syncthreads();
    }
    if (p.penal) {
        // The prompt sets a bit, what follows it counts.  Without branches:
        // tokens of other chunks and places without a token go to words of the
        // lanes' own behind the chunk's.
        auto four = [&](const i32x4 &c, int v) {
            // of a vector that starts early, the tokens of the one before it do
            // not count again
            const int i = ctx_start(v, Lmax), d = i - 4 * v;
            const uint32_t live = 4 * v < L ? (uint32_t)(L - 4 * v) : 0u;
            const int first = 4 * (v - tid);  // of the work-group's vectors
            const bool pre = first < P, post = first + 4 * kThreads > P;
            if (first + 4 * kThreads <= L && pre != post) {
                // all of them tokens, on one side of the prompt's end: half the
                // instructions (7 x 11 rows behind 32768 tokens: 32.8 to 30.1 us)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t off;
                    const bool here = t.place(c[j], V, off);
                    uint32_t *w = s.word + (here ? off : (uint32_t)(T::kTokens + lane));
                    if (pre)
                        atomicOr(w, kPrompt);
                    else
                        atomicAdd(w, 1u);
                }
                return;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t off;
                const bool here = t.place(c[j], V, off) && (uint32_t)(d + j) < live;
                uint32_t *w = s.word + (here ? off : (uint32_t)(T::kTokens + lane));
                const bool prompt = i + j < P;
                if (pre)
                    atomicOr(w, prompt ? kPrompt : 0u);
                if (post)
                    atomicAdd(w, prompt ? 0u : 1u);
            }
        };
        if (Lmax < 4) {
            uint32_t off;
            if (tid < L && t.place(x[tid], V, off)) {
                if (tid < P)
                    atomicOr(&s.word[off], kPrompt);
                else
                    atomicAdd(&s.word[off], 1u);
            }
        } else {
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
                if (4 * q * kThreads < L)
                    four(h.c[q], tid + q * kThreads);
            for (int v = tid + kAhead * kThreads; 4 * (v - tid) < L; v += 8 * kThreads) {
                i32x4 c[8];  // 16 took 1 us off 32768 tokens, and waves off the CUs: 206 to 220 us
                             // for 32 x 201 drafted rows
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    c[q] = *(const i32x4_a *)(x + ctx_start(v + q * kThreads, Lmax));
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (4 * (v - tid + q * kThreads) < L)
                        four(c[q], v + q * kThreads);
            }
        }
        // the draft's nodes, with their tokens' places
        int32_t d_tok = h.tok, d_par = h.par;
        for (int i = tid; i < t.n; i += kThreads) {
            if (i != tid) {
                d_tok = dt[i];
                d_par = dp ? dp[i] : i - 1;
            }
            uint32_t off;
            const bool here = t.place(d_tok, V, off) && i >= 1;
            const uint32_t par = d_par >= 0 && d_par < i ? (uint32_t)d_par : kNone;
            s.node[i] = par | (here ? off : kNone) << 16;
            if (here)
                atomicMin(&s_low, i);
        }
        for (int i = tid; i < (int)path_bytes(t.r1 - t.r0, R) / 4; i += kThreads)
            ((uint32_t *)s.path)[i] = 0u;
        __syncthreads();
        // one of a token's nodes, the first to arrive, stands for it and keeps
        // its count
        if (s_low < R) {
            for (int i = tid; i < t.n; i += kThreads) {
                const uint32_t off = s.node[i] >> 16;
                if (off == kNone)
                    continue;
                const uint32_t w = atomicOr(&s.word[off], kDrafted);
                if (!(w & kDrafted)) {
                    s.count[i] = w & (kCount | kPrompt);
                    s.word[off] = (w & ~(kCount | kPrompt)) | kDrafted | (uint32_t)i;
                }
            }
            __syncthreads();
            for (int i = tid; i < t.n; i += kThreads) {
                const uint32_t nd = s.node[i], off = nd >> 16;
                if (off != kNone)
                    s.node[i] = (nd & 0xFFFFu) | (s.word[off] & kCount) << 16;
            }
        }
    }
    // the list, each lane's tokens together
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
        for (int q = 0; q < kPer / 4; ++q) {
            const u32x4 w = ((const u32x4 *)s.word)[(u * kThreads + tid) * (kPer / 4) + q];
            hit |= ((w.x ? 1u : 0u) | (w.y ? 2u : 0u) | (w.z ? 4u : 0u) | (w.w ? 8u : 0u))
                   << (u * kPer + q * 4);
        }
    // tokens, and << 16 vectors with one (at most 4096 and 512)
    int mine = __popc(hit);
    if (kSplit == 1)
#pragma unroll
        for (int u = 0; u < kU; ++u)
            mine += (hit >> (u * kPer)) & T::kAll ? 1 << 16 : 0;
    const int upto = wave_scan(mine);
    if (lane == 63)
        s_sum[wave] = upto;
    __syncthreads();
    int k = upto - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        k += w < wave ? s_sum[w] : 0;
        total += s_sum[w];
    }
    total &= 0xFFFF;
    if constexpr (kSplit > 0) {
        int v = k >> 16;
        k &= 0xFFFF;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const uint32_t hu = (hit >> (u * kPer)) & T::kAll;
            const uint32_t slot = hu && v < kSlots ? (uint32_t)v : kNoSlot;
            if (kSplit == 1)
                s.slot[u * kThreads + tid] = (uint8_t)slot;
            for (uint32_t h = hu; h; h &= h - 1u) {
                const int j = __ffs(h) - 1;
                const uint32_t at = slot == kNoSlot ? kNone : slot * kPer + j;
                const uint32_t off = (uint32_t)((u * kThreads + tid) * kPer + j);
                if (k < kListed) {
                    ((uint32_t *)s.list)[k] = off | at << 16;
                    s.lword[k] = s.word[off];
                }
                ++k;
            }
            v += hu ? 1 : 0;
        }
    } else {
        k &= 0xFFFF;
        for (uint32_t h = hit; h; h &= h - 1u) {
            const int j = __ffs(h) - 1;
            ((uint16_t *)s.list)[k++] =
                (uint16_t)(((j / kPer) * kThreads + tid) * kPer + j % kPer);
        }
    }
    if (p.penal && s_low < R && tid < t.r1 - t.r0) {
        // each row's path, down to the lowest node with a token of the chunk
        const int low = s_low, row = tid * R;
        for (uint32_t i = (uint32_t)(t.r0 + tid); i != kNone && (int)i >= low;) {
            const uint32_t nd = s.node[i], e = nd >> 16;
            if (e != kNone) {
                if (R > 256)
                    ((uint16_t *)s.path)[row + e] += 1;
                else
                    s.path[row + e] += 1;
            }
            i = nd & 0xFFFFu;
        }
    }
    __syncthreads();
    return total;
}

// A store that a lane can leave out without a branch: an offset behind the row's
// bytes is dropped.
constexpr uint32_t kNowhere = 0x80000000u;
constexpr int kNt = 2;  // nontemporal

template <int kIn, int kOut, int kU, bool kMask, bool kTiny>
__global__ __launch_bounds__(kThreads) void k_process(LogitsParams p) {
    typedef Tile<kIn, kU, kProcessBlk> T;
    typedef Elem<kIn> In;
    typedef Elem<kOut> Out;
    typedef typename Out::type O;
    constexpr int kPer = T::kPer;
    constexpr uint32_t kAll = T::kAll;
    extern __shared__ __align__(16) unsigned char mem[];
    const int tid = threadIdx.x, R = p.a.R, V = p.a.V;
    T t;
    t.init(p);
    Ahead h;
    request(p, t.b, h);
    if (!t.rows(p))
        return;
    Lds s;
    lds_carve(mem, T::kTokens, sizeof(typename In::type), R, p.rows, p.a.n_bias, 0, s);
    // in place without a mask, only the listed tokens are read and written
    const bool sparse = p.in_place && !(kMask && t.masked);
    RowRegs<kU> ra, rb, rc;
    RowStream<kIn, kU, kMask, kTiny> rows;
    rows.init(p, t);
    if (!sparse) {
        rows.next(p, t, ra);
        rows.next(p, t, rb);
    }
    Penalty pe;
    uint32_t hit;
    const int listed = list_tokens<kU, 0>(p, t, s, h, pe, hit);
    const uint16_t *list = (const uint16_t *)s.list;
    if (sparse) {
        if constexpr (kIn == kOut)
            for (int r = t.r0; r < t.r1; ++r) {
                O *dst = (O *)p.out + ((int64_t)t.b * R + r) * V;
                for (int k = tid; k < listed; k += kThreads) {
                    const uint32_t off = list[k];
                    O *d = dst + t.token(off);
                    *d = Out::put(processed(In::get(*d), s.word[off], pe, s,
                                            (r - t.r0) * R, R > 256));
                }
            }
        return;
    }
    typename In::type *stage = (typename In::type *)s.stage;
    const bool edge = any_partial(t);
    O *dst = (O *)p.out + ((int64_t)t.b * R + t.r0) * V;
    auto step = [&](RowRegs<kU> &g, int r) {
        const __amdgpu_buffer_rsrc_t rs =
            __builtin_amdgcn_make_buffer_rsrc(dst, 0, V * (int)sizeof(O), 0x00027000);
        if (edge)
#pragma unroll
            for (int u = 0; u < kU; ++u)
                g.x[u] = own_first<kTiny, T>(V, t.own[u], g.x[u]);
        if (listed > 0) {
#pragma unroll
            for (int u = 0; u < kU; ++u)
                if ((hit >> (u * kPer)) & kAll)
                    ((u32x4 *)stage)[u * kThreads + tid] = g.x[u];
            __syncthreads();
            for (int k = tid; k < listed; k += kThreads) {
                const uint32_t off = list[k];
                const float y = processed(In::get(stage[off]), s.word[off], pe, s,
                                          (r - t.r0) * R, R > 256);
                if constexpr (sizeof(typename In::type) == 4)
                    stage[off] = y;
                else
                    stage[off] = Out::put(y);
            }
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const uint32_t hu = (hit >> (u * kPer)) & kAll;
            const uint32_t ok = allowed_of<kMask>(t, u, g);
            const u32x4 x = g.x[u];
            u32x4 y = x;
            if (hu)
                y = ((const u32x4 *)stage)[u * kThreads + tid];
            uint32_t pk[kPer / 2];  // 16-bit results, in pairs
            if constexpr (kOut == SWITCHSD_F32) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    y[j] = !kMask || ((ok >> j) & 1u) ? y[j] : 0xFF800000u;
            } else {
                constexpr uint32_t kInf = kOut == SWITCHSD_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
#pragma unroll
                for (int q = 0; q < kPer / 2; ++q) {
                    if constexpr (kIn == kOut) {
                        pk[q] = y[q];
                    } else if constexpr (kIn == SWITCHSD_F32) {
                        pk[q] = (uint32_t)Out::put(__uint_as_float(y[2 * q])) |
                                (uint32_t)Out::put(__uint_as_float(y[2 * q + 1])) << 16;
                    } else {
                        pk[q] = (uint32_t)Out::put(In::get((uint16_t)x[q])) |
                                (uint32_t)Out::put(In::get((uint16_t)(x[q] >> 16))) << 16;
                        if (hu)  // listed tokens already have the output's type
                            pk[q] = select16(halves(hu, q), y[q], pk[q]);
                    }
                    if (kMask && ok != kAll)
                        pk[q] = select16(halves(ok, q), pk[q], kInf);
                }
            }
            const bool write = !p.in_place || hu || ok != kAll;
            const uint32_t o = t.own[u] == kAll && write
                                   ? (uint32_t)t.v0[u] * (uint32_t)sizeof(O)
                                   : kNowhere;
            if constexpr (kOut == SWITCHSD_F32)
                __builtin_amdgcn_raw_buffer_store_b128(y, rs, o, 0, kNt);
            else if constexpr (kPer == 8)
                __builtin_amdgcn_raw_buffer_store_b128(u32x4{pk[0], pk[1], pk[2], pk[3]}, rs, o, 0,
                                                       kNt);
            else
                __builtin_amdgcn_raw_buffer_store_b64(u32x2{pk[0], pk[1]}, rs, o, 0, kNt);
            if (edge && t.own[u] != kAll && t.own[u] != 0u && write) {
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if ((t.own[u] >> j) & 1u) {
                        if constexpr (kOut == SWITCHSD_F32)
                            dst[t.v0[u] + j] = __uint_as_float(y[j]);
                        else
                            dst[t.v0[u] + j] = (uint16_t)(pk[j / 2] >> (16 * (j & 1)));
                    }
            }
        }
        dst += V;
    };
    for (int r = t.r0; r < t.r1; r += 3) {
        rows.next(p, t, rc);
        step(ra, r);
        rows.next(p, t, ra);
        if (r + 1 < t.r1)
            step(rb, r + 1);
        rows.next(p, t, rb);
        if (r + 2 < t.r1)
            step(rc, r + 2);
    }
}

// The order key (of its value in bf16) of element j of a vector.
template <int kIn>
__device__ __forceinline__ uint32_t elem_key(const u32x4 &x, int j) {
    typedef Elem<kIn> In;
    if constexpr (kIn == SWITCHSD_F32) {
        return order16(Elem<SWITCHSD_BF16>::put(__uint_as_float(x[j])));
    } else {
        const uint32_t e = (x[j / 2] >> (16 * (j & 1))) & 0xFFFFu;
        if constexpr (kIn == SWITCHSD_BF16)
            return order16(e);
        else
            return order16(Elem<SWITCHSD_BF16>::put(In::get((uint16_t)e)));
    }
}

// The order key of the maximum of kU vectors (0: nothing but NaN).  Rounding to
// bf16 keeps the order, so the maximum is taken on the input's patterns: as
// signed integers where one is not negative, as unsigned ones (the smallest)
// where all are; a positive NaN takes the slow way.
template <int kIn, int kU>
__device__ __forceinline__ uint32_t lane_key(const u32x4 (&x)[kU]) {
    typedef Elem<SWITCHSD_BF16> B;
    constexpr bool k32 = kIn == SWITCHSD_F32;
    constexpr int32_t kTop = k32 ? 0x7F800000 : kIn == SWITCHSD_BF16 ? 0x7F80 : 0x7C00;
    auto smax = [](uint32_t a, uint32_t c) {
        return k32 ? (uint32_t)((int32_t)a > (int32_t)c ? (int32_t)a : (int32_t)c)
                   : pk_max_i16(a, c);
    };
    auto umin = [](uint32_t a, uint32_t c) { return k32 ? (a < c ? a : c) : pk_min_u16(a, c); };
    uint32_t m = x[0].x;
#pragma unroll
    for (int u = 0; u < kU; ++u)
        m = smax(smax(smax(m, x[u].x), x[u].y), smax(x[u].z, x[u].w));
    int32_t mx = (int32_t)m;
    if constexpr (!k32) {
        const int32_t m0 = (int16_t)m, m1 = (int32_t)m >> 16;
        mx = m0 > m1 ? m0 : m1;
    }
    if (mx > kTop) {
        uint32_t k = 0u;
        for (int u = 0; u < kU; ++u)
#pragma unroll
            for (int j = 0; j < Elem<kIn>::per; ++j) {
                const uint32_t e = elem_key<kIn>(x[u], j);
                k = e > k ? e : k;
            }
        return k;
    }
    uint32_t v = (uint32_t)mx;
    if (mx < 0) {
        uint32_t l = x[0].x;
#pragma unroll
        for (int u = 0; u < kU; ++u)
            l = umin(umin(umin(l, x[u].x), x[u].y), umin(x[u].z, x[u].w));
        v = k32 ? l : (l & 0xFFFFu) < (l >> 16) ? l & 0xFFFFu : l >> 16;
    }
    if constexpr (k32)
        return order16(B::put(__uint_as_float(v)));
    else if constexpr (kIn == SWITCHSD_BF16)
        return order16(v);
    else
        return order16(B::put(Elem<kIn>::get((uint16_t)v)));
}

// The lowest token's place with key `top` among a lane's vectors of a piece (the
// first is number `v` of the chunk, the next 64 or kThreads on, see kSplit).
template <int kIn, int kSplit, int kU>
__device__ __forceinline__ uint32_t lane_place(const u32x4 (&x)[kU], uint32_t top, uint32_t v) {
    constexpr int kPer = Elem<kIn>::per;
    uint32_t at = kNone;
#pragma unroll
    for (int u = kU - 1; u >= 0; --u)
#pragma unroll
        for (int j = kPer - 1; j >= 0; --j)
            at = elem_key<kIn>(x[u], j) == top ? (u * kSplit * 64 + v) * kPer + j : at;
    return at;
}

// A wave's maximum of a row in LDS: order key << 15 | place, or | the vector
// that holds it, which is then in LDS too.
constexpr uint32_t kPlaced = 0x80000000u;

// kSplit: waves that share a row.  4: each of them takes a quarter of the
// chunk of every row; 1: a wave takes the whole chunk of every fourth row, in
// four pieces, and closes a row (wave maximum, listed tokens) once per four
// pieces.  A wave holds four pieces in registers; each is requested anew, for
// the row after next in its place, once it has been used.  Whole rows keep the
// vectors with listed tokens in LDS, wave by wave; quarters read those tokens
// beside them (one per lane with the row's other requests).
// kU: vectors of a piece per lane.
// Measured, whole rows / quarters of 128256 tokens: 128 x 2 rows 58.8 / 51.0 us,
// 64 x 6 43.0 / 39.8, 32 x 10 28.4 / 27.8, 32 x 13 31.5 / 32.6, 32 x 16 34.8 /
// 37.3, 32 x 32 56.8 / 62.2, 32 x 201 candidate rows under a grammar 206 / 275;
// whole rows from kWholeRows rows a work-group on.
constexpr int kBufs = 4;
// Waves per SIMD the registers are kept to (floats under a mask need more of
// them).
constexpr int waves_of(int in, int split, bool mask) {
    return in == SWITCHSD_F32 && mask && split == 1 ? 3 : 4;
}

template <int kIn, int kSplit, int kU, bool kMask, bool kTiny>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(kTiny ? 1 : waves_of(kIn, kSplit, kMask)))) void
k_verify(LogitsParams p) {
    constexpr int kP = kWaves / kSplit;    // pieces of a row per wave
    constexpr int kRows = kBufs / kP;      // rows held at once
    constexpr int kStep = kWaves / kSplit; // a wave's rows are this far apart
    constexpr int kLanes = kSplit * 64;    // lanes that share a row's listed tokens
    typedef Tile<kIn, kU, kVerifyBlk> T;
    typedef Elem<kIn> In;
    typedef typename In::type E;
    constexpr int kPer = T::kPer;
    constexpr uint32_t kAll = T::kAll;
    constexpr int kWords = T::kTokens / 32;       // of the chunk's allowed bits
    constexpr int kWordLoads = (kWords + 63) / 64;
    extern __shared__ __align__(16) unsigned char mem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int R = p.a.R, V = p.a.V;
    T t;
    t.init(p);
    Ahead h;
    request(p, t.b, h);
    if (!t.rows(p))
        return;
    Lds s;
    lds_carve(mem, T::kTokens, sizeof(E), R, p.rows, p.a.n_bias, kSplit, s);
    const bool masked = kMask && t.masked;

    // ---- the pieces' vectors: number `n` of a lane starts at token v0 + n *
    // span; a vector that does not exist whole is read as the row's last whole one
    auto vec = [&](int q, int u) {
        return kSplit == 1 ? (uint32_t)((q * kU + u) * 64 + lane)
                           : (uint32_t)((u * kWaves + wave) * 64 + lane);
    };
    const int v0 = (int)t.token(vec(0, 0) * kPer);
    const int span = (kSplit * 64 / kVerifyBlk) << (t.chunk_log + T::kBlkLog);
    auto own = [&](int n) {
        const int left = V - (v0 + n * span);
        return left >= kPer ? kAll : left > 0 ? (1u << left) - 1u : 0u;
    };
    bool part = false;
#pragma unroll
    for (int n = 0; n < kP * kU; ++n)
        part = part || (own(n) != kAll && own(n) != 0u);
    const bool edge = __ballot(part) != 0ull;
    const int first = t.r0 + (kSplit == 1 ? wave : 0);
    const int64_t words = (V + 31) / 32;
    u32x4 x[kBufs][kU];
    uint32_t bw[kRows][kWordLoads];
    E ix[kRows];
    // Row r of the logits (behind the last row: that row).
    auto row_of = [&](int r) { return (int64_t)t.b * R + (r < t.r1 ? r : t.r1 - 1); };
    // All requests are unconditional, so that a wait for one piece leaves the
    // later ones in flight: behind the last row every lane reads that row's
    // first vector.
    auto fetch = [&](int j, int r) {
        const char *src = (const char *)p.a.logits + row_of(r) * V * (int64_t)sizeof(E);
        const bool live = r < t.r1;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int v = v0 + (j % kP * kU + u) * span;
            const int at = v < V - kPer ? v : V - kPer;
            if constexpr (kTiny) {
                union {
                    E e[kPer];
                    u32x4 v;
                } y;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    y.e[i] = ((const E *)src)[v < V && v + i < V ? v + i : 0];
                x[j][u] = y.v;
            } else {
                x[j][u] = __builtin_nontemporal_load(
                    (const u32x4_a *)(src + (live ? (uint32_t)at * (uint32_t)sizeof(E) : 0u)));
            }
        }
    };
    // the words with the allowed bits of the chunk, 32 places each
    uint32_t wat[kWordLoads];
#pragma unroll
    for (int i = 0; i < kWordLoads; ++i) {
        const uint32_t place = (uint32_t)(lane + i * 64) * 32u;
        const uint32_t tok = t.token(place);
        wat[i] = masked && place < (uint32_t)T::kTokens && tok < (uint32_t)V ? tok >> 5 : 0u;
    }
    auto fetch_bits = [&](int i, int r) {
        if constexpr (kMask) {  // (without a mask a word of the nodes' counts)
            const uint32_t *w = masked ? p.a.allowed + row_of(r) * words
                                       : (const uint32_t *)p.a.dn;
#pragma unroll
            for (int q = 0; q < kWordLoads; ++q)
                bw[i][q] = w[wat[q]];
        }
    };
#pragma unroll
    for (int j = 0; j < kBufs; ++j) {
        if (j % kP == 0)
            fetch_bits(j / kP, first + j / kP * kStep);
        fetch(j, first + j / kP * kStep);
    }
    for (int i = tid; i < 2 * p.rows * kSplit; i += kThreads)
        s.key[i] = 0u;
    __syncthreads();
    Penalty pe;
    uint32_t mine;
    const int listed = list_tokens<kU, kSplit>(p, t, s, h, pe, mine);
    const uint32_t *list = (const uint32_t *)s.list;
    const bool fits = listed <= kListed;

    // What is listed or does not exist leaves the maximum (all bits set: a
    // negative NaN), and so does what is not allowed; -inf, which an allowed or a
    // forbidden token may be, matters only where nothing is above it.
    constexpr uint32_t kLow = 0x007Fu;  // the key of -inf
    auto spread = [](uint32_t b, int q) {
        return kIn == SWITCHSD_F32 ? (uint32_t)((int32_t)(b << (31 - q)) >> 31) : halves(b, q);
    };
    u32x4 gone[kU];  // of vectors u * kThreads + tid: with shared rows, this lane's
    uint32_t inner[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        inner[u] = t.own[u] & ~(mine >> (u * kPer));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            gone[u][i] = spread(~inner[u] & kAll, i);
        if (kSplit == 1) {
            if (fits)
                s.gone[u * kThreads + tid] = gone[u];
            s.inner[u * kThreads + tid] = (uint8_t)inner[u];
        }
    }
    if (kSplit == 1)
        __syncthreads();
    uint64_t slots = ~0ull;  // of this lane's vectors in `held`, a byte each
    if (kSplit == 1 && listed > 0 && fits) {
        slots = 0ull;
#pragma unroll
        for (int n = 0; n < kP * kU; ++n)
            slots |= (uint64_t)s.slot[vec(n / kU, n % kU)] << (8 * n);
    }
    u32x4 *held = s.held + wave * kSlots;
    uint32_t *abits = s.bits + wave * kWords;
    auto allowed_at = [&](uint32_t v) {  // the allowed bits of vector v, lowest first
        return (uint32_t)((const uint8_t *)abits)[v * kPer >> 3] >> (v * kPer & 7u);
    };
    const int nth = kSplit == 1 ? lane : tid;
    uint32_t entry0 = 0u, word0 = 0u;  // this lane's first listed token
    if (nth < listed) {
        entry0 = list[nth];
        word0 = s.lword[nth];
    }
    const uint32_t item0 = t.token(entry0 & 0xFFFFu) * (uint32_t)sizeof(E);
    auto fetch_item = [&](int i, int r) {  // (lanes without one: the chunk's first token)
        if constexpr (kSplit != 1)
            ix[i] = *(const E *)((const char *)p.a.logits +
                                 row_of(r) * V * (int64_t)sizeof(E) +
                                 (nth < listed ? item0 : 0u));
    };
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        fetch_item(i, first + i * kStep);

    // ---- the rows
    for (int r = first; r < t.r1; r += kRows * kStep) {
        uint32_t best = 0u, bq = 0u;    // the lane's maximum and its piece
        u32x4 top_x[kU];
#pragma unroll
        for (int j = 0; j < kBufs; ++j) {
            const int q = j % kP, row = r + j / kP * kStep;
            if (kSplit != 1 && row >= t.r1)
                break;
            if (q == 0) {
                best = bq = 0u;
                if constexpr (kMask) {
#pragma unroll
                    for (int i = 0; i < kWordLoads; ++i)
                        if (kWords % 64 == 0 || lane + i * 64 < kWords)
                            abits[lane + i * 64] = bw[j / kP][i];
                    fetch_bits(j / kP, row + kRows * kStep);
                }
                wave_fence();
            }
            u32x4 y[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                y[u] = x[j][u];
                if (edge)
                    y[u] = own_first<kTiny, T>(V, own(q * kU + u), y[u]);
                if (kSplit == 1) {
                    const uint32_t slot = (uint32_t)(slots >> (8 * (q * kU + u))) & 0xFFu;
                    if (slot != kNoSlot)
                        held[slot] = y[u];
                }
                if (kSplit != 1)
                    y[u] |= gone[u];
                else if (fits)
                    y[u] |= s.gone[vec(q, u)];
                else
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        y[u][i] |= spread(~(uint32_t)s.inner[vec(q, u)] & kAll, i);
                if (masked) {
                    const uint32_t no = ~allowed_at(vec(q, u)) & kAll;
                    if (__ballot(no != 0u) != 0ull)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            y[u][i] |= spread(no, i);
                }
            }
            const uint32_t k = lane_key<kIn, kU>(y);
            const bool up = q == 0 || k > best;
            best = up ? k : best;
            bq = up ? (uint32_t)q : bq;
#pragma unroll
            for (int u = 0; u < kU; ++u)
                top_x[u] = up ? y[u] : top_x[u];
            fetch(j, row + kRows * kStep);
            const E x0 = ix[j / kP];
            if (q == kP - 1)
                fetch_item(j / kP, row + kRows * kStep);
            if (q != kP - 1)
                continue;
            uint32_t top = wave_max(best);
            uint32_t forb = kNone;  // this lane's lowest forbidden place
            if (masked && top <= kLow) {
                // nothing above -inf: a forbidden token is -inf too
#pragma unroll
                for (int i = kP * kU - 1; i >= 0; --i) {
                    const uint32_t v = vec(i / kU, i % kU);
                    const uint32_t no =
                        ~allowed_at(v) & (kSplit == 1 ? (uint32_t)s.inner[v] : inner[i % kU]);
                    forb = no ? v * kPer + (uint32_t)__ffs(no) - 1u : forb;
                }
                top = __ballot(forb != kNone) != 0ull ? kLow : top;
            }
            const unsigned long long who = __ballot(best == top);
            const int slot = (row - t.r0) * kSplit + (kSplit == 1 ? 0 : wave);
            if (top > kLow && (who & (who - 1ull)) == 0ull) {
                // one lane holds it: its token is looked up when the rows are done
                if (best == top) {
                    s.key[slot] = (top << 15) | (bq * 64u * kU + vec(0, 0));
#pragma unroll
                    for (int u = 0; u < kU; ++u)
                        ((u32x4 *)s.stage)[slot * kU + u] = top_x[u];
                }
            } else if (top != 0u) {
                uint32_t at = kNone;
                if (best == top)
                    at = lane_place<kIn, kSplit, kU>(top_x, top, bq * 64u * kU + vec(0, 0));
                at = forb < at ? forb : at;
                const uint32_t low = kNone - wave_max(kNone - at);
                if (lane == 0)
                    s.key[slot] = kPlaced | (top << 15) | low;
            }
            wave_fence();
            if ((kSplit == 1 ? 0 : wave * 64) < listed) {
                uint32_t ki = 0u;  // order key, then the lowest place
                auto value = [&](uint32_t place, uint32_t at) {
                    return kSplit == 1 && at != kNone
                               ? ((const E *)held)[at]
                               : ((const E *)p.a.logits)[row_of(row) * V + t.token(place)];
                };
                auto item = [&](E v, uint32_t place, uint32_t w) {
                    const float f = processed(In::get(v), w, pe, s, (row - t.r0) * R, R > 256);
                    const bool ok = !masked || ((abits[place >> 5] >> (place & 31u)) & 1u);
                    const uint32_t o = order16(ok ? Elem<SWITCHSD_BF16>::put(f) : 0xFF80u);
                    const uint32_t k2 = o ? (o << 16) | (kNone - place) : 0u;
                    ki = k2 > ki ? k2 : ki;
                };
                if (fits && kSplit == 1) {
                    // four of the lane's tokens at a time, their reads together
                    for (int i0 = lane; i0 < listed + lane; i0 += 4 * kLanes) {
                        uint32_t e[4], w[4];
                        E v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int c = i0 + i * kLanes < listed ? i0 + i * kLanes : 0;
                            e[i] = list[c];
                            w[i] = s.lword[c];
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[i] = ((const E *)held)[e[i] >> 16 != kNone ? e[i] >> 16 : 0u];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (i0 + i * kLanes < listed)
                                item(e[i] >> 16 != kNone ? v[i] : value(e[i] & 0xFFFFu, kNone),
                                     e[i] & 0xFFFFu, w[i]);
                    }
                } else if (fits) {
                    if (nth < listed)
                        item(x0, entry0 & 0xFFFFu, word0);
                    for (int i = nth + kLanes; i < listed; i += kLanes) {
                        const uint32_t e = list[i];
                        item(value(e & 0xFFFFu, kNone), e & 0xFFFFu, s.lword[i]);
                    }
                } else {
                    // more than the list holds: every token with a word
                    for (int i = nth; i < T::kTokens; i += kLanes)
                        if (s.word[i] != 0u)
                            item(value((uint32_t)i, kNone), (uint32_t)i, s.word[i]);
                }
                ki = wave_max(ki);
                if (lane == 0)
                    s.key[p.rows * kSplit + slot] = ki;
            }
            wave_fence();
        }
    }
    __syncthreads();
    // the places of the maxima that one lane held
    for (int i = tid; i < (t.r1 - t.r0) * kSplit; i += kThreads) {
        const uint32_t e = s.key[i];
        const uint32_t top = (e & ~kPlaced) >> 15;
        uint32_t at = e & 0x7FFFu;
        if (!(e & kPlaced)) {
            u32x4 y[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u)
                y[u] = ((const u32x4 *)s.stage)[i * kU + u];
            at = lane_place<kIn, kSplit, kU>(y, top, at);
        }
        s.key[i] = e != 0u ? (top << 16) | (kNone - at) : 0u;
    }
    __syncthreads();
    if (tid >= 64)
        return;
    // one row per lane (at most kRowGroup = 64 rows)
    const int64_t node = (int64_t)t.b * R + (tid < R ? tid : R - 1);
    const int tok0 = p.a.dtok[node];
    int par0 = tid - 1;
    if (p.a.dpar)
        par0 = p.a.dpar[node];
    if (tid < t.r1 - t.r0) {
        uint32_t k = 0u;
#pragma unroll
        for (int q = 0; q < kSplit; ++q) {
            const uint32_t a = s.key[tid * kSplit + q];
            const uint32_t c = s.key[(p.rows + tid) * kSplit + q];
            k = a > k ? a : k;
            k = c > k ? c : k;
        }
        if (k)
            __hip_atomic_fetch_max(row_keys(p, t.b, (int)(t.chunk % kCopies)) + t.r0 + tid,
                                   ((unsigned long long)order32(k >> 16) << 32) |
                                       (0xFFFFFFFFu - t.token(kNone - (k & 0xFFFFu))),
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (arrive(&p.tickets[(int64_t)t.b * kLineU32],
               (uint32_t)(p.chunks * ((t.n + p.rows - 1) / p.rows))))
        accept(p, t.b, t.n, tok0, par0, mem);
}

// kU: vectors per lane and row (of a piece); kSplit: waves that share a row of
// k_verify, 0: k_process.
template <int kIn, int kOut, int kU, int kSplit, bool kTiny, bool kMask>
int launch(const LogitsParams &p, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)p.a.B * p.groups * p.chunks));
    Lds l;
    const size_t lds = lds_carve(nullptr, kThreads * kU * Elem<kIn>::per,
                                 sizeof(typename Elem<kIn>::type), p.a.R, p.rows, p.a.n_bias,
                                 kSplit, l);
    if constexpr (kSplit > 0)
        hipLaunchKernelGGL((k_verify<kIn, kSplit, kU, kMask, kTiny>), grid, dim3(kThreads), lds,
                           stream, p);
    else
        hipLaunchKernelGGL((k_process<kIn, kOut, kU, kMask, kTiny>), grid, dim3(kThreads), lds,
                           stream, p);
    return hipGetLastError() == hipSuccess ? SWITCHSD_OK : SWITCHSD_EHIP;
}

template <int kIn, int kOut, bool kVerify, bool kMask>
int launch_unroll(const LogitsParams &p, hipStream_t stream) {
    constexpr int kSplit = kVerify ? 4 : 0;
    if (p.a.V < Elem<kIn>::per)
        return launch<kIn, kOut, 1, kSplit, true, kMask>(p, stream);
    if constexpr (kVerify)
        if (p.split == 1)
            return launch<kIn, kOut, 2, 1, false, kMask>(p, stream);
    return p.unroll == 2 ? launch<kIn, kOut, 2, kSplit, false, kMask>(p, stream)
                         : launch<kIn, kOut, 1, kSplit, false, kMask>(p, stream);
}

template <int kIn, int kOut, bool kVerify>
int launch_mask(const LogitsParams &p, hipStream_t stream) {
    return p.a.allowed ? launch_unroll<kIn, kOut, kVerify, true>(p, stream)
                       : launch_unroll<kIn, kOut, kVerify, false>(p, stream);
}

}  // namespace

int launch_logits_kernel(const LogitsParams &p, int32_t out_type, hipStream_t stream) {
    constexpr int BF = SWITCHSD_BF16, HF = SWITCHSD_F16, FF = SWITCHSD_F32;
    const int in = p.a.logits_type;
    if (!p.out)  // verify
        return in == BF   ? launch_mask<BF, BF, true>(p, stream)
               : in == HF ? launch_mask<HF, BF, true>(p, stream)
                          : launch_mask<FF, BF, true>(p, stream);
    if (in == BF)
        return launch_mask<BF, BF, false>(p, stream);
    if (in == HF)
        return out_type == BF ? launch_mask<HF, BF, false>(p, stream)
                              : launch_mask<HF, HF, false>(p, stream);
    return out_type == BF ? launch_mask<FF, BF, false>(p, stream)
                          : launch_mask<FF, FF, false>(p, stream);
}

}  // namespace switchsd
