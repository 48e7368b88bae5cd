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

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// ---- elements

template <int TYPE>
constexpr int kPerVec = TYPE == SWITCHSD_F32 ? 4 : 8;  // elements of 16 bytes
template <int TYPE>
constexpr int kSize = TYPE == SWITCHSD_F32 ? 4 : 2;

typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));

// Rows stand at any element's address; so do their vectors.
template <int TYPE>
__device__ __forceinline__ u32x4 load_vec(const char *row, int64_t vec) {
    if (TYPE == SWITCHSD_F32)
        return *(const u32x4_a4 *)(row + vec * 16);
    return *(const u32x4_a2 *)(row + vec * 16);
}

template <int TYPE>
__device__ __forceinline__ float element(u32x4 x, int e) {
    if (TYPE == SWITCHSD_F32)
        return __builtin_bit_cast(float, (uint32_t)x[e]);
    if (TYPE == SWITCHSD_BF16)
        return __builtin_bit_cast(float, e % 2 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(x[e / 2] >> (e % 2 * 16)));
}

template <int TYPE>
__device__ __forceinline__ float load_logit(const char *row, int64_t at) {
    if (TYPE == SWITCHSD_F32)
        return ((const float *)row)[at];
    const uint16_t v = ((const uint16_t *)row)[at];
    if (TYPE == SWITCHSD_BF16)
        return __builtin_bit_cast(float, (uint32_t)v << 16);
    return (float)__builtin_bit_cast(_Float16, v);
}

template <int TYPE>
__device__ __forceinline__ void store_logit(char *row, int64_t at, float v) {
    if (TYPE == SWITCHSD_F32)
        ((float *)row)[at] = v;
    else if (TYPE == SWITCHSD_BF16)
        ((uint16_t *)row)[at] = __builtin_bit_cast(uint16_t, (__bf16)v);
    else
        ((uint16_t *)row)[at] = __builtin_bit_cast(uint16_t, (_Float16)v);
}

// The vector behind the last whole one, NaN where there is nothing.
template <int TYPE>
__device__ __forceinline__ u32x4 load_last(const char *row, int64_t vec, int V) {
    u32x4 x = u32x4{~0u, ~0u, ~0u, ~0u};
    for (int e = 0; e < kPerVec<TYPE>; ++e) {
        const int64_t v = vec * kPerVec<TYPE> + e;
        if (v >= V)
            break;
        if (TYPE == SWITCHSD_F32)
            x[e] = ((const uint32_t *)row)[v];
        else
            x[e / 2] = (x[e / 2] & ~(0xFFFFu << (e % 2 * 16))) |
                       (uint32_t)((const uint16_t *)row)[v] << (e % 2 * 16);
    }
    return x;
}

// Keys that order logits: larger first (-0 as 0), NaN behind all numbers as 0.
__device__ __forceinline__ uint32_t order_of(float l) {
    if (!(l == l))
        return 0;
    const uint32_t u = __builtin_bit_cast(uint32_t, l + 0.0f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
constexpr uint32_t kMinusInf = ~0xFF800000u;  // order_of(-inf)
// With the lower index first among equals.  Never 0.
__device__ __forceinline__ unsigned long long order_key(float l, uint32_t v) {
    return (unsigned long long)order_of(l) << 32 | (0xFFFFFFFFu - v);
}
__device__ __forceinline__ float key_logit(unsigned long long key) {
    const uint32_t s = (uint32_t)(key >> 32);
    return __builtin_bit_cast(float, s == 0 ? 0x7FC00000u : (s >> 31) ? s & 0x7FFFFFFFu : ~s);
}
__device__ __forceinline__ uint32_t key_index(unsigned long long key) {
    return 0xFFFFFFFFu - (uint32_t)key;
}

// ---- entries

// A sequence's entries: how many, and entry i's row.  Along a path: the walk from
// accept_node to the anchor leaves its nodes in LDS, over which every lane goes
// alike (a parent lies before its node, so a path has no more nodes than
// accept_node + 1).
struct Entries {
    int n;
    bool walked;
};
__device__ __forceinline__ Entries entries_of(const switchsd_logprob_args &a, int b, int from,
                                              uint16_t *parents, uint16_t *path) {
    const int n = a.dn ? clampi(a.dn[b], 1, a.R) : a.R;
    if (!a.accept_node)
        return {n, false};
    const int last = a.accept_node[b];
    if (last < 0 || last >= n || from > last)
        return {0, false};
    if (!a.dpar)
        return {last + 1, false};
    for (int x = threadIdx.x; x <= last; x += kThreads) {
        const int up = a.dpar[(int64_t)b * a.R + x];
        parents[x] = (uint16_t)(up >= 0 && up < x ? up : 0xFFFF);
    }
    __syncthreads();
    int depth = 0;
    for (int x = last; x > 0; ++depth) {
        path[depth] = (uint16_t)x;
        x = parents[x];
        if (x == 0xFFFF)
            return {0, false};
    }
    return {depth + 1, true};
}
__device__ __forceinline__ int row_of(const Entries &n, int i, const uint16_t *path) {
    return !n.walked || i == 0 ? i : path[n.n - 1 - i];
}

// ---- log probabilities

// What a lane (then a wave, then all) has seen of a row: weights 2^((l - ref) c)
// against a reference of its own that follows its largest logit with a delay, their
// sum and the sum of weight times exponent; the largest logit and the vector
// it was first seen in (none while there is no number above -inf).
struct Sums {
    float ref, lim, s, t, mx;
    int vec;
};
// A reference is moved when a weight would pass 2^kDelay (a sum of 2^26 of them is far
// from the largest float).
constexpr float kDelay = 20.0f;
// The exponent that weights and factors stop at: it leaves nothing of a sum (2^46 at most) in
// 32 bits, and an infinite distance, that of a mask of the lowest number, would make NaN of
// what is multiplied with it and then with the weight 0.
constexpr float kNothing = -150.0f;
constexpr float kLargest = 3.402823466e38f;

// The largest of the vector's logits is returned (NaN where all are).
template <int TYPE>
__device__ __forceinline__ float take(Sums &a, u32x4 x, int vec, float c, float delay) {
    constexpr int N = kPerVec<TYPE>;
    float f[N];
#pragma unroll
    for (int e = 0; e < N; ++e)
        f[e] = element<TYPE>(x, e);
    float top = f[0];
#pragma unroll
    for (int e = 1; e < N; ++e)
        top = fmaxf(top, f[e]);
    const bool up = top > a.mx;
    a.mx = up ? top : a.mx;
    a.vec = up ? vec : a.vec;
    if (__any(top > a.lim)) {
        const float ref = fmaxf(a.ref, top);
        const float d = a.ref == -INFINITY ? 0.0f : fmaxf((a.ref - ref) * c, kNothing);
        const float f2 = __builtin_amdgcn_exp2f(d);
        a.t = f2 * (a.t + a.s * d);
        a.s *= f2;
        a.ref = ref;
        a.lim = ref + delay;
    }
    // a vector's own sums first: fewer roundings of the long ones
    float s = 0.0f, t = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        // NaN (and -inf beside itself) weighs nothing: the maximum drops it
        const float y = fmaxf((f[e] - a.ref) * c, kNothing);
        const float w = __builtin_amdgcn_exp2f(y);
        s += w;
        t = fmaf(w, y, t);
    }
    a.s += s;
    a.t += t;
    return top;
}

// How many elements of a wave's vectors are ahead of the given token's logit, in
// vectors before its own (equal ones count) or behind it; its own counts none.  `top`
// are the vectors' largest logits: mostly none of a wave's is that large.
template <int TYPE>
__device__ __forceinline__ int ahead_of(u32x4 x, float top, float lt, int j, int own) {
    int n = 0;
    if (__all(j > own)) {
        if (__any(top > lt))
#pragma unroll
            for (int e = 0; e < kPerVec<TYPE>; ++e)
                n += __popcll(__ballot(element<TYPE>(x, e) > lt));
    } else if (__all(j < own)) {
        if (__any(top >= lt))
#pragma unroll
            for (int e = 0; e < kPerVec<TYPE>; ++e)
                n += __popcll(__ballot(element<TYPE>(x, e) >= lt));
    } else {
#pragma unroll
        for (int e = 0; e < kPerVec<TYPE>; ++e) {
            const float l = element<TYPE>(x, e);
            n += __popcll(__ballot(j < own ? l >= lt : j > own && l > lt));
        }
    }
    return n;
}
// The same of a NaN: every number, and before it every NaN.
template <int TYPE>
__device__ __forceinline__ int ahead_of_nan(u32x4 x, int j, int own) {
    int n = 0;
#pragma unroll
    for (int e = 0; e < kPerVec<TYPE>; ++e) {
        const float l = element<TYPE>(x, e);
        n += __popcll(__ballot(j < own || (j != own && l == l)));
    }
    return n;
}

// Sums against reference `from`, against `to` (not below it).
__device__ __forceinline__ void move(float &s, float &t, float from, float to, float c) {
    const float d = s > 0.0f ? fmaxf((from - to) * c, kNothing) : 0.0f;
    const float f = __builtin_amdgcn_exp2f(d);
    t = f * (t + s * d);
    s *= f;
}

constexpr int kWaves = kThreads / 64;
constexpr int kList = 2048;    // candidates in LDS
constexpr int kGroups = 128;   // pairs of lanes whose largest logits are compared
static_assert(kGroups * 2 == kThreads && SWITCHSD_MAX_TOP <= kGroups, "a group each");

struct Selection {
    unsigned long long firsts[kGroups], list[kList], best[SWITCHSD_MAX_TOP], bar;
    uint16_t winner[kGroups];
    int count, winners, counts[kWaves];
    unsigned long long red[kWaves];
};

// Largest of the lanes' keys.
__device__ __forceinline__ unsigned long long block_max(unsigned long long v,
                                                        unsigned long long *red) {
    for (int d = 32; d; d >>= 1) {
        const unsigned long long o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        red[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w)
        v = red[w] > v ? red[w] : v;
    return v;
}

// The list's k first keys, in order, to best; 0 behind the last.
__device__ __forceinline__ void rank_list(Selection &sel, int count, int k) {
    for (int x = threadIdx.x; x < k; x += kThreads)
        if (x >= count)
            sel.best[x] = 0;
    for (int x = threadIdx.x; x < count; x += kThreads) {
        const unsigned long long mine = sel.list[x];
        int n = 0;
#pragma unroll 4
        for (int y = 0; y < count; ++y)
            n += sel.list[y] > mine ? 1 : 0;
        if (n < k)
            sel.best[n] = mine;
    }
    __syncthreads();
}

// The k first tokens of the row's vectors [j0, j1), in order, to sel.best (0 where
// there are fewer).  The largest logits of 128 pairs of lanes, in sel.firsts, were
// compared: the k-th of them bounds the first tokens from below, and each of
// them lies in one of the k first pairs, so only those pairs' vectors are read again.
template <int TYPE>
__device__ __forceinline__ void select(Selection &sel, const char *row, int V, int j0, int j1,
                                       int k) {
    constexpr int N = kPerVec<TYPE>;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, full = V / N;
    const int v0 = j0 * N, v1 = j1 * N < V ? j1 * N : V;
    {
        const unsigned long long mine = sel.firsts[tid / 2];
        const ulonglong2 *all = (const ulonglong2 *)sel.firsts + tid % 2 * (kGroups / 4);
        int n = 0;
#pragma unroll 8
        for (int g = 0; g < kGroups / 4; ++g) {
            const ulonglong2 o = all[g];
            n += (o.x > mine ? 1 : 0) + (o.y > mine ? 1 : 0);
        }
        n += __shfl_xor(n, 1);
        if (mine && tid % 2 == 0 && n < k) {
            sel.winner[atomicAdd(&sel.winners, 1)] = (uint16_t)(tid / 2);
            if (n == k - 1)
                sel.bar = mine;
        }
    }
    __syncthreads();
    // with fewer than k pairs that hold a number above -inf, every such number is a
    // candidate; else the elements whose (logit, vector) is not behind the k-th's
    const int winners = sel.winners;
    const unsigned long long bar =
        winners < k ? (unsigned long long)(kMinusInf + 1) << 32 : sel.bar;
    // four vectors of a lane are asked for at once
    const uint32_t per = (uint32_t)((j1 - j0 + kThreads - 1) / kThreads) * 2;
    const uint32_t tasks = (uint32_t)winners * per;
    for (uint32_t x0 = 0; x0 < tasks; x0 += 4 * kThreads) {
        u32x4 q[4];
        int at[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t x = x0 + u * kThreads + tid;
            at[u] = -1;
            q[u] = u32x4{~0u, ~0u, ~0u, ~0u};
            if (x < tasks) {
                const uint32_t w = x / per, y = x - w * per;
                const int j = j0 + (int)(y / 2) * kThreads + sel.winner[w] * 2 + (int)(y % 2);
                if (j < j1) {
                    at[u] = j;
                    q[u] = j < full ? load_vec<TYPE>(row, j) : load_last<TYPE>(row, j, V);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (x0 + u * kThreads >= tasks)
                break;
            // of the bar's own logit the vectors up to its own
            const uint32_t least =
                (uint32_t)(bar >> 32) + (0xFFFFFFFFu - (uint32_t)at[u] >= (uint32_t)bar ? 0 : 1);
            unsigned hits = 0;
#pragma unroll
            for (int e = 0; e < N; ++e)
                hits |= order_of(element<TYPE>(q[u], e)) >= least ? 1u << e : 0u;
            if (hits == 0)
                continue;
            int to = atomicAdd(&sel.count, __popc(hits));
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (hits & 1u << e) {
                    if (to < kList)
                        sel.list[to] = order_key(element<TYPE>(q[u], e), at[u] * N + e);
                    ++to;
                }
        }
    }
    __syncthreads();
    int count = sel.count;
    if (count > kList) {
        // more equal or rising candidates than fit: the next one behind the last,
        // k times over the vectors
        unsigned long long last = ~0ull;
        for (int n = 0; n < k; ++n) {
            unsigned long long next = 0;
            for (int v = v0 + tid; v < v1; v += kThreads) {
                const unsigned long long key = order_key(load_logit<TYPE>(row, v), v);
                next = key < last && key > next ? key : next;
            }
            last = block_max(next, sel.red);
            if (tid == 0)
                sel.best[n] = last;
        }
        __syncthreads();
        return;
    }
    // too few numbers: -inf by their index, then NaN by theirs
    for (int what = 0; what < 2 && count < k; ++what) {
        for (int base = v0; base < v1 && count < k; base += kThreads) {
            const int v = base + tid;
            const float l = v < v1 ? load_logit<TYPE>(row, v) : 0.0f;
            const bool hit = v < v1 && (what == 0 ? l == -INFINITY : !(l == l));
            const unsigned long long w = __ballot(hit);
            __syncthreads();
            if (lane == 0)
                sel.counts[wave] = __popcll(w);
            __syncthreads();
            int at = count + __popcll(w & ((1ull << lane) - 1));
            for (int x = 0; x < kWaves; ++x) {
                at += x < wave ? sel.counts[x] : 0;
                count += sel.counts[x];
            }
            if (hit && at < k)
                sel.list[at] = order_key(l, v);
        }
        count = count < k ? count : k;
    }
    __syncthreads();
    rank_list(sel, count, k);
}

// What the pieces of a cut row leave: sums, and the first tokens.
struct Record {
    unsigned long long sums[2];  // (largest, s), (t, ahead)
    unsigned long long best[SWITCHSD_MAX_TOP];
};
static_assert(sizeof(Record) == kLogprobRecord, "size of a piece's record");

__device__ __forceinline__ unsigned long long pair64(float a, uint32_t b) {
    return (unsigned long long)__builtin_bit_cast(uint32_t, a) << 32 | b;
}
__device__ __forceinline__ float high(unsigned long long v) {
    return __builtin_bit_cast(float, (uint32_t)(v >> 32));
}

// Entry (b, i) of the sequence's entries i = s, s + S, ..: a work-group reads a
// row, or with few rows one of `pieces` pieces of it, once; of a cut row the last
// work-group to arrive joins the pieces.  About 13 lane operations an element, the
// exponential among them, which at full rate is what 5 to 6 TB/s of 16-bit logits
// bring: a row is cut rather than left to one compute unit.
//   8 x up to 512 rows of 151936 bf16 logits, one alternative: 233 to 246 us, 4.4 to 4.7 TB/s
// (without ranks 204, 5.3; 8 x up to 256 rows of floats 204).  32 paths of 1 to 9 entries of 128256, 20 alternatives: 29.6 us, of
// which 6.6 for the alternatives and 3.1 for the ranks; the rest is the path, the
// first bytes and the join of the pieces.
template <int TYPE>
__global__ void __launch_bounds__(kThreads, 4) k_logprob(const LogprobParams p) {
    constexpr int N = kPerVec<TYPE>;
    constexpr int U = 4;  // vectors in flight per lane
    const switchsd_logprob_args &a = p.a;
    __shared__ uint16_t parents[SWITCHSD_MAX_R], path[SWITCHSD_MAX_R];
    __shared__ float4 sums[kWaves];
    __shared__ Selection sel;
    __shared__ int s_last;
    const int piece = (int)(blockIdx.x % p.pieces);
    const int64_t of = blockIdx.x / p.pieces;
    // first entries of all sequences before second ones: what paths leave without work
    // lies behind the rest, not on some of the compute units (40.1 -> 37.4 us for 32
    // paths with 8 slots)
    const int b = (int)(of % a.B), s0 = (int)(of / a.B);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Entries all = entries_of(a, b, s0, parents, path);
    const int V = a.V, full = V / N, nv = (V + N - 1) / N, k = p.n_top;
    const int j0 = piece * p.piece_vecs;
    const int j1 = j0 + p.piece_vecs < nv ? j0 + p.piece_vecs : nv;
    const int whole = j1 < full ? j1 : full;
    const float c = p.inv_t * kLog2e, delay = kDelay / c;
    const u32x4 nothing = u32x4{~0u, ~0u, ~0u, ~0u};  // NaN in every type

    for (int i = s0; i < all.n; i += p.slots) {
        const int64_t e = (int64_t)b * a.R + i;
        const char *row = (const char *)a.logits +
                          ((int64_t)b * a.R + row_of(all, i, path)) * V * kSize<TYPE>;
        // the first vectors are asked for before the token, and its logit behind it
        u32x4 x[U];
        const auto ask = [&](int at) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = at + u * kThreads + tid;
                x[u] = nothing;
                if (j < whole)
                    x[u] = load_vec<TYPE>(row, j);
            }
        };
        ask(j0);
        const int tok = a.tokens ? a.tokens[e] : -1;
        const bool in = tok >= 0 && tok < V;
        const int own = tok / N;
        u32x4 beside = nothing;  // the token's vector
        if (in)
            beside = own < full ? load_vec<TYPE>(row, own) : load_last<TYPE>(row, own, V);
        float lt = 0.0f;
#pragma unroll
        for (int x = 0; x < N; ++x)
            lt = in && x == tok % N ? element<TYPE>(beside, x) : lt;
        const bool ranked = p.rank && in;

        __syncthreads();  // the last entry's use of LDS
        if (tid == 0)
            sel.count = sel.winners = 0;
        Sums m = {-INFINITY, -INFINITY, 0.0f, 0.0f, -INFINITY, -1};
        int ahead = 0;
        const auto use = [&](u32x4 x, int j) {
            const float top = take<TYPE>(m, x, j, c, delay);
            if (ranked)
                ahead += lt == lt ? ahead_of<TYPE>(x, top, lt, j, own)
                                  : ahead_of_nan<TYPE>(x, j, own);
        };
        for (int at = j0; at < whole; at += kThreads * U) {
            if (at > j0)
                ask(at);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (at + u * kThreads + wave * 64 < whole) {
                    const int j = at + u * kThreads + tid;
                    use(x[u], j < whole ? j : INT32_MAX);
                }
        }
        if (j1 > full) {
            const int at = (full - j0) % kThreads;  // the lane whose turn it is
            if (at / 64 == wave)
                use(at == tid ? load_last<TYPE>(row, full, V) : nothing,
                    at == tid ? full : INT32_MAX);
        }
        if (ranked && wave == 0 && own >= j0 && own < j1) {  // the token's own vector
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const int v = own * N + x;
                const bool first = order_key(element<TYPE>(beside, x), v) > order_key(lt, tok);
                ahead += v < V && first ? 1 : 0;
            }
        }

        // the wave's sums against its largest logit
        float mx = m.mx;
#pragma unroll
        for (int d = 32; d; d >>= 1)
            mx = fmaxf(mx, __shfl_xor(mx, d));
        move(m.s, m.t, m.ref, mx, c);
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            m.s += __shfl_xor(m.s, d);
            m.t += __shfl_xor(m.t, d);
        }
        if (k > 0) {
            unsigned long long first = m.vec < 0 ? 0 : order_key(m.mx, m.vec);
            const unsigned long long o = __shfl_xor(first, 1);
            first = o > first ? o : first;
            if (tid % 2 == 0)
                sel.firsts[tid / 2] = first;
        }
        if (lane == 0)
            sums[wave] = make_float4(mx, m.s, m.t, __builtin_bit_cast(float, ahead));
        __syncthreads();
        float M = sums[0].x, S = 0.0f, t = 0.0f;
        ahead = 0;
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
            M = fmaxf(M, sums[w].x);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            float4 v = sums[w];
            move(v.y, v.z, v.x, M, c);
            S += v.y;
            t += v.z;
            ahead += __builtin_bit_cast(int, v.w);
        }
        if (k > 0)
            select<TYPE>(sel, row, V, j0, j1, k);

        if (p.pieces > 1) {
            Record *const of_row = (Record *)p.records + e * p.pieces;
            uint32_t *const ticket = p.tickets + e;
            if (wave == 0) {
                Record *mine = of_row + piece;
                if (lane == 0)
                    st_u64(&mine->sums[0], pair64(M, __builtin_bit_cast(uint32_t, S)));
                if (lane == 1)
                    st_u64(&mine->sums[1], pair64(t, (uint32_t)ahead));
                if (lane < k)
                    st_u64(&mine->best[lane], sel.best[lane]);
                const bool last = arrive(ticket, (uint32_t)p.pieces);
                if (lane == 0)
                    s_last = last ? 1 : 0;
            }
            __syncthreads();
            if (!s_last)
                continue;
            if (tid == 0) {
                st_u32(ticket, 0);
                sel.count = 0;
                sel.bar = ~0ull;
            }
            // what the pieces left is asked for together: sums (pieces are few, a lane
            // for each) and the first of the keys
            float pm = -INFINITY, ps = 0.0f, pt = 0.0f;
            ahead = 0;
            unsigned long long keys[2] = {0, 0};
#pragma unroll
            for (int y = 0; y < 2; ++y)
                if (tid + y * kThreads < p.pieces * k)
                    keys[y] = ld_u64(&of_row[(tid + y * kThreads) / k]
                                          .best[(tid + y * kThreads) % k]);
            if (tid < p.pieces) {
                const unsigned long long x = ld_u64(&of_row[tid].sums[0]);
                const unsigned long long y = ld_u64(&of_row[tid].sums[1]);
                pm = high(x);
                ps = __builtin_bit_cast(float, (uint32_t)x);
                pt = high(y);
                ahead = (int)(uint32_t)y;
            }
            mx = pm;
#pragma unroll
            for (int d = 32; d; d >>= 1)
                mx = fmaxf(mx, __shfl_xor(mx, d));
            move(ps, pt, pm, mx, c);
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                ps += __shfl_xor(ps, d);
                pt += __shfl_xor(pt, d);
                ahead += __shfl_xor(ahead, d);
            }
            if (lane == 0)
                sums[wave] = make_float4(mx, ps, pt, __builtin_bit_cast(float, ahead));
            __syncthreads();
            M = sums[0].x;
#pragma unroll
            for (int w = 1; w < kWaves; ++w)
                M = fmaxf(M, sums[w].x);
            S = t = 0.0f;
            ahead = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                float4 v = sums[w];
                move(v.y, v.z, v.x, M, c);
                S += v.y;
                t += v.z;
                ahead += __builtin_bit_cast(int, v.w);
            }
            if (k > 0) {
                // pieces' first ceil(k / pieces) tokens make k together: the last
                // of them bounds the row's
                const int q = (k + p.pieces - 1) / p.pieces - 1, all = p.pieces * k;
                const auto key_of = [&](int x) {
                    return x < kThreads       ? keys[0]
                           : x < 2 * kThreads ? keys[1]
                                              : ld_u64(&of_row[x / k].best[x % k]);
                };
                for (int x = tid; x < all; x += kThreads)
                    if (x % k == q)
                        atomicMin(&sel.bar, key_of(x));
                __syncthreads();
                const unsigned long long bar = sel.bar;
                for (int x = tid; x < all; x += kThreads) {
                    const unsigned long long key = key_of(x);
                    if (key && key >= bar) {
                        const int at = atomicAdd(&sel.count, 1);
                        if (at < kList)
                            sel.list[at] = key;
                    }
                }
                __syncthreads();
                const int count = sel.count;
                if (count <= kList) {
                    rank_list(sel, count, k);
                } else {
                    unsigned long long last = ~0ull;
                    for (int n = 0; n < k; ++n) {
                        unsigned long long next = 0;
                        for (int x = tid; x < p.pieces * k; x += kThreads) {
                            const unsigned long long key = ld_u64(&of_row[x / k].best[x % k]);
                            next = key < last && key > next ? key : next;
                        }
                        last = block_max(next, sel.red);
                        if (tid == 0)
                            sel.best[n] = last;
                    }
                    __syncthreads();
                }
                for (int x = tid; x < p.pieces * k; x += kThreads)
                    st_u64(&of_row[x / k].best[x % k], 0);
            }
            // the workspace is left zeroed
            for (int x = tid; x < p.pieces * 2; x += kThreads)
                st_u64(&of_row[x / 2].sums[x % 2], 0);
        }

        // no finite maximum: all weight on the first one
        const bool flat = !(fabsf(M) < INFINITY);
        const float lnS = flat ? 0.0f : __builtin_amdgcn_logf(S) * kLn2;
        int greedy = 0;
        if (flat) {
            unsigned long long first = 0;
            for (int v = tid; v < V; v += kThreads) {
                const unsigned long long key = order_key(load_logit<TYPE>(row, v), v);
                first = key > first ? key : first;
            }
            greedy = (int)key_index(block_max(first, sel.red));
        }
        const auto logprob = [&](float l, int v) {
            if (flat)
                return v == greedy ? 0.0f : -INFINITY;
            return l == l ? (l - M) * p.inv_t - lnS : -INFINITY;
        };
        if (tid == 0) {
            if (p.rank)
                p.rank[e] = in ? ahead : -1;
            if (p.logprob)
                p.logprob[e] = in ? logprob(lt, tok) : -INFINITY;
            if (p.lse)
                // finite where the maximum is
                p.lse[e] = flat ? M : fminf(fmaxf(M * p.inv_t + lnS, -kLargest), kLargest);
            if (p.entropy)
                p.entropy[e] = flat ? 0.0f : lnS - t / S * kLn2;
        }
        if (tid < k) {
            const unsigned long long key = sel.best[tid];
            const int v = (int)key_index(key);
            if (p.top_ids)
                p.top_ids[e * k + tid] = v;
            if (p.top_logprobs)
                p.top_logprobs[e * k + tid] = logprob(key_logit(key), v);
        }
    }
}

// ---- gradient

// From this |lse| on 32 bits leave too little of the logarithm beside the maximum (2^-15 of p
// below it, up to all of p): the row's sum is taken again.  One of the row's work-groups
// does that and the whole row, since the gradient may take the row's place.  (4 x up to 1024
// rows of 128256 logits at T = 0.001: 1354 us; with the row's first work-group, which is
// always on the same XCD, 6756.)
constexpr float kFar = 1024.0f;

// The maximum of a row and the logarithm of its sum against it.  Every lane of the
// work-group calls it.
template <int TYPE>
__device__ __forceinline__ float2 row_sum(const char *row, int V, float c) {
    constexpr int N = kPerVec<TYPE>;
    __shared__ float red[2][kThreads / 64];
    const int full = V / N, wave = threadIdx.x >> 6;
    float m = -INFINITY, s = 0.0f;
#pragma unroll 4
    for (int j = threadIdx.x; j <= full; j += kThreads) {
        const u32x4 x = j < full ? load_vec<TYPE>(row, j) : load_last<TYPE>(row, j, V);
#pragma unroll
        for (int e = 0; e < N; ++e)
            m = fmaxf(m, element<TYPE>(x, e));
    }
    for (int d = 32; d; d >>= 1)
        m = fmaxf(m, __shfl_xor(m, d));
    red[0][wave] = m;
    __syncthreads();
    for (int w = 0; w < kThreads / 64; ++w)
        m = fmaxf(m, red[0][w]);
#pragma unroll 4
    for (int j = threadIdx.x; j <= full; j += kThreads) {
        const u32x4 x = j < full ? load_vec<TYPE>(row, j) : load_last<TYPE>(row, j, V);
#pragma unroll
        for (int e = 0; e < N; ++e)
            s += __builtin_amdgcn_exp2f(fmaxf((element<TYPE>(x, e) - m) * c, kNothing));
    }
    for (int d = 32; d; d >>= 1)
        s += __shfl_xor(s, d);
    red[1][wave] = s;
    __syncthreads();
    s = 0.0f;
    for (int w = 0; w < kThreads / 64; ++w)
        s += red[1][w];
    return make_float2(m, __builtin_amdgcn_logf(s) * kLn2);
}

// A work-group per entry and piece of its row: one read, one write, bound by the memory.
// 4 x up to 1024 rows of 128256 bf16 logits: 332 to 348 us, 5.3 to 5.5 TB/s; 23 rows of 50257
// floats 4.8; along 32 paths, most of whose work-groups have no entry, 28.
constexpr int kGradVecs = 4;  // vectors of a lane
template <int TYPE>
__global__ void __launch_bounds__(kThreads) k_logprob_grad(const LogprobParams p, int pieces) {
    constexpr int N = kPerVec<TYPE>;
    const switchsd_logprob_args &a = p.a;
    __shared__ uint16_t parents[SWITCHSD_MAX_R], path[SWITCHSD_MAX_R];
    const int64_t e = blockIdx.x / pieces;
    const int piece = (int)(blockIdx.x - e * pieces);
    const int b = (int)(e / a.R), i = (int)(e % a.R);
    const Entries all = entries_of(a, b, i, parents, path);
    if (i >= all.n)
        return;
    const int V = a.V, full = V / N;
    const int64_t at = ((int64_t)b * a.R + row_of(all, i, path)) * V * kSize<TYPE>;
    const char *row = (const char *)a.logits + at;
    char *out = (char *)p.grad + at;
    const float lse = p.in_lse[e];
    const float g = p.g_logprob ? p.g_logprob[e] : 0.0f;
    const float ge = p.g_entropy ? p.g_entropy[e] : 0.0f;
    const float H = p.g_entropy ? p.in_entropy[e] : 0.0f;
    const int tok = p.g_logprob ? a.tokens[e] : -1;
    const bool flat = !(fabsf(lse) < INFINITY);
    // log p = (l - base) / T - low
    const auto slope_of = [&](float l, int v, float base, float low) {
        // NaN and -inf weigh nothing: the maximum drops them
        const float x = fmaxf(fmaf(l - base, p.inv_t, -low), -150.0f);
        const float w = l == l ? __builtin_amdgcn_exp2f(x * kLog2e) : 0.0f;
        const float d = (v == tok ? g : 0.0f) - w * fmaf(ge, x + H, g);
        return flat ? 0.0f : d * p.inv_t;
    };
    if (!flat && fabsf(lse) >= kFar) {
        if (piece != (int)(e % pieces))  // not always the same XCD's
            return;
        const float2 s = row_sum<TYPE>(row, V, p.inv_t * kLog2e);
#pragma unroll 8
        for (int v = threadIdx.x; v < V; v += kThreads)
            store_logit<TYPE>(out, v, slope_of(load_logit<TYPE>(row, v), v, s.x, s.y));
        return;
    }
    const auto slope = [&](float l, int v) { return slope_of(l, v, 0.0f, lse); };
    const int j0 = piece * (kThreads * kGradVecs) + threadIdx.x;
    u32x4 x[kGradVecs];
#pragma unroll
    for (int u = 0; u < kGradVecs; ++u)
        if (j0 + u * kThreads < full)
            x[u] = load_vec<TYPE>(row, j0 + u * kThreads);
#pragma unroll
    for (int u = 0; u < kGradVecs; ++u) {
        const int j = j0 + u * kThreads;
        if (j < full) {
            u32x4 y;
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float d = slope(element<TYPE>(x[u], q), j * N + q);
                if (TYPE == SWITCHSD_F32) {
                    y[q] = __builtin_bit_cast(uint32_t, d);
                } else {
                    const uint16_t h = TYPE == SWITCHSD_BF16
                                           ? __builtin_bit_cast(uint16_t, (__bf16)d)
                                           : __builtin_bit_cast(uint16_t, (_Float16)d);
                    y[q / 2] = q % 2 ? y[q / 2] | (uint32_t)h << 16 : h;
                }
            }
            if (TYPE == SWITCHSD_F32)
                *(u32x4_a4 *)(out + (int64_t)j * 16) = y;
            else
                *(u32x4_a2 *)(out + (int64_t)j * 16) = y;
        } else if (j == full) {
            for (int v = full * N; v < V; ++v)
                store_logit<TYPE>(out, v, slope(load_logit<TYPE>(row, v), v));
        }
    }
}

int launched() { return hipGetLastError() == hipSuccess ? SWITCHSD_OK : SWITCHSD_EHIP; }

template <int TYPE>
int launch_logprob(LogprobParams p, hipStream_t stream) {
    p.slots = logprob_slots(p.a);
    const LogprobCut cut = logprob_cut(p.a, p.records != nullptr);
    p.pieces = cut.pieces;
    p.piece_vecs = cut.vecs;
    const int64_t groups = (int64_t)p.a.B * p.slots * p.pieces;
    hipLaunchKernelGGL((k_logprob<TYPE>), dim3((unsigned)groups), dim3(kThreads), 0, stream, p);
    return launched();
}

template <int TYPE>
int launch_grad(const LogprobParams &p, hipStream_t stream) {
    const int64_t piece = (int64_t)kThreads * kGradVecs * kPerVec<TYPE>;
    const int64_t pieces = (p.a.V + piece) / piece;  // with a place behind the last whole vector
    const int64_t groups = (int64_t)p.a.B * p.a.R * pieces;
    if (groups >= 1 << 24)
        return SWITCHSD_ESHAPE;
    hipLaunchKernelGGL((k_logprob_grad<TYPE>), dim3((unsigned)groups), dim3(kThreads), 0, stream, p,
                       (int)pieces);
    return launched();
}

}  // namespace

int launch_logprob_kernel(const LogprobParams &p, hipStream_t stream) {
    return p.a.logits_type == SWITCHSD_BF16  ? launch_logprob<SWITCHSD_BF16>(p, stream)
           : p.a.logits_type == SWITCHSD_F16 ? launch_logprob<SWITCHSD_F16>(p, stream)
                                             : launch_logprob<SWITCHSD_F32>(p, stream);
}

int launch_logprob_grad_kernel(const LogprobParams &p, hipStream_t stream) {
    return p.a.logits_type == SWITCHSD_BF16  ? launch_grad<SWITCHSD_BF16>(p, stream)
           : p.a.logits_type == SWITCHSD_F16 ? launch_grad<SWITCHSD_F16>(p, stream)
                                             : launch_grad<SWITCHSD_F32>(p, stream);
}

}  // namespace switchsd
