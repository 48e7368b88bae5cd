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

// A lane per 16 bytes of a row's keys or values, so that loads and stores are whole
// vectors whatever the slots' order.  Moves 4 Hkv D bytes in and as many (or half)
// out: bound by its launch for the rows of a step (256 rows of 8 heads of 128: 2.8 us),
// by the memory for prompts (16 of up to 2048 tokens, 8 heads of 64: 19.1 us, 5.3 TB/s;
// of 128: 31.5 us, into 8 bits 38.3, for the division).
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
//
// For a query row q and the keys k_j that it sees, s_j = scale q . k_j, the output is
// sum_j e^(s_j - m) v_j / sum_j e^(s_j - m) for any m: one pass over the keys with a
// running m, the sums multiplied by e^(m - m') when it moves.  All query heads of a head of
// the cache and all new tokens are rows of one matrix, so that a key is read once for
// all of them.  S^T = K Q^T and O^T = V^T P^T: a column of the products is a query
// row, so a lane holds (half of) one row's weights, which are the second product's
// operand as they stand.  Few rows (k_attend_few) are bound by the bytes of the
// cache, many (k_attend_many) by the exponentials and the matrix instructions.

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

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

// The work of a launch, cut on the device: items are (sequence, tile of query
// rows, head of the cache), an item's keys are cut into units, and what a
// work-group takes is found by the sums over all sequences of what comes before it.
// With many items each work-group takes one whole; with few, up to kAttnGroups
// work-groups take equal shares of all units, in order, and k_merge joins what
// was cut.  The host has seen to it that items, and with few of them units, fit 32
// bits.
struct Work {
    uint32_t items, units;  // of all sequences
    int whole;              // one item for each work-group
    uint32_t groups;        // work-groups that have work
};

// What sequence b has: its new rows, keys that there may be (positions of pages that are
// held), tiles of query rows and units of keys (1 at least, so that every row is
// written).  Where the new rows are a good part of the keys and there is no mask, a later
// tile sees more keys: every G tiles, which are TILE tokens, have TILE / UNIT units more
// than the G before them, so that shares of units are shares of work.  (8 prompts in
// chunks of up to 3250 tokens in contexts of 6900, 4 + 1 heads of 128: 140 us; with the
// same units for all tiles 158.)
struct Seq {
    Chunk c;
    int keys, tiles, units, grow;
};
template <int TILE, int UNIT>
__device__ __forceinline__ uint32_t units_of(const AttnParams &p, const Seq &s, int tile) {
    return (uint32_t)(s.units + (TILE > UNIT && s.grow ? s.grow * (tile / p.G) : 0));
}
// Units of the first t tiles, all heads of them.
template <int TILE, int UNIT>
__device__ __forceinline__ uint32_t units_before(const AttnParams &p, const Seq &s, int t) {
    uint32_t n = (uint32_t)t * (uint32_t)s.units;
    if (TILE > UNIT && s.grow) {
        const int k = t / p.G;
        n += (uint32_t)s.grow * ((uint32_t)p.G * ((uint32_t)k * (uint32_t)(k - 1) / 2) +
                                 (uint32_t)(t - k * p.G) * (uint32_t)k);
    }
    return n * (uint32_t)p.a.Hkv;
}
template <int TILE, int UNIT>
__device__ __forceinline__ Seq seq_of(const AttnParams &p, int b) {
    Seq s;
    s.c = chunk_of(p.a, b);
    const int held = clampi(p.a.held[b], 0, p.a.max_pages);
    const int64_t end = (int64_t)s.c.pos + s.c.n, most = (int64_t)held * p.a.page_size;
    s.keys = p.n_slots == 0 ? 0 : (int)(end < most ? end : most);
    s.tiles = (int)(((int64_t)s.c.n * p.G + TILE - 1) / TILE);
    s.units = s.keys > UNIT ? (s.keys + UNIT - 1) / UNIT : 1;
    s.grow = 0;
    // (units are bounded by the pages that there can be, so not where positions have none)
    if (TILE > UNIT && !p.a.mask && s.tiles > p.G && s.c.n > s.keys / 4 && end <= most) {
        s.grow = TILE / UNIT;
        s.units = (s.c.pos + UNIT - 1) / UNIT + s.grow;
    }
    return s;
}

struct PlanShared {
    uint32_t sums[2][kThreads / 64];
    uint32_t off, base;
    int b;
    Seq seq;
};

// A lane's share of the sequences, with what comes before them.
struct Plan {
    Work w;
    int b0, b1;
    Seq seq;                // of b0, where it is the only one
    uint32_t items, units;  // of its sequences
    uint32_t items_before, units_before;
};

template <int TILE, int UNIT>
__device__ __forceinline__ Plan plan(const AttnParams &p, PlanShared &sh) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (p.a.B + kThreads - 1) / kThreads;
    Plan q;
    q.b0 = tid * per < p.a.B ? tid * per : p.a.B;
    q.b1 = q.b0 + per < p.a.B ? q.b0 + per : p.a.B;
    q.items = q.units = 0;
    for (int b = q.b0; b < q.b1; ++b) {
        q.seq = seq_of<TILE, UNIT>(p, b);
        q.items += (uint32_t)(q.seq.tiles * p.a.Hkv);
        q.units += units_before<TILE, UNIT>(p, q.seq, q.seq.tiles);
    }
    uint32_t pi = (uint32_t)wave_scan((int)q.items), pu = (uint32_t)wave_scan((int)q.units);
    if (lane == 63) {
        sh.sums[0][wave] = pi;
        sh.sums[1][wave] = pu;
    }
    __syncthreads();
    uint32_t items = 0, units = 0;
#pragma unroll
    for (int v = 0; v < kThreads / 64; ++v) {
        pi += v < wave ? sh.sums[0][v] : 0;
        pu += v < wave ? sh.sums[1][v] : 0;
        items += sh.sums[0][v];
        units += sh.sums[1][v];
    }
    q.items_before = pi - q.items;
    q.units_before = pu - q.units;
    // the same in every lane, which the compiler is told so that what follows from it
    // stays in scalar registers
    q.w.items = __builtin_amdgcn_readfirstlane(items);
    q.w.units = __builtin_amdgcn_readfirstlane(units);
    q.w.whole = p.whole || q.w.items >= attention_whole(TILE);
    const uint32_t most = q.w.units / kAttnLeast;
    const uint32_t limit = (uint32_t)p.groups;
    q.w.groups = q.w.whole ? q.w.items : most < 1 ? 1 : most < limit ? most : limit;
    return q;
}

// The first unit of work-group g: floor(g U / W); the work-group that unit u is in: the
// last g with g U / W < u + 1.
__device__ __forceinline__ uint32_t start_of(const Work &w, uint32_t g) {
    if (w.units < (1u << 22))  // g and W are at most kAttnGroups
        return g * w.units / w.groups;
    return (uint32_t)((uint64_t)g * w.units / w.groups);
}
__device__ __forceinline__ uint32_t group_of(const Work &w, uint32_t u) {
    if (w.units < (1u << 22))
        return ((u + 1) * w.groups - 1) / w.units;
    return (uint32_t)((((uint64_t)u + 1) * w.groups - 1) / w.units);
}

__device__ __forceinline__ Seq uniform(const Seq &x) {
    Seq s;
    s.c.n = __builtin_amdgcn_readfirstlane(x.c.n);
    s.c.row = __builtin_amdgcn_readfirstlane(x.c.row);
    s.c.pos = __builtin_amdgcn_readfirstlane(x.c.pos);
    s.keys = __builtin_amdgcn_readfirstlane(x.keys);
    s.tiles = __builtin_amdgcn_readfirstlane(x.tiles);
    s.units = __builtin_amdgcn_readfirstlane(x.units);
    s.grow = __builtin_amdgcn_readfirstlane(x.grow);
    return s;
}

// The sequence that item (or unit) `at` lies in, how many come before it there, and
// the units before the sequence.  Every lane of the work-group calls it.
template <int TILE, int UNIT>
__device__ __forceinline__ int find(const AttnParams &p, const Plan &q, bool by_item, uint32_t at,
                                    PlanShared &sh, Seq &seq, uint32_t &off, uint32_t &base) {
    __syncthreads();
    uint32_t before = by_item ? q.items_before : q.units_before;
    if (at >= before && at - before < (by_item ? q.items : q.units)) {
        uint32_t units = q.units_before;
        for (int b = q.b0; b < q.b1; ++b) {
            const Seq s = q.b1 - q.b0 == 1 ? q.seq : seq_of<TILE, UNIT>(p, b);
            const uint32_t all = units_before<TILE, UNIT>(p, s, s.tiles);
            const uint32_t n = by_item ? (uint32_t)(s.tiles * p.a.Hkv) : all;
            if (at - before < n) {
                sh.b = b;
                sh.off = at - before;
                sh.base = units;
                sh.seq = s;
                break;
            }
            before += n;
            units += all;
        }
    }
    __syncthreads();
    off = __builtin_amdgcn_readfirstlane(sh.off);
    base = __builtin_amdgcn_readfirstlane(sh.base);
    seq = uniform(sh.seq);
    return __builtin_amdgcn_readfirstlane(sh.b);
}

// A work-group's way through its units: pieces of items, one after another.
struct Walk {
    int b;
    Seq seq;
    uint32_t off;       // of the sequence's items (units)
    uint32_t u, end;
    int item, ua, ub;   // the present piece: units [ua, ub) of the item
    bool whole, done;   // one item for each work-group; the piece is a whole item
};
template <int TILE, int UNIT>
__device__ __forceinline__ bool begin(const AttnParams &p, PlanShared &sh, Walk &k) {
    const Plan q = plan<TILE, UNIT>(p, sh);
    if (blockIdx.x >= q.w.groups || q.w.items == 0)
        return false;
    k.u = q.w.whole ? 0 : start_of(q.w, blockIdx.x);
    k.end = q.w.whole ? 1 : start_of(q.w, blockIdx.x + 1);
    uint32_t base;
    k.b = find<TILE, UNIT>(p, q, q.w.whole, q.w.whole ? blockIdx.x : k.u, sh, k.seq, k.off, base);
    k.whole = q.w.whole;
    return true;
}
template <int TILE, int UNIT>
__device__ __forceinline__ void piece(const AttnParams &p, Walk &k) {
    const uint32_t left = k.end - k.u;
    if (k.whole) {
        k.item = (int)k.off;
        k.ua = 0;
        k.ub = (int)units_of<TILE, UNIT>(p, k.seq, k.seq.tiles - 1);
        k.done = true;
        return;
    }
    uint32_t off = k.off, nu = (uint32_t)k.seq.units;
    int tiles = 0;
    if (TILE > UNIT && k.seq.grow) {
        // the G tiles with the same units that it lies in: the last ones that no more than
        // `off` units come before
        int lo = 0, hi = (k.seq.tiles - 1) / p.G;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (units_before<TILE, UNIT>(p, k.seq, mid * p.G) <= off)
                lo = mid;
            else
                hi = mid - 1;
        }
        tiles = lo * p.G;
        off -= units_before<TILE, UNIT>(p, k.seq, tiles);
        nu = units_of<TILE, UNIT>(p, k.seq, tiles);
    }
    k.item = tiles * p.a.Hkv + (int)(off / nu);
    k.ua = (int)(off % nu);
    k.ub = left < nu - (uint32_t)k.ua ? k.ua + (int)left : (int)nu;
    k.done = k.ua == 0 && k.ub == (int)nu;
}
template <int TILE, int UNIT>
__device__ __forceinline__ bool next(const AttnParams &p, Walk &k) {
    const uint32_t n = (uint32_t)(k.ub - k.ua);
    if (k.whole)
        return false;
    k.u += n;
    k.off += n;
    if (k.u >= k.end)
        return false;
    while (k.off == units_before<TILE, UNIT>(p, k.seq, k.seq.tiles)) {
        k.off = 0;
        k.seq = uniform(seq_of<TILE, UNIT>(p, ++k.b));  // there are units left
    }
    return true;
}

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int TYPE>
__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    if (TYPE == SWITCHSD_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const f32x2 v = {a, b};
    if (TYPE == SWITCHSD_BF16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

// Sixteen 8-bit floats as two vectors of 16-bit ones, which hold them exactly.
template <int TYPE>
__device__ __forceinline__ void widen(u32x4 x, u32x4 &lo, u32x4 &hi) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (TYPE == SWITCHSD_BF16) {
            w[j * 2] = __builtin_bit_cast(
                uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[j], 1.0f, false));
            w[j * 2 + 1] = __builtin_bit_cast(
                uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[j], 1.0f, true));
        } else {
            w[j * 2] = __builtin_bit_cast(
                uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[j], 1.0f, false));
            w[j * 2 + 1] = __builtin_bit_cast(
                uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[j], 1.0f, true));
        }
    }
    lo = u32x4{w[0], w[1], w[2], w[3]};
    hi = u32x4{w[4], w[5], w[6], w[7]};
}

// Sets the infinities and NaN among eight 16-bit elements to 0; whether there
// were any.
template <int TYPE>
__device__ __forceinline__ bool clear_not_finite(u32x4 &x) {
    const uint32_t e = TYPE == SWITCHSD_BF16 ? 0x7F80u : 0x7C00u;
    bool bad = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool lo = (x[j] & e) == e, hi = (x[j] >> 16 & e) == e;
        x[j] &= (lo ? 0xFFFF0000u : ~0u) & (hi ? 0xFFFFu : ~0u);
        bad |= lo || hi;
    }
    return bad;
}

// An LDS address as the 32 bits that it is.
__device__ __forceinline__ uint32_t lds_offset(const char *at) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)at;
}

// Four 16-bit elements of one column of an LDS tile of rows: of every 16 lanes,
// lane x names the 8 bytes at row x / 4, columns 4 (x % 4) .., and gets the four
// rows of column x.
__device__ __forceinline__ uint2 read_transposed(uint32_t at) {
    typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
    return __builtin_bit_cast(uint2,
                              __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)at));
}

// The kernel's parameters, read from memory again: what was read of them before is not kept
// for what follows.  Left alone the compiler reads all of them at the start and, with
// too few scalar registers for them, carries them in lanes of vector registers through
// everything (as it still does with others of the scalars: 167 for 128-wide heads in the
// form for many, some ten of them moved back in front of every tile's products).
__device__ __forceinline__ const AttnParams &reread() {
    uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(const AttnParams *)(const __attribute__((address_space(4))) AttnParams *)at;
}

// What a lane holds of one query row (its column of the products).
struct Row {
    int64_t row;  // in q and out
    int i, head;  // new token of the sequence, query head
    bool ok;
};
__device__ __forceinline__ Row row_of(const AttnParams &p, const Chunk &c, int h, int m) {
    Row r;
    r.i = m / p.G;
    r.head = h * p.G + m % p.G;
    r.ok = r.i < c.n;
    r.row = (int64_t)c.row + r.i;
    return r;
}

// The query rows as the products' right operand: lane l holds row l % 32, and of
// step kk the 8 elements that the keys' operand has there.
template <bool E4M3, int D>
__device__ __forceinline__ void load_query(const AttnParams &p, const Row &r,
                                           u32x4 (&q)[D / 16]) {
    const int half = (threadIdx.x >> 5) & 1;
    const char *src = (const char *)p.q + (r.row * p.q_stride + (int64_t)r.head * D) * 2;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
        const int d = E4M3 ? kk / 2 * 32 + half * 16 + kk % 2 * 8 : kk * 16 + half * 8;
        q[kk] = r.ok ? *(const u32x4 *)(src + d * 2) : u32x4{0, 0, 0, 0};
    }
}

// The softmax's factor, as what brings products to powers of two: a magnitude that they
// are multiplied with once the maximum is known, and a sign (or 0, with the magnitude
// 1) that the query rows take, so that what is not seen can be -inf before it.
// NaN is a sign too: the rows become NaN (0x7FFF in both types), and what is not seen stays
// -inf.  (Each case has a loop of its own: with one formula for all, 256-wide heads in the
// form for many spill 59 registers instead of 37, 8 chunks of up to 1024 tokens over 4096
// take 1586 us instead of 1224.)
struct Factor {
    float size, sign;
};
__device__ __forceinline__ Factor factor_of(const AttnParams &p, int h) {
    const float f = p.a.scale * kLog2e * (p.k_scale ? p.k_scale[h] : 1.0f);
    return {f == 0.0f || f != f ? 1.0f : fabsf(f),
            f == 0.0f || f != f ? f : f < 0.0f ? -1.0f : 1.0f};
}
template <int N>
__device__ __forceinline__ void apply_sign(u32x4 (&q)[N], float sign) {
    if (sign == 1.0f)  // the same for all lanes; the rows are not waited for
        return;
    if (sign == -1.0f) {
#pragma unroll
        for (int x = 0; x < N; ++x)
            q[x] ^= 0x80008000u;
        return;
    }
    const uint32_t fill = sign == 0.0f ? 0u : 0x7FFF7FFFu;
#pragma unroll
    for (int x = 0; x < N; ++x)
        q[x] = u32x4{fill, fill, fill, fill};
}

// Which of the 32 cache positions from kb on row r sees, of those in `valid`.
__device__ __forceinline__ uint32_t seen_bits(const AttnParams &p, const Chunk &c, const Row &r,
                                              int kb, uint32_t valid) {
    const int j0 = kb - c.pos;  // the first one's place among the new
    uint32_t bits;
    if (!p.a.mask) {
        const int cnt = r.i - j0 + 1;
        bits = cnt >= 32 ? ~0u : cnt > 0 ? (1u << cnt) - 1 : 0u;
    } else {
        const int words = (p.a.R + 31) / 32;
        const uint32_t *row = p.a.mask + r.row * words;
        bits = j0 <= -32 ? ~0u : 0u;
        if (r.ok && j0 > -32) {
            const int w = j0 >= 0 ? j0 / 32 : -1, sh = j0 & 31;
            const uint32_t lo = w < 0 ? ~0u : w < words ? row[w] : 0u;
            const uint32_t hi = sh && w + 1 < words ? row[w + 1] : 0u;
            bits = sh ? lo >> sh | hi << (32 - sh) : lo;
        }
    }
    return r.ok ? bits & valid : 0u;
}

// Products of the keys that the lane's row does not see.
__device__ __forceinline__ void hide(f32x16 &s, uint32_t seen) {
    seen >>= (threadIdx.x >> 5 & 1) * 4;
#pragma unroll
    for (int e = 0; e < 16; ++e)
        s[e] = seen & 1u << (e / 4 * 8 + e % 4) ? s[e] : -INFINITY;
}

// Running softmax of one query row per lane (both halves of a wave hold the same
// rows, each the keys that its half of the products has): m is what the weights are taken
// against, in powers of two: the maximum less kLift, followed with a delay of up to kDelay, so
// that weights go up to 2^(kLift + kDelay).  fp16 ends at 2^16 and has its smallest step at
// 2^-24: the lift keeps small weights, of which there can be many, out of the range where
// their rounding is a good part of them (bf16 has no such range).  (Sums in 32 bits have
// room for them; a row's sums are multiplied a few times in all, not in every other tile.)
template <int TYPE>
constexpr float kLift = TYPE == SWITCHSD_F16 ? 7.0f : 0.0f;
constexpr float kDelay = 8.0f;

__device__ __forceinline__ float other_half(float v) {
    const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v),
                                                    __builtin_bit_cast(uint32_t, v), false, false);
    return __builtin_bit_cast(float, (uint32_t)(threadIdx.x & 32 ? s[0] : s[1]));
}

// The largest of the lane's row's products of 32 N keys, in powers of two, less kLift; moves m
// where it has to, and returns what the sums so far have to be multiplied with (1:
// nothing).
template <int TYPE, int N>
__device__ __forceinline__ float follow(const f32x16 (&s)[N], float factor, float &m, float &l) {
    float top = s[0][0];
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            top = fmaxf(top, s[x][e]);
    top = fmaxf(top, other_half(top)) * factor - kLift<TYPE>;
    float alpha = 1.0f;
    if (__any(top > m + kDelay || (m == -INFINITY && top > m))) {
        const float mn = fmaxf(m, top);
        alpha = m == mn ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= alpha;
    }
    return alpha;
}
// Products -> weights, in 32 bits in s, summed to l; the weights in 16 bits as the
// right operand of 2 N products with 16 keys each.  That rounding is the price of the
// matrix instructions, whose operands are both of the values' type: at most half a step of
// a weight, 2^-8 of it (bf16), or of fp16 2^-11 of it or 2^-32 of the largest weight,
// whichever is more; less for a sum of many.  The sum of the weights is that of the
// unrounded ones.
template <int TYPE, int N>
__device__ __forceinline__ void weigh(f32x16 (&s)[N], float factor, float m, float &l,
                                      u32x4 (&w)[2 * N]) {
    const float base = m == -INFINITY ? 0.0f : m;
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float a = __builtin_amdgcn_exp2f(fmaf(s[x][e], factor, -base));
            const float b = __builtin_amdgcn_exp2f(fmaf(s[x][e + 1], factor, -base));
            sum[0] += a;
            sum[1] += b;
            w[x * 2 + e / 8][e % 8 / 2] = pack2<TYPE>(a, b);
        }
    l += sum[0] + sum[1];
}

// Infinities and NaN among the values of 32 positions that not every row sees were
// taken as 0, since a weight of 0 would carry them to the rows that do not see
// them.  Here they reach the rows that do: whatever the weight, the sum becomes
// what it is with the value itself.
template <int TYPE, bool E4M3, int D>
__device__ __forceinline__ void add_not_finite(const AttnParams &p, int h, int slot,
                                               uint32_t seen, f32x16 (&o)[D / 32]) {
    const int half = (threadIdx.x >> 5) & 1;
    for (int x = 0; x < 32; ++x) {
        const int s = __shfl(slot, x);
        if (s < 0)
            continue;
        const bool on = seen >> x & 1;
        const int64_t at = ((int64_t)s * p.a.Hkv + h) * D + half * 4;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // a rare path: one value at a time, for few registers
                    __builtin_amdgcn_sched_barrier(0);
                    const float v = cached<TYPE, E4M3>(p.v_cache, at + dt * 32 + g * 8 + e);
                    if (on && !(fabsf(v) < INFINITY))
                        o[dt][g * 4 + e] += v;
                }
    }
}

// O^T += V^T P^T of 32 N keys whose values stand in LDS, a row each `pitch` bytes.
// The fragments of the next 16 keys (and 128 columns) are asked for before the
// present ones are multiplied: left alone the compiler waits for each.
template <int TYPE, int D, int N>
__device__ __forceinline__ void add_values(const u32x4 (&w)[2 * N], const char *values, int pitch,
                                           f32x16 (&o)[D / 32]) {
    constexpr int F = D / 32 < 4 ? D / 32 : 4, PARTS = D / 32 / F, STEPS = 2 * N * PARTS;
    const int lane = threadIdx.x & 63, x = lane & 15;
    // the lane's 8 bytes: keys 4 (lane / 32) + x / 4, columns 16 (lane / 16 % 2) + 4 (x % 4)
    const uint32_t at = lds_offset(values) + ((lane >> 5) * 4 + x / 4) * pitch +
                        ((lane >> 4 & 1) * 16 + x % 4 * 4) * 2;
    u32x4 f[2][F];
    const auto ask = [&](int step, u32x4 (&to)[F]) {
        const uint32_t from = at + step / PARTS * 16 * pitch + step % PARTS * (F * 64);
#pragma unroll
        for (int d = 0; d < F; ++d) {
            const uint2 a = read_transposed(from + d * 64);
            const uint2 b = read_transposed(from + 8 * pitch + d * 64);
            to[d] = u32x4{a.x, a.y, b.x, b.y};
        }
    };
    ask(0, f[0]);
#pragma unroll
    for (int step = 0; step < STEPS; ++step) {
        if (step + 1 < STEPS)
            ask(step + 1, f[(step + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < F; ++d)
            o[step % PARTS * F + d] =
                mfma<TYPE>(f[step & 1][d], w[step / PARTS], o[step % PARTS * F + d]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <int D>
__device__ __forceinline__ void scale_rows(f32x16 (&o)[D / 32], float f) {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
        o[dt] *= f;
}

// Where a result goes: out and lse, or the work-group's place among the partial ones.
template <int TYPE, int D, int TILE>
__device__ __forceinline__ void put(const AttnParams &p, const Row &r, int h, int tile_row,
                                    int64_t place, int dt, const f32x16 &o, float m, float l) {
    const int half = (threadIdx.x >> 5) & 1;
    if (!r.ok)
        return;
    if (place >= 0) {
        float *part = p.part + place * (TILE * (D + 2));
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(f32x4 *)(part + tile_row * D + dt * 32 + g * 8 + half * 4) =
                f32x4{o[g * 4], o[g * 4 + 1], o[g * 4 + 2], o[g * 4 + 3]};
        if (dt == 0 && half == 0) {
            part[TILE * D + tile_row] = m;
            part[TILE * D + TILE + tile_row] = l;
        }
        return;
    }
    const float sv = p.v_scale ? p.v_scale[h] : 1.0f;
    const float f = l == 0.0f ? 0.0f : sv / l;
    char *out = (char *)p.out + (r.row * p.a.Hq + r.head) * (D * 2);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        uint2 v;
        v.x = pack2<TYPE>(o[g * 4] * f, o[g * 4 + 1] * f);
        v.y = pack2<TYPE>(o[g * 4 + 2] * f, o[g * 4 + 3] * f);
        if (l == 0.0f)
            v = make_uint2(0, 0);
        *(uint2 *)(out + (dt * 32 + g * 8 + half * 4) * 2) = v;
    }
    if (p.lse && dt == 0 && half == 0)
        p.lse[r.row * p.a.Hq + r.head] =
            l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// The cache offset (in slots) of position pos; < 0 where there is no key.  The table's
// entry is asked for by itself, so that the wait for it can come later.
__device__ __forceinline__ int page_of(const AttnParams &p, int pos) {
    return p.page_log >= 0 ? pos >> p.page_log : pos / p.a.page_size;
}
__device__ __forceinline__ int entry_of(const AttnParams &p, const int32_t *table, int pos,
                                        int keys) {
    return pos < keys ? table[page_of(p, pos)] : -1;
}
__device__ __forceinline__ int slot_in(const AttnParams &p, int entry, int pos, int keys) {
    const int64_t slot = (int64_t)entry * p.a.page_size + (pos - page_of(p, pos) * p.a.page_size);
    return pos < keys && entry >= 0 && slot < p.n_slots ? (int)slot : -1;
}
__device__ __forceinline__ int slot_of(const AttnParams &p, const int32_t *table, int pos,
                                       int keys) {
    return slot_in(p, entry_of(p, table, pos, keys), pos, keys);
}

// Up to 32 query rows (all new tokens and query heads of one head of the
// cache): the four waves take 32 keys each of every unit of 128, keys straight
// into the registers that the products read, values through a part of LDS of
// their own, so that no wave waits for another before the end.  The next unit's keys
// and values are on their way while the present one's are multiplied; the page table's
// entries are read two units ahead, since loads come back in order.
//   32 x 8 rows (32 + 8 heads of 128, bf16) over up to 4096 keys: 91 us, 4.3 TB/s, and
// 8 of k_merge (8-bit keys: 58 together); 96 x 32 heads, one token, over 3682: 219 us, 4.9 TB/s; the first keys
// arrive some 10 us after the launch.  One token over 512 keys: 12.4 us, a chain of
// plan, page table, first keys and the join of four waves.
template <int TYPE, bool E4M3, int D>
__global__ void __launch_bounds__(kThreads, D <= 128 ? 2 : 1) k_attend_few(const AttnParams) {
    constexpr int TILE = 32, UNIT = 128;
    constexpr int CH = E4M3 ? D / 32 : D / 16;  // 16-byte pieces of a row per half wave
    constexpr int PITCH = D * 2 + 32;
    constexpr int COLS = D / 32 < 4 ? D / 32 : 4;  // blocks of 32 columns joined at once
    constexpr int kVBytes = 4 * 32 * PITCH, kOBytes = 4 * COLS * 4 * 64 * 16;
    __shared__ __attribute__((aligned(16))) char lds[kVBytes > kOBytes ? kVBytes : kOBytes];
    __shared__ float sm[4][TILE], sl[4][TILE];
    // wide rows of the query stand in LDS, which all waves read them from: in registers
    // they leave too few for keys and values on their way (67 x 32 heads over 2651 keys
    // of 256: 311 us, so 229)
    constexpr bool kSharedQ = D > 128;
    constexpr int QP = D * 2 + 16, NK = kSharedQ ? 1 : D / 16;
    __shared__ __attribute__((aligned(16))) char sq[kSharedQ ? TILE * QP : 16];
    __shared__ PlanShared sh;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Walk k;
    if (!begin<TILE, UNIT>(reread(), sh, k))
        return;
    char *const values = lds + wave * 32 * PITCH;
    bool first = true;

    do {
        const AttnParams &p = reread();
        piece<TILE, UNIT>(p, k);
        const int b = k.b, item = k.item, ua = k.ua, ub = k.ub, keys = k.seq.keys;
        const Chunk &c = k.seq.c;
        const int h = item % p.a.Hkv, tile = item / p.a.Hkv;
        const int32_t *table = p.a.table + (int64_t)b * p.a.max_pages;
        const Factor fac = factor_of(p, h);
        const float factor = fac.size;

        const Row r = row_of(p, c, h, tile * TILE + (lane & 31));
        u32x4 q[NK], part[4];
        f32x16 o[D / 32];
        float m = -INFINITY, l = 0.0f;
        constexpr int kStep = kThreads * 16 / (D * 2);  // rows that all lanes read at once
        if constexpr (kSharedQ) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const Row y = row_of(p, c, h, tile * TILE + x * kStep + tid / (D / 8));
                part[x] = u32x4{0, 0, 0, 0};
                if (y.ok)
                    part[x] = *(const u32x4 *)((const char *)p.q +
                                               (y.row * p.q_stride + (int64_t)y.head * D) * 2 +
                                               tid % (D / 8) * 16);
            }
            apply_sign(part, fac.sign);
        }
        int at_q = (lane & 31) * QP + half * (E4M3 ? 32 : 16);
        // the query's operand of step kk
        const auto query = [&](int kk) {
            if constexpr (!kSharedQ)
                return q[kk];
            else
                return *(const u32x4 *)(sq + at_q + (E4M3 ? kk / 2 * 64 + kk % 2 * 16 : kk * 32));
        };
        if constexpr (!kSharedQ) {
            load_query<E4M3, D>(p, r, q);
            apply_sign(q, fac.sign);
        }
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
            o[dt] = f32x16{0};

        // a lane's key is its number within 32; both halves of a row are read by
        // the two lanes of its number
        const int kl = wave * 32 + (lane & 31);
        const char *const kbase =
            (const char *)p.k_cache + (int64_t)h * D * (E4M3 ? 1 : 2) + half * 16;
        const char *const vbase =
            (const char *)p.v_cache + (int64_t)h * D * (E4M3 ? 1 : 2) + half * 16;
        const uint32_t row_bytes = (uint32_t)(p.a.Hkv * D * (E4M3 ? 1 : 2));
        u32x4 kr[CH], vr[CH];
        // positions without a key are read from the first slot, and not used
        const auto load = [&](u32x4 (&to)[CH], const char *base, int slot) {
            const char *src = base + (uint64_t)(uint32_t)(slot < 0 ? 0 : slot) * row_bytes;
#pragma unroll
            for (int x = 0; x < CH; ++x)
                to[x] = *(const u32x4 *)(src + x * 32);
        };
        const int stop = keys > 0 ? ub : ua;  // without keys nothing is read
        bool poisoned = false;
        int slot = -1, next = -1, entry = -1;
        if (ua < stop) {
            slot = slot_of(p, table, ua * UNIT + kl, keys);
            next = slot_of(p, table, (ua + 1) * UNIT + kl, keys);
            entry = entry_of(p, table, (ua + 2) * UNIT + kl, keys);
            load(kr, kbase, slot);
            load(vr, vbase, slot);
        }
        if constexpr (kSharedQ) {
            static_assert(!kSharedQ || 4 * kStep == TILE, "four pieces for a lane");
#pragma unroll
            for (int x = 0; x < 4; ++x)
                *(u32x4 *)(sq + (x * kStep + tid / (D / 8)) * QP + tid % (D / 8) * 16) = part[x];
            __syncthreads();
        }
        for (int t = ua; t < stop; ++t) {
            const int kb = t * UNIT + wave * 32;
            const uint32_t valid = (uint32_t)__ballot(slot >= 0);
            const bool plain = valid == ~0u && kb + 31 < c.pos;
            f32x16 s[1] = {f32x16{0}};
            const int ahead = slot_in(p, entry, (t + 2) * UNIT + kl, keys);
            if (kSharedQ)  // read in every unit, not kept in registers
                asm volatile("" : "+v"(at_q));
            // before the next keys and values, which it is not to wait for
            entry = entry_of(p, table, (t + 3) * UNIT + kl, keys);
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                if (E4M3) {
                    u32x4 lo, hi;
                    widen<TYPE>(kr[k], lo, hi);
                    s[0] = mfma<TYPE>(lo, query(k * 2), s[0]);
                    s[0] = mfma<TYPE>(hi, query(k * 2 + 1), s[0]);
                } else {
                    s[0] = mfma<TYPE>(kr[k], query(k), s[0]);
                }
            }
            // behind the last unit nothing more is read (17 x 32 heads over 1481 keys of 128:
            // 33 -> 30 us), but where the branches cost more than the reads: 8-bit keys and
            // 256-wide heads (67 x 32 over 2651: 229 us, with the branches 243)
            const bool more = E4M3 || D > 128 || t + 1 < stop;
            if (more)
                load(kr, kbase, next);
            // values into LDS
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            char *dst = values + (lane & 31) * PITCH;
            if (!plain) {
                bool bad = false;
#pragma unroll
                for (int x = 0; x < CH; ++x) {
                    if (E4M3) {
                        // 0x7F and 0xFF are the NaN, there are no infinities
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if ((vr[x][j / 4] >> (j % 4 * 8) & 0x7Fu) == 0x7Fu) {
                                vr[x][j / 4] &= ~(0xFFu << (j % 4 * 8));
                                bad = true;
                            }
                    } else {
                        bad |= clear_not_finite<TYPE>(vr[x]);
                    }
                }
                poisoned |= __any(bad && slot >= 0);
            }
#pragma unroll
            for (int x = 0; x < CH; ++x) {
                if (E4M3) {
                    u32x4 lo, hi;
                    widen<TYPE>(vr[x], lo, hi);
                    *(u32x4 *)(dst + (x * 32 + half * 16) * 2) = lo;
                    *(u32x4 *)(dst + (x * 32 + half * 16 + 8) * 2) = hi;
                } else {
                    *(u32x4 *)(dst + (x * 16 + half * 8) * 2) = vr[x];
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (more)
                load(vr, vbase, next);
            if (!plain)
                hide(s[0], seen_bits(p, c, r, kb, valid));
            const float alpha = follow<TYPE, 1>(s, factor, m, l);
            if (__any(alpha != 1.0f))
                scale_rows<D>(o, alpha);
            u32x4 weights[2];
            weigh<TYPE, 1>(s, factor, m, l, weights);
            add_values<TYPE, D, 1>(weights, values, PITCH, o);
            slot = next;
            next = ahead;
        }
        if (poisoned) {
            const AttnParams &p = reread();
            for (int t = ua; t < stop; ++t) {
                const int kb = t * UNIT + wave * 32;
                const int at = slot_of(p, table, t * UNIT + kl, keys);
                const uint32_t valid = (uint32_t)__ballot(at >= 0);
                if (valid == ~0u && kb + 31 < c.pos)
                    continue;
                add_not_finite<TYPE, E4M3, D>(p, h, at, seen_bits(p, c, r, kb, valid), o);
            }
        }

        // join the four waves
        const AttnParams &pe = reread();
        const int64_t place = k.done ? -1 : (int64_t)blockIdx.x * 2 + (first ? 0 : 1);
        l += other_half(l);
        const int row = lane & 31;
        if (half == 0) {
            sm[wave][row] = m;
            sl[wave][row] = l;
        }
        __syncthreads();
        float top = sm[0][row];
#pragma unroll
        for (int v = 1; v < 4; ++v)
            top = fmaxf(top, sm[v][row]);
        // a wave whose products were all NaN has the maximum -inf too, and a sum that is NaN
        const float at = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            sum += sl[v][row] * __builtin_amdgcn_exp2f(sm[v][row] - at);
        const float f = __builtin_amdgcn_exp2f(m - at);
        // each wave adds up one block of columns
#pragma unroll
        for (int d0 = 0; d0 < D / 32; d0 += COLS) {
#pragma unroll
            for (int y = 0; y < COLS; ++y)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = o[d0 + y][g * 4 + e] * f;
                    *(f32x4 *)(lds + (((wave * COLS + y) * 4 + g) * 64 + lane) * 16) = v;
                }
            __syncthreads();
            if (wave < COLS) {
                f32x16 t = f32x16{0};
#pragma unroll
                for (int v = 0; v < 4; ++v)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4 y =
                            *(const f32x4 *)(lds + (((v * COLS + wave) * 4 + g) * 64 + lane) * 16);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            t[g * 4 + e] += y[e];
                    }
                put<TYPE, D, TILE>(pe, r, h, row, place, d0 + wave, t, top, sum);
            }
            __syncthreads();
        }
        first = false;
    } while (next<TILE, UNIT>(reread(), k));
}

// Tiles of 128 query rows, 32 for each wave; the four waves share 64 keys and
// values at a time in LDS, two buffers of them, the next ones on their way through
// registers while the present ones are used.  (Loads straight into LDS save those registers,
// but the compiler waits for all of them before any read of LDS.)
//   Chunks of prompts, 32 + 8 heads of 128, bf16: 969 us and more, up to 840 TFLOP/s; 256 x 60
// drafted nodes over up to 2048 keys: 630 us, 530 TFLOP/s.  A wave needs 1024 cycles of
// matrix instructions for a tile of 32 rows and 64 keys, and some 1450 of vector ones (512 of
// them the exponentials), and a SIMD takes 2770 (prompts) to 3400 (trees) for it: the
// rest are waits, and the matrix unit is in use for a third of the time.
template <int TYPE, bool E4M3, int D>
__global__ void __launch_bounds__(kThreads, D <= 128 ? 2 : 1) k_attend_many(const AttnParams) {
    constexpr int TILE = 128, UNIT = 64;
    constexpr int CH = E4M3 ? D / 16 : D / 8;  // 16-byte pieces of a row in the cache
    constexpr int RPI = 64 / CH;               // rows that a wave reads at once
    constexpr int NI = 16 / RPI;               // such reads for its 16 rows
    // rows of keys 16 bytes apart from a multiple of 256, so that 16 of them read at one
    // column lie in different banks; 4 rows of values read at two pairs of pieces too
    constexpr int KP = D * 2 + 16, VP = D * 2 + 64;
    __shared__ __attribute__((aligned(16))) char sk[2][UNIT * KP];
    __shared__ __attribute__((aligned(16))) char sv[2][UNIT * VP];
    __shared__ __attribute__((aligned(16))) uint64_t sflag[2][4];  // keys there are
    __shared__ int s_poison[4];  // each wave's own: it clears it before it stores values
    __shared__ PlanShared sh;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Walk k;
    if (!begin<TILE, UNIT>(reread(), sh, k))
        return;
    bool first = true;

    do {
        const AttnParams &p = reread();
        piece<TILE, UNIT>(p, k);
        const int b = k.b, item = k.item, ua = k.ua, keys = k.seq.keys;
        const Chunk &c = k.seq.c;
        int ub = k.ub;
        // whole items: the last tiles first, which see the most keys without a mask
        const int h = item % p.a.Hkv;
        const int tile = !k.whole && k.seq.grow ? item / p.a.Hkv
                                                : k.seq.tiles - 1 - item / p.a.Hkv;
        const int32_t *table = p.a.table + (int64_t)b * p.a.max_pages;
        const Factor fac = factor_of(p, h);
        const float factor = fac.size;
        // keys that the tile's (the wave's) last row sees
        int lim = keys, wlim = keys;
        if (!p.a.mask) {
            const int i1 = (tile * TILE + TILE - 1) / p.G;
            const int i2 = (tile * TILE + wave * 32 + 31) / p.G;
            const int64_t e1 = (int64_t)c.pos + (i1 < c.n ? i1 + 1 : c.n);
            const int64_t e2 = (int64_t)c.pos + (i2 < c.n ? i2 + 1 : c.n);
            lim = e1 < keys ? (int)e1 : keys;
            wlim = e2 < keys ? (int)e2 : keys;
        }
        const int stop = (lim + UNIT - 1) / UNIT;
        ub = ub < stop ? ub : stop;
        const Row r = row_of(p, c, h, tile * TILE + wave * 32 + (lane & 31));
        const bool rows = __any(r.ok);
        u32x4 q[D / 16];
        load_query<false, D>(p, r, q);
        apply_sign(q, fac.sign);
        f32x16 o[D / 32];
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
            o[dt] = f32x16{0};

        const int piece = lane % CH, sub = lane / CH;
        const char *const kbase =
            (const char *)p.k_cache + (int64_t)h * D * (E4M3 ? 1 : 2) + piece * 16;
        const char *const vbase =
            (const char *)p.v_cache + (int64_t)h * D * (E4M3 ? 1 : 2) + piece * 16;
        const uint32_t row_bytes = (uint32_t)(p.a.Hkv * D * (E4M3 ? 1 : 2));
        u32x4 kr[NI], vr[NI];
        const uint64_t apart = (uint64_t)(vbase - kbase);
        if (lane == 0)
            s_poison[wave] = 0;
        // Slots by batches of four tiles: a lane has the slot of one key, of tile lane / 16
        // of the batch and of the 16 keys there that its wave fetches.  The table's
        // entries are asked for two batches ahead.  Positions without a key are fetched
        // from the first slot, and not used.
        const auto position = [&](int batch) {
            return (ua + batch * 4 + lane / 16) * UNIT + wave * 16 + lane % 16;
        };
        const auto load = [&](int slots, int tile) {
            int of[NI];
#pragma unroll
            for (int x = 0; x < NI; ++x)
                of[x] = __shfl(slots, tile * 16 + x * RPI + sub);
#pragma unroll
            for (int x = 0; x < NI; ++x) {
                const char *from = kbase + (uint64_t)(uint32_t)of[x] * row_bytes;
                kr[x] = *(const u32x4 *)from;
                vr[x] = *(const u32x4 *)(from + apart);
            }
        };
        const auto stash = [&](uint32_t valid, int t) {
            const int buf = t & 1;
            const bool plain = valid == 0xFFFFu && (t + 1) * UNIT <= c.pos;
            bool bad = false;
#pragma unroll
            for (int x = 0; x < NI; ++x) {
                const int row = wave * 16 + x * RPI + sub;
                char *kd = sk[buf] + row * KP, *vd = sv[buf] + row * VP;
                if (E4M3) {
                    u32x4 lo, hi;
                    widen<TYPE>(kr[x], lo, hi);
                    *(u32x4 *)(kd + piece * 32) = lo;
                    *(u32x4 *)(kd + piece * 32 + 16) = hi;
                    widen<TYPE>(vr[x], lo, hi);
                    if (!plain) {
                        bad |= clear_not_finite<TYPE>(lo);
                        bad |= clear_not_finite<TYPE>(hi);
                    }
                    *(u32x4 *)(vd + piece * 32) = lo;
                    *(u32x4 *)(vd + piece * 32 + 16) = hi;
                } else {
                    *(u32x4 *)(kd + piece * 16) = kr[x];
                    if (!plain)
                        bad |= clear_not_finite<TYPE>(vr[x]);
                    *(u32x4 *)(vd + piece * 16) = vr[x];
                }
            }
            if (!plain && __any(bad) && lane == 0)
                s_poison[wave] = 1;
        };

        if (keys == 0)
            ub = ua;
        int slots = 0, next = 0, entry = -1;  // of this batch, the next; the table's behind
        uint64_t valid = 0, valid_next = 0;
        uint64_t all = 0;                     // keys that all four waves have
        const auto slots_of = [&](int from, int batch, uint64_t &there) {
            const int slot = slot_in(p, from, position(batch), lim);
            there = __ballot(slot >= 0);
            if (lane == 0)
                sflag[batch & 1][wave] = there;
            return slot < 0 ? 0 : slot;
        };
        if (ua < ub) {
            const int e0 = entry_of(p, table, position(0), lim);
            entry = entry_of(p, table, position(1), lim);
            next = slots_of(e0, 0, valid_next);
            load(next, 0);
            stash((uint32_t)valid_next & 0xFFFFu, ua);
        }
        for (int t = ua; t < ub; ++t) {
            __syncthreads();
            const int j = (t - ua) & 3, batch = (t - ua) >> 2;
            if (j == 0) {
                const u32x4 *f = (const u32x4 *)sflag[batch & 1];
                const u32x4 both = f[0] & f[1];
                all = (uint64_t)__builtin_amdgcn_readfirstlane(both[1] & both[3]) << 32 |
                      (uint32_t)__builtin_amdgcn_readfirstlane(both[0] & both[2]);
                slots = next;
                valid = valid_next;
                next = slots_of(entry, batch + 1, valid_next);
                entry = entry_of(p, table, position(batch + 2), lim);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (t + 1 < ub)
                load(j < 3 ? slots : next, (j + 1) & 3);
            const int kb = t * UNIT, buf = t & 1;
            if (rows && kb < wlim) {
                const char *const K = sk[buf], *const V = sv[buf];
                // four fragments of the keys ahead of those that are multiplied
                f32x16 s[2];
                s[0] = s[1] = f32x16{0};
                u32x4 f[2][4];
                const auto ask = [&](int step, u32x4 (&to)[4]) {
                    const int row = step / (D / 64) * 32 + (lane & 31);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int kk = step % (D / 64) * 4 + x;
                        to[x] =
                            *(const u32x4 *)(K + row * KP + (kk * 2 + half) * 16);
                    }
                };
                ask(0, f[0]);
#pragma unroll
                for (int step = 0; step < D / 32; ++step) {
                    if (step + 1 < D / 32)
                        ask(step + 1, f[(step + 1) & 1]);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        s[step / (D / 64)] = mfma<TYPE>(f[step & 1][x], q[step % (D / 64) * 4 + x],
                                                        s[step / (D / 64)]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if ((~all >> j * 16 & 0xFFFF) != 0 || kb + UNIT > c.pos) {
                    const uint64_t *f = sflag[batch & 1];
                    const int x = j * 16;
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        hide(s[y],
                             seen_bits(p, c, r, kb + y * 32,
                                       ((uint32_t)(f[y * 2] >> x) & 0xFFFFu) |
                                           (uint32_t)(f[y * 2 + 1] >> x) << 16));
                }
                const float alpha = follow<TYPE, 2>(s, factor, m, l);
                if (__any(alpha != 1.0f))
                    scale_rows<D>(o, alpha);
                u32x4 weights[4];
                weigh<TYPE, 2>(s, factor, m, l, weights);
                add_values<TYPE, D, 2>(weights, V, VP, o);
            }
            if (t + 1 < ub)
                stash((uint32_t)((j < 3 ? valid : valid_next) >> ((j + 1) & 3) * 16) & 0xFFFFu,
                      t + 1);
        }
        __syncthreads();
        const bool poisoned = (s_poison[0] | s_poison[1] | s_poison[2] | s_poison[3]) != 0;
        __syncthreads();  // before the next item's first tile is stored
        if (poisoned) {
            const AttnParams &p = reread();
            for (int kb = ua * UNIT; kb < ub * UNIT && kb < wlim; kb += 32) {
                const int at = slot_of(p, table, kb + (lane & 31), lim);
                const uint32_t valid = (uint32_t)__ballot(at >= 0);
                if (valid != ~0u || kb / UNIT * UNIT + UNIT > c.pos)
                    add_not_finite<TYPE, E4M3, D>(p, h, at, seen_bits(p, c, r, kb, valid), o);
            }
        }

        const AttnParams &pe = reread();
        l += other_half(l);
        const int64_t place = k.done ? -1 : (int64_t)blockIdx.x * 2 + (first ? 0 : 1);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
            put<TYPE, D, TILE>(pe, r, h, wave * 32 + (lane & 31), place, dt, o[dt], m, l);
        first = false;
    } while (next<TILE, UNIT>(reread(), k));
}

// A partial result added to a row's.
__device__ __forceinline__ void add_part(float &m, float &l, f32x4 &o, float pm, float ps,
                                         f32x4 po) {
    const float mn = fmaxf(m, pm), at = mn == -INFINITY ? 0.0f : mn;
    const float f = __builtin_amdgcn_exp2f(m - at), pf = __builtin_amdgcn_exp2f(pm - at);
    m = mn;
    l = l * f + ps * pf;
    o = o * f + po * pf;
}

// Joins the partial results of the items that were cut.  Of a work-group's lanes,
// D / 4 take four elements each of a row; `parts` such groups of lanes take every
// parts-th result of one row, the others another row.
template <int TYPE, int D, int TILE, int UNIT, int kRows>
__global__ void __launch_bounds__(kThreads) k_merge(const AttnParams, int parts,
                                                    uint32_t groups) {
    constexpr int LANES = D / 4, kSets = kThreads / LANES, kLoops = 4 / kRows;
    __shared__ PlanShared sh;
    __shared__ f32x4 so[kThreads];
    __shared__ float2 sml[kThreads];
    const int tid = threadIdx.x;
    const Plan pl = plan<TILE, UNIT>(reread(), sh);
    const AttnParams &p = reread();
    const Work &w = pl.w;
    if (w.whole)
        return;
    const int set = tid / LANES, lane = tid % LANES, d = lane * 4;
    // the row groups of all items in equal shares
    const uint32_t all = w.items * groups;
    const uint32_t from = (uint32_t)((uint64_t)blockIdx.x * all / gridDim.x);
    const uint32_t to = (uint32_t)(((uint64_t)blockIdx.x + 1) * all / gridDim.x);
    uint32_t found = ~0u, item = 0, base = 0;
    Seq s;
    for (uint32_t id = from, n; id < to; id += n) {
        if (id / groups != found) {
            found = id / groups;
            find<TILE, UNIT>(p, pl, true, found, sh, s, item, base);
        }
        n = groups - id % groups;
        n = n < to - id ? n : to - id;
        n = n < kRows ? n : kRows;
        const Chunk &c = s.c;
        uint32_t nu = (uint32_t)s.units, u0 = base + item * nu;
        if (TILE > UNIT && s.grow) {
            const int t = (int)item / p.a.Hkv;
            nu = units_of<TILE, UNIT>(p, s, t);
            u0 = base + units_before<TILE, UNIT>(p, s, t) + item % (uint32_t)p.a.Hkv * nu;
        }
        const uint32_t u1 = u0 + nu;
        const uint32_t g0 = group_of(w, u0), g1 = group_of(w, u1 - 1);
        if (g0 == g1)
            continue;  // one work-group had the whole item
        const bool late = start_of(w, g0) < u0;  // the item is not the first one of g0
        const int h = (int)item % p.a.Hkv;
        const int tile = TILE > UNIT && !s.grow ? s.tiles - 1 - (int)item / p.a.Hkv
                                                : (int)item / p.a.Hkv;
        Row r[kRows];
        int row[kRows];
        bool on[kRows];
        float m[kRows], l[kRows];
        f32x4 o[kRows];
#pragma unroll
        for (int y = 0; y < kRows; ++y) {
            const int at = (int)(id % groups + y) * (kSets / parts) + set / parts;
            r[y] = row_of(p, c, h, tile * TILE + at);
            on[y] = (uint32_t)y < n && at < TILE && r[y].ok;
            row[y] = on[y] ? at : 0;  // read all the same
            m[y] = -INFINITY;
            l[y] = 0.0f;
            o[y] = f32x4{0};
        }
#pragma unroll kLoops
        for (uint32_t g = g0 + set % parts; g <= g1; g += parts) {
            const float *part =
                p.part + ((int64_t)g * 2 + (g == g0 && late ? 1 : 0)) * (TILE * (D + 2));
            float pm[kRows], ps[kRows];
            f32x4 po[kRows];
#pragma unroll
            for (int y = 0; y < kRows; ++y) {
                pm[y] = part[TILE * D + row[y]];
                ps[y] = part[TILE * D + TILE + row[y]];
                po[y] = *(const f32x4 *)(part + row[y] * D + d);
            }
#pragma unroll
            for (int y = 0; y < kRows; ++y)
                add_part(m[y], l[y], o[y], pm[y], ps[y], po[y]);
        }
#pragma unroll
        for (int y = 0; y < kRows; ++y) {
            if (parts > 1) {
                __syncthreads();  // the last row's use of LDS
                so[tid] = o[y];
                sml[tid] = make_float2(m[y], l[y]);
                __syncthreads();
                for (int x = 1; x < parts && set % parts == 0; ++x) {
                    const float2 z = sml[tid + x * LANES];
                    add_part(m[y], l[y], o[y], z.x, z.y, so[tid + x * LANES]);
                }
            }
            if (!on[y] || set % parts)
                continue;
            const float f = l[y] == 0.0f ? 0.0f : (p.v_scale ? p.v_scale[h] : 1.0f) / l[y];
            const f32x4 v = l[y] == 0.0f ? f32x4{0} : o[y] * f;
            *(uint2 *)((char *)p.out + ((r[y].row * p.a.Hq + r[y].head) * D + d) * 2) =
                make_uint2(pack2<TYPE>(v[0], v[1]), pack2<TYPE>(v[2], v[3]));
            if (p.lse && d == 0)
                p.lse[r[y].row * p.a.Hq + r[y].head] =
                    l[y] == 0.0f ? -INFINITY : (m[y] + __builtin_amdgcn_logf(l[y])) * kLn2;
        }
    }
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

template <int TYPE, int D, int TILE, int UNIT>
void launch_merge(const AttnParams &p, int64_t items, hipStream_t stream) {
    constexpr int kSets = kThreads / (D / 4);
    // lanes for a row's results beside each other while there are too few rows
    const int64_t rows = (int64_t)p.a.R * p.G < TILE ? (int64_t)p.a.R * p.G : TILE;
    items = items < attention_whole(TILE) ? items : attention_whole(TILE);
    int parts = 1;
    const auto groups = [&]() { return (rows * parts + kSets - 1) / kSets; };
    while (parts < kSets && parts * items < p.groups && items * groups() < kAttnMerge)
        parts *= 2;
    const int64_t all = items * groups();
    const dim3 g((unsigned)(all < kAttnMerge ? all : kAttnMerge)), t(kThreads);
    // four rows of an item at once where a work-group has eight and more groups of them (242 x
    // 95 rows over 1718 keys: 267 -> 261 us); with fewer, four results of one (3 x 324 over
    // 1749: 36 us, four rows at once 41)
    if (all >= 8 * kAttnMerge)
        hipLaunchKernelGGL((k_merge<TYPE, D, TILE, UNIT, 4>), g, t, 0, stream, p, parts,
                           (uint32_t)groups());
    else
        hipLaunchKernelGGL((k_merge<TYPE, D, TILE, UNIT, 1>), g, t, 0, stream, p, parts,
                           (uint32_t)groups());
}

template <int TYPE, bool E4M3, int D>
int launch_attend(AttnParams p, hipStream_t stream) {
    const int64_t rows = (int64_t)p.a.R * p.G, tile = attention_tile(rows);
    const int64_t whole = attention_whole(tile);
    int64_t items = (int64_t)p.a.B * ((rows + tile - 1) / tile);
    // what a device's cu that does not ascend could ask for is to fit 32 bits too
    if (items * p.a.Hkv >= 1ll << 31)
        return SWITCHSD_ESHAPE;
    const int64_t cut = items * p.a.Hkv;
    // packed: the rows that there are make no more tiles than this
    const int64_t most = (int64_t)p.a.rows * p.G / tile + p.a.B;
    if (p.a.cu && most < items)
        items = most;
    items *= p.a.Hkv;
    const int64_t cap = (int64_t)p.a.max_pages * p.a.page_size;
    const int64_t len = (int64_t)p.a.Lmax + p.a.R;
    const int64_t keys = len < cap ? len : cap;
    // never cut: short contexts, and lengths whose units would not fit 32 bits
    p.whole = keys <= kAttnShort ||
              (cut < whole ? cut : whole) * (keys / 64 + 4) >= (1ll << 31);
    // as many as the device holds at once: two on a compute unit where their registers
    // allow it
    p.groups = D == 256 ? kAttnGroups / 2 : kAttnGroups;
    const int64_t groups = p.whole || items > p.groups ? items : p.groups;
    if (groups >= 1 << 24)
        return SWITCHSD_ESHAPE;
    const dim3 g((unsigned)groups), t(kThreads);
    if (tile == 32) {
        hipLaunchKernelGGL((k_attend_few<TYPE, E4M3, D>), g, t, 0, stream, p);
        if (!p.whole)
            launch_merge<TYPE, D, 32, 128>(p, items, stream);
    } else {
        hipLaunchKernelGGL((k_attend_many<TYPE, E4M3, D>), g, t, 0, stream, p);
        if (!p.whole)
            launch_merge<TYPE, D, 128, 64>(p, items, stream);
    }
    return launched();
}

template <int TYPE, bool E4M3>
int launch_typed(const AttnParams &p, hipStream_t stream) {
    return p.a.D == 64    ? launch_attend<TYPE, E4M3, 64>(p, stream)
           : p.a.D == 128 ? launch_attend<TYPE, E4M3, 128>(p, stream)
                          : launch_attend<TYPE, E4M3, 256>(p, stream);
}

}  // namespace

int launch_attention_kernel(const AttnParams &p, int32_t type, int32_t cache_type,
                            hipStream_t stream) {
    const bool e4m3 = cache_type == SWITCHSD_E4M3;
    if (type == SWITCHSD_BF16)
        return e4m3 ? launch_typed<SWITCHSD_BF16, true>(p, stream)
                    : launch_typed<SWITCHSD_BF16, false>(p, stream);
    return e4m3 ? launch_typed<SWITCHSD_F16, true>(p, stream)
                : launch_typed<SWITCHSD_F16, false>(p, stream);
}

}  // namespace switchsd
