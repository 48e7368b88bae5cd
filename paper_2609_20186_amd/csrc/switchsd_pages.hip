// switchsd_pages.hip -- gfx950 kernels for the bookkeeping of a paged KV cache
// around the speculation-control step: pages, slots and positions of the
// drafted rows (k_page_plan), packed slots of ragged ranges (k_span_slots) and
// the move of the accepted nodes' cache rows (k_compact).
//
// A plan moves a few kilobytes: it is bound by its chain of dependent reads
// (requests, sums over the sequences, pages, slots) and, with several
// work-groups, by the ticket of the last one.  Measured (MI355X), each state
// planned once, so that pages move: 32 sequences of 8 rows 4.8 us, 32 of 201 14.2
// us, 1024 trees of 60 nodes 9.4 us (planned again, when nothing moves: 2.7 and
// 8.8 us for the first and the last).  Every work-group sums over all sequences
// before its own, which grows with the square of their number: 65536 trees of
// 60 nodes take 1.5 ms.  Packed slots write 20 bytes
// a position: 256 prompts of up to 8192 tokens 11 us, 4.0 TB/s.  Cache rows: 16
// x 20 rows of 1 KB in each of 32 planes moved in 6.7 us, 3.1 TB/s.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "switchsd_device.h"
#include "switchsd_internal.h"

namespace switchsd {

namespace {

constexpr int kWaves = kThreads / 64;

// Inclusive sums over the work-group's lanes of (a, b); their totals.
__device__ __forceinline__ void block_scan2(int &a, int &b, int &ta, int &tb,
                                            int (&sh)[2][kWaves]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    a = wave_scan(a);
    b = wave_scan(b);
    if (lane == 63) {
        sh[0][wave] = a;
        sh[1][wave] = b;
    }
    __syncthreads();
    ta = tb = 0;
    int pa = 0, pb = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        pa += w < wave ? sh[0][w] : 0;
        pb += w < wave ? sh[1][w] : 0;
        ta += sh[0][w];
        tb += sh[1][w];
    }
    a += pa;
    b += pb;
    __syncthreads();
}

// What sequence b asks of the ring: its length and nodes, the pages it holds,
// lacks (grow) and gives back (back).  B * max_pages < 2^31, so sums of them
// fit 32 bits.
struct Ask {
    int L, n, held, grow, back;
};
__device__ __forceinline__ Ask page_ask(const PageParams &p, int lengths, int dn, int held) {
    Ask a;
    a.L = clampi(lengths, 0, p.Lmax);
    a.n = clampi(dn, 1, p.R);
    a.held = clampi(held, 0, p.max_pages);
    a.grow = a.back = 0;
    if (a.L > 0) {
        const uint32_t last = (uint32_t)(a.L - 1) + (uint32_t)a.n + (uint32_t)p.page_size - 1u;
        const uint32_t need =
            p.page_log >= 0 ? last >> p.page_log : last / (uint32_t)p.page_size;
        const int pages = need < (uint32_t)p.max_pages ? (int)need : p.max_pages;
        a.grow = pages > a.held ? pages - a.held : 0;
    } else {
        a.back = a.held;
    }
    return a;
}

// What the sequences lane * 4 .. lane * 4 + 3 of those from b0 on ask, requested
// at once (behind b1: nothing).
__device__ __forceinline__ void page_ask4(const PageParams &p, int b0, int b1, Ask (&a)[4]) {
    int len[4], dn[4], held[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int b = b0 + 4 * (int)threadIdx.x + q, c = b < b1 ? b : b1 - 1;
        len[q] = p.lengths[c];
        dn[q] = p.dn[c];
        held[q] = p.held[c];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        a[q] = page_ask(p, len[q], dn[q], held[q]);
        if (b0 + 4 * (int)threadIdx.x + q >= b1)
            a[q].grow = a[q].back = 0;
    }
}

__device__ __forceinline__ uint32_t ring_at(const PageParams &p, int head, int64_t i) {
    // head < ring_pages and i < ring_pages
    const uint32_t k = (uint32_t)head + (uint32_t)i;
    return k >= (uint32_t)p.ring_pages ? k - (uint32_t)p.ring_pages : k;
}

// Pages of one sequence, by the wave: entries held + j, j >= j0, taken from
// the ring, all of a finished sequence's given back.
__device__ __forceinline__ void page_moves(const PageParams &p, int head, int count, int b,
                                           int held, int first, int took, int j0, int back,
                                           int bfirst) {
    const int lane = threadIdx.x & 63;
    int32_t *row = p.table + (int64_t)b * p.max_pages;
    for (int j = j0 + lane; j < took; j += 64)
        row[held + j] = p.ring[ring_at(p, head, first + j)];
    for (int j = lane; j < back; j += 64) {
        const int64_t at = (int64_t)count + bfirst + j;
        if (at < p.ring_pages)
            p.ring[ring_at(p, head, at)] = row[j];
        row[j] = -1;
    }
}

// The slot of cache position `at`.
__device__ __forceinline__ int64_t page_slot(const PageParams &p, int head, int b, uint32_t at,
                                             int held, int first, int took) {
    const uint32_t pg = p.page_log >= 0 ? at >> p.page_log : at / (uint32_t)p.page_size;
    if (pg >= (uint32_t)(held + took))
        return -1;
    const int page = pg < (uint32_t)held ? p.table[(int64_t)b * p.max_pages + pg]
                                         : p.ring[ring_at(p, head, first + (int)pg - held)];
    return (int64_t)page * p.page_size + (at - pg * (uint32_t)p.page_size);
}

// Pages, slots and positions.  Work-group g plans the sequences from g * seqs
// on: it sums what all earlier sequences lack and give back, so that no
// work-group waits for another, and the last one to arrive, when every one has
// read held and the ring's state, writes both anew (a lone one does so at
// once).  A page taken in this call is read from the ring, where nothing is
// written in this call that is read from it: returned pages go behind the free
// ones, and only as far as the ring's end.
// kLanes (R <= 64): a node per lane, 64 / R whole sequences per wave, depths by
// pointer jumping in registers; else nodes in LDS, kPlanNodes at most.
template <bool kLanes>
__global__ __launch_bounds__(kThreads) void k_page_plan(PageParams p) {
    __shared__ int red[2][kWaves];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b0 = blockIdx.x * p.seqs;
    const int ns = p.B - b0 < p.seqs ? p.B - b0 : p.seqs;
    const int h0 = p.ring_state[0], c0 = p.ring_state[1];
    // this lane's sequence (kLanes: its node's), before anything is waited for
    const int per = 64 / p.R;
    int sl = tid, r = 0;
    bool mine = tid < ns;
    if (kLanes) {
        const int i = (int)((uint32_t)lane / (uint32_t)p.R);
        r = lane - i * p.R;
        sl = wave * per + i;
        mine = i < per && sl < ns;
    }
    const int b = b0 + (mine ? sl : 0);
    const int len = p.lengths[b], dn = p.dn[b], hd = p.held[b];
    int par = r - 1;
    if (kLanes && p.dpar && p.positions)
        par = p.dpar[(int64_t)b * p.R + (r < p.R ? r : 0)];
    int ga = 0, ba = 0;  // of the sequences before b0
    if (b0 > 0) {
        for (int t0 = 0; t0 < b0; t0 += 4 * kThreads) {
            Ask a[4];
            page_ask4(p, t0, b0, a);
            ga += a[0].grow + a[1].grow + a[2].grow + a[3].grow;
            ba += a[0].back + a[1].back + a[2].back + a[3].back;
        }
        int tg, tb;
        block_scan2(ga, ba, tg, tb, red);
        ga = tg;
        ba = tb;
    }
    const int head = clampi(h0, 0, p.ring_pages - 1);
    const int count = clampi(c0, 0, p.ring_pages);
    const Ask a = page_ask(p, len, dn, hd);
    const bool lead = mine && r == 0;
    int g = lead ? a.grow : 0, k = lead ? a.back : 0, gt, bt;
    block_scan2(g, k, gt, bt, red);
    const bool served = ga + g <= count;
    const int first = ga + g - a.grow, bfirst = ba + k - a.back;
    const int took = served ? a.grow : 0;
    if (lead)
        p.missing[b] = served ? 0 : a.grow;

    if constexpr (kLanes) {
        // taken pages: two per node's lane, the rest and the returned ones by
        // the wave, sequence by sequence
        int32_t *row = p.table + (int64_t)b * p.max_pages;
        int pg[2];
#pragma unroll
        for (int q = 0; q < 2; ++q)
            pg[q] = p.ring[mine && r + q * p.R < took ? ring_at(p, head, first + r + q * p.R) : 0u];
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (mine && r + q * p.R < took)
                row[a.held + r + q * p.R] = pg[q];
        unsigned long long more = __ballot(lead && (took > 2 * p.R || a.back > 0));
        while (more) {
            const int l = __ffsll((long long)more) - 1;
            more &= more - 1ull;
            page_moves(p, head, count, __shfl(b, l), __shfl(a.held, l), __shfl(first, l),
                       __shfl(took, l), 2 * p.R, __shfl(a.back, l), __shfl(bfirst, l));
        }
        const bool live = mine && a.L > 0 && r < a.n;
        if (p.positions) {
            const bool up = live && par >= 0 && par < r;
            int depth = up ? 1 : 0, anc = up ? lane - r + par : lane;
            for (;;) {
                const int nx = __shfl(anc, anc);
                if (__ballot(nx != anc) == 0ull)
                    break;
                depth += __shfl(depth, anc);
                anc = nx;
            }
            if (mine)
                p.positions[(int64_t)b * p.R + r] = live ? a.L - 1 + depth : -1;
        }
        if (p.slots && mine)
            p.slots[(int64_t)b * p.R + r] =
                live ? page_slot(p, head, b, (uint32_t)(a.L - 1 + r), a.held, first, took) : -1;
    } else {
        __shared__ uint32_t st[2][kPlanNodes];
        __shared__ int s_L[kWaves * 4], s_n[kWaves * 4], s_held[kWaves * 4], s_first[kWaves * 4],
            s_took[kWaves * 4], s_back[kWaves * 4], s_bfirst[kWaves * 4];
        if (tid < ns) {
            s_L[tid] = a.L;
            s_n[tid] = a.n;
            s_held[tid] = a.held;
            s_first[tid] = first;
            s_took[tid] = took;
            s_back[tid] = a.back;
            s_bfirst[tid] = bfirst;
        }
        __syncthreads();
        for (int s = wave; s < ns; s += kWaves)
            page_moves(p, head, count, b0 + s, s_held[s], s_first[s], s_took[s], 0, s_back[s],
                       s_bfirst[s]);
        const int nodes = ns * p.R;
        int cur = 0;
        if (p.positions && p.dpar) {
            // a path ends at the node whose parent is not valid, as at the anchor
            for (int i = tid; i < nodes; i += kThreads) {
                const int s = i / p.R, q = p.dpar[(int64_t)b0 * p.R + i], rr = i - s * p.R;
                const bool up = rr < s_n[s] && q >= 0 && q < rr;
                st[0][i] = up ? kHolds | (1u << 16) | (uint32_t)q : kHolds | (uint32_t)rr;
            }
            __syncthreads();
            for (bool open = true; open; cur ^= 1) {
                bool more = false;
                for (int i = tid; i < nodes; i += kThreads) {
                    const uint32_t s1 = st[cur][i];
                    const uint32_t s2 = st[cur][i / p.R * p.R + (int)(s1 & 0xFFFFu)];
                    st[cur ^ 1][i] = jump_compose(s1, s2);
                    more |= (s1 & 0xFFFFu) != (s2 & 0xFFFFu);
                }
                open = __syncthreads_or(more);
            }
        }
        for (int i = tid; i < nodes; i += kThreads) {
            const int s = i / p.R, rr = i - s * p.R;
            const int64_t o = (int64_t)b0 * p.R + i;
            const bool live = s_L[s] > 0 && rr < s_n[s];
            if (p.positions) {
                const int depth = p.dpar ? (int)((st[cur][i] >> 16) & 0x7FFFu) : rr;
                p.positions[o] = live ? s_L[s] - 1 + depth : -1;
            }
            if (p.slots)
                p.slots[o] = live ? page_slot(p, head, b0 + s, (uint32_t)(s_L[s] - 1 + rr),
                                              s_held[s], s_first[s], s_took[s])
                                  : -1;
        }
    }

    // ---- held and the ring's state, once every work-group has read them
    int popped = lead ? took : 0, z = 0;
    if (gridDim.x > 1) {
        __syncthreads();
        if (tid < 64) {
            const bool last = arrive(p.ticket, gridDim.x);
            if (tid == 0)
                s_last = last;
        }
        __syncthreads();
        if (!s_last)
            return;
        popped = 0;
        int before = 0;
        bt = 0;
        for (int t0 = 0; t0 < p.B; t0 += 4 * kThreads) {
            Ask q[4];
            page_ask4(p, t0, p.B, q);
            int gs = q[0].grow + q[1].grow + q[2].grow + q[3].grow, tg, tb;
            int bs = q[0].back + q[1].back + q[2].back + q[3].back;
            const int own = gs;
            block_scan2(gs, bs, tg, tb, red);
            int upto = before + gs - own;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                upto += q[i].grow;
                const int take = upto <= count ? q[i].grow : 0;
                const int bi = t0 + 4 * tid + i;
                popped += take;
                if (bi < p.B && (take || q[i].back))
                    p.held[bi] = q[i].L > 0 ? q[i].held + take : 0;
            }
            before += tg;
            bt += tb;
        }
    } else if (lead && (took || a.back)) {
        p.held[b] = a.L > 0 ? a.held + took : 0;
    }
    int total, zt;
    block_scan2(popped, z, total, zt, red);
    if (tid == 0) {
        p.ring_state[0] = (int)(((uint32_t)head + (uint32_t)total) % (uint32_t)p.ring_pages);
        // what lies behind the ring's end was not appended and does not count
        const int room = p.ring_pages - count;
        p.ring_state[1] = count - total + (bt < room ? bt : room);
        if (gridDim.x > 1)
            st_u32(p.ticket, 0u);
    }
}

// Packed slots.  A work-group takes the kSpanPart positions that are part
// number `part` of a sequence's range, four consecutive ones per lane, at the
// sum of all earlier sequences' sizes, which it takes itself while what it
// copies is under way.
typedef int32_t i32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef int64_t i64x2_a8 __attribute__((ext_vector_type(2), aligned(8)));

__global__ __launch_bounds__(kThreads) void k_span_slots(SpanParams p) {
    __shared__ int red[2][kWaves];
    const int tid = threadIdx.x;
    const int g = blockIdx.x / p.parts, part = blockIdx.x - g * p.parts;
    const int b0 = g * p.seqs, b1 = b0 + p.seqs < p.B ? b0 + p.seqs : p.B;
    if (part > 0) {
        // most ranges are shorter than the longest that may be
        bool any = false;
        for (int b = b0; b < b1; ++b) {
            const int h = clampi(p.end[b], 0, p.Lmax);
            any = any || h - clampi(p.begin[b], 0, h) > part * kSpanPart;
        }
        if (!any)
            return;
    }
    int before = 0;
    for (int b = b0; b < b1; ++b) {
        const int hi = clampi(p.end[b], 0, p.Lmax), lo = clampi(p.begin[b], 0, hi);
        const int size = hi - lo;
        // this lane's positions lo + k .. lo + k + 3
        const int k = part * kSpanPart + 4 * tid, i = lo + k;
        const int held = p.slots ? clampi(p.held[b], 0, p.max_pages) : 0;
        const int32_t *row = p.table + (int64_t)b * p.max_pages;
        const int32_t *x = p.tokens + (int64_t)b * p.Lmax;
        int page[4], tok[4];
        int64_t slot[4];
        const bool whole = k + 4 <= size;
        if (whole && p.packed) {
            const i32x4_a4 v = *(const i32x4_a4 *)(x + i);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                tok[q] = v[q];
        }
        if (k < size && p.slots) {
            int pg[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                pg[q] = p.page_log >= 0 ? (i + q) >> p.page_log
                                        : (int)((uint32_t)(i + q) / (uint32_t)p.page_size);
                page[q] = held > 0 ? row[pg[q] < held ? pg[q] : 0] : 0;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                slot[q] = pg[q] < held
                              ? (int64_t)page[q] * p.page_size + (i + q - pg[q] * p.page_size)
                              : -1;
        }
        if (b == b0 && b0 > 0) {
            for (int t0 = 0; t0 < b0; t0 += 4 * kThreads) {
                int l[4], h[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = t0 + q * kThreads + tid;
                    l[q] = p.begin[c < b0 ? c : b0 - 1];
                    h[q] = p.end[c < b0 ? c : b0 - 1];
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int e = clampi(h[q], 0, p.Lmax);
                    before += t0 + q * kThreads + tid < b0 ? e - clampi(l[q], 0, e) : 0;
                }
            }
            int z = 0, total, tz;
            block_scan2(before, z, total, tz, red);
            before = total;
        }
        if (part == 0 && tid == 0) {
            p.cu[b] = before;
            if (b == p.B - 1)
                p.cu[p.B] = before + size;
        }
        const int64_t j = (int64_t)before + k;
        if (whole && j + 4 <= p.capacity) {
            if (p.slots) {
                *(i64x2_a8 *)(p.slots + j) = i64x2_a8{slot[0], slot[1]};
                *(i64x2_a8 *)(p.slots + j + 2) = i64x2_a8{slot[2], slot[3]};
            }
            if (p.positions)
                *(i32x4_a4 *)(p.positions + j) = i32x4_a4{i, i + 1, i + 2, i + 3};
            if (p.packed)
                *(i32x4_a4 *)(p.packed + j) = i32x4_a4{tok[0], tok[1], tok[2], tok[3]};
            if (p.seq)
                *(i32x4_a4 *)(p.seq + j) = i32x4_a4{b, b, b, b};
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (k + q < size && j + q < p.capacity) {
                    if (p.slots)
                        p.slots[j + q] = slot[q];
                    if (p.positions)
                        p.positions[j + q] = i + q;
                    if (p.packed)
                        p.packed[j + q] = x[i + q];
                    if (p.seq)
                        p.seq[j + q] = b;
                }
        }
        before += size;
    }
}

// Accepted nodes' cache rows.  A lane moves the same piece (of sizeof(Vec)
// bytes) of every row of its sequence and plane, in path order: the row that
// node j moves to is the source of no later node (nodes ascend along the path,
// so a later source lies beyond j), and the lane itself has read it before if
// it was an earlier one's.  kAhead rows are read before the first of them is
// written, what is left behind those two at a time (a path of 20: 8, 8, 2, 2).
constexpr int kAhead = 8;

template <typename Vec>
__global__ __launch_bounds__(kThreads) void k_compact(CompactParams p) {
    __shared__ int16_t par[SWITCHSD_MAX_R];
    __shared__ int64_t slot[SWITCHSD_MAX_R];
    __shared__ int16_t path[SWITCHSD_MAX_R];  // node at depth d
    __shared__ int64_t src[SWITCHSD_MAX_R], dst[SWITCHSD_MAX_R];
    // bit i: node i does not follow node i - 1 (the anchor does not)
    __shared__ unsigned long long s_heads[SWITCHSD_MAX_R / 64];
    __shared__ int s_m;
    const int tid = threadIdx.x;
    const int b = blockIdx.x / p.blocks, blk = blockIdx.x - b * p.blocks;
    const int64_t base = (int64_t)b * p.R;
    const int n = clampi(p.dn[b], 1, p.R);
    const int a = p.accept_node[b];
    if (a <= 0 || a >= n)
        return;
    for (int i0 = 0; i0 <= a; i0 += kThreads) {
        const int i = i0 + tid;
        int q = -1;
        if (i <= a) {
            q = p.dpar[base + i];
            q = q >= 0 && q < i ? q : -1;
            par[i] = (int16_t)q;
            slot[i] = p.slots[base + i];
        }
        const unsigned long long heads = __ballot(i == 0 || q != i - 1);
        if ((tid & 63) == 0 && i < SWITCHSD_MAX_R)
            s_heads[i >> 6] = heads;
    }
    __syncthreads();
    if (tid < 64) {
        // the path, deepest node first, a run of nodes that follow each other
        // (within 64) at a time: chains and candidates are few runs (a path of 20
        // moved in 4.8 us, node by node in 5.7)
        int depth = 0, cur = a;
        while (cur > 0) {
            const int own = par[cur], top = cur & 63;
            const unsigned long long h = s_heads[cur >> 6] & (~0ull >> (63 - top));
            const int low = h ? cur - top + 63 - __builtin_clzll(h) : cur - top;
            const int run = cur - (low > 0 ? low : 1) + 1;
            if (tid < run)
                path[depth + tid] = (int16_t)(cur - tid);
            depth += run;
            cur = low == 0 ? 0 : low == cur ? own : par[low];
        }
        depth = cur == 0 ? depth : 0;
        // read by other lanes of the wave
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        // the moves that are any, in path order
        int m = 0;
        for (int j0 = 1; j0 <= depth; j0 += 64) {
            const int j = j0 + tid;
            int64_t from = 0, to = 0;
            bool move = false;
            if (j <= depth) {
                from = slot[path[depth - j]];
                to = slot[j];
                move = from != to && from >= 0 && from < p.n_slots && to >= 0 && to < p.n_slots;
            }
            const unsigned long long mask = __ballot(move);
            if (move) {
                const int k = m + __popcll(mask & ((1ull << tid) - 1ull));
                src[k] = from * p.row_vecs;
                dst[k] = to * p.row_vecs;
            }
            m += __popcll(mask);
        }
        if (tid == 0)
            s_m = m;
    }
    __syncthreads();
    const int m = s_m;
    const int64_t u = (int64_t)blk * kThreads + tid;
    if (m == 0 || u >= p.pieces)
        return;
    const int64_t plane = u / p.row_vecs;
    Vec *c = (Vec *)((char *)p.cache + plane * p.plane_stride) + (u - plane * p.row_vecs);
    int j = 0;
    for (; j + kAhead <= m; j += kAhead) {
        Vec v[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
            v[q] = c[src[j + q]];
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
            c[dst[j + q]] = v[q];
    }
    for (; j < m; j += 2) {
        const Vec v = c[src[j]], w = c[src[j + 1 < m ? j + 1 : j]];
        c[dst[j]] = v;
        if (j + 1 < m)
            c[dst[j + 1]] = w;
    }
}

}  // namespace

int launch_page_plan_kernel(const PageParams &p, hipStream_t stream) {
    const dim3 grid((unsigned)((p.B + p.seqs - 1) / p.seqs));
    if (p.R <= 64)
        hipLaunchKernelGGL(k_page_plan<true>, grid, dim3(kThreads), 0, stream, p);
    else
        hipLaunchKernelGGL(k_page_plan<false>, grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError() == hipSuccess ? SWITCHSD_OK : SWITCHSD_EHIP;
}

int launch_span_kernel(const SpanParams &p, hipStream_t stream) {
    const int64_t grid = (int64_t)((p.B + p.seqs - 1) / p.seqs) * p.parts;
    hipLaunchKernelGGL(k_span_slots, dim3((unsigned)grid), dim3(kThreads), 0, stream, p);
    return hipGetLastError() == hipSuccess ? SWITCHSD_OK : SWITCHSD_EHIP;
}

int launch_compact_kernel(const CompactParams &p, bool wide, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)p.B * p.blocks));
    if (wide)
        hipLaunchKernelGGL(k_compact<u32x4>, grid, dim3(kThreads), 0, stream, p);
    else
        hipLaunchKernelGGL(k_compact<uint32_t>, grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError() == hipSuccess ? SWITCHSD_OK : SWITCHSD_EHIP;
}

}  // namespace switchsd
