// switchsd_pages.hip -- gfx950 kernels for the bookkeeping of a paged KV cache
// around the speculation-control step: pages, slots and positions of the
// drafted rows (k_page_plan), packed slots of ragged ranges (k_span_slots) and
// the move of the accepted nodes' cache rows (k_compact).
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "switchsd_device.h"
#include "switchsd_internal.h"

namespace switchsd {

namespace {

constexpr int kWaves = kThreads / 64;

// Sum over the work-group of (a, b); every lane gets both sums.
__device__ __forceinline__ void block_sum2(int &a, int &b, int (&sh)[2][kWaves]) {
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        a += __shfl_xor(a, o);
        b += __shfl_xor(b, o);
    }
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
        sh[0][wave] = a;
        sh[1][wave] = b;
    }
    __syncthreads();
    a = b = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        a += sh[0][w];
        b += sh[1][w];
    }
    __syncthreads();
}

// Inclusive sums over the work-group's lanes of (a, b).
__device__ __forceinline__ void block_scan2(int &a, int &b, int (&sh)[2][kWaves]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int pa = __shfl_up(a, o), pb = __shfl_up(b, o);
        if (lane >= o) {
            a += pa;
            b += pb;
        }
    }
    if (lane == 63) {
        sh[0][wave] = a;
        sh[1][wave] = b;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w)
        if (w < wave) {
            a += sh[0][w];
            b += sh[1][w];
        }
    __syncthreads();
}

// What sequence b asks of the ring: its length and nodes, the pages it holds,
// lacks (grow) and gives back (back).  B * max_pages < 2^31, so sums of them
// fit 32 bits.
struct Ask {
    int L, n, held, grow, back;
};
__device__ __forceinline__ Ask page_ask(const PageParams &p, int b) {
    Ask a;
    a.L = clampi(p.lengths[b], 0, p.Lmax);
    a.n = clampi(p.dn[b], 1, p.R);
    a.held = clampi(p.held[b], 0, p.max_pages);
    a.grow = a.back = 0;
    if (a.L > 0) {
        const uint32_t need =
            ((uint32_t)(a.L - 1) + (uint32_t)a.n + (uint32_t)p.page_size - 1u) /
            (uint32_t)p.page_size;
        const int pages = need < (uint32_t)p.max_pages ? (int)need : p.max_pages;
        a.grow = pages > a.held ? pages - a.held : 0;
    } else {
        a.back = a.held;
    }
    return a;
}

// Pages, slots and positions.  Work-group g plans the sequences from g *
// seqs on (seqs * R <= kPlanNodes, or one sequence): it sums what all earlier
// sequences lack and give back, so that no work-group waits for another, and
// the last one to arrive, when every one has read held and the ring's state,
// writes both anew.  A page taken in this call is read from the ring, where
// nothing is written in this call that is read from it: returned pages go
// behind the free ones, and free and held pages together fit the ring.
__global__ __launch_bounds__(kThreads) void k_page_plan(PageParams p) {
    __shared__ int red[2][kWaves];
    __shared__ uint32_t st[2][kPlanNodes];
    __shared__ int s_L[kThreads], s_n[kThreads], s_held[kThreads], s_first[kThreads],
        s_took[kThreads], s_back[kThreads], s_bfirst[kThreads];
    __shared__ int s_last;
    const int tid = threadIdx.x;
    const int b0 = blockIdx.x * p.seqs;
    const int ns = p.B - b0 < p.seqs ? p.B - b0 : p.seqs;
    const int head = clampi(p.ring_state[0], 0, p.ring_pages - 1);
    const int count = clampi(p.ring_state[1], 0, p.ring_pages);
    int ga = 0, ba = 0;  // of the sequences before b0
    for (int b = tid; b < b0; b += kThreads) {
        const Ask a = page_ask(p, b);
        ga += a.grow;
        ba += a.back;
    }
    block_sum2(ga, ba, red);
    {
        Ask a = {0, 0, 0, 0, 0};
        if (tid < ns)
            a = page_ask(p, b0 + tid);
        int g = a.grow, k = a.back;
        block_scan2(g, k, red);
        if (tid < ns) {
            const bool served = ga + g <= count;
            s_L[tid] = a.L;
            s_n[tid] = a.n;
            s_held[tid] = a.held;
            s_first[tid] = ga + g - a.grow;
            s_took[tid] = served ? a.grow : 0;
            s_back[tid] = a.back;
            s_bfirst[tid] = ba + k - a.back;
            p.missing[b0 + tid] = served ? 0 : a.grow;
        }
    }
    __syncthreads();
    // pages taken and given back, a wave per sequence
    for (int s = tid >> 6; s < ns; s += kWaves) {
        int32_t *row = p.table + (int64_t)(b0 + s) * p.max_pages;
        const int held = s_held[s], took = s_took[s], back = s_back[s];
        for (int j = tid & 63; j < took; j += 64)
            row[held + j] = p.ring[((uint32_t)head + (uint32_t)(s_first[s] + j)) %
                                   (uint32_t)p.ring_pages];
        for (int j = tid & 63; j < back; j += 64) {
            const int64_t at = (int64_t)count + s_bfirst[s] + j;
            if (at < p.ring_pages)
                p.ring[((uint32_t)head + (uint32_t)at) % (uint32_t)p.ring_pages] = row[j];
            row[j] = -1;
        }
    }
    // depths by pointer jumping: every edge holds that leads to a valid parent
    const int nodes = ns * p.R;
    if (p.positions && p.dpar) {
        for (int i = tid; i < nodes; i += kThreads) {
            const int s = i / p.R, r = i - s * p.R;
            const int q = r < s_n[s] ? p.dpar[(int64_t)b0 * p.R + i] : -1;
            const bool up = q >= 0 && q < r;
            // a path ends at the node whose parent is not valid, as at the anchor
            st[0][i] = up ? kHolds | (1u << 16) | (uint32_t)q : kHolds | (uint32_t)r;
        }
        __syncthreads();
    }
    int cur = 0;
    if (p.positions && p.dpar) {
        for (bool open = true; open; cur ^= 1) {
            bool more = false;
            for (int i = tid; i < nodes; i += kThreads) {
                const uint32_t s1 = st[cur][i];
                const int s = i / p.R;
                const uint32_t s2 = st[cur][s * p.R + (int)(s1 & 0xFFFFu)];
                st[cur ^ 1][i] = jump_compose(s1, s2);
                more |= (s1 & 0xFFFFu) != (s2 & 0xFFFFu);
            }
            open = __syncthreads_or(more);
        }
    }
    for (int i = tid; i < nodes; i += kThreads) {
        const int s = i / p.R, r = i - s * p.R;
        const int64_t o = (int64_t)b0 * p.R + i;
        const bool live = s_L[s] > 0 && r < s_n[s];
        if (p.positions) {
            const int depth = p.dpar ? (int)((st[cur][i] >> 16) & 0x7FFFu) : r;
            p.positions[o] = live ? s_L[s] - 1 + depth : -1;
        }
        if (p.slots) {
            int64_t slot = -1;
            if (live) {
                const uint32_t at = (uint32_t)(s_L[s] - 1 + r);
                const uint32_t pg = at / (uint32_t)p.page_size;
                const int held = s_held[s];
                int page = -1;
                bool have = false;
                if (pg < (uint32_t)held) {
                    page = p.table[(int64_t)(b0 + s) * p.max_pages + pg];
                    have = true;
                } else if (pg < (uint32_t)(held + s_took[s])) {
                    page = p.ring[((uint32_t)head + (uint32_t)(s_first[s] + (int)pg - held)) %
                                  (uint32_t)p.ring_pages];
                    have = true;
                }
                if (have)
                    slot = (int64_t)page * p.page_size + (at - pg * (uint32_t)p.page_size);
            }
            p.slots[o] = slot;
        }
    }
    __syncthreads();
    if (tid < 64) {
        const bool last = arrive(p.ticket, gridDim.x);
        if (tid == 0)
            s_last = last;
    }
    __syncthreads();
    if (!s_last)
        return;
    // every work-group has read held and ring_state
    int gt = 0, bt = 0, popped = 0;
    for (int t0 = 0; t0 < p.B; t0 += kThreads) {
        const int b = t0 + tid;
        Ask a = {0, 0, 0, 0, 0};
        if (b < p.B)
            a = page_ask(p, b);
        int g = a.grow, k = a.back;
        block_scan2(g, k, red);
        const bool served = gt + g <= count;
        if (b < p.B && ((served && a.grow) || a.back))
            p.held[b] = a.L > 0 ? a.held + a.grow : 0;
        int pt = served ? a.grow : 0, gk = a.grow;
        block_sum2(pt, gk, red);
        popped += pt;
        gt += gk;
        int bk = a.back, z = 0;
        block_sum2(bk, z, red);
        bt += bk;
    }
    if (tid == 0) {
        p.ring_state[0] = (int)(((uint32_t)head + (uint32_t)popped) % (uint32_t)p.ring_pages);
        const int64_t left = (int64_t)count - popped + bt;
        p.ring_state[1] = left > p.ring_pages ? p.ring_pages : (int)left;
        st_u32(p.ticket, 0u);
    }
}

// Packed slots.  Work-group (sequence group g, part t) writes the t-th
// kSpanPart positions of each of its sequences' ranges, at the sum of all
// earlier sequences' sizes, which it takes itself.
__device__ __forceinline__ void span_of(const SpanParams &p, int b, int &lo, int &size) {
    const int hi = clampi(p.end[b], 0, p.Lmax);
    lo = clampi(p.begin[b], 0, hi);
    size = hi - lo;
}

__global__ __launch_bounds__(kThreads) void k_span_slots(SpanParams p) {
    __shared__ int red[2][kWaves];
    const int tid = threadIdx.x;
    const int g = blockIdx.x / p.parts, part = blockIdx.x - g * p.parts;
    const int b0 = g * p.seqs, b1 = b0 + p.seqs < p.B ? b0 + p.seqs : p.B;
    int before = 0, any = 0;
    for (int b = b0 + tid; b < b1; b += kThreads) {
        int lo, size;
        span_of(p, b, lo, size);
        any |= size > part * kSpanPart;
    }
    if (part > 0 && !__syncthreads_or(any))
        return;
    for (int b = tid; b < b0; b += kThreads) {
        int lo, size;
        span_of(p, b, lo, size);
        before += size;
    }
    int z = 0;
    block_sum2(before, z, red);
    for (int b = b0; b < b1; ++b) {
        int lo, size;
        span_of(p, b, lo, size);
        if (part == 0 && tid == 0) {
            p.cu[b] = before;
            if (b == p.B - 1)
                p.cu[p.B] = before + size;
        }
        const int held = p.slots ? clampi(p.held[b], 0, p.max_pages) : 0;
        const int k1 = size < (part + 1) * kSpanPart ? size : (part + 1) * kSpanPart;
        for (int k = part * kSpanPart + tid; k < k1; k += kThreads) {
            const int64_t j = (int64_t)before + k;
            if (j >= p.capacity)
                break;
            const int i = lo + k;
            if (p.slots) {
                const int pg = (int)((uint32_t)i / (uint32_t)p.page_size);
                int64_t slot = -1;
                if (pg < held)
                    slot = (int64_t)p.table[(int64_t)b * p.max_pages + pg] * p.page_size +
                           (i - pg * p.page_size);
                p.slots[j] = slot;
            }
            if (p.positions)
                p.positions[j] = i;
            if (p.packed)
                p.packed[j] = p.tokens[(int64_t)b * p.Lmax + i];
            if (p.seq)
                p.seq[j] = b;
        }
        before += size;
    }
}

// Accepted nodes' cache rows.  A lane moves the same piece (of sizeof(Vec)
// bytes) of every row of its sequence and plane, in path order: the row that
// node j moves to is the source of no later node (nodes ascend along the path,
// so a later source lies beyond j), and the lane itself has read it before if
// it was an earlier one's.
template <typename Vec>
__global__ __launch_bounds__(kThreads) void k_compact(CompactParams p) {
    __shared__ int64_t src[SWITCHSD_MAX_R], dst[SWITCHSD_MAX_R];
    __shared__ int s_m;
    const int tid = threadIdx.x;
    const int b = blockIdx.x / p.blocks, blk = blockIdx.x - b * p.blocks;
    const int64_t base = (int64_t)b * p.R;
    if (tid == 0) {
        const int n = clampi(p.dn[b], 1, p.R);
        const int a = p.accept_node[b];
        int depth = 0, m = 0;
        if (a > 0 && a < n) {
            int cur = a;
            while (cur > 0) {
                const int q = p.dpar[base + cur];
                if (q < 0 || q >= cur)
                    break;
                cur = q;
                ++depth;
            }
            if (cur != 0)
                depth = 0;
            cur = a;
            for (int j = depth; j > 0; --j) {
                const int64_t from = p.slots[base + cur], to = p.slots[base + j];
                const bool in = from >= 0 && from < p.n_slots && to >= 0 && to < p.n_slots;
                if (from != to && in) {
                    src[m] = from;
                    dst[m] = to;
                    ++m;
                }
                cur = p.dpar[base + cur];
            }
        }
        s_m = m;
    }
    __syncthreads();
    const int m = s_m;
    if (m == 0)
        return;
    const int64_t u = (int64_t)blk * kThreads + tid;
    if (u >= p.pieces)
        return;
    const int plane = (int)(u / p.row_vecs);
    const int64_t piece = u - (int64_t)plane * p.row_vecs;
    Vec *c = (Vec *)((char *)p.cache + (int64_t)plane * p.plane_stride) + piece;
    for (int j = m - 1; j >= 0; --j)  // path order: the list is deepest first
        c[dst[j] * p.row_vecs] = c[src[j] * p.row_vecs];
}

}  // namespace

int launch_page_plan_kernel(const PageParams &p, hipStream_t stream) {
    const int grid = (p.B + p.seqs - 1) / p.seqs;
    hipLaunchKernelGGL(k_page_plan, dim3((unsigned)grid), dim3(kThreads), 0, stream, p);
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
