// Block tables and slot maps from the requests' lengths, in one launch.
//
// need = ceil((len + new) / page); a request gives back held - need pages or takes need - held.  Where its pages lie in the
// list of free ones follows from two sums over the requests before it, so that every result is fixed by the inputs:
//   given back   free_list[n_free + (given by requests before) + k]             k = 0, 1, .. in page order
//   taken        free_list[total - 1 - (taken by requests before) - k]          total = n_free + all that is given back
// Every CTA works out both sums for all requests (a block scan; a few KB from L2) and then takes its share of pages and slots.  Nothing that a CTA
// looks up is written by another one: a page that one request gives back and another takes is read where the former held it, and not in the
// list.  Only counts that are brought up to date in place (held_out, n_free_out) have to wait until all CTAs have read them: those calls
// are one cluster, with a barrier.
//
// What bounds it: latency (lengths, scan, list, slots: dependent steps, and a launch); for prompts the 8 bytes a slot.  256 requests that grow by 16
// rows 8.2 us, 64 prompts of up to 8191 rows in pages of 64 6.5 us (4.2 MB of slots); in one cluster, as in place, 8.8 and 14.4.  The former
// has a hundredth of the slots and takes longer, because CTAs are as many as its slots ask for, two, and nine of its requests end: 4.7 us where no
// page moves, 5.5 where each request takes one (a search for its place in the list, by every slot on it), 8.0 where those are pages that are given back in
// the same call (a second search), 2250 in all; that on 32 CTAs 6.4.
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace orthrus {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kStretch = 256;                    // slots of a long row that a warp maps at a time

struct Entry { uint32_t gives, takes; int need, held; };       // sums before / up to and with the request; need < 0: left alone

__device__ inline unsigned long long warp_scan(unsigned long long x, int lane)
{
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    return x;
}

__global__ void __launch_bounds__(kThreads, 1) page_tables_kernel(const PageTablesParams p, int per, bool in_place)
{
    extern __shared__ Entry entry[];
    __shared__ unsigned long long sum[2][kWarps];
    __shared__ unsigned upto;                    // pages taken by the requests that are served
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = gridDim.x, rank = blockIdx.x;
    if (tid == 0) upto = 0;
    pdl_begin();

    // sums over the requests: a thread's own `per` ones, then the block's
    unsigned long long g = 0, t = 0;
    int flags = 0;
    const int b0 = min(tid * per, p.B), b1 = min(b0 + per, p.B);
    for (int b = b0; b < b1; ++b) {
        const int len = p.cache_len[b], add = p.n_new[b], held = p.held_in[b];
        const long long need = ((long long)len + add + (1 << p.page_shift) - 1) >> p.page_shift;
        const bool ok = len >= 0 && add >= 0 && add <= p.max_new && held >= 0 && held <= p.max_pages && need <= p.max_pages;
        if (!ok) flags |= ORTHRUS_DEV_BAD_CACHE_LEN;
        entry[b] = Entry{0, 0, ok ? (int)need : -1, held};
        if (ok && need < held) g += held - need;
        if (ok && need > held) t += need - held;
    }
    unsigned long long gs = warp_scan(g, lane), ts = warp_scan(t, lane);
    if (lane == 31) { sum[0][warp] = gs; sum[1][warp] = ts; }
    __syncthreads();
    if (warp < 2) sum[warp][lane] = warp_scan(sum[warp][lane], lane);
    __syncthreads();
    gs += (warp ? sum[0][warp - 1] : 0) - g;
    ts += (warp ? sum[1][warp - 1] : 0) - t;
    const unsigned long long given = sum[0][kWarps - 1];
    int n_free = *p.n_free_in;
    if (n_free < 0 || n_free > p.n_pages || given > (unsigned long long)(p.n_pages - n_free)) flags |= ORTHRUS_DEV_NO_PAGES;
    n_free = min(max(n_free, 0), p.n_pages);
    const unsigned total = (unsigned)min((unsigned long long)p.n_pages, n_free + given);
    unsigned most = 0;
    for (int b = b0; b < b1; ++b) {
        Entry e = entry[b];
        const int change = e.need < 0 ? 0 : e.need - e.held;
        if (change > 0) ts += change;
        e.gives = (uint32_t)min(gs, 0xffffffffull);
        e.takes = (uint32_t)min(ts, 0xffffffffull);
        if (change < 0) gs -= change;
        if (change > 0) {
            if (e.takes <= total) most = e.takes;
            else { e.need = -2; flags |= ORTHRUS_DEV_NO_PAGES; }        // not served
        }
        entry[b] = e;
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0 && most) atomicMax(&upto, most);
    flags = __reduce_or_sync(0xffffffffu, (unsigned)flags);
    if (flags && lane == 0 && rank == 0 && p.status) atomicOr(p.status, flags);
    __syncthreads();

    // Page number t of all that are given back, or taken, is a thread's; whose it is, a search in the sums tells.
    auto request_of = [&](unsigned t, auto upto) {             // the first request that upto(request) is above t for
        int lo = 0, n = p.B;
#pragma unroll 1
        while (n > 1) {
            const int half = n >> 1;
            if (upto(lo + half - 1) <= t) { lo += half; n -= half; }
            else n = half;
        }
        return lo;
    };
    const unsigned mine = rank * kThreads + tid, all = C * kThreads;
    const unsigned n_given = (unsigned)min(given, (unsigned long long)(p.n_pages - n_free));
    // where page number t of those that are given back is
    auto given_page = [&](unsigned t) -> const int32_t * {
        const int b = request_of(t, [&](int i) { const Entry &e = entry[i]; return e.gives + (e.need >= 0 ? max(e.held - e.need, 0) : 0); });
        const Entry e = entry[b];
        return p.table + (long long)b * p.max_pages + e.need + (t - e.gives);
    };
#pragma unroll 1
    for (unsigned t = mine; t < n_given; t += all) p.free_list[n_free + t] = __ldcg(given_page(t));
    // where page number t of those that are taken, from the end of the list, is
    auto taken = [&](unsigned t) -> const int32_t * {
        const unsigned at = total - 1 - t;
        if (at < (unsigned)n_free) return p.free_list + at;
        return given_page(at - n_free);
    };
#pragma unroll 1
    for (unsigned t = mine; t < upto; t += all) {
        const int b = request_of(t, [&](int i) { return entry[i].takes; });
        const Entry e = entry[b];
        p.table[(long long)b * p.max_pages + e.held + (t - (e.takes - (unsigned)(e.need - e.held)))] = __ldcg(taken(t));
    }
    // the page of position pos of a request: one that it held, or one that it gets
    auto page_of = [&](const Entry &e, const int32_t *held, int pos) {
        const int j = pos >> p.page_shift;
        return j < e.held ? held + j : taken(e.takes - (unsigned)(e.need - e.held) + (unsigned)(j - e.held));
    };
    const int page_mask = (1 << p.page_shift) - 1;
    if (p.max_new >= kStretch) {
        // long rows: a warp 256 slots of a request, eight lookups of a lane under way together
        const int stretches = (p.max_new + kStretch - 1) / kStretch;
#pragma unroll 1
        for (long long it = rank * kWarps + warp; it < (long long)p.B * stretches; it += C * kWarps) {
            const int b = (int)(it / stretches), i0 = (int)(it - (long long)b * stretches) * kStretch + lane;
            const Entry e = entry[b];
            const int len = p.cache_len[b], n = e.need < 0 ? 0 : p.n_new[b];
            const int32_t *held = p.table + (long long)b * p.max_pages;
            int64_t *out = p.slot_map + (long long)b * p.max_new;
            int32_t page[kStretch / 32];
#pragma unroll
            for (int k = 0; k < kStretch / 32; ++k) page[k] = i0 + k * 32 < n ? __ldcg(page_of(e, held, len + i0 + k * 32)) : -1;
#pragma unroll
            for (int k = 0; k < kStretch / 32; ++k) {
                const int i = i0 + k * 32;
                if (i < p.max_new) out[i] = i < n ? ((long long)page[k] << p.page_shift) + ((len + i) & page_mask) : -1;
            }
        }
    } else {
        // short ones: a thread one at a time of all requests' rows laid end to end, so that all threads are busy
        const long long n_slots = (long long)p.B * p.max_new;
        const int step_b = (int)(all / (unsigned)p.max_new), step_i = (int)(all % (unsigned)p.max_new);
        int b = (int)(mine / (unsigned)p.max_new), i = (int)(mine % (unsigned)p.max_new);
#pragma unroll 4
        for (long long it = mine; it < n_slots; it += all) {
            const Entry e = entry[b];
            const int len = p.cache_len[b], n = e.need < 0 ? 0 : p.n_new[b];
            p.slot_map[it] = i < n ? ((long long)__ldcg(page_of(e, p.table + (long long)b * p.max_pages, len + i)) << p.page_shift) + ((len + i) & page_mask) : -1;
            b += step_b;
            i += step_i;
            if (i >= p.max_new) { i -= p.max_new; ++b; }
        }
    }
    if (in_place) cluster_sync_all();
    for (int r = (int)mine; r < p.B; r += (int)all) {
        const Entry e = entry[r];
        p.granted[r] = e.need < 0 ? 0 : p.n_new[r];
        p.held_out[r] = e.need < 0 ? e.held : e.need;
    }
    if (rank == 0 && tid == 0) *p.n_free_out = (int)(total - upto);
}

}  // namespace

cudaError_t launch_page_tables(const PageTablesParams &p, cudaStream_t st)
{
    // CTAs by the slots to write
    const long long slots = (long long)p.B * p.max_new;
    const bool in_place = p.held_out == p.held_in || p.n_free_out == p.n_free_in;
    int C;
    if (in_place) {
        C = slots <= 8192 ? 1 : slots <= 32768 ? 4 : 8;
        if (slots > 131072 && clusters_resident(16, 1) > 0) C = 16;
    } else {
        const long long want = (slots + 2047) / 2048;
        C = (int)(want < num_sms() ? want : num_sms());
    }
    static std::atomic<uint64_t> done{0};
    const int smem = p.B * (int)sizeof(Entry);
    const cudaError_t e = configure(page_tables_kernel, done, 8192 * (int)sizeof(Entry), true);
    if (e != cudaSuccess) return e;
    const int per = (p.B + kThreads - 1) / kThreads;
    return in_place ? launch_clusters(true, C, page_tables_kernel, dim3(C), kThreads, smem, st, p, per, true)
                    : launch_clusters(true, 1, page_tables_kernel, dim3(C), kThreads, smem, st, p, per, false);
}

}  // namespace orthrus
