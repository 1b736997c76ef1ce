// Attention over the pages of a paged cache, bf16, head_dim 64 and 128, on tcgen05: one new token a request, blocks of either view.
//
//   S [128 rows x 64 keys] = Q K^T          O [128 rows x d] += P V,  P = 2^(S scale - reference)          (S scale in the log2 domain)
//
// One pass over the keys with a running reference and sum; a unit is a request, a KV head and up to 128 of its query rows (G heads by K
// block positions).  Rows that a unit does not have are padding of the MMA, but cost no softmax.
//
// What bounds it: HBM, 4 d bytes per key and KV head, up to some 64 rows; then the softmax (64 exponentials a row and tile) and the MMAs.  For a
// decoding step of 4 to 16 rows warp-level MMAs of 16 rows were built first and taken out: they spend more instructions on a tile than
// one thread here that issues it (32 requests of 1024 to 8192 keys, 4 rows: 109 us against 94).
//
// Work is cut by tiles of 64 keys, not by requests: all tiles of all units lie on one line, and CTA c of n takes the stretch
// [c T / n, (c + 1) T / n).  Every CTA finds its stretch from the lengths themselves, so that the host needs no plan, a captured graph serves any
// lengths, and a batch of unequal requests loads all SMs alike.  A unit that is cut leaves pieces (unnormalised sums with their
// reference) in the workspace; the CTA that finishes last, by the unit's count, joins them in the order of their keys, which fixes the result.
//
// CTA of 192 threads, 113 KB of shared memory and 256 TMEM columns: two fit an SM, so that one's softmax overlaps the other's products, and the
// next call's CTAs can be resident early.
//   warps 0-3  softmax, thread = query row: scores from tensor memory, probabilities back to it as bf16 in their place; also the
//              query rows' way into shared memory, the read-out, and the join
//   warp 4     producer: looks up pages, K and V tiles into a ring of slots, a TMA box per page and 64 columns, running on into the
//              next unit of the stretch
//   warp 5     MMAs: the scores of the next tile are issued ahead of the product of this one
// A row's reference follows its maximum only when that has grown by more than 2^8 since: the output in tensor memory is rescaled rarely,
// numerator and denominator use the same reference, and probabilities stay below 2^8.
// Probabilities are rounded to bf16, the type of the values: the MMA takes operands of one type, and its rate with two products for each (a rounded
// part and the rest) would be half.  The sum is of the unrounded ones.  Outputs are then off by 2.3e-3 of their size in the mean, where their own
// rounding alone makes 1.7e-3 (2000 to 32768 keys).
// Every wait is bounded: on expiry the CTA raises ORTHRUS_DEV_WAIT_TIMEOUT, waits for its copies and MMAs in flight and ends.
#include <cuda.h>
#include <type_traits>
#include "paged_stretch.cuh"

namespace orthrus {
namespace {

constexpr int MROWS = 128, PRODUCER = 4, MMA = 5, NTHREADS = 192;
constexpr float kSlack = 8.f;             // log2 of what a probability may be

__device__ inline void bar_softmax() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ inline bool bar_softmax_and(bool ok) {
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.and.pred q, 1, 128, p;\n"
                 " selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"((uint32_t)ok) : "memory");
    return r != 0;
}

// QR: query rows that have a place, and rows of the products; rows that a unit does not have are whatever lies there, and nobody reads their
// results.  Products of 64 rows have 16 of them in each warp's part of tensor memory (EACH), and take less power than ones of 128, which counts
// where the power limit sets the clock: 32 requests of 1024 to 8192 keys, 4 rows, call after call for a second, 104 us at 1.39 GHz with 128 rows,
// 91 at 1.70 with 64 (a single call 89 either way).
template <int HD, int QR> struct Shape {
    static constexpr int EACH = QR / 4;
    static constexpr int PANELS = HD / 64, QSUB = QR * 128, SUB = KT * 128, SLOT = PANELS * SUB;   // bytes
    static constexpr int NSLOT = (113 * 1024 - PANELS * QSUB - 512) / SLOT;
    static constexpr int OFF_Q = 0, OFF_RING = PANELS * QSUB, OFF_BAR = OFF_RING + NSLOT * SLOT;
    // barriers: slots full, slots empty, scores (two buffers), probabilities (two), a product done, query rows, all products of a
    // unit done (a waiter at the unit's end may find the barrier of the single ones two phases behind), drained
    static constexpr int FULL = 0, EMPTY = NSLOT, SCORES = 2 * NSLOT, PROBS = SCORES + 2, PRODUCT = PROBS + 2, QUERY = PRODUCT + 1,
                         DONE = QUERY + 1, DRAIN = DONE + 1, BARS = DRAIN + 1;
    static constexpr int OFF_MISC = OFF_BAR + BARS * 8, SMEM = OFF_MISC + 16;
    static constexpr uint32_t TM_S = HD, TM_COLS = 256;            // O, then two buffers of scores
    // Up to half as many query rows as have a place: the next unit's go to the other half while this one's are in use, and its first scores follow the
    // last product of this one.  AHEAD: bytes to the other half.  (256 requests of 100 to 500
    // keys 84.2 us without, 80.7 with; 64 of 100 to 4000 93.9 and 90.2.)
    static constexpr int AHEAD_ROWS = QR == 64 ? 32 : 0, AHEAD = QSUB / 2;
    // the join: references and sums of the pieces [piece][row], in the place of the unit's query rows: of all, or of half of each panel
    static constexpr int JOIN = PANELS * QSUB;
    static_assert(NSLOT >= 5 && 2 * (SMEM + 1024) <= 228 * 1024, "two CTAs per SM");
};

template <int HD, int QR>
__global__ void __launch_bounds__(NTHREADS, 2)
paged_attend_tc_kernel(const __grid_constant__ PagedParams p, const __grid_constant__ PagedMaps tm, const __grid_constant__ PagedWork w)
{
    using C = Shape<HD, QR>;
    constexpr int NSLOT = C::NSLOT, PANELS = C::PANELS;
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t sbase = smem_u32(smem);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + C::OFF_MISC);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + C::OFF_MISC + 4);
    int *last_flag = reinterpret_cast<int *>(smem + C::OFF_MISC + 8);
    auto bar = [&](int i) { return sbase + C::OFF_BAR + i * 8; };
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (warp == MMA) {
        if (lane == 0) {
            *abort_flag = (sbase & 1023u) == 0 ? 0 : 1;      // swizzled tiles need 1 KB alignment
            for (int i = 0; i < C::BARS; ++i) mbar_init(bar(i), i == C::PROBS || i == C::PROBS + 1 || i == C::QUERY ? 4 : 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            fence_proxy_async();
        }
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(tmem_slot)), "r"(C::TM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const int U = p.Hkv * w.row_tiles, page = 1 << p.page_shift;
    const bool ahead = w.rows <= C::AHEAD_ROWS;
    Stretch s;
    Piece x;
    // tile number T of the CTA: K in ring item 2 T, V in 2 T + 1; item j in slot j % NSLOT
    if (warp == PRODUCER) {
        // ------------------------------------------------------------------ producer
        bool waited = false;
        auto wait = [&] { griddep_wait(); griddep_launch(); waited = true; };
        int items = 0;
        if (lane == 0) { prefetch_map(&tm.k); prefetch_map(&tm.v); }
        // The stretch is looked for ahead of the wait.  Unless the lengths are promised, it is a guess, which is made again behind the wait if they
        // have changed; the pages are looked up behind it.
        PageWindow pages;
        bool have;
#pragma unroll 1
        for (bool again = false; ; again = true) {
            s = find_stretch(p, U, w.most_pieces);
            have = next_piece(p, s, lane, x);
            if (!p.quiescent && !again) wait();
            if (have) pages.open(p, x, lane);
            if (p.quiescent || again || still_so(p, s, lane)) break;
        }
        const uint64_t policy = policy_evict_first();
        const int box = 1 << w.box_shift;
        bool ok = true;
        while (ok && have) {
            const int h = x.u / w.row_tiles, keys = x.P + x.n;
            for (int t = x.t0; ok && t < x.t1; ++t) {
                const int pos0 = t * KT;
                if (!waited && pos0 + KT > x.P) wait();                                   // rows of the block itself
                const int last = min(pos0 + KT, keys) - 1;
                const int i = lane & 3, pan = lane >> 2;                                  // lane: box and panel
                const int pos = pos0 + (i << w.box_shift), pg = pages.page(p, pos, last, lane);
                const int live = ((last - pos0) >> w.box_shift) + 1;
                const int row = ((pg * p.Hkv + h) << p.page_shift) + (pos & (page - 1));
#pragma unroll
                for (int kind = 0; kind < 2; ++kind) {
                    const int slot = items % NSLOT;
                    if (items >= NSLOT) ok = mbar_wait_warp_call(bar(C::EMPTY + slot), (items / NSLOT + 1) & 1, abort_flag);
                    if (!ok) break;
                    if (lane == 0) mbar_expect_tx(bar(C::FULL + slot), live * box * HD * 2);
                    __syncwarp();
                    if (lane < 4 * PANELS && i < live)
                        tma_load_2d(sbase + C::OFF_RING + slot * C::SLOT + pan * C::SUB + i * (box * 128), kind ? &tm.v : &tm.k, pan * 64, row,
                                    bar(C::FULL + slot), policy);
                    __syncwarp();
                    ++items;
                }
            }
            have = ok && next_piece(p, s, lane, x);
            if (have) pages.open(p, x, lane);
        }
        if (!waited) wait();
        if (*abort_flag && lane == 0)                   // the last copies, before the block can end
            for (int k = max(0, items - NSLOT); k < items; ++k) mbar_wait_long(bar(C::FULL + k % NSLOT), (k / NSLOT) & 1);
        __syncwarp();
    } else if (warp == MMA) {
        // ------------------------------------------------------------------ MMAs
        constexpr uint32_t IDESC_QK = make_idesc(KT, 0, QR), IDESC_PV = make_idesc(HD, 1, QR);
        const uint64_t q_desc = make_desc(sbase + C::OFF_Q, 16, 1024);
        uint32_t q_at = 0;                               // the unit's query rows, in 16 bytes
        bool ok = true;
#pragma unroll 1
        for (bool again = false; ; again = true) {
            s = find_stretch(p, U, w.most_pieces);
            if (!again) griddep_wait();
            if (again || still_so(p, s, lane)) break;
        }
        if (blockIdx.x == 0) tell_requests(p, lane);
        int T = 0, units = 0;
        auto full = [&](int item) { return mbar_wait_warp_call(bar(C::FULL + item % NSLOT), (item / NSLOT) & 1, abort_flag); };
        auto scores = [&](int T) {
            const int slot = 2 * T % NSLOT;
            if (elect_one()) {
                const uint64_t kd = make_desc(sbase + C::OFF_RING + slot * C::SLOT, 16, 1024);
                const uint32_t d = tmem + C::TM_S + (T & 1) * KT;
#pragma unroll
                for (int kk = 0; kk < HD / 16; ++kk)
                    umma_ss(d, q_desc + q_at + (((kk >> 2) * C::QSUB + (kk & 3) * 32) >> 4), kd + (((kk >> 2) * C::SUB + (kk & 3) * 32) >> 4), IDESC_QK, kk > 0);
                umma_commit(bar(C::EMPTY + slot));
                umma_commit(bar(C::SCORES + (T & 1)));
            }
            __syncwarp();
        };
        while (ok && next_piece(p, s, lane, x)) {
            const int tiles = x.t1 - x.t0;
            ok = mbar_wait_warp_call(bar(C::QUERY), units & 1, abort_flag) && full(2 * T);
            if (!ok) break;
            tc_fence_after();
            scores(T);
            for (int t = 0; t < tiles; ++t, ++T) {
                if (t + 1 < tiles) {
                    ok = full(2 * (T + 1));
                    if (!ok) break;
                    scores(T + 1);
                }
                ok = mbar_wait_warp_call(bar(C::PROBS + (T & 1)), (T >> 1) & 1, abort_flag) && full(2 * T + 1);
                if (!ok) break;
                tc_fence_after();
                const int slot = (2 * T + 1) % NSLOT;
                if (elect_one()) {
                    const uint64_t vd = make_desc(sbase + C::OFF_RING + slot * C::SLOT, C::SUB, 1024);
                    const uint32_t a = tmem + C::TM_S + (T & 1) * KT;
#pragma unroll
                    for (int kk = 0; kk < KT / 16; ++kk) umma_ts(tmem, a + kk * 8, vd + (kk * 2048 >> 4), IDESC_PV, t > 0 || kk > 0);
                    umma_commit(bar(C::EMPTY + slot));
                    umma_commit(bar(C::PRODUCT));
                    if (t == tiles - 1) umma_commit(bar(C::DONE));
                }
                __syncwarp();
            }
            ++units;
            if (ahead) q_at ^= C::AHEAD >> 4;
        }
        if (*abort_flag) {                              // the MMAs in flight, before their operands and tensor memory go
            if (elect_one()) umma_commit(bar(C::DRAIN));
            __syncwarp();
            mbar_wait_long(bar(C::DRAIN), 0);
        }
    } else {
        // ------------------------------------------------------------------ softmax
        const int r = lane < C::EACH ? warp * C::EACH + lane : MROWS;                    // (MROWS: none)
        const uint32_t mine = tmem + ((uint32_t)(warp * 32) << 16);
        int T = 0, units = 0;
        struct Rows { int h, r0, rows; long long at; };  // of a unit; `at`: this thread's query row
        auto open = [&](const Piece &x, uint32_t place) {
            Rows u;
            u.h = x.u / w.row_tiles, u.r0 = (x.u - u.h * w.row_tiles) * MROWS;
            u.rows = max(0, min(MROWS, x.n * p.G - u.r0));
            u.at = r < u.rows ? row_offset(p, x.b, u.h, u.r0 + r, HD) : 0;
            // into swizzled panels of 64 columns; a row that does not exist is left as it is
            const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(p.q) + u.at;
            const uint32_t dst = sbase + C::OFF_Q + place + r * 128;
            if (r < u.rows)
#pragma unroll
                for (int c = 0; c < HD / 8; ++c)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + (c >> 3) * C::QSUB + (((c & 7) ^ (r & 7)) << 4)), "l"(src + c * 8) : "memory");
            return u;
        };
        auto opened = [&] {                              // the rows are there
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::QUERY));
        };
        Piece y;                                         // the next unit, and its rows
        Rows next;
        uint32_t place = 0;                              // of this unit's rows
        bool have = false, ok = true;
#pragma unroll 1
        for (int look = 0; ; ++look) {                   // first and, if they have changed, second look at the lengths
            s = find_stretch(p, U, w.most_pieces);
            have = next_piece(p, s, lane, x);
            if (look == 0) griddep_wait();
            if (have) next = open(x, 0);
            if (look > 0 || still_so(p, s, lane)) break;
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
        if (have) opened();
#pragma unroll 1
        while (have) {
            const int h = next.h, r0 = next.r0, rows = next.rows, keys = x.P + x.n;
            const long long at = next.at;
            const bool at_work = warp * C::EACH < rows;       // (other warps have padding only)
            have = next_piece(p, s, lane, y);
            if (ahead && have) next = open(y, place ^ C::AHEAD);
            const int sees = p.causal ? min(keys, x.P + (r0 + r) / p.G + 1) : keys;
            float ref = -INFINITY, l = 0.f;
            for (int t = x.t0; t < x.t1; ++t, ++T) {
                const int pos0 = t * KT;
                const uint32_t ts = mine + C::TM_S + (T & 1) * KT;
                if (!mbar_wait_warp_call(bar(C::SCORES + (T & 1)), (T >> 1) & 1, abort_flag)) { ok = false; break; }
                tc_fence_after();
                if (at_work) {
                    uint32_t raw[KT];
                    float sc[KT];
                    tmem_ld<KT>(ts, raw);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < KT; ++j) sc[j] = __uint_as_float(raw[j]);
                    if (pos0 + KT > x.P) {               // some keys are the block's own, or do not exist
#pragma unroll
                        for (int j = 0; j < KT; ++j) sc[j] = pos0 + j < sees ? sc[j] : -INFINITY;
                    }
                    float top = max3(sc[0], sc[1], sc[2]);
#pragma unroll
                    for (int j = 3; j + 1 < KT; j += 2) top = max3(top, sc[j], sc[j + 1]);
                    top = r < rows ? fmaxf(top, sc[KT - 1]) * p.scale_log2 : -INFINITY;
                    const bool move = top > ref + kSlack || (ref == -INFINITY && top > -INFINITY);
                    if (__any_sync(0xffffffffu, move)) {
                        const float next = move ? top : ref, al = next == -INFINITY ? 1.f : ex2(ref - next);
                        ref = next;
                        l *= al;
                        if (t > x.t0) {
                            // the products so far, which are the sums up to the tile before
                            if (!mbar_wait_warp_call(bar(C::PRODUCT), (T - 1) & 1, abort_flag)) { ok = false; break; }
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < HD; c += 32) {
                                uint32_t o[32];
                                tmem_ld32(mine + c, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * al);
                                tmem_st32(mine + c, o);
                            }
                        }
                    }
                    const float from = r >= rows ? INFINITY : ref == -INFINITY ? 0.f : ref;      // (padding: no probability, which saves power)
                    uint32_t pk[KT / 2];
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < KT; j += 2) {
                        const float a = ex2(fmaf(sc[j], p.scale_log2, -from)), b = ex2(fmaf(sc[j + 1], p.scale_log2, -from));
                        sum[(j >> 1) & 3] += a + b;
                        pk[j >> 1] = pack_bf16(a, b);
                    }
                    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    tmem_st32(ts, pk);
                    tmem_st_wait();
                }
                if (pos0 + KT > keys) {
                    // rows behind the last key, which may hold anything: zero, for the product with their zero probabilities
                    const int item = 2 * T + 1, slot = item % NSLOT;
                    if (!mbar_wait_warp_call(bar(C::FULL + slot), (item / NSLOT) & 1, abort_flag)) { ok = false; break; }
                    const int n0 = keys - pos0, n = (KT - n0) * (HD / 8);
                    for (int e = tid; e < n; e += 128) {
                        const int row = n0 + e / (HD / 8), c = e % (HD / 8);
                        *reinterpret_cast<uint4 *>(smem + C::OFF_RING + slot * C::SLOT + (c >> 3) * C::SUB + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(C::PROBS + (T & 1)));
            }
            if (ok && ahead && have) opened();
            if (ok) ok = mbar_wait_warp_call(bar(C::DONE), units & 1, abort_flag);
            ++units;
            ok = bar_softmax_and(ok);              // (a warp whose wait ran out has come here too: all leave together)
            if (!ok) break;
            tc_fence_after();
            // this thread's row of the output, 64 columns at a time
            auto read_out = [&](auto put) {
#pragma unroll 1
                for (int c = 0; c < HD; c += 64) {
                    uint32_t o[64];
                    tmem_ld<64>(mine + c, o);
                    tmem_ld_wait();
                    put(c, o);
                }
                tc_fence_before();
            };
            const bool uncut = x.t0 == 0 && x.t1 == x.tiles;
            if (uncut && at_work) {
                const float inv = 1.f / l;
                read_out([&](int c, const uint32_t (&o)[64]) {
#pragma unroll
                    for (int j = 0; j < 64; j += 8) {
                        auto two = [&](int i) { return pack_bf16(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv); };
                        st_global_if(r < rows, static_cast<__nv_bfloat16 *>(p.out) + at + c + j, make_uint4(two(j), two(j + 2), two(j + 4), two(j + 6)));
                    }
                });
            }
            if (!uncut) {
                // a piece: [four columns][row], so that a warp's store is 512 contiguous bytes
                const size_t step = piece_floats(w.rows, HD), stats = (size_t)w.rows * HD;
                if (at_work) {
                    float *to = w.pieces + (2 * blockIdx.x + (x.first ? 0 : 1)) * step;
                    if (r < rows) *reinterpret_cast<float2 *>(to + stats + r * 2) = make_float2(ref, l);
                    read_out([&](int c, const uint32_t (&o)[64]) {
#pragma unroll
                        for (int j = 0; j < 64; j += 4)
                            st_global_if(r < rows, to + ((size_t)(c + j) / 4 * w.rows + r) * 4, make_uint4(o[j], o[j + 1], o[j + 2], o[j + 3]));
                    });
                }
                const int c0 = owner(s, x.unit0), n = owner(s, x.unit0 + x.tiles - 1) - c0 + 1;
                bar_softmax();
                if (tid == 0) {
                    *last_flag = last_piece(p.status, c0, n);         // (no other cut unit begins in CTA c0)
                }
                // The join of the CTA that is the last.  Where things lie does not depend on it; vectors of four columns, a row a lane of them
                const int rs = rows > 1 ? 32 - __clz(rows - 1) : 0;                      // log2 of the rows, rounded up
                const int vecs = HD / 4 << rs;
                const float *others = w.pieces + 2 * c0 * step, *first = others + (stretch_start(s, c0) == x.unit0 ? 0 : step);
                auto piece = [&](int k) { return k ? others + 2 * k * step : first; };
                bar_softmax();
                if (*last_flag && rows > 0) {
                    // [piece][row]: references and sums, in the place of the unit's query rows
                    auto st = [&](int e) -> float2 & {
                        const int to = ahead ? place + (e * 8 / C::AHEAD) * C::QSUB + e * 8 % C::AHEAD : e * 8;
                        return *reinterpret_cast<float2 *>(smem + C::OFF_Q + to);
                    };
                    for (int e = tid; e < n << rs; e += 128) {
                        const int k = e >> rs, row = e & ((1 << rs) - 1);
                        if (row < rows) st(e) = __ldcg(reinterpret_cast<const float2 *>(piece(k) + stats) + row);
                    }
                    // IT vectors of UN pieces under way together
                    auto sum_up = [&](auto it, auto un) {
                        constexpr int IT = decltype(it)::value, UN = decltype(un)::value;
#pragma unroll 1
                        for (int e0 = tid; e0 - tid < vecs; e0 += 128 * IT) {
                            float4 acc[IT];
                            float top[IT], sum[IT];
                            int row[IT], off[IT];
#pragma unroll
                            for (int i = 0; i < IT; ++i) {
                                const int e = e0 + i * 128;
                                row[i] = min(e & ((1 << rs) - 1), rows - 1);             // (rows and vectors that do not exist: another, not stored)
                                off[i] = min(e >> rs, HD / 4 - 1) * w.rows + row[i];
                                acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                                top[i] = -INFINITY;
                                sum[i] = 0.f;
                            }
#pragma unroll 1
                            for (int k0 = 0; k0 < n; k0 += UN) {
                                float4 y[UN][IT];
#pragma unroll
                                for (int u = 0; u < UN; ++u) {
                                    const float4 *src = reinterpret_cast<const float4 *>(piece(min(k0 + u, n - 1)));      // (likewise)
#pragma unroll
                                    for (int i = 0; i < IT; ++i) y[u][i] = __ldcg(src + off[i]);
                                }
                                if (k0 == 0) {
                                    if (e0 == tid) bar_softmax();                        // (the references are there)
#pragma unroll 4
                                    for (int k = 0; k < n; ++k)
#pragma unroll
                                        for (int i = 0; i < IT; ++i) top[i] = fmaxf(top[i], st((k << rs) + row[i]).x);
#pragma unroll
                                    for (int i = 0; i < IT; ++i) if (top[i] == -INFINITY) top[i] = 0.f;
                                }
#pragma unroll
                                for (int u = 0; u < UN; ++u)
                                    if (k0 + u < n)
#pragma unroll
                                        for (int i = 0; i < IT; ++i) {
                                            const float2 rf = st(((k0 + u) << rs) + row[i]);
                                            const float al = ex2(rf.x - top[i]);
                                            sum[i] = fmaf(rf.y, al, sum[i]);
                                            acc[i].x = fmaf(y[u][i].x, al, acc[i].x); acc[i].y = fmaf(y[u][i].y, al, acc[i].y);
                                            acc[i].z = fmaf(y[u][i].z, al, acc[i].z); acc[i].w = fmaf(y[u][i].w, al, acc[i].w);
                                        }
                            }
#pragma unroll
                            for (int i = 0; i < IT; ++i) {
                                const int e = e0 + i * 128;
                                if (e >= vecs || (e & ((1 << rs) - 1)) >= rows) continue;
                                const float inv = 1.f / sum[i];
                                *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.out) + row_offset(p, x.b, h, r0 + row[i], HD) + (e >> rs) * 4) =
                                    make_uint2(pack_bf16(acc[i].x * inv, acc[i].y * inv), pack_bf16(acc[i].z * inv, acc[i].w * inv));
                            }
                        }
                    };
                    if (vecs <= 256) sum_up(std::integral_constant<int, 2>(), std::integral_constant<int, 8>());
                    else sum_up(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
                    bar_softmax();                         // (the references' place is query rows' again)
                }
            }
            x = y;
            if (ahead) place ^= C::AHEAD;
            else if (have) { next = open(x, 0); opened(); }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    if (warp == MMA) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::TM_COLS));
    }
    if (tid == 0 && *abort_flag && p.status) atomicOr(p.status, ORTHRUS_DEV_WAIT_TIMEOUT);
}

template <int HD, int QR>
cudaError_t launch_one(const PagedParams &p, const PagedMaps &tm, const PagedWork &w, int ctas, cudaStream_t st)
{
    using C = Shape<HD, QR>;
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = configure(paged_attend_tc_kernel<HD, QR>, done, C::SMEM, false);
    if (e != cudaSuccess) return e;
    return launch_kernel(p.early, paged_attend_tc_kernel<HD, QR>, dim3(ctas), NTHREADS, C::SMEM, st, p, tm, w);
}

}  // namespace

bool page_map(const void *ptr, unsigned d, unsigned long long rows, unsigned box, CUtensorMap *out)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {d, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)d * 2};
    const cuuint32_t boxes[2] = {64, box}, estr[2] = {1, 1};
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(ptr), dims, strides, boxes, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool paged_tc_shape(const orthrus_paged_layer_t &L)
{
    if (L.dtype != ORTHRUS_BF16 || (L.head_dim != 64 && L.head_dim != 128) || L.page_size < 16) return false;
    const long long row_tiles = ((long long)L.n_q_heads / L.n_kv_heads * L.block + MROWS - 1) / MROWS;
    if ((long long)L.batch * L.n_kv_heads * row_tiles * (((long long)L.max_pages * L.page_size + KT - 1) / KT) > 0x7fffffffLL) return false;
    return (unsigned long long)L.n_pages * L.n_kv_heads * L.page_size < 0x7fffffffull && tc_driver_ok();
}

namespace {

int max_len_of(const orthrus_paged_layer_t &L)
{
    const long long n = L.max_len_hint > 0 ? (long long)L.max_len_hint : (long long)L.max_pages * L.page_size - L.block;
    return n > 0 ? (int)n : 0;
}

// Which kernel.  Calls of up to 128 query rows a unit that take a few times as long as a launch go to the keys kernel (attend_keys.cu, over
// pages), whose clusters meet through shared memory: CTAs per unit, or 0.  It gives every request as many CTAs as the longest may need; this
// file's kernel shares the lengths out, and starts and joins in some 5 us more.  Us a call, here and there, 8 KV heads of 4 query heads:
// one request of 2000, 4000, 16000, 32000 keys 10.7 and 5.8, 12.7 and 7.8, 23.9 and 20.2, 33.1 and 37.8; 8 of 500 to 4000 22.1 and
// 20.9, of 1000 to 8000 32.1 and 39.4 (all of 8000 48 and 43); 32 of 125 to 1000 25.2 and 20.9, of 250 to 2000 34.1 and 39.1; blocks of 16, 8 of 500
// to 4000 34.8 and 24.9, 4 of 2000 to 16000 56 and 44, 8 of those 68 and 83; one KV head, 16000 and 60000 keys 20.4 and 19.5, 42 and 67.
// Hence: up to 200 MB of keys and values at the bound (270 MB where rows are many), one request any number, and up to 12 tiles a CTA.
// The host knows the bound and not the lengths, and the line is drawn for unequal ones, where the keys kernel loses most (30 of 32 requests of 1024 to 8192
// keys 88 here and 157 there).  For equal ones it comes too early: 4 requests of 32768 keys, 64 query heads, 89.9 here and 78.4 there, call after call for
// a second at 1785 MHz and 948 W, 1965 MHz and 689 W; 8 of 16000 with 64 rows 99 and 88.
// A bound far above the lengths has its price too: 8 requests of 512 to 4096, blocks of 16, 4 KV heads, 15.4 us, 38 with a bound of 32768; one of
// 4096 9.2 and 15.7.
// ORTHRUS_TC_SMALL_ROWS=0 keeps all calls on this file's kernel, =1 puts there whatever fits (measurement knobs).
int keys_plan(const orthrus_paged_layer_t &L)
{
    const int G = L.n_q_heads / L.n_kv_heads, knob = small_rows_knob();
    if (knob == 0 || !keys_rows(L.head_dim, G, L.block)) return 0;
    const int kb = keys_kb_rows(L.head_dim, G, L.block), tiles = (L.block + kb - 1) / kb;
    if ((long long)L.n_kv_heads * tiles > 65535) return 0;                       // (a dimension of its grid)
    const int max_len = max_len_of(L), S = paged_keys_splits(L, max_len);
    if (S == 0 || knob > 0) return S;
    const long long bytes = 4LL * L.head_dim * L.batch * L.n_kv_heads * tiles * max_len;
    if (bytes > (G * L.block <= 16 ? 200000000LL : 270000000LL) && L.batch * tiles > 1) return 0;
    return ((long long)max_len + L.block + KT - 1) / KT <= 24LL * S ? S : 0;
}

// CTAs of a call, and what its workspace holds: from the shape and the host's bound on the lengths.
struct Grid { int ctas, row_tiles, rows, most_pieces; size_t bytes; };
Grid plan(const orthrus_paged_layer_t &L)
{
    Grid g;
    const int M = L.n_q_heads / L.n_kv_heads * L.block;
    g.row_tiles = (M + MROWS - 1) / MROWS;
    g.rows = M < MROWS ? M : MROWS;
    const long long units = (long long)L.batch * L.n_kv_heads * g.row_tiles;
    const long long tiles = units * (((long long)max_len_of(L) + L.block + KT - 1) / KT);
    // Two CTAs an SM; one where wide units are cut into more pieces than tiles are worth (8 KV heads, 8 requests of 2000 keys, 64 and 128
    // rows 33.5 and 50 us at two, 30.5 and 40 at one; 4 rows 20.6 and 24.6; 32 requests of 1024 to 8192, 64 rows 111 and 147)
    const long long sms = (g.rows <= 16 || tiles >= 32LL * num_sms() ? 2LL : 1LL) * num_sms(), most = sms < kCounts ? sms : kCounts;
    g.ctas = (int)(tiles < 1 ? 1 : tiles < most ? tiles : most);
    // pieces of a unit: what the join has room for, and no more than one CTA adds up in the time the others save
    int padded = 1;
    while (padded < g.rows) padded *= 2;
    const int place = L.head_dim == 128 ? g.rows <= 64 ? Shape<128, 64>::JOIN : Shape<128, 128>::JOIN
                                        : g.rows <= 64 ? Shape<64, 64>::JOIN : Shape<64, 128>::JOIN;
    const int room = (g.rows <= Shape<128, 64>::AHEAD_ROWS ? place / 2 : place) / (padded * 8);
    g.most_pieces = room < kMostPieces ? room : kMostPieces;
    g.bytes = 2 * (size_t)g.ctas * piece_floats(g.rows, L.head_dim) * sizeof(float);
    return g;
}
}  // namespace

size_t paged_tc_workspace_bytes(const orthrus_paged_layer_t &L) { return plan(L).bytes; }

cudaError_t launch_paged_attend_tc(const PagedParams &p, const orthrus_paged_layer_t &L, void *ws_body, cudaStream_t st)
{
    if (const int S = keys_plan(L)) return launch_paged_attend_keys(p, S, st);
    const Grid g = plan(L);
    PagedWork w;
    w.row_tiles = g.row_tiles;
    w.box_shift = p.page_shift < 6 ? p.page_shift : 6;
    w.rows = g.rows;
    w.most_pieces = g.most_pieces;
    w.pieces = static_cast<float *>(ws_body);
    PagedMaps tm;
    const unsigned long long rows = (unsigned long long)L.n_pages * L.n_kv_heads * L.page_size;
    if (!page_map(p.k_pages, p.d, rows, 1u << w.box_shift, &tm.k) || !page_map(p.v_pages, p.d, rows, 1u << w.box_shift, &tm.v))
        return cudaErrorInvalidValue;
    if (p.d == 128) return g.rows <= 64 ? launch_one<128, 64>(p, tm, w, g.ctas, st) : launch_one<128, 128>(p, tm, w, g.ctas, st);
    return g.rows <= 64 ? launch_one<64, 64>(p, tm, w, g.ctas, st) : launch_one<64, 128>(p, tm, w, g.ctas, st);
}

}  // namespace orthrus
