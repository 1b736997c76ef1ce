// Attention over the pages of a paged cache, bf16, head_dim 64 and 128: one new token a request, or a block of up to 64.
//
//   s_j = q . k_j * scale,   m = max s,   out = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m)      (s in the log2 domain)
//
// One pass over the keys with a running maximum and sum.  What bounds it: HBM, 4 d bytes per key and KV head; a decoding step has 1 to
// 16 query rows per KV head, 2 to 32 flops a byte, so that warp-level MMAs of 16 query rows, even half empty, take a tenth of the time
// the keys take to arrive.
//
// Work is cut by tiles of 64 keys, not by requests: all tiles of all units (request, KV head, tile of query rows) lie on one line, and
// CTA c of n takes the stretch [c T / n, (c + 1) T / n).  Every CTA finds its stretch from the lengths themselves, so that the host
// needs no plan, a captured graph serves any lengths, and a batch of unequal requests loads all SMs alike.  A unit that is cut leaves pieces
// (unnormalised sums with their maximum) in the workspace; the CTA that finishes last, by the unit's counter, joins them in the
// order of their keys, which fixes the result.
//
// CTA of 160 threads, two to an SM:
//   warp 4     producer: looks up pages, brings K and V tiles by TMA into a ring (a box per page, 64 rows at most, 128-byte
//              swizzle), running on into the next unit of the stretch while the consumers finish this one
//   warps 0-3  consumers: WR groups of 16 MT query rows, 4 / WR groups of keys of each tile; a warp keeps maximum, sum and
//              output of its own keys in registers and meets the others at the end of a unit only
// Every wait is bounded: on expiry the CTA raises ORTHRUS_DEV_WAIT_TIMEOUT, waits for its copies in flight and ends.
#include <cuda.h>
#include <cmath>
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace orthrus {
namespace {

constexpr int KT = 64;                    // keys per tile
constexpr int CW = 4, PRODUCER = 4, NTHREADS = 160;
constexpr int kLeast = 2;                 // tiles a CTA takes at least, while there are fewer than CTAs

__device__ inline void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ inline void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ inline void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ inline void tma_load_3d(uint32_t dst, const CUtensorMap *tm, int c0, int c1, int c2, uint32_t bar, uint64_t policy) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
                 " [%0], [%1, {%2, %3, %4}], [%5], %6;"
                 ::"r"(dst), "l"(tm), "r"(c0), "r"(c1), "r"(c2), "r"(bar), "l"(policy) : "memory");
}
__device__ inline void bar_consumers() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
// the same, telling whether all of the threads brought `ok`
__device__ inline bool bar_consumers_and(bool ok) {
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.and.pred q, 1, 128, p;\n"
                 " selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"((uint32_t)ok) : "memory");
    return r != 0;
}

struct PagedMaps { CUtensorMap k, v; };
struct PagedWork {
    int row_tiles;           // tiles of query rows of a (request, KV head)
    int box_shift;           // log2 of the rows of a TMA box: min(page, 64)
    int rows;                // query rows a piece holds: min(rows of a tile, K G)
    int *counter;            // [unit]: pieces that are in
    float *pieces;           // [2 CTAs][rows][d], behind them [rows][2] (maximum, sum)
};

// floats of a piece, a multiple of the 16 bytes it is moved in
__host__ __device__ constexpr size_t piece_floats(int rows, int d) { return ((size_t)rows * (d + 2) + 3) / 4 * 4; }

template <int HD, int MT, int WR> struct PagedShape {
    static constexpr int MR = 16 * MT * WR, WK = CW / WR, KW = KT / WK;       // rows of a tile; key groups, keys of one
    static constexpr int TILE = KT * HD * 2;                                  // bytes of a K or V tile
    // the query rows' place is the output's when a unit ends
    static constexpr int Q_BYTES = MR * HD * 2, BUF_BYTES = MR * HD * 4, STAT_BYTES = CW * 16 * MT * 4;
    static constexpr int REST = BUF_BYTES + STAT_BYTES + 2 * MR * 4;
    static constexpr int ROOM = (113 * 1024 - REST - 160) / (2 * TILE), STAGES = ROOM < 6 ? ROOM : 6;
    static constexpr int OFF_BUF = STAGES * 2 * TILE, OFF_Q = OFF_BUF, OFF_STAT = OFF_BUF + BUF_BYTES,
                         OFF_ML = OFF_STAT + STAT_BYTES, OFF_BAR = OFF_ML + 2 * MR * 4;
    static constexpr int SMEM = OFF_BAR + 3 * STAGES * 8 + 16;
    static_assert(STAGES >= 2 && SMEM <= 113 * 1024 && Q_BYTES <= BUF_BYTES, "shared memory of two CTAs");
};

// A CTA's stretch of the line of tiles, piece by piece.  Every warp walks it by itself.
struct Stretch {
    long long T, pos, end, base;     // all tiles; next tile; the stretch's end; first tile of request b
    int n, b, P, rows, tiles;        // CTAs at work; request: its prefix, rows of its block, tiles of one of its units
    int U;                           // units of a request
};
struct Piece { int b, u, P, n, t0, t1, tiles; long long unit0; bool first; };

__device__ inline int tiles_of(int P, int n) { return n > 0 ? (P + n + KT - 1) / KT : 0; }
__device__ inline void load_request(const PagedParams &p, Stretch &s)
{
    bool bad;
    paged_request(p, s.b, s.P, s.rows, bad);
    s.tiles = tiles_of(s.P, s.rows);
}
// `c`: this CTA.  False: nothing to do.
__device__ inline bool find_stretch(const PagedParams &p, int U, int c, int ctas, int lane, bool tell, Stretch &s)
{
    long long sum = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
        int P, n, t = 0;
        bool bad = false;
        if (b0 + lane < p.B) { paged_request(p, b0 + lane, P, n, bad); t = tiles_of(P, n); }
        if (tell && bad && p.status) atomicOr(p.status, ORTHRUS_DEV_BAD_CACHE_LEN);
        sum += __reduce_add_sync(0xffffffffu, (unsigned)t);
    }
    s.U = U;
    s.T = sum * U;
    const long long most = (s.T + kLeast - 1) / kLeast;
    s.n = (int)min((long long)ctas, max(most, 1ll));
    if (c >= s.n || s.T == 0) return false;
    s.pos = s.T * c / s.n;
    s.end = s.T * (c + 1) / s.n;
    // the request that the stretch begins in
    long long run = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
        int P, n, t = 0;
        bool bad;
        if (b0 + lane < p.B) { paged_request(p, b0 + lane, P, n, bad); t = tiles_of(P, n); }
        int upto = t;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += x;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, (run + upto) * U > s.pos);
        if (hit) {
            const int l = __ffs(hit) - 1;
            s.b = b0 + l;
            s.base = (run + __shfl_sync(0xffffffffu, upto - t, l)) * U;
            break;
        }
        run += __shfl_sync(0xffffffffu, upto, 31);
    }
    load_request(p, s);
    return true;
}
__device__ inline bool next_piece(const PagedParams &p, Stretch &s, long long start, Piece &x)
{
    if (s.pos >= s.end) return false;
    while (s.pos >= s.base + (long long)s.tiles * s.U) {
        s.base += (long long)s.tiles * s.U;
        ++s.b;
        load_request(p, s);
    }
    x.b = s.b; x.P = s.P; x.n = s.rows; x.tiles = s.tiles;
    x.u = (int)((s.pos - s.base) / s.tiles);
    x.unit0 = s.base + (long long)x.u * s.tiles;
    x.t0 = (int)(s.pos - x.unit0);
    x.t1 = (int)min((long long)s.tiles, x.t0 + (s.end - s.pos));
    x.first = s.pos == start;
    s.pos += x.t1 - x.t0;
    return true;
}
__device__ inline int owner(const Stretch &s, long long tile) { return (int)(((tile + 1) * s.n - 1) / s.T); }

template <int HD, int MT, int WR>
__global__ void __launch_bounds__(NTHREADS, 2)
paged_attend_kernel(const __grid_constant__ PagedParams p, const __grid_constant__ PagedMaps tm, const __grid_constant__ PagedWork w)
{
    using C = PagedShape<HD, MT, WR>;
    constexpr int STAGES = C::STAGES, TILE = C::TILE, MR = C::MR, WK = C::WK, KW = C::KW, NK = KW / 8, ND = HD / 8;
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t sbase = smem_u32(smem);
    float *buf = reinterpret_cast<float *>(smem + C::OFF_BUF);
    float *stat = reinterpret_cast<float *>(smem + C::OFF_STAT);       // [warp][row of the warp]: maxima
    float *ml = reinterpret_cast<float *>(smem + C::OFF_ML);           // [row]: maximum, then [row]: sum
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + C::OFF_BAR + 3 * STAGES * 8);
    int *last_flag = reinterpret_cast<int *>(smem + C::OFF_BAR + 3 * STAGES * 8 + 4);
    auto bar_k = [&](int s) { return sbase + C::OFF_BAR + s * 8; };
    auto bar_v = [&](int s) { return sbase + C::OFF_BAR + (STAGES + s) * 8; };
    auto bar_free = [&](int s) { return sbase + C::OFF_BAR + (2 * STAGES + s) * 8; };
    auto at = [](int r, int c) { return r * HD + (c ^ ((r & 3) << 3)); };     // output row r, column c: rows shifted against one another
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 0) {
        *abort_flag = (sbase & 1023u) == 0 ? 0 : 1;      // swizzled tiles need 1 KB alignment
        for (int s = 0; s < STAGES; ++s) { mbar_init(bar_k(s), 1); mbar_init(bar_v(s), 1); mbar_init(bar_free(s), CW); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    __syncthreads();
    const int U = p.Hkv * w.row_tiles, page = 1 << p.page_shift;
    Stretch s;
    Piece x;

    if (warp == PRODUCER) {
        // ------------------------------------------------------------------ producer
        bool waited = false;
        auto wait = [&] { griddep_wait(); griddep_launch(); waited = true; };
        if (!p.quiescent) wait();
        int issued = 0;
        if (find_stretch(p, U, blockIdx.x, gridDim.x, lane, blockIdx.x == 0, s)) {
            const long long start = s.pos;
            const uint64_t policy = policy_evict_first();
            const int box = 1 << w.box_shift, boxes = KT >> w.box_shift;
            bool ok = true;
            while (ok && next_piece(p, s, start, x)) {
                const int h = x.u / w.row_tiles, keys = x.P + x.n;
                const int32_t *table = p.table + (long long)x.b * p.max_pages;
                const int n_pages = (keys + page - 1) >> p.page_shift;
                // 32 pages at a time, the next 32 asked for ahead
                int j0 = (x.t0 * KT) >> p.page_shift;
                auto ask = [&](int j) { return j + lane < n_pages ? __ldg(table + j + lane) : 0; };
                int cur = ask(j0), nxt = ask(j0 + 32);
                for (int t = x.t0; ok && t < x.t1; ++t) {
                    const int pos0 = t * KT;
                    if (!waited && pos0 + KT > x.P) wait();       // rows of the block itself
                    const int first = pos0 >> p.page_shift, last = (min(pos0 + KT, keys) - 1) >> p.page_shift;
                    if (last >= j0 + 32) {
                        // (a tile's pages lie in one window: both are multiples of what a tile holds, or one page)
                        j0 += 32;
                        cur = nxt;
                        nxt = ask(j0 + 32);
                    }
                    const int st = issued % STAGES;
                    if (issued >= STAGES) ok = mbar_wait_warp(bar_free(st), (issued / STAGES + 1) & 1, abort_flag);
                    if (!ok) break;
                    const int live = (min(KT, keys - pos0) + box - 1) >> w.box_shift;        // boxes with rows in them
                    if (lane == 0) {
                        mbar_expect_tx(bar_k(st), live * box * HD * 2);
                        mbar_expect_tx(bar_v(st), live * box * HD * 2);
                    }
                    __syncwarp();
                    const int i = lane & 3, kind = lane >> 2;                                 // lanes 0-3: K boxes, 4-7: V boxes
                    const int pos = pos0 + (i << w.box_shift);
                    int pg = __shfl_sync(0xffffffffu, cur, (max(min(pos >> p.page_shift, last), first) - j0) & 31);
                    if (lane < 8 && i < live && i < boxes) {
                        if (pg < 0 || pg >= p.n_pages) {
                            if (p.status) atomicOr(p.status, ORTHRUS_DEV_BAD_PAGE);
                            pg = 0;
                        }
                        const int row = ((pg * p.Hkv + h) << p.page_shift) + (pos & (page - 1));
                        tma_load_3d(sbase + (st * 2 + kind) * TILE + i * (box * HD * 2), kind ? &tm.v : &tm.k, 0, row, 0,
                                    kind ? bar_v(st) : bar_k(st), policy);
                    }
                    __syncwarp();
                    ++issued;
                }
            }
        }
        if (!waited) wait();
        // the last copies, before the block can end (there are none left unless the consumers gave up)
        if (*abort_flag && lane == 0)
            for (int k = max(0, issued - STAGES); k < issued; ++k) {
                mbar_wait_long(bar_k(k % STAGES), (k / STAGES) & 1);
                mbar_wait_long(bar_v(k % STAGES), (k / STAGES) & 1);
            }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ consumers
        griddep_wait();
        const int wr = warp / WK, wk = warp % WK, g = lane >> 2, tq = lane & 3;
        const uint32_t sq = sbase + C::OFF_Q;
        // per-lane parts of the addresses that ldmatrix takes: row, then the swizzled 16-byte chunk
        const int kr = (lane & 7) + ((lane >> 4) << 3), kc = (lane >> 3) & 1;
        const int vr = (lane & 7) + (((lane >> 3) & 1) << 3), vc = lane >> 4;
        const uint32_t k_lane = kr * 128 + ((kc ^ (kr & 7)) << 4), v_lane = vr * 128 + ((vc ^ (vr & 7)) << 4);
        const uint32_t panel = 128u << w.box_shift;
        bool ok = find_stretch(p, U, blockIdx.x, gridDim.x, lane, false, s);
        const long long start = ok ? s.pos : 0;
        int used = 0;
        while (ok && next_piece(p, s, start, x)) {
            const int h = x.u / w.row_tiles, r0 = (x.u - h * w.row_tiles) * MR, M = x.n * p.G, keys = x.P + x.n;
            // the unit's query rows, 128-byte swizzled panels of 64 columns; rows that do not exist are zero
            const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p.q);
            bar_consumers();                       // (the last unit's rows are done with)
            for (int e = tid; e < MR * (HD / 8); e += 128) {
                const int r = e / (HD / 8), c = e % (HD / 8), R = r0 + r, i = R / p.G;
                uint4 val = make_uint4(0, 0, 0, 0);
                if (R < M) val = *reinterpret_cast<const uint4 *>(q + (((long long)x.b * p.K + i) * p.Hq + h * p.G + R - i * p.G) * HD + c * 8);
                *reinterpret_cast<uint4 *>(smem + C::OFF_Q + (c >> 3) * (MR * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = val;
            }
            bar_consumers();
            const int wrow = wr * 16 * MT;         // this warp's rows of the tile
            uint32_t qf[MT == 1 ? HD / 16 : 1][4];
            auto load_q = [&](int mt, int ks, uint32_t (&f)[4]) {
                const int r = wrow + mt * 16 + vr, c = ks * 2 + vc;
                ldmatrix_x4(f, sq + (c >> 3) * (MR * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
            };
            if constexpr (MT == 1)
#pragma unroll
                for (int ks = 0; ks < HD / 16; ++ks) load_q(0, ks, qf[ks]);
            // what the rows of this lane see
            int sees[MT][2];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int i = (r0 + wrow + mt * 16 + g + e * 8) / p.G;
                    sees[mt][e] = p.causal ? min(keys, x.P + i + 1) : keys;
                }
            float o[MT][ND][4], m[MT][2], l[MT][2];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                m[mt][0] = m[mt][1] = -INFINITY;
                l[mt][0] = l[mt][1] = 0.f;
#pragma unroll
                for (int j = 0; j < ND; ++j) o[mt][j][0] = o[mt][j][1] = o[mt][j][2] = o[mt][j][3] = 0.f;
            }
            for (int t = x.t0; t < x.t1; ++t, ++used) {
                const int st = used % STAGES, parity = (used / STAGES) & 1, pos0 = t * KT + wk * KW;
                if (!mbar_wait_warp(bar_k(st), parity, abort_flag)) { ok = false; break; }
                const uint32_t sk = sbase + st * 2 * TILE, sv = sk + TILE;
                // byte offset of a group of 16 keys in a tile of boxes
                auto group = [&](int np) {
                    const int k0 = wk * KW + np * 16, bx = k0 >> w.box_shift;
                    return (uint32_t)(bx * ((HD * 2) << w.box_shift) + (k0 - (bx << w.box_shift)) * 128);
                };
                float sc[MT][NK][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int j = 0; j < NK; ++j) sc[mt][j][0] = sc[mt][j][1] = sc[mt][j][2] = sc[mt][j][3] = 0.f;
#pragma unroll
                for (int ks = 0; ks < HD / 16; ++ks) {
                    uint32_t qa[MT][4];
                    if constexpr (MT > 1)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) load_q(mt, ks, qa[mt]);
#pragma unroll
                    for (int np = 0; np < NK / 2; ++np) {
                        uint32_t kf[4];
                        ldmatrix_x4(kf, ((sk + group(np) + k_lane) ^ (((ks * 2) & 7) << 4)) + (ks >> 2) * panel);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            if constexpr (MT == 1) {
                                mma_bf16(sc[mt][2 * np], qf[ks], kf[0], kf[1]);
                                mma_bf16(sc[mt][2 * np + 1], qf[ks], kf[2], kf[3]);
                            } else {
                                mma_bf16(sc[mt][2 * np], qa[mt], kf[0], kf[1]);
                                mma_bf16(sc[mt][2 * np + 1], qa[mt], kf[2], kf[3]);
                            }
                        }
                    }
                }
                const bool tail = pos0 + KW > x.P;         // some keys are the block's own, or do not exist
                uint32_t pf[MT][NK / 2][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    if (tail) {
#pragma unroll
                        for (int j = 0; j < NK; ++j) {
                            const int pos = pos0 + j * 8 + tq * 2;
                            if (pos >= sees[mt][0]) sc[mt][j][0] = -INFINITY;
                            if (pos + 1 >= sees[mt][0]) sc[mt][j][1] = -INFINITY;
                            if (pos >= sees[mt][1]) sc[mt][j][2] = -INFINITY;
                            if (pos + 1 >= sees[mt][1]) sc[mt][j][3] = -INFINITY;
                        }
                    }
                    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int j = 0; j < NK; ++j) {
                        top[0] = max3(top[0], sc[mt][j][0], sc[mt][j][1]);
                        top[1] = max3(top[1], sc[mt][j][2], sc[mt][j][3]);
                    }
                    float ref[2], al[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 1));
                        top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 2));
                        const float mn = fmaxf(m[mt][e], top[e] * p.scale_log2);
                        ref[e] = mn == -INFINITY ? 0.f : mn;             // (of nothing so far: no factor)
                        al[e] = ex2(m[mt][e] - ref[e]);
                        m[mt][e] = mn;
                    }
                    float sum[2] = {0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < NK; ++j) {
                        const float p0 = ex2(fmaf(sc[mt][j][0], p.scale_log2, -ref[0])), p1 = ex2(fmaf(sc[mt][j][1], p.scale_log2, -ref[0]));
                        const float p2 = ex2(fmaf(sc[mt][j][2], p.scale_log2, -ref[1])), p3 = ex2(fmaf(sc[mt][j][3], p.scale_log2, -ref[1]));
                        sum[0] += p0 + p1;
                        sum[1] += p2 + p3;
                        pf[mt][j >> 1][(j & 1) * 2] = pack_bf16(p0, p1);
                        pf[mt][j >> 1][(j & 1) * 2 + 1] = pack_bf16(p2, p3);
                    }
                    l[mt][0] = l[mt][0] * al[0] + sum[0];
                    l[mt][1] = l[mt][1] * al[1] + sum[1];
                    if (__any_sync(0xffffffffu, al[0] != 1.f || al[1] != 1.f)) {
#pragma unroll
                        for (int j = 0; j < ND; ++j) { o[mt][j][0] *= al[0]; o[mt][j][1] *= al[0]; o[mt][j][2] *= al[1]; o[mt][j][3] *= al[1]; }
                    }
                }
                if (!mbar_wait_warp(bar_v(st), parity, abort_flag)) { ok = false; break; }
                if (pos0 + KW > keys) {
                    // rows behind the last key, which may hold anything: zero, for the product with their zero probabilities
                    for (int r = max(0, keys - pos0); r < KW; ++r) {
                        const int k0 = wk * KW + r, bx = k0 >> w.box_shift;
                        const uint32_t off = st * 2 * TILE + TILE + bx * ((HD * 2) << w.box_shift) + (k0 - (bx << w.box_shift)) * 128;
                        if (lane < HD / 8)
                            *reinterpret_cast<uint4 *>(smem + off + (lane >> 3) * panel + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    __syncwarp();
                }
#pragma unroll
                for (int kk = 0; kk < NK / 2; ++kk)
#pragma unroll
                    for (int dp = 0; dp < HD / 16; ++dp) {
                        uint32_t vf[4];
                        ldmatrix_x4_trans(vf, ((sv + group(kk) + v_lane) ^ (((dp * 2) & 7) << 4)) + (dp >> 2) * panel);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            mma_bf16(o[mt][2 * dp], pf[mt][kk], vf[0], vf[1]);
                            mma_bf16(o[mt][2 * dp + 1], pf[mt][kk], vf[2], vf[3]);
                        }
                    }
                if (pos0 + KW > keys) fence_proxy_async();        // the zeros before the next copy into the slot
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_free(st));
            }
            // the warps' results of their own keys become the unit's (or the piece's): common maximum, then added up in turn
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[mt][e] += __shfl_xor_sync(0xffffffffu, l[mt][e], 1);
                    l[mt][e] += __shfl_xor_sync(0xffffffffu, l[mt][e], 2);
                    if (tq == 0) stat[warp * 16 * MT + mt * 16 + g + e * 8] = m[mt][e];
                }
            ok = bar_consumers_and(ok);            // (a warp whose wait ran out has come here too: all leave together)
            if (!ok) break;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = mt * 16 + g + e * 8;
                    float top = -INFINITY;
#pragma unroll
                    for (int k = 0; k < WK; ++k) top = fmaxf(top, stat[(wr * WK + k) * 16 * MT + r]);
                    const float al = top == -INFINITY ? 0.f : ex2(m[mt][e] - top);
                    l[mt][e] *= al;
                    m[mt][e] = top;
#pragma unroll
                    for (int j = 0; j < ND; ++j) { o[mt][j][e * 2] *= al; o[mt][j][e * 2 + 1] *= al; }
                }
#pragma unroll 1
            for (int k = 0; k < WK; ++k) {
                if (wk == k)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int r = wrow + mt * 16 + g + e * 8;
                            if (r0 + r >= M) continue;
#pragma unroll
                            for (int j = 0; j < ND; ++j) {
                                float2 *dst = reinterpret_cast<float2 *>(buf + at(r, j * 8 + tq * 2));
                                float2 v = make_float2(o[mt][j][e * 2], o[mt][j][e * 2 + 1]);
                                if (k) { const float2 y = *dst; v.x += y.x; v.y += y.y; }
                                *dst = v;
                            }
                            if (tq == 0) { ml[r] = m[mt][e]; ml[MR + r] = l[mt][e] + (k ? ml[MR + r] : 0.f); }
                        }
                bar_consumers();
            }
            const int rows = min(MR, M - r0);
            auto out_row = [&](int r) {
                const int R = r0 + r, i = R / p.G;
                return static_cast<__nv_bfloat16 *>(p.out) + (((long long)x.b * p.K + i) * p.Hq + h * p.G + R - i * p.G) * HD;
            };
            constexpr int VR = HD / 4;             // vectors of four columns in a row
            if (x.t0 == 0 && x.t1 == x.tiles) {
                for (int e = tid; e < rows * VR; e += 128) {
                    const int r = e / VR, c = (e % VR) * 4;
                    const float4 v = *reinterpret_cast<const float4 *>(buf + at(r, c));
                    const float inv = 1.f / ml[MR + r];
                    *reinterpret_cast<uint2 *>(out_row(r) + c) = make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
                }
                continue;
            }
            const size_t step = piece_floats(w.rows, HD);
            auto piece_at = [&](int slot) { return w.pieces + slot * step; };
            float *mine = piece_at(2 * blockIdx.x + (x.first ? 0 : 1));
            for (int e = tid; e < rows * VR; e += 128) {
                const int r = e / VR, c = (e % VR) * 4;
                *reinterpret_cast<float4 *>(mine + r * HD + c) = *reinterpret_cast<const float4 *>(buf + at(r, c));
            }
            if (tid < rows) *reinterpret_cast<float2 *>(mine + (size_t)w.rows * HD + tid * 2) = make_float2(ml[tid], ml[MR + tid]);
            __threadfence();
            bar_consumers();
            const int c0 = owner(s, x.unit0), n = owner(s, x.unit0 + x.tiles - 1) - c0 + 1;
            if (tid == 0) {
                int *counter = w.counter + (long long)x.b * U + x.u;
                const bool last = atomicAdd(counter, 1) == n - 1;
                if (last) { *counter = 0; __threadfence(); }
                *last_flag = last;
            }
            bar_consumers();
            if (!*last_flag) continue;
            __threadfence();
            const int s0 = 2 * c0 + (s.T * c0 / s.n == x.unit0 ? 0 : 1);      // where the first piece is; the others are first in their CTAs
            for (int e = tid; e < rows * VR; e += 128) {
                const int r = e / VR, c = (e % VR) * 4;
                float top = -INFINITY, sum = 0.f;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                for (int k = 0; k < n; ++k)
                    top = fmaxf(top, __ldcg(piece_at(k ? 2 * (c0 + k) : s0) + (size_t)w.rows * HD + r * 2));
#pragma unroll 4
                for (int k = 0; k < n; ++k) {
                    const float *src = piece_at(k ? 2 * (c0 + k) : s0);
                    const float2 st = __ldcg(reinterpret_cast<const float2 *>(src + (size_t)w.rows * HD + r * 2));
                    const float4 y = __ldcg(reinterpret_cast<const float4 *>(src + r * HD + c));
                    const float al = top == -INFINITY ? 0.f : ex2(st.x - top);
                    sum = fmaf(st.y, al, sum);
                    v.x = fmaf(y.x, al, v.x); v.y = fmaf(y.y, al, v.y); v.z = fmaf(y.z, al, v.z); v.w = fmaf(y.w, al, v.w);
                }
                const float inv = 1.f / sum;
                *reinterpret_cast<uint2 *>(out_row(r) + c) = make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
            }
        }
    }
    __syncthreads();
    if (tid == 0 && *abort_flag && p.status) atomicOr(p.status, ORTHRUS_DEV_WAIT_TIMEOUT);
}

int tile_rows(int M) { return M <= 16 ? 16 : M <= 32 ? 32 : 64; }

// CTAs of a call, and what its workspace holds.  From the shape and the host's bound on the lengths.
struct Grid { int ctas, row_tiles, rows; size_t counters, bytes; };
Grid plan(const orthrus_paged_layer_t &L)
{
    Grid g;
    const int M = L.n_q_heads / L.n_kv_heads * L.block, mr = tile_rows(M);
    g.row_tiles = (M + mr - 1) / mr;
    g.rows = M < mr ? M : mr;
    const long long units = (long long)L.batch * L.n_kv_heads * g.row_tiles;
    const long long keys = (L.max_len_hint > 0 ? (long long)L.max_len_hint : (long long)L.max_pages * L.page_size - L.block) + L.block;
    const long long tiles = units * ((keys < 1 ? 1 : keys) + KT - 1) / KT;
    const long long most = 2LL * num_sms();
    g.ctas = (int)(tiles < 1 ? 1 : tiles < most ? tiles : most);
    g.counters = (size_t)((units * 4 + 255) / 256 * 256);
    g.bytes = g.counters + 2 * (size_t)g.ctas * piece_floats(g.rows, L.head_dim) * sizeof(float);
    return g;
}

// [rows][d] as panels of 64 columns: boxes of `box` rows and all columns
bool page_map(void *ptr, unsigned d, unsigned long long rows, unsigned box, CUtensorMap *out)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {64, (cuuint64_t)rows, d / 64};
    const cuuint64_t strides[2] = {(cuuint64_t)d * 2, 128};
    const cuuint32_t boxes[3] = {64, box, d / 64}, estr[3] = {1, 1, 1};
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, ptr, dims, strides, boxes, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD, int MT, int WR>
cudaError_t launch_one(const PagedParams &p, const PagedMaps &tm, const PagedWork &w, int ctas, cudaStream_t st)
{
    using C = PagedShape<HD, MT, WR>;
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = configure(paged_attend_kernel<HD, MT, WR>, done, C::SMEM, false);
    if (e != cudaSuccess) return e;
    return launch_kernel(p.early, paged_attend_kernel<HD, MT, WR>, dim3(ctas), NTHREADS, C::SMEM, st, p, tm, w);
}

}  // namespace

bool paged_tc_shape(const orthrus_paged_layer_t &L)
{
    if (L.dtype != ORTHRUS_BF16 || (L.head_dim != 64 && L.head_dim != 128) || L.page_size < 16) return false;
    return (unsigned long long)L.n_pages * L.n_kv_heads * L.page_size < 0x7fffffffull && tc_driver_ok();
}

size_t paged_tc_workspace_bytes(const orthrus_paged_layer_t &L) { return plan(L).bytes; }

cudaError_t launch_paged_attend_tc(const PagedParams &p, const orthrus_paged_layer_t &L, void *ws_body, cudaStream_t st)
{
    const Grid g = plan(L);
    const int M = p.G * p.K;
    PagedWork w;
    w.row_tiles = g.row_tiles;
    w.box_shift = p.page_shift < 6 ? p.page_shift : 6;
    w.rows = g.rows;
    w.counter = static_cast<int *>(ws_body);
    w.pieces = reinterpret_cast<float *>(static_cast<unsigned char *>(ws_body) + g.counters);
    PagedMaps tm;
    const unsigned long long rows = (unsigned long long)L.n_pages * L.n_kv_heads * L.page_size;
    if (!page_map(L.k_pages, p.d, rows, 1u << w.box_shift, &tm.k) || !page_map(L.v_pages, p.d, rows, 1u << w.box_shift, &tm.v))
        return cudaErrorInvalidValue;
    if (p.d == 128) {
        if (M <= 16) return launch_one<128, 1, 1>(p, tm, w, g.ctas, st);
        if (M <= 32) return launch_one<128, 2, 1>(p, tm, w, g.ctas, st);
        return launch_one<128, 2, 2>(p, tm, w, g.ctas, st);
    }
    if (M <= 16) return launch_one<64, 1, 1>(p, tm, w, g.ctas, st);
    if (M <= 32) return launch_one<64, 2, 1>(p, tm, w, g.ctas, st);
    return launch_one<64, 2, 2>(p, tm, w, g.ctas, st);
}

}  // namespace orthrus
