// How the work of a paged attention call is cut over CTAs, where the pieces of its units lie, and the walk over a request's pages.
#pragma once
#include <cuda.h>
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace orthrus {

constexpr int KT = 64;                    // keys per tile
constexpr int kLeast = 2;                 // tiles a CTA takes at least, while there are fewer than CTAs

struct PagedMaps { CUtensorMap k, v; };
struct PagedWork {
    int row_tiles;           // tiles of query rows of a (request, KV head)
    int box_shift;           // log2 of the rows of a TMA box: min(page, 64)
    int rows;                // query rows a piece holds: min(rows of a tile, K G)
    int most_pieces;         // pieces of a unit
    float *pieces;           // [2 CTAs] pieces: an output [d / 4][rows][4], behind it [rows][2] (reference, sum)
};

// floats of a piece, a multiple of the 16 bytes it is moved in
__host__ __device__ constexpr size_t piece_floats(int rows, int d) { return ((size_t)rows * (d + 2) + 3) / 4 * 4; }

// A CTA's stretch of the line of tiles, piece by piece.  Every warp walks it by itself, 32 requests' lengths in its lanes.  Tile numbers fit 31
// bits (paged_tc_shape sees to it).
struct Stretch {
    int n, q, rem;                   // CTAs at work: the first `rem` take q + 1 tiles, the others q
    int start, pos, end, base;       // the stretch's first, next and end; first tile of request b
    int b, P, rows, tiles;           // request: its prefix, rows of its block, tiles of one of its units
    int U;                           // units of a request
    int b0, lane_P, lane_rows;       // requests [b0, b0 + 32): a lane's
};
struct Piece { int b, u, P, n, t0, t1, tiles, unit0; bool first; };

__device__ inline int tiles_of(int P, int n) { return n > 0 ? (P + n + KT - 1) / KT : 0; }
// requests [b0, b0 + 32) into the lanes; this lane's tiles
__device__ inline int load_requests(const PagedParams &p, Stretch &s, int b0, int lane)
{
    bool bad;
    s.b0 = b0;
    s.lane_P = s.lane_rows = 0;
    if (b0 + lane < p.B) paged_request(p, b0 + lane, s.lane_P, s.lane_rows, bad);
    return tiles_of(s.lane_P, s.lane_rows);
}
// A stretch that was found ahead of the wait for the preceding kernel is one behind it too if the lengths are still the same.
__device__ inline bool still_so(const PagedParams &p, const Stretch &s, int lane)
{
    if (p.B > 32) return false;
    int P = 0, n = 0;
    bool bad;
    if (lane < p.B) paged_request(p, lane, P, n, bad);
    return __all_sync(0xffffffffu, P == s.lane_P && n == s.lane_rows);
}
// lengths out of range, by one warp of a call
__device__ inline void tell_requests(const PagedParams &p, int lane)
{
#pragma unroll 1
    for (int b = lane; b < p.B; b += 32) {
        int P, n;
        bool bad;
        paged_request(p, b, P, n, bad);
        if (bad && p.status) atomicOr(p.status, ORTHRUS_DEV_BAD_CACHE_LEN);
    }
}
__device__ inline void set_request(const PagedParams &p, Stretch &s, int lane)
{
    if (s.b >= s.b0 + 32) load_requests(p, s, s.b, lane);
    s.P = __shfl_sync(0xffffffffu, s.lane_P, s.b - s.b0);
    s.rows = __shfl_sync(0xffffffffu, s.lane_rows, s.b - s.b0);
    s.tiles = tiles_of(s.P, s.rows);
}
__device__ inline int scan_tiles(int t, int lane)
{
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, t, off);
        if (lane >= off) t += x;
    }
    return t;
}
// The stretch of CTA c; end = 0: nothing to do.  As many CTAs are at work as there are, but for two bounds: kLeast tiles each, and no more
// pieces of the longest unit than `most`.  (Out of line, one copy for the warps' roles: a kernel's code has to be short.)
static __device__ __noinline__ Stretch find_stretch(const PagedParams &p, int U, int most)
{
    const int c = blockIdx.x, lane = threadIdx.x & 31;
    Stretch s;
    s.pos = s.end = 0;
    s.U = U;
    // a lane sums up `per` neighbouring requests; up to 32 requests it keeps its own
    const int per = (p.B + 31) / 32;
    int mine = 0, longest = 0;
    if (per == 1) {
        mine = longest = load_requests(p, s, 0, lane);
    } else {
#pragma unroll 4
        for (int i = 0; i < per; ++i) {
            int P = 0, n = 0;
            bool bad;
            if (lane * per + i < p.B) paged_request(p, lane * per + i, P, n, bad);
            const int t = tiles_of(P, n);
            mine += t;
            longest = max(longest, t);
        }
    }
    const int upto = scan_tiles(mine, lane);
    longest = (int)__reduce_max_sync(0xffffffffu, (unsigned)longest);
    const unsigned T = (unsigned)__shfl_sync(0xffffffffu, upto, 31) * U;
    if (T == 0) return s;
    const unsigned share = max((longest + most - 2) / (most - 1), 1);       // tiles of a CTA at least
    const unsigned n = max(min(min(gridDim.x, (T + kLeast - 1) / kLeast), T / share), 1u);
    s.n = (int)n;
    s.q = (int)(T / n);
    s.rem = (int)(T - n * s.q);
    if (c >= s.n) return s;
    s.start = s.pos = c * s.q + min(c, s.rem);
    s.end = s.start + s.q + (c < s.rem);
    // the lane, then the request that the stretch begins in
    const int l = __ffs(__ballot_sync(0xffffffffu, upto * U > s.pos)) - 1;
    int run = __shfl_sync(0xffffffffu, upto - mine, l);
    s.b = l * per;
    if (per > 1) {
#pragma unroll 1
        for (int b0 = l * per; ; b0 += 32) {                  // (it is among the lane's: the loop ends)
            const int t = load_requests(p, s, b0, lane), sum = scan_tiles(t, lane);
            const unsigned hit = __ballot_sync(0xffffffffu, (run + sum) * U > s.pos);
            if (hit || b0 + 32 >= p.B) {
                const int k = hit ? __ffs(hit) - 1 : 0;
                s.b = b0 + k;
                run += __shfl_sync(0xffffffffu, sum - t, k);
                break;
            }
            run += __shfl_sync(0xffffffffu, sum, 31);
        }
    }
    s.base = run * U;
    set_request(p, s, lane);
    return s;
}
__device__ inline bool next_piece(const PagedParams &p, Stretch &s, int lane, Piece &x)
{
    if (s.pos >= s.end) return false;
#pragma unroll 1
    while (s.pos >= s.base + s.tiles * s.U) {
        s.base += s.tiles * s.U;
        ++s.b;
        set_request(p, s, lane);
    }
    x.b = s.b; x.P = s.P; x.n = s.rows; x.tiles = s.tiles;
    x.u = (int)((unsigned)(s.pos - s.base) / (unsigned)s.tiles);
    x.unit0 = s.base + x.u * s.tiles;
    x.t0 = s.pos - x.unit0;
    x.t1 = min(s.tiles, x.t0 + (s.end - s.pos));
    x.first = s.pos == s.start;
    s.pos += x.t1 - x.t0;
    return true;
}
__device__ inline int stretch_start(const Stretch &s, int c) { return c * s.q + min(c, s.rem); }
// the CTA that takes a tile
__device__ inline int owner(const Stretch &s, int tile)
{
    const int longer = s.rem * (s.q + 1);
    return tile < longer ? (int)((unsigned)tile / (unsigned)(s.q + 1)) : s.rem + (int)((unsigned)(tile - longer) / (unsigned)s.q);
}

// Rows of q and out: row R of request b and KV head h
__device__ inline long long row_offset(const PagedParams &p, int b, int h, int R, int d)
{
    const int i = R / p.G;
    return (((long long)b * p.K + i) * p.Hq + h * p.G + R - i * p.G) * d;
}

// The 32 table entries at hand of a warp that walks a request's pages, the next 32 asked for ahead.
struct PageWindow {
    const int32_t *table;
    int n_pages, j0, cur, nxt;
    __device__ int ask(int j, int lane) const { return j + lane < n_pages ? __ldcg(table + j + lane) : 0; }
    __device__ void open(const PagedParams &p, const Piece &x, int lane) {
        table = p.table + (long long)x.b * p.max_pages;
        n_pages = (x.P + x.n + (1 << p.page_shift) - 1) >> p.page_shift;
        j0 = (x.t0 * KT) >> p.page_shift;
        cur = ask(j0, lane);
        nxt = ask(j0 + 32, lane);
    }
    // page of position `pos` of the tile whose last position is `last`, a lane its own `pos`; a tile's pages lie in one window (both are
    // multiples of what a tile holds, or the tile is in one page)
    __device__ int page(const PagedParams &p, int pos, int last, int lane) {
        if ((last >> p.page_shift) >= j0 + 32) { j0 += 32; cur = nxt; nxt = ask(j0 + 32, lane); }
        int pg = __shfl_sync(0xffffffffu, cur, (min(pos, last) >> p.page_shift) - j0);
        if (pg < 0 || pg >= p.n_pages) {
            if (p.status) atomicOr(p.status, ORTHRUS_DEV_BAD_PAGE);
            pg = 0;
        }
        return pg;
    }
};

}  // namespace orthrus
