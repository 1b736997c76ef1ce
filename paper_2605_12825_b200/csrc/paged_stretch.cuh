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
    int *counter;            // [unit]: pieces that are in
    float *pieces;           // [2 CTAs] pieces: an output [d / 4][rows][4], behind it [rows][2] (reference, sum)
};

// floats of a piece, a multiple of the 16 bytes it is moved in
__host__ __device__ constexpr size_t piece_floats(int rows, int d) { return ((size_t)rows * (d + 2) + 3) / 4 * 4; }

// (of numbers that hardly ever pass 32 bits)
__device__ inline long long quotient(long long a, long long b) {
    return (unsigned long long)(a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}

// A CTA's stretch of the line of tiles, piece by piece.  Every warp walks it by itself, 32 requests' lengths in its lanes.
struct Stretch {
    long long T, pos, end, base;     // all tiles; next tile; the stretch's end; first tile of request b
    int n, b, P, rows, tiles;        // CTAs at work; request: its prefix, rows of its block, tiles of one of its units
    int U;                           // units of a request
    int b0, lane_P, lane_rows;       // requests [b0, b0 + 32): a lane's
};
struct Piece { int b, u, P, n, t0, t1, tiles; long long unit0; bool first; };

__device__ inline int tiles_of(int P, int n) { return n > 0 ? (P + n + KT - 1) / KT : 0; }
// requests [b0, b0 + 32) into the lanes; this lane's tiles
__device__ inline int load_requests(const PagedParams &p, Stretch &s, int b0, int lane, bool tell)
{
    bool bad = false;
    s.b0 = b0;
    s.lane_P = s.lane_rows = 0;
    if (b0 + lane < p.B) paged_request(p, b0 + lane, s.lane_P, s.lane_rows, bad);
    if (tell && bad && p.status) atomicOr(p.status, ORTHRUS_DEV_BAD_CACHE_LEN);
    return tiles_of(s.lane_P, s.lane_rows);
}
__device__ inline void set_request(const PagedParams &p, Stretch &s, int lane)
{
    if (s.b >= s.b0 + 32) load_requests(p, s, s.b, lane, false);
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
// The stretch of CTA c; false: nothing to do.  As many CTAs are at work as there are, but for two bounds: kLeast tiles each, and no more pieces
// of the longest unit than `most`.
__device__ inline bool find_stretch(const PagedParams &p, int U, int c, int ctas, int most, int lane, bool tell, Stretch &s)
{
    long long sum = 0;
    int longest = 0, t = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
        t = load_requests(p, s, b0, lane, tell);
        sum += __reduce_add_sync(0xffffffffu, (unsigned)t);
        longest = max(longest, (int)__reduce_max_sync(0xffffffffu, (unsigned)t));
    }
    s.U = U;
    s.T = sum * U;
    if (s.T == 0) return false;
    long long n = min((long long)ctas, (s.T + kLeast - 1) / kLeast);
    n = min(n, max(1ll, quotient(s.T * (most - 1), longest)));
    s.n = (int)n;
    if (c >= s.n) return false;
    s.pos = quotient(s.T * c, n);
    s.end = quotient(s.T * (c + 1), n);
    // the request that the stretch begins in
    long long run = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
        if (p.B > 32) t = load_requests(p, s, b0, lane, false);
        const int upto = scan_tiles(t, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, (run + upto) * U > s.pos);
        if (hit) {
            const int l = __ffs(hit) - 1;
            s.b = b0 + l;
            s.base = (run + __shfl_sync(0xffffffffu, upto - t, l)) * U;
            break;
        }
        run += __shfl_sync(0xffffffffu, upto, 31);
    }
    set_request(p, s, lane);
    return true;
}
__device__ inline bool next_piece(const PagedParams &p, Stretch &s, long long start, int lane, Piece &x)
{
    if (s.pos >= s.end) return false;
    while (s.pos >= s.base + (long long)s.tiles * s.U) {
        s.base += (long long)s.tiles * s.U;
        ++s.b;
        set_request(p, s, lane);
    }
    x.b = s.b; x.P = s.P; x.n = s.rows; x.tiles = s.tiles;
    x.u = (int)quotient(s.pos - s.base, s.tiles);
    x.unit0 = s.base + (long long)x.u * s.tiles;
    x.t0 = (int)(s.pos - x.unit0);
    x.t1 = (int)min((long long)s.tiles, x.t0 + (s.end - s.pos));
    x.first = s.pos == start;
    s.pos += x.t1 - x.t0;
    return true;
}
__device__ inline int owner(const Stretch &s, long long tile) { return (int)quotient((tile + 1) * s.n - 1, s.T); }

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
    __device__ int ask(int j, int lane) const { return j + lane < n_pages ? __ldg(table + j + lane) : 0; }
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
