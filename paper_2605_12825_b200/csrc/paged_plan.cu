// Which kernel serves a call of the paged attention on tensor cores, with how many CTAs, and what its workspace holds.
#include "paged_stretch.cuh"

namespace orthrus {

cudaError_t launch_paged_attend_mma(const PagedParams &p, const PagedWork &w, unsigned long long rows, int ctas, cudaStream_t st);
cudaError_t launch_paged_attend_wide(const PagedParams &p, const PagedWork &w, unsigned long long rows, int ctas, cudaStream_t st);

namespace {

bool narrow(const orthrus_paged_layer_t &L) { return L.n_q_heads / L.n_kv_heads * L.block <= 16; }

// From the shape and the host's bound on the lengths.
PagedGrid plan(const orthrus_paged_layer_t &L)
{
    PagedGrid g;
    const int M = L.n_q_heads / L.n_kv_heads * L.block, mr = narrow(L) ? 16 : 128;
    g.row_tiles = (M + mr - 1) / mr;
    g.rows = M < mr ? M : mr;
    const long long units = (long long)L.batch * L.n_kv_heads * g.row_tiles;
    const long long keys = (L.max_len_hint > 0 ? (long long)L.max_len_hint : (long long)L.max_pages * L.page_size - L.block) + L.block;
    const long long tiles = units * (((keys < 1 ? 1 : keys) + KT - 1) / KT);
    // Two CTAs an SM where there is much to stream; one where latency counts, which halves the pieces to join
    const long long most = (tiles >= 16LL * num_sms() ? 2LL : 1LL) * num_sms();
    g.ctas = (int)(tiles < 1 ? 1 : tiles < most ? tiles : most);
    g.most_pieces = narrow(L) ? kMostNarrow : kMostWide;
    g.counters = (size_t)((units * 4 + 255) / 256 * 256);
    g.bytes = g.counters + 2 * (size_t)g.ctas * piece_floats(g.rows, L.head_dim) * sizeof(float);
    return g;
}

unsigned long long pool_rows(const orthrus_paged_layer_t &L) { return (unsigned long long)L.n_pages * L.n_kv_heads * L.page_size; }

}  // namespace

bool paged_tc_shape(const orthrus_paged_layer_t &L)
{
    if (L.dtype != ORTHRUS_BF16 || (L.head_dim != 64 && L.head_dim != 128) || L.page_size < 16) return false;
    return pool_rows(L) < 0x7fffffffull && tc_driver_ok();
}

size_t paged_tc_workspace_bytes(const orthrus_paged_layer_t &L) { return plan(L).bytes; }

cudaError_t launch_paged_attend_tc(const PagedParams &p, const orthrus_paged_layer_t &L, void *ws_body, cudaStream_t st)
{
    const PagedGrid g = plan(L);
    PagedWork w;
    w.row_tiles = g.row_tiles;
    w.box_shift = p.page_shift < 6 ? p.page_shift : 6;
    w.rows = g.rows;
    w.most_pieces = g.most_pieces;
    w.counter = static_cast<int *>(ws_body);
    w.pieces = reinterpret_cast<float *>(static_cast<unsigned char *>(ws_body) + g.counters);
    set_last_path(narrow(L) ? "mma" : "tcgen05");
    return narrow(L) ? launch_paged_attend_mma(p, w, pool_rows(L), g.ctas, st) : launch_paged_attend_wide(p, w, pool_rows(L), g.ctas, st);
}

}  // namespace orthrus
