// Attention over pages in fp32 arithmetic: the fp32 test mode, and the shapes that the tensor-core kernels do not take (head_dim 32 and
// 256, pages of fewer than 16 positions).
//
// One pass over the keys with a running reference and sum, as elsewhere; a CTA takes four query rows of a unit (request and KV head) and a
// range of its keys, its eight warps eight keys each in turn.  In a warp a lane has d / 32 columns of every key, so that loads are whole rows:
//   scores     32 partial products a lane (8 keys, 4 rows), summed over the lanes by halving: after five exchanges lane 4 j + r has
//              key j's with row r, 31 shuffles for all of them
//   softmax    a lane its one score; maxima over the lanes of a row, sums kept apart until the end
//   values     a weight for each of the 32 pairs by shuffle, d / 32 columns a lane
// The warps' results meet in shared memory, the ranges of a unit in the workspace, where the CTA that is the last joins them in their order.
//
// What bounds it: HBM for up to four rows a unit, then the fp32 pipe (4 d operations a key and row) and the bf16 values' way to
// fp32.  8 KV heads of 4 query heads, 4096 keys: fp32 of 128, 32 requests 168 us (6.4 TB/s); bf16 of 256, one request 31 us, 32 requests 254 us
// (4.2 TB/s); bf16 of 32, 8 requests 34 us.  Pairs of products in one instruction (fma.rn.f32x2) were slower, 292 us for 254.
#include <type_traits>
#include "paged.cuh"

namespace orthrus {
namespace {

constexpr int ROWS = 4, KEYS = 8, WARPS = 8, THREADS = WARPS * 32, CHUNK = WARPS * KEYS;

template <int BYTES> struct Raw;                 // what a lane loads at once
template <> struct Raw<2> { using V = unsigned short; };
template <> struct Raw<4> { using V = unsigned; };
template <> struct Raw<8> { using V = uint2; };
template <> struct Raw<16> { using V = uint4; };
template <int BYTES> __device__ inline typename Raw<BYTES>::V nothing() { return typename Raw<BYTES>::V{}; }

template <typename T> __device__ inline float to_f(T x) { return x; }
template <> __device__ inline float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ inline void put(float *p, float x) { *p = x; }
__device__ inline void put(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }

// A lane's columns: NV vectors of VEC, 32 VEC apart
template <typename T, int DPL> struct Columns {
    static constexpr int VEC = DPL < 16 / (int)sizeof(T) ? DPL : 16 / (int)sizeof(T), NV = DPL / VEC, BYTES = VEC * sizeof(T);
    using V = typename Raw<BYTES>::V;
    __device__ static int first(int v, int lane) { return (v * 32 + lane) * VEC; }
    __device__ static float at(const V &x, int k) {
        if constexpr (sizeof(T) == 4) {
            if constexpr (VEC == 1) return __uint_as_float(x);
            else if constexpr (VEC == 2) return __uint_as_float(k ? x.y : x.x);
            else return __uint_as_float(k == 0 ? x.x : k == 1 ? x.y : k == 2 ? x.z : x.w);
        } else {
            unsigned w;
            if constexpr (VEC <= 2) w = x;
            else if constexpr (VEC == 4) w = k < 2 ? x.x : x.y;
            else w = k < 2 ? x.x : k < 4 ? x.y : k < 6 ? x.z : x.w;
            return __uint_as_float(k & 1 ? w & 0xffff0000u : w << 16);
        }
    }
};

template <typename T, int DPL>
__global__ void __launch_bounds__(THREADS, DPL * sizeof(T) > 16 ? 1 : 2) paged_attend_simt_kernel(const PagedParams p, int row_tiles, float *pieces)
{
    constexpr int D = DPL * 32;
    using C = Columns<T, DPL>;
    using V = typename C::V;
    __shared__ float sO[WARPS][ROWS][D], sM[WARPS][ROWS], sL[WARPS][ROWS];
    __shared__ int is_last;
    pdl_begin();
    const int unit = blockIdx.x / row_tiles, b = unit / p.Hkv, h = unit - b * p.Hkv, r0 = (blockIdx.x - unit * row_tiles) * ROWS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int P, n;
    bool bad;
    paged_request(p, b, P, n, bad);
    if (bad && h == 0 && r0 == 0 && blockIdx.y == 0 && tid == 0) atomicOr(p.status, ORTHRUS_DEV_BAD_CACHE_LEN);
    const int M = n * p.G;
    if (r0 >= M) return;
    // keys that any row of this tile sees, and this CTA's of them
    const unsigned keys = p.causal ? P + min(n, (r0 + ROWS - 1) / p.G + 1) : P + n;
    const unsigned each = ((keys + gridDim.y - 1) / gridDim.y + CHUNK - 1) / CHUNK * CHUNK, parts = (keys + each - 1) / each;
    if (blockIdx.y >= parts) return;
    const int k0 = blockIdx.y * each, k1 = (int)min(keys, k0 + each);
    auto row_at = [&](int R) { return (((long long)b * p.K + R / p.G) * p.Hq + h * p.G + R % p.G) * D; };

    float q[ROWS][DPL], o[ROWS][DPL];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int v = 0; v < C::NV; ++v) {
            const V x = r0 + r < M ? *reinterpret_cast<const V *>(static_cast<const T *>(p.q) + row_at(r0 + r) + C::first(v, lane)) : nothing<C::BYTES>();
#pragma unroll
            for (int k = 0; k < C::VEC; ++k) { q[r][v * C::VEC + k] = C::at(x, k) * p.scale_log2; o[r][v * C::VEC + k] = 0.f; }
        }
    auto sees_of = [&](int r) { return r0 + r >= M ? 0 : p.causal ? P + (r0 + r) / p.G + 1 : P + n; };
    const int my_row = lane & 3, my_key = lane >> 2, my_sees = sees_of(my_row);
    float m = -INFINITY, l = 0.f;                // of row my_row: its reference, and the sum over keys my_key of each eight
    const int32_t *table = p.table + (long long)b * p.max_pages;
    auto page_of = [&](int pos) { return pos < k1 ? __ldcg(table + (pos >> p.page_shift)) : 0; };
    int next = page_of(k0 + warp * KEYS + (lane & 7));
    for (int t0 = k0 + warp * KEYS; t0 < k1; t0 += CHUNK) {
        // the eight keys' rows (lane j: key j's), whose pages were asked for a turn ahead
        const int pos = t0 + (lane & 7), page = next;
        const bool in = page >= 0 && page < p.n_pages, is = pos < k1 && in;
        if (pos < k1 && !in) atomicOr(p.status, ORTHRUS_DEV_BAD_PAGE);
        const long long row = ((((long long)page * p.Hkv + h) << p.page_shift) + (pos & ((1 << p.page_shift) - 1))) * D;
        if (t0 < k1 - CHUNK) next = page_of(pos + CHUNK);
        const unsigned live = __ballot_sync(0xffffffffu, is);
        V kx[KEYS][C::NV], vx[KEYS][C::NV];
        long long at[KEYS];
#pragma unroll
        for (int j = 0; j < KEYS; ++j) at[j] = __shfl_sync(0xffffffffu, row, j) + lane * C::VEC;
        auto load = [&](V (&x)[KEYS][C::NV], const void *pages) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
#pragma unroll
                for (int v = 0; v < C::NV; ++v)
                    x[j][v] = live >> j & 1 ? __ldcg(reinterpret_cast<const V *>(static_cast<const T *>(pages) + at[j] + v * 32 * C::VEC)) : nothing<C::BYTES>();
        };
        load(kx, p.k_pages);
        load(vx, p.v_pages);
        float s[KEYS * ROWS];
#pragma unroll
        for (int j = 0; j < KEYS; ++j)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                float x = 0.f;
#pragma unroll
                for (int c = 0; c < DPL; ++c) x = fmaf(q[r][c], C::at(kx[j][c / C::VEC], c % C::VEC), x);
                s[j * ROWS + r] = x;
            }
#pragma unroll
        for (int off = 16; off; off >>= 1)
#pragma unroll
            for (int i = 0; i < off; ++i) {
                const bool up = lane & off;
                const float keep = up ? s[i + off] : s[i], give = up ? s[i] : s[i + off];
                s[i] = keep + __shfl_xor_sync(0xffffffffu, give, off);
            }
        const float x = t0 + my_key < min(my_sees, k1) && (live >> my_key & 1) ? s[0] : -INFINITY;
        float top = x;
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        const float to = fmaxf(m, top), ref = to == -INFINITY ? 0.f : to;
        if (__any_sync(0xffffffffu, to > m)) {
            const float al = exp2f(m - ref);
            l *= al;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float a = __shfl_sync(0xffffffffu, al, r);
#pragma unroll
                for (int c = 0; c < DPL; ++c) o[r][c] *= a;
            }
            m = to;
        }
        const float w = exp2f(x - ref);
        l += w;
        auto add = [&](auto all) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float y = __shfl_sync(0xffffffffu, w, j * ROWS + r);
                    if (!decltype(all)::value && t0 + j >= sees_of(r)) continue;         // (a value that the row does not see may be anything)
#pragma unroll
                    for (int c = 0; c < DPL; ++c) o[r][c] = fmaf(y, C::at(vx[j][c / C::VEC], c % C::VEC), o[r][c]);
                }
        };
        if (t0 + KEYS <= P) add(std::true_type()); else add(std::false_type());
    }

    // the warps' sums
#pragma unroll
    for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    if (lane < ROWS) { sM[warp][lane] = m; sL[warp][lane] = l; }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int c = 0; c < DPL; ++c) sO[warp][r][C::first(c / C::VEC, lane) + c % C::VEC] = o[r][c];
    __syncthreads();
    constexpr int PIECE = ROWS * (D + 2);
    float *mine = pieces + ((size_t)blockIdx.x * gridDim.y + blockIdx.y) * PIECE;
    for (int e = tid; e < ROWS * D; e += THREADS) {
        const int r = e / D, c = e - r * D;
        float ref = sM[0][r], sum = 0.f, y = 0.f;
#pragma unroll
        for (int k = 1; k < WARPS; ++k) ref = fmaxf(ref, sM[k][r]);
        const float from = ref == -INFINITY ? 0.f : ref;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {
            const float a = exp2f(sM[k][r] - from);
            sum = fmaf(sL[k][r], a, sum);
            y = fmaf(sO[k][r][c], a, y);
        }
        if (parts > 1) {
            mine[e] = y;
            if (c == 0) { mine[ROWS * D + r] = ref; mine[ROWS * D + ROWS + r] = sum; }
        } else if (r0 + r < M) put(static_cast<T *>(p.out) + row_at(r0 + r) + c, y / sum);
    }
    if (parts == 1) return;
    __syncthreads();
    if (tid == 0) is_last = last_piece(p.status, blockIdx.x, (int)parts);
    __syncthreads();
    if (!is_last) return;
    const float *all = pieces + (size_t)blockIdx.x * gridDim.y * PIECE;
    for (int e = tid; e < ROWS * D; e += THREADS) {
        const int r = e / D, c = e - r * D;
        if (r0 + r >= M) break;
        float ref = -INFINITY, sum = 0.f, y = 0.f;
        for (unsigned k = 0; k < parts; ++k) ref = fmaxf(ref, __ldcg(all + k * PIECE + ROWS * D + r));
        if (ref == -INFINITY) ref = 0.f;
#pragma unroll 4
        for (unsigned k = 0; k < parts; ++k) {
            const float *x = all + k * PIECE, a = exp2f(__ldcg(x + ROWS * D + r) - ref);
            sum = fmaf(__ldcg(x + ROWS * D + ROWS + r), a, sum);
            y = fmaf(__ldcg(x + e), a, y);
        }
        put(static_cast<T *>(p.out) + row_at(r0 + r) + c, y / sum);
    }
}

// Units of four rows, and CTAs for each: so many that all SMs have two (of a cut unit there is a count in the workspace's header)
struct Cut { long long units; int row_tiles, parts; };
Cut cut(const orthrus_paged_layer_t &L)
{
    Cut c;
    c.row_tiles = (L.n_q_heads / L.n_kv_heads * L.block + ROWS - 1) / ROWS;
    c.units = (long long)L.batch * L.n_kv_heads * c.row_tiles;
    const long long most = (L.max_len_hint > 0 ? (long long)L.max_len_hint + L.block : (long long)L.max_pages * L.page_size);
    const long long room = 2LL * num_sms() / c.units, chunks = (most + CHUNK - 1) / CHUNK;
    c.parts = (int)(room < chunks ? room : chunks);
    if (c.parts > kMostPieces) c.parts = kMostPieces;
    if (c.parts < 1 || c.units > kCounts) c.parts = 1;
    return c;
}

template <typename T, int DPL> cudaError_t launch_one(const PagedParams &p, const Cut &c, float *pieces, cudaStream_t st)
{
    return launch_kernel(p.early, paged_attend_simt_kernel<T, DPL>, dim3((unsigned)c.units, c.parts), THREADS, 0, st, p, c.row_tiles, pieces);
}
template <typename T> cudaError_t launch_width(const PagedParams &p, const Cut &c, float *pieces, cudaStream_t st)
{
    switch (p.d) {
    case 32: return launch_one<T, 1>(p, c, pieces, st);
    case 64: return launch_one<T, 2>(p, c, pieces, st);
    case 128: return launch_one<T, 4>(p, c, pieces, st);
    default: return launch_one<T, 8>(p, c, pieces, st);
    }
}

}  // namespace

bool paged_simt_shape(const orthrus_paged_layer_t &L) { return cut(L).units <= 0x7fffffffLL; }

size_t paged_simt_workspace_bytes(const orthrus_paged_layer_t &L)
{
    const Cut c = cut(L);
    return c.parts > 1 ? (size_t)c.units * c.parts * ROWS * (L.head_dim + 2) * sizeof(float) : 0;
}

cudaError_t launch_paged_attend_simt(const PagedParams &p, const orthrus_paged_layer_t &L, void *ws_body, cudaStream_t st)
{
    const Cut c = cut(L);
    float *pieces = static_cast<float *>(ws_body);
    return L.dtype == ORTHRUS_FP32 ? launch_width<float>(p, c, pieces, st) : launch_width<__nv_bfloat16>(p, c, pieces, st);
}

}  // namespace orthrus
