// New K/V rows into the pages of a paged cache, alone or with the rotary embedding of the block's queries and keys.
//
// A warp takes a row (block position i of request b) and some of its heads: four column pairs of a head a lane, so that a head
// of 128 takes 16 lanes.  The pairs' frequencies stay in registers, shared out over the lanes that have the same columns of
// different heads; a row's angles are reduced to a turn in
// double (position times frequency reaches tens of thousands of radians, where a float would be off by more than the output's
// rounding) and their sine and cosine taken of what is left, in float for bf16 rows (an error of 2^-22 before a rounding of 2^-9) and in
// double for fp32 ones.  No shared memory, no barrier.
// What bounds it: latency for a decoding batch (slot and length, the angles, the stores), HBM for prompts.  With rotation, bf16: 32 requests' blocks
// of 16 rows, 32 and 8 heads of 128, 4.7 us (of which some 2.5 are a launch); 13 thousand rows of 16 and 4 heads of 128, 33 us, 4.9 TB/s.  fp32 7.3 and 62 us (5.2 TB/s);
// without rotation bf16 2.0 and 11.0, fp32 2.4 and 18.7 us.
#include <cmath>
#include <type_traits>
#include "paged.cuh"

namespace orthrus {
namespace {

template <typename T> struct Lanes;             // four consecutive elements; the type that rotates them
template <> struct Lanes<float> {
    using V = float4;
    using R = double;
    __device__ static void unpack(const V &v, R (&x)[4]) { x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
    __device__ static V pack(const R (&x)[4]) { return make_float4((float)x[0], (float)x[1], (float)x[2], (float)x[3]); }
    __device__ static void turn(double t, R &s, R &c) { sincospi(2.0 * t, &s, &c); }
};
template <> struct Lanes<__nv_bfloat16> {
    using V = uint2;
    using R = float;
    __device__ static void unpack(const V &v, R (&x)[4]) {
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
    }
    __device__ static V pack(const R (&x)[4]) {
        V v;
        reinterpret_cast<__nv_bfloat162 &>(v.x) = __floats2bfloat162_rn(x[0], x[1]);
        reinterpret_cast<__nv_bfloat162 &>(v.y) = __floats2bfloat162_rn(x[2], x[3]);
        return v;
    }
    __device__ static void turn(double t, R &s, R &c) { sincospif(2.f * (float)t, &s, &c); }
};

struct WriteArgs {
    const void *q, *k_blk, *v_blk;
    void *q_out, *k_pages, *v_pages;
    const int64_t *slot_map;
    const int32_t *cache_len;
    int32_t *status;
    long long rows, n_slots;
    int K, Hq, Hkv, page_shift, chunks, per_chunk;     // a row's heads in `chunks` pieces of per_chunk
    double log2_theta;
};

template <typename T, int D, bool ROPE>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) paged_write_kernel(const WriteArgs a)
{
    using R = typename Lanes<T>::R;
    using V = typename Lanes<T>::V;
    constexpr int N = 4, HALF = D / 2, LPH = HALF / N, HPI = 32 / LPH;      // lanes per head, heads per step of a warp
    constexpr int U = 2;                                              // steps whose loads are under way together
    const int lane = threadIdx.x & 31, sub = lane / LPH, c = (lane % LPH) * N;
    // lanes with the same columns of different heads share the angles of these: A each
    constexpr int A = N > HPI ? N / HPI : 1;
    double freq[A];                                                   // turns per position
    if (ROPE)
#pragma unroll
        for (int j = 0; j < A; ++j)
            freq[j] = exp2(-2.0 * (double)(c + min(sub * A + j, N - 1)) / (double)D * a.log2_theta) * 0.15915494309189533577;
    pdl_begin();
    const int Hq = ROPE ? a.Hq : 0, heads = Hq + a.Hkv;
    const T *q = static_cast<const T *>(a.q), *kb = static_cast<const T *>(a.k_blk), *vb = static_cast<const T *>(a.v_blk);
    T *qo = static_cast<T *>(a.q_out), *kp = static_cast<T *>(a.k_pages), *vp = static_cast<T *>(a.v_pages);
    auto at = [](auto *p) { return reinterpret_cast<std::conditional_t<std::is_const_v<std::remove_pointer_t<decltype(p)>>, const V, V> *>(p); };
    const long long n_items = a.rows * a.chunks, stride = (long long)gridDim.x * 8;
    // slot and position of an item's row, an item ahead
    auto look = [&](long long it, long long &slot, int &pos) {
        const long long row = it / a.chunks, b = row / a.K;
        slot = a.slot_map[row];
        pos = ROPE ? max(a.cache_len[b], 0) + (int)(row - b * a.K) : 0;
    };
    long long it = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), slot = -1, next_slot = -1;
    int pos = 0, next_pos = 0;
    if (it < n_items) look(it, next_slot, next_pos);
#pragma unroll 1
    for (; it < n_items; it += stride) {
        slot = next_slot;
        pos = next_pos;
        if (it + stride < n_items) look(it + stride, next_slot, next_pos);
        if (slot < 0) continue;
        const long long row = it / a.chunks;
        const int h0 = (int)(it - row * a.chunks) * a.per_chunk, h1 = min(heads, h0 + a.per_chunk);
        const bool room = slot < a.n_slots;
        if (!room && a.status && lane == 0 && h0 == 0) atomicOr(a.status, ORTHRUS_DEV_BAD_PAGE);
        const long long page = slot >> a.page_shift;
        const int in_page = (int)(slot & ((1 << a.page_shift) - 1));
        R s[N], co[N];
#pragma unroll 1
        for (int hh = h0 + sub; hh - sub < h1; hh += HPI * U) {
            V lo[U], hi[U], vl[U], vh[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = hh + u * HPI;
                if (h >= h1) continue;
                if (h < Hq) {
                    const T *src = q + (row * Hq + h) * D + c;
                    lo[u] = *at(src); hi[u] = *at(src + HALF);
                } else {
                    const long long off = (row * a.Hkv + h - Hq) * D + c;
                    lo[u] = *at(kb + off); hi[u] = *at(kb + off + HALF);
                    vl[u] = *at(vb + off); vh[u] = *at(vb + off + HALF);
                }
            }
            if (ROPE && hh == h0 + sub) {                     // (while the first loads are under way)
                R sa[A], ca[A];
#pragma unroll
                for (int j = 0; j < A; ++j) {
                    const double t = (double)pos * freq[j];
                    Lanes<T>::turn(t - rint(t), sa[j], ca[j]);
                }
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    s[j] = __shfl_sync(0xffffffffu, sa[j % A], lane % LPH + LPH * (j / A));
                    co[j] = __shfl_sync(0xffffffffu, ca[j % A], lane % LPH + LPH * (j / A));
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = hh + u * HPI;
                if (h >= h1) continue;
                if (ROPE) {
                    R x0[N], x1[N], y0[N], y1[N];
                    Lanes<T>::unpack(lo[u], x0);
                    Lanes<T>::unpack(hi[u], x1);
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        y0[j] = x0[j] * co[j] - x1[j] * s[j];
                        y1[j] = x1[j] * co[j] + x0[j] * s[j];
                    }
                    lo[u] = Lanes<T>::pack(y0);
                    hi[u] = Lanes<T>::pack(y1);
                }
                if (h < Hq) {
                    T *dst = qo + (row * Hq + h) * D + c;
                    *at(dst) = lo[u]; *at(dst + HALF) = hi[u];
                } else if (room) {
                    const long long dst = (((page * a.Hkv + h - Hq) << a.page_shift) + in_page) * D + c;
                    *at(kp + dst) = lo[u]; *at(kp + dst + HALF) = hi[u];
                    *at(vp + dst) = vl[u]; *at(vp + dst + HALF) = vh[u];
                }
            }
        }
    }
}

template <typename T, bool ROPE>
cudaError_t launch_width(bool early, int d, int blocks, cudaStream_t st, const WriteArgs &a)
{
    switch (d) {
    case 32: return launch_kernel(early, paged_write_kernel<T, 32, ROPE>, dim3(blocks), 256, 0, st, a);
    case 64: return launch_kernel(early, paged_write_kernel<T, 64, ROPE>, dim3(blocks), 256, 0, st, a);
    case 128: return launch_kernel(early, paged_write_kernel<T, 128, ROPE>, dim3(blocks), 256, 0, st, a);
    default: return launch_kernel(early, paged_write_kernel<T, 256, ROPE>, dim3(blocks), 256, 0, st, a);
    }
}

}  // namespace

cudaError_t launch_paged_kv_write(const orthrus_paged_layer_t &L, const int64_t *slot_map, const void *q, const void *k_blk,
                                  const void *v_blk, double theta, void *q_out, int32_t *status, cudaStream_t st)
{
    WriteArgs a;
    a.q = q; a.k_blk = k_blk; a.v_blk = v_blk; a.q_out = q_out; a.k_pages = L.k_pages; a.v_pages = L.v_pages;
    a.slot_map = slot_map; a.cache_len = L.cache_len; a.status = status;
    a.page_shift = __builtin_ctz((unsigned)L.page_size);
    a.rows = (long long)L.batch * L.block; a.n_slots = (long long)L.n_pages << a.page_shift;
    a.K = L.block; a.Hq = L.n_q_heads; a.Hkv = L.n_kv_heads;
    a.log2_theta = q ? log2(theta) : 0.0;
    // A row's heads by several warps where the rows alone do not fill the GPU
    const int heads = (q ? L.n_q_heads : 0) + L.n_kv_heads, hpi = 256 / L.head_dim;     // (heads per step)
    const long long room = 32LL * num_sms();
    const int least = 2 * hpi;                               // one round of a warp's loads
    long long chunks = (room + a.rows - 1) / a.rows;
    const int most = (heads + least - 1) / least;
    if (chunks > most) chunks = most;
    if (chunks < 1) chunks = 1;
    a.per_chunk = (int)(((heads + chunks - 1) / chunks + least - 1) / least * least);
    a.chunks = (heads + a.per_chunk - 1) / a.per_chunk;
    const long long want = (a.rows * a.chunks + 7) / 8, cap = 32LL * num_sms();
    const int blocks = (int)(want < cap ? want : cap);
    const bool early = !(L.flags & ORTHRUS_LAYER_NO_EARLY_LAUNCH);
    if (L.dtype == ORTHRUS_FP32)
        return q ? launch_width<float, true>(early, L.head_dim, blocks, st, a) : launch_width<float, false>(early, L.head_dim, blocks, st, a);
    return q ? launch_width<__nv_bfloat16, true>(early, L.head_dim, blocks, st, a)
             : launch_width<__nv_bfloat16, false>(early, L.head_dim, blocks, st, a);
}

}  // namespace orthrus
