// Attention over the pages of a paged cache for units of at most 16 query rows, bf16, head_dim 64 and 128: one new token a request at up
// to 16 query heads per KV head, short blocks of narrower groups.
//
//   s_j = q . k_j * scale,   m = max s,   out = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m)      (s in the log2 domain)
//
// One pass over the keys with a running maximum and sum.  What bounds it: HBM, 4 d bytes per key and KV head; 1 to 16 query rows are 2 to
// 32 flops a byte, so that warp-level MMAs of 16 query rows, even half empty, take a tenth of the time the keys take to arrive.
//
// Work is cut by tiles of 64 keys, not by requests: all tiles of all units (request, KV head) lie on one line, and CTA c of n takes the
// stretch [c T / n, (c + 1) T / n).  Every CTA finds its stretch from the lengths themselves, so that the host needs no plan, a captured graph
// serves any lengths, and a batch of unequal requests loads all SMs alike.  A unit that is cut leaves pieces (unnormalised sums with their
// maximum) in the workspace; the CTA that finishes last, by the unit's counter, joins them in the order of their keys, which fixes the result.
//
// CTA of 160 threads, two to an SM:
//   warp 4     producer: looks up pages, brings K and V tiles by TMA into a ring (a box per page, 64 rows at most, 128-byte
//              swizzle), running on into the next unit of the stretch while the consumers finish this one
//   warps 0-3  consumers: 16 keys of each tile; a warp keeps maximum, sum and output of its own keys in registers and meets the
//              others at the end of a unit only
// Every wait is bounded: on expiry the CTA raises ORTHRUS_DEV_WAIT_TIMEOUT, waits for its copies in flight and ends.
#include <cuda.h>
#include "paged_stretch.cuh"

namespace orthrus {
namespace {

constexpr int MR = 16, CW = 4, PRODUCER = 4, NTHREADS = 160;

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

template <int HD> struct Shape {
    static constexpr int TILE = KT * HD * 2;                                  // bytes of a K or V tile
    static constexpr int BUF_BYTES = MR * HD * 4, STAT_BYTES = CW * MR * 4;    // (the query rows are in the output's place until the unit ends)
    static constexpr int ROOM = (113 * 1024 - BUF_BYTES - STAT_BYTES - 2 * MR * 4 - 160) / (2 * TILE), STAGES = ROOM < 6 ? ROOM : 6;
    static constexpr int OFF_BUF = STAGES * 2 * TILE, OFF_STAT = OFF_BUF + BUF_BYTES, OFF_ML = OFF_STAT + STAT_BYTES,
                         OFF_BAR = OFF_ML + 2 * MR * 4;
    static constexpr int SMEM = OFF_BAR + 3 * STAGES * 8 + 16;
    static_assert(STAGES >= 3 && SMEM <= 113 * 1024, "shared memory of two CTAs");
};

template <int HD>
__global__ void __launch_bounds__(NTHREADS, 2)
paged_attend_kernel(const __grid_constant__ PagedParams p, const __grid_constant__ PagedMaps tm, const __grid_constant__ PagedWork w)
{
    using C = Shape<HD>;
    constexpr int STAGES = C::STAGES, TILE = C::TILE, ND = HD / 8;
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t sbase = smem_u32(smem);
    float *buf = reinterpret_cast<float *>(smem + C::OFF_BUF);
    float *stat = reinterpret_cast<float *>(smem + C::OFF_STAT);       // [warp][row]: maxima
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
    const int U = p.Hkv, page = 1 << p.page_shift;
    Stretch s;
    Piece x;

    if (warp == PRODUCER) {
        // ------------------------------------------------------------------ producer
        bool waited = false;
        auto wait = [&] { griddep_wait(); griddep_launch(); waited = true; };
        if (!p.quiescent) wait();
        int issued = 0;
        if (lane == 0) { prefetch_map(&tm.k); prefetch_map(&tm.v); }
        if (find_stretch(p, U, blockIdx.x, gridDim.x, w.most_pieces, lane, blockIdx.x == 0, s)) {
            const long long start = s.pos;
            const uint64_t policy = policy_evict_first();
            const int box = 1 << w.box_shift;
            bool ok = true;
            PageWindow pages;
            while (ok && next_piece(p, s, start, lane, x)) {
                const int h = x.u, keys = x.P + x.n;
                pages.open(p, x, lane);
                for (int t = x.t0; ok && t < x.t1; ++t) {
                    const int pos0 = t * KT;
                    if (!waited && pos0 + KT > x.P) wait();                                   // rows of the block itself
                    const int last = min(pos0 + KT, keys) - 1;
                    const int i = lane & 3, kind = lane >> 2;                                 // lanes 0-3: K boxes, 4-7: V boxes
                    const int pos = pos0 + (i << w.box_shift), pg = pages.page(p, pos, last, lane);
                    const int st = issued % STAGES;
                    if (issued >= STAGES) ok = mbar_wait_warp(bar_free(st), (issued / STAGES + 1) & 1, abort_flag);
                    if (!ok) break;
                    const int live = ((last - pos0) >> w.box_shift) + 1;                      // boxes with rows in them
                    if (lane == 0) {
                        mbar_expect_tx(bar_k(st), live * box * HD * 2);
                        mbar_expect_tx(bar_v(st), live * box * HD * 2);
                    }
                    __syncwarp();
                    if (lane < 8 && i < live) {
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
        const int wk = warp, g = lane >> 2, tq = lane & 3;
        const uint32_t sq = sbase + C::OFF_BUF;
        // per-lane parts of the addresses that ldmatrix takes: row, then the swizzled 16-byte chunk
        const int kr = (lane & 7) + ((lane >> 4) << 3), kc = (lane >> 3) & 1;
        const int vr = (lane & 7) + (((lane >> 3) & 1) << 3), vc = lane >> 4;
        const uint32_t panel = 128u << w.box_shift;
        const uint32_t box_bytes = (uint32_t)(HD * 2) << w.box_shift;
        // this warp's 16 keys in a tile of boxes
        const int bx = (wk * 16) >> w.box_shift;
        const uint32_t group = bx * box_bytes + (wk * 16 - (bx << w.box_shift)) * 128;
        const uint32_t k_lane = group + kr * 128 + ((kc ^ (kr & 7)) << 4), v_lane = group + TILE + vr * 128 + ((vc ^ (vr & 7)) << 4);
        bool ok = find_stretch(p, U, blockIdx.x, gridDim.x, w.most_pieces, lane, false, s);
        const long long start = ok ? s.pos : 0;
        int used = 0;
        while (ok && next_piece(p, s, start, lane, x)) {
            const int h = x.u, M = x.n * p.G, keys = x.P + x.n;
            // the unit's query rows, 128-byte swizzled panels of 64 columns; rows that do not exist are zero
            const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p.q);
            bar_consumers();                       // (the last unit's rows are done with)
            for (int e = tid; e < MR * (HD / 8); e += 128) {
                const int r = e / (HD / 8), c = e % (HD / 8);
                uint4 val = make_uint4(0, 0, 0, 0);
                if (r < M) val = *reinterpret_cast<const uint4 *>(q + row_offset(p, x.b, h, r, HD) + c * 8);
                *reinterpret_cast<uint4 *>(smem + C::OFF_BUF + (c >> 3) * (MR * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = val;
            }
            bar_consumers();
            const uint32_t q_lane = sq + vr * 128 + ((vc ^ (vr & 7)) << 4);
            // what the rows of this lane see
            int sees[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) sees[e] = p.causal ? min(keys, x.P + (g + e * 8) / p.G + 1) : keys;
            float o[ND][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
            for (int j = 0; j < ND; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
            for (int t = x.t0; t < x.t1; ++t, ++used) {
                const int st = used % STAGES, parity = (used / STAGES) & 1, pos0 = t * KT + wk * 16;
                if (!mbar_wait_warp(bar_k(st), parity, abort_flag)) { ok = false; break; }
                const uint32_t sk = sbase + st * 2 * TILE + k_lane, sv = sbase + st * 2 * TILE + v_lane;
                float sc[2][4];
#pragma unroll
                for (int j = 0; j < 2; ++j) sc[j][0] = sc[j][1] = sc[j][2] = sc[j][3] = 0.f;
#pragma unroll
                for (int ks = 0; ks < HD / 16; ++ks) {
                    uint32_t qf[4], kf[4];                 // (the rows' fragments again for every tile: their registers are the output's)
                    ldmatrix_x4(qf, (q_lane ^ (((ks * 2) & 7) << 4)) + (ks >> 2) * (MR * 128));
                    ldmatrix_x4(kf, (sk ^ (((ks * 2) & 7) << 4)) + (ks >> 2) * panel);
                    mma_bf16(sc[0], qf, kf[0], kf[1]);
                    mma_bf16(sc[1], qf, kf[2], kf[3]);
                }
                if (pos0 + 16 > x.P) {                     // some keys are the block's own, or do not exist
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int pos = pos0 + j * 8 + tq * 2;
                        if (pos >= sees[0]) sc[j][0] = -INFINITY;
                        if (pos + 1 >= sees[0]) sc[j][1] = -INFINITY;
                        if (pos >= sees[1]) sc[j][2] = -INFINITY;
                        if (pos + 1 >= sees[1]) sc[j][3] = -INFINITY;
                    }
                }
                float top[2] = {fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[1][0], sc[1][1])),
                                fmaxf(fmaxf(sc[0][2], sc[0][3]), fmaxf(sc[1][2], sc[1][3]))};
                float ref[2], al[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 1));
                    top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 2));
                    const float mn = fmaxf(m[e], top[e] * p.scale_log2);
                    ref[e] = mn == -INFINITY ? 0.f : mn;             // (of nothing so far: no factor)
                    al[e] = ex2(m[e] - ref[e]);
                    m[e] = mn;
                }
                float pr[2][4];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) pr[j][e] = ex2(fmaf(sc[j][e], p.scale_log2, -ref[e >> 1]));
                const uint32_t pf[4] = {pack_bf16(pr[0][0], pr[0][1]), pack_bf16(pr[0][2], pr[0][3]), pack_bf16(pr[1][0], pr[1][1]),
                                        pack_bf16(pr[1][2], pr[1][3])};
                l[0] = fmaf(l[0], al[0], (pr[0][0] + pr[0][1]) + (pr[1][0] + pr[1][1]));
                l[1] = fmaf(l[1], al[1], (pr[0][2] + pr[0][3]) + (pr[1][2] + pr[1][3]));
                if (__any_sync(0xffffffffu, al[0] != 1.f || al[1] != 1.f)) {
#pragma unroll
                    for (int j = 0; j < ND; ++j) { o[j][0] *= al[0]; o[j][1] *= al[0]; o[j][2] *= al[1]; o[j][3] *= al[1]; }
                }
                if (!mbar_wait_warp(bar_v(st), parity, abort_flag)) { ok = false; break; }
                if (pos0 + 16 > keys) {
                    // rows behind the last key, which may hold anything: zero, for the product with their zero probabilities
                    for (int r = max(0, keys - pos0); r < 16; ++r)
                        if (lane < HD / 8)
                            *reinterpret_cast<uint4 *>(smem + (st * 2 + 1) * TILE + group + r * 128 + (lane >> 3) * panel + (lane & 7) * 16) =
                                make_uint4(0, 0, 0, 0);
                    __syncwarp();
                }
#pragma unroll
                for (int dp = 0; dp < HD / 16; ++dp) {
                    uint32_t vf[4];
                    ldmatrix_x4_trans(vf, (sv ^ (((dp * 2) & 7) << 4)) + (dp >> 2) * panel);
                    mma_bf16(o[2 * dp], pf, vf[0], vf[1]);
                    mma_bf16(o[2 * dp + 1], pf, vf[2], vf[3]);
                }
                if (pos0 + 16 > keys) fence_proxy_async();        // the zeros before the next copy into the slot
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_free(st));
            }

            // the warps' results of their own keys become the unit's (or the piece's): common maximum, then added up in turn
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
                l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
                if (tq == 0) stat[warp * MR + g + e * 8] = m[e];
            }
            ok = bar_consumers_and(ok);            // (a warp whose wait ran out has come here too: all leave together)
            if (!ok) break;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = g + e * 8;
                float top = -INFINITY;
#pragma unroll
                for (int k = 0; k < CW; ++k) top = fmaxf(top, stat[k * MR + r]);
                const float al = top == -INFINITY ? 0.f : ex2(m[e] - top);
                l[e] *= al;
                m[e] = top;
#pragma unroll
                for (int j = 0; j < ND; ++j) { o[j][e * 2] *= al; o[j][e * 2 + 1] *= al; }
            }
#pragma unroll 1
            for (int k = 0; k < CW; ++k) {
                if (wk == k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = g + e * 8;
                        if (r >= M) continue;
#pragma unroll
                        for (int j = 0; j < ND; ++j) {
                            float2 *dst = reinterpret_cast<float2 *>(buf + at(r, j * 8 + tq * 2));
                            float2 v = make_float2(o[j][e * 2], o[j][e * 2 + 1]);
                            if (k) { const float2 y = *dst; v.x += y.x; v.y += y.y; }
                            *dst = v;
                        }
                        if (tq == 0) { ml[r] = m[e]; ml[MR + r] = l[e] + (k ? ml[MR + r] : 0.f); }
                    }
                bar_consumers();
            }
            const int rows = min(MR, M);
            auto put = [&](int r, int c, const float4 &v, float inv) {
                *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.out) + row_offset(p, x.b, h, r, HD) + c) =
                    make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
            };
            // VR lanes a row, four columns each
            constexpr int VR = HD / 4, RPW = 128 / VR;
            const int c = (tid % VR) * 4, r_first = tid / VR;
            if (x.t0 == 0 && x.t1 == x.tiles) {
                for (int r = r_first; r < rows; r += RPW)
                    put(r, c, *reinterpret_cast<const float4 *>(buf + at(r, c)), 1.f / ml[MR + r]);
                continue;
            }
            const size_t step = piece_floats(w.rows, HD), stats = (size_t)w.rows * HD;
            float *mine = w.pieces + (2 * blockIdx.x + (x.first ? 0 : 1)) * step;
            for (int r = r_first; r < rows; r += RPW)
                *reinterpret_cast<float4 *>(mine + r * HD + c) = *reinterpret_cast<const float4 *>(buf + at(r, c));
            if (tid < rows) *reinterpret_cast<float2 *>(mine + stats + tid * 2) = make_float2(ml[tid], ml[MR + tid]);
            const int c0 = owner(s, x.unit0), n = owner(s, x.unit0 + x.tiles - 1) - c0 + 1;
            bar_consumers();
            if (tid == 0) {
                int *counter = w.counter + (long long)x.b * U + x.u;
                __threadfence();
                const bool last = atomicAdd(counter, 1) == n - 1;
                if (last) { *counter = 0; __threadfence(); }
                *last_flag = last;
            }
            bar_consumers();
            if (!*last_flag) continue;
            // The first piece is its CTA's first only if the unit begins with the stretch; the others begin theirs.  The lanes of a row hold the
            // weights of its pieces, lane j those of j, j + VR, ...
            const float *first = w.pieces + (2 * c0 + (s.T * c0 / s.n == x.unit0 ? 0 : 1)) * step, *others = w.pieces + 2 * c0 * step;
            auto piece = [&](int k) { return k ? others + 2 * k * step : first; };
            constexpr int HELD = 64 / VR;
            const int j0 = tid % VR;
#pragma unroll 1
            for (int r = r_first; r < rows; r += RPW) {
                float2 st[HELD];
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < HELD; ++i) {
                    const int k = j0 + i * VR;
                    st[i] = k < n ? __ldcg(reinterpret_cast<const float2 *>(piece(k) + stats + r * 2)) : make_float2(-INFINITY, 0.f);
                    top = fmaxf(top, st[i].x);
                }
                const unsigned lanes = VR == 32 ? 0xffffffffu : 0xffffu << (lane & 16);
#pragma unroll
                for (int off = VR / 2; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(lanes, top, off));
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < HELD; ++i) {
                    st[i].x = top == -INFINITY ? 0.f : ex2(st[i].x - top);
                    sum = fmaf(st[i].x, st[i].y, sum);
                }
#pragma unroll
                for (int off = VR / 2; off; off >>= 1) sum += __shfl_xor_sync(lanes, sum, off);
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int i = 0; i < HELD; ++i)
#pragma unroll 1
                    for (int k0 = i * VR; k0 < min(n, (i + 1) * VR); k0 += 16) {
                        float4 y[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (k0 + k < n) y[k] = __ldcg(reinterpret_cast<const float4 *>(piece(k0 + k) + r * HD + c));
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (k0 + k < n) {
                                const float al = __shfl_sync(lanes, st[i].x, (k0 + k) % VR, VR);
                                v.x = fmaf(y[k].x, al, v.x); v.y = fmaf(y[k].y, al, v.y); v.z = fmaf(y[k].z, al, v.z); v.w = fmaf(y[k].w, al, v.w);
                            }
                    }
                put(r, c, v, 1.f / sum);
            }
        }
    }
    __syncthreads();
    if (tid == 0 && *abort_flag && p.status) atomicOr(p.status, ORTHRUS_DEV_WAIT_TIMEOUT);
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

template <int HD>
cudaError_t launch_one(const PagedParams &p, const PagedMaps &tm, const PagedWork &w, int ctas, cudaStream_t st)
{
    using C = Shape<HD>;
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = configure(paged_attend_kernel<HD>, done, C::SMEM, false);
    if (e != cudaSuccess) return e;
    return launch_kernel(p.early, paged_attend_kernel<HD>, dim3(ctas), NTHREADS, C::SMEM, st, p, tm, w);
}

}  // namespace

cudaError_t launch_paged_attend_mma(const PagedParams &p, const PagedWork &w, unsigned long long rows, int ctas, cudaStream_t st)
{
    PagedMaps tm;
    if (!page_map(const_cast<void *>(p.k_pages), p.d, rows, 1u << w.box_shift, &tm.k) ||
        !page_map(const_cast<void *>(p.v_pages), p.d, rows, 1u << w.box_shift, &tm.v))
        return cudaErrorInvalidValue;
    return p.d == 128 ? launch_one<128>(p, tm, w, ctas, st) : launch_one<64>(p, tm, w, ctas, st);
}

}  // namespace orthrus
