// Attention over pages in fp32 arithmetic: the fp32 test mode, and the shapes that the tensor-core kernel does not take (head_dim 32 and
// 256, pages of fewer than 16 positions).  A CTA takes a unit's tile of 16 query rows and walks its keys, 32 at a time, a lane a
// key: scores, the tile's maximum and sum by butterfly reductions, the probabilities broadcast lane by lane for the values.  The keys of a unit
// are not cut over CTAs.  Not tuned.
#include "paged.cuh"

namespace orthrus {
namespace {

constexpr int TN = 32, MT = 16, RW = 4;          // keys per tile, query rows per CTA and per warp

__device__ inline float to_f(float x) { return x; }
__device__ inline float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ inline void put(float *p, float x) { *p = x; }
__device__ inline void put(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }

template <typename T, int DPL>
__global__ void __launch_bounds__(128) paged_attend_simt_kernel(const PagedParams p)
{
    constexpr int D = DPL * 32;
    extern __shared__ float smem[];
    float *sK = smem;                    // [TN][D + 1]
    float *sV = sK + TN * (D + 1);       // [TN][D]
    float *sQ = sV + TN * D;             // [MT][D]
    pdl_begin();
    const int unit = blockIdx.x, b = unit / p.Hkv, h = unit - b * p.Hkv, r0 = blockIdx.y * MT;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int P, n;
    bool bad;
    paged_request(p, b, P, n, bad);
    if (bad && h == 0 && blockIdx.y == 0 && tid == 0 && p.status) atomicOr(p.status, ORTHRUS_DEV_BAD_CACHE_LEN);
    const int M = n * p.G;
    if (r0 >= M) return;
    const T *q = static_cast<const T *>(p.q), *kp = static_cast<const T *>(p.k_pages), *vp = static_cast<const T *>(p.v_pages);
    for (int e = tid; e < MT * D; e += 128) {
        const int R = r0 + e / D, c = e % D;
        sQ[e] = R < M ? to_f(q[(((long long)b * p.K + R / p.G) * p.Hq + h * p.G + R % p.G) * D + c]) : 0.f;
    }
    float o[RW][DPL], m[RW], l[RW];
#pragma unroll
    for (int rr = 0; rr < RW; ++rr) {
        m[rr] = -INFINITY; l[rr] = 0.f;
#pragma unroll
        for (int k = 0; k < DPL; ++k) o[rr][k] = 0.f;
    }
    // keys that any row of this tile sees
    const int keys = p.causal ? P + min(n, (r0 + MT - 1) / p.G + 1) : P + n;
    for (int t0 = 0; t0 < keys; t0 += TN) {
        __syncthreads();
        for (int j = warp; j < TN; j += 4) {
            const int pos = t0 + j;
            const int32_t page = pos < keys ? p.table[(long long)b * p.max_pages + (pos >> p.page_shift)] : -1;
            const bool in = page >= 0 && page < p.n_pages;
            if (pos < keys && !in && lane == 0 && p.status) atomicOr(p.status, ORTHRUS_DEV_BAD_PAGE);
            const long long row = ((((long long)page * p.Hkv + h) << p.page_shift) + (pos & ((1 << p.page_shift) - 1))) * D;
#pragma unroll
            for (int k = 0; k < DPL; ++k) {
                sK[j * (D + 1) + k * 32 + lane] = in ? to_f(kp[row + k * 32 + lane]) : 0.f;
                sV[j * D + k * 32 + lane] = in ? to_f(vp[row + k * 32 + lane]) : 0.f;
            }
        }
        __syncthreads();
#pragma unroll
        for (int rr = 0; rr < RW; ++rr) {
            const int r = warp * RW + rr, R = r0 + r;
            if (R >= M) continue;                        // the same for the whole warp
            const int sees = p.causal ? P + R / p.G + 1 : P + n;
            float s = 0.f;
            const float *qr = sQ + r * D, *kr = sK + lane * (D + 1);
#pragma unroll 8
            for (int c = 0; c < D; ++c) s = fmaf(qr[c], kr[c], s);
            s = t0 + lane < sees ? s * p.scale_log2 : -INFINITY;
            float top = s;
#pragma unroll
            for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float m_new = fmaxf(m[rr], top), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = exp2f(m[rr] - ref), pj = exp2f(s - ref);
            float sum = pj;
#pragma unroll
            for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            l[rr] = l[rr] * alpha + sum;
            m[rr] = m_new;
#pragma unroll
            for (int k = 0; k < DPL; ++k) o[rr][k] *= alpha;
            const int seen = min(TN, sees - t0);
            for (int j = 0; j < seen; ++j) {             // (values behind what the row sees are not touched)
                const float w = __shfl_sync(0xffffffffu, pj, j);
#pragma unroll
                for (int k = 0; k < DPL; ++k) o[rr][k] = fmaf(w, sV[j * D + k * 32 + lane], o[rr][k]);
            }
        }
    }
#pragma unroll
    for (int rr = 0; rr < RW; ++rr) {
        const int R = r0 + warp * RW + rr;
        if (R >= M) continue;
        T *out = static_cast<T *>(p.out) + (((long long)b * p.K + R / p.G) * p.Hq + h * p.G + R % p.G) * D;
#pragma unroll
        for (int k = 0; k < DPL; ++k) put(out + k * 32 + lane, o[rr][k] / l[rr]);
    }
}

template <typename T, int DPL> cudaError_t launch_one(const PagedParams &p, cudaStream_t st)
{
    constexpr int D = DPL * 32, smem = (TN * (D + 1) + TN * D + MT * D) * (int)sizeof(float);
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = configure(paged_attend_simt_kernel<T, DPL>, done, smem, false);
    if (e != cudaSuccess) return e;
    return launch_kernel(p.early, paged_attend_simt_kernel<T, DPL>, dim3(p.B * p.Hkv, (p.K * p.G + MT - 1) / MT), 128, smem, st, p);
}
template <typename T> cudaError_t launch_width(const PagedParams &p, cudaStream_t st)
{
    switch (p.d) {
    case 32: return launch_one<T, 1>(p, st);
    case 64: return launch_one<T, 2>(p, st);
    case 128: return launch_one<T, 4>(p, st);
    default: return launch_one<T, 8>(p, st);
    }
}

}  // namespace

cudaError_t launch_paged_attend_simt(const PagedParams &p, int dtype, cudaStream_t st)
{
    return dtype == ORTHRUS_FP32 ? launch_width<float>(p, st) : launch_width<__nv_bfloat16>(p, st);
}

}  // namespace orthrus
