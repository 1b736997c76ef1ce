// One token per row of logits: temperature, top-k, top-p and min-p, then inversion of the running mass with a given uniform.
//
// Every filter cuts the row, ordered by value falling and id rising, at one place; so does the draw.  A place is a value and a count of
// the ties at it, so that no sorting is needed: it is enough to know, for the values in order, how many tokens have them and what they weigh.
//   1. A cluster of CTAs counts its row's values in shared memory, one pass over the logits.  bf16 has few values: those with magnitude
//      2^-20 to 2^8 and zero have a bin each, what is outside shares four.  Weights are then needed once per value and not once per token (an
//      exponential in double precision for a few thousand values instead of 150 thousand tokens).  fp32: bins of 2^20 neighbouring
//      values, which carry counts and the sum of their tokens' weights; the maximum is found by a pass before.
//   2. Sums over groups of 32 bins go to one CTA, which finds the bin of each cut from them.
//   3. A cut in a bin of many values: another pass counts and weighs 1024 parts of that bin, until a part is one value.
//   4. The CTA that holds the wanted occurrence of the drawn value finds its id.
// Weights are integers, exp((x - max) / T) in steps of 2^-S with 2^S times the vocabulary below 2^63: sums do not depend on the
// order in which atomics arrive, are exact, and a border is off by no more than the weights' own rounding.
//
// What bounds it: one row, latency (five dependent steps at the cluster's barriers); many rows, the atomics in shared memory (one a
// token for bf16, three for fp32 next to an exponential in double).
#include <cooperative_groups.h>
#include <cmath>
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace cg = cooperative_groups;

namespace orthrus {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kParts = 1024;                       // parts of a bin that a cut falls into
constexpr uint32_t kNone = 0xffffffffu;            // no candidate: NaN, -inf

// Values as whole numbers that rise as the value falls; -0 is 0.  Bins of neighbouring ones.
template <typename T> struct Keys;
template <> struct Keys<__nv_bfloat16> {
    static constexpr int N = 8;                                        // elements of 16 bytes
    static constexpr uint32_t LO = 107u << 7, HI = 135u << 7;          // magnitudes 2^-20 and 2^8
    static constexpr int FINE = HI - LO, BINS = 2 * FINE + 5, STEPS = (BINS + 31) / 32, WEIGHED = 4;
    using Raw = uint16_t;
    __device__ static uint32_t key(uint32_t h) {                       // h: the 16 bits
        const uint32_t mag = h & 0x7fff;
        if (mag >= 0x7f80 && h != 0x7f80) return kNone;
        return mag == 0 || !(h & 0x8000) ? 0x7fff - mag : 0x8000 + mag;
    }
    __device__ static double value(uint32_t d) {
        const uint32_t h = d <= 0x7fff ? 0x7fff - d : d;               // (0x8000 + mag are the bits themselves)
        return (double)__uint_as_float(h << 16);
    }
    __device__ static int bin(uint32_t d) {
        if (d == 0x7fff) return FINE + 2;
        const uint32_t mag = d < 0x7fff ? 0x7fff - d : d - 0x8000;
        const int t = (int)(min(max(mag, LO - 1), HI) - (LO - 1));
        return d < 0x7fff ? FINE + 1 - t : FINE + 3 + t;
    }
    // the bin of an element, straight from its bits; < 0: no candidate
    __device__ static int bin_of(uint32_t h) {
        const uint32_t mag = h & 0x7fff;
        const int t = (int)(min(max(mag, LO - 1), HI) - (LO - 1));
        int b = h & 0x8000 ? FINE + 3 + t : FINE + 1 - t;
        if (mag - 1 >= 0x7f7f) b = mag == 0 ? FINE + 2 : h == 0x7f80 ? 0 : -1;
        return b;
    }
    // first value of a bin; which of the bins of many values it is (-1: it is one value)
    __device__ static uint32_t first(int b) {
        if (b == 0) return 0;
        if (b <= FINE) return 0x7fff - (HI - b);
        if (b == FINE + 1) return 0x7fff - (LO - 1);
        if (b == FINE + 2) return 0x7fff;
        if (b == FINE + 3) return 0x8001;
        return 0x8000 + LO + (uint32_t)(b - FINE - 4);
    }
    __device__ static int weighed(int b) { return b == 0 ? 0 : b == FINE + 1 ? 1 : b == FINE + 3 ? 2 : b == BINS - 1 ? 3 : -1; }
    static constexpr int BITS = 15;                                     // a bin has at most 2^BITS values
    template <class F> __device__ static void each(const uint4 &u, F f) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) { f(2 * k, w[k] & 0xffffu); f(2 * k + 1, w[k] >> 16); }
    }
};
template <> struct Keys<float> {
    static constexpr int N = 4;
    static constexpr int BITS = 20, BINS = 4096, STEPS = BINS / 32, WEIGHED = BINS;
    using Raw = uint32_t;
    __device__ static uint32_t key(uint32_t h) {
        const uint32_t mag = h & 0x7fffffffu;
        if (mag >= 0x7f800000u && h != 0x7f800000u) return kNone;
        return mag == 0 || !(h >> 31) ? 0x7fffffffu - mag : h;
    }
    __device__ static double value(uint32_t d) { return (double)__uint_as_float(d <= 0x7fffffffu ? 0x7fffffffu - d : d); }
    __device__ static int bin(uint32_t d) { return (int)(d >> BITS); }
    __device__ static uint32_t first(int b) { return (uint32_t)b << BITS; }
    __device__ static int weighed(int b) { return b; }
    template <class F> __device__ static void each(const uint4 &u, F f) { f(0, u.x); f(1, u.y); f(2, u.z); f(3, u.w); }
};

struct SampleArgs {
    const void *logits;
    long long stride;
    int vocab, scale_bits;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k;
    int32_t *token;
    float *logprob;
};

// A sum of 64 bits as two of 32 that atomics can add to
struct Sum { uint32_t lo, hi; };
__device__ inline void add_to(Sum *s, unsigned long long x) {
    const uint32_t lo = (uint32_t)x, old = atomicAdd(&s->lo, lo), hi = (uint32_t)(x >> 32) + (old + lo < lo);
    if (hi) atomicAdd(&s->hi, hi);
}
__device__ inline unsigned long long whole(const Sum &s) { return (unsigned long long)s.hi << 32 | s.lo; }

// A place in the order: token number `tie` (from 0) of those with key d, which weigh w each; before it, and by its CTAs
struct Place { uint32_t d, tie, count_before, owner, owner_tie; int bin; unsigned long long mass_before, w; };

template <typename T> struct Shared {
    uint32_t count[Keys<T>::STEPS * 32];
    Sum mass[Keys<T>::WEIGHED];
    uint32_t part_count[kParts];
    Sum part_mass[kParts];
    unsigned long long step_mass[Keys<T>::STEPS + 1];    // CTA 0: sums of the groups of 32 bins, then of all before
    uint32_t step_count[Keys<T>::STEPS + 1];
    unsigned long long part_step_mass[kParts / 32 + 1];  // likewise for the parts
    uint32_t part_step_count[kParts / 32 + 1];
    Place place;
    uint32_t top, per_warp[kWarps];
};

enum Mode { BY_COUNT, BY_MASS, BY_KEY };

__device__ inline unsigned long long scan_sum(unsigned long long x, int lane) {
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    return x;
}

template <typename T>
struct Sampler {
    using K = Keys<T>;
    Shared<T> &sh;
    const SampleArgs &a;
    cg::cluster_group cluster;
    const T *row;
    int tid, lane, warp, C, rank;
    int skew, n_vec, v0, v1;               // vector v: elements [v N - skew, v N - skew + N); this CTA's vectors
    uint32_t top;                          // key of the largest
    double x_top, inv_t, scale;

    __device__ void meet() { if (C > 1) cluster.sync(); else __syncthreads(); }
    __device__ Shared<T> *of(int r) { return C > 1 ? cluster.map_shared_rank(&sh, r) : &sh; }
    __device__ double share(uint32_t d) const {            // exp((x - max) / T)
        if (d == top) return 1.0;
        const double y = K::value(d) - x_top;
        return y == -INFINITY ? 0.0 : exp(y * inv_t);
    }
    __device__ unsigned long long weight(uint32_t d) const { return __double2ull_rn(share(d) * scale); }

    // f(element, bits) for the elements of vectors [b, e), lanes and warps (or one warp's lanes) side by side
    template <class F> __device__ void elements(int b, int e, int at, int step, F f) const {
        const uint4 *vec = reinterpret_cast<const uint4 *>(row - skew);
        int v = b + at;
        auto part = [&](int v) {
            const int i0 = v * K::N - skew;
            for (int k = max(0, -i0); k < min(K::N, a.vocab - i0); ++k) f(i0 + k, (uint32_t)reinterpret_cast<const typename K::Raw *>(row)[i0 + k]);
        };
        auto is_whole = [&](int v) { return v * K::N >= skew && v * K::N - skew + K::N <= a.vocab; };
        for (; v + 3 * step < e; v += 4 * step) {
            if (is_whole(v) && is_whole(v + 3 * step)) {
                uint4 u[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) u[q] = __ldg(vec + v + q * step);
#pragma unroll
                for (int q = 0; q < 4; ++q) K::each(u[q], [&](int k, uint32_t h) { f((v + q * step) * K::N - skew + k, h); });
            } else {
#pragma unroll 1
                for (int q = 0; q < 4; ++q) {
                    if (is_whole(v + q * step)) {
                        const uint4 u = __ldg(vec + v + q * step);
                        K::each(u, [&](int k, uint32_t h) { f((v + q * step) * K::N - skew + k, h); });
                    } else part(v + q * step);
                }
            }
        }
        for (; v < e; v += step) {
            if (is_whole(v)) {
                const uint4 u = __ldg(vec + v);
                K::each(u, [&](int k, uint32_t h) { f(v * K::N - skew + k, h); });
            } else part(v);
        }
    }
    template <class F> __device__ void mine(F f) const { elements(v0, v1, tid, kThreads, f); }

    // key of the row's largest, known to every CTA; the barriers of a cluster
    __device__ void find_top() {
        if (tid == 0) sh.top = kNone;
        __syncthreads();
        uint32_t best = kNone;
        mine([&](int, uint32_t h) { best = min(best, K::key(h)); });
        best = __reduce_min_sync(0xffffffffu, best);
        if (lane == 0) atomicMin(&sh.top, best);
        meet();
        top = sh.top;
        for (int r = 0; r < C; ++r) top = min(top, of(r)->top);
        meet();
    }

    // merged count and mass of a bin (or of a part of one); `d`: its first value, `one`: it has no other
    __device__ void merged(bool parts, int b, uint32_t d, bool one, uint32_t &count, unsigned long long &mass) {
        count = 0; mass = 0;
        const int m = parts ? b : K::weighed(b);
        for (int r = 0; r < C; ++r) {
            const Shared<T> *s = of(r);
            count += parts ? s->part_count[b] : s->count[b];
            if (!one) mass += whole(parts ? s->part_mass[b] : s->mass[m]);
        }
        if (one && count) mass = count * weight(d);
    }
    // sums of groups of 32 bins to CTA 0 (groups shared out over warps and CTAs)
    __device__ void sum_steps() {
        Shared<T> *to = of(0);
        for (int s = rank * kWarps + warp; s < K::STEPS; s += C * kWarps) {
            const int b = s * 32 + lane;
            uint32_t count = 0;
            unsigned long long mass = 0;
            if (b < K::BINS) merged(false, b, K::first(b), K::weighed(b) < 0, count, mass);
            count = __reduce_add_sync(0xffffffffu, count);
            if (count) mass = __shfl_sync(0xffffffffu, scan_sum(mass, lane), 31);
            if (lane == 0) { to->step_count[s] = count; to->step_mass[s] = count ? mass : 0; }
        }
    }
    // sums of groups become sums of all groups before; by one warp
    __device__ void run_steps(uint32_t *count, unsigned long long *mass, int n) {
        unsigned long long c_run = 0, m_run = 0;
        for (int s0 = 0; s0 < n; s0 += 32) {
            const int s = s0 + lane;
            const unsigned long long c = s < n ? count[s] : 0, m = s < n ? mass[s] : 0;
            const unsigned long long ci = scan_sum(c, lane), mi = scan_sum(m, lane);
            if (s < n) { count[s] = (uint32_t)(c_run + ci - c); mass[s] = m_run + mi - m; }
            c_run += __shfl_sync(0xffffffffu, ci, 31);
            m_run += __shfl_sync(0xffffffffu, mi, 31);
        }
        if (lane == 0) { count[n] = (uint32_t)c_run; mass[n] = m_run; }
        __syncwarp();
    }
    // By one warp of CTA 0: the bin (or part) in which the running count or mass passes y, or which holds the key y.  p.count_before and
    // p.mass_before: of all before the bins at hand.
    __device__ void search(bool parts, Mode mode, unsigned long long y, int shift, uint32_t base, Place &p, uint32_t &count_at) {
        const uint32_t *sc = parts ? sh.part_step_count : sh.step_count;
        const unsigned long long *sm = parts ? sh.part_step_mass : sh.step_mass;
        const int n = parts ? kParts / 32 : K::STEPS;
        int s = 0;
        if (mode == BY_KEY) s = (parts ? (int)(((uint32_t)y - base) >> shift) : K::bin((uint32_t)y)) >> 5;
        else
            for (int s0 = 0; s0 < n; s0 += 32) {
                const int i = s0 + lane;
                const bool below = i < n && (mode == BY_COUNT ? p.count_before + (unsigned long long)sc[i + 1] <= y : p.mass_before + sm[i + 1] <= y);
                s += __popc(__ballot_sync(0xffffffffu, below));
            }
        s = min(s, n - 1);
        const int b = s * 32 + lane;
        const uint32_t d = parts ? base + ((uint32_t)b << shift) : b < K::BINS ? K::first(b) : kNone;
        uint32_t count = 0;
        unsigned long long mass = 0;
        if (parts || b < K::BINS) merged(parts, b, d, parts ? shift == 0 : K::weighed(b) < 0, count, mass);
        const unsigned long long ci = scan_sum(count, lane), mi = scan_sum(mass, lane);
        const unsigned long long cb = p.count_before + sc[s] + ci - count, mb = p.mass_before + sm[s] + mi - mass;
        unsigned hit;
        if (mode == BY_KEY) hit = 1u << ((parts ? (int)(((uint32_t)y - base) >> shift) : K::bin((uint32_t)y)) & 31);
        else hit = __ballot_sync(0xffffffffu, mode == BY_COUNT ? cb + count > y : mb + mass > y);
        const int l = hit ? __ffs(hit) - 1 : 31;
        p.bin = __shfl_sync(0xffffffffu, b, l);
        p.d = __shfl_sync(0xffffffffu, d, l);
        p.count_before = (uint32_t)__shfl_sync(0xffffffffu, cb, l);
        p.mass_before = __shfl_sync(0xffffffffu, mb, l);
        count_at = __shfl_sync(0xffffffffu, count, l);
    }

    // The place where the running count or mass passes y, or behind the last token with key at most y (BY_KEY).  All CTAs call it
    // alike and learn the answer.
    __device__ Place locate(Mode mode, unsigned long long y) {
        Place p;
        p.count_before = 0; p.mass_before = 0;
        bool parts = false;
        int shift = 0;
        uint32_t base = 0;
        for (;;) {
            if (rank == 0 && warp == 0) {
                uint32_t count_at;
                search(parts, mode, y, shift, base, p, count_at);
                const bool one = parts ? shift == 0 : K::weighed(p.bin) < 0;
                p.w = one ? weight(p.d) : 0;
                p.tie = p.owner = p.owner_tie = 0;
                if (one) {
                    // which of the tokens with this key, and whose it is
                    if (mode == BY_COUNT) p.tie = (uint32_t)(y - p.count_before);
                    else if (mode == BY_MASS) p.tie = p.w ? (uint32_t)min((y - p.mass_before) / p.w, (unsigned long long)count_at - 1) : 0;
                    else p.tie = count_at;                                // (one behind the last of them)
                    const uint32_t c = lane < C ? (parts ? of(lane)->part_count[p.bin] : of(lane)->count[p.bin]) : 0;
                    const uint32_t upto = (uint32_t)scan_sum(c, lane);
                    const unsigned hit = __ballot_sync(0xffffffffu, upto > p.tie);
                    p.owner = hit ? __ffs(hit) - 1 : 0;
                    p.owner_tie = p.tie - __shfl_sync(0xffffffffu, upto - c, p.owner);
                }
                if (lane < C) of(lane)->place = p;
            }
            meet();
            p = sh.place;
            const bool one = parts ? shift == 0 : K::weighed(p.bin) < 0;
            if (one) { meet(); return p; }
            // the bin's parts
            base = p.d;
            shift = parts ? max(0, shift - 10) : max(0, K::BITS - 10);
            parts = true;
            for (int i = tid; i < kParts; i += kThreads) { sh.part_count[i] = 0; sh.part_mass[i] = Sum{0, 0}; }
            __syncthreads();
            const int keep = shift;
            mine([&](int, uint32_t h) {
                const uint32_t d = K::key(h), off = (d - base) >> keep;
                if (d != kNone && d >= base && off < kParts) {
                    atomicAdd(&sh.part_count[off], 1u);
                    if (keep) add_to(&sh.part_mass[off], weight(d));
                }
            });
            meet();
            if (rank == 0) {
                for (int s = warp; s < kParts / 32; s += kWarps) {
                    uint32_t count;
                    unsigned long long mass;
                    merged(true, s * 32 + lane, base + ((uint32_t)(s * 32 + lane) << shift), shift == 0, count, mass);
                    count = __reduce_add_sync(0xffffffffu, count);
                    mass = __shfl_sync(0xffffffffu, scan_sum(mass, lane), 31);
                    if (lane == 0) { sh.part_step_count[s] = count; sh.part_step_mass[s] = mass; }
                }
                __syncthreads();
                if (warp == 0) run_steps(sh.part_step_count, sh.part_step_mass, kParts / 32);
            }
        }
    }

    // the largest key whose share is at least `least` (0 < least <= 1; the share falls as the key rises)
    __device__ uint32_t last_key(double least) const {
        unsigned long long lo = top, hi = sizeof(T) == 2 ? 0xffffu : 0xffffffffu;       // lo qualifies; hi does not (a NaN's place)
        while (hi - lo > 1) {
            const unsigned long long step = (hi - lo + 32) / 33, d = lo + step * (lane + 1);
            const unsigned m = __ballot_sync(0xffffffffu, d < hi && share((uint32_t)d) >= least);
            const int n = __popc(m);                                          // (they are the first ones)
            if (n < 32 && lo + step * (n + 1) < hi) hi = lo + step * (n + 1);
            lo += step * n;
        }
        return (uint32_t)lo;
    }

    // id of the owner_tie-th token with key d among this CTA's; all threads call it
    __device__ void find_token(const Place &p, int32_t *out) {
        const int per = (v1 - v0 + kWarps - 1) / kWarps, b = v0 + warp * per, e = min(v1, b + per);
        uint32_t n = 0;
        elements(b, e, lane, 32, [&](int, uint32_t h) { n += K::key(h) == p.d; });
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) sh.per_warp[warp] = n;
        __syncthreads();
        uint32_t before = 0;
        for (int k = 0; k < warp; ++k) before += sh.per_warp[k];
        if (p.owner_tie < before || p.owner_tie >= before + n) return;
        uint32_t left = p.owner_tie - before;
        // vectors in order, a lane each
        for (int v = b; v < e; v += 32) {
            uint32_t c = 0;
            if (v + lane < e) elements(v + lane, v + lane + 1, 0, 1, [&](int, uint32_t h) { c += K::key(h) == p.d; });
            const uint32_t upto = (uint32_t)scan_sum(c, lane);
            const uint32_t all = __shfl_sync(0xffffffffu, upto, 31);
            if (left < all) {
                if (left >= upto - c && left < upto) {
                    uint32_t k = left - (upto - c);
                    elements(v + lane, v + lane + 1, 0, 1, [&](int i, uint32_t h) { if (K::key(h) == p.d && k-- == 0) *out = i; });
                }
                return;
            }
            left -= all;
        }
    }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_tokens_kernel(const SampleArgs a)
{
    using K = Keys<T>;
    extern __shared__ __align__(16) unsigned char smem[];
    Shared<T> &sh = *reinterpret_cast<Shared<T> *>(smem);
    const int tid = threadIdx.x;
    Sampler<T> s{sh, a, cg::this_cluster()};
    s.C = gridDim.x; s.rank = blockIdx.x;
    s.tid = tid; s.lane = tid & 31; s.warp = tid >> 5;
    const int r = blockIdx.y;
    for (int i = tid; i < K::STEPS * 32; i += kThreads) sh.count[i] = 0;
    for (int i = tid; i < K::WEIGHED; i += kThreads) sh.mass[i] = Sum{0, 0};
    pdl_begin();
    s.row = static_cast<const T *>(a.logits) + r * a.stride;
    s.skew = (int)((reinterpret_cast<uintptr_t>(s.row) & 15) / sizeof(T));
    s.n_vec = (a.vocab + s.skew + K::N - 1) / K::N;
    const int per = (s.n_vec + s.C - 1) / s.C;
    s.v0 = min(s.n_vec, s.rank * per);
    s.v1 = min(s.n_vec, s.v0 + per);
    const float t = a.temperature[r];
    const bool greedy = !(t > 0.f);
    s.inv_t = 1.0 / (greedy ? 1.0 : (double)t);
    s.scale = ldexp(1.0, a.scale_bits);
    const float top_p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
    const int top_k = greedy ? 1 : a.top_k ? a.top_k[r] : 0;
    const double u = fmin(fmax((double)a.u[r], 0.0), 1.0 - 0x1p-24);          // (NaN: 0)
    __syncthreads();

    if constexpr (sizeof(T) == 2) {
        s.mine([&](int, uint32_t h) {
            const int b = K::bin_of(h);
            if (b >= 0) atomicAdd(&sh.count[b], 1u);
        });
        s.meet();
        // the largest: the first bin that is not empty; in the bins of many values (and for their weights) by another look at the elements
        bool many = false;
        for (int k = 0; k < K::WEIGHED; ++k)
            for (int q = 0; q < s.C; ++q) many |= s.of(q)->count[k == 0 ? 0 : k == 1 ? K::FINE + 1 : k == 2 ? K::FINE + 3 : K::BINS - 1] != 0;
        if (many) {
            s.find_top();
        } else {
            if (tid == 0) sh.top = kNone;
            __syncthreads();
            for (int b = tid; b < K::BINS; b += kThreads)
                if (sh.count[b]) { atomicMin(&sh.top, K::first(b)); break; }
            s.meet();
            s.top = sh.top;
            for (int q = 0; q < s.C; ++q) s.top = min(s.top, s.of(q)->top);
        }
        s.x_top = s.top == kNone ? 0.0 : K::value(s.top);
        if (many)
            s.mine([&](int, uint32_t h) {
                const int b = K::bin_of(h), m = b < 0 ? -1 : K::weighed(b);
                if (m >= 0) add_to(&sh.mass[m], s.weight(K::key(h)));
            });
    } else {
        s.find_top();
        s.x_top = s.top == kNone ? 0.0 : K::value(s.top);
        s.mine([&](int, uint32_t h) {
            const uint32_t d = K::key(h);
            if (d == kNone) return;
            const int b = K::bin(d);
            atomicAdd(&sh.count[b], 1u);
            const unsigned long long w = s.weight(d);
            if (w) add_to(&sh.mass[b], w);
        });
    }
    if (s.top == kNone) {
        if (s.rank == 0 && tid == 0) { a.token[r] = 0; if (a.logprob) a.logprob[r] = NAN; }
        s.meet();
        return;
    }
    s.meet();
    s.sum_steps();
    s.meet();
    if (s.rank == 0) {
        if (s.warp == 0) s.run_steps(sh.step_count, sh.step_mass, K::STEPS);
        __syncthreads();
    }
    if (s.C > 1) {
        // (the others need the totals)
        if (s.rank == 0 && s.warp == 0 && s.lane < s.C && s.lane) {
            s.of(s.lane)->step_count[K::STEPS] = sh.step_count[K::STEPS];
            s.of(s.lane)->step_mass[K::STEPS] = sh.step_mass[K::STEPS];
        }
        s.meet();
    }
    const uint32_t tokens = sh.step_count[K::STEPS];
    unsigned long long mass = sh.step_mass[K::STEPS];
    Place cut;
    cut.d = kNone; cut.tie = 0;                       // the last token that is kept: (d, tie)
    bool is_cut = false;
    if (top_k > 0 && (uint32_t)top_k < tokens) {
        cut = s.locate(BY_COUNT, (unsigned long long)top_k - 1);
        mass = cut.mass_before + (cut.tie + 1ull) * cut.w;
        is_cut = true;
    }
    if (top_p < 1.f) {
        const double want = ceil((double)fmaxf(top_p, 0.f) * (double)mass);
        const unsigned long long y = want < 1.0 ? 0 : (unsigned long long)want - 1;
        cut = s.locate(BY_MASS, y);
        mass = cut.mass_before + (cut.tie + 1ull) * cut.w;
        is_cut = true;
    }
    if (min_p > 0.f) {
        if (min_p > 1.f) {
            mass = (unsigned long long)s.scale;       // the first token alone
        } else {
            const uint32_t d = s.last_key((double)min_p);
            if (!is_cut || d < cut.d) {
                const Place q = s.locate(BY_KEY, d);
                mass = q.mass_before + (unsigned long long)q.tie * q.w;
            }
        }
    }
    const Place drawn = s.locate(BY_MASS, (unsigned long long)floor(u * (double)mass));
    if (s.rank == (int)drawn.owner) s.find_token(drawn, a.token + r);
    if (s.rank == 0 && tid == 0 && a.logprob)
        a.logprob[r] = (float)((drawn.d == s.top ? 0.0 : (K::value(drawn.d) - s.x_top) * s.inv_t) - log((double)mass / s.scale));
}

template <typename T>
cudaError_t launch_one(const SampleArgs &a, int rows, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = configure(sample_tokens_kernel<T>, done, (int)sizeof(Shared<T>), true);
    if (e != cudaSuccess) return e;
    // CTAs per row: while they find SMs and have something to count
    int C = 1;
    while (C < 16 && (long long)rows * C * 2 <= 2LL * num_sms() && a.vocab / (C * 2) >= 2048) C *= 2;
    if (C == 16 && clusters_resident(16, 2) < 1) C = 8;
    for (int r0 = 0; r0 < rows; r0 += 65535) {               // (what a grid's second dimension holds)
        const int n = rows - r0 < 65535 ? rows - r0 : 65535;
        SampleArgs b = a;
        b.logits = static_cast<const T *>(a.logits) + r0 * a.stride;
        b.temperature += r0; b.u += r0; b.token += r0;
        if (b.top_k) b.top_k += r0;
        if (b.top_p) b.top_p += r0;
        if (b.min_p) b.min_p += r0;
        if (b.logprob) b.logprob += r0;
        const cudaError_t x = launch_clusters(true, C, sample_tokens_kernel<T>, dim3(C, n), kThreads, sizeof(Shared<T>), st, b);
        if (x != cudaSuccess) return x;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_sample_tokens(const void *logits, int dtype, int rows, int vocab, long long stride, const float *temperature,
                                 const int32_t *top_k, const float *top_p, const float *min_p, const float *u, int32_t *token,
                                 float *logprob, cudaStream_t st)
{
    SampleArgs a;
    a.logits = logits; a.stride = stride; a.vocab = vocab;
    a.scale_bits = 62;
    while ((1ll << (62 - a.scale_bits)) < vocab) --a.scale_bits;       // 2^scale_bits * vocab <= 2^62
    a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.u = u; a.token = token; a.logprob = logprob;
    return dtype == ORTHRUS_FP32 ? launch_one<float>(a, rows, st) : launch_one<__nv_bfloat16>(a, rows, st);
}

}  // namespace orthrus
