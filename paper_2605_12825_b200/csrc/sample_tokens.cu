// One token per row of logits: temperature, top-k, top-p and min-p, then inversion of the running mass with a given uniform.
//
// Every filter cuts the row, ordered by value falling and id rising, at one place; so does the draw.  A place is a value and a count of
// the ties at it, so that no sorting is needed: it is enough to know, for the values in order, how many tokens have them and what they weigh.
//   1. A CTA (few rows: a cluster) counts its row's values in shared memory, one pass over the logits.  bf16 has few values: those with
//      magnitude 2^-24 to 2^8 and zero have a bin each, what is outside shares four.  Weights are then needed once per value and not once per
//      token (an exponential in double precision for a few thousand values instead of 150 thousand tokens).  fp32: bins of 2^16 neighbouring
//      values, magnitudes 2^-8 to 2^8, which carry counts and the sum of their tokens' weights; the maximum is found by a pass before.
//   2. Sums over groups of 32 bins go to one CTA, of which one warp finds the bin of each cut from them, one after the other (all CTAs at each
//      cut, with a barrier between: 18.0 us for 16.3 with one row).
//   3. A cut in a bin of many values needs all CTAs: another pass lists the bin's tokens, which are ranked; if there are too many, it counts and weighs 1024
//      parts of the bin, until a part is one value.
//   4. The wanted occurrence of the drawn value: a pass marks them in a bit map.
// Weights are integers, exp((x - max) / T) in steps of 2^-S with 2^S times the vocabulary at most 2^62: sums do not depend on the
// order in which atomics arrive and are exact; what is off at a border is the weights' own rounding (half a step each, and that of a double: 2^-45
// of the weight where the exponent is largest), and that of the products of u and top_p with a mass, 2^-52 of it.
//
// What bounds it: one row, latency (its steps follow one another at the cluster's barriers); many rows, the atomics in shared memory (one
// a token for bf16, three for fp32 next to an exponential in double): 32 lanes that count in banks of their own take 1.7 clocks of an SM,
// in whatever banks their tokens have 4.0, and 512 rows give some SMs four.  One row of 151936 bf16: 16 us, of which the counts take 2, the sums over
// bins 4, each filter 1, the token 3.4.  512 rows of 128256 bf16: 84 us, of which the counts take 43.  24 rows of
// 32003 fp32 with top-p and min-p: 28 us; 300 of 128256: 274 us, 328 with all filters, most of it the pass that weighs every
// token.  Tokens that are masked out (-inf, or finite and far below) leave the short path with the vector they are in: 512 rows of 128256 bf16 take
// 169 us with 99 % at -inf, 444 with half of them, 693 with 99 % at -1e30, which overflows the list of those and takes another pass; 300 rows of fp32
// 311 and 450.
#include <cooperative_groups.h>
#include <cmath>
#include <cstddef>
#include <type_traits>
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace cg = cooperative_groups;

namespace orthrus {
namespace {

constexpr int kParts = 1024;                       // parts of a bin that a cut falls into, or tokens of one that are listed
constexpr uint32_t kNone = 0xffffffffu;            // no candidate: NaN, -inf

// Values as whole numbers that rise as the value falls (keys); -0 is 0.  Bins of neighbouring ones, by the 16 leading bits: FINE for each
// sign, one for zero, and four wide ones: above, below and (either sign) near zero.
template <typename T> struct Keys {
    static constexpr bool HALF = sizeof(T) == 2;
    static constexpr int N = 16 / sizeof(T);                           // elements of 16 bytes
    static constexpr uint32_t LO = (HALF ? 103u : 119u) << 7, HI = 135u << 7;      // magnitudes 2^-24 or 2^-8, and 2^8
    // Groups of 32 bins in the order of values: above, the positive ones, near zero (positive, zero, negative), the negative ones, below
    static constexpr int FINE = HI - LO, POS = 32, NEAR = POS + FINE, ZERO = NEAR + 1, NEG = NEAR + 32, END = NEG + FINE, STEPS = END / 32 + 1;
    static constexpr int SLOTS = 2 * FINE + 5, WEIGHED = HALF ? 4 : SLOTS;
    static_assert(FINE % 32 == 0, "whole groups");
    static constexpr int LOW = HALF ? 0 : 16;                          // bits behind the leading 16
    static constexpr uint32_t SIGN = HALF ? 0x8000u : 0x80000000u, INF = 0x7f80u << LOW;
    using Raw = std::conditional_t<HALF, uint16_t, uint32_t>;
    __device__ static uint32_t key(uint32_t h) {                       // h: the bits
        const uint32_t mag = h & (SIGN - 1);
        if (mag >= INF && h != INF) return kNone;
        return mag == 0 || !(h & SIGN) ? SIGN - 1 - mag : h;
    }
    __device__ static uint32_t bits(uint32_t d) { return d < SIGN ? SIGN - 1 - d : d; }
    __device__ static double value(uint32_t d) { return (double)__uint_as_float(bits(d) << (16 - LOW)); }
    __device__ static int bin(uint32_t d) {
        if (d == SIGN - 1) return ZERO;
        const bool pos = d < SIGN;
        const uint32_t mag = (pos ? SIGN - 1 - d : d - SIGN) >> LOW;
        if (mag - LO < (uint32_t)FINE) return pos ? POS + (int)(HI - 1 - mag) : NEG + (int)(mag - LO);
        return mag < LO ? (pos ? NEAR : NEAR + 2) : pos ? 0 : END;
    }
    __device__ static bool fine(int b) { return (b >= POS && b < NEAR) || (b >= NEG && b < END); }
    __device__ static bool exists(int b) { return fine(b) || b == 0 || (b >= NEAR && b < NEAR + 3) || b == END; }
    __device__ static bool wide(int b) { return exists(b) && !fine(b) && b != ZERO; }
    __device__ static bool one_value(int b) { return HALF && (fine(b) || b == ZERO); }
    // where the count of a bin that exists is: by magnitude, the positive ones, the negative ones, the other five
    __device__ static int slot(int b) {
        if (b >= POS && b < NEAR) return NEAR - 1 - b;
        if (b >= NEG && b < END) return FINE + (b - NEG);
        return 2 * FINE + (b == 0 ? 0 : b == END ? 4 : b - NEAR + 1);
    }
    __device__ static int weighed(int b) { return HALF ? (b == 0 ? 0 : b == NEAR ? 1 : b == NEAR + 2 ? 2 : 3) : slot(b); }      // its mass
    // the first key behind a bin that exists
    __device__ static uint32_t end(int b) {
        return fine(b) ? first(b) + (1u << LOW) : b == 0 ? first(POS) : b == NEAR ? SIGN - 1 : b == ZERO ? SIGN : b == END ? kNone : first(NEG);
    }
    // log2 of how many keys a bin has at most, and the first
    __device__ static int width(int b) { return wide(b) ? HALF ? 15 : 30 : LOW; }
    __device__ static uint32_t first(int b) {
        const uint32_t more = (1u << LOW) - 1;
        if (b >= POS && b < NEAR) return SIGN - 1 - ((HI - 1 - (b - POS)) << LOW | more);
        if (b >= NEG && b < END) return SIGN + ((LO + (uint32_t)(b - NEG)) << LOW);
        if (b == 0) return 0;
        if (b == NEAR) return SIGN - 1 - (((LO - 1) << LOW) | more);
        if (b == ZERO) return SIGN - 1;
        return b == END ? SIGN + (HI << LOW) : SIGN + 1;
    }
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

// A place in the order: token number `tie` (from 0) of those with key d, which weigh w each; what is before them; its id, where that is known
struct Place { uint32_t d, tie, count_before, count_at, id; int bin; unsigned long long mass_before, w; };

enum Mode { BY_COUNT, BY_MASS, BY_KEY };
// What CTA 0 tells the others: a cut that needs all of them, or the drawn token (stage 4)
struct Order { Place at; unsigned long long y, mass; uint32_t cut; int stage; Mode mode; };

constexpr int kPartSteps = kParts / 32;
template <typename T> struct Shared {
    uint32_t count[Keys<T>::SLOTS + 3];                  // of a bin at its slot (in the end: the bit map)
    Sum mass[Keys<T>::WEIGHED];
    union {
        struct { uint32_t count[kParts]; Sum mass[kParts]; } part;
        struct { uint32_t key[kParts], id[kParts]; unsigned long long w[kParts]; } list;
        uint32_t wide_bits[4 * kParts];                  // first pass over bf16: bits of tokens in the wide bins
    };
    // CTA 0: sums of the groups of 32 bins, then of all before; behind them those of the parts
    unsigned long long step_mass[Keys<T>::STEPS + 1 + kPartSteps + 1];
    uint32_t step_count[Keys<T>::STEPS + 1 + kPartSteps + 1];
    Place place[2];
    Order order;
    uint32_t top, found, per_warp[32];
    // CTA 0 of several: what all of them have counted (a launch of single CTAs leaves out the room for these)
    uint32_t all_count[Keys<T>::STEPS * 32];
    Sum all_mass[Keys<T>::WEIGHED];
};


__device__ inline uint32_t scan_sum(uint32_t x, int lane) {
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    return x;
}
__device__ inline unsigned long long scan_sum(unsigned long long x, int lane) {
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    return x;
}

// sum over a warp, of numbers below 2^63 whose sum is
__device__ inline unsigned long long warp_total(unsigned long long x) {
    const unsigned long long lo = __reduce_add_sync(0xffffffffu, (uint32_t)x & 0xffffff), mid = __reduce_add_sync(0xffffffffu, (uint32_t)(x >> 24) & 0xffffff),
                             hi = __reduce_add_sync(0xffffffffu, (uint32_t)(x >> 48));
    return lo + (mid << 24) + (hi << 48);
}

// kAlone: one CTA a row
template <typename T, int kThreads, bool kAlone>
struct Sampler {
    using K = Keys<T>;
    static constexpr int kWarps = kThreads / 32;
    Shared<T> &sh;
    const SampleArgs &a;
    cg::cluster_group cluster;
    const T *row;
    int tid, lane, warp, C, rank;
    int e0, e1;                            // this CTA's elements
    uint32_t top;                          // key of the largest
    double x_top, inv_t, scale;
    int turn;                              // which of the two places is next (one is written while the other may still be read)

    __device__ void meet() { if (!kAlone) cluster.sync(); else __syncthreads(); }
    __device__ Shared<T> *of(int r) { return !kAlone ? cluster.map_shared_rank(&sh, r) : &sh; }
    // exp((x - max) / T) of a value x that is not the largest.  (NaN, of infinities that cancel: 0)
    __device__ double share_of(double x) const { return exp(fmax((x - x_top) * inv_t, -800.0)); }
    __device__ double share(uint32_t d) const {
        return d == top ? 1.0 : share_of(K::value(d));
    }
    __device__ unsigned long long weight(uint32_t d) const { return __double2ull_rn(share(d) * scale); }

    // f(element, 16 bytes) for the whole vectors among elements [b, e), U loads of a thread under way together; g(element, bits) for the
    // elements in front of and behind them
    template <int U, bool BACK = false, class F, class G> __device__ void vectors(int b, int e, F f, G g) const {
        const int skew = (int)((reinterpret_cast<uintptr_t>(row + b) & 15) / sizeof(T)), head = min((K::N - skew) % K::N, e - b);
        const int n = (e - b - head) / K::N, tail = b + head + n * K::N;
        const uint4 *x = reinterpret_cast<const uint4 *>(row + b + head);
#pragma unroll 1
        for (int v = tid; v < n; v += U * kThreads) {
            uint4 u[U];
#pragma unroll
            for (int q = 0; q < U; ++q) { const int i = min(v + q * kThreads, n - 1); u[q] = __ldcg(x + (BACK ? n - 1 - i : i)); }
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const int i = v + q * kThreads;
                if (i < n) f(b + head + (BACK ? n - 1 - i : i) * K::N, u[q]);
            }
        }
        // (at most N - 1 each, fewer than the threads)
        const int i = tid < head ? b + tid : tid - head < e - tail ? tail + tid - head : -1;
        if (i >= 0) g(i, (uint32_t)reinterpret_cast<const typename K::Raw *>(row)[i]);
    }
    // f(element, bits) for this CTA's elements.  In little code: for what is not done for every row
    template <class F> __device__ void mine(F f) const {
        vectors<4>(e0, e1,
                [&](int i0, uint4 u) {
#pragma unroll 1
                    for (int k = 0; k < K::N; ++k) {
                        f(i0 + k, K::HALF ? u.x & 0xffff : u.x);
                        if (K::HALF) { u.x = __funnelshift_r(u.x, u.y, 16); u.y = __funnelshift_r(u.y, u.z, 16); u.z = __funnelshift_r(u.z, u.w, 16); u.w >>= 16; }
                        else { u.x = u.y; u.y = u.z; u.z = u.w; }
                    }
                },
                f);
    }

    // key of the row's largest, from every CTA's (sh.top, before a barrier)
    __device__ uint32_t top_of_all() {
        const uint32_t x = lane < C ? of(lane)->top : kNone;
        return __reduce_min_sync(0xffffffffu, x);
    }
    __device__ void find_top() {
        float high = -INFINITY;                            // (NaN is passed over)
        vectors<4>(e0, e1,
                [&](int, const uint4 &u) {
                    high = fmaxf(high, fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w))));
                },
                [&](int, uint32_t h) { high = fmaxf(high, __uint_as_float(h)); });
        uint32_t best = K::key(__float_as_uint(high));
        best = __reduce_min_sync(0xffffffffu, best);
        if (lane == 0) atomicMin(&sh.top, best);
    }

    // what is in bin b, of parts if `parts`, by its first value d (`one`: it has no other)
    __device__ void in_bin(bool parts, int b, uint32_t d, bool one, uint32_t &count, unsigned long long &mass) {
        count = parts ? sh.part.count[b] : !kAlone ? sh.all_count[b] : sh.count[K::slot(b)];
        mass = 0;
        if (one) { if (count) mass = count * weight(d); }
        else mass = whole(parts ? sh.part.mass[b] : !kAlone ? sh.all_mass[K::weighed(b)] : sh.mass[K::weighed(b)]);
    }
    // Sums of groups of 32 bins to CTA 0.  One CTA a row: a thread a group, which it walks from a place of its lane's on, in another bank than
    // the other lanes (a warp a group, summed by reductions, takes twice as long with four rows on an SM).
    __device__ void sum_steps_alone() {
#pragma unroll 1
        for (int s = tid; s < K::STEPS; s += kThreads) {
            const bool pos = s >= K::POS / 32 && s < K::NEAR / 32, neg = s >= K::NEG / 32 && s < K::END / 32;
            uint32_t n = 0;
            unsigned long long m = 0;
            if (pos || neg) {
                const int at0 = pos ? K::NEAR - 32 - s * 32 : K::FINE + (s * 32 - K::NEG);           // its slots, which follow one another
                constexpr int J = 4;                       // bins under way together
#pragma unroll 1
                for (int j0 = 0; j0 < 32; j0 += J) {
                    uint32_t count[J], any = 0;
#pragma unroll
                    for (int j = 0; j < J; ++j) { count[j] = sh.count[at0 + ((j0 + j + lane) & 31)]; any |= count[j]; }
                    if (any == 0) continue;
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        const int at = at0 + ((j0 + j + lane) & 31);
                        n += count[j];
                        if constexpr (K::HALF) {
                            const uint32_t h = pos ? K::LO + at : 0x8000u + K::LO + (at - K::FINE);
                            m += count[j] * __double2ull_rn((K::bits(top) == h ? 1.0 : share_of((double)__uint_as_float(h << 16))) * scale);
                        } else {
                            m += whole(sh.mass[at]);
                        }
                    }
                }
            } else {
#pragma unroll 1
                for (int b = s * 32; b < s * 32 + 3; ++b) {
                    uint32_t count = 0;
                    unsigned long long mass = 0;
                    if (K::exists(b)) in_bin(false, b, K::first(b), K::one_value(b), count, mass);
                    n += count;
                    m += mass;
                }
            }
            sh.step_count[s] = n;
            sh.step_mass[s] = m;
        }
    }
    // Several CTAs: a warp a group, groups shared out over all warps; the bins themselves go to CTA 0 too
    __device__ void sum_steps() {
        Shared<T> *to = of(0);
#pragma unroll 1
        for (int s = rank * kWarps + warp; s < K::STEPS; s += C * kWarps) {
            const int b = s * 32 + lane;
            // slot, and, of a fine bin of bf16, the value; groups are of one kind
            const bool pos = s >= K::POS / 32 && s < K::NEAR / 32, neg = s >= K::NEG / 32 && s < K::END / 32, is = pos || neg || K::exists(b);
            const int at = pos ? K::NEAR - 1 - b : neg ? K::FINE + (b - K::NEG) : is ? K::slot(b) : 0;
            const bool one = is && (pos || neg ? K::HALF : K::one_value(b)), wide = is && !one;
            uint32_t count = 0;
            unsigned long long mass = 0;
            const Sum *m = sh.mass + (wide ? K::weighed(b) : 0);
            uint32_t x[8];
            Sum y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {                  // (at most eight CTAs)
                x[i] = is && i < C ? *cluster.map_shared_rank(sh.count + at, i) : 0;
                y[i] = wide && i < C ? *cluster.map_shared_rank(m, i) : Sum{0, 0};
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) { count += x[i]; mass += whole(y[i]); }
            to->all_count[b] = count;
            if (wide) to->all_mass[K::weighed(b)] = Sum{(uint32_t)mass, (uint32_t)(mass >> 32)};
            uint32_t n = 0;
            if (__any_sync(0xffffffffu, count)) {
                if (one) {
                    const uint32_t h = pos ? K::LO + at : neg ? 0x8000u + K::LO + (at - K::FINE) : K::bits(K::first(b));
                    mass = count * __double2ull_rn((K::bits(top) == h ? 1.0 : share_of((double)__uint_as_float(h << 16))) * scale);
                }
                n = __reduce_add_sync(0xffffffffu, count);
                mass = warp_total(mass);
            }
            if (lane == 0) { to->step_count[s] = n; to->step_mass[s] = mass; }
        }
    }
    // the same for the parts, all of which are CTA 0's
    __device__ void sum_parts(uint32_t base, int shift) {
#pragma unroll 1
        for (int s = warp; s < kPartSteps; s += kWarps) {
            uint32_t count;
            unsigned long long mass;
            in_bin(true, s * 32 + lane, base + ((uint32_t)(s * 32 + lane) << shift), shift == 0, count, mass);
            count = __reduce_add_sync(0xffffffffu, count);
            mass = warp_total(mass);
            if (lane == 0) { sh.step_count[K::STEPS + 1 + s] = count; sh.step_mass[K::STEPS + 1 + s] = mass; }
        }
    }
    // sums of groups become sums of all groups before, in place, the total behind them; by one warp of CTA 0
    __device__ void run_steps(bool parts) {
        const int n = parts ? kPartSteps : K::STEPS;
        uint32_t *count = sh.step_count + (parts ? K::STEPS + 1 : 0);
        unsigned long long *mass = sh.step_mass + (parts ? K::STEPS + 1 : 0);
        const int per = (n + 31) / 32, b = min(n, lane * per), e = min(n, b + per);
        uint32_t c = 0;
        unsigned long long m = 0;
        for (int s = b; s < e; ++s) { c += count[s]; m += mass[s]; }
        uint32_t cr = scan_sum(c, lane) - c;
        unsigned long long mr = scan_sum(m, lane) - m;
        for (int s = b; s < e; ++s) {
            const uint32_t x = count[s];
            const unsigned long long y = mass[s];
            count[s] = cr; mass[s] = mr;
            cr += x; mr += y;
        }
        if (lane == 31) { count[n] = cr; mass[n] = mr; }
        __syncwarp();
    }
    // By one warp of CTA 0: the bin (or part) in which the running count or mass passes y, or which holds the key y.  p.count_before and
    // p.mass_before: of all before the bins at hand.
    __device__ void search(bool parts, Mode mode, unsigned long long y, int shift, uint32_t base, Place &p) {
        const uint32_t *sc = sh.step_count + (parts ? K::STEPS + 1 : 0);
        const unsigned long long *sm = sh.step_mass + (parts ? K::STEPS + 1 : 0);
        const int n = parts ? kPartSteps : K::STEPS;
        const int by_key = parts ? (int)(((uint32_t)y - base) >> shift) : K::bin((uint32_t)y);       // (of BY_KEY)
        int s = by_key >> 5;
        if (mode != BY_KEY) {
            uint32_t below = 0;
#pragma unroll 4
            for (int i = lane; i < n; i += 32)
                below += mode == BY_COUNT ? p.count_before + (unsigned long long)sc[i + 1] <= y : p.mass_before + sm[i + 1] <= y;
            s = min((int)__reduce_add_sync(0xffffffffu, below), n - 1);
        }
        const int b = s * 32 + lane;
        const bool is = parts || K::exists(b);
        const uint32_t d = parts ? base + ((uint32_t)b << shift) : is ? K::first(b) : kNone;
        uint32_t count = 0;
        unsigned long long mass = 0;
        if (is) in_bin(parts, b, d, parts ? shift == 0 : K::one_value(b), count, mass);
        const uint32_t cb = p.count_before + sc[s] + scan_sum(count, lane) - count;
        const unsigned long long mb = p.mass_before + sm[s] + scan_sum(mass, lane) - mass;
        const unsigned hit = mode == BY_KEY ? 1u << (by_key & 31)
                                            : __ballot_sync(0xffffffffu, mode == BY_COUNT ? (unsigned long long)cb + count > y : mb + mass > y);
        const int l = hit ? __ffs(hit) - 1 : 31;
        p.bin = __shfl_sync(0xffffffffu, b, l);
        p.d = __shfl_sync(0xffffffffu, d, l);
        p.count_before = __shfl_sync(0xffffffffu, cb, l);
        p.mass_before = __shfl_sync(0xffffffffu, mb, l);
        p.count_at = __shfl_sync(0xffffffffu, count, l);
    }

    // By one warp of CTA 0: which of the tokens with key p.d, of a bin or part that has no other
    __device__ void settle(Mode mode, unsigned long long y, Place &p) const {
        p.w = weight(p.d);
        p.id = kNone;
        p.tie = mode == BY_COUNT ? (uint32_t)(y - p.count_before)
              : mode == BY_KEY ? p.count_at                              // (one behind the last of them)
              : p.w ? (uint32_t)min((y - p.mass_before) / p.w, (unsigned long long)p.count_at - 1) : 0;
    }
    // The place where the running count or mass passes y, or behind the last token with key at most y (BY_KEY), of which bin p.bin is known, which
    // has many values.  All CTAs call it alike and learn the answer.
    __device__ Place refine(Mode mode, unsigned long long y, Place p) {
        if (p.count_at <= kParts) return ranked(mode, y, p);
        int shift = K::width(p.bin);
#pragma unroll 1
        for (;;) {
            // the bin's parts
            const uint32_t base = p.d;
            shift = max(0, shift - 10);
            for (int i = tid; i < kParts; i += kThreads) { sh.part.count[i] = 0; sh.part.mass[i] = Sum{0, 0}; }
            __syncthreads();
            mine([&](int, uint32_t h) {
                const uint32_t d = K::key(h), off = (d - base) >> shift;
                if (d != kNone && d >= base && off < kParts) {
                    atomicAdd(&sh.part.count[off], 1u);
                    if (shift) add_to(&sh.part.mass[off], weight(d));
                }
            });
            if (!kAlone) {
                // to those of CTA 0 (few are not empty: the bin was one of thousands)
                meet();
                if (rank)
                    for (int i = tid; i < kParts; i += kThreads)
                        if (const uint32_t n = sh.part.count[i]) {
                            Shared<T> *to = of(0);
                            atomicAdd(&to->part.count[i], n);
                            const unsigned long long m = whole(sh.part.mass[i]);
                            if (m) add_to(&to->part.mass[i], m);
                        }
            }
            meet();
            if (rank == 0) { sum_parts(base, shift); __syncthreads(); }
            if (rank == 0 && warp == 0) {
                run_steps(true);
                search(true, mode, y, shift, base, p);
                if (shift == 0) settle(mode, y, p);
                if (lane < C) of(lane)->place[turn] = p;
            }
            meet();
            p = sh.place[turn];
            turn ^= 1;
            if (shift == 0) return p;
        }
    }
    // The same among the tokens of bin p.bin, of which there are few: every CTA lists its own, CTA 0 takes them all
    __device__ Place ranked(Mode mode, unsigned long long y, const Place &p) {
        const uint32_t size = K::end(p.bin) - p.d, like = K::bits(p.d);
        auto list = [&](int i, uint32_t h) {
            const uint32_t d = K::key(h);
            if (d - p.d >= size) return;
            const uint32_t at = atomicAdd(&sh.found, 1u);
            if (at < kParts) { sh.list.key[at] = d; sh.list.id[at] = (uint32_t)i; }          // (it is: they have been counted)
        };
        if (!K::HALF && K::fine(p.bin))                    // (the bits' leading half says it)
            vectors<4>(e0, e1,
                    [&](int i0, const uint4 &u) {
                        const uint32_t x = u.x ^ like, y = u.y ^ like, z = u.z ^ like, w = u.w ^ like;
                        if (min(min(x, y), min(z, w)) >> 16) return;
                        uint32_t m = (x >> 16 == 0) | (y >> 16 == 0) << 1 | (z >> 16 == 0) << 2 | (w >> 16 == 0) << 3;
#pragma unroll 1
                        for (; m; m &= m - 1) {
                            const int k = __ffs(m) - 1;
                            list(i0 + k, k == 0 ? u.x : k == 1 ? u.y : k == 2 ? u.z : u.w);
                        }
                    },
                    list);
        else mine(list);
        meet();
        if (rank == 0) {
            uint32_t n = min(sh.found, (uint32_t)kParts), own = n;
            if (!kAlone) {
                const uint32_t upto = scan_sum(lane < C ? of(lane)->found : 0, lane);
                n = min(__shfl_sync(0xffffffffu, upto, 31), (uint32_t)kParts);
                uint32_t end[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) end[i] = __shfl_sync(0xffffffffu, upto, i);      // (at most eight CTAs)
                for (uint32_t j = own + tid; j < n; j += kThreads) {
                    int r = 0;
                    uint32_t before = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) if (j >= end[i]) { r = i + 1; before = end[i]; }
                    const Shared<T> *from = of(r);
                    sh.list.key[j] = from->list.key[j - before];
                    sh.list.id[j] = from->list.id[j - before];
                }
                __syncthreads();
            }
            for (uint32_t j = tid; j < n; j += kThreads) sh.list.w[j] = weight(sh.list.key[j]);
            __syncthreads();
            // (up to n: BY_KEY asks for a place behind a key that may have no token)
            for (uint32_t j = tid; j < n + (mode == BY_KEY); j += kThreads) {
                if (mode == BY_KEY && j < n) continue;
                const uint32_t d = j < n ? sh.list.key[j] : (uint32_t)y, id = j < n ? sh.list.id[j] : kNone;
                uint32_t before = 0, tie = 0;
                unsigned long long mass = 0;
#pragma unroll 4
                for (uint32_t k = 0; k < n; ++k) {
                    const uint32_t x = sh.list.key[k];
                    const bool lower = x < d, same = x == d && sh.list.id[k] < id;
                    before += lower;
                    tie += same;
                    if (lower) mass += sh.list.w[k];
                }
                Place q = p;
                q.d = d; q.tie = tie; q.id = id;
                q.w = j < n ? sh.list.w[j] : weight(d);
                q.count_before += before;
                q.mass_before += mass;
                const unsigned long long c = (unsigned long long)q.count_before + tie, m = q.mass_before + tie * q.w;
                if (mode == BY_COUNT ? c == y : mode == BY_MASS ? m <= y && y < m + q.w : true)
                    for (int r = 0; r < C; ++r) of(r)->place[turn] = q;
            }
        }
        meet();
        const Place q = sh.place[turn];
        turn ^= 1;
        return q;
    }

    // the largest key whose share is at least `least` (0 < least <= 1; the share falls as the key rises)
    __device__ uint32_t last_key(double least) const {
        unsigned long long lo = top, hi = sizeof(T) == 2 ? 0xffffu : 0xffffffffu;       // lo qualifies; hi does not (a NaN's place)
        {
            // it is almost always among the 32 keys around max + T ln(least)
            const float x = (float)(x_top + (double)logf((float)least) / inv_t);
            const unsigned long long g = K::key(__float_as_uint(x) >> (16 - K::LOW)), d0 = g > lo + 16 && g < hi ? g - 16 : lo, d = d0 + lane;
            const int n = __popc(__ballot_sync(0xffffffffu, d < hi && share((uint32_t)d) >= least));
            if (n > 0 && n < 32) return (uint32_t)d0 + n - 1;
        }
#pragma unroll 1
        while (hi - lo > 1) {
            const unsigned long long step = (hi - lo + 32) / 33, d = lo + step * (lane + 1);
            const unsigned m = __ballot_sync(0xffffffffu, d < hi && share((uint32_t)d) >= least);
            const int n = __popc(m);                                          // (they are the first ones)
            if (n < 32 && lo + step * (n + 1) < hi) hi = lo + step * (n + 1);
            lo += step * n;
        }
        return (uint32_t)lo;
    }

    // Id of the tie-th token with key d, by the CTA that has it: a bit map of them, a stretch of elements at a time
    __device__ void find_token(const Place &p, int32_t *out) {
        // a stretch per CTA at a time (so that half of a row is read on average); the bits are where the counts were
        const int room = min(32768, ((a.vocab + C - 1) / C + 31) & ~31);
        static_assert(32768 <= K::SLOTS * 32, "bit map");
        // (both zeros are one key)
        const uint32_t bits = K::bits(p.d) * (K::HALF ? 0x10001u : 1u), mask = K::bits(p.d) ? 0xffffffffu : (K::SIGN - 1) * (K::HALF ? 0x10001u : 1u);
        uint32_t before = 0;                               // those of earlier stretches
#pragma unroll 1
        for (int b = rank; ; b += C) {                     // (every CTA as often: they tell one another how many there are)
            const int lo = (int)min((long long)a.vocab, (long long)b * room), hi = min(a.vocab, lo + room);
            __syncthreads();
            for (int i = tid; i < room / 32; i += kThreads) sh.count[i] = 0;
            __syncthreads();
            auto put = [&](int i) { atomicOr(&sh.count[(i - lo) >> 5], 1u << ((i - lo) & 31)); };
            vectors<4>(lo, hi,
                    [&](int i0, const uint4 &u) {
                        uint32_t w[4] = {(u.x ^ bits) & mask, (u.y ^ bits) & mask, (u.z ^ bits) & mask, (u.w ^ bits) & mask};
                        if constexpr (K::HALF) {
                            uint32_t eq = 0;               // (a bit an element)
#pragma unroll
                            for (int q = 0; q < 4; ++q) { const uint32_t e = __vseteq2(w[q], 0); eq |= ((e | e >> 15) & 3) << (2 * q); }
                            while (eq) { put(i0 + __ffs(eq) - 1); eq &= eq - 1; }
                        } else {
#pragma unroll
                            for (int q = 0; q < 4; ++q) if (w[q] == 0) put(i0 + q);
                        }
                    },
                    [&](int i, uint32_t h) { if (K::key(h) == p.d) put(i); });
            __syncthreads();
            // how many: of a thread's words, of the threads in front of it, of the CTAs in front of this one
            const int words = (hi - lo + 31) / 32, per = (words + kThreads - 1) / kThreads, w0 = min(words, tid * per), w1 = min(words, w0 + per);
            uint32_t n = 0;
            for (int i = w0; i < w1; ++i) n += __popc(sh.count[i]);
            const uint32_t upto = scan_sum(n, lane);
            if (lane == 31) sh.per_warp[warp] = upto;
            __syncthreads();
            uint32_t mine = 0, all = 0;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) { if (k < warp) mine += sh.per_warp[k]; all += sh.per_warp[k]; }
            if (!kAlone) {
                if (tid == 0) sh.found = all;
                meet();
                const uint32_t others = lane < C ? of(lane)->found : 0, sum = scan_sum(others, lane);
                mine += __shfl_sync(0xffffffffu, sum - others, rank);
                all = __shfl_sync(0xffffffffu, sum, 31);
                meet();
            }
            uint32_t left = p.tie - before - mine - (upto - n);        // (huge, if it is in front)
            if (p.tie >= before && left < n)
                for (int i = w0; ; ++i) {
                    const uint32_t w = sh.count[i], c = __popc(w);
                    if (left < c) { *out = lo + i * 32 + (int)__fns(w, 0, (int)left + 1); break; }
                    left -= c;
                }
            before += all;
            if (p.tie < before || (long long)(b - rank + C) * room >= a.vocab) return;
        }
    }
};

template <typename T, int kThreads, bool kAlone>
__global__ void __launch_bounds__(kThreads, kThreads > 256 ? 1 : Keys<T>::HALF ? 4 : 3) sample_tokens_kernel(const SampleArgs a)
{
    using K = Keys<T>;
    extern __shared__ __align__(16) unsigned char smem[];
    Shared<T> &sh = *reinterpret_cast<Shared<T> *>(smem);
    const int tid = threadIdx.x;
    Sampler<T, kThreads, kAlone> s{sh, a, cg::this_cluster()};
    s.C = gridDim.x; s.rank = blockIdx.x; s.turn = 0;
    s.tid = tid; s.lane = tid & 31; s.warp = tid >> 5;
    const int r = blockIdx.y;
    for (int i = tid; i < K::SLOTS; i += kThreads) sh.count[i] = 0;
    for (int i = tid; i < K::WEIGHED; i += kThreads) sh.mass[i] = Sum{0, 0};
    if (tid == 0) sh.top = kNone;
    pdl_begin();
    s.row = static_cast<const T *>(a.logits) + r * a.stride;
    const int per = (a.vocab + s.C - 1) / s.C;
    s.e0 = min(a.vocab, s.rank * per);
    s.e1 = min(a.vocab, s.e0 + per);
    const float t = a.temperature[r];
    const bool greedy = !(t > 0.f);
    s.inv_t = 1.0 / (greedy ? 1.0 : (double)t);
    s.scale = ldexp(1.0, a.scale_bits);
    const float top_p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
    const int top_k = greedy ? 1 : a.top_k ? a.top_k[r] : 0;
    const double u = fmin(fmax((double)a.u[r], 0.0), 1.0 - 0x1p-24);          // (NaN: 0)
    __syncthreads();

    bool wait = true;                                 // there are counts or sums that other CTAs may still be at
    auto weigh = [&] { s.x_top = s.top == kNone ? 0.0 : K::value(s.top); };
    if constexpr (K::HALF) {
        if (tid == 0) sh.found = 0;
        __syncthreads();
        // zero, and what has no bin of its own (whose weights are needed one by one: a list of them); hardly ever
        __nv_bfloat162 high = __halves2bfloat162(__ushort_as_bfloat16(0xff80), __ushort_as_bfloat16(0xff80));     // (NaN is passed over)
        uint32_t best = kNone;
        auto rare = [&](uint32_t h) {
            const uint32_t d = K::key(h);
            if (d == kNone) return;
            best = min(best, d);
            const int b = K::bin(d);
            atomicAdd(&sh.count[K::slot(b)], 1u);
            if (b == K::ZERO || K::one_value(b)) return;
            const uint32_t at = atomicAdd(&sh.found, 1u);
            if (at < 4 * kParts) sh.wide_bits[at] = h;
        };
        // Two elements less LO each, both with bins of their own: a magnitude of 12 bits and the sign on top.  The slot is the magnitude's, FINE
        // further on for a negative one, so the sign moves down to bit 12.  (What a token costs here is instructions.)
        static_assert(K::FINE == 0x1000, "12 bits");
        auto add = [&](uint32_t t) {
            const uint32_t v = (t & 0x0fff0fff) | (t >> 3 & ~0x0fff0fffu);        // (bits 13 to 15 of the lower one are not its own)
            atomicAdd(reinterpret_cast<uint32_t *>(reinterpret_cast<char *>(sh.count) + (v << 2 & 0x7ffc)), 1u);
            atomicAdd(reinterpret_cast<uint32_t *>(reinterpret_cast<char *>(sh.count) + (v >> 14 & ~3u)), 1u);
        };
        // (from the row's end: its beginning, where the drawn token is looked for first, is then what L2 has of it; 88.8 us for 86.9)
        s.template vectors<4, true>(s.e0, s.e1,
                  [&](int i0, const uint4 &u) {
                      // a magnitude below LO or from HI on leaves one of the bits 12 to 14 (a borrow from the upper element does not hide the
                      // lower one's)
                      constexpr uint32_t LO2 = K::LO * 0x10001u;
                      const uint32_t x = u.x - LO2, y = u.y - LO2, z = u.z - LO2, w = u.w - LO2;
                      auto pair = [](uint32_t v) { return *reinterpret_cast<__nv_bfloat162 *>(&v); };
                      high = __hmax2(high, __hmax2(__hmax2(pair(u.x), pair(u.y)), __hmax2(pair(u.z), pair(u.w))));
                      if (((x | y | z | w) & 0x70007000) == 0) {
                          add(x); add(y); add(z); add(w);
                      } else {
#pragma unroll 1
                          for (int k = 0; k < K::N; ++k) rare((uint32_t)reinterpret_cast<const uint16_t *>(s.row)[i0 + k]);
                      }
                  },
                  [&](int, uint32_t h) { rare(h); });
        best = min(best, min(K::key(__bfloat16_as_ushort(high.x)), K::key(__bfloat16_as_ushort(high.y))));
        best = __reduce_min_sync(0xffffffffu, best);
        if (s.lane == 0) atomicMin(&sh.top, best);
        s.meet();
        s.top = s.top_of_all();
        weigh();
        const uint32_t listed = sh.found;
        auto weigh_one = [&](uint32_t h) {
            const uint32_t d = K::key(h);
            if (d != kNone && K::wide(K::bin(d))) add_to(&sh.mass[K::weighed(K::bin(d))], s.weight(d));
        };
        if (!kAlone) wait = __any_sync(0xffffffffu, s.lane < s.C && s.of(s.lane)->found);
        if (listed <= 4 * kParts) for (uint32_t j = tid; j < listed; j += kThreads) weigh_one(sh.wide_bits[j]);
        else s.mine([&](int, uint32_t h) { weigh_one(h); });
    } else {
        s.find_top();
        s.meet();
        s.top = s.top_of_all();
        weigh();
        const auto one = [&](uint32_t h) {
            const uint32_t d = K::key(h);
            if (d == kNone) return;
            const int b = K::bin(d);
            atomicAdd(&sh.count[K::slot(b)], 1u);
            const unsigned long long w = s.weight(d);
            if (w) add_to(&sh.mass[K::weighed(b)], w);
        };
        // four tokens that are not far from zero, whose exponentials and atomics are under way together (what a token costs here is instructions)
        const auto four = [&](const uint4 &u) {
            const uint32_t h[4] = {u.x, u.y, u.z, u.w};
            uint32_t at[4], far = 0, lo[4], old[4], hi[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t mag = h[j] & 0x7fffffff, lead = mag >> 16;
                const bool neg = h[j] >> 31;
                far |= lead >= K::HI;
                // (below LO the slots of the bins near zero)
                at[j] = lead >= K::LO ? lead - K::LO + (neg ? K::FINE : 0) : 2 * K::FINE + (mag == 0 ? 2 : neg ? 3 : 1);
            }
            if (far) {
#pragma unroll 1
                for (int j = 0; j < 4; ++j) one(j == 0 ? u.x : j == 1 ? u.y : j == 2 ? u.z : u.w);
                return;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) atomicAdd(&sh.count[at[j]], 1u);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned long long w = __double2ull_rn(s.share_of((double)__uint_as_float(h[j])) * s.scale);
                lo[j] = (uint32_t)w;
                hi[j] = (uint32_t)(w >> 32);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) old[j] = lo[j] ? atomicAdd(&sh.mass[at[j]].lo, lo[j]) : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (const uint32_t x = hi[j] + (old[j] + lo[j] < old[j])) atomicAdd(&sh.mass[at[j]].hi, x);
        };
        s.template vectors<2>(s.e0, s.e1, [&](int, const uint4 &u) { four(u); }, [&](int, uint32_t h) { one(h); });
    }
    if (s.top == kNone) {
        if (s.rank == 0 && tid == 0) { a.token[r] = 0; if (a.logprob) a.logprob[r] = NAN; }
        s.meet();
        return;
    }
    if (wait) s.meet();
    if constexpr (kAlone) s.sum_steps_alone(); else s.sum_steps();
    s.meet();
    // Top-k, top-p, min-p, the draw.  One warp makes them one after the other as long as they fall into bins of one value.
    const bool lead = s.rank == 0 && s.warp == 0;
    Place at;                                         // the last token that is kept, then the drawn one
    uint32_t tokens = 0, cut = kNone;                 // key of the former
    unsigned long long mass = 0, y = 0;
    int stage = 0;
    Mode mode = BY_MASS;
    if (lead) {
        s.run_steps(false);
        tokens = sh.step_count[K::STEPS];
        mass = sh.step_mass[K::STEPS];
    }
    auto keep = [&] {
        mass = at.mass_before + ((unsigned long long)at.tie + (mode == BY_KEY ? 0 : 1)) * at.w;
        cut = at.d;
    };
#pragma unroll 1
    for (;;) {
        if (lead) {
#pragma unroll 1
            for (; stage < 4; ++stage) {
                mode = BY_MASS;
                if (stage == 0) {
                    if (top_k <= 0 || (uint32_t)top_k >= tokens) continue;
                    mode = BY_COUNT;
                    y = (unsigned long long)top_k - 1;
                } else if (stage == 1) {
                    if (!(top_p < 1.f)) continue;
                    const double want = ceil((double)fmaxf(top_p, 0.f) * (double)mass);
                    y = want < 1.0 ? 0 : (unsigned long long)want - 1;
                } else if (stage == 2) {
                    if (!(min_p > 0.f)) continue;
                    if (min_p > 1.f) { mass = (unsigned long long)s.scale; continue; }        // the first token alone
                    const uint32_t d = s.last_key((double)min_p);
                    if (d >= cut) continue;
                    mode = BY_KEY;
                    y = d;
                } else {
                    y = (unsigned long long)floor(u * (double)mass);
                }
                at.count_before = 0;
                at.mass_before = 0;
                s.search(false, mode, y, 0, 0, at);
                if (!K::one_value(at.bin)) break;
                s.settle(mode, y, at);
                if (stage < 3) keep();
            }
            if (s.lane < s.C) s.of(s.lane)->order = Order{at, y, mass, cut, stage, mode};
        }
        if (tid == 0) sh.found = 0;
        s.meet();
        at = sh.order.at; y = sh.order.y; mass = sh.order.mass; cut = sh.order.cut; stage = sh.order.stage; mode = sh.order.mode;
        if (stage == 4) break;
        at = s.refine(mode, y, at);
        if (stage == 3) break;
        keep();
        ++stage;
    }
    const Place drawn = at;
    if (drawn.id == kNone) s.find_token(drawn, a.token + r);
    else if (s.rank == 0 && tid == 0) a.token[r] = (int32_t)drawn.id;
    if (s.rank == 0 && tid == 0 && a.logprob)
        a.logprob[r] = (float)((drawn.d == s.top ? 0.0 : (K::value(drawn.d) - s.x_top) * s.inv_t) - log((double)mass / s.scale));
}

template <typename T, int kThreads, bool kAlone>
cudaError_t launch_one(const SampleArgs &a, int rows, int C, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    const size_t smem = C > 1 ? sizeof(Shared<T>) : offsetof(Shared<T>, all_count);
    const cudaError_t e = configure(sample_tokens_kernel<T, kThreads, kAlone>, done, (int)smem, false);
    if (e != cudaSuccess) return e;
    for (int r0 = 0; r0 < rows; r0 += 65535) {               // (what a grid's second dimension holds)
        const int n = rows - r0 < 65535 ? rows - r0 : 65535;
        SampleArgs b = a;
        b.logits = static_cast<const T *>(a.logits) + r0 * a.stride;
        b.temperature += r0; b.u += r0; b.token += r0;
        if (b.top_k) b.top_k += r0;
        if (b.top_p) b.top_p += r0;
        if (b.min_p) b.min_p += r0;
        if (b.logprob) b.logprob += r0;
        const cudaError_t x = launch_clusters(true, C, sample_tokens_kernel<T, kThreads, kAlone>, dim3(C, n), kThreads, smem, st, b);
        if (x != cudaSuccess) return x;
    }
    return cudaSuccess;
}

// CTAs per row: several while they find SMs of their own and have something to count.  fp32 rows with an SM of their own have all its threads,
// which wait for exponentials and atomics (75 rows of 128256 163 us with 256 threads, 85 with 1024; 148 of 32000 46 and 29; 75 of 8000 16.1 and 14.0).  bf16 rows
// gain little (36.9 and 34.3; 75 of 8000 13.3 and 14.8) and keep to 256.
template <typename T> cudaError_t launch_type(const SampleArgs &a, int rows, cudaStream_t st)
{
    int C = 1;
    while (C < 8 && (long long)rows * C * 2 <= num_sms() && a.vocab / (C * 2) >= 2048) C *= 2;
    if (C > 1) return launch_one<T, 512, false>(a, rows, C, st);
    if constexpr (!Keys<T>::HALF)
        if (rows <= num_sms()) return launch_one<T, 1024, true>(a, rows, 1, st);
    return launch_one<T, 256, true>(a, rows, 1, st);
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
    return dtype == ORTHRUS_FP32 ? launch_type<float>(a, rows, st) : launch_type<__nv_bfloat16>(a, rows, st);
}

}  // namespace orthrus
