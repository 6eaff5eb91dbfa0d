// Losses of tokens and their gradients (zkdl_token_logprobs, zkdl_token_logprobs_backward, zkdl_policy_loss, zkdl_preference_loss).
//
// A row of logits x gives, with u = x / temperature and c = max_j x_j, the sum S = sum_j exp(u_j - u_c) and with it the token's
// log-probability and every p_j = exp(u_j - u_c) / S.  All of it is bound by memory: 2 or 4 bytes an entry read (and written) against about
// 18 operations' time (the exponential counts four, and a gradient has it twice).  So a row is read once, all its loads under way before the
// first is looked at, and stays in registers and LDS until its gradient leaves (k_loss_rows, k_loss_small); only rows that are longer, few or
// wanted together (the preference's sums need all of them before the first gradient) are read twice (k_loss_part, k_loss_slope).  Rates
// beside the kernels: MI355X, where a copy of 1 GiB moves 5.2 TB/s.
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "layer8.cuh"
#include "vec8.cuh"

namespace {

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float INF = __builtin_huge_valf(), NAN32 = __builtin_nanf("");

__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }    // 1 ulp; 0 below 2^-126, where nothing is left of a probability

// Integers of 32 or 64 bits, without a branch: loads of several are under way at once.
struct Ints {
    const void* p;
    int wide;       // 0 or 1
    __device__ __forceinline__ int64_t at(uint64_t i) const {
        const uint32_t* q = (const uint32_t*)p + (i << wide);
        const uint32_t low = q[0], high = q[wide];
        return (int64_t)((uint64_t)(wide ? high : (uint32_t)((int32_t)low >> 31)) << 32 | low);
    }
};

struct LossArgs {
    uint64_t rows;
    uint32_t cols;
    float inv_tau, k;            // 1 / temperature; log2(e) / temperature
    float times, step;           // top is the largest logit times `times`, and p_j = exp2((x_j times - top) step - log_sum log2(e)):
                                 // 1 / temperature and log2(e) where the caller has top, 1 and log2(e) / temperature where it stays here
    double inv_tau64;
    Ints tokens;
    Ints offsets;                // preference: rows outside [offsets[0], offsets[last]) count for nothing
    uint64_t last;
    float *logp, *top, *log_sum; // may be null
    double* logp64;              // preference: for the pairs' sums
    float* dlogp;                // preference: zeros, for the pairs to fill in
    // policy
    const float *old_logp, *advantage, *ref_logp, *weight;
    double every, low, high, kl; // the weight where there are none; 1 - clip_low, 1 + clip_high
    float* terms;                // [3][rows]: weighted loss, divergence, clipped
    int past;                    // the gradient goes past the caches (where a kernel has that)
};

enum { ROWS_LOGP, ROWS_POLICY, ROWS_SLOPE };

// The row's token, or -1 where the row counts for nothing.
__device__ __forceinline__ int64_t token_of(const LossArgs& a, uint64_t r) {
    const int64_t y = a.tokens.at(r);
    if (!a.offsets.p) return y;
    const int64_t lo = a.offsets.at(0), hi = a.offsets.at(a.last);
    return (int64_t)r < lo || (int64_t)r >= hi ? -1 : y;
}

// Terms are exp2((x - c) k): the difference first, so that rows of the type's lowest value (masks) and of its largest stay in the range.
__device__ __forceinline__ float term_of(float x, float c, float k) { return exp2_raw((x - c) * k); }

// x times - top, the product rounded by itself as top was: of the row's largest nothing is left.  (With what a fused product has beyond 32 bits all p_j
// of a row would be off by a factor, up to exp(2^-24 |top|).)
__device__ __forceinline__ float below_top(float x, float times, float top) {
#pragma clang fp contract(off)
    const float u = x * times;
    return u - top;
}

// The logarithm of a row's sum, and what is taken from it, in 64 bits: in 32 the last places of log_sum and logp are a millionth at 10, which a loss has in
// every ratio and, of sums that cancel, in its first places (policy, 2000 x 4001 16-bit entries, a loss of 0.03: off by 2.1e-9, from log-probabilities
// rounded to 32 bits by 5.6e-9).  The logarithm is the exponent and that of a number next to 1, which 32 bits hold to 2^-25.  The sum itself is in 32
// bits, and so is k, whose rounding all terms share: both stay in logp (4096 x 131072 entries: off by -5e-8 on average over the rows).
struct RowStats {
    float top, log_sum;
    double logp;
};
__device__ __forceinline__ RowStats row_stats(const LossArgs& a, float c, float sum, int64_t y, float xy) {
    const float m = __builtin_amdgcn_frexp_mantf(sum);          // 1/2 <= m < 1
    const bool low = m < .70710678f;
    const double log_sum = ((double)(__builtin_amdgcn_frexp_expf(sum) - low) + (double)__builtin_amdgcn_logf(low ? 2 * m : m)) * 0.69314718055994530942;
    RowStats s;
    s.log_sum = (float)log_sum;
    s.top = c * a.times;
    s.logp = ((double)xy - (double)c) * a.inv_tau64 - log_sum;
    if (!(sum < INF)) s.top = s.log_sum = NAN32;          // a NaN, +infinity, or nothing but -infinity
    if (!(sum < INF) || y >= (int64_t)a.cols) s.logp = NAN32;
    return s;
}

// em = exp(d) - 1, of grown = exp(d), and exp(d) - 1 - d: where d is small by the series, which is off by d^3 / 60 < 2^-35 of it; the difference in 64 bits by 2^-52 of 1,
// 2^-31 of it at most.
__device__ __forceinline__ double divergence_of(double d, double grown, double& em) {
    const double small = d * d * fma(d, fma(d, 1. / 24, 1. / 6), .5);
    const bool near = fabs(d) < 0x1p-10;
    em = near ? small + d : grown - 1;
    return near ? small : em < INF ? em - d : em;       // (d may be infinite: a token that cannot be)
}

// A number that the lane next door has, of each pair of lanes.
__device__ __forceinline__ double next_door(double x) {
    const auto swap = [](int w) { return __builtin_amdgcn_mov_dpp(w, 0xB1, 0xF, 0xF, true); };
    return __hiloint2double(swap(__double2hiint(x)), swap(__double2loint(x)));
}

// What the policy loss has of a row beside its logits, asked for before they are looked at.
struct PolicyRow {
    float w, adv, old, ref;
};
template <int MODE>
__device__ __forceinline__ PolicyRow policy_of(const LossArgs& a, uint64_t r) {
    if constexpr (MODE != ROWS_POLICY) return {0.f, 0.f, 0.f, 0.f};
    return {a.weight ? a.weight[r] : 1.f, a.advantage[r], a.old_logp[r], a.ref_logp ? a.ref_logp[r] : 0.f};
}
// One row's share of the policy loss; returns dlogp.  In 64 bits up to the three terms and dlogp, which are rounded once, with the weight in them: a
// ratio or a divergence beyond 2^128 may have a weight that brings it back, and the terms' sum may be much smaller than they are (the
// loss of 4096 x 131072 16-bit entries, terms of 0.6 and a sum of 0.01: off by 1.2e-9, with shares in 32 bits by 1.4e-9).  What is loaded is widened
// here and not where it is asked for, which would wait for it (4096 x 1024 32-bit entries 12.0 us, 12.6 that way).  PAIRS: of two lanes, which have the same
// row, one takes the ratio's exponential and the other the divergence's, where the vector operations show (2^20 rows of 32 with a reference
// 97 us; both in every lane 101, in 32 bits 89).
template <bool PAIRS = false>
__device__ __forceinline__ float policy_row(const LossArgs& a, const PolicyRow& row, double logp, float (&term)[3]) {
    const double w = a.weight ? (double)row.w : a.every, adv = row.adv;
    if (row.w == 0) {           // whatever the rest is
        term[0] = term[1] = term[2] = 0.f;
        return 0.f;
    }
    double ratio, grown = 0.;
    if constexpr (PAIRS) {
        const bool odd = threadIdx.x & 1;
        const double mine = exp(odd ? (double)row.ref - logp : logp - (double)row.old), other = next_door(mine);
        ratio = odd ? other : mine;
        grown = odd ? mine : other;
    } else {
        ratio = exp(logp - (double)row.old);
        if (a.ref_logp) grown = exp((double)row.ref - logp);
    }
    const bool up = adv > 0 && ratio > a.high, down = adv < 0 && ratio < a.low, clipped = up || down;
    const double gain = adv == 0 ? 0. : (up ? a.high : down ? a.low : ratio) * adv;
    double slope = clipped || adv == 0 ? 0. : -adv * ratio, div = 0.;
    if (a.ref_logp) {
        double em;
        div = divergence_of((double)row.ref - logp, grown, em);
        if (a.kl != 0) slope = fma(-a.kl, em, slope);
    }
    term[0] = (float)(w * (a.kl != 0 ? fma(a.kl, div, -gain) : -gain));     // (a divergence without end that nobody asked for stays out)
    term[1] = (float)(w * div);
    term[2] = clipped ? (float)w : 0.f;
    return (float)(w * slope);
}
__device__ __forceinline__ void put_terms(const LossArgs& a, uint64_t r, const float (&term)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) a.terms[i * a.rows + r] = term[i];
}

// A number that all lanes of the wave have, in a scalar register.
__device__ __forceinline__ float of_wave(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
    return x;
}
// over the G threads of a row, a block's waves with one store each
template <int G, bool MAX>
__device__ __forceinline__ float row_reduce(float x, float* s) {
    x = MAX ? wave_max(x) : l8_wave_sum(x);
    if constexpr (G > 64) {
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
        __syncthreads();
        x = s[0];
#pragma unroll
        for (int i = 1; i < G / 64; ++i) x = MAX ? fmaxf(x, s[i]) : x + s[i];
    }
    return x;
}

template <class T>
__device__ __forceinline__ float max8(float c, const Raw8<T>& v) {
    float f[8];
    floats8(v, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) c = fmaxf(c, f[i]);
    return c;
}
// -co p_j of eight entries; the token's own entry is put over it by the same thread afterwards.
template <class T>
__device__ __forceinline__ void slope8(const Raw8<T>& v, float c, float k, float co_inv, float (&f)[8]) {
    floats8(v, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = term_of(f[i], c, k) * -co_inv;
}
template <class T>
__device__ __forceinline__ void put_one(T* to, float x) {
    T o;
    l8_put(x, o);
    *to = o;
}
// The part of a vector at the row's end that no other thread has.
template <class T>
__device__ __forceinline__ void put_end(T* row, const L8At& end, const float (&f)[8]) {
    if (!end.live) return;
    if (end.dup == 0) {
        l8_store(row + end.start, 8, f);
        return;
    }
#pragma unroll
    for (int i = 1; i < 8; ++i)
        if ((uint32_t)i >= end.dup) put_one(row + end.start + i, f[i]);
}

// A thread's offset in bytes, opaque, so that it stays the 32-bit offset that the instructions below take.
template <class T>
__device__ __forceinline__ uint32_t own_offset(uint32_t t) {
    uint32_t o = t * 8 * (uint32_t)sizeof(T);
    asm("" : "+v"(o));
    return o;
}
// Eight items, `lane` bytes behind p + n, p and n being the whole wave's: the instruction adds the lane's own offset, and no vector has an address
// of 64 bits of its own.
template <class T>
__device__ __forceinline__ Raw8<T> load8_at(const T* p, uint32_t n, uint32_t lane) {
    uint64_t at = (uint64_t)(p + n);
    asm("" : "+s"(at));
    const auto* q = (const __attribute__((address_space(1))) QuadAnywhere*)(at + lane);
    Raw8<T> v;
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) v.q[h] = q[h];
    return v;
}
template <bool PAST = false, class T>
__device__ __forceinline__ void store8_at(T* p, uint32_t n, uint32_t lane, const float (&f)[8]) {
    uint64_t at = (uint64_t)(p + n);
    asm("" : "+s"(at));
    auto* q = (__attribute__((address_space(1))) QuadAnywhere*)(at + lane);
    Raw8<T> w;
    pack8(f, w);
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        if (PAST) __builtin_nontemporal_store(w.q[h], q + h);
        else q[h] = w.q[h];
    }
}
// A thread's vector in LDS, 16 bytes of it next to the other threads'.
template <class T, int N>
__device__ __forceinline__ void put_lds(Quad (*to)[N], uint32_t t, const Raw8<T>& v) {
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) to[h][t] = v.q[h];
}
template <class T, int N>
__device__ __forceinline__ Raw8<T> get_lds(Quad (*from)[N], uint32_t t) {
    Raw8<T> v;
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) v.q[h] = from[h][t];
    return v;
}
// Where vector k of a row lies: rows begin with different ones.  Blocks run side by side, and rows of a power of two of bytes would have all of them
// ask the same memory channels at once.
template <int G, int WHOLE>
__device__ __forceinline__ uint32_t place_of(int k, uint32_t turn) {
    const uint32_t i = k + turn;
    return (i < (uint32_t)WHOLE ? i : i - WHOLE) * (8 * G);
}
template <class T, int G, int WHOLE>
__device__ __forceinline__ void put_zeros(T* to, uint32_t mine, uint32_t turn, bool ends, const L8At& end) {
    const float zero[8] = {};
#pragma unroll 4
    for (int k = 0; k < WHOLE; ++k) store8_at(to, place_of<G, WHOLE>(k, turn), mine, zero);
    if (ends) put_end(to, end, zero);
}

// ---------------------------------------------------------------------------
// Rows that stay on the chip: G threads a row (a wave: four rows a block) with WHOLE vectors of eight each, and one at the row's end:
// 8 G WHOLE <= cols < 8 G (WHOLE + 1), cols > 256.  The vectors are in registers, but for the last of the longest rows, which lie in LDS: so two
// blocks of 512 threads with 128 registers each, and half of the LDS, have room in a compute unit up to rows of 256 kB, and one of them has
// memory at work while the other computes.  (As many instances as there are lengths: with a count that the kernel learns when it runs, the
// vectors' registers were copied and spilled.)  Bound by memory: log-probabilities of 4096 x 32768 16-bit entries, a quarter of the rows
// not read, 38.3 us (5.2 TB/s); the policy's gradient of 4096 x 131072, a quarter zeros, 360 us (5.2 TB/s), of 4096 x 16384 49 us (5.5 TB/s).
// ---------------------------------------------------------------------------
constexpr int loss_threads(int G) { return G < 256 ? 256 : G; }
// vectors in registers, by what else a thread holds, and in LDS, of which a compute unit has 160 kB
template <class T>
constexpr int loss_regs(int whole) { return whole <= 32 / (int)sizeof(T) ? whole : whole <= 50 / (int)sizeof(T) ? 32 / (int)sizeof(T) : whole - 18 / (int)sizeof(T); }
template <class T, int MODE, int G, int WHOLE>
__global__ __launch_bounds__(loss_threads(G), G == 512 ? 4 : 1) void k_loss_rows(LossArgs a, L8Mat<const T> x, L8Mat<T> out) {
    constexpr int GROUPS = loss_threads(G) / G, REGS = loss_regs<T>(WHOLE), STORED = WHOLE - REGS;
    constexpr uint32_t EACH = 8 * G;
    __shared__ float s_max[G / 64], s_sum[G / 64];
    __shared__ Quad s_v[STORED ? STORED * (sizeof(T) / 2) : 1][STORED ? G : 1];
    const uint32_t t = threadIdx.x % G, mine = own_offset<T>(t);
    const uint32_t group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / G);
    const bool ends = WHOLE * EACH < a.cols;
    const L8At end = l8_at(WHOLE * EACH + t * 8, a.cols);
    const uint64_t r = ((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * GROUPS + group;       // (a loop over rows would keep its constants in registers)
    if (r >= a.rows) return;
    const uint32_t turn = G > 64 && WHOLE > 1 ? (uint32_t)r % (WHOLE ? WHOLE : 1) : 0;
    const int64_t y = token_of(a, r);
    T* const to = out.p + r * out.rs;
    float term[3] = {0.f, 0.f, 0.f};
    RowStats st = {0.f, 0.f, 0.};
    if (y >= 0) {
        const T* const row = x.p + r * x.rs;
        Raw8<T> v[REGS ? REGS : 1], last;
        float c = -INF, sum = 0.f;
#pragma unroll
        for (int k = 0; k < STORED; ++k) v[k] = load8_at(row, place_of<G, WHOLE>(REGS + k, turn), mine);
#pragma unroll
        for (int k = STORED; k < REGS; ++k) v[k] = load8_at(row, place_of<G, WHOLE>(k, turn), mine);
#pragma unroll
        for (int k = 0; k < STORED; ++k) {
            c = max8(c, v[k]);
            put_lds<T>(&s_v[k * (sizeof(T) / 2)], t, v[k]);
            const T* rest = row;
            asm volatile("" : "+s"(rest), "+v"(c));        // the next load waits for this vector's maximum: its registers are that load's
            v[k] = load8_at(rest, place_of<G, WHOLE>(k, turn), mine);
        }
        if (ends) last = load8(row + end.start);
        const float xy = l8_f32(row[y < (int64_t)a.cols ? y : 0]);
        const PolicyRow given = policy_of<MODE>(a, r);
#pragma unroll
        for (int k = 0; k < REGS; ++k) {
            c = max8(c, v[(k + STORED) % (REGS ? REGS : 1)]);       // in the order in which they were asked for
            if (STORED) __builtin_amdgcn_sched_barrier(0);
        }
        if (ends) c = max8(c, last);
        c = of_wave(row_reduce<G, true>(c, s_max));
#pragma unroll
        for (int k = 0; k < WHOLE; ++k) {
            float f[8];
            if (k < REGS) {
                keep_packed(v[k < REGS ? k : 0]);
                floats8(v[k < REGS ? k : 0], f);
            } else {
                floats8(get_lds<T>(&s_v[(k < REGS ? 0 : k - REGS) * (sizeof(T) / 2)], t), f);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += term_of(f[i], c, a.k);
            if (STORED) __builtin_amdgcn_sched_barrier(0);      // one vector's floats at a time: no registers are left for more
        }
        if (ends) {         // what another thread has, or nobody, stays out
            float f[8];
            if (STORED) last = load8(row + end.start);          // (read again: the registers are the others')
            else keep_packed(last);
            floats8(last, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += end.live && (uint32_t)i >= end.dup ? term_of(f[i], c, a.k) : 0.f;
        }
        sum = of_wave(row_reduce<G, false>(sum, s_sum));
        st = row_stats(a, c, sum, y, xy);
        if (MODE == ROWS_POLICY) {
            const float dlogp = policy_row(a, given, st.logp, term);
            const float co = dlogp * a.inv_tau, co_inv = of_wave(co / sum);
            if (out.p && dlogp != 0) {
                float f[8];
                const auto put_all = [&](auto past) {
#pragma unroll
                    for (int k = 0; k < WHOLE; ++k) {
                        if (k < REGS) {
                            keep_packed(v[k < REGS ? k : 0]);
                            slope8(v[k < REGS ? k : 0], c, a.k, co_inv, f);
                        } else {
                            slope8(get_lds<T>(&s_v[(k < REGS ? 0 : k - REGS) * (sizeof(T) / 2)], t), c, a.k, co_inv, f);
                        }
                        store8_at<decltype(past)::value>(to, place_of<G, WHOLE>(k, turn), mine, f);
                        if (STORED) __builtin_amdgcn_sched_barrier(0);
                    }
                };
                if (STORED && sizeof(T) == 2 && a.past) put_all(std::true_type());
                else put_all(std::false_type());
                if (ends) {
                    if (STORED) last = load8(row + end.start);
                    else keep_packed(last);
                    slope8(last, c, a.k, co_inv, f);
                    put_end(to, end, f);
                }
                if (y < (int64_t)a.cols && t == (uint32_t)y / 8 % G) put_one(to + y, fmaf(-co_inv, term_of(xy, c, a.k), co));
            } else if (out.p) {
                put_zeros<T, G, WHOLE>(to, mine, turn, ends, end);
            }
        }
    } else if (MODE == ROWS_POLICY && out.p) {
        put_zeros<T, G, WHOLE>(to, mine, turn, ends, end);
    }
    if (t == 0) {
        if (a.logp) a.logp[r] = (float)st.logp;
        if (a.logp64) a.logp64[r] = st.logp;
        if (a.top) a.top[r] = st.top;
        if (a.log_sum) a.log_sum[r] = st.log_sum;
        if (a.dlogp) a.dlogp[r] = 0.f;
        if (MODE == ROWS_POLICY) put_terms(a, r, term);
    }
}

// ---------------------------------------------------------------------------
// Rows of up to 8 G entries for G = 8, 16 or 32 lanes: as many rows in a wave as fit, a vector of eight (or what there is) a lane.
// ROWS_SLOPE: the gradient from dlogp, top and log_sum alone.  2^20 rows of 128 32-bit entries: log-probabilities 112 us (4.8 TB/s), gradient
// 191 us (5.6 TB/s), policy 223 us.
// ---------------------------------------------------------------------------
template <int G, bool MAX>
__device__ __forceinline__ float lanes_reduce(float x) {
#pragma unroll
    for (int d = G / 2; d; d >>= 1) {
        const float y = __shfl_xor(x, d, 64);
        x = MAX ? fmaxf(x, y) : x + y;
    }
    return x;
}
template <class T, int MODE, int G>
__global__ __launch_bounds__(256) void k_loss_small(LossArgs a, const float* dlogp_in, const float* top, const float* log_sum, L8Mat<const T> x, L8Mat<T> out) {
    const uint32_t t = threadIdx.x % G, j = t * 8;
    const uint64_t r = ((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * (256 / G) + threadIdx.x / G;
    if (r >= a.rows) return;
    const int n = j < a.cols ? (int)min(8u, a.cols - j) : 0;
    const int64_t y = token_of(a, r);
    float f[8], term[3] = {0.f, 0.f, 0.f}, dlogp = 0.f, co_inv = 0.f;
    RowStats st = {0.f, 0.f, 0.};
    if (MODE == ROWS_SLOPE) dlogp = y < 0 ? 0.f : dlogp_in[r];
    const bool bad = y >= (int64_t)a.cols, live = MODE == ROWS_SLOPE ? dlogp != 0 : y >= 0;
    if (live) {
        const T* const row = x.p + r * x.rs;
        l8_load(row + (n ? j : 0), n, f);
        if (MODE == ROWS_SLOPE) {
            const float norm = log_sum[r] * LOG2E;
            float c = top[r], times = a.times, k = a.step;
            if (fabsf(c) == INF) {          // as in slope_far
                c = -INF;
#pragma unroll
                for (int i = 0; i < 8; ++i) c = fmaxf(c, i < n ? f[i] : -INF);
                c = lanes_reduce<G, true>(c);
                times = 1.f;
                k = a.k;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = exp2_raw(fmaf(below_top(f[i], times, c), k, -norm));
            if (bad) dlogp = NAN32;
            co_inv = dlogp * a.inv_tau;
        } else {
            const float xy = l8_f32(row[bad ? 0 : y]);
            const PolicyRow given = policy_of<MODE>(a, r);
            float c = -INF, sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) c = fmaxf(c, i < n ? f[i] : -INF);
            c = lanes_reduce<G, true>(c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[i] = term_of(f[i], c, a.k);
                sum += i < n ? f[i] : 0.f;
            }
            sum = lanes_reduce<G, false>(sum);
            st = row_stats(a, c, sum, y, xy);
            if (MODE == ROWS_POLICY) {
                dlogp = policy_row<true>(a, given, st.logp, term);
                co_inv = dlogp * a.inv_tau / sum;
            }
        }
    }
    if (MODE != ROWS_SLOPE && t == 0) {
        if (a.logp) a.logp[r] = (float)st.logp;
        if (a.logp64) a.logp64[r] = st.logp;
        if (a.top) a.top[r] = st.top;
        if (a.log_sum) a.log_sum[r] = st.log_sum;
        if (a.dlogp) a.dlogp[r] = 0.f;
        if (MODE == ROWS_POLICY) put_terms(a, r, term);
    }
    if (MODE != ROWS_LOGP && out.p && n) {
        const float co = dlogp * a.inv_tau;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f[i] = dlogp == 0 ? 0.f : f[i] * -co_inv;
            f[i] += dlogp != 0 && (uint64_t)y == j + i ? co : 0.f;
        }
        l8_store(out.p + r * out.rs + j, n, f);
    }
}

// ---------------------------------------------------------------------------
// Rows in parts: few long rows on many blocks, and rows longer than the chip holds.  A block has 2048 ITEMS entries of a row: their
// largest, and the sum of exp2((x - largest) k).  One row of 131072: 3.8 us, and 2.5 for joining its 16 parts (launches and trips to
// memory); 1024 such rows of 16 bits 52 us (5.2 TB/s).
// ---------------------------------------------------------------------------
struct Part {
    float top, sum;
};
// FULL: the row does not end in it, so that no load waits for a branch.
template <class T, int ITEMS, bool FULL>
__device__ __forceinline__ void part_of(const LossArgs& a, const T* row, uint32_t q, float& c, float& sum, float* s_max, float* s_sum) {
    float f[ITEMS][8];
    int n[ITEMS];
    if constexpr (FULL) {
        Raw8<T> v[ITEMS];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) v[k] = load8_at(row + (uint64_t)q * (ITEMS * 2048), k * 2048, own_offset<T>(threadIdx.x));
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            n[k] = 8;
            floats8(v[k], f[k]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const uint64_t j = ((uint64_t)(q * ITEMS + k) * 256 + threadIdx.x) * 8;
            n[k] = j < a.cols ? (int)min((uint64_t)8, a.cols - j) : 0;
            l8_load(row + (n[k] ? j : 0), n[k], f[k]);
        }
    }
    c = -INF;
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) c = fmaxf(c, FULL || i < n[k] ? f[k][i] : -INF);
    c = of_wave(row_reduce<256, true>(c, s_max));
    if (c == -INF) {        // nothing but -infinity, which adds nothing, or NaN
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (FULL || i < n[k]) && f[k][i] != f[k][i] ? NAN32 : 0.f;
    } else {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += FULL || i < n[k] ? term_of(f[k][i], c, a.k) : 0.f;
    }
    sum = row_reduce<256, false>(sum, s_sum);
}
template <class T, int ITEMS>
__global__ __launch_bounds__(256) void k_loss_part(LossArgs a, L8Mat<const T> x, Part* part, uint32_t parts) {
    __shared__ float s_max[4], s_sum[4];
    for (uint64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        if (token_of(a, r) < 0) continue;
        const T* row = x.p + r * x.rs;
        for (uint32_t q = blockIdx.x; q < parts; q += gridDim.x) {
            float c, sum;
            if ((uint64_t)(q + 1) * ITEMS * 2048 <= a.cols) part_of<T, ITEMS, true>(a, row, q, c, sum, s_max, s_sum);
            else part_of<T, ITEMS, false>(a, row, q, c, sum, s_max, s_sum);
            if (threadIdx.x == 0) part[r * parts + q] = {c, sum};
            __syncthreads();
        }
    }
}

// A row's parts together, a block a row; of the policy loss the row's terms and dlogp as well.
template <class T, int MODE>
__global__ __launch_bounds__(256) void k_loss_join(LossArgs a, L8Mat<const T> x, const Part* part, uint32_t parts) {
    __shared__ float s_max[4], s_sum[4];
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t y = token_of(a, r);
        RowStats st = {0.f, 0.f, 0.};
        float term[3] = {0.f, 0.f, 0.f}, dlogp = 0.f;
        if (y >= 0) {
            const float xy = l8_f32(x.p[r * x.rs + (y < (int64_t)a.cols ? y : 0)]);
            const PolicyRow given = policy_of<MODE>(a, r);
            float c = -INF, sum = 0.f;
            for (uint32_t q = threadIdx.x; q < parts; q += 256) c = fmaxf(c, part[r * parts + q].top);
            c = row_reduce<256, true>(c, s_max);
            for (uint32_t q = threadIdx.x; q < parts; q += 256) {
                const Part p = part[r * parts + q];
                sum = fmaf(p.sum, term_of(p.top, c, a.k), sum);
            }
            sum = row_reduce<256, false>(sum, s_sum);
            st = row_stats(a, c, sum, y, xy);
            if (MODE == ROWS_POLICY) dlogp = policy_row(a, given, st.logp, term);
        }
        if (threadIdx.x == 0) {
            if (a.logp) a.logp[r] = (float)st.logp;
            if (a.logp64) a.logp64[r] = st.logp;
            if (a.top) a.top[r] = st.top;
            if (a.log_sum) a.log_sum[r] = st.log_sum;
            if (a.dlogp) a.dlogp[r] = dlogp;
            if (MODE == ROWS_POLICY) put_terms(a, r, term);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// Sums over rows, in 64 bits and always in the same order
// ---------------------------------------------------------------------------
__device__ __forceinline__ double wave_sum64(double x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}
// N sums over a block of WAVES waves; s: N times as many numbers
template <int N, int WAVES>
__device__ __forceinline__ void block_sums64(double (&x)[N], double (*s)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = wave_sum64(x[i]);
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6][i] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x[i] += s[w][i];
    }
}
// out[b] = the sum of in[b][0 .. n), a block each
template <class IN, class OUT>
__global__ __launch_bounds__(1024) void k_loss_sum(const IN* in, uint64_t n, uint64_t per, OUT* out) {
    __shared__ double s[16][1];
    const uint64_t lo = blockIdx.x * per, hi = min(n, lo + per);
    double x[1] = {0};
    for (uint64_t i = lo + threadIdx.x; i < hi; i += 1024) x[0] += (double)in[blockIdx.y * n + i];
    block_sums64<1, 16>(x, s);
    if (threadIdx.x == 0) out[(uint64_t)blockIdx.y * gridDim.x + blockIdx.x] = (OUT)x[0];
}

// ---------------------------------------------------------------------------
// The gradient of the logits from dlogp, top and log_sum: a wave has 2048 entries of a row, four loads under way.  Bound by memory: 2048 x 65536
// 32-bit entries 193 us (5.6 TB/s); behind the forward pass of 4096 x 32768 16-bit entries 63 us (7.2 TB/s: the logits are still in the
// last-level cache).
// ---------------------------------------------------------------------------
struct SlopeRow {
    float co, times, step, top, norm;   // p_j = exp2((x_j times - top) step - norm)
    int64_t y;
    bool none, bad;                     // zeros, NaN
};
template <class T, bool FULL, bool PAST>
__device__ __forceinline__ void slope_of(const SlopeRow& s, const T* row, T* to, uint32_t cols, uint32_t at, uint32_t lane) {
    float f[4][8];
    int n[4];
    const uint32_t mine = own_offset<T>(lane);
    if constexpr (FULL) {
        if (!s.none) {
            Raw8<T> v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = load8_at(row + at, k * 512, mine);
#pragma unroll
            for (int k = 0; k < 4; ++k) floats8(v[k], f[k]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint64_t j = (uint64_t)at + (k * 64 + lane) * 8;
            n[k] = j < cols ? (int)min((uint64_t)8, cols - j) : 0;
            if (!s.none) l8_load(row + (n[k] ? j : 0), n[k], f[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint64_t j = (uint64_t)at + (k * 64 + lane) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[k][i] = s.none ? 0.f : exp2_raw(fmaf(below_top(f[k][i], s.times, s.top), s.step, -s.norm)) * (s.bad ? NAN32 : -s.co);
        if ((uint64_t)s.y - j < 8 && !s.bad && !s.none) {       // the token's own entry
#pragma unroll
            for (int i = 0; i < 8; ++i) f[k][i] += (uint64_t)s.y - j == i ? s.co : 0.f;
        }
        if (FULL) store8_at<PAST>(to + at, k * 512, mine, f[k]);
        else l8_store(to + (n[k] ? j : 0), n[k], f[k]);
    }
}
// The same where logits / temperature, and with it top, are beyond 32 bits: from the row's largest logit c, p_j = exp2((x_j - c) k - norm).  Rare (rows of
// nothing but a mask of the lowest value), and apart from the rest, whose registers it would take.
template <class T>
__device__ __forceinline__ void slope_far(const SlopeRow& s, float k, const T* row, T* to, uint32_t cols, uint32_t first, uint32_t step, uint32_t lane) {
    asm volatile("" : "+v"(lane));
    float c = -INF;
#pragma unroll 1
    for (uint32_t j = lane; j < cols; j += 64) c = fmaxf(c, l8_f32(row[j]));
#pragma unroll 1
    for (int d = 32; d; d >>= 1) c = fmaxf(c, __int_as_float(__builtin_amdgcn_ds_bpermute((int)((lane ^ d) * 4), __float_as_int(c))));
    c = of_wave(c);
#pragma unroll 1
    for (uint64_t at = first; at < cols; at += step)
#pragma unroll 1
        for (uint64_t j = at + lane; j < min(at + 2048, (uint64_t)cols); j += 64) {
            const float p = exp2_raw(fmaf(l8_f32(row[j]) - c, k, -s.norm));
            put_one(to + j, s.bad ? NAN32 : (uint64_t)s.y == j ? fmaf(-p, s.co, s.co) : -p * s.co);
        }
}
template <class T>
__global__ __launch_bounds__(256) void k_loss_slope(LossArgs a, const float* dlogp, const float* top, const float* log_sum, L8Mat<const T> x, L8Mat<T> out,
                                                    uint32_t segs, uint32_t waves, const float* losses, uint64_t pairs, float* loss) {
    if (losses && blockIdx.x == 0 && blockIdx.y == 0) {         // the preference's loss, beside the gradient
        __shared__ double s_loss[4][1];
        double sum[1] = {0};
        for (uint64_t i = threadIdx.x; i < pairs; i += 256) sum[0] += (double)losses[i];
        block_sums64<1, 4>(sum, s_loss);
        if (threadIdx.x == 0) *loss = (float)sum[0];
    }
    // waves: of a row in one block, 1, 2 or 4
    const uint32_t per = 4 / waves, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (uint64_t r = (uint64_t)blockIdx.y * per + wave / waves; r < a.rows; r += (uint64_t)gridDim.y * per) {
        SlopeRow s;
        const float d = dlogp[r];
        s.y = token_of(a, r);
        s.co = d * a.inv_tau;
        s.none = s.y < 0 || d == 0;
        s.bad = s.y >= (int64_t)a.cols;
        s.times = a.times;
        s.step = a.step;
        s.top = top[r];
        s.norm = log_sum[r] * LOG2E;
        if (!s.none && fabsf(s.top) == INF) {
            slope_far(s, a.k, x.p + r * x.rs, out.p + r * out.rs, a.cols, (blockIdx.x * waves + wave % waves) * 2048, gridDim.x * waves * 2048, lane);
            continue;
        }
        for (uint32_t q = blockIdx.x * waves + wave % waves; q < segs; q += gridDim.x * waves) {
            if ((uint64_t)(q + 1) * 2048 <= a.cols) {
                if (sizeof(T) == 2 && a.past) slope_of<T, true, true>(s, x.p + r * x.rs, out.p + r * out.rs, a.cols, q * 2048, lane);
                else slope_of<T, true, false>(s, x.p + r * x.rs, out.p + r * out.rs, a.cols, q * 2048, lane);
            } else slope_of<T, false, false>(s, x.p + r * x.rs, out.p + r * out.rs, a.cols, q * 2048, lane);
        }
    }
}

// ---------------------------------------------------------------------------
// A pair of sequences, a block each: its margin, its share of the loss, and dlogp of its rows.  Three trips to memory behind one another and the
// logistic function in 64 bits: 16 pairs of 240 rows 5.3 us.
// ---------------------------------------------------------------------------
struct PairArgs {
    uint64_t rows, pairs;
    Ints tokens, offsets;
    const double* logp;         // (as they came out of the rows: what rounding took from each would be in the margin, where the sums cancel)
    const float *ref_logp, *weight;
    int form, average;
    float every, beta, target, smoothing;
    float *margin, *losses, *dlogp;
};
template <int N>
__global__ __launch_bounds__(N) void k_loss_pair(PairArgs a) {
    __shared__ double s[N / 64][4];
    for (uint64_t i = blockIdx.x; i < a.pairs; i += gridDim.x) {
        uint64_t at[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int64_t o = a.offsets.at(2 * i + k);
            at[k] = o < 0 ? 0 : min((uint64_t)o, a.rows);
        }
        at[1] = max(at[1], at[0]);
        double x[4] = {0, 0, 0, 0};         // of either sequence the sum, and the rows that count
#pragma unroll 4
        for (uint64_t r = at[0] + threadIdx.x; r < at[2]; r += N) {
            const int64_t y = a.tokens.at(r);
            const double p = a.logp[r];        // (no load waits for the token)
            const float q = a.ref_logp ? a.ref_logp[r] : 0.f;
            const double d = y >= 0 ? p - (double)q : 0., one = y >= 0 ? 1. : 0.;
            const bool second = r >= at[1];
            x[0] += second ? 0. : d;
            x[1] += second ? d : 0.;
            x[2] += second ? 0. : one;
            x[3] += second ? one : 0.;
        }
        block_sums64<4, N / 64>(x, s);
        const double share[2] = {a.average ? 1 / fmax(x[2], 1.) : 1., a.average ? 1 / fmax(x[3], 1.) : 1.}, h[2] = {x[0] * share[0], x[1] * share[1]};
        const double margin = a.beta * (h[0] - h[1]), m = margin - a.target, w = a.weight ? (double)a.weight[i] : (double)a.every;
        double each, slope;
        if (a.form == ZKDL_PREF_LOGISTIC) {
            const double small = log1p(exp(-fabs(m)));          // log(1 + exp(-|m|))
            const double toward = fmax(-m, 0.) + small, away = fmax(m, 0.) + small;
            // (margins may be infinite: a sequence that cannot be)
            each = (a.smoothing < 1 ? (1 - a.smoothing) * toward : 0.) + (a.smoothing > 0 ? a.smoothing * away : 0.);
            slope = a.smoothing - 1 / (1 + exp(m));
        } else if (a.form == ZKDL_PREF_HINGE) {
            each = m >= 0 ? 0 : -m;
            slope = m >= 0 ? 0 : m < 0 ? -1 : m;
        } else {
            each = m * m;
            slope = 2 * m;
        }
        if (m != m) each = slope = m;
        if (w == 0) each = slope = 0;       // whatever the sequences hold
        if (threadIdx.x == 0) {
            if (a.margin) a.margin[i] = (float)margin;
            a.losses[i] = (float)(w * each);
        }
        if (a.dlogp) {
            const float d0 = (float)(w * slope * a.beta * share[0]), d1 = (float)(-w * slope * a.beta * share[1]);
#pragma unroll 4
            for (uint64_t r = at[0] + threadIdx.x; r < at[2]; r += N) a.dlogp[r] = a.tokens.at(r) < 0 ? 0.f : r >= at[1] ? d1 : d0;
        }
        __syncthreads();        // s is the next pair's
    }
}

// ---- launches ----------------------------------------------------------------------
// Whether rows stay on the chip, or go in parts: in registers rows below 136 kB are faster there however few they are (one row of 32768 16-bit entries
// 5.3 us against 8.2, 1024 of them 15 / 17.5; with the policy's gradient 8.6 / 14.3 and 25 / 43).  With a part of the row in LDS, up to
// 256 kB, only where a second read is saved, which a gradient needs, and rows enough to fill the device (policy, 131072 16-bit entries, in
// LDS / in parts: 128 rows 29.5 / 24.8, 256 rows 37.9 / 41.6, 1024 rows 130 / 155; log-probabilities of 1024 rows 73 / 52).
template <class T>
bool rows_fit(const LossArgs& a, bool slope) {
    constexpr uint32_t most = 32 / sizeof(T);       // vectors in registers
    return a.cols < 4096 * (most + 1) || (slope && a.rows >= 192 && a.cols <= 4096 * 2 * most);
}

template <class T, int MODE, int G, int WHOLE>
void launch_rows_of(zkdl_ctx* ctx, const LossArgs& a, L8Mat<const T> x, L8Mat<T> out) {
    const uint64_t blocks = l8_ceil(a.rows, loss_threads(G) / G), wide = blocks < (1u << 20) ? blocks : 1u << 20;
    hipLaunchKernelGGL((k_loss_rows<T, MODE, G, WHOLE>), dim3((unsigned)wide, (unsigned)l8_ceil(blocks, wide)), dim3(loss_threads(G)), 0, ctx->stream, a, x, out);
}
template <class T, int MODE, int G, int WHOLE, int LAST>
void launch_rows_from(zkdl_ctx* ctx, const LossArgs& a, L8Mat<const T> x, L8Mat<T> out) {
    if (a.cols / (8 * G) == WHOLE) launch_rows_of<T, MODE, G, WHOLE>(ctx, a, x, out);
    else if constexpr (WHOLE < LAST) launch_rows_from<T, MODE, G, WHOLE + 1, LAST>(ctx, a, x, out);
}
// Rows of 256 entries and less; 2^20 rows of 32 took 242 us with a wave each, 4 * 2^20 rows of 7 in parts 44 ms.
constexpr uint32_t LOSS_SMALL = 256;
template <class T, int MODE>
void launch_small(zkdl_ctx* ctx, const LossArgs& a, const float* dlogp, const float* top, const float* log_sum, L8Mat<const T> x, L8Mat<T> out) {
    const auto go = [&](auto g) {
        constexpr int G = decltype(g)::value;
        const uint64_t blocks = l8_ceil(a.rows, 256 / G), wide = blocks < (1u << 20) ? blocks : 1u << 20;
        hipLaunchKernelGGL((k_loss_small<T, MODE, G>), dim3((unsigned)wide, (unsigned)l8_ceil(blocks, wide)), dim3(256), 0, ctx->stream, a, dlogp, top, log_sum, x, out);
    };
    if (a.cols <= 64) go(std::integral_constant<int, 8>());
    else if (a.cols <= 128) go(std::integral_constant<int, 16>());
    else go(std::integral_constant<int, 32>());
}

// Few threads a row, with many vectors each, where there are rows enough to fill the device: more rows are under way at once, and fewer
// threads wait for one another.
template <class T, int MODE>
void launch_rows(zkdl_ctx* ctx, const LossArgs& a, L8Mat<const T> x, L8Mat<T> out) {
    constexpr int MOST = 32 / sizeof(T);        // vectors in registers
    const bool many = a.rows >= 1024;
    if (a.cols <= LOSS_SMALL) launch_small<T, MODE>(ctx, a, nullptr, nullptr, nullptr, x, out);
    else if (a.cols < 2048 || (many && a.cols < 4096)) launch_rows_from<T, MODE, 64, 0, 7>(ctx, a, x, out);
    else if (a.cols < 8192 || (many && a.cols < 2048 * (MOST / 2 + 1))) launch_rows_from<T, MODE, 256, 1, MOST / 2>(ctx, a, x, out);
    else launch_rows_from<T, MODE, 512, 2, MODE == ROWS_LOGP ? MOST : 2 * MOST>(ctx, a, x, out);
}

// Logits that the last-level cache (256 MiB) holds, but not beside their gradient, are still there for the second read if the gradient goes past
// it: preference loss of 4096 x 32768 16-bit entries 131 us / 106 past it, with the gradient read once behind it 285 / 275.  Below 128 MiB
// the gradient's reader finds it in the cache (64 MiB 71 / 75), far above 256 it makes no difference.  32-bit entries leave a thread as two pieces of
// 16 bytes, half of what lies between its neighbours' each: past the cache such halves cost a third more (below).
template <class T>
bool slope_past(const LossArgs& a) {
    const uint64_t bytes = a.rows * a.cols * sizeof(T);
    return sizeof(T) == 2 && bytes > (uint64_t)128 << 20 && bytes <= (uint64_t)288 << 20;
}
template <class T>
void launch_slope(zkdl_ctx* ctx, LossArgs a, const float* dlogp, const float* top, const float* log_sum, L8Mat<const T> x, L8Mat<T> out,
                  const float* losses = nullptr, uint64_t pairs = 0, float* loss = nullptr) {
    if (a.cols <= LOSS_SMALL && !losses) return launch_small<T, ROWS_SLOPE>(ctx, a, dlogp, top, log_sum, x, out);
    a.past = slope_past<T>(a);
    const uint32_t segs = (uint32_t)l8_ceil(a.cols, 2048), waves = segs >= 4 ? 4 : segs >= 2 ? 2 : 1;
    const uint64_t gx = l8_ceil(segs, waves), gy = l8_ceil(a.rows, 4 / waves);
    hipLaunchKernelGGL((k_loss_slope<T>), dim3((unsigned)(gx < 1024 ? gx : 1024), (unsigned)(gy < 4096 ? gy : 4096)), dim3(256), 0, ctx->stream, a, dlogp, top,
                       log_sum, x, out, segs, waves, losses, pairs, loss);
}

// `sets` sums over n values each, one behind the other
int launch_sum(zkdl_ctx* ctx, const float* in, uint64_t n, unsigned sets, float* out) {
    constexpr uint64_t per = 1 << 14;
    const uint64_t blocks = l8_ceil(n, per) < 4096 ? l8_ceil(n, per) : 4096;
    if (blocks <= 1) {
        hipLaunchKernelGGL((k_loss_sum<float, float>), dim3(1, sets), dim3(1024), 0, ctx->stream, in, n, n, out);
        return ZKDL_OK;
    }
    double* mid = (double*)zk_alloc_scratch(ctx, blocks * sets * 8);
    if (!mid) return ZKDL_ENOMEM;
    hipLaunchKernelGGL((k_loss_sum<float, double>), dim3((unsigned)blocks, sets), dim3(1024), 0, ctx->stream, in, n, l8_ceil(n, blocks), mid);
    hipLaunchKernelGGL((k_loss_sum<double, float>), dim3(1, sets), dim3(1024), 0, ctx->stream, mid, blocks, blocks, out);
    zk_free(ctx, mid);
    return ZKDL_OK;
}

template <class T, int MODE>
int launch_parts(zkdl_ctx* ctx, const LossArgs& a, L8Mat<const T> x) {
    const uint32_t parts = (uint32_t)l8_ceil(a.cols, 2048 * 4);
    Part* part = (Part*)zk_alloc_scratch(ctx, a.rows * parts * sizeof(Part));
    if (!part) return ZKDL_ENOMEM;
    const dim3 grid(parts < 65535 ? parts : 65535, (unsigned)(a.rows < 256 ? a.rows : 256));
    hipLaunchKernelGGL((k_loss_part<T, 4>), grid, dim3(256), 0, ctx->stream, a, x, part, parts);
    hipLaunchKernelGGL((k_loss_join<T, MODE>), dim3((unsigned)(a.rows < 65536 ? a.rows : 65536)), dim3(256), 0, ctx->stream, a, x, part, parts);
    zk_free(ctx, part);
    return ZKDL_OK;
}

bool ints_ok(int dtype) { return dtype == ZKDL_I32 || dtype == ZKDL_I64; }
// Above 2^120 a term would be there whose distance from the largest logit is beyond 32 bits.
bool good_tau(float tau) { return tau >= FLT_MIN && tau <= 0x1p120f && 1.f / tau <= FLT_MAX; }
bool rows_ok(const zkdl_mat* m) { return l8_mat_ok(m, false) && l8_is_float(m->dtype) && m->stack == 1 && (m->rows == 0 || m->cols > 0); }
bool slope_ok(const zkdl_mat* d, const zkdl_mat* x) { return !d || (l8_mat_ok(d, true) && d->dtype == x->dtype && l8_same_shape(d, x)); }

LossArgs loss_args(const zkdl_mat* x, const void* tokens, int tokens_dtype, float tau) {
    LossArgs a = {};
    a.rows = x->rows;
    a.cols = (uint32_t)x->cols;
    a.inv_tau = 1.f / tau;
    a.inv_tau64 = 1 / (double)tau;
    a.k = (float)(1.4426950408889634 / tau);
    a.times = a.inv_tau;
    a.step = LOG2E;
    a.tokens = {tokens, tokens_dtype == ZKDL_I64};
    return a;
}

template <class F>
int by_type(int dtype, F&& go) {
    switch (dtype) {
        case ZKDL_F32: return go(float{});
        case ZKDL_F16: return go(__half{});
        default: return go(bf16_t{});
    }
}

// Scratch that goes back to the context whatever happens.
struct Scratch {
    zkdl_ctx* ctx;
    float* p;
    Scratch(zkdl_ctx* c, size_t floats) : ctx(c), p((float*)zk_alloc_scratch(c, floats * 4)) {}
    ~Scratch() { zk_free(ctx, p); }
    Scratch(const Scratch&) = delete;
};

template <class T>
int policy(zkdl_ctx* ctx, LossArgs a, const zkdl_mat* logits, float* sums, const zkdl_mat* dlogits) {
    const bool fit = rows_fit<T>(a, dlogits);
    Scratch s(ctx, a.rows * (fit || !dlogits ? 3 : 6));
    if (!s.p) return ZKDL_ENOMEM;
    a.terms = s.p;
    // rows in LDS (launch_rows): 1024 x 131072 16-bit entries 134 us / 126 past the cache, with the gradient read once behind it 249 / 242; 256 x
    // 131072, which stay in the cache for that, 64 / 68; 4096 x 49152 32-bit entries 320 / 425
    a.past = sizeof(T) == 2 && a.rows * a.cols * sizeof(T) > (uint64_t)128 << 20;
    if (fit) {
        launch_rows<T, ROWS_POLICY>(ctx, a, l8_mat<const T>(logits), l8_mat<T>(dlogits));
    } else {
        if (dlogits) {
            a.dlogp = s.p + 3 * a.rows;
            a.top = s.p + 4 * a.rows;
            a.log_sum = s.p + 5 * a.rows;
            a.times = 1;
            a.step = a.k;
        }
        const int rc = launch_parts<T, ROWS_POLICY>(ctx, a, l8_mat<const T>(logits));
        if (rc != ZKDL_OK) return rc;
        if (dlogits) launch_slope<T>(ctx, a, a.dlogp, a.top, a.log_sum, l8_mat<const T>(logits), l8_mat<T>(dlogits));
    }
    return launch_sum(ctx, a.terms, a.rows, 3, sums);
}

template <class T>
int preference(zkdl_ctx* ctx, LossArgs a, const zkdl_mat* logits, const zkdl_preference* p, float* loss, float* margin, float* logp, const zkdl_mat* dlogits) {
    Scratch s(ctx, (a.rows ? a.rows : 1) * 5 + p->pairs);
    if (!s.p) return ZKDL_ENOMEM;
    a.logp = logp;
    a.logp64 = (double*)s.p;
    a.dlogp = s.p + 2 * a.rows;
    a.top = s.p + 3 * a.rows;
    a.log_sum = s.p + 4 * a.rows;
    a.times = 1;
    a.step = a.k;
    a.offsets = {p->offsets, p->offsets_dtype == ZKDL_I64};
    a.last = 2 * p->pairs;
    float* losses = s.p + 5 * a.rows;
    if (a.rows) {
        if (rows_fit<T>(a, false)) {
            launch_rows<T, ROWS_LOGP>(ctx, a, l8_mat<const T>(logits), L8Mat<T>{nullptr, 0, 0});
        } else {
            const int rc = launch_parts<T, ROWS_LOGP>(ctx, a, l8_mat<const T>(logits));
            if (rc != ZKDL_OK) return rc;
        }
    }
    PairArgs q = {a.rows, p->pairs, a.tokens, a.offsets, a.logp64, p->ref_logp, p->weight, p->form, p->average, 1.f / (float)p->pairs, p->beta, p->target,
                  p->smoothing, margin, losses, dlogits ? a.dlogp : nullptr};
    if (p->pairs) {
        // threads by the rows of a pair (8192 of them 37 us with 256 threads)
        const dim3 grid((unsigned)(p->pairs < 65536 ? p->pairs : 65536));
        if (a.rows / p->pairs < 1024) hipLaunchKernelGGL((k_loss_pair<256>), grid, dim3(256), 0, ctx->stream, q);
        else hipLaunchKernelGGL((k_loss_pair<1024>), grid, dim3(1024), 0, ctx->stream, q);
    }
    const bool few = dlogits && a.rows && p->pairs <= 4096 && a.cols > LOSS_SMALL;         // pairs whose losses one block adds up while others are at the gradient
    a.offsets.p = nullptr;          // dlogp is 0 where rows are in no sequence
    if (dlogits && a.rows)
        launch_slope<T>(ctx, a, a.dlogp, a.top, a.log_sum, l8_mat<const T>(logits), l8_mat<T>(dlogits), few ? losses : nullptr, p->pairs, loss);
    return few ? (int)ZKDL_OK : launch_sum(ctx, losses, p->pairs, 1, loss);
}

}  // namespace

extern "C" int zkdl_token_logprobs(zkdl_ctx* ctx, const zkdl_mat* logits, const void* tokens, int tokens_dtype, float temperature, float* logp, float* top,
                                   float* log_sum) try {
    if (!ctx || !rows_ok(logits) || !ints_ok(tokens_dtype) || !good_tau(temperature)) return ZKDL_EINVAL;
    if (logits->rows == 0) return ZKDL_OK;
    if (!tokens || !logp) return ZKDL_EINVAL;
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    LossArgs a = loss_args(logits, tokens, tokens_dtype, temperature);
    a.logp = logp;
    a.top = top;
    a.log_sum = log_sum;
    const int rc = by_type(logits->dtype, [&](auto t) {
        using T = decltype(t);
        if (!rows_fit<T>(a, false)) return launch_parts<T, ROWS_LOGP>(ctx, a, l8_mat<const T>(logits));
        launch_rows<T, ROWS_LOGP>(ctx, a, l8_mat<const T>(logits), L8Mat<T>{nullptr, 0, 0});
        return (int)ZKDL_OK;
    });
    if (rc != ZKDL_OK) return rc;
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}

extern "C" int zkdl_token_logprobs_backward(zkdl_ctx* ctx, const float* dlogp, const zkdl_mat* logits, const void* tokens, int tokens_dtype, const float* top,
                                            const float* log_sum, float temperature, const zkdl_mat* dlogits) try {
    if (!ctx || !rows_ok(logits) || !ints_ok(tokens_dtype) || !good_tau(temperature) || !dlogits || !slope_ok(dlogits, logits)) return ZKDL_EINVAL;
    if (logits->rows == 0) return ZKDL_OK;
    if (!dlogp || !tokens || !top || !log_sum) return ZKDL_EINVAL;
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    const LossArgs a = loss_args(logits, tokens, tokens_dtype, temperature);
    by_type(logits->dtype, [&](auto t) {
        using T = decltype(t);
        launch_slope<T>(ctx, a, dlogp, top, log_sum, l8_mat<const T>(logits), l8_mat<T>(dlogits));
        return 0;
    });
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}

extern "C" int zkdl_policy_loss(zkdl_ctx* ctx, const zkdl_mat* logits, const void* tokens, int tokens_dtype, const zkdl_policy* terms, float* sums, float* logp,
                                const zkdl_mat* dlogits) try {
    if (!ctx || !rows_ok(logits) || !ints_ok(tokens_dtype) || !terms || !good_tau(terms->temperature) || !slope_ok(dlogits, logits) || !sums) return ZKDL_EINVAL;
    if (!(terms->clip_low >= 0 && terms->clip_low <= 1) || !(terms->clip_high >= 0 && terms->clip_high <= FLT_MAX) || !std::isfinite(terms->kl) ||
        (terms->kl != 0 && logits->rows && !terms->ref_logp))
        return ZKDL_EINVAL;
    if (logits->rows && (!tokens || !terms->old_logp || !terms->advantage)) return ZKDL_EINVAL;
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    LossArgs a = loss_args(logits, tokens, tokens_dtype, terms->temperature);
    a.logp = logp;
    a.old_logp = terms->old_logp;
    a.advantage = terms->advantage;
    a.ref_logp = terms->ref_logp;
    a.weight = terms->weight;
    a.every = 1 / (double)logits->rows;
    a.low = 1 - (double)terms->clip_low;
    a.high = 1 + (double)terms->clip_high;
    a.kl = terms->kl;
    const int rc = logits->rows == 0 ? launch_sum(ctx, nullptr, 0, 3, sums)
                                     : by_type(logits->dtype, [&](auto t) { return policy<decltype(t)>(ctx, a, logits, sums, dlogits); });
    if (rc != ZKDL_OK) return rc;
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}

extern "C" int zkdl_preference_loss(zkdl_ctx* ctx, const zkdl_mat* logits, const void* tokens, int tokens_dtype, const zkdl_preference* terms, float* loss,
                                    float* margin, float* logp, const zkdl_mat* dlogits) try {
    if (!ctx || !rows_ok(logits) || !ints_ok(tokens_dtype) || !terms || !good_tau(terms->temperature) || !slope_ok(dlogits, logits) || !loss) return ZKDL_EINVAL;
    if (!ints_ok(terms->offsets_dtype) || terms->reserved != 0 || terms->form < ZKDL_PREF_LOGISTIC || terms->form > ZKDL_PREF_SQUARE || !terms->offsets ||
        !std::isfinite(terms->beta) || !std::isfinite(terms->target) || !(terms->smoothing >= 0 && terms->smoothing <= 1) ||
        (terms->smoothing != 0 && terms->form != ZKDL_PREF_LOGISTIC))
        return ZKDL_EINVAL;
    if (terms->pairs >= (uint64_t)1 << 31 || (logits->rows && !tokens)) return ZKDL_EINVAL;
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    const LossArgs a = loss_args(logits, tokens, tokens_dtype, terms->temperature);
    const int rc = by_type(logits->dtype, [&](auto t) {
        using T = decltype(t);
        return preference<T>(ctx, a, logits, terms, loss, margin, logp, dlogits);
    });
    if (rc != ZKDL_OK) return rc;
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}
