// The end of a training step: the norm of all gradients (zkdl_gradient_norm) and AdamW over many tensors (zkdl_adamw_step).
//
// Both are bound by memory: an entry of a step in 32 bits is 28 bytes moved for about 40 vector operations, with 8-bit states 14 bytes
// (16-bit gradients) for about 80, ten of them in 64 bits.  A launch takes many tensors: their addresses stand in its arguments (4 kB at most, so nothing is copied to the device
// and nothing is kept of a call), and a block finds its tensor by the number of its chunk.
#include <cfloat>
#include <cmath>
#include <algorithm>
#include <type_traits>

#include "layer8.cuh"
#include "vec8.cuh"

namespace {

// The tensor that chunk c is of: first[] rises, first[0] = 0 <= c < first[count].
template <int N>
__device__ __forceinline__ uint32_t tensor_of(const uint32_t (&first)[N], uint32_t count, uint32_t c) {
    uint32_t lo = 0, hi = count;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (first[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

// ---------------------------------------------------------------------------
// Norm: squares in 64 bits, so that no gradient in the range of 32 bits leaves it.  0.8 GB of 16-bit gradients 136 us (5.9 TB/s) and 5 for the
// join; 34 MB in 32 bits 5.9 us and 2.3.
// ---------------------------------------------------------------------------
constexpr uint32_t NORM_TENSORS = 160, NORM_ITEMS = 4, NORM_CHUNK = 256 * 8 * NORM_ITEMS, NORM_BLOCKS = 2048;
struct NormArgs {
    const void* p[NORM_TENSORS];
    uint64_t n[NORM_TENSORS];
    uint32_t first[NORM_TENSORS + 1];
    uint8_t dtype[NORM_TENSORS];
    uint32_t count;
    double* part;       // a sum for each block
};
static_assert(sizeof(NormArgs) <= 4096 - 256, "a launch's arguments");

__device__ __forceinline__ double block_sum(double x, double* s) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0;
    for (uint32_t i = 0; i < blockDim.x / 64; ++i) x += s[i];
    return x;
}

template <class T>
__device__ __forceinline__ void add_squares(const T* p, uint64_t n, uint64_t at, double (&sum)[2]) {
    float f[NORM_ITEMS][8];
    if (at + NORM_CHUNK <= n) {
        L8Vec<T> v[NORM_ITEMS];
#pragma unroll
        for (int k = 0; k < (int)NORM_ITEMS; ++k) v[k] = l8_raw(p + at + (k * 256 + threadIdx.x) * 8);
#pragma unroll
        for (int k = 0; k < (int)NORM_ITEMS; ++k) l8_floats(v[k], f[k]);
    } else {
#pragma unroll
        for (int k = 0; k < (int)NORM_ITEMS; ++k) {
            const uint64_t j = at + (k * 256 + threadIdx.x) * 8;
            const int left = j < n ? (int)min((uint64_t)8, n - j) : 0;
            l8_load(p + (left ? j : 0), left, f[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < (int)NORM_ITEMS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double g = f[k][i];
            sum[i & 1] = fma(g, g, sum[i & 1]);
        }
}
__global__ __launch_bounds__(256) void k_norm_part(NormArgs a) {
    __shared__ double s[4];
    double sum[2] = {0, 0};
    for (uint32_t c = blockIdx.x; c < a.first[a.count]; c += gridDim.x) {
        const uint32_t i = tensor_of(a.first, a.count, c);
        const uint64_t at = (uint64_t)(c - a.first[i]) * NORM_CHUNK;
        switch (a.dtype[i]) {
            case L8_F32: add_squares((const float*)a.p[i], a.n[i], at, sum); break;
            case L8_F16: add_squares((const __half*)a.p[i], a.n[i], at, sum); break;
            default: add_squares((const bf16_t*)a.p[i], a.n[i], at, sum);
        }
    }
    const double x = block_sum(sum[0] + sum[1], s);
    if (threadIdx.x == 0) a.part[blockIdx.x] = x;
}
__global__ __launch_bounds__(1024) void k_norm_join(const double* part, uint64_t n, float limit, float* norm, float* factor) {
    __shared__ double s[16];
    double x = 0;
    for (uint64_t i = threadIdx.x; i < n; i += 1024) x += part[i];
    x = sqrt(block_sum(x, s));
    if (threadIdx.x == 0) {
        const float f = (float)x;
        *norm = f;
        if (factor) *factor = !(f < __builtin_huge_valf()) ? __builtin_nanf("") : x > (double)limit ? (float)((double)limit / x) : 1.f;
    }
}

// ---------------------------------------------------------------------------
// AdamW.  2^28 entries (MI355X, a copy moves 5.2 TB/s): all in 32 bits 1375 us (5.5 TB/s); 8-bit states with 32-bit gradients 775 us (5.5), with 16-bit
// gradients 685 us (5.5), all parameters and gradients in 16 bits 540 us (5.0: here the vector operations show).  The moments are taken
// in 64 bits because the codes' rounding has to come out the same for whoever computes the step.
// ---------------------------------------------------------------------------
constexpr uint32_t ADAM_ITEMS = 2, ADAM_CHUNK = 256 * 8 * ADAM_ITEMS, ADAM_BLOCK8 = 256;
struct AdamTensor {
    void* param;
    const void* grad;
    void *m, *v;
    uint64_t n;
};
struct AdamTensor8 : AdamTensor {
    uint8_t *m_scale, *v_scale;
    float *m_value, *v_value;
    uint32_t number;        // of the tensor in the call: its random bits
};
// BITS: of the states
template <int BITS>
struct AdamArgs {
    typedef std::conditional_t<BITS == 32, AdamTensor, AdamTensor8> Tensor;
    static constexpr uint32_t TENSORS = BITS == 32 ? 80 : 40;
    Tensor t[TENSORS];
    uint32_t first[TENSORS + 1];
    uint32_t count, seed_lo, seed_hi, step;
    double lr, decay, beta1, beta2, root2, scale;       // root2: (1 - beta2)^(1/2); scale: of rate, root and eps
    const int64_t* step_ptr;
    const float *lr_ptr, *factor;
    float eps;
    float rate, root, keep;     // scale lr / (1 - beta1^t), scale (1 - beta2^t)^(-1/2), 1 - lr decay
};
static_assert(sizeof(AdamArgs<32>) <= 4096 - 256 && sizeof(AdamArgs<8>) <= 4096 - 256, "a launch's arguments");

// What the step's number and the learning rate give: on the host, or, where they are read from device memory, in every block.
struct AdamRates {
    float rate, root, keep;
};
static __host__ __device__ inline double power_of(double b, uint32_t t) {       // by squaring: the same on either side
    double r = 1;
    for (; t; t >>= 1) {
        if (t & 1) r = r * b;
        b = b * b;
    }
    return r;
}
static __host__ __device__ inline AdamRates adam_rates(double lr, double decay, double beta1, double beta2, double scale, uint32_t t) {
    AdamRates r;
    r.rate = (float)(scale * lr / (1 - power_of(beta1, t)));
    r.root = (float)(scale / sqrt(1 - power_of(beta2, t)));
    r.keep = (float)fma(-lr, decay, 1.0);       // (rounded once, on either side)
    return r;
}

__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x9E3779B1u;
    x ^= x >> 15;
    x *= 0x85A308D3u;
    return x ^ x >> 16;
}

// 8-bit floats: 3 mantissa bits and LOG exponent bits, the largest of which is the binade of scale byte e.
template <int LOG>
struct Float8 {
    static constexpr uint32_t LAST = (1u << LOG) - 1;
    // of a block whose largest magnitude is `top` (the bits of a float)
    static __device__ __forceinline__ uint32_t scale(uint32_t top) {
        const uint32_t e = max(40u, (top + 0xFFFFFu) >> 23);
        return e > 254 ? 255u : e;
    }
    // A code's bits are those of a float's exponent and mantissa: that float (subnormal where the code's exponent is 0) times 2^(e - LAST) is its value.
    // NaN where the block holds none.
    static __device__ __forceinline__ double unit(uint32_t e) {
        const double u = __hiloint2double((int)((1023 - LAST + e) << 20), 0);
        return e == 255 ? (double)__builtin_nanf("") : u;
    }
    // code of the magnitude with the bits u; r: 16 random bits; WHOLE: where the code's exponent is known not to be 0
    static __device__ __forceinline__ uint32_t smallest(uint32_t e) { return (e - LAST + 1) << 23; }
    template <bool WHOLE>
    static __device__ __forceinline__ uint32_t code(uint32_t u, uint32_t e, uint32_t r) {
        const uint32_t base = (e - LAST) << 23;
        const uint32_t whole = (u - base + (r << 4 | 8)) >> 20;
        if (WHOLE) return whole;
        const float place = __uint_as_float(u) * __uint_as_float((254 - (e - LAST - 2)) << 23);
        const uint32_t part = (uint32_t)(int)(place + fmaf((float)r, 0x1p-16f, 0x1p-17f));
        return u >= smallest(e) ? whole : part;
    }
};
typedef Float8<4> M8;
typedef Float8<5> V8;
// Entry q of eight codes as the float that a code's bits are: moved to the sign, the exponent's last bits and the mantissa's first
__device__ __forceinline__ float m_float(const uint32_t (&w)[2], int q) {
    const uint32_t high = w[q / 4] << (24 - 8 * (q % 4));
    return __uint_as_float((uint32_t)((int32_t)high >> 4) & 0x87F00000u);
}
__device__ __forceinline__ float v_float(const uint32_t (&w)[2], int q) {
    const uint32_t x = q % 4 == 3 ? w[q / 4] >> 4 : w[q / 4] << (20 - 8 * (q % 4) & 31);
    return __uint_as_float(x & 0x0FF00000u);
}

struct __attribute__((packed, aligned(1))) Codes8 {
    uint32_t w[2];
};
__device__ __forceinline__ Codes8 load_codes(const uint8_t* p, int n) {
    Codes8 c = {{0, 0}};
    if (n >= 8) return *(const Codes8*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) c.w[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
    return c;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int n, const Codes8& c) {
    if (n >= 8) {
        *(Codes8*)p = c;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = (uint8_t)(c.w[i / 4] >> (8 * (i % 4)));
}
// Codes of eight entries, with their random bits: the upper 16 of m, the lower ones of v.
template <class F, bool WHOLE>
__device__ __forceinline__ void put_codes(const float (&x)[8], uint32_t e, const uint32_t (&r)[8], Codes8& to) {
    to = {{0, 0}};
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const uint32_t u = l8_mag(x[q]);
        uint32_t c;
        if constexpr (F::LAST == M8::LAST) c = F::template code<WHOLE>(u, e, r[q] >> 16) | (__float_as_uint(x[q]) >> 24 & 128u);
        else c = WHOLE ? F::template code<WHOLE>(u, e, r[q] & 0xFFFFu) : max(F::template code<WHOLE>(u, e, r[q] & 0xFFFFu), min(u, 1u));       // a second moment that is there does not vanish
        to.w[q / 4] |= c << (8 * (q % 4));
    }
}
// over the 32 lanes that share a block of 256 entries
__device__ __forceinline__ uint32_t half_wave_max(uint32_t x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, d, 64));
    return x;
}

// 1 ulp.  The instruction takes what is below 2^-126 for 0, which leaves nothing to divide by where eps is as small as such a root: SMALL.
template <bool SMALL>
__device__ __forceinline__ float root_of(float v) {
    if (!SMALL) return __builtin_amdgcn_sqrtf(v);
    const bool small = v < FLT_MIN;
    const float r = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v);
    return small ? r * 0x1p-32f : r;
}
// BITS: of the states.  A thread has eight adjacent entries of every 2048; 32 threads have a block of an 8-bit state.  FULL: the tensor does not end in
// the chunk, so that no load waits for a branch.  SMALL: roots of subnormal numbers (2 to 3 % of the time where they are not asked for).
struct AdamJob {
    double b1, b2, c1, c2;      // m <- b1 m + c1 grad, v <- b2 v + (c2 grad)^2: the gradients' factor is in c1 and c2
    AdamRates rates;
    float eps;
    uint32_t key;
    bool go;
};
template <bool FULL, class T>
__device__ __forceinline__ Raw8<T> load_raw(const T* p, int n) {
    if constexpr (FULL) return load8(p);
    float f[8];
    Raw8<T> v;
    l8_load(p, n, f);
    pack8(f, v);        // (exactly: they came from T)
    return v;
}
template <bool FULL, class T>
__device__ __forceinline__ void store_entries(T* p, int n, const float (&f)[8]) {
    if constexpr (FULL) store8(p, f);
    else l8_store(p, n, f);
}
template <class P, class G, int BITS, bool FULL, bool SMALL>
__device__ __forceinline__ void adam_chunk(const AdamJob& a, const typename AdamArgs<BITS>::Tensor& t, uint64_t at) {
    P* const param = (P*)t.param;
    const G* const grad = (const G*)t.grad;
    Raw8<P> praw[ADAM_ITEMS];
    Raw8<G> graw[ADAM_ITEMS];
    Raw8<float> mraw[BITS == 32 ? ADAM_ITEMS : 1], vraw[BITS == 32 ? ADAM_ITEMS : 1];
    Codes8 mcode[ADAM_ITEMS], vcode[ADAM_ITEMS];
    uint32_t mscale[ADAM_ITEMS], vscale[ADAM_ITEMS];
    int n[ADAM_ITEMS];
    uint64_t j[ADAM_ITEMS];
#pragma unroll
    for (int k = 0; k < (int)ADAM_ITEMS; ++k) {
        j[k] = at + k * 2048;
        n[k] = FULL ? 8 : j[k] < t.n ? (int)min((uint64_t)8, t.n - j[k]) : 0;
        if (!n[k]) j[k] = 0;
        if constexpr (BITS == 32) {
            mraw[k] = load_raw<FULL>((const float*)t.m + j[k], n[k]);
            vraw[k] = load_raw<FULL>((const float*)t.v + j[k], n[k]);
        } else {
            mscale[k] = n[k] ? t.m_scale[j[k] / ADAM_BLOCK8] : 0;
            vscale[k] = n[k] ? t.v_scale[j[k] / ADAM_BLOCK8] : 0;
            mcode[k] = load_codes((const uint8_t*)t.m + j[k], n[k]);
            vcode[k] = load_codes((const uint8_t*)t.v + j[k], n[k]);
        }
        praw[k] = load_raw<FULL>(param + j[k], n[k]);
        graw[k] = load_raw<FULL>(grad + j[k], n[k]);
    }
#pragma unroll
    for (int k = 0; k < (int)ADAM_ITEMS; ++k) {
        float p[8], g[8], m[8], v[8];
        double b1 = a.b1, b2 = a.b2;
        uint32_t em = 0, ev = 0;
        if constexpr (BITS == 32) {
            floats8(mraw[k], m);
            floats8(vraw[k], v);
        } else {
            em = max(40u, mscale[k]);
            ev = max(40u, vscale[k]);
            b1 *= M8::unit(em);
            b2 *= V8::unit(ev);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                m[q] = m_float(mcode[k].w, q);
                v[q] = v_float(vcode[k].w, q);
            }
        }
        if (a.go) {
            floats8(praw[k], p);
            floats8(graw[k], g);
            uint32_t tm = 0, tv = 0;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const double d = (double)g[q], d2 = a.c2 * d;
                m[q] = (float)fma(a.c1, d, b1 * (double)m[q]);
                v[q] = (float)fma(d2, d2, b2 * (double)v[q]);
                const float below = fmaf(root_of<SMALL>(v[q]), a.rates.root, a.eps);
                p[q] = fmaf(-a.rates.rate * m[q], __builtin_amdgcn_rcpf(below), p[q] * a.rates.keep);
                if (BITS == 8 && (FULL || q < n[k])) {
                    tm = max(tm, l8_mag(m[q]));
                    tv = max(tv, l8_mag(v[q]));
                }
            }
            store_entries<FULL>(param + j[k], n[k], p);
            if constexpr (BITS == 32) {
                store_entries<FULL>((float*)t.m + j[k], n[k], m);
                store_entries<FULL>((float*)t.v + j[k], n[k], v);
            } else {
                em = M8::scale(half_wave_max(tm));
                ev = V8::scale(half_wave_max(tv));
                const uint64_t block = j[k] / ADAM_BLOCK8;
                const uint32_t first = mix(a.key ^ (uint32_t)block) + (uint32_t)(j[k] % ADAM_BLOCK8) * 0x9E3779B1u;
                uint32_t lm = ~0u, lv = ~0u, r[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    r[q] = mix(first + (uint32_t)q * 0x9E3779B1u);
                    lm = min(lm, l8_mag(m[q]));
                    lv = min(lv, l8_mag(v[q]));
                }
                // codes with exponent 0 cost half as much again and are rare (below 2^-14 or 2^-30 of the block's largest): a wave without any goes without
                if (__any(lm < M8::smallest(em))) put_codes<M8, false>(m, em, r, mcode[k]);
                else put_codes<M8, true>(m, em, r, mcode[k]);
                if (__any(lv < V8::smallest(ev))) put_codes<V8, false>(v, ev, r, vcode[k]);
                else put_codes<V8, true>(v, ev, r, vcode[k]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    mcode[k].w[h] = em == 255 ? 0 : mcode[k].w[h];
                    vcode[k].w[h] = ev == 255 ? 0 : vcode[k].w[h];
                }
                store_codes((uint8_t*)t.m + j[k], n[k], mcode[k]);
                store_codes((uint8_t*)t.v + j[k], n[k], vcode[k]);
                if ((threadIdx.x & 31) == 0 && n[k]) {
                    t.m_scale[block] = (uint8_t)em;
                    t.v_scale[block] = (uint8_t)ev;
                }
            }
        }
        if constexpr (BITS == 8) {
            if (t.m_value) {
                const double u = M8::unit(em);
#pragma unroll
                for (int q = 0; q < 8; ++q) m[q] = (float)(u * (double)m_float(mcode[k].w, q));
                store_entries<FULL>(t.m_value + j[k], n[k], m);
            }
            if (t.v_value) {
                const double u = V8::unit(ev);
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = (float)(u * (double)v_float(vcode[k].w, q));
                store_entries<FULL>(t.v_value + j[k], n[k], v);
            }
        }
    }
}

// BITS: of the states; SMALL: as in adam_chunk
template <class P, class G, int BITS, bool SMALL>
__global__ __launch_bounds__(256) void k_adamw(AdamArgs<BITS> a) {
    __shared__ AdamRates s_rates;
    const uint32_t i = tensor_of(a.first, a.count, blockIdx.x);
    const auto& t = a.t[i];
    uint32_t step = a.step;
    AdamRates rates = {a.rate, a.root, a.keep};
    bool go = true;
    if (a.step_ptr) {
        const int64_t v = *a.step_ptr;
        go = v >= 1 && v < (int64_t)1 << 31;
        step = go ? (uint32_t)v : 1;
    }
    if (a.step_ptr || a.lr_ptr) {
        if (threadIdx.x == 0) s_rates = adam_rates(a.lr_ptr ? (double)*a.lr_ptr : a.lr, a.decay, a.beta1, a.beta2, a.scale, step);
        __syncthreads();
        rates = s_rates;
    }
    double factor = 1;
    if (a.factor) {
        const float f = *a.factor;
        go = go && fabsf(f) < __builtin_huge_valf();
        factor = f;
    }
    if (BITS == 32 && !go) return;
    uint32_t key = 0;
    if constexpr (BITS == 8) key = mix(mix(mix(mix(a.seed_lo) ^ a.seed_hi) ^ step) ^ t.number);
    const uint64_t at = (uint64_t)(blockIdx.x - a.first[i]) * ADAM_CHUNK + threadIdx.x * 8;
    const AdamJob job = {a.beta1, a.beta2, (1 - a.beta1) * factor, a.root2 * factor, rates, a.eps, key, go};
    if ((uint64_t)(blockIdx.x - a.first[i] + 1) * ADAM_CHUNK <= t.n) adam_chunk<P, G, BITS, true, SMALL>(job, t, at);
    else adam_chunk<P, G, BITS, false, SMALL>(job, t, at);
}

template <class F>
void by_type(int dtype, F&& go) {
    switch (dtype) {
        case ZKDL_F32: go(float{}); break;
        case ZKDL_F16: go(__half{}); break;
        default: go(bf16_t{});
    }
}
uint64_t item_bytes(int dtype) { return dtype == ZKDL_F32 ? 4 : 2; }

// Memory that a call reads or writes: nothing that is written may overlap anything else.
struct Span {
    uint64_t lo, hi;
    bool out;
    bool operator<(const Span& o) const { return lo < o.lo; }
};
// runs: where the spans of one kind begin, and their end.  Tensors of a kind mostly lie in the order in which they were made, so the runs are
// merged: 8000 spans of 1000 tensors would take longer to sort than their update.
bool spans_apart(std::vector<Span>& s, std::vector<size_t> runs) {
    for (size_t i = 0; i + 1 < runs.size(); ++i)
        if (!std::is_sorted(s.begin() + runs[i], s.begin() + runs[i + 1])) std::sort(s.begin() + runs[i], s.begin() + runs[i + 1]);
    while (runs.size() > 2) {
        std::vector<size_t> left;
        for (size_t i = 0; i + 1 < runs.size(); i += 2) {
            left.push_back(runs[i]);
            if (i + 2 < runs.size()) std::inplace_merge(s.begin() + runs[i], s.begin() + runs[i + 1], s.begin() + runs[i + 2]);
        }
        left.push_back(runs.back());
        runs.swap(left);
    }
    uint64_t any = 0, outs = 0;      // where what came before ends
    for (const Span& x : s) {
        if (x.lo < (x.out ? any : outs)) return false;
        any = std::max(any, x.hi);
        if (x.out) outs = std::max(outs, x.hi);
    }
    return true;
}

template <int BITS>
void adamw(zkdl_ctx* ctx, const zkdl_adamw_tensor* tensors, size_t count, const zkdl_adamw* how) {
    AdamArgs<BITS> a = {};
    a.seed_lo = (uint32_t)how->seed;
    a.seed_hi = (uint32_t)(how->seed >> 32);
    a.step = how->step_ptr ? 1 : (uint32_t)how->step;
    a.lr = how->lr_ptr ? 0 : how->lr;
    a.decay = how->decay;
    a.beta1 = how->beta1;
    a.beta2 = how->beta2;
    a.root2 = std::sqrt(1 - how->beta2);
    a.step_ptr = how->step_ptr;
    a.lr_ptr = how->lr_ptr;
    a.factor = how->factor;
    a.scale = how->eps < 0x1p64 ? 1 : 0x1p-64;      // the reciprocal of what is above 2^126 would be 0
    a.eps = (float)(how->eps * a.scale);
    const AdamRates rates = adam_rates(a.lr, a.decay, a.beta1, a.beta2, a.scale, a.step);
    a.rate = rates.rate;
    a.root = rates.root;
    a.keep = rates.keep;
    // a subnormal v, below 2^-126, divided by 1 - beta2^t, which is 1 - beta2 at least, has a root below 2^-26 of eps: half a unit of 32 bits is not reached
    const bool small = how->eps * a.root2 < 0x1p-37;
    // tensors of the same types share launches
    const int types[3] = {ZKDL_F32, ZKDL_F16, ZKDL_BF16};
    uint32_t there = 0;
    const auto kind = [&](const zkdl_adamw_tensor& t) {
        const auto at = [&](int dtype) { return dtype == ZKDL_F32 ? 0 : dtype == ZKDL_F16 ? 1 : 2; };
        return 3 * at(t.param_dtype) + at(t.grad_dtype);
    };
    for (size_t i = 0; i < count; ++i) there |= 1u << kind(tensors[i]);
    for (int k = 0; k < 9; ++k) {
        if (!(there >> k & 1)) continue;
        const auto flush = [&] {
            if (!a.count) return;
            by_type(types[k / 3], [&](auto p) {
                by_type(types[k % 3], [&](auto g) {
                    const auto kernel = small ? k_adamw<decltype(p), decltype(g), BITS, true> : k_adamw<decltype(p), decltype(g), BITS, false>;
                    hipLaunchKernelGGL(kernel, dim3(a.first[a.count]), dim3(256), 0, ctx->stream, a);
                });
            });
            a.count = 0;
        };
        for (size_t i = 0; i < count; ++i) {
            const zkdl_adamw_tensor& t = tensors[i];
            if (kind(t) != k || !t.n) continue;
            const uint64_t chunks = l8_ceil(t.n, ADAM_CHUNK);
            if (a.count == a.TENSORS || (a.count && a.first[a.count] + chunks >= (uint64_t)1 << 23)) flush();
            auto& to = a.t[a.count];
            to.param = t.param;
            to.grad = t.grad;
            to.m = t.m;
            to.v = t.v;
            to.n = t.n;
            if constexpr (BITS == 8) {
                to.m_scale = t.m_scale;
                to.v_scale = t.v_scale;
                to.m_value = t.m_value;
                to.v_value = t.v_value;
                to.number = (uint32_t)i;
            }
            a.first[a.count + 1] = a.first[a.count] + (uint32_t)chunks;
            ++a.count;
        }
        flush();
    }
}

}  // namespace

extern "C" int zkdl_gradient_norm(zkdl_ctx* ctx, const zkdl_vec* tensors, size_t count, float limit, float* norm, float* factor) try {
    if (!ctx || (count && !tensors) || !norm || !(limit > 0)) return ZKDL_EINVAL;
    uint64_t total = 0;
    for (size_t i = 0; i < count; ++i) {
        const zkdl_vec& t = tensors[i];
        if (!l8_is_float(t.dtype) || t.reserved != 0 || (t.n && !t.data) || t.n >= (uint64_t)1 << 40) return ZKDL_EINVAL;
        if (l8_ceil(t.n, NORM_CHUNK) >= (uint64_t)1 << 31) return ZKDL_ETOOBIG;
        total += l8_ceil(t.n, NORM_CHUNK);
    }
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    // blocks of all launches: each has NORM_BLOCKS at most
    const uint64_t most = (l8_ceil(count, NORM_TENSORS) + 2 * l8_ceil(total, (uint64_t)1 << 31) + 1) * NORM_BLOCKS;
    double* part = (double*)zk_alloc_scratch(ctx, std::min(most, total + 1) * 8);
    if (!part) return ZKDL_ENOMEM;
    NormArgs a;
    a.count = 0;
    a.first[0] = 0;
    uint64_t blocks = 0;
    const auto flush = [&] {
        if (!a.count) return;
        const uint32_t grid = std::min(a.first[a.count], NORM_BLOCKS);
        a.part = part + blocks;
        hipLaunchKernelGGL(k_norm_part, dim3(grid), dim3(256), 0, ctx->stream, a);
        blocks += grid;
        a.count = 0;
    };
    for (size_t i = 0; i < count; ++i) {
        const zkdl_vec& t = tensors[i];
        if (!t.n) continue;
        const uint64_t chunks = l8_ceil(t.n, NORM_CHUNK);
        if (a.count == NORM_TENSORS || (a.count && a.first[a.count] + chunks >= (uint64_t)1 << 31)) flush();
        a.p[a.count] = t.data;
        a.n[a.count] = t.n;
        a.dtype[a.count] = t.dtype == ZKDL_F32 ? L8_F32 : t.dtype == ZKDL_F16 ? L8_F16 : L8_BF16;
        a.first[a.count + 1] = a.first[a.count] + (uint32_t)chunks;
        ++a.count;
    }
    flush();
    hipLaunchKernelGGL(k_norm_join, dim3(1), dim3(1024), 0, ctx->stream, part, blocks, limit, norm, factor);
    zk_free(ctx, part);
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}

extern "C" int zkdl_adamw_step(zkdl_ctx* ctx, const zkdl_adamw_tensor* tensors, size_t count, const zkdl_adamw* how) try {
    if (!ctx || (count && !tensors) || !how || how->reserved != 0 || (how->bits != 32 && how->bits != 8)) return ZKDL_EINVAL;
    if (!(how->beta1 >= 0 && how->beta1 < 1) || !(how->beta2 >= 0 && how->beta2 < 1) || !((float)how->eps >= FLT_MIN && (float)how->eps <= FLT_MAX) ||
        !std::isfinite(how->decay) || (!how->lr_ptr && !std::isfinite(how->lr)) || (!how->step_ptr && (how->step < 1 || how->step >= (int64_t)1 << 31)))
        return ZKDL_EINVAL;
    if (count >= (size_t)1 << 31) return ZKDL_EINVAL;
    for (size_t i = 0; i < count; ++i) {
        const zkdl_adamw_tensor& t = tensors[i];
        if (!l8_is_float(t.param_dtype) || !l8_is_float(t.grad_dtype) || t.n >= (uint64_t)1 << 40) return ZKDL_EINVAL;
        if (how->bits == 32 && (t.m_value || t.v_value)) return ZKDL_EINVAL;
        if (!t.n) continue;
        if (!t.param || !t.grad || !t.m || !t.v || (how->bits == 8 && (!t.m_scale || !t.v_scale))) return ZKDL_EINVAL;
        if (l8_ceil(t.n, ADAM_CHUNK) >= (uint64_t)1 << 23) return ZKDL_ETOOBIG;      // a launch's threads are counted in 32 bits
    }
    std::vector<Span> spans;
    std::vector<size_t> runs;
    spans.reserve((how->bits == 8 ? 8 : 4) * count + 3);
    const auto span = [&](const void* p, uint64_t bytes, bool out) {
        if (bytes && p) spans.push_back({(uint64_t)p, (uint64_t)p + bytes, out});
    };
    const auto run = [&](auto of) {
        runs.push_back(spans.size());
        for (size_t i = 0; i < count; ++i) of(tensors[i]);
    };
    typedef const zkdl_adamw_tensor& Tensor;
    const uint64_t state = how->bits == 32 ? 4 : 1;
    run([&](Tensor t) { span(t.param, t.n * item_bytes(t.param_dtype), true); });
    run([&](Tensor t) { span(t.grad, t.n * item_bytes(t.grad_dtype), false); });
    run([&](Tensor t) { span(t.m, t.n * state, true); });
    run([&](Tensor t) { span(t.v, t.n * state, true); });
    if (how->bits == 8) {
        run([&](Tensor t) { span(t.m_scale, l8_ceil(t.n, ADAM_BLOCK8), true); });
        run([&](Tensor t) { span(t.v_scale, l8_ceil(t.n, ADAM_BLOCK8), true); });
        run([&](Tensor t) { span(t.m_value, t.n * 4, true); });
        run([&](Tensor t) { span(t.v_value, t.n * 4, true); });
    }
    runs.push_back(spans.size());
    span(how->step_ptr, 8, false);
    span(how->lr_ptr, 4, false);
    span(how->factor, 4, false);
    runs.push_back(spans.size());
    if (!spans_apart(spans, std::move(runs))) return ZKDL_EINVAL;
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    if (how->bits == 32) adamw<32>(ctx, tensors, count, how);
    else adamw<8>(ctx, tensors, count, how);
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}
