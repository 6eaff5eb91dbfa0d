// What the kernels of the 8-bit layers (k_layer8.hip, k_matmul8.hip) share: matrices as kernels see them, items of the three
// floating types, reductions over a wave.
#pragma once
#include <hip/hip_fp16.h>

#include "zkdl_internal.h"

enum L8Type { L8_F32 = 0, L8_F16 = 1, L8_BF16 = 2 };
struct bf16_t {
    uint16_t v;
};

// A stack of matrices: item (s, i, j) at p + s * ss + i * rs + j.
template <class T>
struct L8Mat {
    T* p;
    uint64_t rs, ss;
};
template <class T>
static inline L8Mat<T> l8_mat(const zkdl_mat* m) {
    L8Mat<T> r = {nullptr, 0, 0};
    if (m) {
        r.p = (T*)m->data;
        r.rs = m->row_stride;
        r.ss = m->stack_stride;
    }
    return r;
}

static __device__ __forceinline__ float l8_f32(float x) { return x; }
static __device__ __forceinline__ float l8_f32(__half x) { return __half2float(x); }
static __device__ __forceinline__ float l8_f32(bf16_t x) { return __uint_as_float((uint32_t)x.v << 16); }
// One rounding, to nearest even, where a result leaves for memory.
static __device__ __forceinline__ void l8_put(float x, float& o) { o = x; }
static __device__ __forceinline__ void l8_put(float x, __half& o) {
    asm("" : "+v"(x));      // a 32-bit value of its own: a product in front would be rounded once, to 16 bits, otherwise
    o = __float2half(x);
}
static __device__ __forceinline__ void l8_put(float x, bf16_t& o) { o.v = __builtin_bit_cast(uint16_t, (__bf16)x); }

// Eight adjacent items, at any address: the memory system takes 16 bytes at once also where they are not aligned.
template <class T>
struct __attribute__((packed, aligned(1))) L8Vec {
    T v[8];
};
// f[0..8) = p[0..n), zeros behind
template <class T>
static __device__ __forceinline__ void l8_load(const T* p, int n, float (&f)[8]) {
    if (n >= 8) {
        const L8Vec<T> x = *(const L8Vec<T>*)p;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = l8_f32(x.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < n ? l8_f32(p[i]) : 0.f;
    }
}
// The eight items that a thread at column j of a row of `cols` >= 8 looks at: those from j on, or the row's last eight, of which
// the first `dup` belong to another thread (all of them where j is behind the end).  So every load takes eight items, none waits for
// a branch, and what two threads write twice is the same.
struct L8At {
    uint32_t start, dup;
    bool live;
};
static __device__ __forceinline__ L8At l8_at(uint32_t j, uint32_t cols) {
    L8At r;
    r.start = min(j, cols - 8);
    r.dup = j - r.start;
    r.live = j < cols;
    return r;
}
template <class T>
static __device__ __forceinline__ L8Vec<T> l8_raw(const T* p) { return *(const L8Vec<T>*)p; }
template <class T>
static __device__ __forceinline__ void l8_floats(const L8Vec<T>& x, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = l8_f32(x.v[i]);
}

template <class T>
static __device__ __forceinline__ void l8_store(T* p, int n, const float (&f)[8]) {
    L8Vec<T> x;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        T o;
        l8_put(f[i], o);
        x.v[i] = o;
    }
    if (n >= 8) {
        *(L8Vec<T>*)p = x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = x.v[i];
    }
}
struct __attribute__((packed, aligned(1))) L8Bytes {
    uint32_t lo, hi;
};
static __device__ __forceinline__ void l8_store_q(int8_t* p, int n, const int (&q)[8]) {
    L8Bytes w;
    w.lo = (q[0] & 255) | (q[1] & 255) << 8 | (q[2] & 255) << 16 | (uint32_t)q[3] << 24;
    w.hi = (q[4] & 255) | (q[5] & 255) << 8 | (q[6] & 255) << 16 | (uint32_t)q[7] << 24;
    if (n >= 8) {
        *(L8Bytes*)p = w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (int8_t)q[i];
    }
}

// |x| as a number whose order as an integer is that of the magnitudes, infinity above all finite ones and NaN above that.
static __device__ __forceinline__ uint32_t l8_mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }
constexpr uint32_t L8_INF = 0x7f800000u;

// How the values of a row (column) whose largest magnitude is `top` become 8-bit integers.
struct L8Quant {
    float pre, inv;     // q = rint((v * pre) * inv)
    bool finite;
};
static __device__ __forceinline__ L8Quant l8_quant(uint32_t top) {
    L8Quant r;
    r.finite = top < L8_INF;
    const float a = __uint_as_float(top);
    // 127 / a overflows for the smallest a; times 2^100 both stay normal, exactly
    r.pre = a < 0x1p-100f ? 0x1p100f : 1.f;
    r.inv = top == 0 || !r.finite ? 0.f : 127.f / (a * r.pre);
    return r;
}
static __device__ __forceinline__ int l8_round(float v, const L8Quant& c) {
    const float q = rintf(v * c.pre * c.inv);
    return (int)(c.finite ? q : 0.f);      // (a choice of values, not a branch for each entry)
}

static __device__ __forceinline__ float l8_wave_sum(float x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}
static __device__ __forceinline__ uint32_t l8_wave_max(uint32_t x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, d, 64));
    return x;
}

typedef int v4i __attribute__((ext_vector_type(4)));
struct __attribute__((packed, aligned(1))) M8Bytes {
    uint32_t v[4];
};
// 16 bytes of a stored matrix from (r, c) on, zeros outside rows x cols
static __device__ __forceinline__ v4i m8_fetch(const int8_t* p, uint64_t rs, uint32_t r, uint32_t rows, uint32_t c, uint32_t cols) {
    v4i x = {0, 0, 0, 0};
    if (r < rows && c < cols) {
        const int8_t* at = p + r * rs + c;
        if (cols - c >= 16) {
            const M8Bytes y = *(const M8Bytes*)at;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (int)y.v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (c + i < cols) x[i / 4] |= (int)((uint32_t)(uint8_t)at[i] << (8 * (i % 4)));
        }
    }
    return x;
}

// Rows of whole 16 bytes at multiples of 16, zeros behind the last column: what k_m8_tile can fetch of any matrix.
struct M8PackArgs {
    const int8_t* p;
    uint64_t rs, ss;
    uint64_t rows, stack, pitch;
    uint32_t cols;
    int8_t* out;
};
static __device__ __forceinline__ void m8_pack(const M8PackArgs& a, uint32_t block, uint32_t blocks) {
    const uint64_t pieces = a.pitch / 16, n = a.stack * a.rows * pieces;
    for (uint64_t i = block * 256ull + threadIdx.x; i < n; i += blocks * 256ull) {
        const uint64_t row = i / pieces, c = i % pieces * 16;
        *(v4i*)(a.out + i * 16) = m8_fetch(a.p + row / a.rows * a.ss, a.rs, (uint32_t)(row % a.rows), (uint32_t)a.rows, (uint32_t)c, a.cols);
    }
}

// ---- host side -------------------------------------------------------------------
// The context's device is the current one while this lives: its stream may be the device's default one.
struct L8Device {
    int before = -1;
    hipError_t err;
    explicit L8Device(const zkdl_ctx* ctx) {
        int now = -1;
        err = hipGetDevice(&now);
        if (err == hipSuccess && now != ctx->device) {
            err = hipSetDevice(ctx->device);
            if (err == hipSuccess) before = now;
        }
    }
    ~L8Device() {
        if (before >= 0) (void)hipSetDevice(before);
    }
};
static inline bool l8_is_float(int dtype) { return dtype == ZKDL_F32 || dtype == ZKDL_F16 || dtype == ZKDL_BF16; }
// A matrix that a kernel can address; an output's items are all different ones.
static inline bool l8_mat_ok(const zkdl_mat* m, bool output) {
    if (!m || m->reserved != 0) return false;
    const uint64_t lim = (uint64_t)1 << 31, far = (uint64_t)1 << 40;
    if (m->rows >= lim || m->cols >= lim || m->stack >= lim) return false;
    if (m->rows == 0 || m->cols == 0 || m->stack == 0) return true;
    if (!m->data || (m->rows > 1 && m->row_stride >= far) || (m->stack > 1 && m->stack_stride >= far)) return false;
    if (!output) return true;
    return (m->rows == 1 || m->row_stride >= m->cols) && (m->stack == 1 || m->stack_stride >= (m->rows - 1) * m->row_stride + m->cols);
}
static inline bool l8_same_shape(const zkdl_mat* a, const zkdl_mat* b) {
    return a->stack == b->stack && a->rows == b->rows && a->cols == b->cols;
}
static inline uint64_t l8_ceil(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// ---- k_layer8.hip ------------------------------------------------------------------
// zkdl_quantize_i8 behind its checks, on matrices with entries
int zk_quantize_i8(zkdl_ctx* ctx, const zkdl_mat* x, int axis, const float* mult, const zkdl_mat* q, float* scale, const zkdl_mat* values);
// What the gradients of a small layer need first, in one launch: dy w_scale quantised by rows (q, t), a_scale dy by columns (p, u), and the
// matrices that have to be packed for the tiles.
struct L8Prepare {
    const zkdl_mat *dy, *q, *p;
    const float *a_scale, *w_scale;
    float *t, *u;
    M8PackArgs pack[2];
    int packs;
};
bool zk_prepare_fits(const zkdl_mat* dy);
int zk_prepare(zkdl_ctx* ctx, const L8Prepare& job);
// the two quantisations alone, for gradients of many rows
bool zk_quantize_both_fits(const zkdl_mat* dy);
int zk_quantize_both(zkdl_ctx* ctx, const L8Prepare& job);
