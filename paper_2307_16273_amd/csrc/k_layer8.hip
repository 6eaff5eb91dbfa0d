// Quantisation to 8 bits and the norm between 8-bit layers (zkdl_quantize_i8, zkdl_rmsnorm_i8, zkdl_rmsnorm_i8_backward).
// Every kernel here is bound by memory: a value costs a few instructions and 2 to 9 bytes, so a row is read once, kept in
// registers while its maximum (and mean square) is reduced, and written once.  Of a card that copies 5.0 TB/s from and to memory: norm of
// 8192 x 4096 bf16 with residual and all outputs 58 us (5.2 TB/s), its gradients 57 us (4.7), 4096 x 4096 bf16 by rows 15.1 us (5.6, part
// of it from the last-level cache), 8 x 1024 x 1024 f32 by columns 15.3 us (4.9).  One token of 4096 takes the kernel 3.7 us, all of it
// latency: launch, a load, a reduction, a store.
#include <float.h>

#include "layer8.cuh"

// ---------------------------------------------------------------------------
// Rows: v = (x [+ residual]) * w, largest |v| of the row, q = rint(v * 127 / that).
// A row belongs to G threads (a wave, or a block) and each of them keeps ITEMS vectors of 8 values, all of whose loads are
// under way before the first is looked at; ITEMS = 0 is for rows too long for the registers, which are read twice, and for
// rows of fewer than 8.
// ---------------------------------------------------------------------------
struct L8RowArgs {
    uint64_t rows, per_stack;     // rows in all, rows of a matrix
    uint32_t cols;
    const void* w;                // norm: cols weights; else cols multipliers for each matrix, or null
    int w_f32;                    // w is 32 bits (else the values' type)
    uint64_t w_stack;             // items of w for each matrix
    float eps;
    float* scale;
    float* rstd;
};

template <class T>
static __device__ __forceinline__ void l8_weights(const L8RowArgs& a, uint64_t s, uint32_t j, int n, float (&f)[8]) {
    if (!a.w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 1.f;
    } else if (a.w_f32) {
        l8_load((const float*)a.w + s * a.w_stack + j, n, f);
    } else {
        l8_load((const T*)a.w + s * a.w_stack + j, n, f);
    }
}

// threads of a block: four waves, or one group if that is larger
constexpr int l8_threads(int group) { return group < 256 ? 256 : group; }
// columns that a group of threads holds with `items` vectors of 8 each; every choice of a kernel below asks this and no number of its own
constexpr uint64_t l8_covers(int group, int items) { return (uint64_t)group * items * 8; }

// sum and maximum over the G threads of a row
template <int G>
static __device__ __forceinline__ void l8_row_reduce(float& sum, uint32_t& top) {
    sum = l8_wave_sum(sum);
    top = l8_wave_max(top);
    if constexpr (G > 64) {
        __shared__ float s_sum[G / 64];
        __shared__ uint32_t s_top[G / 64];
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
            s_sum[threadIdx.x >> 6] = sum;
            s_top[threadIdx.x >> 6] = top;
        }
        __syncthreads();
        sum = 0.f;
        top = 0;
#pragma unroll
        for (int i = 0; i < G / 64; ++i) {
            sum += s_sum[i];
            top = max(top, s_top[i]);
        }
    }
}

// the mean square's root when the squares, or their mean with eps, left the range (or an input did): once more, 2^-80 smaller.  (At that scale
// the sum is at least 2^-64, so an eps that underflows there is lost beside it in any case.)
template <class T, int G>
static __device__ __forceinline__ float l8_rstd_again(const T* x, const T* r, uint32_t cols, float eps, uint32_t t) {
    float again = 0.f;
    uint32_t unused = 0;
#pragma unroll 1
    for (uint32_t j = t * 8; j < cols; j += G * 8) {
        float h[8], b[8] = {};
        const int n = (int)min(cols - j, 8u);
        l8_load(x + j, n, h);
        if (r) l8_load(r + j, n, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float y = (h[i] + b[i]) * 0x1p-80f;
            again = fmaf(y, y, again);
        }
    }
    l8_row_reduce<G>(again, unused);
    return 0x1p-80f / sqrtf(again / (float)cols + eps * 0x1p-80f * 0x1p-80f);
}

template <class T, bool NORM, int G, int ITEMS>
static __device__ __forceinline__ void l8_rows(const L8RowArgs& a, const L8Mat<const T>& x, const L8Mat<const T>& res, const L8Mat<int8_t>& q,
                                               const L8Mat<T>& total, const L8Mat<T>& values, uint32_t block, uint32_t blocks) {
    constexpr int GROUPS = l8_threads(G) / G;
    const uint32_t t = threadIdx.x % G;
    const uint64_t step = (uint64_t)blocks * GROUPS;
    // all groups of a block take as many turns: the reductions of a block-wide group meet at barriers
    for (uint64_t r0 = (uint64_t)block * GROUPS; r0 < a.rows; r0 += step) {
        const uint64_t r = r0 + threadIdx.x / G;
        if (GROUPS > 1 && r >= a.rows) continue;
        const uint64_t s = r / a.per_stack, m = r % a.per_stack;
        const T* xr = x.p + s * x.ss + m * x.rs;
        const T* rr = NORM && res.p ? res.p + s * res.ss + m * res.rs : nullptr;
        T* tr = NORM && total.p ? total.p + s * total.ss + m * total.rs : nullptr;
        float keep[ITEMS ? ITEMS : 1][8];
        float ss = 0.f;
        uint32_t top = 0;
        if constexpr (ITEMS > 0) {
            L8At at[ITEMS];
            L8Vec<T> xv[ITEMS], rv[ITEMS], wt[ITEMS];
            L8Vec<float> wf[ITEMS];
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                at[k] = l8_at((k * G + t) * 8, a.cols);
                xv[k] = l8_raw(xr + at[k].start);
            }
            if (NORM && rr) {
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) rv[k] = l8_raw(rr + at[k].start);
            }
            if (a.w && a.w_f32) {
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) wf[k] = l8_raw((const float*)a.w + s * a.w_stack + at[k].start);
            } else if (NORM && a.w) {
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) wt[k] = l8_raw((const T*)a.w + at[k].start);
            }
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                float(&v)[8] = keep[k];
                l8_floats(xv[k], v);
                if (NORM) {
                    if (rr) {
                        float b[8];
                        l8_floats(rv[k], b);
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] += b[i];
                    }
                    if (tr && at[k].live) l8_store(tr + at[k].start, 8, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) ss = fmaf(v[i], (uint32_t)i < at[k].dup ? 0.f : v[i], ss);
                }
                if (a.w) {
                    float w[8];
                    if (a.w_f32) l8_floats(wf[k], w);
                    else if (NORM) l8_floats(wt[k], w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= w[i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, l8_mag(v[i]));
            }
        } else {
            for (uint32_t j = t * 8; j < a.cols; j += G * 8) {
                const int n = (int)min(a.cols - j, 8u);
                float v[8], w[8];
                l8_load(xr + j, n, v);
                if (rr) {
                    l8_load(rr + j, n, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] += w[i];
                }
                if (tr) l8_store(tr + j, n, v);
                l8_weights<T>(a, s, j, n, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (NORM) ss = fmaf(v[i], v[i], ss);
                    top = max(top, l8_mag(v[i] * w[i]));
                }
            }
        }
        l8_row_reduce<G>(ss, top);
        float rstd = 1.f;
        if (NORM) {
            const float ms = ss / (float)a.cols + a.eps;
            rstd = l8_mag(ms) >= L8_INF ? l8_rstd_again<T, G>(xr, rr, a.cols, a.eps, t) : 1.f / sqrtf(ms);
        }
        const L8Quant c = l8_quant(top);
        float scale = __uint_as_float(top) / 127.f;
        if (NORM) scale = __uint_as_float(top) * rstd / 127.f;
        if (!c.finite) scale = __uint_as_float(0x7fc00000u);
        if (t == 0) {
            a.scale[r] = scale;
            if (NORM && a.rstd) a.rstd[r] = rstd;
        }
        int8_t* qr = q.p + s * q.ss + m * q.rs;
        T* vr = values.p ? values.p + s * values.ss + m * values.rs : nullptr;
        auto second = [&](uint32_t j, int n, float (&v)[8]) {
            int iq[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) iq[i] = l8_round(v[i], c);
            l8_store_q(qr + j, n, iq);
            if (vr) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = (float)iq[i] * scale;
                l8_store(vr + j, n, v);
            }
        };
        if constexpr (ITEMS > 0) {
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const L8At p = l8_at((k * G + t) * 8, a.cols);
                if (p.live) second(p.start, 8, keep[k]);
            }
        } else {
            for (uint32_t j = t * 8; j < a.cols; j += G * 8) {
                const int n = (int)min(a.cols - j, 8u);
                float v[8], w[8];
                l8_load(xr + j, n, v);
                if (rr) {
                    l8_load(rr + j, n, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] += w[i];
                }
                l8_weights<T>(a, s, j, n, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= w[i];
                second(j, n, v);
            }
        }
    }
}

template <class T, bool NORM, int G, int ITEMS>
__global__ __launch_bounds__(l8_threads(G)) void k_l8_rows(L8RowArgs a, L8Mat<const T> x, L8Mat<const T> res, L8Mat<int8_t> q, L8Mat<T> total,
                                                           L8Mat<T> values) {
    l8_rows<T, NORM, G, ITEMS>(a, x, res, q, total, values, blockIdx.x, gridDim.x);
}

// zeros by a kernel and not by a memory operation: the calls may be captured into a graph
__global__ __launch_bounds__(256) void k_l8_zero(float* p, uint64_t n) {
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < n; i += gridDim.x * 256ull) p[i] = 0.f;
}

// blocks of a launch that walks over `units` of work: enough to fill the device several times over
static unsigned l8_grid(uint64_t units) { return (unsigned)(units < 65536 ? units : 65536); }

template <class T, bool NORM>
static void l8_launch_rows(zkdl_ctx* ctx, const L8RowArgs& a, L8Mat<const T> x, L8Mat<const T> res, L8Mat<int8_t> q, L8Mat<T> total,
                           L8Mat<T> values) {
    const uint32_t n = a.cols;
#define L8_ROWS(G, ITEMS)                                                                                                              \
    hipLaunchKernelGGL((k_l8_rows<T, NORM, G, ITEMS>), dim3(l8_grid(l8_ceil(a.rows, l8_threads(G) / G))), dim3(l8_threads(G)), 0, ctx->stream, a, x, \
                       res, q, total, values)
#define L8_ROWS_TO(G, ITEMS) if (n <= l8_covers(G, ITEMS)) L8_ROWS(G, ITEMS)
    if (n < 8) L8_ROWS(64, 0);
    else L8_ROWS_TO(64, 1);
    else L8_ROWS_TO(64, 2);
    else L8_ROWS_TO(256, 1);
    else L8_ROWS_TO(256, 2);
    else L8_ROWS_TO(512, 2);
    else L8_ROWS_TO(1024, 2);
    else L8_ROWS(1024, 0);
#undef L8_ROWS_TO
#undef L8_ROWS
}

// ---------------------------------------------------------------------------
// Columns: a block looks at 64 columns x a chunk of rows; largest magnitudes of the chunks, then the values once more (they
// come from the last-level cache for anything below 256 MB).  A chunk that is a whole column needs no second launch.
// ---------------------------------------------------------------------------
constexpr int L8_COL_T = 8, L8_COL_R = 32;      // 8 threads of 8 columns, 32 rows at a time
struct L8ColArgs {
    uint64_t rows, chunk;         // chunk: rows of a block
    uint32_t cols, chunks;
    const float* mult;            // rows for each matrix, or null
    uint32_t* part;               // [stack][parts][cols] largest magnitudes
    uint32_t parts;
    float* scale;                 // [stack][cols]
};

// four rows of a thread: read before the first of them is looked at
template <class T>
struct L8ColRows {
    L8Vec<T> v[4];
    float w[4];
    __device__ __forceinline__ void fetch(const L8Mat<const T>& x, const T* p, const float* mu, uint64_t m, uint64_t hi) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = l8_raw(p + min(m + k * L8_COL_R, hi - 1) * x.rs);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = 1.f;
        if (mu) {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = mu[min(m + k * L8_COL_R, hi - 1)];
        }
    }
};

// f(m, v) for the thread's rows m, m + 32, .. < hi.  WIDE: there are 8 columns and more; the last eight of a row start where that many are
// left (what two threads both have, both write alike), and `first` holds the first four rows.
template <class T, bool WIDE, class F>
static __device__ __forceinline__ void l8_col_walk(const L8ColArgs& a, const L8Mat<const T>& x, uint64_t s, uint64_t m, uint64_t hi, uint32_t j,
                                                   L8ColRows<T> first, F f) {
    const T* p = x.p + s * x.ss + j;
    const float* mu = a.mult ? a.mult + s * a.rows : nullptr;
    if constexpr (WIDE) {
        for (bool more = false; m < hi; m += 4 * L8_COL_R, more = true) {
            if (more) first.fetch(x, p, mu, m, hi);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (m + k * L8_COL_R >= hi) break;
                float g[8];
                l8_floats(first.v[k], g);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] *= first.w[k];
                f(m + k * L8_COL_R, g);
            }
        }
    } else {
        for (; m < hi; m += L8_COL_R) {
            float g[8];
            l8_load(p + m * x.rs, (int)a.cols, g);
            if (mu) {
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] *= mu[m];
            }
            f(m, g);
        }
    }
}

// MODE 0: largest magnitudes of a chunk -> part; 1: quantise a chunk; 2: both, the chunk being all rows
template <class T, int MODE, bool WIDE>
__global__ __launch_bounds__(256) void k_l8_cols(L8ColArgs a, L8Mat<const T> x, L8Mat<int8_t> q, L8Mat<T> values) {
    __shared__ uint32_t s_top[L8_COL_R][L8_COL_T * 8 + 1];
    __shared__ float s_pre[L8_COL_T * 8], s_inv[L8_COL_T * 8], s_scale[L8_COL_T * 8];
    const uint32_t tx = threadIdx.x % L8_COL_T, ty = threadIdx.x / L8_COL_T;
    const uint32_t c0 = blockIdx.x * (L8_COL_T * 8);
    // threadIdx.x < 64 also: the column whose magnitude that thread finishes
    const uint32_t j = WIDE ? l8_at(c0 + tx * 8, a.cols).start : 0, mine = WIDE ? l8_at(c0 + (threadIdx.x & 56), a.cols).start + (threadIdx.x & 7) : threadIdx.x;
    const uint64_t s = blockIdx.z;
    const uint64_t lo = blockIdx.y * a.chunk, hi = min(lo + a.chunk, a.rows);
    const bool live = c0 + tx * 8 < a.cols;
    const int n = WIDE ? 8 : (int)a.cols;
    uint32_t top[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    L8ColRows<T> first;
    if (WIDE && lo < hi) first.fetch(x, x.p + s * x.ss + j, a.mult ? a.mult + s * a.rows : nullptr, lo + ty, hi);
    if (MODE != 1) {
        if (live)
            l8_col_walk<T, WIDE>(a, x, s, lo + ty, hi, j, first, [&](uint64_t, float(&v)[8]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) top[i] = max(top[i], l8_mag(v[i]));
            });
    } else if (live) {
        for (uint32_t k = ty; k < a.parts; k += L8_COL_R) {
            const uint32_t* p = a.part + (s * a.parts + k) * a.cols + j;
            if constexpr (WIDE) {
                const M8Bytes b = *(const M8Bytes*)p, c = *(const M8Bytes*)(p + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) top[i] = max(top[i], b.v[i]), top[4 + i] = max(top[4 + i], c.v[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < n) top[i] = max(top[i], p[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) s_top[ty][tx * 8 + i] = top[i];
    __syncthreads();
    if (threadIdx.x < L8_COL_T * 8) {
        uint32_t b = 0;
        for (int k = 0; k < L8_COL_R; ++k) b = max(b, s_top[k][threadIdx.x]);
        const bool in = WIDE ? c0 + (threadIdx.x & 56) < a.cols : threadIdx.x < a.cols;
        if (MODE == 0) {
            if (in) a.part[(s * a.parts + blockIdx.y) * a.cols + mine] = b;
        } else {
            const L8Quant c = l8_quant(b);
            const float scale = c.finite ? __uint_as_float(b) / 127.f : __uint_as_float(0x7fc00000u);
            s_pre[threadIdx.x] = c.pre;
            s_inv[threadIdx.x] = c.inv;
            s_scale[threadIdx.x] = scale;
            if (in && blockIdx.y == 0) a.scale[s * a.cols + mine] = scale;
        }
    }
    if (MODE == 0) return;
    __syncthreads();
    if (!live) return;
    L8Quant c[8];
    float scale[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        scale[i] = s_scale[tx * 8 + i];
        c[i].pre = s_pre[tx * 8 + i];
        c[i].inv = s_inv[tx * 8 + i];
        c[i].finite = scale[i] == scale[i];
    }
    l8_col_walk<T, WIDE>(a, x, s, lo + ty, hi, j, first, [&](uint64_t m, float(&v)[8]) {
        int iq[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) iq[i] = l8_round(v[i], c[i]);
        l8_store_q(q.p + s * q.ss + m * q.rs + j, n, iq);
        if (values.p) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)iq[i] * scale[i];
            l8_store(values.p + s * values.ss + m * values.rs + j, n, v);
        }
    });
}

// The same with the columns kept in registers between the two looks at them, for up to 2048 rows: a block has 8 CT columns, 256 rows at a
// time.  CT = 4 reads whole lines; CT = 1 is for matrices of few columns, which would otherwise leave most of the device idle.
constexpr int L8_ONCE_R = 256, L8_ONCE_ITEMS = 8;
template <class T, int CT, int ITEMS>
static __device__ __forceinline__ void l8_cols_once(const L8ColArgs& a, const L8Mat<const T>& x, const L8Mat<int8_t>& q, const L8Mat<T>& values,
                                                    uint64_t s, uint32_t block) {
    constexpr int WAVES = CT * L8_ONCE_R / 64;
    __shared__ uint32_t s_top[WAVES][CT * 8];
    __shared__ float s_pre[CT * 8], s_inv[CT * 8], s_scale[CT * 8];
    const uint32_t tx = threadIdx.x % CT, ty = threadIdx.x / CT;
    const L8At at = l8_at(block * (CT * 8) + tx * 8, a.cols);
    const T* p = x.p + s * x.ss + at.start;
    const float* mu = a.mult ? a.mult + s * a.rows : nullptr;
    L8Vec<T> raw[ITEMS];
    float w[ITEMS], v[ITEMS][8];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) raw[k] = l8_raw(p + min(ty + (uint64_t)k * L8_ONCE_R, a.rows - 1) * x.rs);
    if (mu) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) w[k] = mu[min(ty + (uint64_t)k * L8_ONCE_R, a.rows - 1)];
    }
    uint32_t top[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        l8_floats(raw[k], v[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (mu) v[k][i] *= w[k];
            top[i] = max(top[i], l8_mag(v[k][i]));
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int d = CT; d < 64; d <<= 1) top[i] = max(top[i], (uint32_t)__shfl_xor((int)top[i], d, 64));
    }
    if ((threadIdx.x & 63) < CT) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_top[threadIdx.x >> 6][tx * 8 + i] = top[i];
    }
    __syncthreads();
    if (threadIdx.x < CT * 8) {
        uint32_t b = 0;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) b = max(b, s_top[k][threadIdx.x]);
        const L8Quant c = l8_quant(b);
        s_pre[threadIdx.x] = c.pre;
        s_inv[threadIdx.x] = c.inv;
        s_scale[threadIdx.x] = c.finite ? __uint_as_float(b) / 127.f : __uint_as_float(0x7fc00000u);
    }
    __syncthreads();
    if (!at.live) return;
    L8Quant c[8];
    float scale[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        scale[i] = s_scale[tx * 8 + i];
        c[i].pre = s_pre[tx * 8 + i];
        c[i].inv = s_inv[tx * 8 + i];
        c[i].finite = scale[i] == scale[i];
    }
    if (ty == 0) l8_store(a.scale + s * a.cols + at.start, 8, scale);
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const uint64_t m = ty + (uint64_t)k * L8_ONCE_R;
        if (m >= a.rows) break;
        int iq[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) iq[i] = l8_round(v[k][i], c[i]);
        l8_store_q(q.p + s * q.ss + m * q.rs + at.start, 8, iq);
        if (values.p) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)iq[i] * scale[i];
            l8_store(values.p + s * values.ss + m * values.rs + at.start, 8, f);
        }
    }
}
template <class T, int CT, int ITEMS>
__global__ __launch_bounds__(CT * L8_ONCE_R) void k_l8_cols_once(L8ColArgs a, L8Mat<const T> x, L8Mat<int8_t> q, L8Mat<T> values) {
    l8_cols_once<T, CT, ITEMS>(a, x, q, values, blockIdx.z, blockIdx.x);
}

// four blocks for each compute unit, of 64 rows and more
static void l8_col_chunks(L8ColArgs& a, uint64_t tiles) {
    uint64_t chunks = l8_ceil(1024, tiles);
    if (chunks > l8_ceil(a.rows, 64)) chunks = l8_ceil(a.rows, 64);
    if (chunks < 1) chunks = 1;
    a.chunk = l8_ceil(l8_ceil(a.rows, chunks), L8_COL_R) * L8_COL_R;
    a.chunks = (uint32_t)l8_ceil(a.rows, a.chunk);
}

template <class T>
static int l8_quant_cols(zkdl_ctx* ctx, const zkdl_mat* x, const float* mult, const zkdl_mat* q, float* scale, const zkdl_mat* values) {
    L8ColArgs a = {};
    a.rows = x->rows;
    a.cols = (uint32_t)x->cols;
    a.mult = mult;
    a.scale = scale;
    a.part = nullptr;
    const uint64_t tiles = l8_ceil(x->cols, L8_COL_T * 8);
    const bool wide = x->cols >= 8;
    // the grid's axes hold 65535 blocks: matrices of a longer stack go in launches of their own
    for (uint64_t s0 = 0; s0 < x->stack; s0 += 65535) {
        const uint64_t ns = x->stack - s0 < 65535 ? x->stack - s0 : 65535;
        l8_col_chunks(a, tiles * ns);
        a.parts = a.chunks;
        L8Mat<const T> mx = l8_mat<const T>(x);
        L8Mat<int8_t> mq = l8_mat<int8_t>(q);
        L8Mat<T> mv = l8_mat<T>(values);
        mx.p += s0 * mx.ss;
        mq.p += s0 * mq.ss;
        if (mv.p) mv.p += s0 * mv.ss;
        a.mult = mult ? mult + s0 * x->rows : nullptr;
        a.scale = scale + s0 * x->cols;
        const dim3 grid((unsigned)tiles, a.chunks, (unsigned)ns);
        if (wide && x->rows <= L8_ONCE_R * L8_ONCE_ITEMS) {
#define L8_ONCE(CT, ITEMS) \
    hipLaunchKernelGGL((k_l8_cols_once<T, CT, ITEMS>), dim3((unsigned)l8_ceil(x->cols, CT * 8), 1, (unsigned)ns), dim3(CT * L8_ONCE_R), 0, ctx->stream, a, mx, mq, mv)
            if (l8_ceil(x->cols, 32) * ns < 64 && x->rows <= 4 * L8_ONCE_R) {
                if (x->rows <= 2 * L8_ONCE_R) L8_ONCE(1, 2);
                else L8_ONCE(1, 4);
            } else if (x->rows <= L8_ONCE_R) L8_ONCE(4, 1);
            else if (x->rows <= 2 * L8_ONCE_R) L8_ONCE(4, 2);
            else if (x->rows <= 4 * L8_ONCE_R) L8_ONCE(4, 4);
            else L8_ONCE(4, 8);
#undef L8_ONCE
            continue;
        }
        if (a.chunks == 1) {
            hipLaunchKernelGGL((wide ? k_l8_cols<T, 2, true> : k_l8_cols<T, 2, false>), grid, dim3(256), 0, ctx->stream, a, mx, mq, mv);
            continue;
        }
        a.part = (uint32_t*)zk_alloc_scratch(ctx, ns * a.chunks * x->cols * 4);
        if (!a.part) return ZKDL_ENOMEM;
        hipLaunchKernelGGL((wide ? k_l8_cols<T, 0, true> : k_l8_cols<T, 0, false>), grid, dim3(256), 0, ctx->stream, a, mx, mq, mv);
        hipLaunchKernelGGL((wide ? k_l8_cols<T, 1, true> : k_l8_cols<T, 1, false>), grid, dim3(256), 0, ctx->stream, a, mx, mq, mv);
        zk_free(ctx, a.part);
    }
    return ZKDL_OK;
}

template <class T>
static int l8_quantize(zkdl_ctx* ctx, const zkdl_mat* x, int axis, const float* mult, const zkdl_mat* q, float* scale, const zkdl_mat* values) {
    if (axis == 0) return l8_quant_cols<T>(ctx, x, mult, q, scale, values);
    L8RowArgs a = {};
    a.rows = x->stack * x->rows;
    a.per_stack = x->rows;
    a.cols = (uint32_t)x->cols;
    a.w = mult;
    a.w_f32 = 1;
    a.w_stack = x->cols;
    a.scale = scale;
    l8_launch_rows<T, false>(ctx, a, l8_mat<const T>(x), L8Mat<const T>{nullptr, 0, 0}, l8_mat<int8_t>(q), L8Mat<T>{nullptr, 0, 0}, l8_mat<T>(values));
    return ZKDL_OK;
}

int zk_quantize_i8(zkdl_ctx* ctx, const zkdl_mat* x, int axis, const float* mult, const zkdl_mat* q, float* scale, const zkdl_mat* values) {
    switch (x->dtype) {
        case ZKDL_F32: return l8_quantize<float>(ctx, x, axis, mult, q, scale, values);
        case ZKDL_F16: return l8_quantize<__half>(ctx, x, axis, mult, q, scale, values);
        default: return l8_quantize<bf16_t>(ctx, x, axis, mult, q, scale, values);
    }
}

extern "C" int zkdl_quantize_i8(zkdl_ctx* ctx, const zkdl_mat* x, int axis, const float* mult, const zkdl_mat* q, float* scale,
                                const zkdl_mat* values) try {
    if (!ctx || !l8_mat_ok(x, false) || !l8_mat_ok(q, true) || !l8_is_float(x->dtype) || q->dtype != ZKDL_I8 || !l8_same_shape(x, q) ||
        (axis != 0 && axis != 1))
        return ZKDL_EINVAL;
    if (values && (!l8_mat_ok(values, true) || values->dtype != x->dtype || !l8_same_shape(x, values))) return ZKDL_EINVAL;
    const uint64_t scales = x->stack * (axis ? x->rows : x->cols);
    if (scales && !scale) return ZKDL_EINVAL;
    if (axis == 0 && x->cols >= (uint64_t)1 << 27) return ZKDL_ETOOBIG;     // a launch's threads are counted in 32 bits
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    if (scales && (axis ? x->cols : x->rows) == 0) {        // scales of nothing
        hipLaunchKernelGGL(k_l8_zero, dim3(l8_grid(l8_ceil(scales, 256))), dim3(256), 0, ctx->stream, scale, scales);
        ZK_HIP(ctx, hipGetLastError());
        return ZKDL_OK;
    }
    if (!scales) return ZKDL_OK;
    const int rc = zk_quantize_i8(ctx, x, axis, mult, q, scale, values);
    if (rc != ZKDL_OK) return rc;
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}

extern "C" int zkdl_rmsnorm_i8(zkdl_ctx* ctx, const zkdl_mat* x, const zkdl_mat* residual, const void* weight, int weight_dtype, float eps,
                               const zkdl_mat* q, float* scale, float* rstd, const zkdl_mat* total, const zkdl_mat* values) try {
    if (!ctx || !l8_mat_ok(x, false) || !l8_mat_ok(q, true) || !l8_is_float(x->dtype) || q->dtype != ZKDL_I8 || !l8_same_shape(x, q) ||
        x->stack != 1)
        return ZKDL_EINVAL;
    if (residual && (!l8_mat_ok(residual, false) || residual->dtype != x->dtype || !l8_same_shape(x, residual))) return ZKDL_EINVAL;
    for (const zkdl_mat* o : {total, values})
        if (o && (!l8_mat_ok(o, true) || o->dtype != x->dtype || !l8_same_shape(x, o))) return ZKDL_EINVAL;
    if (weight_dtype != ZKDL_F32 && weight_dtype != x->dtype) return ZKDL_EINVAL;
    if (!(eps >= FLT_MIN) || !(eps <= FLT_MAX)) return ZKDL_EINVAL;
    if (x->rows == 0) return ZKDL_OK;
    if (x->cols == 0 || !weight || !scale) return ZKDL_EINVAL;      // the mean over no entries is no number
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    L8RowArgs a = {};
    a.rows = a.per_stack = x->rows;
    a.cols = (uint32_t)x->cols;
    a.w = weight;
    a.w_f32 = weight_dtype == ZKDL_F32;
    a.eps = eps;
    a.scale = scale;
    a.rstd = rstd;
    auto go = [&](auto t) {
        using T = decltype(t);
        l8_launch_rows<T, true>(ctx, a, l8_mat<const T>(x), l8_mat<const T>(residual), l8_mat<int8_t>(q), l8_mat<T>(total), l8_mat<T>(values));
    };
    if (x->dtype == ZKDL_F32) go(float{});
    else if (x->dtype == ZKDL_F16) go(__half{});
    else go(bf16_t{});
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}

// ---------------------------------------------------------------------------
// Both quantisations of a large gradient: by rows (times the columns' scales), and, in the same pass, the largest magnitudes of the columns
// (times the rows' scales), each thread its own columns over all of its block's rows; then by columns.  The gradient is read twice instead
// of three times.
// ---------------------------------------------------------------------------
template <class T>
struct L8BothArgs {
    uint64_t rows;
    uint32_t cols;
    const float *row_mult, *col_mult;     // a factor for each row (for the columns' codes), for each column (for the rows')
    float* scale;                         // of the rows
    uint32_t* part;                       // [blocks][cols]
    L8Mat<const T> x;
    L8Mat<int8_t> q;
};
template <class T, int G, int ITEMS>
__global__ __launch_bounds__(l8_threads(G)) void k_l8_both(L8BothArgs<T> a) {
    constexpr int GROUPS = l8_threads(G) / G;
    const uint32_t t = threadIdx.x % G;
    uint32_t tops[ITEMS][8] = {};
    float w[ITEMS][8];
    L8At at[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        at[k] = l8_at((k * G + t) * 8, a.cols);
        l8_floats(l8_raw(a.col_mult + at[k].start), w[k]);
    }
    const uint64_t step = (uint64_t)gridDim.x * GROUPS;
    for (uint64_t r0 = (uint64_t)blockIdx.x * GROUPS; r0 < a.rows; r0 += step) {
        const uint64_t m = r0 + threadIdx.x / G;
        if (GROUPS > 1 && m >= a.rows) continue;
        const float f = a.row_mult[m];
        L8Vec<T> xv[ITEMS];
        float v[ITEMS][8], unused = 0.f;
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) xv[k] = l8_raw(a.x.p + m * a.x.rs + at[k].start);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            l8_floats(xv[k], v[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                tops[k][i] = max(tops[k][i], l8_mag(v[k][i] * f));
                v[k][i] *= w[k][i];
                top = max(top, l8_mag(v[k][i]));
            }
        }
        l8_row_reduce<G>(unused, top);
        const L8Quant c = l8_quant(top);
        if (t == 0) a.scale[m] = c.finite ? __uint_as_float(top) / 127.f : __uint_as_float(0x7fc00000u);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            int iq[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) iq[i] = l8_round(v[k][i], c);
            if (at[k].live) l8_store_q(a.q.p + m * a.q.rs + at[k].start, 8, iq);
        }
    }
    if constexpr (GROUPS > 1) {
        __shared__ uint32_t s_tops[GROUPS][G * ITEMS * 8];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at[k].live) s_tops[threadIdx.x / G][at[k].start + i] = tops[k][i];
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < a.cols; j += l8_threads(G)) {
            uint32_t b = 0;
            for (int k = 0; k < GROUPS; ++k) b = max(b, s_tops[k][j]);
            a.part[(uint64_t)blockIdx.x * a.cols + j] = b;
        }
    } else {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
            if (at[k].live) {
#pragma unroll
                for (int i = 0; i < 8; ++i) a.part[(uint64_t)blockIdx.x * a.cols + at[k].start + i] = tops[k][i];
            }
    }
}
// of the blocks' parts the first: 32 columns x 32 runs of parts
__global__ __launch_bounds__(1024) void k_l8_max_parts(uint32_t* part, uint32_t parts, uint32_t cols) {
    __shared__ uint32_t s[32][33];
    const uint32_t tx = threadIdx.x & 31, ty = threadIdx.x >> 5, j = blockIdx.x * 32 + tx;
    uint32_t b = 0;
    if (j < cols) {
#pragma unroll 8
        for (uint32_t k = ty; k < parts; k += 32) b = max(b, part[(uint64_t)k * cols + j]);
    }
    s[ty][tx] = b;
    __syncthreads();
    if (ty == 0 && j < cols) {
        for (int k = 0; k < 32; ++k) b = max(b, s[k][tx]);
        part[j] = b;
    }
}

template <class T>
static int l8_both(zkdl_ctx* ctx, const L8Prepare& job) {
    const zkdl_mat* x = job.dy;
    L8BothArgs<T> a = {x->rows, (uint32_t)x->cols, job.a_scale, job.w_scale, job.t, nullptr, l8_mat<const T>(x), l8_mat<int8_t>(job.q)};
    const uint32_t n = a.cols;
    uint64_t blocks = l8_ceil(a.rows, n <= l8_covers(64, 2) ? 4 : 1);
    if (blocks > 768) blocks = 768;
    a.part = (uint32_t*)zk_alloc_scratch(ctx, blocks * n * 4);
    if (!a.part) return ZKDL_ENOMEM;
#define L8_BOTH(G, ITEMS)           \
    if (n <= l8_covers(G, ITEMS)) \
    hipLaunchKernelGGL((k_l8_both<T, G, ITEMS>), dim3((unsigned)blocks), dim3(l8_threads(G)), 0, ctx->stream, a)
    L8_BOTH(64, 1);
    else L8_BOTH(64, 2);
    else L8_BOTH(256, 1);
    else L8_BOTH(256, 2);
    else L8_BOTH(512, 2);
    else L8_BOTH(1024, 2);
#undef L8_BOTH
    hipLaunchKernelGGL(k_l8_max_parts, dim3((unsigned)l8_ceil(n, 32)), dim3(1024), 0, ctx->stream, a.part, (uint32_t)blocks, n);
    L8ColArgs c = {};
    c.rows = a.rows;
    c.cols = n;
    c.mult = job.a_scale;
    c.scale = job.u;
    c.part = a.part;
    c.parts = 1;
    l8_col_chunks(c, l8_ceil(n, L8_COL_T * 8));
    hipLaunchKernelGGL((k_l8_cols<T, 1, true>), dim3((unsigned)l8_ceil(n, L8_COL_T * 8), c.chunks, 1), dim3(256), 0, ctx->stream, c, l8_mat<const T>(x),
                       l8_mat<int8_t>(job.p), L8Mat<T>{nullptr, 0, 0});
    zk_free(ctx, a.part);
    return ZKDL_OK;
}
bool zk_quantize_both_fits(const zkdl_mat* dy) { return dy->stack == 1 && dy->cols >= 8 && dy->cols <= l8_covers(1024, 2); }
int zk_quantize_both(zkdl_ctx* ctx, const L8Prepare& job) {
    switch (job.dy->dtype) {
        case ZKDL_F32: return l8_both<float>(ctx, job);
        case ZKDL_F16: return l8_both<__half>(ctx, job);
        default: return l8_both<bf16_t>(ctx, job);
    }
}

// ---------------------------------------------------------------------------
// L8Prepare: blocks for each of its parts
// ---------------------------------------------------------------------------
template <class T>
struct L8PrepareArgs {
    L8RowArgs rows;
    L8ColArgs cols;
    L8Mat<const T> dy;
    L8Mat<int8_t> q, p;
    M8PackArgs pack[2];
    uint32_t first[4];      // first block of the columns, of the two packings, and their end
};
template <class T, int G, int ITEMS, int COL_ITEMS>
__global__ __launch_bounds__(256) void k_l8_prepare(L8PrepareArgs<T> a) {
    const L8Mat<T> none = {nullptr, 0, 0};
    const uint32_t b = blockIdx.x;
    if (b < a.first[0]) l8_rows<T, false, G, ITEMS>(a.rows, a.dy, L8Mat<const T>{nullptr, 0, 0}, a.q, none, none, b, a.first[0]);
    else if (b < a.first[1]) l8_cols_once<T, 1, COL_ITEMS>(a.cols, a.dy, a.p, none, 0, b - a.first[0]);
    else if (b < a.first[2]) m8_pack(a.pack[0], b - a.first[1], a.first[2] - a.first[1]);
    else m8_pack(a.pack[1], b - a.first[2], a.first[3] - a.first[2]);
}

// false: nothing was launched, no kernel holds so many rows and columns
template <class T>
static bool l8_prepare(zkdl_ctx* ctx, const L8Prepare& j) {
    L8PrepareArgs<T> a = {};
    a.rows.rows = a.rows.per_stack = j.dy->rows;
    a.rows.cols = (uint32_t)j.dy->cols;
    a.rows.w = j.w_scale;
    a.rows.w_f32 = 1;
    a.rows.w_stack = j.dy->cols;
    a.rows.scale = j.t;
    a.cols.rows = a.cols.chunk = j.dy->rows;
    a.cols.cols = (uint32_t)j.dy->cols;
    a.cols.chunks = 1;
    a.cols.mult = j.a_scale;
    a.cols.scale = j.u;
    a.dy = l8_mat<const T>(j.dy);
    a.q = l8_mat<int8_t>(j.q);
    a.p = l8_mat<int8_t>(j.p);
    const uint64_t n = j.dy->cols;
    a.first[0] = (uint32_t)l8_ceil(j.dy->rows, n <= l8_covers(64, 2) ? 4 : 1);
    a.first[1] = a.first[0] + (uint32_t)l8_ceil(n, 8);
    for (int i = 0; i < 2; ++i) {
        a.pack[i] = j.pack[i];
        const uint64_t pieces = i < j.packs ? j.pack[i].stack * j.pack[i].rows * (j.pack[i].pitch / 16) : 0, blocks = l8_ceil(pieces, 256);
        a.first[2 + i] = a.first[1 + i] + (uint32_t)(blocks < 4096 ? blocks : 4096);
    }
#define L8_PREPARE(G, ITEMS, COL_ITEMS)                                                            \
    if (n <= l8_covers(G, ITEMS) && j.dy->rows <= (uint64_t)COL_ITEMS * L8_ONCE_R)                 \
    hipLaunchKernelGGL((k_l8_prepare<T, G, ITEMS, COL_ITEMS>), dim3(a.first[3]), dim3(256), 0, ctx->stream, a)
    L8_PREPARE(64, 1, 4);
    else L8_PREPARE(64, 2, 4);
    else L8_PREPARE(256, 1, 4);
    else L8_PREPARE(256, 2, 4);
    else L8_PREPARE(256, 4, 4);
    else L8_PREPARE(64, 2, 8);
    else L8_PREPARE(256, 1, 8);
    else L8_PREPARE(256, 2, 8);     // (1025 to 1279 rows: the entries allow up to 2557 columns)
    else return false;
#undef L8_PREPARE
    return true;
}

// Rows of one group's registers, columns of a block's, and no more entries than reading the columns eight at a time is worth: whole calls
// of zkdl_matmul_i8_backward (us, a launch for each step / all in one), rows x in x out: 1024 x 2048 x 2048 34.4 / 34.1, 300 x 500 x 8192
// 34.7 / 32.7, 512 x 512 x 8192 36 / 40; with more than 2048 columns of more than 1024 rows 1025 x 64 x 2557 33.5 / 26.7, 1152 x 1024 x 2112
// 32.8 / 31.6.
bool zk_prepare_fits(const zkdl_mat* dy) {
    return dy->stack == 1 && dy->cols >= 8 && dy->cols <= l8_covers(256, 4) && dy->rows >= 1 && dy->rows <= 8 * L8_ONCE_R &&
           dy->rows * dy->cols <= (uint64_t)5 << 19;
}
int zk_prepare(zkdl_ctx* ctx, const L8Prepare& job) {
    bool held;
    switch (job.dy->dtype) {
        case ZKDL_F32: held = l8_prepare<float>(ctx, job); break;
        case ZKDL_F16: held = l8_prepare<__half>(ctx, job); break;
        default: held = l8_prepare<bf16_t>(ctx, job);
    }
    return held ? ZKDL_OK : ZKDL_ETOOBIG;
}

// ---------------------------------------------------------------------------
// Gradients of the norm.  A group of G threads walks over rows with fixed columns for each thread, so that its share of
// dweight stays in registers; the blocks' shares are summed by a second kernel, always in the same order.
// ---------------------------------------------------------------------------
struct L8BackArgs {
    uint64_t rows;
    uint32_t cols;
    const void* w;
    int w_f32;
    const float* rstd;
    float* part;        // [blocks][cols], or null
    float* dweight;     // not null: blocks from row_blocks on sum it up by columns
    uint32_t row_blocks;
};

// dweight of 64 columns, straight from the gradients: 32 rows at a time
template <class T>
static __device__ __forceinline__ void l8_dweight_cols(const L8BackArgs& a, const L8Mat<const T>& dy, const L8Mat<const T>& h, uint32_t block) {
    __shared__ float s[32][65];
    const uint32_t tx = threadIdx.x % 8, ty = threadIdx.x / 8;
    const L8At at = l8_at(block * 64 + tx * 8, a.cols);
    float dw[8] = {};
    for (uint64_t m = ty; m < a.rows; m += 128) {
        L8Vec<T> gv[4], hv[4];
        float r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint64_t i = min(m + k * 32, a.rows - 1);
            gv[k] = l8_raw(dy.p + i * dy.rs + at.start);
            hv[k] = l8_raw(h.p + i * h.rs + at.start);
            r[k] = a.rstd[i];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (m + k * 32 >= a.rows) break;
            float g[8], n[8];
            l8_floats(gv[k], g);
            l8_floats(hv[k], n);
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[i] = fmaf(g[i], n[i] * r[k], dw[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) s[ty][tx * 8 + i] = dw[i];
    __syncthreads();
    if (ty == 0 && at.live) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dw[i] = 0.f;
            for (int k = 0; k < 32; ++k) dw[i] += s[k][tx * 8 + i];
        }
        l8_store(a.dweight + at.start, 8, dw);
    }
}

template <class T, int G, int ITEMS>
__global__ __launch_bounds__(l8_threads(G)) void k_l8_norm_back(L8BackArgs a, L8Mat<const T> dy, L8Mat<const T> h, L8Mat<const T> dt, L8Mat<T> dx) {
    constexpr int GROUPS = l8_threads(G) / G;
    const uint32_t t = threadIdx.x % G;
    L8RowArgs wa = {};
    wa.w = a.w;
    wa.w_f32 = a.w_f32;
    if (G <= 256 && blockIdx.x >= a.row_blocks) {
        l8_dweight_cols(a, dy, h, blockIdx.x - a.row_blocks);
        return;
    }
    float dw[ITEMS][8] = {}, w[ITEMS][8];
    L8At at[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        at[k] = l8_at((k * G + t) * 8, a.cols);
        l8_weights<T>(wa, 0, at[k].start, 8, w[k]);
    }
    const uint64_t step = (uint64_t)a.row_blocks * GROUPS;
    const float over = 1.f / (float)a.cols;
    for (uint64_t r0 = (uint64_t)blockIdx.x * GROUPS; r0 < a.rows; r0 += step) {
        const uint64_t m = r0 + threadIdx.x / G;
        if (GROUPS > 1 && m >= a.rows) continue;
        const float rstd = a.rstd[m];
        float g[ITEMS][8], n[ITEMS][8];
        float dot = 0.f;
        uint32_t unused = 0;
        L8Vec<T> gv[ITEMS], hv[ITEMS], ev[ITEMS];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) gv[k] = l8_raw(dy.p + m * dy.rs + at[k].start);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) hv[k] = l8_raw(h.p + m * h.rs + at[k].start);
        if (dt.p) {
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) ev[k] = l8_raw(dt.p + m * dt.rs + at[k].start);
        }
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            l8_floats(gv[k], g[k]);
            l8_floats(hv[k], n[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[k][i] *= rstd;
                dw[k][i] = fmaf(g[k][i], n[k][i], dw[k][i]);
                g[k][i] *= w[k][i];
                dot = fmaf(g[k][i], (uint32_t)i < at[k].dup ? 0.f : n[k][i], dot);
            }
        }
        l8_row_reduce<G>(dot, unused);
        dot *= over;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = rstd * fmaf(-n[k][i], dot, g[k][i]);
            if (dt.p) {
                float e[8];
                l8_floats(ev[k], e);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] += e[i];
            }
            if (at[k].live) l8_store(dx.p + m * dx.rs + at[k].start, 8, d);
        }
    }
    if (!a.part) return;
    if constexpr (GROUPS > 1) {
        __shared__ float s_dw[GROUPS][G * ITEMS * 8];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at[k].live) s_dw[threadIdx.x / G][at[k].start + i] = dw[k][i];
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < a.cols; j += l8_threads(G)) {
            float s = 0.f;
            for (int k = 0; k < GROUPS; ++k) s += s_dw[k][j];
            a.part[(uint64_t)blockIdx.x * a.cols + j] = s;
        }
    } else {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
            if (at[k].live) l8_store(a.part + (uint64_t)blockIdx.x * a.cols + at[k].start, 8, dw[k]);
    }
}

// Rows too long for the registers: dx with the row read twice, and dweight by columns.
template <class T>
__global__ __launch_bounds__(256) void k_l8_norm_back_long(L8BackArgs a, L8Mat<const T> dy, L8Mat<const T> h, L8Mat<const T> dt, L8Mat<T> dx) {
    L8RowArgs wa = {};
    wa.w = a.w;
    wa.w_f32 = a.w_f32;
    const float over = 1.f / (float)a.cols;
    for (uint64_t m = blockIdx.x; m < a.rows; m += gridDim.x) {
        const float rstd = a.rstd[m];
        float dot = 0.f;
        uint32_t unused = 0;
        auto at = [&](uint32_t j, int c, float (&g)[8], float (&n)[8]) {
            float w[8];
            l8_load(dy.p + m * dy.rs + j, c, g);
            l8_load(h.p + m * h.rs + j, c, n);
            l8_weights<T>(wa, 0, j, c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] *= rstd;
                g[i] *= w[i];
            }
        };
        for (uint32_t j = threadIdx.x * 8; j < a.cols; j += 2048) {
            float g[8], n[8];
            at(j, (int)min(a.cols - j, 8u), g, n);
#pragma unroll
            for (int i = 0; i < 8; ++i) dot = fmaf(g[i], n[i], dot);
        }
        l8_row_reduce<256>(dot, unused);
        dot *= over;
        for (uint32_t j = threadIdx.x * 8; j < a.cols; j += 2048) {
            const int c = (int)min(a.cols - j, 8u);
            float g[8], n[8];
            at(j, c, g, n);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = rstd * fmaf(-n[i], dot, g[i]);
            if (dt.p) {
                float e[8];
                l8_load(dt.p + m * dt.rs + j, c, e);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] += e[i];
            }
            l8_store(dx.p + m * dx.rs + j, c, g);
        }
    }
}

template <class T>
__global__ __launch_bounds__(256) void k_l8_dweight_long(L8BackArgs a, L8Mat<const T> dy, L8Mat<const T> h) {
    const uint64_t j = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (j >= a.cols) return;
    const int c = (int)min(a.cols - j, (uint64_t)8);
    float dw[8] = {};
    for (uint64_t m = blockIdx.y; m < a.rows; m += gridDim.y) {
        float g[8], n[8];
        l8_load(dy.p + m * dy.rs + j, c, g);
        l8_load(h.p + m * h.rs + j, c, n);
        const float rstd = a.rstd[m];
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[i] = fmaf(g[i], n[i] * rstd, dw[i]);
    }
    l8_store(a.part + blockIdx.y * (uint64_t)a.cols + j, c, dw);
}

// out[j] = sum over the blocks' shares: 32 columns x 32 runs of shares, the runs' sums added in their order
__global__ __launch_bounds__(1024) void k_l8_sum_shares(const float* part, uint32_t shares, uint32_t cols, float* out) {
    __shared__ float s[32][33];
    const uint32_t tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    for (uint64_t j0 = (uint64_t)blockIdx.x * 32; j0 < cols; j0 += gridDim.x * 32ull) {
        const uint64_t j = j0 + tx;
        float x = 0.f;
        if (j < cols) {
#pragma unroll 8
            for (uint32_t k = ty; k < shares; k += 32) x += part[(uint64_t)k * cols + j];
        }
        __syncthreads();
        s[ty][tx] = x;
        __syncthreads();
        if (ty == 0 && j < cols) {
            x = 0.f;
            for (int k = 0; k < 32; ++k) x += s[k][tx];
            out[j] = x;
        }
    }
}

template <class T>
static int l8_norm_back(zkdl_ctx* ctx, L8BackArgs a, const zkdl_mat* dy, const zkdl_mat* h, const zkdl_mat* dt, const zkdl_mat* dx, float* dweight) {
    const uint32_t n = a.cols;
    const bool wave = n <= l8_covers(64, 2), regs = n >= 8 && n <= l8_covers(1024, 2);
    uint64_t blocks = l8_ceil(a.rows, wave ? 4 : 1);
    if (blocks > 768) blocks = 768;
    const uint64_t col_rows = a.rows < 64 ? a.rows : 64;
    a.row_blocks = (uint32_t)blocks;
    // The gradients of few rows are summed by columns in blocks of the same launch, which read them once more, from L2; otherwise the blocks'
    // shares are summed by a second one.  Whole calls (us, second launch / same launch) with 128, 1024, 4096 columns: 64 rows 8.2 / 4.9,
    // 8.6 / 5.0, 8.5 / 5.0; 512 rows 8.4 / 6.8, 8.4 / 7.2, 11.2 / 8.1; 1024 rows 8.6 / 10.6, 8.4 / 11.3, 14.4 / 14.1.
    const bool together = dweight && n >= 8 && n <= l8_covers(256, 2) && a.rows <= 512;
    if (together) {
        a.dweight = dweight;
        blocks += l8_ceil(n, 64);
    } else if (dweight) {
        a.part = (float*)zk_alloc_scratch(ctx, (regs ? blocks : col_rows) * n * 4);
        if (!a.part) return ZKDL_ENOMEM;
    }
    const L8Mat<const T> mdy = l8_mat<const T>(dy), mh = l8_mat<const T>(h), mdt = l8_mat<const T>(dt);
    const L8Mat<T> mdx = l8_mat<T>(dx);
#define L8_BACK(G, ITEMS)           \
    if (n <= l8_covers(G, ITEMS)) \
    hipLaunchKernelGGL((k_l8_norm_back<T, G, ITEMS>), dim3((unsigned)blocks), dim3(l8_threads(G)), 0, ctx->stream, a, mdy, mh, mdt, mdx)
    if (!regs) {
        hipLaunchKernelGGL((k_l8_norm_back_long<T>), dim3(l8_grid(a.rows)), dim3(256), 0, ctx->stream, a, mdy, mh, mdt, mdx);
        if (dweight) hipLaunchKernelGGL((k_l8_dweight_long<T>), dim3((unsigned)l8_ceil(n, 2048), (unsigned)col_rows), dim3(256), 0, ctx->stream, a, mdy, mh);
    } else L8_BACK(64, 1);
    else L8_BACK(64, 2);
    else L8_BACK(256, 1);
    else L8_BACK(256, 2);
    else L8_BACK(512, 2);
    else L8_BACK(1024, 2);
#undef L8_BACK
    if (a.part)
        hipLaunchKernelGGL(k_l8_sum_shares, dim3(l8_grid(l8_ceil(n, 32))), dim3(1024), 0, ctx->stream, a.part, (uint32_t)(regs ? blocks : col_rows), n, dweight);
    zk_free(ctx, a.part);
    return ZKDL_OK;
}

extern "C" int zkdl_rmsnorm_i8_backward(zkdl_ctx* ctx, const zkdl_mat* dy, const zkdl_mat* h, const void* weight, int weight_dtype,
                                        const float* rstd, const zkdl_mat* dtotal, const zkdl_mat* dx, float* dweight) try {
    if (!ctx || !l8_mat_ok(dy, false) || !l8_mat_ok(h, false) || !l8_mat_ok(dx, true) || !l8_is_float(dy->dtype) || h->dtype != dy->dtype ||
        dx->dtype != dy->dtype || !l8_same_shape(dy, h) || !l8_same_shape(dy, dx) || dy->stack != 1)
        return ZKDL_EINVAL;
    if (dtotal && (!l8_mat_ok(dtotal, false) || dtotal->dtype != dy->dtype || !l8_same_shape(dy, dtotal))) return ZKDL_EINVAL;
    if ((weight_dtype != ZKDL_F32 && weight_dtype != dy->dtype) || dy->cols == 0 || !weight) return ZKDL_EINVAL;
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    if (dy->rows == 0) {
        if (dweight) hipLaunchKernelGGL(k_l8_zero, dim3(l8_grid(l8_ceil(dy->cols, 256))), dim3(256), 0, ctx->stream, dweight, dy->cols);
        ZK_HIP(ctx, hipGetLastError());
        return ZKDL_OK;
    }
    if (!rstd) return ZKDL_EINVAL;
    L8BackArgs a = {dy->rows, (uint32_t)dy->cols, weight, weight_dtype == ZKDL_F32, rstd, nullptr, nullptr, 0};
    int rc;
    if (dy->dtype == ZKDL_F32) rc = l8_norm_back<float>(ctx, a, dy, h, dtotal, dx, dweight);
    else if (dy->dtype == ZKDL_F16) rc = l8_norm_back<__half>(ctx, a, dy, h, dtotal, dx, dweight);
    else rc = l8_norm_back<bf16_t>(ctx, a, dy, h, dtotal, dx, dweight);
    if (rc != ZKDL_OK) return rc;
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}
