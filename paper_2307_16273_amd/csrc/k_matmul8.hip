// Products of 8-bit integers with exact 32-bit accumulators on the matrix cores (zkdl_matmul_i8, zkdl_matmul_i8_backward).
//
// v_mfma_i32_16x16x64_i8 takes 64 products of each of 16 x 16 entries; a lane holds 16 adjacent k of one row of op(A) and of
// one column of op(B).  An operand whose memory runs along k is read that way (16 bytes a lane); for the other layout a tile
// stands in LDS as it does in memory, row by row of k, and ds_read_b64_tr_b8 turns 8 x 16 bytes while it reads them: in each
// group of 16 lanes, lanes 2r and 2r+1 point at 16 bytes of row r and lane c receives the eight bytes of column c.
#include "layer8.cuh"

typedef int v2i __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v2i lds_v2i;

struct M8Args {
    const int8_t *a, *b;
    uint64_t a_rs, a_ss, b_rs, b_ss;   // strides of the stored matrices, bytes
    void* out;
    uint64_t o_rs, o_ss;               // items
    int o_type;                        // zkdl_dtype
    const float *sa, *sb;
    uint32_t M, N, K;
};

// the block's tile: matrix, first row, first column
static __device__ __forceinline__ void m8_tile(const M8Args& p, uint32_t bm, uint32_t bn, uint64_t& s, uint32_t& m0, uint32_t& n0) {
    const uint32_t gm = (p.M + bm - 1) / bm, gn = (p.N + bn - 1) / bn, t = blockIdx.x % (gm * gn);
    s = blockIdx.x / (gm * gn);
    m0 = t / gn * bm;
    n0 = t % gn * bn;
}

static __device__ __forceinline__ void m8_store(const M8Args& p, uint64_t s, uint32_t i, uint32_t j, int acc) {
    const uint64_t at = s * p.o_ss + i * p.o_rs + j;
    if (p.o_type == ZKDL_I32) {
        ((int*)p.out)[at] = acc;
        return;
    }
    float f = (float)acc;
    if (p.sa) f *= p.sa[s * p.M + i];
    if (p.sb) f *= p.sb[s * p.N + j];
    if (p.o_type == ZKDL_F32) l8_put(f, ((float*)p.out)[at]);
    else if (p.o_type == ZKDL_F16) l8_put(f, ((__half*)p.out)[at]);
    else l8_put(f, ((bf16_t*)p.out)[at]);
}

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

// 64 x 64 entries a block, four waves of 32 x 32; tiles of 64 k go through registers into LDS, so any address and any edge
// will do.  AT: op(A) runs along m in memory, BN: op(B) along n.
constexpr int M8_PITCH = 80;     // bytes of a tile's row in LDS: 64 and 16 that keep the rows' banks apart
template <bool AT, bool BN>
__global__ __launch_bounds__(256) void k_m8_any(M8Args p) {
    __shared__ __align__(16) int8_t s_a[64 * M8_PITCH], s_b[64 * M8_PITCH];
    const uint32_t t = threadIdx.x, l = t & 63, w = t >> 6, g = l >> 4, i16 = l & 15;
    uint64_t s;
    uint32_t m0, n0;
    m8_tile(p, 64, 64, s, m0, n0);
    const uint32_t wm = (w >> 1) * 32, wn = (w & 1) * 32;
    const int8_t *a = p.a + s * p.a_ss, *b = p.b + s * p.b_ss;
    v4i acc[2][2] = {};
    for (uint32_t k0 = 0; k0 < p.K; k0 += 64) {
        const uint32_t r = t >> 2, c = (t & 3) * 16;
        const v4i va = AT ? m8_fetch(a, p.a_rs, k0 + r, p.K, m0 + c, p.M) : m8_fetch(a, p.a_rs, m0 + r, p.M, k0 + c, p.K);
        const v4i vb = BN ? m8_fetch(b, p.b_rs, k0 + r, p.K, n0 + c, p.N) : m8_fetch(b, p.b_rs, n0 + r, p.N, k0 + c, p.K);
        __syncthreads();
        *(v4i*)(s_a + r * M8_PITCH + c) = va;
        *(v4i*)(s_b + r * M8_PITCH + c) = vb;
        __syncthreads();
        v4i fa[2], fb[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            auto frag = [&](bool turned, int8_t* tile, uint32_t at) {
                if (!turned) return *(const v4i*)(tile + (at + i16) * M8_PITCH + g * 16);
                v4i f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const v2i y = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i*)(tile + (16 * g + 8 * h + (i16 >> 1)) * M8_PITCH + at + (i16 & 1) * 8));
                    f[2 * h] = y[0];
                    f[2 * h + 1] = y[1];
                }
                return f;
            };
            fa[x] = frag(AT, s_a, wm + x * 16);
            fb[x] = frag(BN, s_b, wn + x * 16);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[y], fa[x], acc[x][y], 0, 0, 0);
    }
    // the tile comes out turned: a lane has four adjacent columns of one row
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const uint32_t i = m0 + wm + x * 16 + i16;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t j = n0 + wn + y * 16 + g * 4 + e;
                if (i < p.M && j < p.N) m8_store(p, s, i, j, acc[x][y][e]);
            }
        }
}

// a launch's blocks are counted in 32 bits of threads
constexpr uint64_t M8_MAX_TILES = (uint64_t)1 << 24;

static int m8_launch(zkdl_ctx* ctx, const M8Args& p, bool at, bool bn, uint64_t stack) {
    const uint64_t tiles = l8_ceil(p.M, 64) * l8_ceil(p.N, 64);
    if (tiles >= M8_MAX_TILES || stack >= M8_MAX_TILES || tiles * stack >= M8_MAX_TILES) return ZKDL_ETOOBIG;
    const dim3 grid((unsigned)(tiles * stack));
    if (at && bn) hipLaunchKernelGGL((k_m8_any<true, true>), grid, dim3(256), 0, ctx->stream, p);
    else if (at) hipLaunchKernelGGL((k_m8_any<true, false>), grid, dim3(256), 0, ctx->stream, p);
    else if (bn) hipLaunchKernelGGL((k_m8_any<false, true>), grid, dim3(256), 0, ctx->stream, p);
    else hipLaunchKernelGGL((k_m8_any<false, false>), grid, dim3(256), 0, ctx->stream, p);
    return ZKDL_OK;
}

// a and b behind the checks; out may be empty
static int m8_product(zkdl_ctx* ctx, const zkdl_mat* a, const zkdl_mat* b, int trans_a, int trans_b, const float* sa, const float* sb,
                      const zkdl_mat* out) {
    if (out->stack == 0 || out->rows == 0 || out->cols == 0) return ZKDL_OK;
    M8Args p;
    p.a = (const int8_t*)a->data;
    p.b = (const int8_t*)b->data;
    p.a_rs = a->row_stride;
    p.a_ss = a->stack_stride;
    p.b_rs = b->row_stride;
    p.b_ss = b->stack_stride;
    p.out = out->data;
    p.o_rs = out->row_stride;
    p.o_ss = out->stack_stride;
    p.o_type = out->dtype;
    p.sa = sa;
    p.sb = sb;
    p.M = (uint32_t)out->rows;
    p.N = (uint32_t)out->cols;
    p.K = (uint32_t)(trans_a ? a->rows : a->cols);
    return m8_launch(ctx, p, trans_a != 0, trans_b == 0, out->stack);
}

// sums of this many products of magnitude 2^14 stay within 31 bits
constexpr uint64_t M8_MAX_K = ((uint64_t)1 << 17) - 1;

extern "C" int zkdl_matmul_i8(zkdl_ctx* ctx, const zkdl_mat* a, const zkdl_mat* b, int trans_a, int trans_b, const float* a_scale,
                              const float* b_scale, const zkdl_mat* out) try {
    if (!ctx || !l8_mat_ok(a, false) || !l8_mat_ok(b, false) || !l8_mat_ok(out, true) || a->dtype != ZKDL_I8 || b->dtype != ZKDL_I8)
        return ZKDL_EINVAL;
    if (out->dtype != ZKDL_I32 && !l8_is_float(out->dtype)) return ZKDL_EINVAL;
    if (out->dtype == ZKDL_I32 && (a_scale || b_scale)) return ZKDL_EINVAL;
    const uint64_t m = trans_a ? a->cols : a->rows, k = trans_a ? a->rows : a->cols, kb = trans_b ? b->cols : b->rows,
                   n = trans_b ? b->rows : b->cols;
    if (k != kb || out->rows != m || out->cols != n || a->stack != b->stack || out->stack != a->stack) return ZKDL_EINVAL;
    if (k > M8_MAX_K) return ZKDL_ETOOBIG;
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    const int rc = m8_product(ctx, a, b, trans_a, trans_b, a_scale, b_scale, out);
    if (rc != ZKDL_OK) return rc;
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}

extern "C" int zkdl_matmul_i8_backward(zkdl_ctx* ctx, const zkdl_mat* dy, const zkdl_mat* a, const zkdl_mat* w, int trans_w,
                                       const float* a_scale, const float* w_scale, const zkdl_mat* da, const zkdl_mat* dw) try {
    if (!ctx || !l8_mat_ok(dy, false) || !l8_mat_ok(a, false) || !l8_mat_ok(w, false) || !l8_is_float(dy->dtype) || a->dtype != ZKDL_I8 ||
        w->dtype != ZKDL_I8)
        return ZKDL_EINVAL;
    const uint64_t m = a->rows, k = a->cols, n = trans_w ? w->rows : w->cols, kw = trans_w ? w->cols : w->rows, st = dy->stack;
    if (kw != k || dy->rows != m || dy->cols != n || a->stack != st || w->stack != st) return ZKDL_EINVAL;
    if (da && (!l8_mat_ok(da, true) || da->dtype != dy->dtype || !l8_same_shape(da, a))) return ZKDL_EINVAL;
    if (dw && (!l8_mat_ok(dw, true) || dw->dtype != ZKDL_F32 || !l8_same_shape(dw, w))) return ZKDL_EINVAL;
    if (m > M8_MAX_K || n > M8_MAX_K) return ZKDL_ETOOBIG;
    if (st == 0 || (!da && !dw)) return ZKDL_OK;
    if ((m && !a_scale) || (n && !w_scale)) return ZKDL_EINVAL;
    L8Device dev(ctx);
    ZK_HIP(ctx, dev.err);
    // the quantised gradient: rows of whole 16 bytes
    const uint64_t pitch = l8_ceil(n ? n : 1, 16) * 16;
    int8_t* q = (int8_t*)zk_alloc(ctx, st * m * pitch);
    float* scale = q ? (float*)zk_alloc(ctx, st * (m > n ? m : n) * 4) : nullptr;
    int rc = q && scale ? ZKDL_OK : ZKDL_ENOMEM;
    const zkdl_mat mq = {q, st, m, n, pitch, m * pitch, ZKDL_I8, 0};
    if (rc == ZKDL_OK && da) {
        if (m && n) rc = zk_quantize_i8(ctx, dy, 1, w_scale, &mq, scale, nullptr);
        if (rc == ZKDL_OK) rc = m8_product(ctx, &mq, w, 0, !trans_w, n ? scale : nullptr, nullptr, da);
    }
    if (rc == ZKDL_OK && dw) {
        if (m && n) rc = zk_quantize_i8(ctx, dy, 0, a_scale, &mq, scale, nullptr);
        if (rc == ZKDL_OK) {
            if (trans_w) rc = m8_product(ctx, &mq, a, 1, 0, m ? scale : nullptr, nullptr, dw);
            else rc = m8_product(ctx, a, &mq, 1, 0, nullptr, m ? scale : nullptr, dw);
        }
    }
    zk_free(ctx, scale);
    zk_free(ctx, q);
    if (rc != ZKDL_OK) return rc;
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}
