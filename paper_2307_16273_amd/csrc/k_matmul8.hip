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
    int o_vec;                         // four adjacent items may be stored at once
    const float *sa, *sb;
    uint32_t M, N, K;
};

// The block's tile: matrix, first row, first column.  Blocks go round the eight dies; each die takes a run of tiles that lie together,
// eight rows of tiles at a time, so that its L2 serves a tile's neighbours.
static __device__ __forceinline__ void m8_tile(const M8Args& p, uint32_t bm, uint32_t bn, uint64_t& s, uint32_t& m0, uint32_t& n0) {
    const uint32_t gm = (p.M + bm - 1) / bm, gn = (p.N + bn - 1) / bn, run = gridDim.x / 8;
    uint32_t id = blockIdx.x;
    if (id < run * 8) id = id % 8 * run + id / 8;
    s = id / (gm * gn);
    id %= gm * gn;
    const uint32_t first = id / (8 * gn) * 8, rows = min(gm - first, 8u), at = id - first * gn;
    m0 = (first + at % rows) * bm;
    n0 = at / rows * bn;
}

template <class T>
struct alignas(4 * sizeof(T)) M8Four {
    T v[4];
};
// Four adjacent columns of a row: the accumulators, or (acc sa) sb, each product rounded to 32 bits and once more to out's type.
template <class T>
static __device__ __forceinline__ void m8_store4(T* o, int n, bool vec, const v4i& acc, float sa, const float (&sb)[4]) {
    M8Four<T> x;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (__is_same(T, int)) x.v[e] = acc[e];
        else l8_put((float)acc[e] * sa * sb[e], x.v[e]);
    }
    if (vec && n >= 4) {
        *(M8Four<T>*)o = x;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) o[e] = x.v[e];
    }
}
// A wave's fragments, 16 rows and 16 columns apart; the lane's first row and column are (i, j): the products come out turned, so that a
// lane has four adjacent columns of one row.  inside: no fragment crosses an edge and items may be stored by fours.  All scales are read
// before the first store: a load behind stores waits for them.
template <class T, int FM, int FN>
static __device__ __forceinline__ void m8_store_as(const M8Args& p, uint64_t s, uint32_t i, uint32_t j, bool inside, const v4i (&acc)[FM][FN]) {
    float sa[FM], sb[FN][4];
#pragma unroll
    for (int x = 0; x < FM; ++x) sa[x] = 1.f;
#pragma unroll
    for (int y = 0; y < FN; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) sb[y][e] = 1.f;
    if constexpr (!__is_same(T, int)) {
        if (p.sa) {
            const float* q = p.sa + s * p.M;
#pragma unroll
            for (int x = 0; x < FM; ++x) sa[x] = q[min(i + x * 16, p.M - 1)];
        }
        if (p.sb) {
            const float* q = p.sb + s * p.N;
#pragma unroll
            for (int y = 0; y < FN; ++y)
#pragma unroll
                for (int e = 0; e < 4; ++e) sb[y][e] = q[min(j + y * 16 + e, p.N - 1)];
        }
    }
    T* o = (T*)p.out + s * p.o_ss + i * p.o_rs + j;
    if (inside) {
#pragma unroll
        for (int x = 0; x < FM; ++x)
#pragma unroll
            for (int y = 0; y < FN; ++y) m8_store4(o + x * 16 * p.o_rs + y * 16, 4, true, acc[x][y], sa[x], sb[y]);
    } else {
#pragma unroll
        for (int x = 0; x < FM; ++x)
#pragma unroll
            for (int y = 0; y < FN; ++y)
                if (i + x * 16 < p.M && j + y * 16 < p.N)
                    m8_store4(o + x * 16 * p.o_rs + y * 16, (int)min(p.N - j - y * 16, 4u), p.o_vec != 0, acc[x][y], sa[x], sb[y]);
    }
}
template <int FM, int FN>
static __device__ __forceinline__ void m8_store_tile(const M8Args& p, uint64_t s, uint32_t i, uint32_t j, bool inside, const v4i (&acc)[FM][FN]) {
    switch (p.o_type) {
        case ZKDL_I32: m8_store_as<int>(p, s, i, j, inside, acc); break;
        case ZKDL_F32: m8_store_as<float>(p, s, i, j, inside, acc); break;
        case ZKDL_F16: m8_store_as<__half>(p, s, i, j, inside, acc); break;
        default: m8_store_as<bf16_t>(p, s, i, j, inside, acc);
    }
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
    m8_store_tile<2, 2>(p, s, m0 + wm + i16, n0 + wn + g * 4, false, acc);
}

// ---------------------------------------------------------------------------
// Tiles whose operands lie at multiples of 16 bytes: the memory system writes them into LDS by itself (16 bytes a lane, in
// the order of the lanes), a stage of 128 k while the one before it is multiplied.  A lane chooses which 16 bytes it fetches, so
// that the rows of a fragment lie in different banks: chunk c of row r stands at c ^ swizzle(r).
// ---------------------------------------------------------------------------
static __device__ __align__(16) const uint32_t m8_zeros[4] = {0, 0, 0, 0};
typedef const __attribute__((address_space(1))) void* glb_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;

// An operand's tile: R rows of op(A) (columns of op(B)), BK = 128 k, for T threads.  TURN: memory runs along the rows.
template <int R, bool TURN, int T>
struct M8Tile {
    static constexpr int BK = 128, BYTES = R * BK, LOADS = BYTES / 16 / T, CHUNKS = (TURN ? R : BK) / 16;
    uint32_t off[LOADS];
    // The banks hold 256 bytes, and a quarter wave's reads are to cover them: 16 rows' chunks of 16 bytes each, of two
    // groups of lanes
    static __device__ __forceinline__ uint32_t swizzle(uint32_t r) {
        if (!TURN) return (r >> 1) & 7;
        if (CHUNKS >= 16) return (r & 7) | ((r >> 4) & 1) << 3;
        if (CHUNKS == 8) return ((r >> 1) & 3) | ((r >> 4) & 1) << 2;
        return ((r >> 2) & 1) | ((r >> 4) & 1) << 1;
    }
    static __device__ __forceinline__ void place(uint32_t i, uint32_t t, uint32_t& r, uint32_t& c) {
        const uint32_t at = i * T + t;
        r = at / CHUNKS;
        c = ((at % CHUNKS) ^ swizzle(r)) * 16;
    }
    // rows: how many of the tile's there are; the last ones stand in for those that are not (their sums are not stored)
    __device__ __forceinline__ void init(uint32_t t, uint64_t rs, uint32_t rows) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            uint32_t r, c;
            place(i, t, r, c);
            off[i] = TURN ? (uint32_t)(r * rs) + min(c, rows - 16) : (uint32_t)(min(r, rows - 1) * rs) + c;
        }
    }
    __device__ __forceinline__ void load(const int8_t* p, int8_t* lds, uint32_t w) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) __builtin_amdgcn_global_load_lds((glb_ptr)(p + off[i]), (lds_ptr)(lds + (i * T + w * 64) * 16), 16, 0, 0);
    }
    // the last stage: zeros from k = `left` on
    __device__ __forceinline__ void load_part(const int8_t* p, int8_t* lds, uint32_t w, uint32_t t, uint32_t left) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            uint32_t r, c;
            place(i, t, r, c);
            const int8_t* q = (TURN ? r : c) < left ? p + off[i] : (const int8_t*)m8_zeros;
            __builtin_amdgcn_global_load_lds((glb_ptr)q, (lds_ptr)(lds + (i * T + w * 64) * 16), 16, 0, 0);
        }
    }
    // the fragment of rows at .. at + 15, k from 64 kk on
    static __device__ __forceinline__ v4i frag(const int8_t* lds, uint32_t at, int kk, uint32_t g, uint32_t i16) {
        if constexpr (!TURN) {
            const uint32_t r = at + i16;
            return *(const v4i*)(lds + r * BK + (((kk * 4 + g) ^ swizzle(r)) * 16));
        } else {
            v4i f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t r = kk * 64 + 16 * g + 8 * h + (i16 >> 1);
                const v2i y = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i*)(lds + r * R + (((at >> 4) ^ swizzle(r)) * 16) + (i16 & 1) * 8));
                f[2 * h] = y[0];
                f[2 * h + 1] = y[1];
            }
            return f;
        }
    }
};

template <int BM, int BN, int WM, int WN, int STAGES, bool AT, bool BT>
__global__ __launch_bounds__(WM * WN * 64) void k_m8_tile(M8Args p) {
    constexpr int T = WM * WN * 64, FM = BM / WM / 16, FN = BN / WN / 16;
    using OA = M8Tile<BM, AT, T>;
    using OB = M8Tile<BN, BT, T>;
    constexpr int STAGE = OA::BYTES + OB::BYTES, LOADS = OA::LOADS + OB::LOADS;
    __shared__ __align__(16) int8_t lds[STAGES * STAGE];
    const uint32_t t = threadIdx.x, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), g = l >> 4, i16 = l & 15;
    uint64_t s;
    uint32_t m0, n0;
    m8_tile(p, BM, BN, s, m0, n0);
    const uint32_t wm = w / WN * (BM / WM), wn = w % WN * (BN / WN);
    OA oa;
    OB ob;
    oa.init(t, p.a_rs, min(p.M - m0, (uint32_t)BM));
    ob.init(t, p.b_rs, min(p.N - n0, (uint32_t)BN));
    const int8_t* pa = p.a + s * p.a_ss + (AT ? (uint64_t)m0 : m0 * p.a_rs);
    const int8_t* pb = p.b + s * p.b_ss + (BT ? (uint64_t)n0 : n0 * p.b_rs);
    const uint64_t step_a = AT ? 128 * p.a_rs : 128, step_b = BT ? 128 * p.b_rs : 128;
    const uint32_t stages = (p.K + 127) / 128;
    uint32_t ahead = 0, in = 0, out = 0;
    auto load = [&]() {
        if (ahead < stages) {
            int8_t* q = lds + in * STAGE;
            const uint32_t left = p.K - ahead * 128;
            if (left >= 128) {
                oa.load(pa, q, w);
                ob.load(pb, q + OA::BYTES, w);
            } else {
                oa.load_part(pa, q, w, t, left);
                ob.load_part(pb, q + OA::BYTES, w, t, left);
            }
            pa += step_a;
            pb += step_b;
            in = in == STAGES - 1 ? 0 : in + 1;
        }
        ++ahead;
    };
    v4i acc[FM][FN] = {};
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) load();
    for (uint32_t k = 0; k < stages; ++k) {
        // stage k has landed when no more is under way than the stages behind it; then everybody has also left stage k - 1
        if (STAGES > 2 && stages - 1 - k >= STAGES - 2) {
            constexpr int V = (STAGES - 2) * LOADS;
            static_assert(V < 64, "counts to 63");
            __builtin_amdgcn_s_waitcnt(0x0f70 | (V & 15) | (V >> 4) << 14);
        } else {
            __builtin_amdgcn_s_waitcnt(0x0f70);
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        load();
        const int8_t* la = lds + out * STAGE;
        const int8_t* lb = la + OA::BYTES;
        out = out == STAGES - 1 ? 0 : out + 1;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            v4i fa[FM], fb[FN];
#pragma unroll
            for (int y = 0; y < FN; ++y) fb[y] = OB::frag(lb, wn + y * 16, kk, g, i16);
#pragma unroll
            for (int x = 0; x < FM; ++x) fa[x] = OA::frag(la, wm + x * 16, kk, g, i16);
            __builtin_amdgcn_s_setprio(1);      // the wave whose operands are there goes first: the others read meanwhile
#pragma unroll
            for (int x = 0; x < FM; ++x)
#pragma unroll
                for (int y = 0; y < FN; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[y], fa[x], acc[x][y], 0, 0, 0);
            __builtin_amdgcn_s_setprio(0);
        }
    }
    m8_store_tile<FM, FN>(p, s, m0 + wm + i16, n0 + wn + g * 4, p.o_vec && m0 + BM <= p.M && n0 + BN <= p.N, acc);
}

// ---------------------------------------------------------------------------
// Few rows (a batch of tokens): bound by reading op(B) once.  A block has 16 FM rows and 16 NC columns and its eight waves share out
// k, 64 at a time; operands go straight into registers (op(B) through a wave's own piece of LDS where it has to be turned), many
// loads under way at once, and the waves' sums are added at the end.
// ---------------------------------------------------------------------------
template <int FM, int NC, int U, bool AT, bool BT>
__global__ __launch_bounds__(512) void k_m8_few(M8Args p) {
    constexpr int W = 8, BYTES = 1024 * NC;      // of a wave's tile of 64 k
    __shared__ __align__(16) int8_t turn[BT ? W * BYTES : 16];
    __shared__ __align__(16) int sums[W][FM * NC][64][4];
    const uint32_t t = threadIdx.x, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), g = l >> 4, i16 = l & 15;
    uint64_t s;
    uint32_t m0, n0;
    m8_tile(p, 16 * FM, 16 * NC, s, m0, n0);
    const int8_t *a = p.a + s * p.a_ss, *b = p.b + s * p.b_ss;
    v4i acc[FM][NC] = {};
    const uint32_t steps = (p.K + 63) / 64;
    int8_t* mine = turn + (BT ? w * BYTES : 0);
    for (uint32_t k0 = w; k0 < steps; k0 += W * U) {
        v4i fa[U][FM], fb[U][NC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t k = (k0 + u * W) * 64;
#pragma unroll
            for (int y = 0; y < NC; ++y) {
                if (BT) {       // 64 rows of k, 16 NC columns each: lane's piece
                    const uint32_t at = y * 64 + l, r = at / NC, c = at % NC * 16;
                    fb[u][y] = m8_fetch(b, p.b_rs, k + r, p.K, n0 + c, p.N);
                } else {
                    fb[u][y] = m8_fetch(b, p.b_rs, n0 + y * 16 + i16, p.N, k + g * 16, p.K);
                }
            }
#pragma unroll
            for (int x = 0; x < FM; ++x) {
                if (AT) {
                    const uint32_t i = m0 + x * 16 + i16;
                    v4i f = {0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint32_t kk = k + g * 16 + e;
                        if (i < p.M && kk < p.K) f[e / 4] |= (int)((uint32_t)(uint8_t)a[kk * p.a_rs + i] << (8 * (e % 4)));
                    }
                    fa[u][x] = f;
                } else {
                    fa[u][x] = m8_fetch(a, p.a_rs, m0 + x * 16 + i16, p.M, k + g * 16, p.K);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            v4i f[NC];
            if (BT) {
                // a wave's own LDS: its operations there keep their order
#pragma unroll
                for (int y = 0; y < NC; ++y) *(v4i*)(mine + (y * 64 + l) * 16) = fb[u][y];
                asm volatile("" ::: "memory");
#pragma unroll
                for (int y = 0; y < NC; ++y)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t r = 16 * g + 8 * h + (i16 >> 1);
                        const v2i z = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i*)(mine + r * (16 * NC) + y * 16 + (i16 & 1) * 8));
                        f[y][2 * h] = z[0];
                        f[y][2 * h + 1] = z[1];
                    }
                asm volatile("" ::: "memory");
            } else {
#pragma unroll
                for (int y = 0; y < NC; ++y) f[y] = fb[u][y];
            }
#pragma unroll
            for (int x = 0; x < FM; ++x)
#pragma unroll
                for (int y = 0; y < NC; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f[y], fa[u][x], acc[x][y], 0, 0, 0);
        }
    }
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < NC; ++y) *(v4i*)sums[w][x * NC + y][l] = acc[x][y];
    __syncthreads();
    // fragment f of the sums goes to wave f (mod 8)
#pragma unroll
    for (int f0 = 0; f0 < FM * NC; f0 += W) {
        const uint32_t f = f0 + w;
        if (f < FM * NC) {
            v4i v[1][1] = {};
#pragma unroll
            for (int q = 0; q < W; ++q) v[0][0] += *(const v4i*)sums[q][f][l];
            m8_store_tile<1, 1>(p, s, m0 + f / NC * 16 + i16, n0 + f % NC * 16 + g * 4, false, v);
        }
    }
}

// a launch's blocks are counted in 32 bits of threads
constexpr uint64_t M8_MAX_TILES = (uint64_t)1 << 23;

template <bool AT, bool BT>
static int m8_launch(zkdl_ctx* ctx, const M8Args& p, uint64_t stack, bool whole) {
    int bm = 64, bn = 64, threads = 256;
    void (*kernel)(M8Args) = k_m8_any<AT, BT>;
    auto tiles = [&](uint64_t m, uint64_t n) { return l8_ceil(p.M, m) * l8_ceil(p.N, n) * stack; };
    if (p.M <= 16) {
        constexpr int NC = BT ? 2 : 1;
        kernel = k_m8_few<1, NC, 8, AT, BT>;
        bm = 16, bn = 16 * NC, threads = 512;
    } else if (whole) {
        if (tiles(256, 256) >= 200) {
            kernel = k_m8_tile<256, 256, 2, 4, 2, AT, BT>;
            bm = bn = 256, threads = 512;
        } else if (tiles(128, 128) >= 200) {
            kernel = k_m8_tile<128, 128, 2, 2, 2, AT, BT>;
            bm = bn = 128;
        } else {
            kernel = k_m8_tile<64, 64, 2, 2, 4, AT, BT>;
        }
    }
    if (l8_ceil(p.M, bm) * l8_ceil(p.N, bn) >= M8_MAX_TILES || stack >= M8_MAX_TILES || tiles(bm, bn) >= M8_MAX_TILES) return ZKDL_ETOOBIG;
    hipLaunchKernelGGL(kernel, dim3((unsigned)tiles(bm, bn)), dim3(threads), 0, ctx->stream, p);
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
    const uint64_t item = out->dtype == ZKDL_I32 || out->dtype == ZKDL_F32 ? 4 : 2;
    p.o_vec = p.o_rs % 4 == 0 && (out->stack == 1 || p.o_ss % 4 == 0) && (uintptr_t)p.out % (4 * item) == 0;
    // operands that k_m8_tile can fetch: whole 16 bytes along memory, and rows of a tile within 32 bits
    auto whole = [&](const zkdl_mat* m) {
        return (uintptr_t)m->data % 16 == 0 && m->row_stride % 16 == 0 && (m->stack == 1 || m->stack_stride % 16 == 0) && m->cols % 16 == 0 &&
               m->row_stride < (uint64_t)1 << 23;
    };
    const bool w = p.K > 0 && whole(a) && whole(b);
    if (trans_a && !trans_b) return m8_launch<true, true>(ctx, p, out->stack, w);
    if (trans_a) return m8_launch<true, false>(ctx, p, out->stack, w);
    if (!trans_b) return m8_launch<false, true>(ctx, p, out->stack, w);
    return m8_launch<false, false>(ctx, p, out->stack, w);
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
