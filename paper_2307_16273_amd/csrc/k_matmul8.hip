// Products of 8-bit integers with exact 32-bit accumulators on the matrix cores (zkdl_matmul_i8, zkdl_matmul_i8_backward).
//
// v_mfma_i32_16x16x64_i8 takes 64 products of each of 16 x 16 entries; a lane holds 16 adjacent k of one row of op(A) and of
// one column of op(B).  An operand whose memory runs along k is read that way (16 bytes a lane); for the other layout a tile
// stands in LDS as it does in memory, row by row of k, and ds_read_b64_tr_b8 turns 8 x 16 bytes while it reads them: in each
// group of 16 lanes, lanes 2r and 2r+1 point at 16 bytes of row r and lane c receives the eight bytes of column c.
#include "layer8.cuh"

typedef int v2i __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v2i lds_v2i;

struct M8Args {
    const int8_t *a, *b;
    uint64_t a_rs, a_ss, b_rs, b_ss;   // strides of the stored matrices, bytes
    void* out;
    uint64_t o_rs, o_ss;               // items
    int o_type;                        // zkdl_dtype
    const float *sa, *sb;
    uint32_t M, N, K;
    uint32_t all;       // not 0: the matrices of the stack are slices of K out of so many k, the last one what is left
};

// The block's tile: matrix, first row, first column.  Blocks go round the eight dies; each die takes a run of tiles that lie together,
// eight rows of tiles at a time, so that its L2 serves a tile's neighbours.
static __device__ __forceinline__ void m8_tile(const M8Args& p, uint32_t bm, uint32_t bn, uint32_t id, uint32_t blocks, uint64_t& s, uint32_t& m0,
                                               uint32_t& n0) {
    const uint32_t gm = (p.M + bm - 1) / bm, gn = (p.N + bn - 1) / bn, run = blocks / 8;
    if (id < run * 8) id = id % 8 * run + id / 8;
    s = id / (gm * gn);
    id %= gm * gn;
    const uint32_t first = id / (8 * gn) * 8, rows = min(gm - first, 8u), at = id - first * gn;
    m0 = (first + at % rows) * bm;
    n0 = at / rows * bn;
}

template <class T>
struct __attribute__((packed, aligned(1))) M8Four {      // at any address
    T v[4];
};
// Four adjacent columns of a row: the accumulators, or (acc sa) sb, each product rounded to 32 bits and once more to out's type.
template <class T>
static __device__ __forceinline__ void m8_store4(T* o, int n, const v4i& acc, float sa, const float (&sb)[4]) {
    M8Four<T> x;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        T y;
        if constexpr (__is_same(T, int)) y = acc[e];
        else l8_put((float)acc[e] * sa * sb[e], y);
        x.v[e] = y;
    }
    if (n >= 4) {
        *(M8Four<T>*)o = x;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) o[e] = x.v[e];
    }
}
// A wave's fragments, 16 rows and 16 columns apart; the lane's first row and column are (i, j): the products come out turned, so that a
// lane has four adjacent columns of one row.  inside: no fragment crosses an edge.  All scales are read
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
    if constexpr (sizeof(T) == 2 && FN % 2 == 0) {
        if (inside) {
            // Of two fragments side by side every other sixteen lanes' columns change places, so that a lane has eight adjacent ones and
            // stores 16 bytes (us, 8 / 16 bytes a lane: 8192 x 4096 x 4096 126 / 118, 8192 x 128 x 8192 45 / 35, 4718 x 31 x 4544 25.5 / 21.4).
            const uint32_t odd = (threadIdx.x >> 4) & 1;
            T* q = o + (odd ? 12 : 0);
#pragma unroll
            for (int x = 0; x < FM; ++x)
#pragma unroll
                for (int y = 0; y < FN; y += 2) {
                    uint32_t v[2][2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        M8Four<T> f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) l8_put((float)acc[x][y + h][e] * sa[x] * sb[y + h][e], f.v[e]);
                        __builtin_memcpy(v[h], &f, 8);
                    }
                    M8Bytes w;
#pragma unroll
                    for (int d = 0; d < 2; ++d) {
                        const auto r = __builtin_amdgcn_permlane16_swap(v[0][d], v[1][d], false, false);
                        w.v[d] = r[0];
                        w.v[2 + d] = r[1];
                    }
                    *(M8Bytes*)(q + x * 16 * p.o_rs + y * 16) = w;
                }
            return;
        }
    }
    if (inside) {
#pragma unroll
        for (int x = 0; x < FM; ++x)
#pragma unroll
            for (int y = 0; y < FN; ++y) m8_store4(o + x * 16 * p.o_rs + y * 16, 4, acc[x][y], sa[x], sb[y]);
    } else {
#pragma unroll
        for (int x = 0; x < FM; ++x)
#pragma unroll
            for (int y = 0; y < FN; ++y)
                if (i + x * 16 < p.M && j + y * 16 < p.N)
                    m8_store4(o + x * 16 * p.o_rs + y * 16, (int)min(p.N - j - y * 16, 4u), acc[x][y], sa[x], sb[y]);
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
    // rows: how many of the tile's there are; the last ones stand in for those that are not (their sums are not stored).  Along memory
    // they come in whole 16s.
    __device__ __forceinline__ void init(uint32_t t, uint64_t rs, uint32_t rows) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            uint32_t r, c;
            place(i, t, r, c);
            off[i] = TURN ? (uint32_t)(r * rs) + min(c, ((rows + 15) & ~15u) - 16) : (uint32_t)(min(r, rows - 1) * rs) + c;
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

// BM x BN entries, WM x WN waves.  256 x 256 with 8 waves of 128 x 64: 8192 x 4096 x 4096 in 117 to 119 us whatever the layouts, 2.3 POP/s;
// the products alone, nothing loaded or read, take 95 us (85 on zeros: the clock gives way), so what is left is the loads' and LDS' share
// (a stage is 2048 cycles of products, and 1536 of fragments and 512 of loads in LDS) and a tile's first loads and last stores.
template <int BM, int BN, int WM, int WN, int STAGES, bool AT, bool BT>
static __device__ __forceinline__ void m8_tile_block(const M8Args& p, int8_t* lds, uint32_t block, uint32_t blocks) {
    constexpr int T = WM * WN * 64, FM = BM / WM / 16, FN = BN / WN / 16;
    using OA = M8Tile<BM, AT, T>;
    using OB = M8Tile<BN, BT, T>;
    constexpr int STAGE = OA::BYTES + OB::BYTES, LOADS = OA::LOADS + OB::LOADS;
    constexpr bool BIG = FM * FN > 16;
    const uint32_t t = threadIdx.x, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), g = l >> 4, i16 = l & 15;
    uint64_t s;
    uint32_t m0, n0;
    m8_tile(p, BM, BN, block, blocks, s, m0, n0);
    const uint32_t K = p.all ? min(p.K, p.all - (uint32_t)s * p.K) : p.K;
    const uint32_t wm = w / WN * (BM / WM), wn = w % WN * (BN / WN);
    OA oa;
    OB ob;
    oa.init(t, p.a_rs, min(p.M - m0, (uint32_t)BM));
    ob.init(t, p.b_rs, min(p.N - n0, (uint32_t)BN));
    const uint64_t step_a = AT ? 128 * p.a_rs : 128, step_b = BT ? 128 * p.b_rs : 128;
    const uint32_t stages = (K + 127) / 128;
    const int8_t* pa = p.a + s * p.a_ss + (AT ? (uint64_t)m0 : m0 * p.a_rs);
    const int8_t* pb = p.b + s * p.b_ss + (BT ? (uint64_t)n0 : n0 * p.b_rs);
    uint32_t ahead = 0, in = 0, out = 0;
    auto load = [&]() {
        if (ahead < stages) {
            int8_t* q = lds + in;
            const uint32_t left = K - ahead * 128;
            if (left >= 128) {
                oa.load(pa, q, w);
                ob.load(pb, q + OA::BYTES, w);
            } else {
                oa.load_part(pa, q, w, t, left);
                ob.load_part(pb, q + OA::BYTES, w, t, left);
            }
            pa += step_a;
            pb += step_b;
            in = in == (STAGES - 1) * STAGE ? 0 : in + STAGE;
        }
        ++ahead;
    };
    v4i acc[FM][FN] = {};
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) load();
    for (uint32_t k = 0; k < stages; ++k) {
        // stage k has landed when no more is under way than the stages behind it
        if (STAGES > 2 && stages - 1 - k >= STAGES - 2) {
            constexpr int V = (STAGES - 2) * LOADS;
            static_assert(V < 64, "counts to 63");
            __builtin_amdgcn_s_waitcnt(0x0f70 | (V & 15) | (V >> 4) << 14);
        } else {
            __builtin_amdgcn_s_waitcnt(0x0f70);
        }
        // Behind the barrier everybody has left stage k - 1, which the next loads write over: this wave's reads of it have arrived (lgkmcnt 0;
        // its products have used them, but the compiler may move products behind the barrier).
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xc07f);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int8_t* la = lds + out;
        const int8_t* lb = la + OA::BYTES;
        out = out == (STAGES - 1) * STAGE ? 0 : out + STAGE;
        v4i fa[2][FM], fb[2][FN];
        auto frags = [&](int q) {
#pragma unroll
            for (int y = 0; y < FN; ++y) fb[q][y] = OB::frag(lb, wn + y * 16, q, g, i16);
#pragma unroll
            for (int x = 0; x < FM; ++x) fa[q][x] = OA::frag(la, wm + x * 16, q, g, i16);
        };
        auto mul = [&](int q) {
            if (BIG) __builtin_amdgcn_s_setprio(1);      // the wave whose operands are there goes first: the others read meanwhile
#pragma unroll
            for (int x = 0; x < FM; ++x)
#pragma unroll
                for (int y = 0; y < FN; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[q][y], fa[q][x], acc[x][y], 0, 0, 0);
            if (BIG) __builtin_amdgcn_s_setprio(0);
        };
        // Fragments come before the next stage's loads, whose addresses are worked out while they are on their way; both halves of a
        // stage's where they fit the registers beside the sums.  8192 x 4096 x 4096, us, loads first / like this: op(A) op(B) along k
        // 122 / 115, op(B) across 137 / 111, both across 140 / 114; 128 x 128 tiles 135 / 123, 158 / 127, 160 / 131.
        frags(0);
        if (!BIG) frags(1);
        load();
        mul(0);
        if (BIG) frags(1);
        mul(1);
    }
    m8_store_tile<FM, FN>(p, s, m0 + wm + i16, n0 + wn + g * 4, m0 + BM <= p.M && n0 + BN <= p.N, acc);
}

template <int BM, int BN, int WM, int WN, int STAGES, bool AT, bool BT>
__global__ __launch_bounds__(WM * WN * 64) void k_m8_tile(M8Args p) {
    __shared__ __align__(16) int8_t lds[STAGES * (BM + BN) * 128];
    m8_tile_block<BM, BN, WM, WN, STAGES, AT, BT>(p, lds, blockIdx.x, gridDim.x);
}

// The two products of a small layer's gradients in one launch: blocks for da, then for dw, whose operands both run across k.
struct M8Pair {
    M8Args da, dw;
    uint32_t da_blocks;
};
template <bool BT>
__global__ __launch_bounds__(256) void k_m8_pair(M8Pair p) {
    __shared__ __align__(16) int8_t lds[4 * 128 * 128];
    if (blockIdx.x < p.da_blocks) m8_tile_block<64, 64, 2, 2, 4, false, BT>(p.da, lds, blockIdx.x, p.da_blocks);
    else m8_tile_block<64, 64, 2, 2, 4, true, true>(p.dw, lds, blockIdx.x - p.da_blocks, gridDim.x - p.da_blocks);
}

// ---------------------------------------------------------------------------
// Small products, any address: bound by latency and by reading the operands once (one row through 4096 x 4096, output channels first: 5.4 us
// a call, 3.1 TB/s).  A block has 16 FM rows and 16 FN columns and its eight
// waves share out k, 64 at a time; U such steps are under way at once, straight into registers (through a wave's own piece of LDS where an
// operand has to be turned), and the waves' sums are added at the end.
// ---------------------------------------------------------------------------

// the 16 bytes moved towards the lower ones by sh, zeros behind them
static __device__ __forceinline__ v4i m8_shift(const v4i& f, uint32_t sh) {
    const uint64_t lo = (uint32_t)f[0] | (uint64_t)(uint32_t)f[1] << 32, hi = (uint32_t)f[2] | (uint64_t)(uint32_t)f[3] << 32;
    uint64_t nl = lo, nh = hi;
    if (sh >= 16) nl = nh = 0;
    else if (sh >= 8) nl = hi >> (8 * (sh - 8)), nh = 0;
    else if (sh) nl = lo >> (8 * sh) | hi << (64 - 8 * sh), nh = hi >> (8 * sh);
    return v4i{(int)(uint32_t)nl, (int)(uint32_t)(nl >> 32), (int)(uint32_t)nh, (int)(uint32_t)(nh >> 32)};
}

// A wave's share of one operand: F fragments of 16 rows of op(A) (columns of op(B)) from `at` on.  Loads wait for no branch: what lies
// behind an edge is read from inside the matrix and shifted out (along memory) or never stored.
template <int F, bool TURN>
struct M8Few {
    const int8_t* p;
    uint64_t rs;
    uint32_t at, rows, K, l;
    // whether that holds: at least 16 entries along memory
    __device__ __forceinline__ bool plain() const { return (TURN ? rows : K) >= 16; }
    // whether pieces of the tile cross the edge along memory
    __device__ __forceinline__ bool ragged() const { return TURN && at + 16 * F > rows; }
    __device__ __forceinline__ void load(uint32_t k, v4i (&f)[F]) const {
#pragma unroll
        for (int x = 0; x < F; ++x) {
            const int8_t* q;
            if (TURN) {
                const uint32_t piece = x * 64 + l;
                q = p + min(k + piece / F, K - 1) * rs + min(at + piece % F * 16, rows - 16);
            } else {
                q = p + min(at + x * 16 + (l & 15), rows - 1) * rs + min(k + (l >> 4) * 16, K - 16);
            }
            const M8Bytes y = *(const M8Bytes*)q;
#pragma unroll
            for (int i = 0; i < 4; ++i) f[x][i] = (int)y.v[i];
        }
    }
    __device__ __forceinline__ void load_guarded(uint32_t k, v4i (&f)[F]) const {
#pragma unroll
        for (int x = 0; x < F; ++x) {
            const uint32_t piece = x * 64 + l;
            f[x] = TURN ? m8_fetch(p, rs, k + piece / F, K, at + piece % F * 16, rows)
                        : m8_fetch(p, rs, at + x * 16 + (l & 15), rows, k + (l >> 4) * 16, K);
        }
    }
    // the last, partial step of load(): entries from K on become zeros
    __device__ __forceinline__ void cut(uint32_t k, v4i (&f)[F]) const {
#pragma unroll
        for (int x = 0; x < F; ++x) {
            if (TURN) {
                if (k + (x * 64 + l) / F >= K) f[x] = v4i{0, 0, 0, 0};
            } else {
                const uint32_t from = k + (l >> 4) * 16;
                f[x] = m8_shift(f[x], from + 16 > K ? from + 16 - K : 0);
            }
        }
    }
    // ragged(): the pieces to their places
    __device__ __forceinline__ void place(v4i (&f)[F]) const {
#pragma unroll
        for (int x = 0; x < F; ++x) {
            const uint32_t from = at + (x * 64 + l) % F * 16;
            f[x] = m8_shift(f[x], from + 16 > rows ? from + 16 - rows : 0);
        }
    }
    // turned: from pieces of rows of k to fragments, by way of the wave's own LDS, whose operations keep their order
    static __device__ __forceinline__ void turn(int8_t* mine, uint32_t l, v4i (&f)[F]) {
        if (!TURN) return;
        const uint32_t g = l >> 4, i16 = l & 15;
#pragma unroll
        for (int x = 0; x < F; ++x) *(v4i*)(mine + (x * 64 + l) * 16) = f[x];
        asm volatile("" ::: "memory");
#pragma unroll
        for (int x = 0; x < F; ++x)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v2i z = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i*)(mine + (16 * g + 8 * h + (i16 >> 1)) * (16 * F) + x * 16 + (i16 & 1) * 8));
                f[x][2 * h] = z[0];
                f[x][2 * h + 1] = z[1];
            }
        asm volatile("" ::: "memory");
    }
};

template <int FM, int FN, int U, bool AT, bool BT>
__global__ __launch_bounds__(512) void k_m8_few(M8Args p) {
    constexpr int W = 8, TURN_A = AT ? 1024 * FM : 0, TURN_B = BT ? 1024 * FN : 0, SUMS = FM * FN * 1024;
    __shared__ __align__(16) int8_t lds[W * (SUMS > TURN_A + TURN_B ? SUMS : TURN_A + TURN_B)];
    const uint32_t t = threadIdx.x, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), g = l >> 4, i16 = l & 15;
    uint64_t s;
    uint32_t m0, n0;
    m8_tile(p, 16 * FM, 16 * FN, blockIdx.x, gridDim.x, s, m0, n0);
    const M8Few<FM, AT> a = {p.a + s * p.a_ss, p.a_rs, m0, p.M, p.K, l};
    const M8Few<FN, BT> b = {p.b + s * p.b_ss, p.b_rs, n0, p.N, p.K, l};
    int8_t *turn_a = lds + w * (TURN_A + TURN_B), *turn_b = turn_a + TURN_A;
    v4i acc[FM][FN] = {};
    const uint32_t steps = (p.K + 63) / 64;
    auto mul = [&](v4i(&fa)[FM], v4i(&fb)[FN]) {
        M8Few<FM, AT>::turn(turn_a, l, fa);
        M8Few<FN, BT>::turn(turn_b, l, fb);
#pragma unroll
        for (int x = 0; x < FM; ++x)
#pragma unroll
            for (int y = 0; y < FN; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[y], fa[x], acc[x][y], 0, 0, 0);
    };
    if (a.plain() && b.plain()) {
        const bool ragged_a = a.ragged(), ragged_b = b.ragged();
        for (uint32_t k0 = w; k0 < steps; k0 += W * U) {
            v4i fa[U][FM], fb[U][FN];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                // (steps behind the end read the last one again: their k is looked at below)
                const uint32_t k = min(k0 + u * W, steps - 1) * 64;
                b.load(k, fb[u]);
                a.load(k, fa[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (k0 + u * W >= steps) break;
                const uint32_t k = (k0 + u * W) * 64;
                if (k + 64 > p.K) {
                    a.cut(k, fa[u]);
                    b.cut(k, fb[u]);
                }
                if (ragged_a) a.place(fa[u]);
                if (ragged_b) b.place(fb[u]);
                mul(fa[u], fb[u]);
            }
        }
    } else {
        for (uint32_t k0 = w; k0 < steps; k0 += W) {
            v4i fa[FM], fb[FN];
            a.load_guarded(k0 * 64, fa);
            b.load_guarded(k0 * 64, fb);
            mul(fa, fb);
        }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FN; ++y) *(v4i*)(lds + ((w * FM * FN + x * FN + y) * 64 + l) * 16) = acc[x][y];
    __syncthreads();
    // fragment f of the sums goes to wave f (mod 8)
#pragma unroll
    for (int f0 = 0; f0 < FM * FN; f0 += W) {
        const uint32_t f = f0 + w;
        if (f < FM * FN) {
            v4i v[1][1] = {};
#pragma unroll
            for (int q = 0; q < W; ++q) v[0][0] += *(const v4i*)(lds + ((q * FM * FN + f) * 64 + l) * 16);
            m8_store_tile<1, 1>(p, s, m0 + f / FN * 16 + i16, n0 + f % FN * 16 + g * 4, false, v);
        }
    }
}

// The sums of the slices of a long k, 32-bit integers [slices][M][N]: out = (their sum sa) sb
__global__ __launch_bounds__(256) void k_m8_join(M8Args p, const int* parts, uint32_t slices) {
    const uint32_t n4 = (p.N + 3) / 4;
    const uint64_t n = (uint64_t)p.M * n4, each = (uint64_t)p.M * p.N;
    for (uint64_t at = blockIdx.x * 256ull + threadIdx.x; at < n; at += gridDim.x * 256ull) {
        const uint32_t i = (uint32_t)(at / n4), j = (uint32_t)(at % n4) * 4;
        const int* q = parts + (uint64_t)i * p.N + j;
        v4i acc[1][1] = {};
        if (j + 4 <= p.N) {
#pragma unroll 8
            for (uint32_t s = 0; s < slices; ++s) {
                const M8Bytes x = *(const M8Bytes*)(q + s * each);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[0][0][e] += (int)x.v[e];
            }
        } else {
            for (uint32_t s = 0; s < slices; ++s)
                for (uint32_t e = 0; j + e < p.N; ++e) acc[0][0][e] += q[s * each + e];
        }
        m8_store_tile<1, 1>(p, 0, i, j, false, acc);
    }
}

__global__ __launch_bounds__(256) void k_m8_pack(M8PackArgs a) { m8_pack(a, blockIdx.x, gridDim.x); }

// a launch's blocks are counted in 32 bits of threads
constexpr uint64_t M8_MAX_TILES = (uint64_t)1 << 23;
enum M8Choice { M8_FEW1, M8_FEW2, M8_TILE64, M8_TILE128, M8_TILE256 };

template <bool AT, bool BT>
static int m8_launch(zkdl_ctx* ctx, const M8Args& p, uint64_t stack, int choice) {
    int bm = 0, bn = 0, threads = 0;
    void (*kernel)(M8Args) = nullptr;
    auto few = [&](void (*k)(M8Args), int fm, int fn) { kernel = k, bm = 16 * fm, bn = 16 * fn, threads = 512; };
    auto tile = [&](void (*k)(M8Args), int m, int n, int t) { kernel = k, bm = m, bn = n, threads = t; };
    switch (choice) {
        case M8_FEW1: few(k_m8_few<1, BT ? 2 : 1, 8, AT, BT>, 1, BT ? 2 : 1); break;
        case M8_FEW2: few(k_m8_few<2, 2, 4, AT, BT>, 2, 2); break;
        case M8_TILE64: tile(k_m8_tile<64, 64, 2, 2, 4, AT, BT>, 64, 64, 256); break;
        case M8_TILE128: tile(k_m8_tile<128, 128, 2, 2, 2, AT, BT>, 128, 128, 256); break;
        default: tile(k_m8_tile<256, 256, 2, 4, 2, AT, BT>, 256, 256, 512);
    }
    const uint64_t tiles = l8_ceil(p.M, bm) * l8_ceil(p.N, bn);
    if (tiles >= M8_MAX_TILES || stack >= M8_MAX_TILES || tiles * stack >= M8_MAX_TILES) return ZKDL_ETOOBIG;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles * stack)), dim3(threads), 0, ctx->stream, p);
    return ZKDL_OK;
}

// Which kernel.  whole: both operands can be fetched by k_m8_tile as they are; across: one of them does not run along k.  Times in us on
// the way back to back, launch included (a launch alone 4):
//  - up to 16 rows or columns, blocks of 16 (FEW1 / FEW2 / TILE64): 1 x 4096 x 4096 along k 5.7 / 7.5 / 10.8, across 9.2 / 9.2 / 16.5;
//  - up to 64 with an operand across and a long k, blocks of 32 (FEW2 / TILE64): 64 x 4096 x 4096 11.5 / 17.2, both along k 10.6 / 10.9;
//    not with more tiles (8 products of 64 x 1024 x 1024 9.9 / 5.4) or a k that is cut in slices (64 x 8192 x 4096 18 / 12);
//  - operands that have to be packed first, FEW2 / TILE64 with the packing: 64 x 4001 x 4001 23 / 27, 260 x 515 x 515 13 / 11 (along k),
//    10 / 12 (one across), 130 x 1001 x 1001 10 / 13, 260 x 1001 x 1001 17 / 13;
//  - pair: products that may share a launch by tiles of 64, which spares 3: gradients of (rows, in, out, tiles of 128 / the pair) 64 x 768 x 2944
//    19.5 / 14.9, 256 x 2048 x 2048 19.9 / 17.2, 3000 x 1000 x 700 48.7 / 45.3, but 1000 x 2000 x 2000 37.1 / 38.4;
//  - tiles of 64, 128, 256 (4096 x 4096 weights, along k): 256 rows 11 / 27 / 52, 512 16 / 28 / 53, 1024 30 / 30 / 55, 2048 58 / 36 / 57,
//    4096 114 / 66 / 61, 8192 208 / 128 / 114.  That is by how many fit the 256 compute units at once, two of the smaller ones each.
//  - operands that cannot be packed for the tiles (m8_packs) go to k_m8_few, which takes any strides.
static int m8_choose(uint64_t m, uint64_t n, uint64_t k, uint64_t stack, bool whole, bool across, bool packs = true, bool pair = false) {
    const uint64_t few = m < n ? m : n;
    if (few <= 16) return M8_FEW1;
    if (!packs) return M8_FEW2;
    auto tiles = [&](uint64_t x) { return l8_ceil(m, x) * l8_ceil(n, x) * stack; };
    const uint64_t t64 = tiles(64), t128 = tiles(128), t256 = tiles(256), work = m * n * k * stack;
    if (whole ? few <= 64 && across && k >= 2048 && k <= 4096 && t64 <= 64 : work <= (uint64_t)1 << (few <= 64 ? 30 : 27)) return M8_FEW2;
    const uint64_t c64 = t64 <= 256 ? 11 : 15 * l8_ceil(t64, 512), c128 = t128 <= 256 ? 28 : 34 * l8_ceil(t128, 512), c256 = 54 * l8_ceil(t256, 256);
    const uint64_t spare = pair && work <= (uint64_t)3 << 30 ? 3 : 0;
    return c64 <= c128 + spare && c64 <= c256 + spare ? M8_TILE64 : c128 <= c256 ? M8_TILE128 : M8_TILE256;
}

// How many slices of k tiles of 64 are worth, joined by a second launch: few tiles would leave most of the device idle over a long k.
// Whole calls (us, one launch / slices), both operands along k: 256 x 256 with k = 2048 6.7 / 7.5, 4096 10.6 / 8.2, 8192 18.6 / 8.7, 65536
// 129 / 15; 512 x 512 with k = 4096 10.6 / 12.0, 8192 18.7 / 13.2; 1024 x 1024 with k = 8192 19.2 / 19.4 (across 30.7 / 26.3), 65536 131 / 100.
// fresh: an operand that the launch before wrote, which comes from farther away: gradients of 64 x 768 x 2944 22.8 / 19.3 (23 stages of one
// of them), 4000 x 200 x 1000 47 / 41 (32), 4718 x 4544 x 31 51 / 45 (37).
// (A join inside the launch, by the last block of a tile, was no faster: what passes between the dies has to go past their caches.)
static uint64_t m8_slices(uint64_t m, uint64_t n, uint64_t k, bool fresh) {
    const uint64_t t64 = l8_ceil(m, 64) * l8_ceil(n, 64), stages = l8_ceil(k, 128);
    if (stages < (t64 <= 16 ? (fresh ? 16 : 24) : t64 <= 128 ? (fresh ? 20 : 40) : 64) || t64 > 256) return 1;
    uint64_t slices = 512 / t64;
    if (slices > stages / 4) slices = stages / 4;
    if (slices < 2) return 1;
    // every slice has entries: slices of whole stages, as many as those make
    return l8_ceil(k, l8_ceil(l8_ceil(k, slices), 128) * 128);
}

// Operands that k_m8_tile can fetch: whole 16 bytes along memory, rows of a tile within 32 bits.  Along k one of the two has to end in
// zeros or at a multiple of 16: a packed or a turned one does.
static bool m8_whole(const zkdl_mat* m, bool padded) {
    return (uintptr_t)m->data % 16 == 0 && m->row_stride % 16 == 0 && (m->stack == 1 || m->stack_stride % 16 == 0) && (padded || m->cols % 16 == 0) &&
           m->row_stride < (uint64_t)1 << 23;
}
// Whether a packed copy of so many columns is one that k_m8_tile can fetch.
static bool m8_packs(uint64_t cols) { return l8_ceil(cols, 16) * 16 < (uint64_t)1 << 23; }
// Memory for a packed copy of m, which is to be what args say; m becomes the copy.
static int m8_pack_for(zkdl_ctx* ctx, zkdl_mat* m, M8PackArgs* args) {
    if (!m8_packs(m->cols)) return ZKDL_ETOOBIG;
    const uint64_t pitch = l8_ceil(m->cols, 16) * 16;
    void* out = zk_alloc_scratch(ctx, m->stack * m->rows * pitch);
    if (!out) return ZKDL_ENOMEM;
    *args = {(const int8_t*)m->data, m->row_stride, m->stack_stride, m->rows, m->stack, pitch, (uint32_t)m->cols, (int8_t*)out};
    m->data = out;
    m->row_stride = pitch;
    m->stack_stride = m->rows * pitch;
    return ZKDL_OK;
}
static void m8_launch_pack(zkdl_ctx* ctx, const M8PackArgs& args) {
    const uint64_t blocks = l8_ceil(args.stack * args.rows * (args.pitch / 16), 256);
    hipLaunchKernelGGL(k_m8_pack, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, ctx->stream, args);
}
static M8Args m8_args(const zkdl_mat* out, uint32_t k, const float* sa, const float* sb) {
    M8Args p = {};
    p.out = out->data;
    p.o_rs = out->row_stride;
    p.o_ss = out->stack_stride;
    p.o_type = out->dtype;
    p.sa = sa;
    p.sb = sb;
    p.M = (uint32_t)out->rows;
    p.N = (uint32_t)out->cols;
    p.K = k;
    return p;
}
static void m8_operands(M8Args& p, const zkdl_mat* a, const zkdl_mat* b) {
    p.a = (const int8_t*)a->data;
    p.b = (const int8_t*)b->data;
    p.a_rs = a->row_stride;
    p.a_ss = a->stack_stride;
    p.b_rs = b->row_stride;
    p.b_ss = b->stack_stride;
}

// A product that tiles of 64 take in slices of k: p becomes their stack, whose 32-bit sums `parts` gets and m8_join adds up into what p was.
struct M8Slices {
    uint64_t count = 1;
    int* parts = nullptr;
    M8Args joined;
};
static int m8_slice(zkdl_ctx* ctx, M8Args& p, bool trans_a, bool trans_b, bool fresh, M8Slices& s) {
    s.count = m8_slices(p.M, p.N, p.K, fresh);
    s.joined = p;
    if (s.count == 1) return ZKDL_OK;
    s.parts = (int*)zk_alloc_scratch(ctx, s.count * p.M * p.N * 4);
    if (!s.parts) return ZKDL_ENOMEM;
    p.all = p.K;
    p.K = (uint32_t)(l8_ceil(l8_ceil(p.K, s.count), 128) * 128);
    p.a_ss = trans_a ? p.K * p.a_rs : p.K;
    p.b_ss = trans_b ? p.K : p.K * p.b_rs;
    p.out = s.parts;
    p.o_type = ZKDL_I32;
    p.o_rs = p.N;
    p.o_ss = (uint64_t)p.M * p.N;
    p.sa = p.sb = nullptr;
    return ZKDL_OK;
}
static void m8_join(zkdl_ctx* ctx, const M8Slices& s) {
    if (!s.parts) return;
    const uint64_t blocks = l8_ceil((uint64_t)s.joined.M * l8_ceil(s.joined.N, 4), 256);
    hipLaunchKernelGGL(k_m8_join, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, ctx->stream, s.joined, s.parts, (uint32_t)s.count);
}

// The product of operands as the chosen kernel wants them, a long k in slices.
static int m8_run(zkdl_ctx* ctx, M8Args p, bool trans_a, bool trans_b, uint64_t stack, bool fresh, int choice) {
    M8Slices sl;
    int rc = choice == M8_TILE64 && stack == 1 ? m8_slice(ctx, p, trans_a, trans_b, fresh, sl) : ZKDL_OK;
    if (rc != ZKDL_OK) return rc;
    stack *= sl.count;
    if (trans_a && !trans_b) rc = m8_launch<true, true>(ctx, p, stack, choice);
    else if (trans_a) rc = m8_launch<true, false>(ctx, p, stack, choice);
    else if (!trans_b) rc = m8_launch<false, true>(ctx, p, stack, choice);
    else rc = m8_launch<false, false>(ctx, p, stack, choice);
    if (rc == ZKDL_OK) m8_join(ctx, sl);
    zk_free(ctx, sl.parts);
    return rc;
}

// a and b behind the checks; out may be empty.  padded 1, 2: a, b is the context's own memory, whose rows go on to a multiple of 16.
static int m8_product(zkdl_ctx* ctx, const zkdl_mat* a, const zkdl_mat* b, int trans_a, int trans_b, const float* sa, const float* sb,
                      const zkdl_mat* out, int padded) {
    if (out->stack == 0 || out->rows == 0 || out->cols == 0) return ZKDL_OK;
    M8Args p = m8_args(out, (uint32_t)(trans_a ? a->rows : a->cols), sa, sb);
    const bool wa = m8_whole(a, padded == 1), wb = m8_whole(b, padded == 2);
    const bool packs = (wa || m8_packs(a->cols)) && (wb || m8_packs(b->cols));
    const int choice = p.K ? m8_choose(p.M, p.N, p.K, out->stack, wa && wb, trans_a || !trans_b, packs) : M8_FEW1;
    zkdl_mat pa = *a, pb = *b;
    void* packed[2] = {nullptr, nullptr};
    if (choice >= M8_TILE64) {
        for (int i = 0; i < 2; ++i) {
            if (i ? wb : wa) continue;
            M8PackArgs args;
            const int rc = m8_pack_for(ctx, i ? &pb : &pa, &args);
            if (rc != ZKDL_OK) {
                zk_free(ctx, packed[0]);
                return rc;
            }
            packed[i] = args.out;
            m8_launch_pack(ctx, args);
        }
    }
    m8_operands(p, &pa, &pb);
    const int rc = m8_run(ctx, p, trans_a != 0, trans_b != 0, out->stack, padded != 0, choice);
    zk_free(ctx, packed[0]);
    zk_free(ctx, packed[1]);
    return rc;
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
    const int rc = m8_product(ctx, a, b, trans_a, trans_b, a_scale, b_scale, out, 0);
    if (rc != ZKDL_OK) return rc;
    ZK_HIP(ctx, hipGetLastError());
    return ZKDL_OK;
} catch (...) {
    return ZKDL_ENOMEM;
}

static int m8_both_gradients(zkdl_ctx* ctx, const zkdl_mat* dy, const zkdl_mat* a, const zkdl_mat* w, int trans_w, const float* a_scale,
                             const float* w_scale, const zkdl_mat* da, const zkdl_mat* dw, int c_da, int c_dw) {
    const uint64_t m = dy->rows, n = dy->cols, pitch = l8_ceil(n, 16) * 16, codes = l8_ceil(m * pitch, 256) * 256;
    int8_t* mem = (int8_t*)zk_alloc_scratch(ctx, 2 * codes + (m + n) * 4);      // q, p, t, u
    if (!mem) return ZKDL_ENOMEM;
    const zkdl_mat q = {mem, 1, m, n, pitch, 0, ZKDL_I8, 0}, p = {mem + codes, 1, m, n, pitch, 0, ZKDL_I8, 0};
    L8Prepare job = {};
    job.dy = dy;
    job.q = &q;
    job.p = &p;
    job.a_scale = a_scale;
    job.w_scale = w_scale;
    job.t = (float*)(mem + 2 * codes);
    job.u = job.t + m;
    const bool one = zk_prepare_fits(dy), tiles64 = c_da <= M8_TILE64 && c_dw <= M8_TILE64;
    zkdl_mat pa = *a, pw = *w;
    int rc = ZKDL_OK;
    if (!one) rc = zk_quantize_both(ctx, job);
    if (!one && !tiles64) {
        if (rc == ZKDL_OK) rc = m8_product(ctx, &q, w, 0, !trans_w, job.t, nullptr, da, 1);
        if (rc == ZKDL_OK)
            rc = trans_w ? m8_product(ctx, &p, a, 1, 0, job.u, nullptr, dw, 1) : m8_product(ctx, a, &p, 1, 0, nullptr, job.u, dw, 2);
        zk_free(ctx, mem);
        return rc;
    }
    for (zkdl_mat* x : {&pa, &pw})
        if (rc == ZKDL_OK && !m8_whole(x, false)) {
            rc = m8_pack_for(ctx, x, &job.pack[job.packs]);
            if (rc == ZKDL_OK) ++job.packs;
        }
    if (rc == ZKDL_OK) {
        if (one) rc = zk_prepare(ctx, job);
        else
            for (int i = 0; i < job.packs; ++i) m8_launch_pack(ctx, job.pack[i]);
    }
    if (rc == ZKDL_OK) {
        M8Pair pair;
        pair.da = m8_args(da, (uint32_t)n, job.t, nullptr);
        m8_operands(pair.da, &q, &pw);
        pair.dw = m8_args(dw, (uint32_t)m, trans_w ? job.u : nullptr, trans_w ? nullptr : job.u);
        if (trans_w) m8_operands(pair.dw, &p, &pa);
        else m8_operands(pair.dw, &pa, &p);
        if (!tiles64) {
            rc = m8_run(ctx, pair.da, false, !trans_w, 1, true, c_da < M8_TILE64 ? M8_TILE64 : c_da);
            if (rc == ZKDL_OK) rc = m8_run(ctx, pair.dw, true, false, 1, true, c_dw < M8_TILE64 ? M8_TILE64 : c_dw);
        } else {
            M8Slices s_da, s_dw;
            rc = m8_slice(ctx, pair.da, false, !trans_w, true, s_da);
            if (rc == ZKDL_OK) rc = m8_slice(ctx, pair.dw, true, false, true, s_dw);
            const uint64_t b_da = l8_ceil(da->rows, 64) * l8_ceil(da->cols, 64) * s_da.count, b_dw = l8_ceil(dw->rows, 64) * l8_ceil(dw->cols, 64) * s_dw.count;
            if (rc == ZKDL_OK && (b_da >= M8_MAX_TILES || b_da + b_dw >= M8_MAX_TILES)) rc = ZKDL_ETOOBIG;
            if (rc == ZKDL_OK) {
                pair.da_blocks = (uint32_t)b_da;
                const dim3 grid((unsigned)(b_da + b_dw));
                if (trans_w) hipLaunchKernelGGL(k_m8_pair<true>, grid, dim3(256), 0, ctx->stream, pair);
                else hipLaunchKernelGGL(k_m8_pair<false>, grid, dim3(256), 0, ctx->stream, pair);
                m8_join(ctx, s_da);
                m8_join(ctx, s_dw);
            }
            zk_free(ctx, s_da.parts);
            zk_free(ctx, s_dw.parts);
        }
    }
    for (int i = 0; i < job.packs; ++i) zk_free(ctx, job.pack[i].out);
    zk_free(ctx, mem);
    return rc;
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
    // Both gradients of a small layer: everything in front of the products in one launch, and the products in another where both take tiles
    // of 64.  Whole calls (us, a launch for each step / like this), rows x in x out: 33 x 100 x 70 14.3 / 7.8, 64 x 1024 x 1024 15.1 / 9.7,
    // 333 x 1000 x 517 22.3 / 9.6, 1024 x 1024 x 1024 21.9 / 15.8, 1000 x 1000 x 1000 30.7 / 18.4.
    // Two reads of a larger gradient instead of three, (three / two): 2100 x 256 x 256 21.3 / 19.3, 4000 x 64 x 64 20.0 / 18.7, 3500 x 64 x 8000
    // 72.6 / 68.2, whose products share a launch; with larger tiles 2500 x 1000 x 1000 50.3 / 53.2, 4096 x 4096 x 4096 157.4 / 155.0,
    // 8192 x 1024 x 1024 77.7 / 65.8.
    if (da && dw && k && n && m && st == 1 && m8_packs(k)) {
        // (tiles of 64 for few rows as well: a product of their own kernel costs a launch more)
        const int c_da = m8_choose(m, k, n, 1, true, false, true, true), c_dw = m8_choose(dw->rows, dw->cols, m, 1, true, false, true, true);
        if (zk_prepare_fits(dy) || (zk_quantize_both_fits(dy) && (m >= 4096 || (c_da <= M8_TILE64 && c_dw <= M8_TILE64)))) {
            const int rc = m8_both_gradients(ctx, dy, a, w, trans_w, a_scale, w_scale, da, dw, c_da, c_dw);
            if (rc != ZKDL_OK) return rc;
            ZK_HIP(ctx, hipGetLastError());
            return ZKDL_OK;
        }
    }
    // the quantised gradient: rows of whole 16 bytes
    const uint64_t pitch = l8_ceil(n ? n : 1, 16) * 16;
    int8_t* q = (int8_t*)zk_alloc_scratch(ctx, st * m * pitch);
    float* scale = q ? (float*)zk_alloc_scratch(ctx, st * (m > n ? m : n) * 4) : nullptr;
    int rc = q && scale ? ZKDL_OK : ZKDL_ENOMEM;
    const zkdl_mat mq = {q, st, m, n, pitch, m * pitch, ZKDL_I8, 0};
    if (rc == ZKDL_OK && da) {
        if (m && n) rc = zk_quantize_i8(ctx, dy, 1, w_scale, &mq, scale, nullptr);
        if (rc == ZKDL_OK) rc = m8_product(ctx, &mq, w, 0, !trans_w, n ? scale : nullptr, nullptr, da, 1);
    }
    if (rc == ZKDL_OK && dw) {
        if (m && n) rc = zk_quantize_i8(ctx, dy, 0, a_scale, &mq, scale, nullptr);
        if (rc == ZKDL_OK) {
            if (trans_w) rc = m8_product(ctx, &mq, a, 1, 0, m ? scale : nullptr, nullptr, dw, 1);
            else rc = m8_product(ctx, a, &mq, 1, 0, nullptr, m ? scale : nullptr, dw, 2);
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
