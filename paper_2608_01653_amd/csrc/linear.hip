// INT8 products of token codes with linear weights, one layer or grouped by expert,
// and their epilogue: z = fma(float(acc), fl((s / b) w_scale), bias), the gated unit,
// one rounding to the output type.
//
// Operand roles: the weights are the MFMA's first operand, the tokens its second, so
// an accumulator lane holds one token and runs of four adjacent channels, which it
// stores as one piece.  The contraction index inside a 64-byte step is the same
// permutation on both sides, which an integer sum does not see.
#include "../../include/hatq.h"
#include "hatq_device.h"
#include "linear.h"
#include "linear_device.h"

namespace hatq {
namespace {

typedef int v16i __attribute__((ext_vector_type(16)));

#define HATQ_LDS(p) ((__attribute__((address_space(3))) void *)(p))
#define HATQ_GLOBAL(p) ((__attribute__((address_space(1))) const void *)(p))

// At most N of this wave's memory operations under way, none of its LDS reads.
template <int N>
__device__ __forceinline__ void wait_vmcnt_lds() {
    static_assert(N >= 0 && N < 64, "vmcnt");
    // s_waitcnt simm16 (gfx9): vmcnt[3:0], expcnt[6:4]=7, lgkmcnt[11:8]=0, vmcnt_hi[15:14]
    __builtin_amdgcn_s_waitcnt((N & 15) | 0x70 | ((N >> 4) << 14));
}

// A bare barrier (loads to LDS stay under way over it), and no access moved across it.
__device__ __forceinline__ void block_barrier() {
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// ---- which rows a tile has --------------------------------------------------------
struct RowTile {
    int expert;     // -1: rows past the last end, written 0
    int row0, end;  // rows [row0, min(row0 + BM, end))
};

// Row tiles of BM rows, each expert's rows starting a tile of their own, and the rows
// past the last end after them.  Every lane of the wave takes part, 64 experts at a
// time; the ends are clamped here, so any contents give rows in [0, rows).
template <int BM>
struct RowTiles {
    const LinearArgs &a;
    const int lane;
    int end, begin, n, first;   // this lane's expert of the 64 looked at last
    int last = 0, tiles = 0;    // rows and tiles up to the end of those

    __device__ RowTiles(const LinearArgs &args) : a(args), lane(threadIdx.x & 63) {}

    __device__ void look(int base) {
        const int i = base + lane;
        end = i < a.experts ? a.ends[i] : 0;
        end = wave_scan(max(min(end, a.rows), last), [](int x, int y) { return max(x, y); });
        begin = __builtin_amdgcn_update_dpp(0, end, 0x138, 0xF, 0xF, false);   // wave_shr 1
        if (lane == 0) begin = last;
        n = (end - begin + BM - 1) / BM;
        const int c = wave_scan(n, [](int x, int y) { return x + y; });
        first = tiles + c - n;
        last = __builtin_amdgcn_readlane(end, 63);
        tiles += __builtin_amdgcn_readlane(c, 63);
    }

    // All the row tiles.
    __device__ int total() {
        if (!a.ends) return (a.rows + BM - 1) / BM;
        for (int base = 0; base < a.experts; base += 64) look(base);
        return tiles + (a.rows - last + BM - 1) / BM;
    }

    // Tile t < total(), after total().
    __device__ RowTile find(int t) {
        if (!a.ends) return {0, t * BM, a.rows};
        if (t >= tiles) return {-1, last + (t - tiles) * BM, a.rows};
        const bool again = a.experts > 64;
        if (again) last = tiles = 0;
        for (int base = 0;; base += 64) {
            if (again) look(base);
            const uint64_t hit = __ballot(t >= first && t < first + n);
            if (hit) {
                const int l = __builtin_ctzll(hit);
                return {base + l, __builtin_amdgcn_readlane(begin, l) + (t - __builtin_amdgcn_readlane(first, l)) * BM,
                        __builtin_amdgcn_readlane(end, l)};
            }
        }
    }
};

// Upper bound of the row tiles over any ends (host).
int64_t most_row_tiles(const LinearArgs &a, int bm) {
    const int64_t full = (a.rows + bm - 1) / bm;
    if (!a.ends) return full;
    // each group adds at most one part tile, and there are at most `rows` groups
    const int64_t groups = a.experts + 1 < a.rows ? a.experts + 1 : a.rows;
    return a.rows / bm + groups;
}

// Token of an output row; -1 for an empty one.
__device__ __forceinline__ int token_of(const LinearArgs &a, int row) {
    if (!a.src) return row;
    const int t = a.src[row];
    return (unsigned)t < (unsigned)a.x_rows ? t : -1;
}

// ---- epilogue -----------------------------------------------------------------------
// g[j] = g[j] / (1 + exp(-g[j])) u[j], each operation as its fp32 function: the same bits as
// g / (1 + expf(-g)) u.  exp(-g) = 2^n 2^f: p = fl(-g log2 e), n = rne(p) in the low bits of
// p + 1.5 2^23, and f = (p - n) + the product's rest, so its error does not grow with |g|;
// |g| < 87 keeps 2^n 2^f normal and n its exponent's shift.  The quotient is g times the
// reciprocal with one step of correction.  Groups with a larger gate, an infinity or a NaN
// divide.  (The exponential and reciprocal alone, with p for n + f, lost up to 60 ulp at g =
// -80 and moved a code of the next layer now and then.  Whole call of 8192 x 4096 -> 2 x 8192: 516
// us with them, 529 so, 545 with the division for every element.)
__device__ __forceinline__ void gated4(float *g, const float *u) {
    float m = 0.0f, y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float p = g[j] * -1.44269504f, t = p + HATQ_MAGIC;
        // (log2 e = 1.44269504f + 1.92596303e-8f - 4.2e-16)
        const float f = __builtin_fmaf(g[j], -1.92596303e-8f, __builtin_fmaf(g[j], -1.44269504f, -p)) + (p - (t - HATQ_MAGIC));
        const float e = __uint_as_float((__float_as_uint(t) << 23) + __float_as_uint(__builtin_amdgcn_exp2f(f)));
        const float d = 1.0f + e, r = __builtin_amdgcn_rcpf(d), q = g[j] * r;
        y[j] = __builtin_fmaf(__builtin_fmaf(-q, d, g[j]), r, q);
        m = __builtin_elementwise_maximum(m, fabsf(g[j]));
    }
    if (!(m < 87.0f)) {
        asm volatile("");   // a branch: else the compiler divides for every group and selects
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = g[j] / (1.0f + expf(-g[j]));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = y[j] * u[j];
}

// z of four adjacent packed columns with factors at w_scale and bias (memory or LDS); s =
// the token's scale times 1/b, a power of two: exact unless it is below 2^-126.
__device__ __forceinline__ void dequant4(const float *w_scale, const float *bias, const int *acc, float s, float *z) {
    const float4 w = *reinterpret_cast<const float4 *>(w_scale), b = *reinterpret_cast<const float4 *>(bias);
    z[0] = __builtin_fmaf((float)acc[0], s * w.x, b.x);
    z[1] = __builtin_fmaf((float)acc[1], s * w.y, b.y);
    z[2] = __builtin_fmaf((float)acc[2], s * w.z, b.z);
    z[3] = __builtin_fmaf((float)acc[3], s * w.w, b.w);
}

template <typename T>
__device__ __forceinline__ void put4(const LinearArgs &a, int64_t row, int c, const float *z) {
    T *y = static_cast<T *>(a.y) + row * a.y_stride + c;
    if (c + 4 <= a.cout) {
        store4(y, z);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < a.cout) y[j] = from_float<T>(z[j]);
    }
}
__device__ __forceinline__ void put4(const LinearArgs &a, int64_t row, int c, const float *z) {
    if (a.y_type == kBf16) put4<bf16_t>(a, row, c, z);
    else if (a.y_type == kF16) put4<_Float16>(a, row, c, z);
    else put4<float>(a, row, c, z);
}

// Rows of a tile past the last end: BN outputs each of zeros.
__device__ void zero_tile(const LinearArgs &a, int row0, int rows, int c0, int cols) {
    const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int groups = cols / 4;
    for (int u = threadIdx.x; u < rows * groups; u += blockDim.x) {
        const int r = u / groups, c = c0 + (u - r * groups) * 4;
        if (c < a.cout) put4(a, row0 + r, c, z);
    }
}

// The outputs of one 16 x 16 accumulator of the layer with factors at w_scale and bias:
// this lane's row (written if below end), channels 16 c16 + 4 (lane / 16) and on.
template <int G>
__device__ __forceinline__ void finish16(const LinearArgs &a, const float *w_scale, const float *bias, const v4i (&sum)[G],
                                         float scale, int row, int end, int c16, int block0, int lane) {
    float z[2][4];
    const int p = block0 * 16 + (lane >> 4) * 4, c = c16 * 16 + (lane >> 4) * 4;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const int q[4] = {sum[g][0], sum[g][1], sum[g][2], sum[g][3]};
        dequant4(w_scale + p + 32 * g, bias + p + 32 * g, q, scale, z[g]);
    }
    if (G == 2) gated4(z[0], z[1]);
    if (row < end && c < a.cout) put4(a, row, c, z[0]);
}

// A token's row, and the elements that it has (none for an empty one).
template <typename T>
struct TokenRow {
    const T *p;
    int n;
};
template <typename T>
__device__ __forceinline__ TokenRow<T> token_row(const TokenArgs &x, int row) {
    return {static_cast<const T *>(x.x) + max(row, 0) * x.x_stride, row < 0 ? 0 : x.cin};
}

// The codes of a token's chunks (load_chunks), to LDS.
template <int CH, int THREADS>
__device__ __forceinline__ void store_chunks(int8_t *to, int k_stride, int t, const float (&v)[8 * CH], float sigma, float s) {
    const float r = sigma * (1.0f / s);
    const bool plain = token_plain(s);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * THREADS + t;
        const uint2 q = token_codes8(&v[8 * i], sigma, s, r, plain);
        if (c < k_stride >> 3) *reinterpret_cast<uint2 *>(to + c * 8) = q;
    }
}

// ---- few rows -------------------------------------------------------------------------
// Eight waves, WK of them on one group of 16 output channels (gated: of their gates and
// their values) by 16 MT rows: they take the contraction 64 bytes in turn and add up in
// LDS; 8 / WK groups a block.  The weights go from memory to registers in runs of 1 KB,
// U of them in flight a wave: the kernel is bound by their bytes.  WK is large where the
// groups alone would not fill the card.  13 rows, 4096 -> 2 x 8192 gated: 13.3 us, 5.1 TB/s
// of weights (a large copy moves 5.1).  Tried without gain: 4, 12 and 16 runs in flight,
// nontemporal loads (13.3 us).
template <int MT, int G, int U>
__global__ void __launch_bounds__(512) linear_stream_kernel(const LinearArgs a, int wk) {
    constexpr int WAVES = 8;
    __shared__ v4i part[WAVES][MT][G][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = WAVES / wk, groups = (a.cout + 16 * per - 1) / (16 * per);
    const int bid = blockIdx.y * gridDim.x + blockIdx.x;
    const int t = bid / groups, g0 = (bid - t * groups) * per;
    RowTiles<16 * MT> tiles(a);
    if (t >= tiles.total()) return;
    const RowTile r = tiles.find(t);
    const int rows = min(r.end - r.row0, 16 * MT);
    if (r.expert < 0) return zero_tile(a, r.row0, rows, g0 * 16, 16 * per);

    const int nks = a.k_stride >> 6, first = wave & (wk - 1);
    const int c16 = min(g0 + wave / wk, (a.cout + 15) / 16 - 1);    // (a wave past the last group repeats it)
    const int block0 = G == 1 ? c16 : (c16 >> 1) * 4 + (c16 & 1);   // of 16 packed columns
    const int8_t *w = a.wp + ((int64_t)r.expert * a.cout_pad + block0 * 16) * a.k_stride + lane * 16;
    const int64_t value = (int64_t)32 * a.k_stride;   // from the gates' columns to the values'
    const int8_t *x[MT];
    float s[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int tok = token_of(a, r.row0 + min(16 * m + (lane & 15), rows - 1));
        x[m] = a.xq + (int64_t)max(tok, 0) * a.k_stride + (lane >> 4) * 16;
        s[m] = tok < 0 ? 0.0f : a.sx[tok] * a.inv_b;
    }
    v4i acc[MT][G];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int g = 0; g < G; ++g) acc[m][g] = v4i{0, 0, 0, 0};
    for (int k0 = first; k0 < nks; k0 += wk * U) {
        v4i fw[U][G], fx[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = min(k0 + wk * u, nks - 1);
#pragma unroll
            for (int g = 0; g < G; ++g) fw[u][g] = *reinterpret_cast<const v4i *>(w + g * value + (int64_t)k * 1024);
#pragma unroll
            for (int m = 0; m < MT; ++m) fx[u][m] = *reinterpret_cast<const v4i *>(x[m] + k * 64);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k0 + wk * u >= nks) break;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int g = 0; g < G; ++g)
                    acc[m][g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u][g], fx[u][m], acc[m][g], 0, 0, 0);
        }
    }
    if (wk > 1) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int g = 0; g < G; ++g) part[wave][m][g][lane] = acc[m][g];
        __syncthreads();
    }
    const float *w_scale = a.w_scale + (int64_t)r.expert * a.cout_pad, *bias = a.bias + (int64_t)r.expert * a.cout_pad;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if ((m & (wk - 1)) != first) continue;   // a group's waves share its row tiles
        float z[2][4];
        const int p = block0 * 16 + (lane >> 4) * 4;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            v4i sum = acc[m][g];
            if (wk > 1) {
                sum = part[wave - first][m][g][lane];
                for (int k = 1; k < wk; ++k) sum += part[wave - first + k][m][g][lane];
            }
            const int q[4] = {sum[0], sum[1], sum[2], sum[3]};
            dequant4(w_scale + p + 32 * g, bias + p + 32 * g, q, s[m], z[g]);
        }
        if (G == 2) gated4(z[0], z[1]);
        const int row = 16 * m + (lane & 15), c = c16 * 16 + (lane >> 4) * 4;
        if (row < rows && c < a.cout && c16 == g0 + wave / wk) put4(a, r.row0 + row, c, z[0]);
    }
}

// ---- few tokens, floats in ------------------------------------------------------------
// At most 16 rows, one layer, with the tokens' quantization in front: every block makes
// the codes of its rows itself, in LDS, while its first weights are on their way.  All
// eight waves share a row (a lane CH chunks of 8 elements, one row after the other) and
// then the contraction of 16 output channels.  One launch instead of two, and no codes
// in memory.
template <typename T, int G, int CH>
__global__ void __launch_bounds__(512) linear_token_kernel(const LinearArgs a, const TokenArgs x) {
    constexpr int WAVES = 8, U = 8;
    extern __shared__ __attribute__((aligned(16))) int8_t lds[];
    v4i(*part)[G][64] = reinterpret_cast<v4i(*)[G][64]>(lds);                // [WAVES][G][64]
    float *scale = reinterpret_cast<float *>(lds + WAVES * G * 1024);          // [16]
    float *most = scale + 16;                                                  // [WAVES]
    int8_t *codes = lds + WAVES * G * 1024 + 128;                              // [rows][k_stride + 16]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c16 = blockIdx.x, rows = a.rows;
    const int pitch = a.k_stride + 16;   // 16 rows' pieces then lie in different banks

    TokenRow<T> token = token_row<T>(x, 0);
    Raw8<T> raw[CH] = {};
    load_chunks<T, CH, 512>(token.p, token.n, threadIdx.x, raw);

    const int nks = a.k_stride >> 6;
    const int block0 = G == 1 ? c16 : (c16 >> 1) * 4 + (c16 & 1);   // of 16 packed columns
    const int8_t *w = a.wp + (int64_t)block0 * 16 * a.k_stride + lane * 16;
    const int64_t value = (int64_t)32 * a.k_stride;   // from the gates' columns to the values'
    v4i fw[U][G];
    auto weights = [&](int k0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int g = 0; g < G; ++g)
                fw[u][g] = *reinterpret_cast<const v4i *>(w + g * value + (int64_t)min(k0 + WAVES * u, nks - 1) * 1024);
    };
    weights(wave);
    __builtin_amdgcn_sched_barrier(0);   // the first weights are under way

    for (int row = 0; row < rows; ++row) {
        float v[8 * CH];
        chunk_values<T, CH, 512>(token.p, token.n, threadIdx.x, raw, v);
        if (row + 1 < rows) {   // the next row, under way over this one's codes
            token = token_row<T>(x, row + 1);
            load_chunks<T, CH, 512>(token.p, token.n, threadIdx.x, raw);
        }
        const float sigma = token_butterfly(v, lane, x.log_b);
        float m = token_max(v);
        if (row) __syncthreads();   // the row before has been read
        if (lane == 0) most[wave] = m;
        __syncthreads();
        m = most[0];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) m = __builtin_elementwise_maximum(m, most[k]);
        const float s = token_scale(m);
        if (threadIdx.x == 0) scale[row] = s * a.inv_b;
        store_chunks<CH, 512>(codes + row * pitch, a.k_stride, threadIdx.x, v, sigma, s);
    }
    __syncthreads();

    const int mine = min(lane & 15, rows - 1);
    const int8_t *from = codes + mine * pitch + (lane >> 4) * 16;
    v4i acc[G];
#pragma unroll
    for (int g = 0; g < G; ++g) acc[g] = v4i{0, 0, 0, 0};
    for (int k0 = wave; k0 < nks; k0 += WAVES * U) {
        if (k0 != wave) weights(k0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k0 + WAVES * u >= nks) break;
            const v4i fx = *reinterpret_cast<const v4i *>(from + (k0 + WAVES * u) * 64);
#pragma unroll
            for (int g = 0; g < G; ++g) acc[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u][g], fx, acc[g], 0, 0, 0);
        }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) part[wave][g][lane] = acc[g];
    __syncthreads();
    if (wave != 0) return;
    v4i sum[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        sum[g] = part[0][g][lane];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) sum[g] += part[k][g][lane];
    }
    finish16<G>(a, a.w_scale, a.bias, sum, scale[mine], lane & 15, rows, c16, block0, lane);
}

// ---- small layers, floats in ------------------------------------------------------------
// A contraction of at most 2048: a block quantizes 16 rows (of one expert), a wave a
// row at a time (all of a wave's rows loaded at once), into LDS, and then each wave takes
// groups of 16 output channels over the whole contraction, the weights straight from the
// L2s.  blockIdx.y: `per` of the groups, a multiple of the waves.  Bound by latency (a row
// in, its maximum, the weights' first bytes) until the weights' repeated reads take over:
// 6144 rows, 320 -> 320, float32, 9.6 us (its 15.8 MB would take 3.1), 12-13 us as two
// kernels.
template <typename T, int G, int CH>
__global__ void __launch_bounds__(512) linear_small_kernel(const LinearArgs a, const TokenArgs x, int per) {
    constexpr int WAVES = 8, U = 8, ROWS = 16, TURNS = ROWS / WAVES;
    __shared__ __attribute__((aligned(16))) int8_t codes[ROWS * (512 * CH + 16)];
    __shared__ float scale[ROWS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    RowTiles<ROWS> tiles(a);
    if ((int)blockIdx.x >= tiles.total()) return;
    const RowTile r = tiles.find(blockIdx.x);
    const int row0 = r.row0, rows = min(r.end - row0, ROWS);
    if (r.expert < 0) return zero_tile(a, row0, rows, blockIdx.y * per * 16, per * 16);
    const int64_t first = (int64_t)r.expert * a.cout_pad;   // of this expert's columns
    const int nks = a.k_stride >> 6, pitch = a.k_stride + 16;
    const int end = min(((int)blockIdx.y + 1) * per, (a.cout + 15) / 16);
    int c16 = blockIdx.y * per + wave;

    TokenRow<T> token[TURNS];
    Raw8<T> raw[TURNS][CH] = {};
#pragma unroll
    for (int i = 0; i < TURNS; ++i) token[i] = token_row<T>(x, token_of(a, row0 + min(wave + WAVES * i, rows - 1)));
#pragma unroll
    for (int i = 0; i < TURNS; ++i) load_chunks<T, CH, 64>(token[i].p, token[i].n, lane, raw[i]);

    const int64_t value = (int64_t)32 * a.k_stride;   // from the gates' columns to the values'
    v4i fw[U][G];
    auto weights = [&](int c, int k0) {
        const int block0 = G == 1 ? c : (c >> 1) * 4 + (c & 1);
        const int8_t *w = a.wp + (first + block0 * 16) * a.k_stride + lane * 16;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int g = 0; g < G; ++g)
                fw[u][g] = *reinterpret_cast<const v4i *>(w + g * value + min(k0 + u, nks - 1) * 1024);
    };
    if (c16 < end) weights(c16, 0);
    __builtin_amdgcn_sched_barrier(0);   // the first weights are under way

#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        const int row = wave + WAVES * i;
        if (row >= rows) break;
        float v[8 * CH];
        chunk_values<T, CH, 64>(token[i].p, token[i].n, lane, raw[i], v);
        const float sigma = token_butterfly(v, lane, x.log_b);
        const float s = token_scale(token_max(v));
        if (lane == 0) scale[row] = s * a.inv_b;
        store_chunks<CH, 64>(codes + row * pitch, a.k_stride, lane, v, sigma, s);
    }
    __syncthreads();

    const int mine = min(lane & 15, rows - 1);
    const int8_t *from = codes + mine * pitch + (lane >> 4) * 16;
    while (c16 < end) {
        v4i acc[G];
#pragma unroll
        for (int g = 0; g < G; ++g) acc[g] = v4i{0, 0, 0, 0};
        for (int k0 = 0; k0 < nks; k0 += U) {
            if (k0) weights(c16, k0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (k0 + u >= nks) break;
                const v4i fx = *reinterpret_cast<const v4i *>(from + (k0 + u) * 64);
#pragma unroll
                for (int g = 0; g < G; ++g) acc[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u][g], fx, acc[g], 0, 0, 0);
            }
        }
        const int c = c16;
        c16 += WAVES;
        if (c16 < end) weights(c16, 0);   // the next group's, under way over the stores
        finish16<G>(a, a.w_scale + first, a.bias + first, acc, scale[mine], row0 + (lane & 15), row0 + rows, c,
                    G == 1 ? c : (c >> 1) * 4 + (c & 1), lane);
    }
}

// ---- many rows --------------------------------------------------------------------------
// Block index -> tile.  Blocks bid, bid + 8, ... run on one XCD; each XCD takes a
// contiguous range of v, and v goes down 8 row tiles before the next column tile, so
// the 32 tiles that an XCD's CUs hold at once read 8 row and 4 column operands.
struct TileIndex {
    int t, tn;
};
__device__ __forceinline__ TileIndex tile_index(int bid, int tiles_m, int tiles_n) {
    const int nt = tiles_m * tiles_n, xcd = bid & 7, q = nt >> 3, rest = nt & 7;
    const int v = xcd * q + min(xcd, rest) + (bid >> 3);
    const int band = v / (8 * tiles_n), in = v - band * 8 * tiles_n;
    const int high = min(8, tiles_m - band * 8);
    const int tn = in / high;
    return {band * 8 + in - tn * high, tn};
}

// Stores 32 rows of COLS outputs, fp32 in LDS rows of COLS + 4, to y: lanes take 16-byte
// pieces, so a store instruction writes whole runs of rows.  PARTS waves share the rows.
template <typename T, int COLS, int PARTS>
__device__ void store_rows(const LinearArgs &a, const float *from, int64_t row0, int rows, int c0, int lane, int part) {
    constexpr int E = 16 / sizeof(T), PER = COLS / E;     // elements of a piece, pieces of a row
    constexpr int STEP = 64 / PER, PIECES = 32 / STEP;    // rows that a wave's piece covers, such pieces
    if (c0 >= a.cout) return;
    const int r0 = lane / PER, c = lane % PER * E;
    T *to = static_cast<T *>(a.y) + (row0 + r0) * a.y_stride + c0 + c;
    from += r0 * (COLS + 4) + c;
    const int64_t step = STEP * a.y_stride;
    auto piece = [&](int u, float *z) {
#pragma unroll
        for (int e = 0; e < E; e += 4)
            *reinterpret_cast<float4 *>(z + e) = *reinterpret_cast<const float4 *>(from + u * STEP * (COLS + 4) + e);
    };
    if (c0 + COLS <= a.cout && rows >= 32 && PIECES % PARTS == 0) {
        to += part * step;
#pragma unroll
        for (int k = 0; k < PIECES / PARTS; ++k) {
            float z[E];
            piece(k * PARTS + part, z);
            store16(to, z);
            to += PARTS * step;
        }
        return;
    }
    for (int u = part; u < PIECES; u += PARTS) {
        if (u * STEP + r0 >= rows) continue;
        float z[E];
        piece(u, z);
        T *at = to + u * step;
        if (c0 + c + E <= a.cout) {
            store16(at, z);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (c0 + c + e < a.cout) at[e] = from_float<T>(z[e]);
        }
    }
}

// Tiles of BM rows x BN packed columns by WM x WN waves of FM x FN MFMAs of 32 x 32,
// the contraction in steps of 64 bytes through a ring of STAGES LDS buffers that are
// filled by direct-to-LDS loads.  A row's four 16-byte pieces of a step are permuted
// by the row (piece c of row m at place c ^ (m >> 2 & 3)), so 16 rows' pieces, what the
// 64 banks deliver at once, do not meet in a bank; the weights lie in memory as they are read.
//
// Each half step's fragments are read while the half before runs on the matrix
// cores, and the one barrier of a step stands between its halves: the reads of a
// buffer end before it, the loads that refill that buffer and the reads of the next
// one begin after it.
//
// 4096 x 4096 x 4096, bf16 out: 64 us, 2.1 POP/s; 8192 x 4096 x 16384 gated: 505 us, 2.18
// POP/s (the INT8 library product of that size, which writes plain sums, 2.24).  There the
// matrix cores are busy 60 % of the cycles at 1.6 GHz, where power holds the clock (2.4
// nominal).  (After a pause the clock takes some hundred calls to settle; before, the
// same take up to 80 and 550 us.)  Wave tiles of 64 x 64 in blocks of 128 x
// 256, two a CU, are 3 % behind 128 x 64 in 256 x 256 where all tiles are whole, and ahead
// elsewhere: 32768 rows over 64 experts 175 us against 200.  Tried without gain: five
// stages, wave priorities, 16 waves on 256 x 256, float32 stores without LDS, codes laid
// out in the weights' order (3-5 % for whole tiles; rows gathered by expert cannot).
//
// Few tiles: KG such groups of waves share a tile, each a run of the contraction with a
// ring of its own, and add up in LDS.  A step costs a group about 0.17 us of LDS and
// barrier latency however few MFMAs it has; the groups of a CU overlap it.  965 rows, 6656
// -> 2 x 161: tiles of 32 x 64 11.0 us, of 64 x 64 15.9 (96 of the 256 CUs), of 64 x 128
// without groups 24.9; five stages 11.3.
template <int WM, int WN, int FM, int FN, int STAGES, int KG, int G>
__global__ void __launch_bounds__(64 * WM * WN * KG) linear_tile_kernel(const LinearArgs a) {
    constexpr int NW = WM * WN, BM = WM * FM * 32, BN = WN * FN * 32;
    constexpr int A_INSTR = BM / 16 / NW, B_INSTR = BN / 16 / NW, PER_STAGE = A_INSTR + B_INSTR;
    constexpr int STAGE_BYTES = (BM + BN) * 64;
    constexpr int COLS = FN / G * 32;   // outputs of a wave's row
    static_assert(A_INSTR * NW * 16 == BM && B_INSTR * NW * 16 == BN && FN % G == 0, "tile");
    constexpr int RING = STAGES * STAGE_BYTES;
    static_assert(NW * 32 * (COLS + 4) * 4 <= KG * RING, "output staging");
    static_assert(KG == 1 || (4 % KG == 0 && KG * NW * FM * FN * 4096 <= KG * RING), "partial sums");
    static_assert(BN <= 256 && BM <= 64 * NW * KG && NW * KG >= 2, "a wave's load of the factors");
    // the ring, then the columns' scales and biases, [2][BN] floats, and the tokens' scales.
    // (One array: with a second LDS object the compiler waits for every load under way
    // before each read.)
    __shared__ __attribute__((aligned(1024))) int8_t lds[KG * RING + 8 * BN + 4 * BM];
    float4 *factor = reinterpret_cast<float4 *>(lds + KG * RING);
    float *scales = reinterpret_cast<float *>(lds + KG * RING + 8 * BN);
    const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kg = all / NW, wave = all % NW, wm = wave / WN, wn = wave % WN;
    int8_t *ring = lds + kg * RING;

    const int tiles_n = (a.cout_pad + BN - 1) / BN;
    const int bid = blockIdx.y * gridDim.x + blockIdx.x;
    RowTiles<BM> row_tiles(a);
    const int tiles_m = row_tiles.total();
    if (bid >= tiles_m * tiles_n) return;
    const TileIndex ti = tile_index(bid, tiles_m, tiles_n);
    const int tn = ti.tn;
    const RowTile r = row_tiles.find(ti.t);
    const int rows = min(r.end - r.row0, BM);
    if (r.expert < 0) return zero_tile(a, r.row0, rows, tn * BN / G, BN / G);

    // the tokens of this lane's pieces of the operand, and of a row of the tile
    const int mine_row = all * 64 + lane;
    int tok_a[A_INSTR], tok_row = r.row0 + min(mine_row, rows - 1);
#pragma unroll
    for (int j = 0; j < A_INSTR; ++j) tok_a[j] = r.row0 + min(16 * (wave + NW * j) + (lane >> 2), rows - 1);
    if (a.src) {   // (all loaded before one is looked at)
        tok_row = a.src[tok_row];
#pragma unroll
        for (int j = 0; j < A_INSTR; ++j) tok_a[j] = a.src[tok_a[j]];
        if ((unsigned)tok_row >= (unsigned)a.x_rows) tok_row = -1;
#pragma unroll
        for (int j = 0; j < A_INSTR; ++j)
            if ((unsigned)tok_a[j] >= (unsigned)a.x_rows) tok_a[j] = -1;
    }

    // Column factors and token scales, wanted at the end: direct loads to LDS as well, older than
    // the ring's, so that the ring's first wait ends them and no tile starts by waiting for them.
    if (all < 2 && lane < BN / 4) {
        const float *from = (all ? a.bias : a.w_scale) + (int64_t)r.expert * a.cout_pad + min(tn * BN + lane * 4, a.cout_pad - 4);
        __builtin_amdgcn_global_load_lds(HATQ_GLOBAL(from), HATQ_LDS(lds + KG * RING + all * 4 * BN), 16, 0, 0);
    }
    if (mine_row < BM) {
        if (tok_row < 0) scales[mine_row] = 0.0f;
        else __builtin_amdgcn_global_load_lds(HATQ_GLOBAL(a.sx + tok_row), HATQ_LDS(scales + all * 64), 4, 0, 0);
    }
    // this group's steps: `nks` of them from k0, in a loop of `turns` for every group
    const int steps = a.k_stride >> 6, turns = (steps + KG - 1) / KG;
    const int k0 = min(kg * turns, steps - 1), nks = max(min(steps - kg * turns, turns), 0);
    const int8_t *pa[A_INSTR], *pb[B_INSTR];
#pragma unroll
    for (int j = 0; j < A_INSTR; ++j) {
        const int m = 16 * (wave + NW * j) + (lane >> 2);
        pa[j] = a.xq + (int64_t)max(tok_a[j], 0) * a.k_stride + k0 * 64 + 16 * ((lane & 3) ^ ((m >> 2) & 3));
    }
#pragma unroll
    for (int j = 0; j < B_INSTR; ++j) {
        const int block = min(tn * (BN / 16) + wave + NW * j, a.cout_pad / 16 - 1);
        pb[j] = a.wp + ((int64_t)r.expert * a.cout_pad + block * 16) * a.k_stride + k0 * 1024 + lane * 16;
    }
    // Loads the step that the pointers are at into a buffer; `more`: go on to the next.
    // (Past the last step the last one is loaded again, so that every step has the same
    // loads and waits; nothing reads those copies.)
    auto issue = [&](int8_t *to, bool more) {
#pragma unroll
        for (int j = 0; j < A_INSTR; ++j) {
            __builtin_amdgcn_global_load_lds(HATQ_GLOBAL(pa[j]), HATQ_LDS(to + 1024 * (wave + NW * j)), 16, 0, 0);
            pa[j] += more ? 64 : 0;
        }
#pragma unroll
        for (int j = 0; j < B_INSTR; ++j) {
            __builtin_amdgcn_global_load_lds(HATQ_GLOBAL(pb[j]), HATQ_LDS(to + BM * 64 + 1024 * (wave + NW * j)), 16, 0, 0);
            pb[j] += more ? 1024 : 0;
        }
    };
    int fa[2], fb[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c = 2 * h + (lane >> 5), m = wm * FM * 32 + (lane & 31);
        fa[h] = m * 64 + 16 * (c ^ ((m >> 2) & 3));
        fb[h] = BM * 64 + (wn * FN * 2 + ((lane >> 4) & 1)) * 1024 + c * 256 + (lane & 15) * 16;
    }
    v4i xa[2][FM], wb[2][FN];
    auto read = [&](const int8_t *from, int h, int k) {
        if (k < FN) wb[h][k] = *reinterpret_cast<const v4i *>(from + fb[h] + k * 2048);
        else if (k < FN + FM) xa[h][k - FN] = *reinterpret_cast<const v4i *>(from + fa[h] + (k - FN) * 2048);
    };
    v16i acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[j][i][e] = 0;
    // The MFMAs of half h, with the reads of the other half's fragments two by two between
    // the first of them (left to itself the compiler moves the reads down to their use).
    auto half = [&](int h, const int8_t *next) {
#pragma unroll
        for (int k = 0; k < FM * FN; ++k) {
            const int j = k / FM, i = k % FM;
            acc[j][i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wb[h][j], xa[h][i], acc[j][i], 0, 0, 0);
            if (2 * k < FM + FN) {
                read(next, 1 - h, 2 * k);
                read(next, 1 - h, 2 * k + 1);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

#pragma unroll
    for (int k = 0; k < STAGES; ++k) issue(ring + k * STAGE_BYTES, k + 1 < nks);
    wait_vmcnt_lds<(STAGES - 1) * PER_STAGE>();
    block_barrier();
#pragma unroll
    for (int k = 0; k < FM + FN; ++k) read(ring, 0, k);
    int at = 0;   // this step's buffer
    for (int ks = 0; ks < turns; ++ks) {
        int8_t *now = ring + at;
        at = at + STAGE_BYTES == RING ? 0 : at + STAGE_BYTES;
        if (KG == 1 || ks < nks) half(0, now);
        // the next step's loads have landed (STAGES - 2 later ones under way), this buffer
        // has been read: by every wave, past the barrier
        wait_vmcnt_lds<(STAGES - 2) * PER_STAGE>();
        block_barrier();
        issue(now, ks + STAGES + 1 < nks);
        if (KG == 1 || ks < nks) half(1, ring + at);
    }
    wait_vmcnt_lds<0>();
    block_barrier();   // no load is under way into the buffers that stage the outputs

    if constexpr (KG > 1) {
        // partial sums [KG][NW][FN][FM][4][64]; group kg adds up the quads q = kg mod KG
        v4i *part = reinterpret_cast<v4i *>(lds);
        auto quad = [&](int k, int j, int i, int q) { return part + ((((k * NW + wave) * FN + j) * FM + i) * 4 + q) * 64 + lane; };
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *quad(kg, j, i, q) = v4i{acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]};
        __syncthreads();
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int u = 0; u < 4 / KG; ++u) {
                    // (the sum of quad u KG + kg goes to the registers of quad u)
                    v4i sum = *quad(0, j, i, u * KG + kg);
#pragma unroll
                    for (int k = 1; k < KG; ++k) sum += *quad(k, j, i, u * KG + kg);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[j][i][4 * u + e] = sum[e];
                }
        __syncthreads();
    }

    float scale[FM];   // of this lane's tokens
#pragma unroll
    for (int i = 0; i < FM; ++i) scale[i] = scales[(wm * FM + i) * 32 + (lane & 31)] * a.inv_b;
    float *mine = reinterpret_cast<float *>(lds) + wave * 32 * (COLS + 4);
    const int c0 = (tn * BN + wn * FN * 32) / G;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int first = (wm * FM + i) * 32, n = min(rows - first, 32);
        if (KG == 1 && n <= 0) break;
#pragma unroll
        for (int j = 0; j < FN; j += G)
#pragma unroll
            for (int u = 0; u < 4 / KG; ++u) {
                // element 0's column: rows 8 q + 4 (lane / 32) of the 32 x 32 tile
                const int in = 8 * (u * KG + kg) + 4 * (lane >> 5);
                const float4 *f = factor + ((wn * FN + j) * 32 + in) / 4;
                float z[2][4];
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const int v[4] = {acc[j + g][i][4 * u], acc[j + g][i][4 * u + 1], acc[j + g][i][4 * u + 2],
                                      acc[j + g][i][4 * u + 3]};
                    dequant4(reinterpret_cast<const float *>(f + 8 * g), reinterpret_cast<const float *>(f + BN / 4 + 8 * g), v,
                             scale[i], z[g]);
                }
                if (G == 2) gated4(z[0], z[1]);
                *reinterpret_cast<float4 *>(mine + (lane & 31) * (COLS + 4) + j / G * 32 + in) =
                    make_float4(z[0][0], z[0][1], z[0][2], z[0][3]);
            }
        // (one group: a wave's LDS accesses are in order, so its rows are whole when it reads them)
        if (KG > 1) __syncthreads();
        if (a.y_type == kBf16) store_rows<bf16_t, COLS, KG>(a, mine, r.row0 + first, n, c0, lane, kg);
        else if (a.y_type == kF16) store_rows<_Float16, COLS, KG>(a, mine, r.row0 + first, n, c0, lane, kg);
        else store_rows<float, COLS, KG>(a, mine, r.row0 + first, n, c0, lane, kg);
        if (KG > 1 && i + 1 < FM) __syncthreads();
    }
}

template <int MT, int U>
void stream(const LinearArgs &a, hipStream_t st, int wk) {
    const int cols = 16 * 8 / wk;
    const dim3 grid = grid_of(most_row_tiles(a, 16 * MT) * ((a.cout + cols - 1) / cols));
    if (a.gated) linear_stream_kernel<MT, 2, U><<<grid, 512, 0, st>>>(a, wk);
    else linear_stream_kernel<MT, 1, U><<<grid, 512, 0, st>>>(a, wk);
}

template <typename T, int CH>
void token(const LinearArgs &a, const TokenArgs &x, hipStream_t st) {
    const int grid = (a.cout + 15) / 16;
    const size_t bytes = 8 * (a.gated ? 2 : 1) * 1024 + 128 + (size_t)a.rows * (a.k_stride + 16);
    if (a.gated) linear_token_kernel<T, 2, CH><<<grid, 512, bytes, st>>>(a, x);
    else linear_token_kernel<T, 1, CH><<<grid, 512, bytes, st>>>(a, x);
}

template <typename T, int CH>
void small(const LinearArgs &a, const TokenArgs &x, hipStream_t st) {
    // Column ranges, each of which quantizes the rows again: up to 512 blocks, two a CU, as the
    // card holds at once of a plain layer's with one and two chunks a lane and of a gated one's
    // with one (bf16, 512 -> 256, 6144 rows: 384 blocks 8.8 us, 768 11.0).  The other forms'
    // registers (138 to 207) leave one block a CU: more than 256 of theirs go in two rounds.
    const int groups = (a.cout + 15) / 16, blocks = (int)most_row_tiles(a, 16);
    const int most = blocks < 512 ? 512 / blocks : 1, ranges = (groups + 7) / 8 < most ? (groups + 7) / 8 : most;
    const int per = ((groups + ranges - 1) / ranges + 7) / 8 * 8;
    const dim3 grid(blocks, (groups + per - 1) / per);
    if (a.gated) linear_small_kernel<T, 2, CH><<<grid, 512, 0, st>>>(a, x, per);
    else linear_small_kernel<T, 1, CH><<<grid, 512, 0, st>>>(a, x, per);
}

template <typename T>
void token(const LinearArgs &a, const TokenArgs &x, hipStream_t st) {
    const TokenChoice c = choose_tokens(a);
    if (c.small) {
        if (c.ch == 1) small<T, 1>(a, x, st);
        else if (c.ch == 2) small<T, 2>(a, x, st);
        else small<T, 4>(a, x, st);
    } else {
        if (c.ch == 1) token<T, 1>(a, x, st);
        else if (c.ch == 2) token<T, 2>(a, x, st);
        else token<T, 4>(a, x, st);
    }
}

template <int WM, int WN, int FM, int FN, int STAGES, int KG = 1>
void tile(const LinearArgs &a, hipStream_t st) {
    constexpr int BM = WM * FM * 32, BN = WN * FN * 32;
    const dim3 grid = grid_of(most_row_tiles(a, BM) * ((a.cout_pad + BN - 1) / BN));
    if (a.gated) linear_tile_kernel<WM, WN, FM, FN, STAGES, KG, 2><<<grid, 64 * WM * WN * KG, 0, st>>>(a);
    else linear_tile_kernel<WM, WN, FM, FN, STAGES, KG, 1><<<grid, 64 * WM * WN * KG, 0, st>>>(a);
}

}  // namespace

hipError_t launch_linear_tokens(const LinearArgs &a, const TokenArgs &x, hipStream_t st) {
    if (x.x_type == kF32) token<float>(a, x, st);
    else if (x.x_type == kBf16) token<bf16_t>(a, x, st);
    else token<_Float16>(a, x, st);
    return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs &a, hipStream_t st) {
    const LinearChoice c = choose_linear(a);
    switch (c.kernel) {
        case kTile32x64: tile<1, 1, 1, 2, 3, 4>(a, st); break;
        case kTile64x64: tile<2, 1, 1, 2, 3, 4>(a, st); break;
        case kTile64x128: tile<2, 2, 1, 2, 3>(a, st); break;
        case kTile128x128: tile<2, 2, 2, 2, 3>(a, st); break;
        case kTile128x256: tile<2, 4, 2, 2, 3>(a, st); break;
        case kTile256x256: tile<2, 4, 4, 2, 4>(a, st); break;
        case kStream16: stream<1, 8>(a, st, c.waves); break;
        case kStream32: stream<2, 4>(a, st, c.waves); break;
    }
    return hipGetLastError();
}

}  // namespace hatq
