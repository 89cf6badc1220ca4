// Linear layers of 4-bit weights with a scale for each group of input channels, over a few
// tokens in INT8 codes:
//   z = (s / b) sum_g w_scale[c][g] float(sum_{d in g} q[d] wq[c][d]) + bias
// Exact INT32 sums in each group (INT8 matrix instructions, 64 channels a step; a code enters
// as 16 times itself, the upper half of a byte), fp32 sums over the groups.
//
// Packed weights: 16 channels by 128 input channels, 1 KB in lane order: lane 16 u + c has
// channel c and input channels 16 u .. 16 u + 15 of both 64-channel steps, 8 bytes each;
// byte b of a step's word w holds the codes of input channels 8 w + b (low half) and 8 w + 4
// + b.  Their scales: [4][steps with scales of their own][4 channels] bf16, lane 16 u + c
// takes the u-th part, which belongs to the channels of its sums.  A gated layer's channels
// go 16 gates, 16 values in turn.
#include "linear4.h"

#include "../../include/hatq.h"
#include "linear_device.h"

namespace hatq {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
constexpr int kWaves = 8;
constexpr int kThreads = 256;

// One tile of 16 channels by 128 input channels as it lies in memory: codes, and the scales
// of this lane's sums (S = 2: of both steps, 1: of the whole).
template <int S>
struct Tile {
    v4u code;
    uint32_t scale[2 * S];
};
template <int S>
__device__ __forceinline__ void load_tile(const uint8_t *code, const uint16_t *scale, int lane, Tile<S> &t) {
    t.code = *reinterpret_cast<const v4u *>(code + lane * 16);
    const uint16_t *s = scale + (lane >> 4) * (4 * S);
    if constexpr (S == 2) {
        const v4u w = *reinterpret_cast<const v4u *>(s);
#pragma unroll
        for (int i = 0; i < 4; ++i) t.scale[i] = w[i];
    } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(s);
        t.scale[0] = w.x;
        t.scale[1] = w.y;
    }
}
__device__ __forceinline__ float bf16_of(const uint32_t *w, int j) {
    return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
}

// The tile's products with MT times 16 tokens, x: their codes of both steps.
template <int S, int MT>
__device__ __forceinline__ void multiply(const Tile<S> &t, const v4i (&x)[MT][2], v4f (&acc)[MT]) {
    v4i w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            w[k][2 * i] = (int)((t.code[2 * k + i] << 4) & 0xf0f0f0f0u);
            w[k][2 * i + 1] = (int)(t.code[2 * k + i] & 0xf0f0f0f0u);
        }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        v4i sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[0], x[m][0], v4i{0, 0, 0, 0}, 0, 0, 0);
        if constexpr (S == 2) {
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[m][r] = __builtin_fmaf((float)sum[r], bf16_of(t.scale, r), acc[m][r]);
            sum = v4i{0, 0, 0, 0};
        }
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[1], x[m][1], sum, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            acc[m][r] = __builtin_fmaf((float)sum[r], bf16_of(t.scale, 4 * (S - 1) + r), acc[m][r]);
    }
}

// This lane's outputs of one 16 x 16 tile: channels 16 c16 + 4 (lane / 16) and on of `row`.
// s: the token's scale / b.
template <int G>
__device__ __forceinline__ void finish(const Linear4Args &a, const v4f (&sum)[G], float s, int row, int c16, int lane) {
    float z[2][4];
    const int c = c16 * 16 + (lane >> 4) * 4;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const float4 b = *reinterpret_cast<const float4 *>(a.bias + (c16 * G + g) * 16 + (lane >> 4) * 4);
        const float bias[4] = {b.x, b.y, b.z, b.w};
        // (the codes came 16 times too large)
#pragma unroll
        for (int r = 0; r < 4; ++r) z[g][r] = __builtin_fmaf(sum[g][r] * 0.0625f, s, bias[r]);
    }
    if (G == 2) gated4(z[0], z[1]);
    if (row < a.rows && c < a.cout) put4(a, row, c, z[0]);
}

// ---- a few tokens, floats in -----------------------------------------------------------
// Every block takes 16 channels (gated: and their values), quantizes the rows itself while
// its first weights are under way, and its waves take the tiles in turn.  Bound by latency up to
// about 8 MB of weights: 1 token, 4096 -> 4096, 4.6 us for 8.9 MB, an empty launch 2 to 2.5.
template <typename T, int G, int S, int CH>
__global__ void __launch_bounds__(64 * kWaves) linear4_token_kernel(const Linear4Args a, const TokenArgs x) {
    constexpr int U = 4;
    extern __shared__ __attribute__((aligned(16))) int8_t lds[];
    v4f(*part)[G][64] = reinterpret_cast<v4f(*)[G][64]>(lds);            // [kWaves][G][64]
    float *scale = reinterpret_cast<float *>(lds + kWaves * G * 1024);      // [16]
    float *most = scale + 16;                                              // [kWaves]
    int8_t *codes = lds + kWaves * G * 1024 + 128;                          // [rows][k_stride + 16]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c16 = blockIdx.x, rows = a.rows;
    const int pitch = a.k_stride + 16;   // 16 rows' pieces then lie in different banks
    TokenRow<T> token = token_row<T>(x, 0);
    Raw8<T> raw[CH] = {};
    load_chunks<T, CH, 512>(token.p, token.n, threadIdx.x, raw);

    const int tiles = a.k_stride >> 7;
    const uint8_t *w = a.wp + (int64_t)c16 * G * tiles * 1024;
    const uint16_t *ws = a.w_scale + (int64_t)c16 * G * tiles * (16 * S);
    Tile<S> t[U][G];
    auto weights = [&](int k0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int k = g * tiles + min(k0 + kWaves * u, tiles - 1);
                load_tile<S>(w + (int64_t)k * 1024, ws + (int64_t)k * (16 * S), lane, t[u][g]);
            }
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
        for (int k = 1; k < kWaves; ++k) m = __builtin_elementwise_maximum(m, most[k]);
        const float s = token_scale(m);
        if (threadIdx.x == 0) scale[row] = s * a.inv_b;
        store_chunks<CH, 512>(codes + row * pitch, a.k_stride, threadIdx.x, v, sigma, s);
    }
    __syncthreads();

    const int mine = min(lane & 15, rows - 1);
    const int8_t *from = codes + mine * pitch + (lane >> 4) * 16;
    v4f acc[G][1];
#pragma unroll
    for (int g = 0; g < G; ++g) acc[g][0] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = wave; k0 < tiles; k0 += kWaves * U) {
        if (k0 != wave) weights(k0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k0 + kWaves * u >= tiles) break;
            const v4i *c = reinterpret_cast<const v4i *>(from + (k0 + kWaves * u) * 128);
            const v4i fx[1][2] = {{c[0], c[4]}};
#pragma unroll
            for (int g = 0; g < G; ++g) multiply<S, 1>(t[u][g], fx, acc[g]);
        }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) part[wave][g][lane] = acc[g][0];
    __syncthreads();
    if (wave != 0) return;
    v4f sum[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        sum[g] = part[0][g][lane];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) sum[g] += part[k][g][lane];
    }
    finish<G>(a, sum, scale[mine], (lane & 15) < rows ? lane & 15 : rows, c16, lane);
}

// ---- more tokens of a short contraction, floats in ------------------------------------------
// A contraction of at most 2048: a block quantizes 16 rows, a wave a row at a time (both of a
// wave's rows loaded at once), into LDS, and then each wave takes groups of 16 channels over
// the whole contraction.  blockIdx.y: `per` of the groups, a multiple of the waves.  One launch
// instead of two; bound by latency (row, maximum, codes, then the groups' tiles): 77 rows, 1000 ->
// 1001, float32, 6.8 us.
template <typename T, int G, int S, int CH>
__global__ void __launch_bounds__(64 * kWaves) linear4_small_kernel(const Linear4Args a, const TokenArgs x, int per) {
    constexpr int U = 4, ROWS = 16, TURNS = ROWS / kWaves;
    __shared__ __attribute__((aligned(16))) int8_t codes[ROWS * (512 * CH + 16)];
    __shared__ float scale[ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = blockIdx.x * ROWS, rows = min(a.rows - row0, ROWS);
    const int tiles = a.k_stride >> 7, pitch = a.k_stride + 16;
    const int end = min(((int)blockIdx.y + 1) * per, (a.cout + 15) / 16);
    int c16 = blockIdx.y * per + wave;

    TokenRow<T> token[TURNS];
    Raw8<T> raw[TURNS][CH] = {};
#pragma unroll
    for (int i = 0; i < TURNS; ++i) token[i] = token_row<T>(x, row0 + min(wave + kWaves * i, rows - 1));
#pragma unroll
    for (int i = 0; i < TURNS; ++i) load_chunks<T, CH, 64>(token[i].p, token[i].n, lane, raw[i]);

    Tile<S> t[U][G];
    auto weights = [&](int c, int k0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int64_t k = (int64_t)(c * G + g) * tiles + min(k0 + u, tiles - 1);
                load_tile<S>(a.wp + k * 1024, a.w_scale + k * (16 * S), lane, t[u][g]);
            }
    };
    if (c16 < end) weights(c16, 0);
    __builtin_amdgcn_sched_barrier(0);   // the first weights are under way

#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        const int row = wave + kWaves * i;
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
        v4f acc[G][1];
#pragma unroll
        for (int g = 0; g < G; ++g) acc[g][0] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        for (int k0 = 0; k0 < tiles; k0 += U) {
            if (k0) weights(c16, k0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (k0 + u >= tiles) break;
                const v4i *c = reinterpret_cast<const v4i *>(from + (k0 + u) * 128);
                const v4i fx[1][2] = {{c[0], c[4]}};
#pragma unroll
                for (int g = 0; g < G; ++g) multiply<S, 1>(t[u][g], fx, acc[g]);
            }
        }
        const int c = c16;
        c16 += kWaves;
        if (c16 < end) weights(c16, 0);   // the next group's, under way over the stores
        v4f sum[G];
#pragma unroll
        for (int g = 0; g < G; ++g) sum[g] = acc[g][0];
        finish<G>(a, sum, scale[mine], (lane & 15) < rows ? row0 + (lane & 15) : a.rows, c, lane);
    }
}

// ---- codes from memory ------------------------------------------------------------------
// Waves of a block take G groups of 16 channels by 16 MT rows, `wk` of them the tiles of the
// contraction in turn (they add up in LDS), the others channels further on.  Adjacent groups (and
// a gated layer's gates and values) share the rows' codes: of those a wave reads 2 KB for 1 KB of
// weights and 16 rows, and of long calls they are what the L2s give.
// Few rows are bound by the weights' bytes: 6 rows, 8192 -> 2 x 16384, 25.4 us for 143 MB, 5.6
// TB/s; many by the codes' loads, and by a conversion and a multiply-add for each sum and group:
// 128 rows of 8192 -> 2 x 16384 63 us, 1090 TOP/s, as 2048 rows of 4096 -> 4096, 68 us.  (The next
// step's loads over this one's products, in registers of their own: 5 to 12 % behind.)
// The codes lie as the operands are, 1 KB for 16 rows by 64 input channels: by rows, adjacent
// lanes are in 16 lines, a load is 64 accesses of the CU's cache instead of 16, and those bound
// the same two calls at 94 and 97 us.  Adjacent blocks go to one die each, so the tiles of rows
// that share weights meet in its L2 (17 rows of 16384 -> 16384 32.7 -> 30.4 us).
template <int G, int S, int MT, bool GATED>
__global__ void __launch_bounds__(64 * kWaves) linear4_stream_kernel(const Linear4Args a, int wk) {
    constexpr int U = MT == 1 ? 4 : MT == 4 ? 1 : 2;              // tiles loaded at once
    constexpr int R = GATED ? 2 : 1, N = G / R;             // products an output, output groups a wave
    extern __shared__ __attribute__((aligned(16))) int8_t lds[];
    v4f(*part)[G][MT][64] = reinterpret_cast<v4f(*)[G][MT][64]>(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part_k = wave & (wk - 1);
    const int row_tiles = (a.rows + 16 * MT - 1) / (16 * MT), groups = (a.cout + 15) / 16, sets = (groups + N - 1) / N;
    int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t per = ((int64_t)gridDim.y * gridDim.x) >> 3;
    if (block < 8 * per) block = (block & 7) * per + (block >> 3);
    const int row0 = (int)(block % row_tiles) * (16 * MT);
    const int64_t c16_ = block / row_tiles * (kWaves / wk) + wave / wk;
    const int c16 = (int)(c16_ < sets ? c16_ : sets - 1);
    // (past the last group: the last one again, not stored)
    const auto group = [&](int g) { return min(c16 * N + g / R, groups - 1) * R + g % R; };
    const int tiles = a.k_stride >> 7;
    const int8_t *from[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
        from[m] = a.xq + (int64_t)min((row0 >> 4) + m, (a.rows - 1) >> 4) * 16 * a.k_stride + lane * 16;
    v4f acc[G][MT];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[g][m] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = part_k; k0 < tiles; k0 += wk * U) {
        Tile<S> t[U][G];
        v4i fx[U][MT][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = min(k0 + wk * u, tiles - 1);
#pragma unroll
            for (int g = 0; g < G; ++g)
                load_tile<S>(a.wp + ((int64_t)group(g) * tiles + k) * 1024, a.w_scale + ((int64_t)group(g) * tiles + k) * (16 * S), lane,
                             t[u][g]);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const v4i *c = reinterpret_cast<const v4i *>(from[m] + k * 2048);
                fx[u][m][0] = c[0];
                fx[u][m][1] = c[64];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k0 + wk * u >= tiles) break;
#pragma unroll
            for (int g = 0; g < G; ++g) multiply<S, MT>(t[u][g], fx[u], acc[g]);
        }
    }
    if (wk > 1) {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int m = 0; m < MT; ++m) part[wave][g][m][lane] = acc[g][m];
        __syncthreads();
        if (part_k) return;
        for (int k = 1; k < wk; ++k)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[g][m] += part[wave + k][g][m][lane];
    }
    if (c16_ >= sets) return;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int row = row0 + 16 * m + (lane & 15);
        const float s = a.sx[min(row, a.rows - 1)] * a.inv_b;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v4f sum[R];
#pragma unroll
            for (int r = 0; r < R; ++r) sum[r] = acc[n * R + r][m];
            if (c16 * N + n < groups) finish<R>(a, sum, s, row, c16 * N + n, lane);
        }
    }
}

// ---- weights --------------------------------------------------------------------------
// Held channel of packed column p, or -1 in the padding.
__device__ __forceinline__ int held_channel(const Linear4PrepArgs &a, int p) {
    if (!a.gated) return p < a.cout ? p : -1;
    const int c = (p >> 5) * 16 + (p & 15);
    return c >= a.cout ? -1 : (p & 16) ? a.cout + c : c;
}

// Where packed column p keeps the code of input channel d: its byte, and the bits in it.
__device__ __forceinline__ int64_t code_byte(const Linear4PrepArgs &a, int p, int d) {
    const int step = (d >> 6) & 1, chunk = (d >> 4) & 3, w = (d >> 3) & 1;
    return ((int64_t)(p >> 4) * (a.k_stride >> 7) + (d >> 7)) * 1024 + (chunk * 16 + (p & 15)) * 16 + step * 8 + w * 4 + (d & 3);
}
__device__ __forceinline__ int64_t scale_index(const Linear4PrepArgs &a, int p, int g) {
    const int S = 128 / a.group, c = p & 15;
    return (((int64_t)(p >> 4) * (a.k_stride >> 7) + g / S) * 4 + (c >> 2)) * (4 * S) + g % S * 4 + (c & 3);
}

template <typename T>
__device__ float transformed4(const T *w, int d, int b) {
    const int first = d & ~(b - 1), i = d & (b - 1);
    double acc = 0.0;
    for (int j = 0; j < b; ++j) {
        const double e = (double)to_float(w[first + j]);
        acc += (__popc(i & j) & 1) ? -e : e;
    }
    return (float)acc;
}

// Floats: one wave a packed column and group.  W' = B w in fp64, rounded once to fp32; its
// scale bf16(fl32(max |W'| / 7)), at least 2^-100, codes clamp(rne(fl32(W' / s)), -7, 7).
template <typename T>
__global__ void __launch_bounds__(kThreads) linear4_prepare_kernel(const Linear4PrepArgs a) {
    const int groups = a.k_stride / a.group;
    const int64_t unit = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
    if (unit >= (int64_t)a.cout_pad * groups) return;
    const int lane = threadIdx.x & 63, p = (int)(unit / groups), g = (int)(unit - (int64_t)p * groups);
    const int ch = held_channel(a, p), per = a.group >> 6;   // values a lane
    float v[2] = {0.0f, 0.0f};
    for (int i = 0; i < per; ++i) {
        const int d = g * a.group + i * 64 + lane;
        if (ch >= 0 && d < a.cin) v[i] = transformed4(static_cast<const T *>(a.w) + (int64_t)ch * a.cin, d, a.hblock);
    }
    const float m = token_max(v);       // NaN kept
    const bool fine = m < __builtin_inff();
    const float s = fmaxf(__uint_as_float(bf16_pair(m / 7.0f, 0.0f) << 16), 0x1p-100f);
    for (int i = 0; i < per; ++i) {
        const int q = fine ? (int)__builtin_amdgcn_fmed3f(rintf(v[i] / s), -7.0f, 7.0f) : 0;
        // two codes a byte: input channels d and d + 4, lanes 4 apart
        const int other = __shfl_xor(q, 4, 64);
        if (!(lane & 4)) a.wpack[code_byte(a, p, g * a.group + i * 64 + lane)] = (uint8_t)((q & 15) | (other & 15) << 4);
    }
    if (lane == 0)
        a.w_scale[scale_index(a, p, g)] = ch < 0 ? (uint16_t)0 : fine ? (uint16_t)(__float_as_uint(s) >> 16) : (uint16_t)0x7fc0;
    if (lane == 0 && g == 0) a.bias[p] = ch >= 0 && a.bias_in ? a.bias_in[ch] : 0.0f;
}

// Codes that are there already: a lane the 16 packed bytes of its channel and chunk, a wave the
// 1 KB of 16 channels by 128 input channels, and their scales.  134 million codes in 90 us (a byte a
// lane: 1286), 2.2 TB/s of lines that 16 channels' rows share.
__global__ void __launch_bounds__(kThreads) linear4_pack_kernel(const Linear4PrepArgs a) {
    const int tiles = a.k_stride >> 7, S = 128 / a.group;
    const int64_t unit = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
    if (unit >= (int64_t)(a.cout_pad >> 4) * tiles) return;
    const int lane = threadIdx.x & 63, p16 = (int)(unit / tiles), k = (int)(unit - (int64_t)p16 * tiles);
    const int ch = held_channel(a, p16 * 16 + (lane & 15)), given = (a.cin + a.group - 1) / a.group;
    const bool whole = (reinterpret_cast<uintptr_t>(a.codes) & 15) == 0 && a.cin % 16 == 0;
    uint32_t out[4];
#pragma unroll
    for (int step = 0; step < 2; ++step) {
        const int d = k * 128 + step * 64 + (lane >> 4) * 16;
        const int8_t *from = a.codes + (int64_t)ch * a.cin + d;
        int8_t q[16] = {};
        if (ch >= 0 && d < a.cin) {
            if (whole) {
                *reinterpret_cast<v4u *>(q) = *reinterpret_cast<const v4u *>(from);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (d + j < a.cin) q[j] = from[j];
            }
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            uint32_t word = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int code = max(-8, min(7, (int)q[8 * w + j]));
                word |= (uint32_t)(code & 15) << ((j & 3) * 8 + (j & 4));
            }
            out[step * 2 + w] = word;
        }
    }
    *reinterpret_cast<v4u *>(a.wpack + unit * 1024 + lane * 16) = v4u{out[0], out[1], out[2], out[3]};
    if (lane < 16 * S) {
        // [4][S][4 channels]
        const int c = (lane / (4 * S)) * 4 + (lane & 3), g = k * S + (lane >> 2) % S;
        const int own = held_channel(a, p16 * 16 + c);
        a.w_scale[unit * (16 * S) + lane] = own >= 0 && g < given ? a.scale_in[(int64_t)own * given + g] : (uint16_t)0;
    }
    if (k == 0 && lane < 16) a.bias[p16 * 16 + lane] = ch >= 0 && a.bias_in ? a.bias_in[ch] : 0.0f;
}

template <typename T>
void prepare(const Linear4PrepArgs &a, hipStream_t st) {
    const int64_t units = (int64_t)a.cout_pad * (a.k_stride / a.group);
    linear4_prepare_kernel<T><<<grid_of((units + kThreads / 64 - 1) / (kThreads / 64)), kThreads, 0, st>>>(a);
}

template <typename T, int G, int S>
void token(const Linear4Args &a, const TokenArgs &x, hipStream_t st) {
    // A row or a few of a contraction that its split over 8 waves shortens go to the kernel of a
    // block a group (us, that one and the other: 1 row, 1024 -> 4096 3.9 and 4.8; 2 rows, 2048 ->
    // 4096 4.9 and 6.5; 4 rows, 2048 -> 4096 6.3 and 6.5; 16 rows, 1024 -> 4096 14.6 and 6.3; 1 row,
    // 1024 -> 16384 6.5 and 5.0).
    if (a.k_stride <= 512 || (a.k_stride <= 2048 && (a.rows >= 4 || a.cout > 8192))) {
        // column ranges, each of which quantizes the rows again: up to 512 blocks
        const int groups = (a.cout + 15) / 16, blocks = (a.rows + 15) / 16;
        const int most = blocks < 512 ? 512 / blocks : 1, ranges = (groups + 7) / 8 < most ? (groups + 7) / 8 : most;
        const int per = ((groups + ranges - 1) / ranges + 7) / 8 * 8;
        const dim3 grid(blocks, (groups + per - 1) / per);
        if (a.k_stride <= 512) linear4_small_kernel<T, G, S, 1><<<grid, 512, 0, st>>>(a, x, per);
        else if (a.k_stride <= 1024) linear4_small_kernel<T, G, S, 2><<<grid, 512, 0, st>>>(a, x, per);
        else linear4_small_kernel<T, G, S, 4><<<grid, 512, 0, st>>>(a, x, per);
        return;
    }
    const int grid = (a.cout + 15) / 16;
    const size_t bytes = kWaves * G * 1024 + 128 + (size_t)a.rows * (a.k_stride + 16);
    if (a.k_stride <= 4096) linear4_token_kernel<T, G, S, 1><<<grid, 512, bytes, st>>>(a, x);
    else if (a.k_stride <= 8192) linear4_token_kernel<T, G, S, 2><<<grid, 512, bytes, st>>>(a, x);
    else linear4_token_kernel<T, G, S, 4><<<grid, 512, bytes, st>>>(a, x);
}
template <int G, int S>
void token(const Linear4Args &a, const TokenArgs &x, hipStream_t st) {
    if (x.x_type == kF32) token<float, G, S>(a, x, st);
    else if (x.x_type == kBf16) token<bf16_t, G, S>(a, x, st);
    else token<_Float16, G, S>(a, x, st);
}

template <int G, int S, int MT, bool GATED>
void stream(const Linear4Args &a, hipStream_t st) {
    constexpr int N = GATED ? G / 2 : G;
    const int64_t groups = (a.cout + 15) / 16, sets = (groups + N - 1) / N;
    const int64_t row_tiles = (a.rows + 16 * MT - 1) / (16 * MT);
    const int tiles = a.k_stride >> 7;
    // waves on one set of groups while the sets do not fill the card, and while each has a tile
    int wk = 1;
    while (wk < kWaves && 2 * wk <= tiles && sets * row_tiles * wk < 4096) wk *= 2;
    const int cols = kWaves / wk;
    const size_t bytes = wk > 1 ? (size_t)kWaves * G * MT * 1024 : 0;
    linear4_stream_kernel<G, S, MT, GATED><<<grid_of((sets + cols - 1) / cols * row_tiles), 512, bytes, st>>>(a, wk);
}
// Two groups a wave of more than 16 rows, where they leave the card 256 sets; a gated layer's pair
// always.  In us at 1, 2 and 4 groups: 16 rows of 8192 -> 16384 16.3, 17.1, 18.0; 64 rows of 4096
// -> 4096 (128 sets of 2) 10.5, 12.5, 16.2; 128 of 16384 -> 4096 (256 of 2) 33.5, 29.1, 34.6; 128 of
// 4096 -> 16384 28.4, 24.8, 31.8; 512 of 4096 -> 4096 30.5, 26.6, 33.4.
template <int S, int MT>
void stream(const Linear4Args &a, hipStream_t st) {
    const int64_t sets = ((a.cout + 15) / 16 + 1) / 2, row_tiles = (a.rows + 16 * MT - 1) / (16 * MT);
    if (a.gated) return stream<2, S, MT, true>(a, st);
    if constexpr (MT > 1)
        if (sets * row_tiles >= 256) return stream<2, S, MT, false>(a, st);
    stream<1, S, MT, false>(a, st);
}
template <int S>
void stream(const Linear4Args &a, hipStream_t st) {
    if (a.rows <= 16) stream<S, 1>(a, st);
    else if (a.rows <= 32) stream<S, 2>(a, st);
    else stream<S, 4>(a, st);
}

}  // namespace

// Which tokens the product's blocks quantize themselves.  (us in a graph, so and through memory,
// bf16, 128 input channels a scale.)
// Contractions up to 1024: a pass of the small kernel over all tiles of 16 rows by 16 outputs is
// shorter than two launches up to 2^22 tiles' input channels, 2^23 of at most 256 groups: 16 rows,
// 512 -> 4096 4.8 and 5.7; 128, 1024 -> 4096 6.8 and 9.9; 77, 1024 -> 16384 12.7 and 12.2; 512, 1024
// -> 4096 11.3 and 12.8; 512, 256 -> 16384 18.4 and 15.6; 4096, 512 -> 512 7.9 and 14.3, 512 -> 4096
// 33.8 and 32.2.  Up to 2048: few rows (4 rows, 2048 -> 16384 7.6 and 7.9, 16 rows 9.7 and 8.1, gated
// 4 rows 9.3 and 7.0), and of more than 64 rows with few outputs (77, 2048 -> 4096 9.1 and 10.6; 512,
// 2048 -> 512 8.7 and 10.5; 32, 2048 -> 4096 8.8 and 7.5; gated 77, 2048 -> 2048 11.6 and 10.3).
// Longer ones: where every block quantizes all rows, up to 16 K codes, but 8 K of more than 512
// blocks: 4 rows, 4096 -> 4096 6.9 and 7.7; 1 row, 16384 -> 4096 11.2 and 13.4; 1 row, 8192 -> 16384
// 16.1 and 16.1; 4 rows, 4096 -> 16384 13.8 and 10.9; 1 row, 16384 -> 16384 38.9 and 26.3.
bool linear4_takes_tokens(int32_t rows, int32_t cout, int32_t gated, int32_t k_stride) {
    if (k_stride > 2048) return (int64_t)rows * k_stride <= (cout <= 8192 ? HATQ_TOKEN_CODES : HATQ_TOKEN_CODES / 2);
    if (rows < 4) return true;
    const int64_t groups = (int64_t)((cout + 15) / 16) * (gated ? 2 : 1), work = ((int64_t)rows + 15) / 16 * groups * k_stride;
    if (k_stride > 1024) return rows > 64 && !gated && groups <= 256 && work <= 1 << 23;
    return work <= (groups <= 256 ? 1 << 23 : 1 << 22);
}

hipError_t launch_linear4_prepare(const Linear4PrepArgs &a, hipStream_t st) {
    if (a.codes) {
        const int64_t units = (int64_t)(a.cout_pad >> 4) * (a.k_stride >> 7);
        linear4_pack_kernel<<<grid_of((units + kThreads / 64 - 1) / (kThreads / 64)), kThreads, 0, st>>>(a);
    } else if (a.w_type == kBf16) {
        prepare<bf16_t>(a, st);
    } else if (a.w_type == kF16) {
        prepare<_Float16>(a, st);
    } else {
        prepare<float>(a, st);
    }
    return hipGetLastError();
}

hipError_t launch_linear4_tokens(const Linear4Args &a, const TokenArgs &x, hipStream_t st) {
    if (a.gated) a.group == 64 ? token<2, 2>(a, x, st) : token<2, 1>(a, x, st);
    else a.group == 64 ? token<1, 2>(a, x, st) : token<1, 1>(a, x, st);
    return hipGetLastError();
}

hipError_t launch_linear4(const Linear4Args &a, hipStream_t st) {
    a.group == 64 ? stream<2>(a, st) : stream<1>(a, st);
    return hipGetLastError();
}

}  // namespace hatq
