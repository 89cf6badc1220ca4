// Attention over a 4-bit cache.
//
// Scores in the transformed basis (the orders' b cancel against one 1/b):
//   t[i][p] = scale/b sum_g s_k[p][g] sum_{d in g} (B q_i)[d] c_k[p][d]
//   y_i     = (1/b) B (sum_p w[i][p] s_v[p][g] c_v[p][d]),   w = softmax over p
// so the cache is never transformed: the queries are on the way in, the sums on the way
// out.  Both live in registers as matrix operands: positions are the rows of the first
// product and the contraction of the second, and the 32 positions of a step are dealt to the
// rows so that a lane's scores are the second product's operand as they are.
//
// First product: the query in whole numbers of ND bytes (16 or 24 bits of its largest
// value), INT8 matrix instructions on the bytes against the codes; sums are exact, the
// query's rounding is half a step, 2^-16 or 2^-24 of its largest value.
// Second product: weights w s_v in float16 against the codes in float16, exact.  A weight is
// kept relative to the largest of w s_v (not of w), so the float16 range holds whatever the
// scales are (2^-100 to 2^100): off by 2^-11 of each weight or 2^-25 of the largest.  For float16 and float32 results
// NP = 2 halves carry 22 bits of it.
#include "cache4_device.h"

#ifndef HATQ_ATTENTION_PART
#define HATQ_ATTENTION_PART 2
#endif

namespace hatq {
namespace {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.44269504088896341f;

// Over the four chunks of a column (lanes 16 apart).
__device__ __forceinline__ float chunks_max(float v) {
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const uint32_t w = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float chunks_maximum(float v) {   // NaN kept
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __builtin_elementwise_maximum(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const uint32_t w = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return __builtin_elementwise_maximum(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float chunks_sum(float v) {
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const uint32_t w = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// ---- which rows a tile has --------------------------------------------------------
// COLS columns of one sequence: column c is query row c / share, head c % share of the
// cached head's.
struct ColTile {
    int seq;            // -1: none
    int row0, count;    // the sequence's rows of the call
    int col0;
};
template <int COLS>
__device__ __forceinline__ ColTile col_tile(const AttentionArgs &a, int64_t t) {
    if (!a.at.ends) {
        const int count = a.at.rows / a.at.batch, per = (int)(((int64_t)count * a.share + COLS - 1) / COLS);
        const int64_t seq = t / per;
        if (seq >= a.at.batch) return {-1, 0, 0, 0};
        return {(int)seq, (int)seq * count, count, (int)(t - seq * per) * COLS};
    }
    const int lane = threadIdx.x & 63;
    int last = 0, tiles = 0;
    for (int base = 0; base < a.at.batch; base += 64) {
        const int i = base + lane;
        int end = i < a.at.batch ? a.at.ends[i] : 0;
        end = wave_scan(max(min(end, a.at.rows), last), [](int x, int y) { return max(x, y); });
        int begin = __builtin_amdgcn_update_dpp(0, end, 0x138, 0xF, 0xF, false);   // wave_shr 1
        if (lane == 0) begin = last;
        const int n = (int)(((int64_t)(end - begin) * a.share + COLS - 1) / COLS);
        const int c = wave_scan(n, [](int x, int y) { return x + y; });
        const int first = tiles + c - n;
        const uint64_t hit = __ballot(t >= first && t < first + n);
        if (hit) {
            const int l = __builtin_ctzll(hit), b = __builtin_amdgcn_readlane(begin, l);
            return {base + l, b, __builtin_amdgcn_readlane(end, l) - b,
                    (int)(t - __builtin_amdgcn_readlane(first, l)) * COLS};
        }
        last = __builtin_amdgcn_readlane(end, 63);
        tiles += __builtin_amdgcn_readlane(c, 63);
    }
    return {-1, 0, 0, 0};
}

// ---- sixteen columns of queries -----------------------------------------------------
template <int NB, int ND>
struct Query {
    v4i digit[ND][NB];      // most significant first
    float step;             // of the whole numbers, with the scores' factor
    int pos, from;          // last and first position seen
};

template <int NB, int ND>
__device__ __forceinline__ void load_query(const AttentionArgs &a, const ColTile &t, int head, int length, int col,
                                           Query<NB, ND> &q) {
    const int lane = threadIdx.x & 63, chunk = lane >> 4;
    const int c = min(t.col0 + col + (lane & 15), t.count * a.share - 1);
    const int i = c / a.share, g = c - i * a.share;
    float v[NB][16];
    const int64_t at = (int64_t)(t.row0 + i) * a.q.row + (int64_t)(head * a.share + g) * a.q.head;
#pragma unroll
    for (int b = 0; b < NB; ++b) load_head16(a.q, at, b * 64 + chunk * 16, a.c.dim, v[b]);
    head_butterfly(v, a.c.log_b, chunk, ChunksApart{});
    float m = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 16; ++j) m = __builtin_elementwise_maximum(m, fabsf(v[b][j]));
    m = chunks_maximum(m);
    // whole numbers of at most 127 2^(8 (ND - 1)): their lower bytes, signed, carry no further
    constexpr float kMost = ND == 2 ? 32512.0f : 8323072.0f;
    const float up = m > 0x1p-100f ? kMost / m : 0.0f;      // (below, its scores are taken as 0)
    const float factor = a.scale * kLog2e * __uint_as_float((uint32_t)(127 - a.c.log_b) << 23);
    // the codes come 16 times too large; a query that is not finite has scores NaN
    q.step = m < __builtin_inff() ? m * (1.0f / (kMost * 16.0f)) * factor : __builtin_nanf("");
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t d[ND][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                int n = (int)rintf(v[b][4 * w + j] * up);
#pragma unroll
                for (int k = ND - 1; k > 0; --k) {
                    d[k][j] = (uint32_t)n;
                    n = (n + 128) >> 8;
                }
                d[0][j] = (uint32_t)n;
            }
#pragma unroll
            for (int k = 0; k < ND; ++k) q.digit[k][b][w] = (int)pack_low_bytes(d[k][0], d[k][1], d[k][2], d[k][3]);
        }
    q.pos = a.causal ? length - t.count + i : length - 1;
    q.from = a.window ? max(q.pos - a.window + 1, 0) : 0;
}

// ---- running result of sixteen columns ------------------------------------------------
template <int NB>
struct Sums {
    v4f o[NB][4];       // [block][channel of the run]: runs are rows, columns lanes
    float m, l;         // the largest log2 of a weight so far; this lane's sum of weights
};

// One step's operands as they lie in memory.
template <int NB>
struct Step {
    v4u key[NB], value[NB], key_scale[NB], value_scale[NB];
    bool lacks;         // a page is not there
    bool there;         // the page of this lane's eight scores is
};

template <int NB>
__device__ __forceinline__ void load_step(const Cache4 &c, const Places4 &at, int seq, int head, int p0, Step<NB> &s) {
    // (the step's positions start at a multiple of 32: a page holds a half of it at least)
    const int lane = threadIdx.x & 63;
    const int slot = p0 >> c.log_page, slot2 = (p0 + 16) >> c.log_page;
    const int32_t *table = at.table + (int64_t)seq * at.width;
    int pa = table[min(slot, at.width - 1)], pb = table[min(slot2, at.width - 1)];
    const bool in_a = slot < at.width && (unsigned)pa < (unsigned)c.pages;
    const bool in_b = slot2 < at.width && (unsigned)pb < (unsigned)c.pages;
    s.lacks = !(in_a && in_b);
    const int mask = (1 << c.log_page) - 1;
    const int64_t oa = page_offset<NB>(c, in_a ? pa : 0, head), ob = page_offset<NB>(c, in_b ? pb : 0, head);
    const int octet_k = (lane & 15) >> 2, octet_v = lane >> 4;      // of the step's four
    s.there = octet_v < 2 ? in_a : in_b;
    const uint8_t *k = c.buf + (octet_k < 2 ? oa : ob) + (((p0 + 8 * octet_k) & mask) >> 3) * (NB * kOctet) +
                       (lane >> 4) * 64 + (lane & 3) * 16;
    const uint8_t *v = c.buf + (octet_v < 2 ? oa : ob) + (((p0 + 8 * octet_v) & mask) >> 3) * (NB * kOctet);
#pragma unroll
    for (int b = 0; b < NB; ++b) s.key[b] = *reinterpret_cast<const v4u *>(k + b * kKeyCodes);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        s.key_scale[b] = *reinterpret_cast<const v4u *>(v + NB * 512 + b * 16);
        s.value_scale[b] = *reinterpret_cast<const v4u *>(v + NB * 512 + (NB + b) * 16);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
        s.value[b] = *reinterpret_cast<const v4u *>(v + NB * kKeyCodes + b * 256 + (lane & 15) * 16);
}

__device__ __forceinline__ float scale_of(const v4u &w, int j) {
    return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
}

// One step of 32 positions from p0 on by NQ times sixteen columns.  EDGE: some of them may be
// hidden from some columns.
template <int NB, int ND, int NP, int NQ, bool EDGE>
__device__ __forceinline__ void step(const Step<NB> &s, const Query<NB, ND> (&q)[NQ], int p0, Sums<NB> (&sum)[NQ]) {
    const int lane = threadIdx.x & 63;
    const int first = p0 + 8 * (lane >> 4);
    // scales of this lane's eight positions; log2 of the values' largest, to 0.09 from below
    float lv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float most = scale_of(s.value_scale[0], j);
#pragma unroll
        for (int b = 1; b < NB; ++b) most = fmaxf(most, scale_of(s.value_scale[b], j));
        lv[j] = __builtin_fmaf((float)__float_as_int(most), 0x1p-23f, -127.0f);
    }
    v4i key[2][NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                key[h][b][2 * w] = (int)((s.key[b][2 * h + w] << 4) & 0xf0f0f0f0u);
                key[h][b][2 * w + 1] = (int)(s.key[b][2 * h + w] & 0xf0f0f0f0u);
            }
    v8h code[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v2h pair[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // 1024 + code + 8 as float16, less 1032
                const uint32_t bits = ((s.value[b][i] >> (4 * j)) & 0x000f000fu) | 0x64006400u;
                pair[i] = __builtin_bit_cast(v2h, bits) - v2h{(_Float16)1032.0f, (_Float16)1032.0f};
            }
            code[b][j] = v8h{pair[0][0], pair[0][1], pair[1][0], pair[1][1], pair[2][0], pair[2][1], pair[3][0], pair[3][1]};
        }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        float t[8];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v4i acc[ND];
#pragma unroll
                for (int k = 0; k < ND; ++k)
                    acc[k] = __builtin_amdgcn_mfma_i32_16x16x64_i8(key[h][b], q[n].digit[k][b], v4i{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    // |sum of one byte's products| < 2^20: two bytes' fit 31 bits
                    float f = (float)(acc[ND - 2][r] * 256 + acc[ND - 1][r]);
                    if (ND == 3) f = __builtin_fmaf((float)acc[0][r], 65536.0f, f);
                    const float w = scale_of(s.key_scale[b], 4 * h + r);
                    t[4 * h + r] = b == 0 ? f * w : __builtin_fmaf(f, w, t[4 * h + r]);
                }
            }
        float most = kLowest;
        bool seen[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            t[j] *= q[n].step;
            if (EDGE) {
                seen[j] = s.there && first + j <= q[n].pos && first + j >= q[n].from;
                t[j] = seen[j] ? t[j] : -__builtin_inff();
                most = fmaxf(most, seen[j] ? t[j] + lv[j] : kLowest);
            } else {
                most = fmaxf(most, t[j] + lv[j]);
            }
        }
        most = chunks_max(most);
        Sums<NB> &o = sum[n];
        if (__any(most > o.m)) {
            const float m = fmaxf(o.m, most), down = __builtin_amdgcn_exp2f(o.m - m);
            o.m = m;
            o.l *= down;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) o.o[b][j] *= down;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            t[j] = __builtin_amdgcn_exp2f(t[j] - o.m);
            o.l += t[j];
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            v8h high, low;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float w = t[j] * scale_of(s.value_scale[b], j);
                if (EDGE) w = seen[j] ? w : 0.0f;      // (a hidden position's scale may be anything)
                // (one rounded product for both halves: else one of them is made by v_fma_mixlo, which
                // rounds the exact product, and a tie goes up in one and down in the other)
                if (NP == 2) asm("" : "+v"(w));
                high[j] = (_Float16)w;
                if (NP == 2) low[j] = (_Float16)(w - (float)high[j]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                o.o[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(code[b][j], high, o.o[b][j], 0, 0, 0);
                if (NP == 2) o.o[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(code[b][j], low, o.o[b][j], 0, 0, 0);
            }
        }
    }
}

// Positions [from, to) that some column of a wave sees, `from` a multiple of 32.
template <int NB, int ND, int NP, int NQ>
__device__ __forceinline__ void walk(const AttentionArgs &a, int seq, int head, const Query<NB, ND> (&q)[NQ], int from,
                                     int to, int stride, int sure_from, int sure_to, Sums<NB> (&sum)[NQ]) {
    if (from >= to) return;
    Step<NB> s[2];
    load_step<NB>(a.c, a.at, seq, head, from, s[0]);
    for (int p = from; p < to; p += stride) {
        const int next = p + stride < to ? p + stride : p;
        load_step<NB>(a.c, a.at, seq, head, next, s[1]);
        // every column sees positions [sure_from, sure_to)
        if (p >= sure_from && p + 32 <= sure_to && !s[0].lacks) step<NB, ND, NP, NQ, false>(s[0], q, p, sum);
        else step<NB, ND, NP, NQ, true>(s[0], q, p, sum);
        s[0] = s[1];
    }
}

// Sums of a column whose m and l are whole: transformed, divided, stored.
template <int NB>
__device__ __forceinline__ void store_columns(const AttentionArgs &a, const ColTile &t, int head, int col,
                                              const v4f (&o)[NB][4], float l) {
    const int lane = threadIdx.x & 63, chunk = lane >> 4, c = t.col0 + col + (lane & 15);
    float v[NB][16];
    // (l = 0: no position is seen, and the sums are 0)
    const float by = l == 0.0f ? 0.0f : __uint_as_float((uint32_t)(127 - a.c.log_b) << 23) / l;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[b][4 * r + j] = o[b][j][r];
    head_butterfly(v, a.c.log_b, chunk, ChunksApart{});
    if (c >= t.count * a.share) return;
    const int i = c / a.share, g = c - i * a.share;
    const int64_t at = (int64_t)(t.row0 + i) * a.y.row + (int64_t)(head * a.share + g) * a.y.head;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[b][j] *= by;
        store_head16(a.y, at, b * 64 + chunk * 16, a.c.dim, v[b]);
    }
}

// Length of a sequence in the cache, by its table at most.
__device__ __forceinline__ int length_of(const AttentionArgs &a, int seq) {
    const int64_t most = (int64_t)a.at.width << a.c.log_page;
    const int n = max(a.at.lens[seq], 0);
    return n < most ? n : (int)most;
}

// Sums of `waves` waves (a power of two) of one tile into wave 0's: scaled to the same
// maximum and added by halves.  lds: waves * 128 bytes, and waves / 2 * NB * 4 KB.
template <int NB>
__device__ __forceinline__ void join_waves(Sums<NB> &s, int wave, int waves, char *lds) {
    float *ml = reinterpret_cast<float *>(lds);
    v4f *sums = reinterpret_cast<v4f *>(lds + waves * 128);
    const int lane = threadIdx.x & 63, col = lane & 15;
    const float l = chunks_sum(s.l);
    if (lane < 16) {
        ml[wave * 32 + col] = s.m;
        ml[wave * 32 + 16 + col] = l;
    }
    __syncthreads();
    float m = kLowest, all = 0.0f;
    for (int w = 0; w < waves; ++w) m = fmaxf(m, ml[w * 32 + col]);
    for (int w = 0; w < waves; ++w) all += ml[w * 32 + 16 + col] * __builtin_amdgcn_exp2f(ml[w * 32 + col] - m);
    const float down = __builtin_amdgcn_exp2f(s.m - m);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) s.o[b][j] *= down;
    s.m = m;
    s.l = all;
    for (int h = waves >> 1; h; h >>= 1) {
        if (wave >= h && wave < 2 * h) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) sums[(((wave - h) * NB + b) * 4 + j) * 64 + lane] = s.o[b][j];
        }
        __syncthreads();
        if (wave < h) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) s.o[b][j] += sums[((wave * NB + b) * 4 + j) * 64 + lane];
        }
        __syncthreads();
    }
}

// Sixteen columns a block, its waves each every W-th step of the block's share of the
// positions.
template <int NB, int ND, int NP>
__global__ void __launch_bounds__(512) attention4_kernel(const AttentionArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int split = (int)(block % a.splits), head = (int)(block / a.splits % a.c.heads);
    const int64_t tile = block / a.splits / a.c.heads;
    const ColTile t = col_tile<16>(a, tile);
    if (t.seq < 0) return;
    const int length = length_of(a, t.seq);
    Query<NB, ND> q[1];
    load_query<NB, ND>(a, t, head, length, 0, q[0]);
    // rows of the first and last column
    const int i0 = t.col0 / a.share, i1 = (min(t.col0 + 16, t.count * a.share) - 1) / a.share;
    int from = 0, to = length, sure_from = 0, sure_to = length;
    if (a.causal) {
        to = min(length, length - t.count + i1 + 1);
        sure_to = length - t.count + i0 + 1;
        if (a.window) {
            from = max(length - t.count + i0 - a.window + 1, 0) & ~31;
            sure_from = length - t.count + i1 - a.window + 1;
        }
    }
    const int64_t steps = to > from ? (to - from + 31) >> 5 : 0;
    const int begin = (int)(steps * split / a.splits), end = (int)(steps * (split + 1) / a.splits);
    Sums<NB> s[1];
    s[0].m = kLowest;
    s[0].l = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[0].o[b][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const int last = end == steps ? to : from + 32 * end;
    walk<NB, ND, NP, 1>(a, t.seq, head, q, from + 32 * (begin + wave), last, 32 * waves, sure_from, sure_to, s);
    join_waves<NB>(s[0], wave, waves, lds);
    if (wave) return;
    if (a.splits == 1) {
        store_columns<NB>(a, t, head, 0, s[0].o, s[0].l);
        return;
    }
    char *part = static_cast<char *>(a.ws) + ((tile * a.c.heads + head) * a.splits + split) * (int64_t)(NB * 4096 + 128);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) reinterpret_cast<v4f *>(part)[(b * 4 + j) * 64 + lane] = s[0].o[b][j];
    float *ml = reinterpret_cast<float *>(part + NB * 4096);
    if (lane < 16) {
        ml[lane] = s[0].m;
        ml[16 + lane] = s[0].l;
    }
}

// The partial results of a tile's splits, joined.
template <int NB>
__global__ void __launch_bounds__(512) attention4_join_kernel(const AttentionArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int head = (int)(block % a.c.heads);
    const int64_t tile = block / a.c.heads;
    const ColTile t = col_tile<16>(a, tile);
    if (t.seq < 0) return;
    const char *parts = static_cast<const char *>(a.ws) + (tile * a.c.heads + head) * a.splits * (int64_t)(NB * 4096 + 128);
    Sums<NB> s;
    s.m = kLowest;
    s.l = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) s.o[b][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = wave; k < a.splits; k += waves) {
        const char *part = parts + k * (int64_t)(NB * 4096 + 128);
        const float *ml = reinterpret_cast<const float *>(part + NB * 4096);
        const float m = ml[lane & 15], l = ml[16 + (lane & 15)];
        const float top = fmaxf(s.m, m), mine = __builtin_amdgcn_exp2f(s.m - top), its = __builtin_amdgcn_exp2f(m - top);
        s.m = top;
        // (join_waves adds the four chunks' l)
        s.l = s.l * mine + (lane < 16 ? l * its : 0.0f);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                s.o[b][j] = s.o[b][j] * mine + reinterpret_cast<const v4f *>(part)[(b * 4 + j) * 64 + lane] * its;
    }
    join_waves<NB>(s, wave, waves, lds);
    if (wave == 0) store_columns<NB>(a, t, head, 0, s.o, s.l);
}

// Many query rows: each wave 16 NQ columns of its own over all their positions; the waves of
// a block have adjacent columns and meet the same pages in its caches.
template <int NB, int ND, int NP, int NQ>
__global__ void __launch_bounds__(64 * kWideWaves) attention4_wide_kernel(const AttentionArgs a) {
    constexpr int COLS = 16 * NQ, WAVES = kWideWaves;
    const int wave = threadIdx.x >> 6;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int head = (int)(block % a.c.heads);
    ColTile t = col_tile<COLS * WAVES>(a, block / a.c.heads);
    if (t.seq < 0) return;
    t.col0 += wave * COLS;
    const int cols = t.count * a.share;
    if (t.col0 >= cols) return;
    const int length = length_of(a, t.seq);
    Query<NB, ND> q[NQ];
    Sums<NB> s[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        load_query<NB, ND>(a, t, head, length, 16 * n, q[n]);
        s[n].m = kLowest;
        s[n].l = 0.0f;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[n].o[b][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int i0 = t.col0 / a.share, i1 = (min(t.col0 + COLS, cols) - 1) / a.share;
    int from = 0, to = length, sure_from = 0, sure_to = length;
    if (a.causal) {
        to = min(length, length - t.count + i1 + 1);
        sure_to = length - t.count + i0 + 1;
        if (a.window) {
            from = max(length - t.count + i0 - a.window + 1, 0) & ~31;
            sure_from = length - t.count + i1 - a.window + 1;
        }
    }
    walk<NB, ND, NP, NQ>(a, t.seq, head, q, from, to, 32, sure_from, sure_to, s);
#pragma unroll
    for (int n = 0; n < NQ; ++n)
        if (t.col0 + 16 * n < cols) store_columns<NB>(a, t, head, 16 * n, s[n].o, chunks_sum(s[n].l));
}

dim3 blocks_of(int64_t n) {
    const int64_t x = n < (1 << 20) ? n : 1 << 20;
    return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}

template <int NB, int ND, int NP>
hipError_t launch(const AttentionArgs &a, const AttentionPlan &p, hipStream_t st) {
    if (p.wide) {
        constexpr int NQ = wide_cols(64 * NB) / 16;
        attention4_wide_kernel<NB, ND, NP, NQ><<<blocks_of(p.tiles * a.c.heads), 64 * kWideWaves, 0, st>>>(a);
        return hipGetLastError();
    }
    const size_t lds = (size_t)p.waves * (NB * 2048 + 128);
    attention4_kernel<NB, ND, NP><<<blocks_of(p.tiles * a.c.heads * p.splits), p.waves * 64, lds, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    attention4_join_kernel<NB><<<blocks_of(p.tiles * a.c.heads), p.waves * 64, lds, st>>>(a);
    return hipGetLastError();
}

}  // namespace

// One compilation a head size of 64 HATQ_ATTENTION_PART channels.
#define HATQ_LAUNCH2(n) launch_attention4_##n
#define HATQ_LAUNCH(n) HATQ_LAUNCH2(n)
hipError_t HATQ_LAUNCH(HATQ_ATTENTION_PART)(const AttentionArgs &a, const AttentionPlan &p, hipStream_t st) {
    constexpr int NB = HATQ_ATTENTION_PART;
    return a.q.type == kBf16 && a.y.type == kBf16 ? launch<NB, 2, 1>(a, p, st) : launch<NB, 3, 2>(a, p, st);
}

}  // namespace hatq
