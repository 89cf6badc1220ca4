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
// First product: the codes in float16, exact, against the query in two float16 halves, 22
// bits (many rows of bf16: one half, 11 bits) or 2^-38 of its largest value, after a power of two that
// puts that at 2^13 to 2^14; fp32 sums.
// Second product: weights w s_v in float16 against the codes in float16, exact.  A weight is
// kept in a unit that the largest w s_v (not w) so far passes by 2^12 to 2^15, so that the
// largest fits float16 whatever the scales are (2^-100 to 2^100) and small ones have all of its
// range below: off by 2^-11 of each (for float16 and float32 results in NP = 2 halves, 2^-21; bf16
// outputs round by 2^-8 themselves, and two halves, of the queries too, take 13 % more for 64 tokens
// of 16384 positions and 43 % for prompts), or by half of float16's least step, 2^-37 of the
// largest.  One unit serves a head's groups of 64 channels, so the largest is that of all of them: a
// group whose scales are that far below another's is lost.
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

__device__ __forceinline__ int wave_of_block() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Over the four chunks of a column (lanes 16 apart).  Maxima keep NaN, here and below: one
// instruction for three values, and where a score is NaN the column's results are.
__device__ __forceinline__ float chunks_max(float v) {
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

// a b and c d as two float16: the sum with 0 lets the compiler join a product and its rounding in
// one instruction, and it keeps the waits that a matrix instruction needs behind it.
__device__ __forceinline__ uint32_t product_pair(float a, float b, float c, float d) {
    return __builtin_bit_cast(uint32_t, v2h{(_Float16)__builtin_fmaf(a, b, 0.0f), (_Float16)__builtin_fmaf(c, d, 0.0f)});
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
struct Query {
    float step;             // of the products, with the scores' factor and log2 e
    int pos, from;          // last and first position seen
};

// Eight codes in each half byte of a word to float16: 1024 + code + 8 or 1024 + 16 (code + 8),
// less what is too much.  XOR: their code is two's complement, not code + 8.  The pairs come
// as half bytes (0, 4), (1, 5), (2, 6), (3, 7).
template <bool XOR>
__device__ __forceinline__ void unpack8(uint32_t x, v2h (&out)[4]) {
    const uint32_t low = XOR ? 0x64086408u : 0x64006400u, high = XOR ? 0x64806480u : 0x64006400u;
    const v2h sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f}, c72 = {(_Float16)-72.0f, (_Float16)-72.0f},
              c1032 = {(_Float16)1032.0f, (_Float16)1032.0f};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t w = k ? x >> 8 : x;
        // (and, then exclusive or, in one instruction)
        out[2 * k] = __builtin_bit_cast(v2h, __builtin_amdgcn_bitop3_b32(w, 0x000f000fu, low, 0x6a)) - c1032;
        out[2 * k + 1] = __builtin_elementwise_fma(
            __builtin_bit_cast(v2h, __builtin_amdgcn_bitop3_b32(w, 0x00f000f0u, high, 0x6a)), sixteenth, c72);
    }
}
__device__ __forceinline__ v8h join8(const v2h (&p)[4]) {
    return v8h{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}
// Which of eight adjacent channels the i-th value of a key's unpacked word is: its half bytes
// hold channels 0, 4, 1, 5, 2, 6, 3, 7.
__device__ __forceinline__ constexpr int key_channel(int i) { return (i >> 1) % 2 * 4 + (i >> 2) + (i & 1) * 2; }

// The operand of 16 columns, [NB][2 steps of 32 channels][2 halves][64 lanes], and then
// their steps, in LDS.
template <int NB>
constexpr int kQueryBytes = NB * 4096 + 64;
// Halves of the query that count: both, or one for many columns of bf16, where the second's
// products would take a third of the matrix instructions for bits that a bf16 output hides.
template <int NP, int NQ>
constexpr int kQueryHalves = NP == 1 && NQ > 1 ? 1 : 2;

template <int NB>
__device__ __forceinline__ void make_query(const AttentionArgs &a, const ColTile &t, int head, int col, char *lds) {
    const int lane = threadIdx.x & 63, chunk = lane >> 4;
    const int c = min(t.col0 + col + (lane & 15), t.count * a.share - 1);
    const int i = c / a.share, g = c - i * a.share;
    float v[NB][16];
    const int64_t at = (int64_t)(t.row0 + i) * a.q.row + (int64_t)(head * a.share + g) * a.q.head;
    load_head<NB>(a.q, at, chunk, a.c.dim, v, [] {});
    head_butterfly(v, a.c.log_b, ChunksApart{});
    float m = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 16; ++j) m = __builtin_elementwise_maximum(m, fabsf(v[b][j]));
    m = chunks_max(m);
    const int up = 14 - __builtin_amdgcn_frexp_expf(m);
    const float factor = a.scale * kLog2e * __uint_as_float((uint32_t)(127 - a.c.log_b) << 23);
    // (a query that is not finite has scores NaN)
    if (chunk == 0)
        reinterpret_cast<float *>(lds + NB * 4096)[lane] =
            m < __builtin_inff() ? __builtin_amdgcn_ldexpf(factor, -up) : __builtin_nanf("");
    v8h *const to = reinterpret_cast<v8h *>(lds);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            v8h half[2];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = __builtin_amdgcn_ldexpf(v[b][8 * w + key_channel(j)], up);
                half[0][j] = (_Float16)x;
                half[1][j] = (_Float16)(x - (float)half[0][j]);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) to[((b * 2 + w) * 2 + k) * 64 + lane] = half[k];
        }
}

// The first position that a row at `pos` sees.
__device__ __forceinline__ int first_seen(int pos, int window) { return window <= 0 || window > pos ? 0 : pos - window + 1; }

// The positions that this lane's column sees.
template <int NB>
__device__ __forceinline__ void see(const AttentionArgs &a, const ColTile &t, int length, int col, Query &q) {
    const int c = min(t.col0 + col + (int)(threadIdx.x & 15), t.count * a.share - 1);
    q.pos = a.causal ? length - t.count + c / a.share : length - 1;
    q.from = first_seen(q.pos, a.window);
}

// ---- running result of sixteen columns ------------------------------------------------
template <int NB>
struct Sums {
    v4f o[NB][4];       // [block][channel of the run]: runs are rows, columns lanes
    float m, l;         // log2 of the unit of a weight; this lane's sum of weights, times kSumDown
};
// log2 of where the unit is put, below the largest weight, and of where that may grow to before the
// unit follows.  (2^7 and 2^15 took as long, and kept 5 bits less of small weights.)
constexpr float kUnitBelow = 12.0f, kUnitFollows = 15.0f;
// From here on (a score's magnitude, times log2 e) float32 no longer holds a unit to a small part of a
// power of two.
constexpr float kLargeScore = 0x1p20f;
// A weight without its scale is up to 2^115: sums of 2^24 of them stay finite.
constexpr int kSumDownLog = 12;
constexpr float kSumDown = 0x1p-12f;

// One step's operands as they lie in memory.  Each part is loaded again, for the step after,
// as soon as it has been used, so a step's loads are under way over the rest of the step
// before and no second set of registers is kept.
template <int NB>
struct Step {
    v4u key[NB], key_scale[NB], value_scale[NB], value[NB];
};

// A step's pages: of its two halves where pages have 16 positions, else one.
struct Pages {
    int a, b;
};
template <bool HALF>
__device__ __forceinline__ Pages pages_of(const Cache4 &c, const Places4 &at, const int32_t *table, int p0) {
    const int slot = p0 >> c.log_page, slot2 = (p0 + 16) >> c.log_page;
    const int a = slot < at.width ? table[slot] : -1;
    return {a, !HALF ? a : slot2 < at.width ? table[slot2] : -1};
}

// Where the parts of a step are: this lane's octets of the keys and the values, at `base` or,
// where pages have 16 positions, `half` on for the lanes of the second half.
struct StepAt {
    const uint8_t *base;
    int64_t half;
    bool lacks;         // a page is not there
    bool there;         // the page of this lane's eight scores is
};

// The parts of a lane's addresses that are the same for every step.
struct LaneAt {
    uint32_t key, value, run;
    bool key_half, value_half;      // in the second page of a step
};
template <int NB, bool HALF>
__device__ __forceinline__ LaneAt lane_at() {
    const uint32_t lane = threadIdx.x & 63, octet_k = (lane & 15) >> 2, octet_v = lane >> 4;
    const uint32_t mask = HALF ? 1 : 3;
    const uint32_t v = (octet_v & mask) * (NB * kOctet);
    return {(octet_k & mask) * (NB * kOctet) + (lane >> 4) * 64 + (lane & 3) * 16, v + NB * 512, v + NB * kKeyCodes + (lane & 15) * 16,
            octet_k >= 2, octet_v >= 2};
}

template <int NB, bool HALF>
__device__ __forceinline__ StepAt step_at(const Cache4 &c, int64_t head0, const LaneAt &lane, const Pages &p, int p0) {
    const bool in_a = (unsigned)p.a < (unsigned)c.pages, in_b = (unsigned)p.b < (unsigned)c.pages;
    const int64_t page = (int64_t)c.heads * ((int64_t)(NB * kOctet) << (c.log_page - 3));
    const int mask = (1 << c.log_page) - 1;
    const uint8_t *base = c.buf + head0 + ((p0 & mask) >> 3) * (NB * kOctet) + (in_a ? p.a : 0) * page;
    if constexpr (HALF) {
        return {base, ((int64_t)(in_b ? p.b : 0) - (in_a ? p.a : 0)) * page, !(in_a && in_b), lane.value_half ? in_b : in_a};
    } else {
        return {base, 0, !in_a, in_a};
    }
}
template <bool HALF>
__device__ __forceinline__ v4u load_part(const StepAt &at, uint32_t offset, bool second) {
    const uint8_t *base = at.base;
    if constexpr (HALF) base += second ? at.half : 0;
    return *reinterpret_cast<const v4u *>(base + offset);
}
template <int NB, bool HALF>
__device__ __forceinline__ void load_keys(const StepAt &at, const LaneAt &lane, int b, Step<NB> &s) {
    s.key[b] = load_part<HALF>(at, lane.key + b * kKeyCodes, lane.key_half);
}
template <int NB, bool HALF>
__device__ __forceinline__ void load_scales(const StepAt &at, const LaneAt &lane, int which, v4u (&to)[NB]) {
#pragma unroll
    for (int b = 0; b < NB; ++b) to[b] = load_part<HALF>(at, lane.value + (which * NB + b) * 16, lane.value_half);
}
template <int NB, bool HALF>
__device__ __forceinline__ void load_values(const StepAt &at, const LaneAt &lane, int b, Step<NB> &s) {
    s.value[b] = load_part<HALF>(at, lane.run + b * 256, lane.value_half);
}

__device__ __forceinline__ float scale_of(const v4u &w, int j) {
    return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
}

// One step of 32 positions from p0 on by NQ times sixteen columns, and the next one's loads.
// EDGE: some positions may be hidden from some columns.  large: 1 once a column's largest score
// was kLargeScore or more.
template <int NB, int NP, int NQ, bool EDGE, bool HALF>
__device__ __forceinline__ void step(Step<NB> &s, const StepAt &here, const StepAt &next, const LaneAt &mine, const Query (&q)[NQ],
                                     const char *query, int p0, Sums<NB> (&sum)[NQ], uint32_t &large) {
    const int lane = threadIdx.x & 63;
    const int first = p0 + 8 * (lane >> 4);
    float t[NQ][8];
    uint32_t x_at = lane * 16;
    asm volatile("" : "+v"(x_at));      // read in every step: kept over the loop, the query's registers spill
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        v4f acc[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) acc[n][h] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            v8h key[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v2h pair[4];
                unpack8<true>(s.key[b][2 * h + w], pair);
                key[h] = join8(pair);
            }
            if (w) load_keys<NB, HALF>(next, mine, b, s);
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int k = 0; k < kQueryHalves<NP, NQ>; ++k) {
                    const v8h x = *reinterpret_cast<const v8h *>(query + n * kQueryBytes<NB> + ((b * 2 + w) * 2 + k) * 1024 + x_at);
#pragma unroll
                    for (int h = 0; h < 2; ++h) acc[n][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key[h], x, acc[n][h], 0, 0, 0);
                }
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = acc[n][j >> 2][j & 3], w = scale_of(s.key_scale[b], j);
                t[n][j] = b == 0 ? f * w : __builtin_fmaf(f, w, t[n][j]);
            }
    }
    load_scales<NB, HALF>(next, mine, 0, s.key_scale);
    // log2 of the largest scale of a value, to 0.09 from below, from its bf16 bits; one column
    // tile takes it as they are, 128 (127 + log2), and many spare the registers of 128 times
    // their steps, which spill
    constexpr bool kBits = NQ == 1;
    float lv[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        typedef uint16_t v2s __attribute__((ext_vector_type(2)));
        // (a word by itself: a cast of a vector's element takes the first one's)
        const auto pair = [&](int b) {
            const uint32_t w = s.value_scale[b][i];
            return __builtin_bit_cast(v2s, w);
        };
        v2s most = pair(0);
#pragma unroll
        for (int b = 1; b < NB; ++b) most = __builtin_elementwise_max(most, pair(b));
#pragma unroll
        for (int k = 0; k < 2; ++k)
            lv[2 * i + k] = kBits ? (float)most[k] : __builtin_fmaf((float)most[k], 0x1p-7f, -127.0f);
    }
    uint32_t seen[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        Sums<NB> &o = sum[n];
        float most = -__builtin_inff();
        if (EDGE) {
            // positions first + j that the column sees, as bits
            const int lo = min(max(q[n].from - first, 0), 8), hi = min(max(q[n].pos + 1 - first, 0), 8);
            seen[n] = here.there ? ((1u << hi) - 1) & ~((1u << lo) - 1) : 0u;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float x = __builtin_fmaf(t[n][j], kBits ? q[n].step * 128.0f : q[n].step, lv[j]);
            most = __builtin_elementwise_maximum(most, !EDGE || (seen[n] >> j & 1) ? x : -__builtin_inff());
        }
        most = chunks_max(most);
        if (kBits) most = __builtin_fmaf(most, 0x1p-7f, -127.0f);
        // (A weight may be up to 2^15 of the unit before the unit follows: float16 has room for
        // that, and most columns' largest grows by less after its first step.)
        if (__builtin_expect(__any(most > o.m + kUnitFollows) || large, 0)) {
            // (NaN stays; two float32 steps less, so that rounding does not leave the largest below)
            const float to = __builtin_fmaf(fabsf(most), -0x1p-22f, most - kUnitBelow);
            const float m = to <= o.m ? o.m : to, down = __builtin_amdgcn_exp2f(o.m - m);
            o.m = m;
            o.l *= down;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) o.o[b][j] *= down;
            if (__any(fabsf(most) >= kLargeScore && most > -__builtin_inff())) large = 1;
        }
        // (a step's weights among themselves first: alone, small ones are lost beside a large sum)
        float all = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) t[n][j] = __builtin_fmaf(t[n][j], q[n].step, -o.m);
        if (__builtin_expect(large != 0, 0)) {
            // The unit may be off by several powers of two, as the scores themselves are: a weight
            // above 2^15 of it is taken as that much, for float16 would not hold it.
#pragma unroll
            for (int j = 0; j < 8; ++j)
                t[n][j] = __builtin_elementwise_minimum(
                    t[n][j], kBits ? __builtin_fmaf(lv[j], -0x1p-7f, kUnitFollows + 127.0f) : kUnitFollows - lv[j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float p = __builtin_amdgcn_exp2f(t[n][j]);
            t[n][j] = !EDGE || (seen[n] >> j & 1) ? p : 0.0f;
            all = j ? all + t[n][j] : t[n][j];
        }
        o.l = __builtin_fmaf(all, kSumDown, o.l);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        v8h weight[NQ][NP];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            // (a hidden position's scale may be anything)
            const auto scale = [&](int j) { return !EDGE || (seen[n] >> j & 1) ? scale_of(s.value_scale[b], j) : 0.0f; };
            if constexpr (NP == 1 && NQ == 1) {
                uint32_t pair[4];
#pragma unroll
                for (int j = 0; j < 8; j += 2) pair[j >> 1] = product_pair(t[n][j], scale(j), t[n][j + 1], scale(j + 1));
                weight[n][0] = __builtin_bit_cast(v8h, v4u{pair[0], pair[1], pair[2], pair[3]});
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float w = t[n][j] * scale(j);
                    // (one rounded product for both halves: else one of them is made by v_fma_mixlo, which
                    // rounds the exact product, and a tie goes up in one and down in the other)
                    if (NP == 2) asm("" : "+v"(w));
                    weight[n][0][j] = (_Float16)w;
                    if (NP == 2) weight[n][NP - 1][j] = (_Float16)(w - (float)weight[n][0][j]);
                }
            }
        }
        v2h code[4][4];     // [word: positions][channel of the run]
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack8<false>(s.value[b][i], code[i]);
        load_values<NB, HALF>(next, mine, b, s);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const v2h word[4] = {code[0][j], code[1][j], code[2][j], code[3][j]};
            const v8h x = join8(word);
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int k = 0; k < NP; ++k)
                    sum[n].o[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, weight[n][k], sum[n].o[b][j], 0, 0, 0);
        }
    }
    load_scales<NB, HALF>(next, mine, 1, s.value_scale);
}

// Every stride-th step of the positions [from, to) that some column of a wave sees, `from` a
// multiple of 32; every column sees all of [sure_from, sure_to).  The first step's loads are
// made at once, before the queries.
template <int NB, bool HALF>
struct Walk {
    const AttentionArgs &a;
    const int32_t *table;
    const int64_t head0;
    const int from, to, stride;
    const LaneAt mine;
    Step<NB> s;
    StepAt here;
    Pages pages;
    uint32_t large = 0;

    // (the step after a wave's last one: the same again, not used)
    __device__ __forceinline__ int after(int p) const { return p + stride < to ? p + stride : p; }

    __device__ __forceinline__ Walk(const AttentionArgs &args, int seq, int head, int begin, int end, int by)
        : a(args), table(args.at.table + (int64_t)seq * args.at.width), head0(page_offset<NB>(args.c, 0, head)), from(begin),
          to(end), stride(by), mine(lane_at<NB, HALF>()) {
        if (from >= to) return;
        here = step_at<NB, HALF>(a.c, head0, mine, pages_of<HALF>(a.c, a.at, table, from), from);
#pragma unroll
        for (int b = 0; b < NB; ++b) load_keys<NB, HALF>(here, mine, b, s);
        load_scales<NB, HALF>(here, mine, 0, s.key_scale);
        load_scales<NB, HALF>(here, mine, 1, s.value_scale);
#pragma unroll
        for (int b = 0; b < NB; ++b) load_values<NB, HALF>(here, mine, b, s);
        pages = pages_of<HALF>(a.c, a.at, table, after(from));
        __builtin_amdgcn_sched_barrier(0);
    }

    template <int NP, int NQ, bool EDGE>
    __device__ __forceinline__ void one(int p, const Query (&q)[NQ], const char *query, Sums<NB> (&sum)[NQ]) {
        const StepAt next = step_at<NB, HALF>(a.c, head0, mine, pages, after(p));
        pages = pages_of<HALF>(a.c, a.at, table, after(after(p)));
        step<NB, NP, NQ, EDGE, HALF>(s, here, next, mine, q, query, p, sum, large);
        here = next;
    }
    template <int NP, int NQ>
    __device__ __forceinline__ void run(const Query (&q)[NQ], const char *query, int sure_from, int sure_to, Sums<NB> (&sum)[NQ]) {
        const auto sure = [&](int p) { return p >= sure_from && p + 32 <= sure_to && !here.lacks; };
        // (a loop each: as the branches of one, the compiler makes both kinds' common parts first and
        // keeps all of them)
        for (int p = from; p < to;) {
            for (; p < to && sure(p); p += stride) one<NP, NQ, false>(p, q, query, sum);
            for (; p < to && !sure(p); p += stride) one<NP, NQ, true>(p, q, query, sum);
        }
    }
};

// Sums of a column whose m and l are whole: transformed, divided, stored.
template <int NB>
__device__ __forceinline__ void store_columns(const AttentionArgs &a, const ColTile &t, int head, int col,
                                              const v4f (&o)[NB][4], float l) {
    const int lane = threadIdx.x & 63, chunk = lane >> 4, c = t.col0 + col + (lane & 15);
    float v[NB][16];
    // (l = 0: no position is seen, and the sums are 0)
    const float by = l == 0.0f ? 0.0f : __uint_as_float((uint32_t)(127 - kSumDownLog - a.c.log_b) << 23) / l;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[b][4 * r + j] = o[b][j][r];
    head_butterfly(v, a.c.log_b, ChunksApart{});
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

// Sums of `waves` waves of one tile into wave 0's: every wave leaves its own in LDS, every
// thread adds the waves' values of some of them.  lds: waves * (NB * 4 KB + 128 bytes), not in
// use by others.
template <int NB>
__device__ __forceinline__ void join_waves(Sums<NB> &s, int wave, int waves, char *lds) {
    if (waves == 1) {
        s.l = chunks_sum(s.l);
        return;
    }
    v4f *const sums = reinterpret_cast<v4f *>(lds);
    float *const ml = reinterpret_cast<float *>(lds + waves * (NB * 4096));
    const int lane = threadIdx.x & 63, col = lane & 15;
    const float l = chunks_sum(s.l);
    if (lane < 16) {
        ml[wave * 32 + col] = s.m;
        ml[wave * 32 + 16 + col] = l;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[((wave * NB + b) * 4 + j) * 64 + lane] = s.o[b][j];
    __syncthreads();
    float m = kLowest, all = 0.0f;
    for (int w = 0; w < waves; ++w) m = fmaxf(m, ml[w * 32 + col]);
    for (int i = wave; i < NB * 4; i += waves) {
        v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int w = 0; w < waves; ++w) x += sums[(w * NB * 4 + i) * 64 + lane] * __builtin_amdgcn_exp2f(ml[w * 32 + col] - m);
        // (in the first wave's place, which no other thread reads here)
        sums[i * 64 + lane] = x;
    }
    if (wave == 0)
        for (int w = 0; w < waves; ++w) all += ml[w * 32 + 16 + col] * __builtin_amdgcn_exp2f(ml[w * 32 + col] - m);
    s.m = m;
    s.l = all;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) s.o[b][j] = sums[(b * 4 + j) * 64 + lane];
    }
}

// 16 NQ columns a block, its waves each every W-th step of the block's share of the
// positions.  NQ > 1 where there are many columns: a step's codes are unpacked once for all of
// them.  (Its waves share the positions there too, not the columns: blocks then last a
// fourth as long, and the last ones of a full card leave less of it idle.)
// What bounds it: few columns, the cache's bytes while enough waves have a step of 4 KB under
// way each (64 sequences of 16384, 8 heads of 128 channels: 226 us for 1.09 GB, 4.8 TB/s), behind 6
// to 8 us for the query, the first loads and the waves' sums (2 sequences of 131072, 4 heads:
// 44 us for 143 MB); many columns, the vector instructions of weights and codes beside the matrix
// ones, and blocks of unlike length (the last 1365 rows of prompts of 5461 to 8192 positions, three of
// them, 16 heads over 2 of 128: 355 us, 580 TFLOP/s of 1200 that a large float16 product reaches).
template <int NB, int NP, int NQ, bool HALF>
__global__ void __launch_bounds__(NQ > 1 ? 256 : NB <= 2 ? 1024 : 512) __attribute__((amdgpu_waves_per_eu(NB <= 2 && NQ == 1 ? 4 : 2)))
attention4_kernel(const AttentionArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int waves = blockDim.x >> 6, wave = wave_of_block(), lane = threadIdx.x & 63;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int split = (int)(block % a.splits), head = (int)(block / a.splits % a.c.heads);
    const int64_t tile = block / a.splits / a.c.heads;
    const ColTile t = col_tile<16 * NQ>(a, tile);
    if (t.seq < 0) return;
    const int length = max(a.at.lens[t.seq], 0), cols = t.count * a.share;
    const int most = a.at.width << a.c.log_page;    // positions of a table, up to 2^30
    // rows of the first and last column
    const int i0 = t.col0 / a.share, i1 = (min(t.col0 + 16 * NQ, cols) - 1) / a.share;
    int from = 0, to = length, sure_from = 0, sure_to = length;
    if (a.causal) {
        to = min(length, length - t.count + i1 + 1);
        sure_to = length - t.count + i0 + 1;
        from = first_seen(length - t.count + i0, a.window) & ~31;
        sure_from = first_seen(length - t.count + i1, a.window);
    }
    // (a length may pass its table: its rows' positions count from there all the same)
    to = min(to, most);
    from = min(from, to);
    const int64_t steps = to > from ? (to - from + 31) >> 5 : 0;
    const int begin = (int)(steps * split / a.splits), end = (int)(steps * (split + 1) / a.splits);
    Walk<NB, HALF> walk(a, t.seq, head, from + 32 * (begin + wave), end == steps ? to : from + 32 * end, 32 * waves);
    Query q[NQ];
    Sums<NB> s[NQ];
    // (sixteen columns a wave, NQ waves at least: made by all, it would take as long as two steps)
    char *const query = lds;
    if (wave < NQ) make_query<NB>(a, t, head, 16 * wave, query + wave * kQueryBytes<NB>);
#pragma unroll
    for (int n = 0; n < NQ; ++n) see<NB>(a, t, length, 16 * n, q[n]);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NQ; ++n)
        q[n].step = *reinterpret_cast<const float *>(query + n * kQueryBytes<NB> + NB * 4096 + 4 * (lane & 15));
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        s[n].m = kLowest;
        s[n].l = 0.0f;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[n].o[b][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
    walk.template run<NP, NQ>(q, query, sure_from, sure_to, s);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        __syncthreads();    // the LDS of before has been read
        join_waves<NB>(s[n], wave, waves, lds);
        if (wave == 0 && a.splits == 1 && t.col0 + 16 * n < cols) store_columns<NB>(a, t, head, 16 * n, s[n].o, s[n].l);
    }
    if (wave || a.splits == 1) return;
    // (NQ = 1)
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
__global__ void __launch_bounds__(1024) attention4_join_kernel(const AttentionArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int waves = blockDim.x >> 6, wave = wave_of_block(), lane = threadIdx.x & 63;
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
    // (two parts under way at once: 2 sequences of 131072 48.9 -> 48.1 us; heads of more than 128
    // channels have no registers for it)
    constexpr int kParts = NB <= 2 ? 2 : 1;
#pragma unroll kParts
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

dim3 blocks_of(int64_t n) {
    const int64_t x = n < (1 << 20) ? n : 1 << 20;
    return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}

template <int NB, int NP, bool HALF>
hipError_t launch(const AttentionArgs &a, const AttentionPlan &p, hipStream_t st) {
    constexpr int NQ = wide_cols(64 * NB) / 16;
    const size_t join = p.waves > 1 ? (size_t)p.waves * (NB * 4096 + 128) : 0, query = (size_t)(p.cols / 16) * kQueryBytes<NB>;
    const size_t lds = join > query ? join : query;
    const dim3 grid = blocks_of(p.tiles * a.c.heads * p.splits);
    if (NQ == 1 || p.cols == 16) attention4_kernel<NB, NP, 1, HALF><<<grid, p.waves * 64, lds, st>>>(a);
    else attention4_kernel<NB, NP, NQ, HALF><<<grid, p.waves * 64, lds, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    attention4_join_kernel<NB><<<blocks_of(p.tiles * a.c.heads), p.waves * 64, join, st>>>(a);
    return hipGetLastError();
}

}  // namespace

// One compilation a head size of 64 HATQ_ATTENTION_PART channels.
#define HATQ_LAUNCH2(n) launch_attention4_##n
#define HATQ_LAUNCH(n) HATQ_LAUNCH2(n)
hipError_t HATQ_LAUNCH(HATQ_ATTENTION_PART)(const AttentionArgs &a, const AttentionPlan &p, hipStream_t st) {
    constexpr int NB = HATQ_ATTENTION_PART;
    const bool half = a.c.log_page == 4;
    if (a.q.type == kBf16 && a.y.type == kBf16) return half ? launch<NB, 1, true>(a, p, st) : launch<NB, 1, false>(a, p, st);
    return half ? launch<NB, 2, true>(a, p, st) : launch<NB, 2, false>(a, p, st);
}

}  // namespace hatq
