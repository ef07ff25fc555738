// The chosen experts of few rows: up and gate product, activation and weight, down
// product and the sum over a row's experts, in two launches (include/mp_layers.h).
//
// Bound by reading the chosen experts' weights, once.  Every workgroup finds the
// experts that some row chose and the rows of each from idx by itself (a count
// and a scan in LDS), so that no launch is spent on it.
//   up:    a workgroup has 32 weight rows of an expert (16 of the gate and their 16
//          of the other half), its wavefronts share K; h = act(.) * weight is left
//          as a sum of bf16 terms.
//   down:  a workgroup has 32 output columns and a share of the (expert, step of K)
//          items, its wavefronts a run of them; what they add to each row is
//          joined in LDS, and the shares by the workgroup that ends last.
// Products run on v_mfma_f32_16x16x32_bf16, weights first, so that a lane's
// accumulators are neighbouring columns of one row.  4-bit weights are exact in
// bf16, and so are 8-bit rows; fp32 values (rows, and h) are taken as sums of three
// bf16 terms, which are exact.  (h with two terms, 16 bits, is a third less to load:
// 2 of 8 experts for one row 15.9 us for 16.2, 8 of 64 for 16 8-bit rows 47.9 for 51.9, 4
// of 64 for 64 rows 165 for 170; h in fp32, taken apart by the second launch, 17.4, 56.5
// and 167.)
// 8-bit rows times 4-bit weights go the same way.  v_mfma_scale_f32_16x16x128_f8f6f4
// takes them as they are, but adds each 8 neighbouring products of a lane to some 15 bits
// below the largest (448 * 6 + 0.125 * 0.5 is 448 * 6): sums off by 2^-17 of their size, in
// 52 us for 59 (8 of 64 experts for 16 rows, both launches).
#include "layers_internal.hpp"

namespace mp {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 256;
constexpr int kWaves = kBlock / kWave;
constexpr int kStep = 128;    // elements of K of a step, 32 for a quarter of the lanes
constexpr int kCols = 32;     // weight rows of a workgroup
constexpr int64_t kUpGrid = 512;  // workgroups of the first launch, at most
constexpr int kLine = 36;     // floats of a row's sums in LDS

// 2^(s - 127) (s = 0 is subnormal); NaN for 255.
__device__ inline float scale_value(uint32_t s) {
    return __uint_as_float(s == 255 ? 0x7FC00000u : (s ? s << 23 : 0x00400000u));
}

// ---- the rows of every expert ------------------------------------------------------
// In LDS: the pairs (row, choice) of each expert that has any.  A choice that repeats
// an expert of its row is left out; its weight goes to the first.
struct Lists {
    int* first;      // [E + 1] first place of an expert's pairs
    int* cursor;     // [E] (the count, at first)
    int* active;     // [E] experts that have pairs, in order
    int* chosen;     // [P] expert of a pair, or -1
    int* pairs;      // [P] by expert
    int* total;      // [1] how many are active
    float* given;    // [P] the choices' weights
    float* weight;   // [P] a pair's: that of its choice and of later ones of its expert
};
__host__ __device__ inline int list_words(int E, int P) { return 3 * E + 4 * P + 2; }

__device__ inline Lists carve(int* lds, int E, int P) {
    Lists l;
    l.first = lds;
    l.cursor = l.first + E + 1;
    l.active = l.cursor + E;
    l.chosen = l.active + E;
    l.pairs = l.chosen + P;
    l.total = l.pairs + P;
    l.given = reinterpret_cast<float*>(l.total + 1);
    l.weight = l.given + P;
    return l;
}

__device__ inline void find_rows(const ExpertParams& p, const Lists& l) {
    const int tid = threadIdx.x, lane = tid & 63;
    for (int i = tid; i < p.P; i += kBlock) {
        const int e = p.idx[i];
        l.chosen[i] = e >= 0 && e < p.E ? e : -1;
        l.given[i] = p.weight[i];
    }
    for (int e = tid; e < p.E; e += kBlock) l.cursor[e] = 0;
    __syncthreads();
    for (int i = tid; i < p.P; i += kBlock) {
        const int e = l.chosen[i], r0 = i - i % p.k;
        bool again = e < 0;
        float weight = l.given[i];
        for (int j = r0; j < i; ++j) again |= l.chosen[j] == e;
        for (int j = i + 1; j < r0 + p.k; ++j) weight += l.chosen[j] == e ? l.given[j] : 0.f;
        l.pairs[i] = again ? -1 : e;
        l.weight[i] = weight;
    }
    __syncthreads();
    for (int i = tid; i < p.P; i += kBlock) {
        l.chosen[i] = l.pairs[i];
        if (l.pairs[i] >= 0) atomicAdd(&l.cursor[l.pairs[i]], 1);
    }
    __syncthreads();
    if (tid < 64) {  // a wavefront's scan, 64 experts at a time
        int places = 0, experts = 0;
        for (int e0 = 0; e0 < p.E; e0 += 64) {
            const int e = e0 + lane, n = e < p.E ? l.cursor[e] : 0;
            int sum = n;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_up(sum, o);
                if (lane >= o) sum += v;
            }
            const uint64_t some = __ballot(n > 0);
            if (e < p.E) {
                l.first[e] = places + sum - n;
                l.cursor[e] = places + sum - n;
            }
            if (n > 0) l.active[experts + (int)count_below(some)] = e;
            places += __shfl(sum, 63);
            experts += __popcll(some);
        }
        if (lane == 0) {
            l.first[p.E] = places;
            *l.total = experts;
        }
    }
    __syncthreads();
    // (the order of an expert's pairs is left open: each has its own row of h and of
    // the sums, whatever its place in a product)
    for (int i = tid; i < p.P; i += kBlock)
        if (l.chosen[i] >= 0) l.pairs[atomicAdd(&l.cursor[l.chosen[i]], 1)] = i;
    __syncthreads();
}

// Words of the lists that the second launch takes over.
__host__ __device__ inline int kept_words(int E, int P) { return 2 * E + P + 2; }

__device__ inline void keep_rows(const ExpertParams& p, const Lists& l) {
    const int tid = threadIdx.x;
    int* to = p.lists;
    for (int e = tid; e <= p.E; e += kBlock) to[e] = l.first[e];
    for (int a = tid; a < *l.total; a += kBlock) to[p.E + 1 + a] = l.active[a];
    for (int i = tid; i < l.first[p.E]; i += kBlock) to[2 * p.E + 1 + i] = l.pairs[i];
    if (tid == 0) to[2 * p.E + 1 + p.P] = *l.total;
}

// The kept lists in LDS: first, active, pairs and total, in this order.
template <int BLOCK>
__device__ inline Lists take_rows(const ExpertParams& p, int* lds) {
    for (int i = threadIdx.x; i < kept_words(p.E, p.P); i += BLOCK) lds[i] = p.lists[i];
    Lists l = {};
    l.first = lds;
    l.active = lds + p.E + 1;
    l.pairs = l.active + p.E;
    l.total = l.pairs + p.P;
    return l;
}

// ---- operands ------------------------------------------------------------------------
// A step's 128 elements of K lie on four quarters of the lanes; quarter q has, in its
// i-th of four products, the elements at(i, q) .. + 7.  Any order will do that both
// operands share: 4-bit weights take a whole block to a lane (16 bytes), bf16 ones
// go through memory by whole lines.
// kFull: all steps of a load end below `end`, which no row is shorter than.  kEnd:
// places past the row read its last whole 8 elements (or its last block) instead, to
// be shifted into place or dropped once they are there.  kShort: rows of fewer than
// 8 elements, one by one.  But for those no load has a branch around it, or a use of
// what it loads: either made each wait for the one before (70 us against 36 for 56
// experts of 16 rows).
enum Reach { kFull, kEnd, kShort };

// What a lane keeps of 8 elements from k on that were read from min(k, K - 8) on:
// `skip` of them are before k, and all are dropped from `end` on.
struct Place {
    int start, skip;
};
__device__ inline Place place(int k, int end, int K) {
    const int last = K - 8;
    Place p;
    p.start = k < last ? k : last;
    p.skip = k < end ? k - p.start : 8;
    return p;
}
// Elements skip .. skip+7 of 8 words, zeros after the last.
__device__ inline void shift_words(uint32_t (&w)[8], int skip) {
#pragma unroll
    for (int by = 4; by; by >>= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = skip & by ? (i + by < 8 ? w[i + by] : 0u) : w[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = skip >= 8 ? 0u : w[i];
}
// The same of 8 halves in 4 words.
__device__ inline void shift_halves(uint32_t (&w)[4], int skip) {
#pragma unroll
    for (int by = 2; by; by >>= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = skip & (2 * by) ? (i + by < 4 ? w[i + by] : 0u) : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t next = i < 3 ? w[i + 1] : 0u;
        w[i] = skip & 1 ? (w[i] >> 16) | (next << 16) : w[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = skip >= 8 ? 0u : w[i];
}

// Eight bf16 elements from k on; of rows shorter than 8 one by one.
template <Reach R>
__device__ inline void load_bf16(uint32_t (&w)[4], const uint16_t* p, int k, int end, int K) {
    if constexpr (R != kShort) {
        __builtin_memcpy(w, p + (R == kFull ? k : place(k, end, K).start), 16);
    } else {
        uint16_t u[8] = {};
        for (int i = 0; i < 8; ++i)
            if (k + i < end) u[i] = p[k + i];
        __builtin_memcpy(w, u, 16);
    }
}
template <Reach R>
__device__ inline bf16x8 take_bf16(const uint32_t (&w)[4], int k, int end, int K) {
    uint32_t t[4] = {w[0], w[1], w[2], w[3]};
    if (R == kEnd) shift_halves(t, place(k, end, K).skip);
    return __builtin_bit_cast(bf16x8, t);
}

struct WeightsMx4 {
    template <int U>
    struct Raw {
        uint32_t c[U][4];
        uint32_t s[U];  // the scales of each step's blocks
    };
    struct Row {
        const uint8_t* codes;
        const uint8_t* scales;
    };
    __device__ static int at(int i, int q) { return 32 * q + 8 * i; }
    __device__ static Row row(const void* w, const uint8_t* scales, int64_t r, int K) {
        const int64_t KB = (K + 31) / 32;
        return Row{static_cast<const uint8_t*>(w) + r * KB * 16, scales + r * KB};
    }
    // (the scales of U whole steps are one load: as many requests as rows)
    template <int U, Reach R>
    __device__ static void load(Raw<U>& r, const Row& w, int s, int q, int end, int K) {
        const int last = (K + 31) / 32 - 1;
        if (R == kFull) __builtin_memcpy(r.s, w.scales + 4 * s, 4 * U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            int b = 4 * (s + u) + q;
            if (R != kFull) {
                b = b < last ? b : last;
                r.s[u] = w.scales[b];
            }
            __builtin_memcpy(r.c[u], w.codes + b * 16, 16);
        }
    }
    // (blocks from `end` on are dropped)
    template <int U, Reach R>
    __device__ static uint32_t scale(const Raw<U>& r, int u, int s, int q, int end) {
        return R == kFull ? (r.s[u] >> (8 * q)) & 255 : (kStep * (s + u) + 32 * q < end ? r.s[u] : 0u);
    }
    template <int U, Reach R>
    __device__ static void codes(const Raw<U>& r, int u, int s, int q, int end, uint32_t (&c)[4]) {
        const bool on = R == kFull || kStep * (s + u) + 32 * q < end;
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = on ? r.c[u][i] : 0u;
    }
    template <int U, Reach R>
    __device__ static void unpack(const Raw<U>& r, int u, int s, int q, int end, int,
                                  bf16x8 (&v)[4]) {
        const float f = scale_value(scale<U, R>(r, u, s, q, end));
        uint32_t c[4];
        codes<U, R>(r, u, s, q, end, c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bf16x2 t[4];
            t[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], f, 0);
            t[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], f, 1);
            t[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], f, 2);
            t[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], f, 3);
            __builtin_memcpy(&v[i], t, 16);
        }
    }
};

struct WeightsBf16 {
    template <int U>
    struct Raw {
        uint32_t v[U][4][4];
    };
    typedef const uint16_t* Row;
    __device__ static int at(int i, int q) { return 32 * i + 8 * q; }
    __device__ static Row row(const void* w, const uint8_t*, int64_t r, int K) {
        return static_cast<const uint16_t*>(w) + r * K;
    }
    template <int U, Reach R>
    __device__ static void load(Raw<U>& r, const Row& w, int s, int q, int end, int K) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                load_bf16<R>(r.v[u][i], w, kStep * (s + u) + at(i, q), end, K);
    }
    template <int U, Reach R>
    __device__ static void unpack(const Raw<U>& r, int u, int s, int q, int end, int K,
                                  bf16x8 (&v)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = take_bf16<R>(r.v[u][i], kStep * (s + u) + at(i, q), end, K);
    }
};

// An fp32 value as a sum of three bf16 terms: its upper 16 bits, and so on of what is
// left.  They are exact, but for bits below 2^-133, the least that bf16 holds.  An
// infinity or NaN is its first term.
constexpr int kTermsF32 = 3;
__device__ inline void split(float x, uint16_t (&t)[kTermsF32]) {
    const uint32_t u = __float_as_uint(x);
    float r = x - __uint_as_float(u & 0xFFFF0000u);
    const bool finite = (u & 0x7F800000u) != 0x7F800000u;
    // (the bits of a NaN may all lie in the lower half)
    t[0] = (uint16_t)((u >> 16) | (!finite && (u & 0xFFFF) ? 0x40u : 0u));
    r = finite ? r : 0.f;
    const uint32_t m = __float_as_uint(r);
    t[1] = (uint16_t)(m >> 16);
    t[2] = (uint16_t)pack_bf16(r - __uint_as_float(m & 0xFFFF0000u), 0.f);
}

// Rows: kTerms bf16 terms of every element.
struct RowsF32 {
    static constexpr int kTerms = kTermsF32;
    template <int U>
    struct Raw {
        uint32_t v[U][4][8];
    };
    typedef const float* Row;
    __device__ static Row row(const ExpertParams& p, int r) {
        return static_cast<const float*>(p.x) + r * p.ldx;
    }
    template <typename W, int U, Reach R>
    __device__ static void load(Raw<U>& r, const ExpertParams&, Row x, int s, int q, int end,
                                int K) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = kStep * (s + u) + W::at(i, q);
                if constexpr (R != kShort) {
                    __builtin_memcpy(r.v[u][i], x + (R == kFull ? k : place(k, end, K).start), 32);
                } else {
                    for (int j = 0; j < 8; ++j)
                        r.v[u][i][j] = k + j < end ? __float_as_uint(x[k + j]) : 0u;
                }
            }
    }
    template <typename W, int U, Reach R>
    __device__ static void unpack(const Raw<U>& r, int u, int i, int s, int q, int end, int K,
                                  bf16x8 (&v)[kTerms]) {
        uint32_t f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = r.v[u][i][j];
        if (R == kEnd)
            shift_words(f, place(kStep * (s + u) + W::at(i, q), end, K).skip);
        uint16_t t[kTerms][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint16_t w[kTerms];
            split(__uint_as_float(f[j]), w);
#pragma unroll
            for (int m = 0; m < kTerms; ++m) t[m][j] = w[m];
        }
#pragma unroll
        for (int m = 0; m < kTerms; ++m) __builtin_memcpy(&v[m], t[m], 16);
    }
};

struct RowsBf16 {
    static constexpr int kTerms = 1;
    template <int U>
    struct Raw {
        uint32_t v[U][4][4];
    };
    typedef const uint16_t* Row;
    __device__ static Row row(const ExpertParams& p, int r) {
        return static_cast<const uint16_t*>(p.x) + r * p.ldx;
    }
    template <typename W, int U, Reach R>
    __device__ static void load(Raw<U>& r, const ExpertParams&, Row x, int s, int q, int end,
                                int K) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                load_bf16<R>(r.v[u][i], x, kStep * (s + u) + W::at(i, q), end, K);
    }
    template <typename W, int U, Reach R>
    __device__ static void unpack(const Raw<U>& r, int u, int i, int s, int q, int end, int K,
                                  bf16x8 (&v)[1]) {
        v[0] = take_bf16<R>(r.v[u][i], kStep * (s + u) + W::at(i, q), end, K);
    }
};

struct RowsMx8 {
    static constexpr int kTerms = 1;
    template <int U>
    struct Raw {
        uint32_t c[U][4][2];
        uint32_t s[U];  // the scales of each step's blocks
    };
    struct Row {
        const uint8_t* codes;
        const uint8_t* scales;
    };
    __device__ static Row row(const ExpertParams& p, int r) {
        const int64_t KB = (p.K + 31) / 32;
        return Row{static_cast<const uint8_t*>(p.x) + r * KB * 32, p.x_scales + r * KB};
    }
    template <typename W, int U, Reach R>
    __device__ static void load(Raw<U>& r, const ExpertParams&, const Row& x, int s, int q, int end,
                                int K) {
        const int last = (K + 31) / 32 - 1;
        // (places of an element in blocks that are not there: of the last one)
        const auto in_row = [&](int k) { return R == kFull || k / 32 <= last ? k : 32 * last + k % 32; };
        if (R == kFull) __builtin_memcpy(r.s, x.scales + 4 * s, 4 * U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k0 = kStep * (s + u);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                __builtin_memcpy(r.c[u][i], x.codes + in_row(k0 + W::at(i, q)), 8);
            if (R != kFull) {
                uint32_t b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] = x.scales[in_row(k0 + 32 * i) / 32];
                r.s[u] = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
            }
        }
    }
    template <typename W, int U, Reach R>
    __device__ static void unpack(const Raw<U>& r, int u, int i, int s, int q, int end, int,
                                  bf16x8 (&v)[1]) {
        const int k = W::at(i, q);
        const bool on = R == kFull || kStep * (s + u) + k < end;
        const float f = scale_value(on ? (r.s[u] >> (k / 32 * 8)) & 255 : 0u);
        const uint32_t c0 = on ? r.c[u][i][0] : 0u, c1 = on ? r.c[u][i][1] : 0u;
        bf16x2 t[4];
        t[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, f, false);
        t[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, f, true);
        t[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, f, false);
        t[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, f, true);
        __builtin_memcpy(&v[0], t, 16);
    }
};

// Rows of h: a plane for each term, filled up with zeros to whole steps.
struct RowsOfH {
    static constexpr int kTerms = kTermsF32;
    template <int U>
    struct Raw {
        uint32_t v[U][kTermsF32][4][4];
    };
    typedef const uint16_t* Row;
    template <typename W, int U, Reach R>
    __device__ static void load(Raw<U>& r, const ExpertParams& p, Row x, int s, int q, int, int) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (steps that are not there: the last one, dropped)
            const int at = R == kFull || kStep * (s + u) < p.Hp ? s + u : p.Hp / kStep - 1;
#pragma unroll
            for (int m = 0; m < kTerms; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    __builtin_memcpy(r.v[u][m][i],
                                     x + (int64_t)m * p.P * p.Hp + kStep * at + W::at(i, q), 16);
        }
    }
    template <typename W, int U, Reach R>
    __device__ static void unpack(const Raw<U>& r, int u, int i, int s, int q, int end, int,
                                  bf16x8 (&v)[kTerms]) {
        const bool on = R == kFull || kStep * (s + u) + W::at(i, q) < end;
#pragma unroll
        for (int m = 0; m < kTerms; ++m) {
            uint32_t t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] = on ? r.v[u][m][i][j] : 0u;
            v[m] = __builtin_bit_cast(bf16x8, t);
        }
    }
};

// Steps whose loads are under way together: as many as about 120 registers hold (of 104
// h with 4-bit weights would have one: 8 of 64 experts for 16 8-bit rows 56.8 us for 52.5).
template <typename W, typename X, int M>
constexpr int steps_at_once() {
    constexpr int bytes = (int)(2 * sizeof(typename W::template Raw<1>) +
                                M * sizeof(typename X::template Raw<1>));
    return 4 * bytes <= 480 ? 4 : (2 * bytes <= 480 ? 2 : 1);
}

// acc[t][m] += weight rows w[t] (this lane's of each 16) times rows x[m] (this lane's
// of each 16): U steps from s on, without elements from `end` on.
template <typename W, typename X, int M, int U, Reach R>
__device__ inline void multiply_steps(const ExpertParams& p, const typename W::Row (&w)[2],
                                      const typename X::Row (&x)[M], int K, int s, int end,
                                      f32x4 (&acc)[2][M]) {
    const int q = (threadIdx.x & 63) >> 4;
    typename W::template Raw<U> rw[2];
    typename X::template Raw<U> rx[M];
#pragma unroll
    for (int t = 0; t < 2; ++t) W::template load<U, R>(rw[t], w[t], s, q, end, K);
#pragma unroll
    for (int m = 0; m < M; ++m) X::template load<W, U, R>(rx[m], p, x[m], s, q, end, K);
    __builtin_amdgcn_sched_barrier(0);  // (the compiler would spread them to save registers)
#pragma unroll
    for (int u = 0; u < U; ++u) {
        bf16x8 a[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t) W::template unpack<U, R>(rw[t], u, s, q, end, K, a[t]);
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bf16x8 b[X::kTerms];
                X::template unpack<W, U, R>(rx[m], u, i, s, q, end, K, b);
#pragma unroll
                for (int c = X::kTerms - 1; c >= 0; --c)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        acc[t][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t][i], b[c], acc[t][m],
                                                                            0, 0, 0);
            }
    }
}

// Steps s .. s1-1 of K elements.
template <typename W, typename X, int M>
__device__ inline void multiply(const ExpertParams& p, const typename W::Row (&w)[2],
                                const typename X::Row (&x)[M], int K, int s, int s1,
                                f32x4 (&acc)[2][M]) {
    constexpr int U = steps_at_once<W, X, M>();
    const int end = s1 * kStep < K ? s1 * kStep : K;
    for (; (s + U) * kStep <= end; s += U) multiply_steps<W, X, M, U, kFull>(p, w, x, K, s, end, acc);
    if constexpr (U > 2) {
        if ((s + 2) * kStep <= end) {
            multiply_steps<W, X, M, 2, kFull>(p, w, x, K, s, end, acc);
            s += 2;
        }
    }
    if constexpr (U > 1) {
        if ((s + 1) * kStep <= end) {
            multiply_steps<W, X, M, 1, kFull>(p, w, x, K, s, end, acc);
            ++s;
        }
    }
    if (s * kStep >= end) return;
    if (K >= 8) multiply_steps<W, X, M, 1, kEnd>(p, w, x, K, s, end, acc);
    else multiply_steps<W, X, M, 1, kShort>(p, w, x, K, s, end, acc);
}

// ---- up ---------------------------------------------------------------------------------
__device__ inline float activate(float z, int act) {
    if (act == MP_ACT_RELU) return z < 0.f ? 0.f : z;  // (NaN stays)
    if (act == MP_ACT_SILU) return z / (1.f + expf(-z));
    if (act == MP_ACT_GELU) return 0.5f * z * erfcf(z * -0.707106781f);
    return z;
}

// The pairs n0 .. n0 + 16 M - 1 of expert e and the weight rows of a tile.
template <typename W, typename X, bool GATED, int M>
__device__ inline void up_rows(const ExpertParams& p, const Lists& l, int e, int tile, int n0,
                               float* sums) {
    constexpr int COLS = GATED ? 16 : 32;  // columns of h
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int begin = l.first[e], n = l.first[e + 1] - begin;
    const int64_t rows = (int64_t)(1 + GATED) * p.H;
    typename W::Row w[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        int c = tile * COLS + (GATED ? 0 : 16 * t) + (lane & 15);
        c = c < p.H ? c : p.H - 1;  // (columns past the last are not stored)
        w[t] = W::row(p.w1, p.w1_scales, e * rows + (GATED ? t * (int64_t)p.H : 0) + c, p.K);
    }
    typename X::Row x[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {  // (lanes without a pair take the first one again)
        const int at = n0 + 16 * m + (lane & 15);
        x[m] = X::row(p, l.pairs[begin + (at < n ? at : n0)] / p.k);
    }
    f32x4 acc[2][M] = {};
    const int steps = (p.K + kStep - 1) / kStep;
    multiply<W, X, M>(p, w, x, p.K, steps * wave / kWaves, steps * (wave + 1) / kWaves, acc);

    // the wavefronts' sums: [wave][t][m][i][lane]
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sums[((((wave * 2 + t) * M + m) * 4 + i) << 6) + lane] = acc[t][m][i];
    __syncthreads();
    const int i = threadIdx.x >> 6;
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const int at = n0 + 16 * m + (lane & 15);
        if (at >= n || i >= 4) continue;
        const int pair = l.pairs[begin + at];
        float z[2] = {0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 2; ++t)
            for (int v = 0; v < kWaves; ++v)
                z[t] += sums[((((v * 2 + t) * M + m) * 4 + i) << 6) + lane];
        const float weight = l.weight[pair];
        const int c = 4 * (lane >> 4) + i;
#pragma unroll
        for (int t = 0; t < (GATED ? 1 : 2); ++t) {
            float h = activate(z[t], p.act);
            if (GATED) h *= z[1];
            h *= weight;
            const int col = tile * COLS + 16 * t + c;
            if (col >= p.H) continue;
            uint16_t term[kTermsF32];
            split(h, term);
#pragma unroll
            for (int v = 0; v < kTermsF32; ++v)
                p.h[((int64_t)v * p.P + pair) * p.Hp + col] = term[v];
        }
    }
}

// M: products of 16 rows side by side (1 where there are no more rows).  Workgroups
// go through the (expert, tile) items by the grid, so that finding the rows is paid
// once by each.
template <typename W, typename X, bool GATED, int M>
__global__ __launch_bounds__(kBlock) void expert_up(ExpertParams p, int tiles) {
    extern __shared__ int lds[];
    const Lists l = carve(lds, p.E, p.P);
    float* sums = reinterpret_cast<float*>(lds + (list_words(p.E, p.P) + 3) / 4 * 4);
    find_rows(p, l);
    if (blockIdx.x == 0) {  // (for the second launch)
        keep_rows(p, l);
        for (int c = threadIdx.x; c < (p.Fo + kCols - 1) / kCols; c += kBlock) p.arrived[c] = 0;
    }
    const int items = *l.total * tiles;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int slot = item / tiles, tile = item - slot * tiles;
        const int e = l.active[slot], n = l.first[e + 1] - l.first[e];
        // (the weights of more than 16 M rows are read again, from the caches)
        int n0 = 0;
        for (; n0 + 16 * (M - 1) < n; n0 += 16 * M) up_rows<W, X, GATED, M>(p, l, e, tile, n0, sums);
        if (M > 1 && n0 < n) up_rows<W, X, GATED, 1>(p, l, e, tile, n0, sums);
        if (tile == tiles - 1) {  // zeros fill the last step of the rows of h
            const int more = p.Hp - p.H;
            for (int i = threadIdx.x; i < n * more; i += kBlock)
                for (int v = 0; v < kTermsF32; ++v)
                    p.h[((int64_t)v * p.P + l.pairs[l.first[e] + i / more]) * p.Hp + p.H +
                        i % more] = 0;
        }
    }
}

// ---- down -----------------------------------------------------------------------------
// The sums of this wavefront for the pairs n0 .. of expert e, steps s0 .. s1-1.
template <typename W, typename X, int M>
__device__ inline void down_rows(const ExpertParams& p, const Lists& l, int e, int n0, int c0, int s0,
                                 int s1, float* mine) {
    const int lane = threadIdx.x & 63;
    const int begin = l.first[e], n = l.first[e + 1] - begin;
    typename W::Row w[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        int c = c0 + 16 * t + (lane & 15);
        c = c < p.Fo ? c : p.Fo - 1;
        w[t] = W::row(p.w2, p.w2_scales, (int64_t)e * p.Fo + c, p.H);
    }
    typename X::Row x[M];
    bool has[M];
    int row[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const int at = n0 + 16 * m + (lane & 15);
        has[m] = at < n;  // (others take the first one again)
        const int pair = l.pairs[begin + (has[m] ? at : n0)];
        x[m] = p.h + (int64_t)pair * p.Hp;
        row[m] = pair / p.k;
    }
    f32x4 acc[2][M] = {};
    multiply<W, X, M>(p, w, x, p.H, s0, s1, acc);
#pragma unroll
    for (int m = 0; m < M; ++m) {
        if (!has[m]) continue;
#pragma unroll
        for (int t = 0; t < 2; ++t) {  // (rows of an expert's pairs differ)
            f32x4* to = reinterpret_cast<f32x4*>(&mine[row[m] * kLine + 16 * t + 4 * (lane >> 4)]);
            *to += acc[t][m];
        }
    }
}

template <typename W, typename X, int M, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void expert_down(ExpertParams p) {
    constexpr int BLOCK = WAVES * 64;
    extern __shared__ int lds[];
    __shared__ int s_last;
    const Lists l = take_rows<BLOCK>(p, lds);
    float* sums = reinterpret_cast<float*>(lds + (kept_words(p.E, p.P) + 3) / 4 * 4);
    const int tid = threadIdx.x, wave = tid >> 6;
    const int tile = blockIdx.x / p.splits, share = blockIdx.x - tile * p.splits, c0 = tile * kCols;
    float* mine = sums + wave * p.N * kLine;
    for (int i = tid; i < WAVES * p.N * kLine; i += BLOCK) sums[i] = 0.f;
    __syncthreads();
    // items: an expert and as many steps as are loaded at once
    constexpr int U = steps_at_once<W, X, M>();
    const int steps = p.Hp / kStep, per = (steps + U - 1) / U;
    const int items = *l.total * per, runs = p.splits * WAVES, run = share * WAVES + wave;
    const int hi = (int)((int64_t)items * (run + 1) / runs);
    for (int at = (int)((int64_t)items * run / runs); at < hi;) {
        const int slot = at / per, i0 = at - slot * per;
        const int i1 = hi - at < per - i0 ? i0 + (hi - at) : per;
        const int s0 = i0 * U, s1 = i1 * U < steps ? i1 * U : steps;
        const int e = l.active[slot];
        const int n = l.first[e + 1] - l.first[e];
        int n0 = 0;
        for (; n0 + 16 * (M - 1) < n; n0 += 16 * M) down_rows<W, X, M>(p, l, e, n0, c0, s0, s1, mine);
        if (M > 1 && n0 < n) down_rows<W, X, 1>(p, l, e, n0, c0, s0, s1, mine);
        at += i1 - i0;
    }
    __syncthreads();
    const int64_t size = (int64_t)p.N * kCols;
    float* part = p.part + (int64_t)tile * p.splits * size;
    for (int i = tid; i < p.N * kCols; i += BLOCK) {
        const int r = i / kCols, c = i % kCols;
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) s += sums[(v * p.N + r) * kLine + c];
        if (p.splits > 1)
            __hip_atomic_store(&part[share * size + i], s, __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
        else sums[r * kLine + c] = s;  // (this thread's own)
    }
    if (p.splits > 1) {
        // The last of a tile's workgroups adds the shares, in order.  They are stored and
        // loaded by agent-scope atomics, that is in memory that all XCDs see alike, and
        // every thread waits for its stores before the workgroup is counted: so no
        // fence has to write back and drop the L2 (with __threadfence on both sides
        // this launch took 45 us for one row, now 9).
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0)
            s_last = __hip_atomic_fetch_add(&p.arrived[tile], 1, __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT) == p.splits - 1;
        __syncthreads();
        if (!s_last) return;
    }
    // (all shares of several elements are under way together; one after the other, both
    // launches took 21.9 us for 20.0 for 7 odd rows, eight shares, 172 for 166 for 64 rows
    // of 4 of 64 experts)
    constexpr int ITEMS = M == 1 ? 1 : 4, SHARES = M == 1 ? 8 : 4;
    for (int i0 = tid; i0 < p.N * kCols; i0 += ITEMS * BLOCK) {
        float s[ITEMS] = {};
        if (p.splits > 1) {
            for (int v0 = 0; v0 < p.splits; v0 += SHARES) {
                float t[ITEMS][SHARES];
#pragma unroll
                for (int b = 0; b < ITEMS; ++b) {
                    const int i = i0 + b * BLOCK;
#pragma unroll
                    for (int u = 0; u < SHARES; ++u)  // (what is not there: the last again)
                        t[b][u] = __hip_atomic_load(
                            &part[(v0 + u < p.splits ? v0 + u : p.splits - 1) * size +
                                  (i < p.N * kCols ? i : i0)],
                            __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
#pragma unroll
                for (int b = 0; b < ITEMS; ++b)
#pragma unroll
                    for (int u = 0; u < SHARES; ++u) s[b] += v0 + u < p.splits ? t[b][u] : 0.f;
            }
        }
#pragma unroll
        for (int b = 0; b < ITEMS; ++b) {
            const int i = i0 + b * BLOCK, r = i / kCols, c = i % kCols;
            if (i >= p.N * kCols || c0 + c >= p.Fo) continue;
            float o = p.splits > 1 ? s[b] : sums[r * kLine + c];
            if (p.out_bf16) {
                if (p.residual)
                    o += load_one<BF16>(static_cast<const uint16_t*>(p.residual) + r * p.ldr + c0 + c);
                store_one<BF16>(static_cast<uint16_t*>(p.out) + (int64_t)r * p.Fo + c0 + c, o);
            } else {
                if (p.residual) o += static_cast<const float*>(p.residual)[r * p.ldr + c0 + c];
                static_cast<float*>(p.out)[(int64_t)r * p.Fo + c0 + c] = o;
            }
        }
    }
}

size_t in_16(int words) { return (size_t)(words + 3) / 4 * 16; }

template <typename W, typename X, int M>
void launch_up(const ExpertParams& p, hipStream_t s) {
    const int tiles = (int)ceil_div(p.H, p.gated ? 16 : 32);
    const int64_t items = (int64_t)(p.E < p.P ? p.E : p.P) * tiles;
    const dim3 g((unsigned)(items < kUpGrid ? items : kUpGrid));
    const size_t lds = in_16(list_words(p.E, p.P)) + (size_t)kWaves * 2 * M * 4 * 64 * 4;
    if (p.gated) hipLaunchKernelGGL((expert_up<W, X, true, M>), g, dim3(kBlock), lds, s, p, tiles);
    else hipLaunchKernelGGL((expert_up<W, X, false, M>), g, dim3(kBlock), lds, s, p, tiles);
}

template <typename W, int M>
hipError_t launch(const ExpertParams& p, int rows, hipStream_t s) {
    if (rows == kRowsMx8) launch_up<W, RowsMx8, M>(p, s);
    else if (rows == kRowsBf16) launch_up<W, RowsBf16, M>(p, s);
    else launch_up<W, RowsF32, M>(p, s);
    const dim3 g((unsigned)(ceil_div(p.Fo, kCols) * p.splits));
    constexpr int D = M == 1 ? 8 : 4;  // wavefronts of a workgroup: their sums fit into LDS
    const size_t lds = in_16(kept_words(p.E, p.P)) + (size_t)D * p.N * kLine * 4;
    hipLaunchKernelGGL((expert_down<W, RowsOfH, M, D>), g, dim3(D * 64), lds, s, p);
    return hipGetLastError();
}

}  // namespace

// Workgroups that share the second product's work for a tile of columns.
int expert_splits(int64_t Fo) {
    const int64_t tiles = ceil_div(Fo, kCols);
    int64_t n = ceil_div(256, tiles);
    return (int)(n > 16 ? 16 : n);
}

hipError_t launch_experts(const ExpertParams& p, int rows, int mx4, hipStream_t s) {
    if (mx4) return p.N > 16 ? launch<WeightsMx4, 2>(p, rows, s) : launch<WeightsMx4, 1>(p, rows, s);
    return p.N > 16 ? launch<WeightsBf16, 2>(p, rows, s) : launch<WeightsBf16, 1>(p, rows, s);
}

size_t expert_list_bytes(int64_t E, int64_t P) { return (size_t)kept_words((int)E, (int)P) * 4; }
size_t expert_h_bytes(int64_t P, int64_t Hp) { return (size_t)kTermsF32 * (size_t)P * (size_t)Hp * 2; }

}  // namespace mp
