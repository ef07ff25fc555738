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
// bf16, and so are 8-bit rows; fp32 values are taken as sums of bf16 terms, three
// of which are exact (two, off by 2^-16, where the result is bf16).  8-bit rows
// times 4-bit weights are v_mfma_scale_f32_16x16x128_f8f6f4's, as they are.
#include "layers_internal.hpp"

namespace mp {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 256;
constexpr int kWaves = kBlock / kWave;
constexpr int kStep = 128;    // elements of K of a step, 32 for a quarter of the lanes
constexpr int kE4M3 = 0, kE2M1 = 4;  // operand formats of the scaled products
constexpr int kCols = 32;     // weight rows of a workgroup
constexpr int64_t kUpGrid = 1024;  // workgroups of the first launch, at most
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
// FULL: the step ends within K.  Only such loads are many at a time, without branches
// and without a use of what they load: a branch around a load, or a shift of a scale
// in it, made each wait for the one before (70 us against 30 for 56 experts of 16 rows).

// Eight bf16 elements k .. k+7 of a row of K, zero past its end.
template <bool FULL>
__device__ inline bf16x8 load_bf16(const uint16_t* p, int k, int K) {
    uint16_t u[8] = {};
    if (FULL || k + 8 <= K) {
        __builtin_memcpy(u, p + k, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < K) u[i] = p[k + i];
    }
    bf16x8 v;
    __builtin_memcpy(&v, u, 16);
    return v;
}

struct WeightsMx4 {
    static constexpr bool kMx4 = true;
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
    // (the scales of U steps are one load: as many requests as rows)
    template <int U, bool FULL>
    __device__ static void load(Raw<U>& r, const Row& w, int s, int q, int K) {
        const int KB = (K + 31) / 32, b = 4 * s + q;
        if (FULL) {
            __builtin_memcpy(r.s, w.scales + 4 * s, 4 * U);
#pragma unroll
            for (int u = 0; u < U; ++u) __builtin_memcpy(r.c[u], w.codes + (b + 4 * u) * 16, 16);
        } else {
            r = Raw<U>{};
            if (b < KB) {
                __builtin_memcpy(r.c[0], w.codes + b * 16, 16);
                r.s[0] = (uint32_t)w.scales[b] << (8 * q);
            }
        }
    }
    template <int U>
    __device__ static void unpack(const Raw<U>& r, int u, int q, bf16x8 (&v)[4]) {
        const float f = scale_value((r.s[u] >> (8 * q)) & 255);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bf16x2 t[4];
            t[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.c[u][i], f, 0);
            t[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.c[u][i], f, 1);
            t[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.c[u][i], f, 2);
            t[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.c[u][i], f, 3);
            __builtin_memcpy(&v[i], t, 16);
        }
    }
};

struct WeightsBf16 {
    static constexpr bool kMx4 = false;
    template <int U>
    struct Raw {
        bf16x8 v[U][4];
    };
    typedef const uint16_t* Row;
    __device__ static int at(int i, int q) { return 32 * i + 8 * q; }
    __device__ static Row row(const void* w, const uint8_t*, int64_t r, int K) {
        return static_cast<const uint16_t*>(w) + r * K;
    }
    template <int U, bool FULL>
    __device__ static void load(Raw<U>& r, const Row& w, int s, int q, int K) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r.v[u][i] = load_bf16<FULL>(w, kStep * (s + u) + at(i, q), K);
    }
    template <int U>
    __device__ static void unpack(const Raw<U>& r, int u, int, bf16x8 (&v)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = r.v[u][i];
    }
};

// An fp32 value as a sum of bf16 terms: its upper 16 bits, and so on of what is
// left; of two terms the second is rounded.  Three are exact.  An infinity or NaN
// is its first term.
template <int T>
__device__ inline void split(float x, uint16_t (&t)[T]) {
    const uint32_t u = __float_as_uint(x);
    float r = x - __uint_as_float(u & 0xFFFF0000u);
    const bool finite = (u & 0x7F800000u) != 0x7F800000u;
    // (the bits of a NaN may all lie in the lower half)
    t[0] = (uint16_t)((u >> 16) | (!finite && (u & 0xFFFF) ? 0x40u : 0u));
    r = finite ? r : 0.f;
    if constexpr (T == 3) {
        const uint32_t m = __float_as_uint(r);
        t[1] = (uint16_t)(m >> 16);
        r -= __uint_as_float(m & 0xFFFF0000u);
    }
    t[T - 1] = (uint16_t)pack_bf16(r, 0.f);
}

// Rows: kTerms bf16 terms of every element.
template <int TERMS>
struct RowsF32 {
    static constexpr int kTerms = TERMS;
    template <typename W>
    static constexpr bool kScaled = false;
    template <int U>
    struct Raw {
        float v[U][4][8];
    };
    typedef const float* Row;
    __device__ static Row row(const ExpertParams& p, int r) {
        return static_cast<const float*>(p.x) + r * p.ldx;
    }
    template <typename W, int U, bool FULL>
    __device__ static void load(Raw<U>& r, const ExpertParams&, Row x, int s, int q, int K) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = kStep * (s + u) + W::at(i, q);
                if (FULL) {
                    __builtin_memcpy(r.v[u][i], x + k, 32);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) r.v[u][i][j] = k + j < K ? x[k + j] : 0.f;
                }
            }
    }
    template <typename W, int U>
    __device__ static void unpack(const Raw<U>& r, int u, int i, int, bf16x8 (&v)[TERMS]) {
        uint16_t t[TERMS][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint16_t w[TERMS];
            split<TERMS>(r.v[u][i][j], w);
#pragma unroll
            for (int m = 0; m < TERMS; ++m) t[m][j] = w[m];
        }
#pragma unroll
        for (int m = 0; m < TERMS; ++m) __builtin_memcpy(&v[m], t[m], 16);
    }
};

struct RowsBf16 {
    static constexpr int kTerms = 1;
    template <typename W>
    static constexpr bool kScaled = false;
    template <int U>
    struct Raw {
        bf16x8 v[U][4];
    };
    typedef const uint16_t* Row;
    __device__ static Row row(const ExpertParams& p, int r) {
        return static_cast<const uint16_t*>(p.x) + r * p.ldx;
    }
    template <typename W, int U, bool FULL>
    __device__ static void load(Raw<U>& r, const ExpertParams&, Row x, int s, int q, int K) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r.v[u][i] = load_bf16<FULL>(x, kStep * (s + u) + W::at(i, q), K);
    }
    template <typename W, int U>
    __device__ static void unpack(const Raw<U>& r, int u, int i, int, bf16x8 (&v)[1]) {
        v[0] = r.v[u][i];
    }
};

struct RowsMx8 {
    static constexpr int kTerms = 1;
    // Whether products with these weights take codes and scales as they are.
    template <typename W>
    static constexpr bool kScaled = W::kMx4;
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
    template <typename W, int U, bool FULL>
    __device__ static void load(Raw<U>& r, const ExpertParams&, const Row& x, int s, int q, int K) {
        const int KB = (K + 31) / 32;
        if (FULL) __builtin_memcpy(r.s, x.scales + 4 * s, 4 * U);
        else r = Raw<U>{};
#pragma unroll
        for (int u = 0; u < U; ++u)
            if constexpr (kScaled<W>) {
                // 8-bit codes k = 16 q .. + 15 and 64 + 16 q .. + 15
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const int k = kStep * (s + u) + 32 * i + 16 * q;
                    if (FULL || k / 32 < KB) __builtin_memcpy(r.c[u][i], x.codes + k, 16);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = kStep * (s + u) + W::at(i, q);
                    if (FULL || k / 32 < KB) __builtin_memcpy(r.c[u][i], x.codes + k, 8);
                }
            }
        if (!FULL) {
            for (int i = 0; i < 4; ++i)
                if (4 * s + i < KB) r.s[0] |= (uint32_t)x.scales[4 * s + i] << (8 * i);
        }
    }
    template <typename W, int U>
    __device__ static void unpack(const Raw<U>& r, int u, int i, int q, bf16x8 (&v)[1]) {
        const float f = scale_value((r.s[u] >> (W::at(i, q) / 32 * 8)) & 255);
        bf16x2 t[4];
        t[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.c[u][i][0], f, false);
        t[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.c[u][i][0], f, true);
        t[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.c[u][i][1], f, false);
        t[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.c[u][i][1], f, true);
        __builtin_memcpy(&v[0], t, 16);
    }
};

// Rows of h: TERMS planes, filled up with zeros to whole steps.
template <int TERMS>
struct RowsOfH {
    static constexpr int kTerms = TERMS;
    template <typename W>
    static constexpr bool kScaled = false;
    template <int U>
    struct Raw {
        bf16x8 v[U][TERMS][4];
    };
    typedef const uint16_t* Row;
    template <typename W, int U, bool FULL>
    __device__ static void load(Raw<U>& r, const ExpertParams& p, Row x, int s, int q, int) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int m = 0; m < TERMS; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    __builtin_memcpy(&r.v[u][m][i],
                                     x + (int64_t)m * p.P * p.Hp + kStep * (s + u) + W::at(i, q),
                                     16);
    }
    template <typename W, int U>
    __device__ static void unpack(const Raw<U>& r, int u, int i, int, bf16x8 (&v)[TERMS]) {
#pragma unroll
        for (int m = 0; m < TERMS; ++m) v[m] = r.v[u][m][i];
    }
};

// Steps whose loads are under way together: as many as about 104 registers hold.
template <typename W, typename X, int M>
constexpr int steps_at_once() {
    constexpr int bytes = (int)(2 * sizeof(typename W::template Raw<1>) +
                                M * sizeof(typename X::template Raw<1>));
    return 4 * bytes <= 416 ? 4 : (2 * bytes <= 416 ? 2 : 1);
}

// acc[t][m] += weight rows w[t] (this lane's of each 16) times rows x[m] (this lane's
// of each 16): U steps from s on.
template <typename W, typename X, int M, int U, bool FULL>
__device__ inline void multiply_steps(const ExpertParams& p, const typename W::Row (&w)[2],
                                      const typename X::Row (&x)[M], int K, int s,
                                      f32x4 (&acc)[2][M]) {
    const int q = (threadIdx.x & 63) >> 4;
    typename W::template Raw<U> rw[2];
    typename X::template Raw<U> rx[M];
#pragma unroll
    for (int t = 0; t < 2; ++t) W::template load<U, FULL>(rw[t], w[t], s, q, K);
#pragma unroll
    for (int m = 0; m < M; ++m) X::template load<W, U, FULL>(rx[m], p, x[m], s, q, K);
    __builtin_amdgcn_sched_barrier(0);  // (the compiler would spread them to save registers)
    if constexpr (X::template kScaled<W>) {
        // lane quarter q has the scales of block q
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint32_t* c = rw[t].c[u];
                    i32x8 a = {(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0}, b;
                    __builtin_memcpy(&b, rx[m].c[u], 32);
                    acc[t][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        a, b, acc[t][m], kE2M1, kE4M3, 0, (int)(rw[t].s[u] >> (8 * q)), 0,
                        (int)(rx[m].s[u] >> (8 * q)));
                }
        return;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        bf16x8 a[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t) W::template unpack<U>(rw[t], u, q, a[t]);
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bf16x8 b[X::kTerms];
                X::template unpack<W, U>(rx[m], u, i, q, b);
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
    const int full = K / kStep < s1 ? K / kStep : s1;
    for (; s + U <= full; s += U) multiply_steps<W, X, M, U, true>(p, w, x, K, s, acc);
    if constexpr (U > 2) {
        if (s + 2 <= full) {
            multiply_steps<W, X, M, 2, true>(p, w, x, K, s, acc);
            s += 2;
        }
    }
    if (U > 1 && s < full) multiply_steps<W, X, M, 1, true>(p, w, x, K, s++, acc);
    if (s < s1) multiply_steps<W, X, M, 1, false>(p, w, x, K, s, acc);
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
        if (at >= n) continue;
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
            uint16_t term[3];
            if (p.planes == 3) {
                split<3>(h, term);
            } else {
                uint16_t two[2];
                split<2>(h, two);
                term[0] = two[0];
                term[1] = two[1];
                term[2] = 0;
            }
            for (int v = 0; v < p.planes; ++v)
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
                for (int v = 0; v < p.planes; ++v)
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
        // this launch took 45 us for one row, now 7).
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0)
            s_last = __hip_atomic_fetch_add(&p.arrived[tile], 1, __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT) == p.splits - 1;
        __syncthreads();
        if (!s_last) return;
    }
    for (int i = tid; i < p.N * kCols; i += BLOCK) {
        const int r = i / kCols, c = i % kCols;
        if (c0 + c >= p.Fo) continue;
        float s = 0.f;
        if (p.splits > 1) {
            for (int v = 0; v < p.splits; ++v)
                s += __hip_atomic_load(&part[v * size + i], __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
        } else {
            s = sums[r * kLine + c];
        }
        if (p.out_bf16) {
            if (p.residual)
                s += load_one<BF16>(static_cast<const uint16_t*>(p.residual) + r * p.ldr + c0 + c);
            store_one<BF16>(static_cast<uint16_t*>(p.out) + (int64_t)r * p.Fo + c0 + c, s);
        } else {
            if (p.residual) s += static_cast<const float*>(p.residual)[r * p.ldr + c0 + c];
            static_cast<float*>(p.out)[(int64_t)r * p.Fo + c0 + c] = s;
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
    else if (p.planes == 3) launch_up<W, RowsF32<3>, M>(p, s);
    else launch_up<W, RowsF32<2>, M>(p, s);
    const dim3 g((unsigned)(ceil_div(p.Fo, kCols) * p.splits));
    constexpr int D = M == 1 ? 8 : 4;  // wavefronts of a workgroup: their sums fit into LDS
    const size_t lds = in_16(kept_words(p.E, p.P)) + (size_t)D * p.N * kLine * 4;
    if (p.planes == 3)
        hipLaunchKernelGGL((expert_down<W, RowsOfH<3>, M, D>), g, dim3(D * 64), lds, s, p);
    else
        hipLaunchKernelGGL((expert_down<W, RowsOfH<2>, M, D>), g, dim3(D * 64), lds, s, p);
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

}  // namespace mp
