// Internal declarations shared by the operators of include/mp_layers.h.
#pragma once

#include "mp_internal.hpp"
#include "mp_layers.h"

namespace mp {

// ---- element types -----------------------------------------------------------
// V consecutive elements at the alignment of one (gfx950 takes unaligned
// global accesses) as floats.  bf16 is the upper half of a float; rounding back
// is the hardware's, to nearest even.
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct F32 {
    typedef float raw;
};
struct BF16 {
    typedef uint16_t raw;
};

__device__ inline uint32_t pack_bf16(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

template <int BYTES>
struct Raw {
    uint32_t w[BYTES / 4];
};
template <>
struct Raw<2> {
    uint16_t w[1];
};

// The raw bits of V elements of type T.
template <typename T, int V>
using RawOf = Raw<(int)sizeof(typename T::raw) * V>;

template <typename T, int V>
__device__ inline RawOf<T, V> load_raw(const typename T::raw* p) {
    RawOf<T, V> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}

template <typename T, int V>
__device__ inline void to_floats(const RawOf<T, V>& r, float (&v)[V]) {
    if constexpr (sizeof(typename T::raw) == 4) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = __uint_as_float(r.w[i]);
    } else if constexpr (V == 1) {
        v[0] = __uint_as_float((uint32_t)r.w[0] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            v[2 * i] = __uint_as_float(r.w[i] << 16);
            v[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
        }
    }
}

template <typename T, int V>
__device__ inline RawOf<T, V> from_floats(const float (&v)[V]) {
    RawOf<T, V> r;
    if constexpr (sizeof(typename T::raw) == 4) {
#pragma unroll
        for (int i = 0; i < V; ++i) r.w[i] = __float_as_uint(v[i]);
    } else if constexpr (V == 1) {
        r.w[0] = (uint16_t)pack_bf16(v[0], 0.f);
    } else {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) r.w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    }
    return r;
}

template <typename T, int V>
__device__ inline void load_floats(const typename T::raw* p, float (&v)[V]) {
    to_floats<T, V>(load_raw<T, V>(p), v);
}

template <typename T, int V>
__device__ inline void store_floats(typename T::raw* p, const float (&v)[V]) {
    const RawOf<T, V> r = from_floats<T, V>(v);
    __builtin_memcpy(p, &r, sizeof(r));
}

template <typename T>
__device__ inline float load_one(const typename T::raw* p) {
    if constexpr (sizeof(typename T::raw) == 4) return *p;
    else return __uint_as_float((uint32_t)*p << 16);
}

template <typename T>
__device__ inline void store_one(typename T::raw* p, float v) {
    if constexpr (sizeof(typename T::raw) == 4) *p = v;
    else *p = (uint16_t)pack_bf16(v, 0.f);
}

// ---- dropout (dropout.hip) -----------------------------------------------------
struct DropoutParams {
    const void* x;
    const void* residual;  // nullptr: none
    const int32_t* ids;    // nullptr: the row's number
    const int64_t* step;   // nullptr: 0
    void* out;
    int64_t N, F, ldx, ldr, ldo;
    uint32_t limit;        // an element stays iff its 16-bit word is at least this
    float scale;
    uint64_t seed, offset;
};
hipError_t launch_dropout(const DropoutParams& p, int dtype, int whole_rows, hipStream_t s);

// ---- group norm (norm.hip) -------------------------------------------------------
// How a call of these sizes is cut up.
struct NormShape {
    int V;                  // channels of a thread's chunk
    // short segments (unit = 0: groups too wide, every segment is a long one)
    int unit, tile_groups, tiles, cpr, slots, lpg, short_blocks;
    int64_t lmax;           // rows of the longest short segment
    size_t lds;
    // long segments (long_tiles = 0: there can be none)
    int64_t tile_rows, apply_rows, long_tiles, col_tile, stat_line, places;
    int col_tiles, long_lpg;
    size_t long_lds;
};
NormShape norm_shape(int64_t N, int64_t S, int64_t F, int64_t G, int dtype, int backward);

struct NormParams {
    const void* ptr;
    int rp64;
    const void* x;
    const void* dout;    // backward
    int64_t N, S, F, ldx, G;
    int cg;              // channels of a group
    const float* gamma;  // nullptr: 1
    const float* beta;   // nullptr: 0
    float eps;
    int act;
    void* out;           // or dx (nullptr: not wanted)
    int out_bf16;
    float* mean;
    float* rstd;
    // workspace: partial statistics of the tiles, the segments' mean gradients,
    // lines of dgamma and dbeta (nullptr: not wanted)
    float* stats;
    float* ca;
    float* cb;
    float* part;
    int* flags;          // [short_blocks]: the short path's workgroups met a long segment
    // of the NormShape, filled by the launch
    int64_t lmax, tile_rows, apply_rows, stat_line, places;
    int tile_groups, cpr, slots, lpg, short_blocks;
};
hipError_t launch_norm(NormParams p, const NormShape& h, int dtype, bool backward, float* dgamma,
                       float* dbeta, hipStream_t s);

// ---- router (route.hip) ----------------------------------------------------------
struct RouteParams {
    const void* logits;
    const uint8_t* mask;  // nullptr: every row
    int64_t N, E, ldl, k;
    int renorm;
    int32_t* idx;         // forward: out; backward: in
    float* weight;
    int32_t* counts;      // [E + 1]
    float* loss;          // [2]
    float* part;          // [route_blocks][2 E + 2] partial sums
    const float* dweight; // nullptr: 0
    const float* dloss;   // nullptr: 0
    void* dlogits;
};
int route_blocks(int64_t N, int64_t E);
hipError_t launch_route(const RouteParams& p, int dtype, hipStream_t s);
hipError_t launch_route_backward(const RouteParams& p, int dtype, hipStream_t s);

// ---- microscaled 4-bit floating point (mx.hip) -------------------------------------
struct MxParams {
    const void* seg;
    int seg64;
    int64_t T, N;
    const void* x;
    int64_t ldx;
    int K, KB, Fo;
    const uint8_t* w_codes;   // [T, Fo, KB * 16]
    const uint8_t* w_scales;  // [T, Fo, KB]
    uint8_t* x_codes;         // workspace [N, KB * 16]
    uint8_t* x_scales;        // workspace [N, KB]
    uint32_t* x_words;        // workspace [KS, N]: the scales by steps of four blocks
    uint32_t* w_words;        // workspace [T, KS, Fo]
    void* out;
};
hipError_t launch_mx_quantize(const void* x, int dtype, int64_t N, int64_t K, int64_t ldx,
                              uint8_t* codes, uint8_t* scales, void* values, hipStream_t s);
hipError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t N, int64_t K,
                                void* out, int dtype, hipStream_t s);
// Whether a product of these sizes has no more tiles than a launch can hold.
bool mx_product_fits(int64_t T, int64_t N, int64_t K, int64_t Fo);
hipError_t launch_mx_product(const MxParams& p, int x_dtype, int out_dtype, hipStream_t s);

}  // namespace mp
