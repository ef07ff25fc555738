// Root-mean-square norm with the residual's addition, its result in the rows' type
// or in 8 bits with a scale for 32 values, and its gradients
// (include/mp_layers.h).
//
// A row lies in the registers of a team of L threads, CH chunks of V elements
// each, from its only load to its last store: lanes of a wavefront for rows of up
// to 64 chunks (64 / L rows a wavefront), a wavefront up to 256, else a
// workgroup.  Bound by memory: 512 MB of rows of 256 to 16,384 in 190 to 250 us, the
// gradients in 290 to 385 (4.2 to 5.7 TB/s).  Of longer rows, and in the fp32 gradient of
// 8,193 to 16,384, some registers go through scratch memory: forward of 32,768 fp32
// 268 us, of 65,536 339 (4.0 and 3.2 TB/s).
#include "layers_internal.hpp"

namespace mp {
namespace {

constexpr int kBlock = 256;
constexpr int64_t kMaxGrid = int64_t(1) << 21;  // (a launch has fewer than 2^32 threads)
constexpr int kWide = 1024;  // threads of a row too long for fewer

// Sum over a team of L threads, the same in all of them.
template <int L, int BLOCK>
__device__ inline float team_sum(float v, float* lds) {
    if constexpr (L <= 64) {
        return reduce_sum<L>(v);
    } else {
        v = reduce_sum<64>(v);
        __syncthreads();  // (the sums before have been read)
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < BLOCK / 64; ++w) s += lds[w];
        return s;
    }
}

// Chunk j of a row of F >= V elements begins at j V, but the last one of a row
// that is no multiple of V ends with the row: its first `skip` elements belong to
// the chunk before, and both write the same there.
template <int V>
__device__ inline int chunk_at(int j, int F, int& skip) {
    const int c = j * V, last = F - V;
    skip = c > last ? c - last : 0;
    return c > last ? last : c;
}

template <int V>
__device__ inline void store_as(void* out, int bf16, int64_t at, const float (&v)[V]) {
    if (bf16) store_floats<BF16, V>(static_cast<uint16_t*>(out) + at, v);
    else store_floats<F32, V>(static_cast<float*>(out) + at, v);
}

// Values k0 .. k0+V-1 of a row of F, zero past its end.
template <typename T, int V>
__device__ inline void load_to(const typename T::raw* p, int k0, int F, float (&v)[V]) {
    if (k0 + V <= F) {
        load_floats<T, V>(p + k0, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = k0 + i < F ? load_one<T>(p + k0 + i) : 0.f;
    }
}
template <int V>
__device__ inline void store_to(void* out, int bf16, int64_t row, int k0, int F,
                                const float (&v)[V]) {
    if (k0 + V <= F) {
        store_as<V>(out, bf16, row + k0, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (k0 + i >= F) continue;
            if (bf16) store_one<BF16>(static_cast<uint16_t*>(out) + row + k0 + i, v[i]);
            else store_one<F32>(static_cast<float*>(out) + row + k0 + i, v[i]);
        }
    }
}

// The value of an E4M3 code: magnitude bits e (4) and m (3) are m 2^-9 (e = 0) or
// (8 + m) 2^(e - 10); NaN where all seven are set.
__device__ inline float e4m3_value(uint32_t c) {
    const uint32_t e = (c >> 3) & 15, m = c & 7;
    float a = e ? __uint_as_float(((e + 120) << 23) | (m << 20)) : (float)m * 0x1p-9f;
    a = (c & 127) == 127 ? __builtin_nanf("") : a;
    return c & 128 ? -a : a;
}
// 2^(s - 127) (s = 0 is subnormal); NaN for 255.
__device__ inline float scale_value(uint32_t s) {
    return __uint_as_float(s == 255 ? 0x7FC00000u : (s ? s << 23 : 0x00400000u));
}

// Eight of the 32 values of four neighbouring lanes -> codes and the scale: the
// largest magnitude's exponent less 8, so that it lands in [256, 512); magnitudes
// above 448 saturate.
__device__ inline void quantize8(const float (&v)[8], uint32_t (&c)[2], uint32_t& s) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        m = m > a ? m : a;
    }
    m = reduce_max<4>(m);
    const uint32_t e = m >> 23;
    s = e == 255 ? 255u : (e > 8 ? e - 8 : 0);
    // (divided by 2^(s - 127); nothing of a block of NaN but its scale counts)
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        q[i] = __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(v[i], 127 - (int)s), -448.f, 448.f);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i], q[4 * i + 1], 0, false);
        c[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i + 2], q[4 * i + 3], w, true);
    }
}

// 1 / sqrt(mean of squares + eps) where the sum of squares has overflowed although
// the row is finite: again with values times 2^-76 (65536 squares of at most
// 2^(2 * 52) stay finite).
template <int V, int CH>
__device__ inline float squares_scaled(const float (&t)[CH][V], const int (&skip)[CH]) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float a = t[k][i] * 0x1p-76f;
            s = i >= skip[k] ? __builtin_fmaf(a, a, s) : s;
        }
    return s;
}

// Q8: chunks of 8 that end past the row are filled with zeros, so that blocks of
// 32 lie in four lanes.
template <typename T, int V, int L, int CH, int BLOCK, bool Q8>
__device__ inline void norm_row(const RmsParams& P, int64_t r, float* lds) {
    const int sub = threadIdx.x % L;
    const int F = (int)P.F;
    // (teams are whole in a wavefront or the workgroup: those past the last row take
    // part in the sums with zeros)
    const bool on = r < P.N;
    const typename T::raw* x = static_cast<const typename T::raw*>(P.x) + r * P.ldx;
    const typename T::raw* res = static_cast<const typename T::raw*>(P.residual) + r * P.ldr;

    float t[CH][V];
    int skip[CH];
    int at[CH];
    bool has[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int j = k * L + sub;
        has[k] = on && j * V < F;
        if (Q8) {
            at[k] = j * V;
            skip[k] = 0;
        } else {
            at[k] = chunk_at<V>(j, F, skip[k]);
        }
        if (has[k]) {
            if (Q8) load_to<T, V>(x, at[k], F, t[k]);
            else load_floats<T, V>(x + at[k], t[k]);
        } else {
            skip[k] = V;
#pragma unroll
            for (int i = 0; i < V; ++i) t[k][i] = 0.f;
        }
    }
    if (P.residual) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (!has[k]) continue;
            float v[V];
            if (Q8) load_to<T, V>(res, at[k], F, v);
            else load_floats<T, V>(res + at[k], v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += t[k][i];
            // the norm is that of the sum as it is stored, which the gradient reads
            to_floats<T, V>(from_floats<T, V>(v), t[k]);
        }
    }
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) s = i >= skip[k] ? __builtin_fmaf(t[k][i], t[k][i], s) : s;
    s = team_sum<L, BLOCK>(s, lds);
    const float n = (float)F;
    float rstd = 1.f / sqrtf(s / n + P.eps);
    if (s == __builtin_inff()) {  // (the same for the whole team)
        s = squares_scaled<V, CH>(t, skip);
        s = team_sum<L, BLOCK>(s, lds);
        rstd = 0x1p-76f / sqrtf(s / n + P.eps * 0x1p-76f * 0x1p-76f);
    }
    // (stores begin after the sum: every load of the row has returned, so that total
    // may be x or residual)
    if (on && sub == 0 && P.rstd) P.rstd[r] = rstd;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        if (!Q8 && !has[k]) continue;
        if (has[k] && P.total) store_to<V>(P.total, sizeof(typename T::raw) == 2, r * P.F, at[k], F, t[k]);
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = t[k][i] * rstd;
        if (P.weight && has[k]) {
            float w[V];
            if (Q8) load_to<F32, V>(P.weight, at[k], F, w);
            else load_floats<F32, V>(P.weight + at[k], w);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] *= w[i];
        }
        if constexpr (Q8) {
            if (at[k] + V > F) {  // (zeros past the row also where rstd is NaN)
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = at[k] + i < F ? v[i] : 0.f;
            }
            uint32_t c[2], sc;
            quantize8(v, c, sc);
            const int KB = (F + 31) / 32, b = at[k] / 32;
            if (on && b < KB) {  // (a last block's lanes past the row write its zeros)
                *reinterpret_cast<uint2*>(P.codes + r * KB * 32 + at[k]) = make_uint2(c[0], c[1]);
                if ((sub & 3) == 0) P.scales[r * KB + b] = (uint8_t)sc;
            }
            if (P.out && has[k]) {
                const float f = scale_value(sc);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = e4m3_value(c[i / 4] >> (8 * (i % 4))) * f;
                store_to<V>(P.out, P.out_bf16, r * P.F, at[k], F, v);
            }
        } else {
            store_as<V>(P.out, P.out_bf16, r * P.F + at[k], v);
        }
    }
}

template <typename T, int V, int L, int CH, int BLOCK, bool Q8>
__global__ __launch_bounds__(BLOCK) void rms_fwd(RmsParams P) {
    __shared__ float lds[BLOCK / 64];
    constexpr int TEAMS = BLOCK / L;
    const int64_t groups = (P.N + TEAMS - 1) / TEAMS;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x)
        norm_row<T, V, L, CH, BLOCK, Q8>(P, g * TEAMS + threadIdx.x / L, lds);
}

// dx = rstd (g - xhat mean(g xhat)) + dtotal with g = dout weight; a team's rows
// are blockIdx.x * TEAMS + its number, and so on by the grid, and its partial
// dweight stays in registers until the workgroup's teams are added up in order.
template <typename T, int V, int L, int CH, int BLOCK>
__global__ __launch_bounds__(BLOCK) void rms_bwd(RmsParams P) {
    __shared__ float lds[BLOCK / 64];
    __shared__ float s_dw[L <= 64 ? BLOCK * V : 1];
    constexpr int TEAMS = BLOCK / L;
    const int sub = threadIdx.x % L, team = threadIdx.x / L;
    const int F = (int)P.F;
    float w[CH][V], dw[CH][V];
    int skip[CH];
    int at[CH];
    bool col[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int j = k * L + sub;
        col[k] = j * V < F;
        at[k] = chunk_at<V>(j, F, skip[k]);
        if (!col[k]) skip[k] = V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[k][i] = 1.f;
            dw[k][i] = 0.f;
        }
        if (P.weight && col[k]) load_floats<F32, V>(P.weight + at[k], w[k]);
    }
    const float inv = 1.f / (float)F;
    const int64_t groups = (P.N + TEAMS - 1) / TEAMS;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t r = g * TEAMS + team;
        const bool on = r < P.N;
        const typename T::raw* x = static_cast<const typename T::raw*>(P.x) + r * P.ldx;
        const typename T::raw* d = static_cast<const typename T::raw*>(P.dout) + r * P.F;
        float t[CH][V], v[CH][V];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (on && col[k]) {
                load_floats<T, V>(x + at[k], t[k]);
                load_floats<T, V>(d + at[k], v[k]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) t[k][i] = v[k][i] = 0.f;
            }
        }
        const float rstd = on ? P.rstd[r] : 0.f;
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                t[k][i] *= rstd;  // xhat
                dw[k][i] = __builtin_fmaf(v[k][i], t[k][i], dw[k][i]);
                v[k][i] *= w[k][i];
                s = i >= skip[k] ? __builtin_fmaf(v[k][i], t[k][i], s) : s;
            }
        if (!P.out) continue;
        s = team_sum<L, BLOCK>(s, lds) * inv;
        if (!on) continue;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (!col[k]) continue;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = rstd * __builtin_fmaf(-t[k][i], s, v[k][i]);
            if (P.dtotal) {
                float e[V];
                load_floats<T, V>(static_cast<const typename T::raw*>(P.dtotal) + r * P.F + at[k], e);
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] += e[i];
            }
            store_as<V>(P.out, P.out_bf16, r * P.F + at[k], o);
        }
    }
    if (!P.dweight) return;
    float* to = gridDim.x == 1 ? P.dweight : P.part + (int64_t)blockIdx.x * P.F;
    if constexpr (L <= 64) {
        // (the teams of a workgroup, in order)
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) s_dw[threadIdx.x * V + i] = dw[k][i];
            __syncthreads();
            for (int e = threadIdx.x; e < L * V; e += BLOCK) {
                const int j = k * L + e / V;
                int sk;
                const int c = chunk_at<V>(j, F, sk) + e % V;
                if (j * V >= F || e % V < sk) continue;
                float s = 0.f;
                for (int q = 0; q < TEAMS; ++q) s += s_dw[q * L * V + e];
                to[c] = s;
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < CH; ++k)
            if (col[k]) store_floats<F32, V>(to + at[k], dw[k]);
    }
}

// Rows too long for the registers (dw, and both operands): read twice, the second time
// from the caches.  (512 MB of rows of 32,768 fp32: 647 us, and bf16 576.)
template <typename T, int V>
__device__ inline void grad_row(const RmsParams& P, int64_t r, float* lds) {
    const int F = (int)P.F, per = (F + V - 1) / V;
    const typename T::raw* x = static_cast<const typename T::raw*>(P.x) + r * P.ldx;
    const typename T::raw* d = static_cast<const typename T::raw*>(P.dout) + r * P.F;
    const float rstd = P.rstd[r];
    float s = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 2
        for (int j = threadIdx.x; j < per; j += kWide) {
            int skip;
            const int at = chunk_at<V>(j, F, skip);
            float t[V], v[V], w[V];
            load_floats<T, V>(x + at, t);
            load_floats<T, V>(d + at, v);
            if (P.weight) {
                load_floats<F32, V>(P.weight + at, w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] *= w[i];
            }
            if (pass == 0) {
#pragma unroll
                for (int i = 0; i < V; ++i) s = i >= skip ? __builtin_fmaf(v[i], t[i] * rstd, s) : s;
                continue;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = rstd * __builtin_fmaf(-(t[i] * rstd), s, v[i]);
            if (P.dtotal) {
                load_floats<T, V>(static_cast<const typename T::raw*>(P.dtotal) + r * P.F + at, w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] += w[i];
            }
            store_as<V>(P.out, P.out_bf16, r * P.F + at, v);
        }
        if (pass == 0) s = team_sum<kWide, kWide>(s, lds) / (float)F;
    }
}

template <typename T, int V>
__global__ __launch_bounds__(kWide) void rms_bwd_wide(RmsParams P) {
    __shared__ float lds[kWide / 64];
    for (int64_t r = blockIdx.x; r < P.N; r += gridDim.x) grad_row<T, V>(P, r, lds);
}

// Their dweight: blockIdx.x a tile of columns, blockIdx.y a share of the rows.
template <typename T, int V>
__global__ __launch_bounds__(kBlock) void rms_dw_wide(RmsParams P, int64_t rows) {
    const int F = (int)P.F, j = (int)blockIdx.x * kBlock + (int)threadIdx.x;
    if (j * V >= F) return;
    int skip;
    const int at = chunk_at<V>(j, F, skip);
    const int64_t r0 = (int64_t)blockIdx.y * rows, r1 = r0 + rows < P.N ? r0 + rows : P.N;
    float dw[V] = {};
#pragma unroll 2
    for (int64_t r = r0; r < r1; ++r) {
        const float rstd = P.rstd[r];
        float t[V], v[V];
        load_floats<T, V>(static_cast<const typename T::raw*>(P.x) + r * P.ldx + at, t);
        load_floats<T, V>(static_cast<const typename T::raw*>(P.dout) + r * P.F + at, v);
#pragma unroll
        for (int i = 0; i < V; ++i) dw[i] = __builtin_fmaf(v[i], t[i] * rstd, dw[i]);
    }
    store_floats<F32, V>((gridDim.y == 1 ? P.dweight : P.part + (int64_t)blockIdx.y * P.F) + at, dw);
}

// Lines of partial sums added in order: 32 columns a workgroup, 32 ranges of lines.
__global__ __launch_bounds__(1024) void rms_join(const float* part, int64_t lines, int64_t F,
                                                 float* out) {
    __shared__ float s_sum[32][33];
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + c;
    float s = 0.f;
    if (col < F) {
#pragma unroll 8
        for (int64_t b = q; b < lines; b += 32) s += part[b * F + col];
    }
    s_sum[q][c] = s;
    __syncthreads();
    if (q == 0 && col < F) {
        for (int i = 1; i < 32; ++i) s += s_sum[i][c];
        out[col] = s;
    }
}

// A thread takes eight values.
template <typename T>
__global__ __launch_bounds__(kBlock) void mx8_dequantize(const uint8_t* codes,
                                                         const uint8_t* scales, int64_t N,
                                                         int64_t K, typename T::raw* out) {
    const int64_t KB = (K + 31) / 32, per = KB * 4;
    for (int64_t l = (int64_t)blockIdx.x * kBlock + threadIdx.x; l < N * per;
         l += (int64_t)gridDim.x * kBlock) {
        const int64_t r = l / per, j = l - r * per;
        if (8 * j >= K) continue;
        const float f = scale_value(scales[r * KB + j / 4]);
        uint32_t c[2];
        __builtin_memcpy(c, codes + r * KB * 32 + 8 * j, 8);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e4m3_value(c[i / 4] >> (8 * (i % 4))) * f;
        store_to<8>(out, sizeof(typename T::raw) == 2, r * K, 8 * j, K, v);
    }
}

unsigned at_most(int64_t blocks) { return (unsigned)(blocks < kMaxGrid ? blocks : kMaxGrid); }

// How a row is laid out: elements of a chunk, threads of a team, chunks of a thread.
struct RmsShape {
    int V, L, CH, block;
};
RmsShape rms_shape(int64_t F, int dtype, bool q8) {
    RmsShape h{};
    h.V = q8 ? 8 : (dtype == MP_BF16 ? 8 : 4);
    if (!q8 && F < h.V) h.V = 1;
    const int64_t per = ceil_div(F, h.V);
    h.block = kBlock;
    h.CH = 1;
    h.L = q8 ? 4 : 1;
    while (h.L < 64 && h.L < per) h.L *= 2;
    if (per <= 64) return h;
    if (per <= 256) {
        h.CH = per <= 128 ? 2 : 4;
        return h;
    }
    h.L = h.block = per <= 1024 ? 256 : 1024;
    h.CH = (int)ceil_div(per, h.L);
    h.CH = h.CH <= 2 ? 2 : (h.CH <= 4 ? 4 : (h.CH <= 8 ? 8 : 16));
    return h;
}

#define MP_RMS_WIDE(CALL, T, V)                              \
    if (h.block == 1024) {                                   \
        if (h.CH == 2) CALL(T, V, 1024, 2, 1024);            \
        else if (h.CH == 4) CALL(T, V, 1024, 4, 1024);       \
        else if (h.CH == 8) CALL(T, V, 1024, 8, 1024);       \
        else if constexpr (V == 4) CALL(T, V, 1024, 16, 1024); \
    } else if (h.block == kBlock && h.L == kBlock) {         \
        if (h.CH == 2) CALL(T, V, kBlock, 2, kBlock);        \
        else CALL(T, V, kBlock, 4, kBlock);                  \
    } else if (h.L == 64) {                                  \
        if (h.CH == 1) CALL(T, V, 64, 1, kBlock);            \
        else if (h.CH == 2) CALL(T, V, 64, 2, kBlock);       \
        else CALL(T, V, 64, 4, kBlock);                      \
    } else if (h.L == 32) CALL(T, V, 32, 1, kBlock);         \
    else if (h.L == 16) CALL(T, V, 16, 1, kBlock);           \
    else if (h.L == 8) CALL(T, V, 8, 1, kBlock);             \
    else if (h.L == 4) CALL(T, V, 4, 1, kBlock);

template <typename T, int V>
void launch_fwd(const RmsParams& p, const RmsShape& h, hipStream_t s) {
    const dim3 g(at_most(ceil_div(p.N, h.block / h.L)));
#define MP_RMS_FWD(T, V, L, CH, B) \
    hipLaunchKernelGGL((rms_fwd<T, V, L, CH, B, false>), g, dim3(B), 0, s, p)
    if constexpr (V == 1) {
        if (h.L == 8) MP_RMS_FWD(T, 1, 8, 1, kBlock);
        else if (h.L == 4) MP_RMS_FWD(T, 1, 4, 1, kBlock);
        else if (h.L == 2) MP_RMS_FWD(T, 1, 2, 1, kBlock);
        else MP_RMS_FWD(T, 1, 1, 1, kBlock);
    } else {
        MP_RMS_WIDE(MP_RMS_FWD, T, V)
        else if (h.L == 2) MP_RMS_FWD(T, V, 2, 1, kBlock);
        else MP_RMS_FWD(T, V, 1, 1, kBlock);
    }
#undef MP_RMS_FWD
}

template <typename T>
void launch_q8(const RmsParams& p, const RmsShape& h, hipStream_t s) {
    const dim3 g(at_most(ceil_div(p.N, h.block / h.L)));
#define MP_RMS_Q8(T, V, L, CH, B) \
    hipLaunchKernelGGL((rms_fwd<T, V, L, CH, B, true>), g, dim3(B), 0, s, p)
    MP_RMS_WIDE(MP_RMS_Q8, T, 8)
#undef MP_RMS_Q8
}

template <typename T, int V>
void launch_bwd(const RmsParams& p, const RmsShape& h, int64_t blocks, hipStream_t s) {
    const dim3 g((unsigned)blocks);
#define MP_RMS_BWD(T, V, L, CH, B)                                                     \
    do {                                                                               \
        if constexpr (CH * V <= 16 || B < 1024)                                        \
            hipLaunchKernelGGL((rms_bwd<T, V, L, CH, B>), g, dim3(B), 0, s, p);        \
    } while (0)
    if constexpr (V == 1) {
        if (h.L == 8) MP_RMS_BWD(T, 1, 8, 1, kBlock);
        else if (h.L == 4) MP_RMS_BWD(T, 1, 4, 1, kBlock);
        else if (h.L == 2) MP_RMS_BWD(T, 1, 2, 1, kBlock);
        else MP_RMS_BWD(T, 1, 1, 1, kBlock);
    } else {
        MP_RMS_WIDE(MP_RMS_BWD, T, V)
        else if (h.L == 2) MP_RMS_BWD(T, V, 2, 1, kBlock);
        else MP_RMS_BWD(T, V, 1, 1, kBlock);
    }
#undef MP_RMS_BWD
}

// Backward rows of more than 16 elements a thread.
bool wide(const RmsShape& h) { return h.CH * h.V > 16 && h.block == 1024; }
int64_t wide_rows(int64_t N) { return N > 16 * 64 ? ceil_div(N, 64) : 16; }

template <typename T, int V>
void launch_bwd_wide(const RmsParams& p, int64_t parts, hipStream_t s) {
    if (p.out && p.N > 0)
        hipLaunchKernelGGL((rms_bwd_wide<T, V>), dim3(at_most(p.N)), dim3(kWide), 0, s, p);
    if (p.dweight)
        hipLaunchKernelGGL((rms_dw_wide<T, V>),
                           dim3((unsigned)ceil_div(p.F, V * kBlock), (unsigned)parts), dim3(kBlock),
                           0, s, p, wide_rows(p.N));
}

}  // namespace

int64_t rms_parts(int64_t N, int64_t F, int dtype) {
    const RmsShape h = rms_shape(F, dtype, false);
    if (wide(h)) return N < 1 ? 1 : ceil_div(N, wide_rows(N));
    const int64_t groups = ceil_div(N, h.block / h.L);
    // (2.4M rows of 100 fp32 with 768, 1,024 and 2,048 workgroups: 564, 580 and 643 us;
    // 169,343 of 256 bf16 without dtotal 53, 49 and 43, and the lines' sum 5, 5 and 10; with
    // dtotal 72 and 5 at 1,024)
    const int64_t most = h.block == 1024 ? 512 : 1024;
    return groups < 1 ? 1 : (groups < most ? groups : most);
}

hipError_t launch_rms(const RmsParams& p, int dtype, hipStream_t s) {
    if (p.N <= 0) return hipSuccess;
    const RmsShape h = rms_shape(p.F, dtype, p.codes != nullptr);
    if (p.codes) {
        if (dtype == MP_BF16) launch_q8<BF16>(p, h, s);
        else launch_q8<F32>(p, h, s);
    } else if (h.V == 1) {
        if (dtype == MP_BF16) launch_fwd<BF16, 1>(p, h, s);
        else launch_fwd<F32, 1>(p, h, s);
    } else {
        if (dtype == MP_BF16) launch_fwd<BF16, 8>(p, h, s);
        else launch_fwd<F32, 4>(p, h, s);
    }
    return hipGetLastError();
}

hipError_t launch_rms_backward(const RmsParams& p, int dtype, hipStream_t s) {
    const RmsShape h = rms_shape(p.F, dtype, false);
    const int64_t blocks = rms_parts(p.N, p.F, dtype);
    if (wide(h)) {
        if (dtype == MP_BF16) launch_bwd_wide<BF16, 8>(p, blocks, s);
        else launch_bwd_wide<F32, 4>(p, blocks, s);
    } else if (h.V == 1) {
        if (dtype == MP_BF16) launch_bwd<BF16, 1>(p, h, blocks, s);
        else launch_bwd<F32, 1>(p, h, blocks, s);
    } else {
        if (dtype == MP_BF16) launch_bwd<BF16, 8>(p, h, blocks, s);
        else launch_bwd<F32, 4>(p, h, blocks, s);
    }
    if (p.dweight && blocks > 1)
        hipLaunchKernelGGL(rms_join, dim3((unsigned)ceil_div(p.F, 32)), dim3(1024), 0, s, p.part,
                           blocks, p.F, p.dweight);
    return hipGetLastError();
}

hipError_t launch_mx8_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t N, int64_t K,
                                 void* out, int dtype, hipStream_t s) {
    if (N <= 0) return hipSuccess;
    const int64_t blocks = ceil_div(N * ceil_div(K, 32) * 4, kBlock);
    const dim3 g((unsigned)(blocks < 65536 ? blocks : 65536));
    if (dtype == MP_BF16)
        hipLaunchKernelGGL((mx8_dequantize<BF16>), g, dim3(kBlock), 0, s, codes, scales, N, K,
                           static_cast<uint16_t*>(out));
    else
        hipLaunchKernelGGL((mx8_dequantize<F32>), g, dim3(kBlock), 0, s, codes, scales, N, K,
                           static_cast<float*>(out));
    return hipGetLastError();
}

}  // namespace mp
