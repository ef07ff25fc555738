// Dropout from a counter-based generator (include/mp_layers.h states which
// random word belongs to which element).
//
// One call of Philox4x32-10 gives eight 16-bit words, one for each of eight
// consecutive element numbers, so a thread takes one such block: with bf16 one
// 16-byte load and store, and 20 32-bit products of which the first two
// rounds' upper halves are the same for all threads.  Sixteen bits an element
// keep it bound by memory: with 32 the generator alone would take about as
// long as moving bf16 elements does.
#include "layers_internal.hpp"

namespace mp {
namespace {

constexpr int kBlock = 256;
constexpr int kWords = 8;  // elements of a Philox block
constexpr int64_t kMaxGrid = int64_t(1) << 22;

// Ten rounds: (c0, c1, c2, c3) <- (hi(M1 c2) ^ c1 ^ k0, lo(M1 c2),
// hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)), the key stepping by two odd constants.
__device__ inline void philox(uint64_t block, uint64_t key, uint64_t t, uint32_t (&w)[4]) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32);
    uint32_t c2 = (uint32_t)t, c3 = (uint32_t)(t >> 32);
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)p1;
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0;
    w[1] = c1;
    w[2] = c2;
    w[3] = c3;
}

// Bit i: element i of the block stays.
__device__ inline uint32_t keep_bits(uint64_t block, uint64_t key, uint64_t t, uint32_t limit) {
    uint32_t w[4], m = 0;
    philox(block, key, t, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m |= (uint32_t)((w[i] & 0xFFFFu) >= limit) << (2 * i);
        m |= (uint32_t)((w[i] >> 16) >= limit) << (2 * i + 1);
    }
    return m;
}

__device__ inline uint64_t draw_of(const DropoutParams& P) {
    return P.offset + (P.step ? (uint64_t)*P.step : 0);
}

// v <- the elements that stay, scaled, plus the residual.  The sum is one
// fused operation, as exact as can be.
template <bool RES, int V>
__device__ inline void apply(float (&v)[V], const float (&r)[V], uint32_t m, float scale) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float k = (m >> i) & 1 ? v[i] : 0.f;  // a select: infinities and NaN go too
        v[i] = RES ? __builtin_fmaf(k, scale, r[i]) : k * scale;
    }
}

// Elements f0 .. f0+7 of a row, those in [0, F) of them.
template <typename T, bool RES>
__device__ inline void drop_chunk(const typename T::raw* x, const typename T::raw* res,
                                  typename T::raw* out, int64_t f0, int64_t F, uint32_t m,
                                  float scale) {
    if (f0 >= 0 && f0 + kWords <= F) {
        float v[kWords], r[kWords] = {};
        load_floats<T, kWords>(x + f0, v);
        if (RES) load_floats<T, kWords>(res + f0, r);
        apply<RES>(v, r, m, scale);
        store_floats<T, kWords>(out + f0, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        const int64_t f = f0 + i;
        if (f < 0 || f >= F) continue;
        float v[1] = {load_one<T>(x + f)}, r[1] = {RES ? load_one<T>(res + f) : 0.f};
        apply<RES>(v, r, m >> i, scale);
        store_one<T>(out + f, v[0]);
    }
}

// Contiguous tables without ids: element numbers are places.  Bound by memory: 2.4M x
// 100 bf16 with a residual 252 us (5.8 TB/s), without 162 us (6.0 TB/s).
template <typename T, bool RES>
__global__ __launch_bounds__(kBlock) void dropout_flat(DropoutParams P) {
    typedef typename T::raw raw;
    const int64_t n = P.N * P.F, blocks = (n + kWords - 1) / kWords;
    const uint64_t t = draw_of(P);
    const raw* x = static_cast<const raw*>(P.x);
    const raw* res = static_cast<const raw*>(P.residual);
    raw* out = static_cast<raw*>(P.out);
    for (int64_t b = (int64_t)blockIdx.x * kBlock + threadIdx.x; b < blocks;
         b += (int64_t)gridDim.x * kBlock)
        drop_chunk<T, RES>(x, res, out, b * kWords, n,
                           keep_bits((uint64_t)b, P.seed, t, P.limit), P.scale);
}

// Any strides and ids: a workgroup takes whole rows, a thread one Philox block
// of a row (of F elements a row has at most (F + 14) / 8, as it may begin
// inside one).  ROWS: one word for the row, and the chunks begin with it.  (2.4M rows by
// ids: 128 bf16 247 us, 5.1 TB/s; 100 bf16, whose chunks are cut at both ends of a row,
// 365 us, 2.7 TB/s.  Whole rows of 100 bf16 270 us.)
template <typename T, bool RES, bool ROWS>
__global__ __launch_bounds__(kBlock) void dropout_rows(DropoutParams P, uint32_t cpr,
                                                       uint32_t rows_per_block) {
    typedef typename T::raw raw;
    const uint64_t t = draw_of(P);
    const int64_t groups = (P.N + rows_per_block - 1) / rows_per_block;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t r0 = g * rows_per_block;
        const uint32_t nr =
            (uint32_t)(P.N - r0 < (int64_t)rows_per_block ? P.N - r0 : rows_per_block);
        for (uint32_t l = threadIdx.x; l < nr * cpr; l += kBlock) {
            const uint32_t dr = l / cpr, j = l - dr * cpr;
            const int64_t r = r0 + dr;
            const uint64_t id = P.ids ? (uint64_t)(uint32_t)P.ids[r] : (uint64_t)r;
            int64_t f0;
            uint32_t m;
            if (ROWS) {
                const uint32_t w = keep_bits(id >> 3, P.seed, t, P.limit);
                m = 0u - ((w >> (id & 7)) & 1u);
                f0 = (int64_t)j * kWords;
            } else {
                const uint64_t e0 = id * (uint64_t)P.F, b = (e0 >> 3) + j;
                f0 = (int64_t)(b * kWords - e0);
                if (f0 >= P.F) continue;
                m = keep_bits(b, P.seed, t, P.limit);
            }
            drop_chunk<T, RES>(static_cast<const raw*>(P.x) + r * P.ldx,
                               static_cast<const raw*>(P.residual) + (RES ? r * P.ldr : 0),
                               static_cast<raw*>(P.out) + r * P.ldo, f0, P.F, m, P.scale);
        }
    }
}

// One element a row, as edge weights have, without a stride: every row has a
// Philox block of its own, so the generator's products bound it; a thread
// takes four rows with 16-byte loads (124M fp32 weights, calls in a row: 290 us, 5.1
// TB/s; one row a thread by dropout_rows 1061 us).
template <typename T, bool RES>
__global__ __launch_bounds__(kBlock) void dropout_scalars(DropoutParams P) {
    typedef typename T::raw raw;
    const uint64_t t = draw_of(P);
    const raw* x = static_cast<const raw*>(P.x);
    const raw* res = static_cast<const raw*>(P.residual);
    raw* out = static_cast<raw*>(P.out);
    const int64_t groups = (P.N + 3) / 4;
    for (int64_t g = (int64_t)blockIdx.x * kBlock + threadIdx.x; g < groups;
         g += (int64_t)gridDim.x * kBlock) {
        const int64_t r0 = 4 * g;
        const bool whole = r0 + 4 <= P.N;
        int32_t id[4] = {0, 0, 0, 0};
        float v[4] = {}, r[4] = {};
        if (whole) {
            __builtin_memcpy(id, P.ids + r0, sizeof(id));
            load_floats<T, 4>(x + r0, v);
            if (RES) load_floats<T, 4>(res + r0, r);
        } else {
            for (int i = 0; i < 4; ++i)
                if (r0 + i < P.N) {
                    id[i] = P.ids[r0 + i];
                    v[i] = load_one<T>(x + r0 + i);
                    if (RES) r[i] = load_one<T>(res + r0 + i);
                }
        }
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t e = (uint32_t)id[i];
            uint32_t w[4];
            philox(e >> 3, P.seed, t, w);
            const uint32_t a = e & 2 ? w[1] : w[0], b = e & 2 ? w[3] : w[2];
            const uint32_t word = ((e & 4 ? b : a) >> (16 * (e & 1))) & 0xFFFFu;
            m |= (uint32_t)(word >= P.limit) << i;
        }
        apply<RES>(v, r, m, P.scale);
        if (whole) {
            store_floats<T, 4>(out + r0, v);
        } else {
            for (int i = 0; i < 4; ++i)
                if (r0 + i < P.N) store_one<T>(out + r0 + i, v[i]);
        }
    }
}

template <typename T, bool RES>
void launch(const DropoutParams& p, int whole_rows, hipStream_t s) {
    const int64_t F = p.F;
    const bool dense = p.N <= 1 || (p.ldx == F && p.ldo == F && (!RES || p.ldr == F));
    if (dense && !p.ids && (!whole_rows || F == 1)) {  // (of one element a row is an element)
        const int64_t blocks = ceil_div(p.N * F, (int64_t)kWords * kBlock);
        hipLaunchKernelGGL((dropout_flat<T, RES>),
                           dim3((unsigned)(blocks < kMaxGrid ? blocks : kMaxGrid)), dim3(kBlock),
                           0, s, p);
        return;
    }
    if (F == 1 && dense && p.ids) {
        const int64_t blocks = ceil_div(p.N, (int64_t)4 * kBlock);
        hipLaunchKernelGGL((dropout_scalars<T, RES>), dim3((unsigned)blocks), dim3(kBlock), 0, s,
                           p);
        return;
    }
    const int64_t cpr = whole_rows || F % kWords == 0 ? ceil_div(F, kWords) : (F + 14) / kWords;
    const int64_t rpb = cpr >= kBlock ? 1 : kBlock / cpr;
    const int64_t groups = ceil_div(p.N, rpb);
    const dim3 g((unsigned)(groups < kMaxGrid ? groups : kMaxGrid)), b(kBlock);
    if (whole_rows)
        hipLaunchKernelGGL((dropout_rows<T, RES, true>), g, b, 0, s, p, (uint32_t)cpr,
                           (uint32_t)rpb);
    else
        hipLaunchKernelGGL((dropout_rows<T, RES, false>), g, b, 0, s, p, (uint32_t)cpr,
                           (uint32_t)rpb);
}

}  // namespace

hipError_t launch_dropout(const DropoutParams& p, int dtype, int whole_rows, hipStream_t s) {
    if (p.N <= 0) return hipSuccess;
    if (dtype == MP_BF16) {
        if (p.residual) launch<BF16, true>(p, whole_rows, s);
        else launch<BF16, false>(p, whole_rows, s);
    } else {
        if (p.residual) launch<F32, true>(p, whole_rows, s);
        else launch<F32, false>(p, whole_rows, s);
    }
    return hipGetLastError();
}

}  // namespace mp
