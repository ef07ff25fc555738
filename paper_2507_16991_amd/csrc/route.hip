// Softmax router: the k largest logits of each row, their weights, per-expert
// counts, balance and z loss, and the gradient (include/mp_layers.h).
//
// A row lies on L lanes of a wavefront with V experts each (V = 8: one 16-byte
// load of bf16), so 64 / L rows go through every instruction and nothing
// passes through LDS until the workgroup's sums are joined at the end.  Choosing
// is k rounds of a maximum over the V keys of a lane and, by DPP, over the L
// lanes.  A key orders the logits as unsigned integers; a bf16 key carries
// the expert in its lower half, so that one maximum finds value and place,
// an fp32 key takes a second round for the lowest place of the maximum.
// Sums of probabilities stay in registers of the lane that owns the expert, counts
// are integer atomics in LDS (one a choice; in registers they cost an addition
// an expert and round: 33 -> 29 us for 169k rows of 64 bf16 experts, k = 8); each
// workgroup leaves one line of partial sums, and a workgroup of a second launch
// adds them in order (a small call has one workgroup, which ends by itself).
#include "layers_internal.hpp"

namespace mp {
namespace {

constexpr int kBlock = 512;
constexpr int kWaves = kBlock / kWave;
constexpr int kFinish = 1024;  // threads of the launch that adds the partial sums

// exp(x) for x <= 0 (and NaN): 2^(x log2 e) with the product's rounding error
// put back to first order, relative error about 2^-23.
__device__ inline float exp_neg(float x) {
    const float c = 1.44269502f, c_low = 1.92596303e-8f;  // log2 e
    const float y = x * c;
    const float r = __builtin_fmaf(x, c_low, __builtin_fmaf(x, c, -y));
    const float v = __builtin_amdgcn_exp2f(y);
    // (at -inf the error term is NaN and the power 0)
    return v > 0.f ? __builtin_fmaf(v, r * 0.693147181f, v) : v;
}

// ---- keys ------------------------------------------------------------------------
// Unsigned order of floats (-0 made +0 by the caller), NaN above all; 0 for
// -inf, which is never chosen.
__device__ inline uint32_t order(float v) {
    const uint32_t u = __float_as_uint(v);
    uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    k = v != v ? 0xFFFFFFFFu : k;
    return v == -__builtin_inff() ? 0u : k;
}
__device__ inline float value_of(uint32_t k) {
    return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}

// The L lanes' V experts of row r; -inf where there are none or the row takes
// no part.
template <typename T, int V>
__device__ inline void load_row(const RouteParams& P, int64_t r, int sub, float (&l)[V]) {
    const bool on = r < P.N && (!P.mask || P.mask[r]);
    const typename T::raw* p = static_cast<const typename T::raw*>(P.logits) + r * P.ldl;
    const int e0 = sub * V;
    if (on && e0 + V <= P.E) {
        load_floats<T, V>(p + e0, l);
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
            l[v] = on && e0 + v < P.E ? load_one<T>(p + e0 + v) : -__builtin_inff();
    }
}

// ---- the losses from the sums over all rows ------------------------------------------
// s_p, s_c: sums of probabilities and counts by expert, in LDS; all threads.
template <int BLOCK>
__device__ inline void finish(const RouteParams& P, const float* s_p, const int32_t* s_c, float z,
                              int rows, float* s_red) {
    const int tid = threadIdx.x, E = (int)P.E;
    float dot = 0.f;
    int total = 0;
    for (int e = tid; e < E; e += BLOCK) {
        dot += (float)s_c[e] * s_p[e];
        total += s_c[e];
        P.counts[e] = s_c[e];
    }
    dot = reduce_sum<64>(dot);
    total = (int)reduce_add<64>((uint32_t)total);
    if ((tid & 63) == 0) {
        s_red[2 * (tid >> 6)] = dot;
        s_red[2 * (tid >> 6) + 1] = __int_as_float(total);
    }
    __syncthreads();
    if (tid == 0) {
        float d = 0.f;
        int t = 0;
        for (int w = 0; w < BLOCK / 64; ++w) {
            d += s_red[2 * w];
            t += __float_as_int(s_red[2 * w + 1]);
        }
        P.counts[E] = rows;
        const float n = (float)(rows > 0 ? rows : 1);
        P.loss[0] = rows > 0 ? (float)E * (d / (float)t / n) : 0.f;
        P.loss[1] = rows > 0 ? z / n : 0.f;
    }
}

template <typename T, int V, int L>
__global__ __launch_bounds__(kBlock) void route_fwd(RouteParams P) {
    constexpr int RW = kWave / L;             // rows of a wavefront
    constexpr bool kPlace = sizeof(typename T::raw) == 2;  // keys carry the expert
    __shared__ float s_sum[kBlock * V];       // [wave][row slot][L V experts]
    __shared__ float s_p[L * V];
    __shared__ int32_t s_c[L * V];
    __shared__ float s_z[kWaves];
    __shared__ int s_rows[kWaves];
    __shared__ float s_red[2 * kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int sub = lane % L, slot = lane / L;
    const int E = (int)P.E, k = (int)P.k;

    float psum[V] = {};
    float zsum = 0.f;
    int rows = 0;
    for (int e = tid; e < L * V; e += kBlock) s_c[e] = 0;
    __syncthreads();

    const int64_t groups = (P.N + RW - 1) / RW;
    for (int64_t g = (int64_t)blockIdx.x * kWaves + wave; g < groups;
         g += (int64_t)gridDim.x * kWaves) {
        const int64_t r = g * RW + slot;
        float l[V];
        load_row<T, V>(P, r, sub, l);
        uint32_t key[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            key[v] = order(l[v] + 0.f);  // (-0 + 0 = +0)
            if (kPlace && key[v]) key[v] = (key[v] & 0xFFFF0000u) | (0xFFFFu - (sub * V + v));
        }
        float big = 0.f, chosen = 0.f, my_w = 0.f;
        int my_e = -1;
        bool part = false;
        for (int j = 0; j < k; ++j) {
            uint32_t m = key[0];
#pragma unroll
            for (int v = 1; v < V; ++v) m = m > key[v] ? m : key[v];
            m = reduce_max<L>(m);
            uint32_t e;
            if (kPlace) {
                e = 0xFFFFu - (m & 0xFFFFu);
            } else {
                e = 0xFFFFFFFFu;
#pragma unroll
                for (int v = V - 1; v >= 0; --v) e = key[v] == m ? sub * V + v : e;
                e = reduce_min<L>(e);
            }
            const bool real = m != 0;
            const uint32_t bits = __float_as_uint(value_of(m));
            const float val = __uint_as_float(kPlace ? bits & 0xFFFF0000u : bits);
            if (j == 0) {
                big = real ? val : 0.f;
                part = real;
            }
            const float w = real ? exp_neg(val - big) : 0.f;
            chosen += w;
            const bool mine = j % L == sub;
            my_w = mine ? w : my_w;
            my_e = mine ? (real ? (int)e : -1) : my_e;
#pragma unroll
            for (int v = 0; v < V; ++v)  // (keys with their place differ, but for 0)
                key[v] = (kPlace ? key[v] == m : (int)e == sub * V + v) ? 0u : key[v];
            // a row of more choices than lanes is written as it fills them
            if (k > L && (j % L == L - 1 || j == k - 1)) {
                const int at = j - j % L + sub;
                if (r < P.N && at <= j) {
                    P.idx[r * k + at] = my_e;
                    P.weight[r * k + at] = my_w;
                    if (my_e >= 0) atomicAdd(&s_c[my_e], 1);
                }
            }
        }
        float tot = 0.f, p[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            p[v] = part ? exp_neg(l[v] - big) : 0.f;
            tot += p[v];
        }
        tot = reduce_sum<L>(tot);
        const float inv = part ? 1.f / tot : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) psum[v] = __builtin_fmaf(p[v], inv, psum[v]);
        if (part && sub == 0) {
            const float lse = big + logf(tot);
            zsum = __builtin_fmaf(lse, lse, zsum);
            ++rows;
        }
        const float norm = part ? 1.f / (P.renorm ? chosen : tot) : 0.f;
        if (k <= L) {
            if (r < P.N && sub < k) {
                P.idx[r * k + sub] = my_e;
                P.weight[r * k + sub] = my_w * norm;
                if (my_e >= 0) atomicAdd(&s_c[my_e], 1);
            }
        } else if (r < P.N) {
            for (int j = sub; j < k; j += L) P.weight[r * k + j] *= norm;  // this lane's own
        }
    }

    // the workgroup's sums of probabilities, row slots in order
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) s_sum[(wave * RW + slot) * (L * V) + sub * V + v] = psum[v];
    __syncthreads();
    for (int e = tid; e < E; e += kBlock) {
        float s = 0.f;
        for (int i = 0; i < kWaves * RW; ++i) s += s_sum[i * (L * V) + e];
        s_p[e] = s;
    }
    zsum = reduce_sum<64>(zsum);
    rows = (int)reduce_add<64>((uint32_t)rows);
    if (lane == 0) {
        s_z[wave] = zsum;
        s_rows[wave] = rows;
    }
    __syncthreads();
    float z = 0.f;
    int n = 0;
    for (int w = 0; w < kWaves; ++w) {
        z += s_z[w];
        n += s_rows[w];
    }
    if (gridDim.x == 1) {
        finish<kBlock>(P, s_p, s_c, z, n, s_red);
        return;
    }
    float* part_p = P.part + (int64_t)blockIdx.x * (2 * E + 2);
    for (int e = tid; e < E; e += kBlock) {
        part_p[e] = s_p[e];
        part_p[E + e] = __int_as_float(s_c[e]);
    }
    if (tid == 0) {
        part_p[2 * E] = z;
        part_p[2 * E + 1] = __int_as_float(n);
    }
}

// The partial sums of `blocks` workgroups added in order: an expert has as many
// threads as the workgroup allows, each a range of the lines.
__global__ __launch_bounds__(kFinish) void route_finish(RouteParams P, int blocks) {
    __shared__ float s_sum[kFinish], s_p[1024];
    __shared__ int32_t s_cnt[kFinish], s_c[1024];
    __shared__ float s_z[kFinish / 64], s_red[2 * kFinish / 64];
    __shared__ int s_rows[kFinish / 64];
    const int tid = threadIdx.x, E = (int)P.E;
    int cols = 1;
    while (cols < E) cols *= 2;  // at most 1024
    const int ranges = kFinish / cols, e = tid % cols, q = tid / cols;
    const int64_t line = 2 * E + 2;
    float p = 0.f;
    int32_t c = 0;
    if (e < E) {
#pragma unroll 8
        for (int b = q; b < blocks; b += ranges) {
            p += P.part[b * line + e];
            c += __float_as_int(P.part[b * line + E + e]);
        }
    }
    s_sum[tid] = p;
    s_cnt[tid] = c;
    float z = 0.f;
    int n = 0;
    for (int b = tid; b < blocks; b += kFinish) {
        z += P.part[b * line + 2 * E];
        n += __float_as_int(P.part[b * line + 2 * E + 1]);
    }
    z = reduce_sum<64>(z);
    n = (int)reduce_add<64>((uint32_t)n);
    if ((tid & 63) == 0) {
        s_z[tid >> 6] = z;
        s_rows[tid >> 6] = n;
    }
    __syncthreads();
    if (q == 0 && e < E) {
        for (int i = 1; i < ranges; ++i) {
            p += s_sum[i * cols + e];
            c += s_cnt[i * cols + e];
        }
        s_p[e] = p;
        s_c[e] = c;
    }
    z = 0.f;
    n = 0;
    for (int w = 0; w < kFinish / 64; ++w) {
        z += s_z[w];
        n += s_rows[w];
    }
    __syncthreads();
    finish<kFinish>(P, s_p, s_c, z, n, s_red);
}

// dL/dlogits: with p the softmax, d_e = dL/dp_e of the balance loss and S =
// sum_j w_j dw_j,
//   p_e (d_e - sum p d + 2 dz lse / R)  [- p_e S without renorm]
//   + w_j (dw_j - S)  [w_j dw_j without renorm] where e is the row's j-th choice.
// Bound by its vector instructions, k V comparisons a lane: 169k rows of 64 bf16
// experts, k = 8, 30 us (60 MB).
template <typename T, int V, int L>
__global__ __launch_bounds__(kBlock) void route_bwd(RouteParams P) {
    constexpr int RW = kWave / L;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int sub = lane % L, slot = lane / L;
    const int E = (int)P.E, k = (int)P.k;
    const int R = P.counts[E] > 0 ? P.counts[E] : 1;
    const float db = P.dloss ? P.dloss[0] : 0.f;
    const float dz = P.dloss ? 2.f * P.dloss[1] / (float)R : 0.f;
    float d[V];
    int total = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = sub * V + v;
        const int c = e < E ? P.counts[e] : 0;
        d[v] = (float)c;
        total += c;
    }
    total = (int)reduce_add<L>((uint32_t)total);
    const float scale = total > 0 ? db * (float)E / (float)total / (float)R : 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) d[v] *= scale;

    const int64_t groups = (P.N + RW - 1) / RW;
    for (int64_t g = (int64_t)blockIdx.x * kWaves + wave; g < groups;
         g += (int64_t)gridDim.x * kWaves) {
        const int64_t r = g * RW + slot;
        float l[V];
        load_row<T, V>(P, r, sub, l);
        float big = l[0];
        uint32_t any = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            big = fmaxf(big, l[v]);
            any |= l[v] != -__builtin_inff();  // (NaN: the row takes part)
        }
        big = reduce_fmax<L>(big);
        const bool part = reduce_max<L>(any) != 0;
        float tot = 0.f, pd = 0.f, p[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            p[v] = part ? exp_neg(l[v] - big) : 0.f;
            tot += p[v];
            pd = __builtin_fmaf(p[v], d[v], pd);
        }
        tot = reduce_sum<L>(tot);
        pd = reduce_sum<L>(pd);
        const float inv = part ? 1.f / tot : 0.f;
        const float lse = part ? big + logf(tot) : 0.f;
        float c = __builtin_fmaf(dz, lse, -pd * inv);  // what every p_e is multiplied by, but d_e
        float S = 0.f;
        if (P.dweight) {
            for (int j = sub; j < k; j += L)
                if (r < P.N && P.idx[r * k + j] >= 0)
                    S = __builtin_fmaf(P.weight[r * k + j], P.dweight[r * k + j], S);
            S = reduce_sum<L>(S);
            if (!P.renorm) c -= S;
        }
        float dl[V];
#pragma unroll
        for (int v = 0; v < V; ++v) dl[v] = part ? p[v] * inv * (d[v] + c) : 0.f;
        if (P.dweight) {
            for (int j0 = 0; j0 < k; j0 += L) {
                const int j = j0 + sub;
                int e = -1;
                float t = 0.f;
                if (r < P.N && j < k && part) {
                    e = P.idx[r * k + j];
                    t = P.weight[r * k + j] * (P.dweight[r * k + j] - (P.renorm ? S : 0.f));
                }
                const int n = k - j0 < L ? k - j0 : L;
                for (int i = 0; i < n; ++i) {
                    const int ei = __shfl(e, slot * L + i);
                    const float ti = __shfl(t, slot * L + i);
#pragma unroll
                    for (int v = 0; v < V; ++v) dl[v] += ei == sub * V + v ? ti : 0.f;
                }
            }
        }
        if (r >= P.N) continue;
        typename T::raw* out = static_cast<typename T::raw*>(P.dlogits) + r * E;
        const int e0 = sub * V;
        if (e0 + V <= E) {
            store_floats<T, V>(out + e0, dl);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (e0 + v < E) store_one<T>(out + e0 + v, dl[v]);
        }
    }
}

// Lanes of a row and experts of a lane: 8 experts a lane up to 512, else 16.
int lanes_of(int64_t E) {
    int l = 1;
    while (l < 64 && l * 8 < E) l *= 2;
    return l;
}

template <typename T>
void launch(const RouteParams& p, bool backward, int blocks, hipStream_t s) {
    const dim3 g((unsigned)blocks), b(kBlock);
#define MP_ROUTE(V, L)                                                              \
    if (backward) hipLaunchKernelGGL((route_bwd<T, V, L>), g, b, 0, s, p);          \
    else hipLaunchKernelGGL((route_fwd<T, V, L>), g, b, 0, s, p);                   \
    break
    if (p.E > 512) {
        switch (0) {
            default: MP_ROUTE(16, 64);
        }
        return;
    }
    switch (lanes_of(p.E)) {
        case 1: MP_ROUTE(8, 1);
        case 2: MP_ROUTE(8, 2);
        case 4: MP_ROUTE(8, 4);
        case 8: MP_ROUTE(8, 8);
        case 16: MP_ROUTE(8, 16);
        case 32: MP_ROUTE(8, 32);
        default: MP_ROUTE(8, 64);
    }
#undef MP_ROUTE
}

}  // namespace

// Workgroups of the forward: one for up to 16 wavefronts' rows (no second
// launch), else at most 512, fewer where a line of partial sums is long.  (bf16, k = 8,
// 65536 / E against 512 of them: 16,384 x 256 25 and 30 us.  Tables of many rows and
// experts pay for it: 131,072 x 256 106 and 89 us, 32,768 x 1024 287 and 118.)
int route_blocks(int64_t N, int64_t E) {
    const int64_t groups = ceil_div(N, kWave / lanes_of(E));
    if (groups <= 2 * kWaves) return 1;
    int64_t most = 65536 / E;
    if (most > 512) most = 512;
    const int64_t blocks = ceil_div(groups, kWaves);
    return (int)(blocks < most ? blocks : most);
}

hipError_t launch_route(const RouteParams& p, int dtype, hipStream_t s) {
    const int blocks = route_blocks(p.N, p.E);
    if (dtype == MP_BF16) launch<BF16>(p, false, blocks, s);
    else launch<F32>(p, false, blocks, s);
    if (blocks > 1)
        hipLaunchKernelGGL(route_finish, dim3(1), dim3(kFinish), 0, s, p, blocks);
    return hipGetLastError();
}

hipError_t launch_route_backward(const RouteParams& p, int dtype, hipStream_t s) {
    if (p.N <= 0) return hipSuccess;
    const int64_t blocks = ceil_div(ceil_div(p.N, kWave / lanes_of(p.E)), kWaves);
    const int grid = (int)(blocks < 2048 ? blocks : 2048);
    if (dtype == MP_BF16) launch<BF16>(p, true, grid, s);
    else launch<F32>(p, true, grid, s);
    return hipGetLastError();
}

}  // namespace mp
