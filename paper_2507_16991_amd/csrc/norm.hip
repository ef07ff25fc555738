// Group norm with an activation over segments of consecutive rows, channels
// last, and its gradients (include/mp_layers.h).
//
// Bound by memory (gelu also by its arithmetic), so what counts is how often
// the rows are read.  Segment lengths are on the device; two paths share them
// out by length:
//   * short segments: a unit (a wavefront, or a workgroup) takes a whole
//     segment and keeps its rows in registers, raw, from the statistics to the
//     normalisation: one read, one write.  What does not fit in the registers
//     is read again from the caches.
//   * long segments (more than lmax rows): tiles of `tile_rows` rows, whatever
//     the segments' lengths, leave partial statistics (norm_long_stats), a
//     workgroup joins those of a segment (norm_long_join), and the tiles
//     are normalised by a second read (norm_long_apply).  tile_rows <= lmax, so
//     a tile meets at most two long segments and its partials have two fixed
//     places.
// A thread owns a chunk of V channels (16 bytes) and every slots-th row, so
// groups of any width cost nothing in the loops: sums are per channel, and
// channels are added up to groups in LDS.  Rows whose width is no multiple of V
// end with a chunk moved back to end with the row; the channels that it shares
// with the chunk before it are left out of the sums and stored twice, equal.
// Variances are taken about means: the short path holds the rows and
// subtracts the mean, the long path joins (count, mean, M2) of batches of eight
// rows by  mean = a + d nb / n,  M2 = M2a + M2b + d^2 na nb / n,  d = b - a.
#include "layers_internal.hpp"

namespace mp {
namespace {

constexpr int kLong = 256;        // threads of the long path's workgroups
constexpr int kRows = 8;          // rows that a thread has in registers
constexpr int kPad = 8;           // LDS line of a thread's v-th channel: UNIT + 8 floats,
                                  // so that consecutive channels lie on consecutive banks
constexpr int kJoin = 256;

// ---- activations ----------------------------------------------------------------------
// The standard normal distribution and density at z.  With a = |z| and t =
// 1 / (1 + 0.29 a), Q(a) = 1 - Phi(a) = exp(-a^2 / 2) t P(t): a least-maximum
// fit of degree 6 made for this file (error 8e-8 against Q, 6e-5 of Q out to
// a = 14).  The exponential serves the density too.
__device__ inline void normal(float z, float& Phi, float& e) {
    const float a = fabsf(z);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.29f, a, 1.f));
    float q = -0.0884251818060875f;
    q = __builtin_fmaf(q, t, 0.2835124135017395f);
    q = __builtin_fmaf(q, t, -0.09134544432163239f);
    q = __builtin_fmaf(q, t, 0.17835062742233276f);
    q = __builtin_fmaf(q, t, 0.10107331722974777f);
    q = __builtin_fmaf(q, t, 0.11683434993028641f);
    e = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
    q *= t * e;
    Phi = z < 0.f ? q : 1.f - q;
}

// 1 / (1 + exp(-z)); exp overflows to infinity and its reciprocal is 0.
__device__ inline float sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z));
}

template <int V>
__device__ inline void activate(float (&z)[V], int act) {
    if (act == MP_ACT_RELU) {
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = z[v] < 0.f ? 0.f : z[v];  // (keeps NaN)
    } else if (act == MP_ACT_SILU) {
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] *= sigmoid(z[v]);
    } else if (act == MP_ACT_GELU) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float Phi, e;
            normal(z[v], Phi, e);
            z[v] *= Phi;
        }
    }
}

// d <- d * act'(z)
template <int V>
__device__ inline void slope(float (&d)[V], const float (&z)[V], int act) {
    if (act == MP_ACT_RELU) {
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = z[v] > 0.f ? d[v] : 0.f;
    } else if (act == MP_ACT_SILU) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float g = sigmoid(z[v]);
            d[v] *= __builtin_fmaf(z[v] * g, 1.f - g, g);
        }
    } else if (act == MP_ACT_GELU) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float Phi, e;
            normal(z[v], Phi, e);
            d[v] *= __builtin_fmaf(0.398942280f * z[v], e, Phi);
        }
    }
}

// ---- segments ---------------------------------------------------------------------------
__device__ inline int64_t offset_of(const NormParams& P, int64_t s) {
    const int64_t v = P.rp64 ? static_cast<const int64_t*>(P.ptr)[s]
                             : (int64_t)static_cast<const int32_t*>(P.ptr)[s];
    return v < 0 ? 0 : (v > P.N ? P.N : v);
}

// The last segment that begins at or before `row`: 64 offsets a step.
__device__ inline int64_t segment_of(const NormParams& P, int64_t row) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = P.S;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        const uint64_t before = __ballot(at < hi && offset_of(P, at) <= row);
        const int n = before ? 64 - __builtin_clzll(before) : 1;
        lo += (n - 1) * step;
        if (hi > lo + step) hi = lo + step;
    }
    return lo;
}

// ---- a thread's chunk of channels ------------------------------------------------------------
// Columns [c0, c0 + W) are cut into cpr chunks of V; thread t of a unit has
// chunk t % cpr and row slot t / cpr (slots of them; threads beyond are idle).
template <int V>
struct Chunk {
    int k, slot, c, skip;  // c: first column within the tile; skip: columns of the chunk before
    bool on;
    __device__ Chunk(int t, int cpr, int slots, int W) {
        k = t % cpr;
        slot = t / cpr;
        on = slot < slots;
        const int c0 = k * V;
        c = c0 + V <= W ? c0 : W - V;
        skip = c0 - c;
    }
};

// Floats of a unit: ent[v * (UNIT + kPad) + t] is the v-th channel of thread t.
template <int V, int UNIT>
__device__ inline int place(int slot, int c, int cpr, int W) {
    const int k = c / V < cpr - 1 ? c / V : cpr - 1;
    const int v = k == cpr - 1 && cpr * V > W ? c - (W - V) : c - k * V;
    return v * (UNIT + kPad) + slot * cpr + k;
}

// For each of `groups` ranges of columns (range(g, b, e): [b, e)) the sum over
// slots and columns of get(slot, place); put(g, sum) by one thread.  lpg (a power of
// two, at most 64) neighbouring threads of the unit's UNIT share a range.
template <int V, int UNIT, typename Range, typename Get, typename Put>
__device__ inline void group_sums(int t, int lpg, int groups, int slots, int cpr, int W,
                                  Range range, Get get, Put put) {
    const int l = t & (lpg - 1), per = UNIT / lpg;
    for (int g0 = 0; g0 < groups; g0 += per) {
        const int g = g0 + t / lpg;
        float s = 0.f;
        if (g < groups) {
            int b, e;
            range(g, b, e);
            const int w = e - b, ds = lpg / w, dc = lpg - ds * w;
            int slot = l / w, c = l - slot * w;
            while (slot < slots) {
                s += get(slot, place<V, UNIT>(slot, b + c, cpr, W));
                slot += ds;
                c += dc;
                if (c >= w) {
                    c -= w;
                    ++slot;
                }
            }
        }
        for (int o = lpg >> 1; o > 0; o >>= 1) s += __shfl_xor(s, o);
        if (l == 0 && g < groups) put(g, s);
    }
}

// All threads of a unit have done what they wrote to LDS.  The LDS operations
// of one wavefront complete in order: there only the compiler is held back.
template <int UNIT>
__device__ inline void unit_sync() {
    if constexpr (UNIT == kWave) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
        __syncthreads();
    }
}

__device__ inline int rows_of_slot(int64_t n, int slot, int slots) {
    return n > slot ? (int)((n - slot + slots - 1) / slots) : 0;
}

// ---- short segments ----------------------------------------------------------------------
// blockIdx.y: a tile of whole groups (the last one moved back to end with the
// last group).  BWD: workgroup blockIdx.x leaves its sums of da xhat and da in
// line blockIdx.x of P.part.
template <typename T, int V, int UNIT, bool BWD>
__global__ __launch_bounds__(UNIT < 256 ? 256 : UNIT) void norm_short(NormParams P) {
    typedef typename T::raw raw;
    constexpr int BLOCK = UNIT < 256 ? 256 : UNIT, UNITS = BLOCK / UNIT;
    constexpr int ENT = V * (UNIT + kPad);
    extern __shared__ float s_mem[];
    const int t = threadIdx.x % UNIT, u = threadIdx.x / UNIT;
    const int cg = P.cg, gt = P.tile_groups;
    const int g0 = (int)blockIdx.y * gt <= (int)P.G - gt ? (int)blockIdx.y * gt : (int)P.G - gt;
    const int own = (int)blockIdx.y * gt * cg - g0 * cg;  // columns of the tile before
    const int W = gt * cg, cpr = P.cpr, slots = P.slots;
    const int64_t c0 = (int64_t)g0 * cg;
    float* ent = s_mem + u * ((BWD ? 2 : 1) * ENT + 2 * gt);
    float* ent2 = ent + ENT;  // (BWD)
    float* s_a = ent + (BWD ? 2 : 1) * ENT;
    float* s_b = s_a + gt;
    const Chunk<V> ck(t, cpr, slots, W);
    const auto range = [&](int g, int& b, int& e) {
        b = g * cg;
        e = b + cg;
    };

    float gamma[V], beta[V];
    int lg[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        gamma[v] = P.gamma ? P.gamma[c0 + ck.c + v] : 1.f;
        beta[v] = P.beta ? P.beta[c0 + ck.c + v] : 0.f;
        lg[v] = (ck.c + v) / cg;
    }
    float sum_g[V] = {}, sum_b[V] = {};  // BWD: over all segments of the unit

    const raw* x = static_cast<const raw*>(P.x) + c0 + ck.c;
    for (int64_t s = (int64_t)blockIdx.x * UNITS + u; s < P.S; s += (int64_t)gridDim.x * UNITS) {
        const int64_t b = offset_of(P, s), n = offset_of(P, s + 1) - b;
        if (n > P.lmax) continue;
        if (n <= 0) {
            if (!BWD)
                for (int g = t; g < gt; g += UNIT) {
                    P.mean[s * P.G + g0 + g] = 0.f;
                    P.rstd[s * P.G + g0 + g] = 0.f;
                }
            continue;
        }
        const float inv = 1.f / ((float)n * (float)cg);
        const int mine = ck.on ? rows_of_slot(n, ck.slot, slots) : 0;
        const int64_t r0 = b + ck.slot;
        RawOf<T, V> xr[kRows], dr[kRows];
        const raw* d = static_cast<const raw*>(P.dout) + c0 + ck.c;
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (i < mine) {
                const int64_t r = r0 + (int64_t)i * slots;
                xr[i] = load_raw<T, V>(x + r * P.ldx);
                if (BWD) dr[i] = load_raw<T, V>(d + r * P.F);
            }
        // every row of the thread: those in registers, then the others
        const auto each = [&](auto f) {
#pragma unroll
            for (int i = 0; i < kRows; ++i)
                if (i < mine) f(r0 + (int64_t)i * slots, xr[i], dr[i]);
            for (int i = kRows; i < mine; ++i) {
                const int64_t r = r0 + (int64_t)i * slots;
                const RawOf<T, V> a = load_raw<T, V>(x + r * P.ldx);
                RawOf<T, V> e{};
                if (BWD) e = load_raw<T, V>(d + r * P.F);
                f(r, a, e);
            }
        };
        const auto at = [&](int slot, int p) { return ent[p]; };
        if constexpr (!BWD) {
            float q[V] = {};
            each([&](int64_t, const RawOf<T, V>& a, const RawOf<T, V>&) {
                float f[V];
                to_floats<T, V>(a, f);
#pragma unroll
                for (int v = 0; v < V; ++v) q[v] += f[v];
            });
#pragma unroll
            for (int v = 0; v < V; ++v) ent[v * (UNIT + kPad) + t] = q[v];
            unit_sync<UNIT>();
            group_sums<V, UNIT>(t, P.lpg, gt, slots, cpr, W, range, at,
                                [&](int g, float sum) { s_a[g] = sum * inv; });
            unit_sync<UNIT>();
            float mean[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                mean[v] = s_a[lg[v]];
                q[v] = 0.f;
            }
            each([&](int64_t, const RawOf<T, V>& a, const RawOf<T, V>&) {
                float f[V];
                to_floats<T, V>(a, f);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float e = f[v] - mean[v];
                    q[v] = __builtin_fmaf(e, e, q[v]);
                }
            });
#pragma unroll
            for (int v = 0; v < V; ++v) ent[v * (UNIT + kPad) + t] = q[v];
            unit_sync<UNIT>();
            group_sums<V, UNIT>(t, P.lpg, gt, slots, cpr, W, range, at, [&](int g, float sum) {
                const float rs = 1.f / sqrtf(sum * inv + P.eps);
                s_b[g] = rs;
                P.mean[s * P.G + g0 + g] = s_a[g];
                P.rstd[s * P.G + g0 + g] = rs;
            });
            unit_sync<UNIT>();
            float scale[V];
#pragma unroll
            for (int v = 0; v < V; ++v) scale[v] = s_b[lg[v]] * gamma[v];
            each([&](int64_t r, const RawOf<T, V>& a, const RawOf<T, V>&) {
                float f[V];
                to_floats<T, V>(a, f);
#pragma unroll
                for (int v = 0; v < V; ++v)
                    f[v] = __builtin_fmaf(f[v] - mean[v], scale[v], beta[v]);
                activate<V>(f, P.act);
                if (P.out_bf16) store_floats<BF16, V>(static_cast<uint16_t*>(P.out) + r * P.F + c0 + ck.c, f);
                else store_floats<F32, V>(static_cast<float*>(P.out) + r * P.F + c0 + ck.c, f);
            });
        } else {
            float mean[V], rstd[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                mean[v] = P.mean[s * P.G + g0 + lg[v]];
                rstd[v] = P.rstd[s * P.G + g0 + lg[v]];
            }
            float qg[V] = {}, qb[V] = {};
            const auto grads = [&](const RawOf<T, V>& a, const RawOf<T, V>& e, float (&xh)[V],
                                   float (&da)[V]) {
                float z[V];
                to_floats<T, V>(a, xh);
                to_floats<T, V>(e, da);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    xh[v] = (xh[v] - mean[v]) * rstd[v];
                    z[v] = __builtin_fmaf(xh[v], gamma[v], beta[v]);
                }
                slope<V>(da, z, P.act);
            };
            each([&](int64_t, const RawOf<T, V>& a, const RawOf<T, V>& e) {
                float xh[V], da[V];
                grads(a, e, xh, da);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    qb[v] += da[v];
                    qg[v] = __builtin_fmaf(da[v], xh[v], qg[v]);
                }
            });
#pragma unroll
            for (int v = 0; v < V; ++v) {
                ent[v * (UNIT + kPad) + t] = gamma[v] * qb[v];
                ent2[v * (UNIT + kPad) + t] = gamma[v] * qg[v];
                sum_b[v] += qb[v];
                sum_g[v] += qg[v];
            }
            if (P.out) {
                unit_sync<UNIT>();
                group_sums<V, UNIT>(t, P.lpg, gt, slots, cpr, W, range, at,
                                    [&](int g, float sum) { s_a[g] = sum * inv; });
                group_sums<V, UNIT>(t, P.lpg, gt, slots, cpr, W, range,
                                    [&](int, int p) { return ent2[p]; },
                                    [&](int g, float sum) { s_b[g] = sum * inv; });
                unit_sync<UNIT>();
                float ca[V], cb[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    ca[v] = s_a[lg[v]];
                    cb[v] = s_b[lg[v]];
                }
                each([&](int64_t r, const RawOf<T, V>& a, const RawOf<T, V>& e) {
                    float xh[V], da[V];
                    grads(a, e, xh, da);
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        da[v] = rstd[v] * (__builtin_fmaf(gamma[v], da[v], -ca[v]) - xh[v] * cb[v]);
                    if (P.out_bf16) store_floats<BF16, V>(static_cast<uint16_t*>(P.out) + r * P.F + c0 + ck.c, da);
                    else store_floats<F32, V>(static_cast<float*>(P.out) + r * P.F + c0 + ck.c, da);
                });
            }
        }
    }
    if constexpr (BWD) {
        if (!P.part) return;
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ent[v * (UNIT + kPad) + t] = sum_g[v];
            ent2[v * (UNIT + kPad) + t] = sum_b[v];
        }
        __syncthreads();
        float* line = P.part + (int64_t)blockIdx.x * 2 * P.F + c0;
        for (int c = own + (int)threadIdx.x; c < W; c += BLOCK) {
            float a = 0.f, e = 0.f;
            for (int j = 0; j < UNITS; ++j)
                for (int i = 0; i < slots; ++i) {
                    const float* p = s_mem + j * (2 * ENT + 2 * gt) + place<V, UNIT>(i, c, cpr, W);
                    a += p[0];
                    e += p[ENT];
                }
            line[c] = a;
            line[P.F + c] = e;
        }
    }
}

// ---- long segments ---------------------------------------------------------------------
// The long segments of rows [row0, row1) in order: f(segment, first row, end,
// whether it has begun before or at row0).  At most two, as tile_rows <= lmax.
template <typename Fn>
__device__ inline void long_segments(const NormParams& P, int64_t row0, int64_t row1, Fn f) {
    const int lane = threadIdx.x & 63;
    int64_t s0 = segment_of(P, row0);
    while (s0 < P.S) {
        const int64_t s = s0 + lane;
        const int64_t b = s < P.S ? offset_of(P, s) : row1;
        const int64_t e = s < P.S ? offset_of(P, s + 1) : row1;
        uint64_t hit = __ballot(b < row1 && e > row0 && e - b > P.lmax);
        const bool more = __ballot(b >= row1) == 0;
        while (hit) {
            const int i = __builtin_ctzll(hit);
            hit &= hit - 1;
            const int64_t sb = offset_of(P, s0 + i), se = offset_of(P, s0 + i + 1);
            f(s0 + i, sb > row0 ? sb : row0, se < row1 ? se : row1, sb <= row0);
        }
        if (!more) break;
        s0 += 64;
    }
}

// Column tile blockIdx.y of the long path: kLong * V columns.
template <int V>
struct LongTile {
    int64_t c0;
    int W, cpr, slots, skip0, ga, gn;
    __device__ LongTile(const NormParams& P) {
        const int CT = kLong * V;
        const int64_t begin = (int64_t)blockIdx.y * CT;
        c0 = P.F - begin < V ? P.F - V : begin;  // (a narrow last tile moves back to a chunk's width)
        skip0 = (int)(begin - c0);
        W = (int)(P.F - c0 < CT ? P.F - c0 : CT);
        cpr = (W + V - 1) / V;
        slots = kLong / cpr;
        ga = (int)(begin / P.cg);
        gn = (int)((c0 + W - 1) / P.cg) - ga + 1;
    }
};

// Partials of rows [row0, row1) of a segment: place `seg_slot` (two a tile), then
// blockIdx.y + group: {mean, M2} or {sum gamma da, sum gamma da xhat}.
template <typename T, int V, bool BWD>
__global__ __launch_bounds__(kLong) void norm_long_stats(NormParams P) {
    typedef typename T::raw raw;
    constexpr int UNIT = kLong, ENT = V * (UNIT + kPad);
    __shared__ float ent[ENT], ent2[ENT];
    extern __shared__ float s_a[];  // [groups of a tile]
    const int t = threadIdx.x;
    const LongTile<V> lt(P);
    const Chunk<V> ck(t, lt.cpr, lt.slots, lt.W);
    const int64_t row0 = (int64_t)blockIdx.x * P.tile_rows;
    const int64_t row1 = row0 + P.tile_rows < P.N ? row0 + P.tile_rows : P.N;
    const int64_t cc = lt.c0 + ck.c;
    const auto range = [&](int g, int& b, int& e) {
        const int64_t gb = (int64_t)(lt.ga + g) * P.cg - lt.c0, ge = gb + P.cg;
        b = gb > lt.skip0 ? (int)gb : lt.skip0;
        e = ge < lt.W ? (int)ge : lt.W;
    };
    float gamma[V], beta[V];
    int lg[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        gamma[v] = P.gamma ? P.gamma[cc + v] : 1.f;
        beta[v] = P.beta ? P.beta[cc + v] : 0.f;
        lg[v] = (int)((cc + v) / P.cg);
    }
    float sum_g[V] = {}, sum_b[V] = {};
    const raw* x = static_cast<const raw*>(P.x) + cc;
    const raw* d = static_cast<const raw*>(P.dout) + cc;

    long_segments(P, row0, row1, [&](int64_t s, int64_t b, int64_t e, bool began) {
        const int64_t n = e - b;
        const int mine = ck.on ? rows_of_slot(n, ck.slot, lt.slots) : 0;
        const int64_t r0 = b + ck.slot;
        float A[V] = {}, B[V] = {};  // mean and M2, or the sums of da and da xhat
        float mean[V], rstd[V];
        if (BWD) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                mean[v] = P.mean[s * P.G + lg[v]];
                rstd[v] = P.rstd[s * P.G + lg[v]];
            }
        }
        for (int i0 = 0; i0 < mine; i0 += kRows) {
            const int nb = mine - i0 < kRows ? mine - i0 : kRows;
            RawOf<T, V> xr[kRows], dr[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                // (past the end: the last row again, weighted by nothing)
                const int64_t r = r0 + (int64_t)(i0 + (i < nb ? i : nb - 1)) * lt.slots;
                xr[i] = load_raw<T, V>(x + r * P.ldx);
                if (BWD) dr[i] = load_raw<T, V>(d + r * P.F);
            }
            if constexpr (!BWD) {
                const float fn = (float)nb, f0 = (float)i0;
                const float inb = 1.f / fn, share = fn / (f0 + fn);
                float m[V] = {}, q[V] = {};
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    float f[V];
                    to_floats<T, V>(xr[i], f);
#pragma unroll
                    for (int v = 0; v < V; ++v) m[v] += i < nb ? f[v] : 0.f;
                }
#pragma unroll
                for (int v = 0; v < V; ++v) m[v] *= inb;
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    float f[V];
                    to_floats<T, V>(xr[i], f);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float u = i < nb ? f[v] - m[v] : 0.f;
                        q[v] = __builtin_fmaf(u, u, q[v]);
                    }
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float u = m[v] - A[v];
                    A[v] = i0 ? __builtin_fmaf(u, share, A[v]) : m[v];
                    B[v] += __builtin_fmaf(u * u, f0 * share, q[v]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    if (i >= nb) break;
                    float xh[V], da[V], z[V];
                    to_floats<T, V>(xr[i], xh);
                    to_floats<T, V>(dr[i], da);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        xh[v] = (xh[v] - mean[v]) * rstd[v];
                        z[v] = __builtin_fmaf(xh[v], gamma[v], beta[v]);
                    }
                    slope<V>(da, z, P.act);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        A[v] += da[v];
                        B[v] = __builtin_fmaf(da[v], xh[v], B[v]);
                    }
                }
            }
        }
        __syncthreads();  // the segment before has been added up
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ent[v * (UNIT + kPad) + t] = BWD ? gamma[v] * A[v] : A[v];
            ent2[v * (UNIT + kPad) + t] = BWD ? gamma[v] * B[v] : B[v];
            sum_b[v] += A[v];
            sum_g[v] += B[v];
        }
        __syncthreads();
        float2* out = reinterpret_cast<float2*>(P.stats) +
                      ((int64_t)blockIdx.x * 2 + (began ? 0 : 1)) * P.stat_line + blockIdx.y + lt.ga;
        if constexpr (BWD) {
            group_sums<V, UNIT>(t, P.lpg, lt.gn, lt.slots, lt.cpr, lt.W, range,
                                [&](int, int p) { return ent[p]; },
                                [&](int g, float sum) { out[g].x = sum; });
            group_sums<V, UNIT>(t, P.lpg, lt.gn, lt.slots, lt.cpr, lt.W, range,
                                [&](int, int p) { return ent2[p]; },
                                [&](int g, float sum) { out[g].y = sum; });
        } else {
            group_sums<V, UNIT>(
                t, P.lpg, lt.gn, lt.slots, lt.cpr, lt.W, range,
                [&](int slot, int p) { return (float)rows_of_slot(n, slot, lt.slots) * ent[p]; },
                [&](int g, float sum) {
                    int gb, ge;
                    range(g, gb, ge);
                    s_a[g] = sum / ((float)n * (float)(ge - gb));
                });
            __syncthreads();
            // (the column decides the group, so its mean comes by the range)
            const int l = t & (P.lpg - 1), per = UNIT / P.lpg;
            for (int g1 = 0; g1 < lt.gn; g1 += per) {
                const int g = g1 + t / P.lpg;
                float sum = 0.f;
                if (g < lt.gn) {
                    int gb, ge;
                    range(g, gb, ge);
                    const float m = s_a[g];
                    const int w = ge - gb, ds = P.lpg / w, dc = P.lpg - ds * w;
                    int slot = l / w, c = l - slot * w;
                    while (slot < lt.slots) {
                        const int p = place<V, UNIT>(slot, gb + c, lt.cpr, lt.W);
                        const int rows = rows_of_slot(n, slot, lt.slots);
                        const float u = ent[p] - m;
                        sum += rows > 0 ? __builtin_fmaf(u * u, (float)rows, ent2[p]) : 0.f;
                        slot += ds;
                        c += dc;
                        if (c >= w) {
                            c -= w;
                            ++slot;
                        }
                    }
                }
                for (int o = P.lpg >> 1; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
                if (l == 0 && g < lt.gn) out[g] = make_float2(s_a[g], sum);
            }
        }
    });
    if constexpr (BWD) {
        if (!P.part) return;
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ent[v * (UNIT + kPad) + t] = sum_g[v];
            ent2[v * (UNIT + kPad) + t] = sum_b[v];
        }
        __syncthreads();
        float* line = P.part + ((int64_t)P.short_blocks + blockIdx.x) * 2 * P.F + lt.c0;
        for (int c = lt.skip0 + t; c < lt.W; c += UNIT) {
            float a = 0.f, e = 0.f;
            for (int i = 0; i < lt.slots; ++i) {
                const int p = place<V, UNIT>(i, c, lt.cpr, lt.W);
                a += ent[p];
                e += ent2[p];
            }
            line[c] = a;
            line[P.F + c] = e;
        }
    }
}

// The partials of every long segment joined: mean and rstd, or the means of
// gamma da and gamma da xhat (P.ca, P.cb).  A workgroup looks for its segments
// among 256 at a time; gw (a power of two) threads have neighbouring groups, and
// kJoin / gw share a group's partials.
template <bool BWD>
__global__ __launch_bounds__(kJoin) void norm_long_join(NormParams P, int gw, int64_t col_tile) {
    __shared__ float s_sum[kJoin], s_sum2[kJoin];
    __shared__ int64_t s_seg[kJoin];
    __shared__ int s_n;
    const int t = threadIdx.x, gi = t & (gw - 1), q = t / gw, Q = kJoin / gw;
    for (int64_t base = blockIdx.x; base < P.S; base += (int64_t)gridDim.x * kJoin) {
        __syncthreads();
        if (t == 0) s_n = 0;
        __syncthreads();
        const int64_t mine = base + (int64_t)t * gridDim.x;
        const int64_t rows = mine < P.S ? offset_of(P, mine + 1) - offset_of(P, mine) : 0;
        if (rows > P.lmax) s_seg[atomicAdd(&s_n, 1)] = mine;  // (any order: each is done by itself)
        if (!BWD && P.lmax == 0 && mine < P.S && rows <= 0)   // (else the short path's)
            for (int64_t g = 0; g < P.G; ++g) P.mean[mine * P.G + g] = P.rstd[mine * P.G + g] = 0.f;
        __syncthreads();
        const int found = s_n;
        for (int j = 0; j < found; ++j) {
            const int64_t s = s_seg[j], b = offset_of(P, s), e = offset_of(P, s + 1);
            const int64_t t0 = b / P.tile_rows, t1 = (e - 1) / P.tile_rows;
            for (int64_t g1 = 0; g1 < P.G; g1 += gw) {
                const int64_t g = g1 + gi;
                const bool ok = g < P.G;
                const int64_t cb = g * P.cg, ce = cb + P.cg;
                const int64_t y0 = cb / col_tile, ny = ok ? (ce - 1) / col_tile - y0 + 1 : 0;
                const int64_t parts = (t1 - t0 + 1) * ny;
                const auto each = [&](auto f) {
#pragma unroll 4
                    for (int64_t i = q; i < parts; i += Q) {
                        const int64_t tile = t0 + i / ny, y = y0 + i % ny;
                        const int64_t at = tile * 2 + (b > tile * P.tile_rows ? 1 : 0);
                        const float2 v = reinterpret_cast<const float2*>(P.stats)[at * P.stat_line + y + g];
                        const int64_t ra = tile * P.tile_rows > b ? tile * P.tile_rows : b;
                        const int64_t rb = (tile + 1) * P.tile_rows < e ? (tile + 1) * P.tile_rows : e;
                        const int64_t ca = y * col_tile > cb ? y * col_tile : cb;
                        const int64_t cz = (y + 1) * col_tile < ce ? (y + 1) * col_tile : ce;
                        f(v, (float)(rb - ra) * (float)(cz - ca));
                    }
                };
                const auto total = [&](float* s_v, float v) {
                    __syncthreads();
                    s_v[t] = v;
                    __syncthreads();
                    for (int o = Q / 2; o > 0; o >>= 1) {
                        if (q < o) s_v[t] += s_v[t + o * gw];
                        __syncthreads();
                    }
                    return s_v[gi];
                };
                const float inv = 1.f / ((float)(e - b) * (float)P.cg);
                if constexpr (BWD) {
                    float A = 0.f, B = 0.f;
                    each([&](float2 v, float) {
                        A += v.x;
                        B += v.y;
                    });
                    A = total(s_sum, A) * inv;
                    B = total(s_sum2, B) * inv;
                    if (q == 0 && ok) {
                        P.ca[s * P.G + g] = A;
                        P.cb[s * P.G + g] = B;
                    }
                } else {
                    float m = 0.f, M2 = 0.f;
                    each([&](float2 v, float n) { m = __builtin_fmaf(v.x, n, m); });
                    m = total(s_sum, m) * inv;
                    each([&](float2 v, float n) {
                        const float u = v.x - m;
                        M2 += __builtin_fmaf(u * u, n, v.y);
                    });
                    M2 = total(s_sum2, M2) * inv;
                    if (q == 0 && ok) {
                        P.mean[s * P.G + g] = m;
                        P.rstd[s * P.G + g] = 1.f / sqrtf(M2 + P.eps);
                    }
                }
            }
        }
    }
}

// The tiles again, from the last to the first (the last are still in the caches):
// out, or dx.
template <typename T, int V, bool BWD>
__global__ __launch_bounds__(kLong) void norm_long_apply(NormParams P) {
    typedef typename T::raw raw;
    const int t = threadIdx.x;
    const LongTile<V> lt(P);
    const Chunk<V> ck(t, lt.cpr, lt.slots, lt.W);
    const int64_t tile = (int64_t)gridDim.x - 1 - blockIdx.x;
    const int64_t row0 = tile * P.tile_rows;
    const int64_t row1 = row0 + P.tile_rows < P.N ? row0 + P.tile_rows : P.N;
    const int64_t cc = lt.c0 + ck.c;
    float gamma[V], beta[V];
    int lg[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        gamma[v] = P.gamma ? P.gamma[cc + v] : 1.f;
        beta[v] = P.beta ? P.beta[cc + v] : 0.f;
        lg[v] = (int)((cc + v) / P.cg);
    }
    const raw* x = static_cast<const raw*>(P.x) + cc;
    const raw* d = static_cast<const raw*>(P.dout) + cc;
    long_segments(P, row0, row1, [&](int64_t s, int64_t b, int64_t e, bool) {
        if (!ck.on) return;
        float mean[V], rstd[V], ca[V], cb[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            mean[v] = P.mean[s * P.G + lg[v]];
            rstd[v] = P.rstd[s * P.G + lg[v]];
            ca[v] = BWD ? P.ca[s * P.G + lg[v]] : 0.f;
            cb[v] = BWD ? P.cb[s * P.G + lg[v]] : 0.f;
            if (!BWD) rstd[v] *= gamma[v];
        }
#pragma unroll 4
        for (int64_t r = b + ck.slot; r < e; r += lt.slots) {
            float f[V];
            load_floats<T, V>(x + r * P.ldx, f);
            if constexpr (!BWD) {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    f[v] = __builtin_fmaf(f[v] - mean[v], rstd[v], beta[v]);
                activate<V>(f, P.act);
            } else {
                float da[V], z[V];
                load_floats<T, V>(d + r * P.F, da);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    f[v] = (f[v] - mean[v]) * rstd[v];
                    z[v] = __builtin_fmaf(f[v], gamma[v], beta[v]);
                }
                slope<V>(da, z, P.act);
#pragma unroll
                for (int v = 0; v < V; ++v)
                    f[v] = rstd[v] * (__builtin_fmaf(gamma[v], da[v], -ca[v]) - f[v] * cb[v]);
            }
            if (P.out_bf16) store_floats<BF16, V>(static_cast<uint16_t*>(P.out) + r * P.F + cc, f);
            else store_floats<F32, V>(static_cast<float*>(P.out) + r * P.F + cc, f);
        }
    });
}

// dgamma and dbeta: the lines of P.part added up in order, 64 columns a workgroup,
// a sixteenth of the lines a wavefront.
constexpr int kGradWaves = 16;
__global__ __launch_bounds__(kGradWaves * kWave) void norm_param_grads(NormParams P, int64_t lines,
                                                                       float* dgamma,
                                                                       float* dbeta) {
    __shared__ float s_sum[kGradWaves][kWave];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * kWave + lane, n = 2 * P.F;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < n) {
        int64_t i = w;
        for (; i + 7 * kGradWaves < lines; i += 8 * kGradWaves) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = P.part[(i + j * kGradWaves) * n + c];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j & 3] += v[j];
        }
        for (; i < lines; i += kGradWaves) s[0] += P.part[i * n + c];
    }
    s_sum[w][lane] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (w == 0 && c < n) {
        float r = s_sum[0][lane];
        for (int j = 1; j < kGradWaves; ++j) r += s_sum[j][lane];
        if (c < P.F) dgamma[c] = r;
        else dbeta[c - P.F] = r;
    }
}

// ---- shapes of the launches ------------------------------------------------------------
int pow2_below(int64_t v, int most) {
    int p = 1;
    while (2 * p <= v && 2 * p <= most) p *= 2;
    return p;
}

}  // namespace

// V: 16 bytes of a row, or single elements for rows narrower than that.  The
// unit is the smallest that holds a row's chunks and one and a half average
// segments in registers, else 256 threads (1024 for rows that need them).
NormShape norm_shape(int64_t N, int64_t S, int64_t F, int64_t G, int dtype, int backward) {
    NormShape h{};
    const int64_t cg = F / G;
    const int wide = dtype == MP_BF16 ? 8 : 4;
    h.V = F >= wide ? wide : 1;
    h.tile_rows = 1;
    // short path: whole groups in tiles of at most `unit` chunks
    const int64_t most = 1024 * (int64_t)h.V;
    if (cg <= most) {
        const int64_t tiles = ceil_div(G, most / cg);
        h.tile_groups = (int)ceil_div(G, tiles);
        h.tiles = (int)ceil_div(G, h.tile_groups);
        const int64_t W = h.tile_groups * cg;
        h.cpr = (int)ceil_div(W, h.V);
        h.unit = 0;
        for (int u : {64, 256}) {
            if (u < h.cpr) continue;
            if (kRows * (u / h.cpr) * S * 2 >= 3 * N) {
                h.unit = u;
                break;
            }
        }
        if (!h.unit) h.unit = h.cpr <= 256 ? 256 : 1024;
        h.slots = h.unit / h.cpr;
        h.lmax = 4 * kRows * h.slots;
        h.lpg = pow2_below(h.unit / h.tile_groups, 64);
        const int64_t units = h.unit < 256 ? 256 / h.unit : 1;
        const int64_t cap = backward ? 1024 : (int64_t(1) << 20);
        const int64_t blocks = ceil_div(S, units);
        h.short_blocks = (int)(blocks < cap ? blocks : cap);
        h.lds = (size_t)units * ((backward ? 2 : 1) * h.V * (h.unit + kPad) + 2 * h.tile_groups) * 4;
    }
    h.col_tile = kLong * (int64_t)h.V;
    if (N > h.lmax) {
        int64_t r = ceil_div(N, 2048);
        if (r < 32) r = 32;
        if (r > h.lmax) r = h.lmax > 0 ? h.lmax : 1;
        h.tile_rows = r;
        h.long_tiles = ceil_div(N, r);
        h.col_tiles = (int)ceil_div(F, h.col_tile);
        h.stat_line = h.col_tiles + G;
        // threads of a group: as many as a full column tile's groups leave
        const int64_t gn = h.col_tiles > 1 ? ceil_div(h.col_tile, cg) + 1 : G;
        h.long_lpg = pow2_below(kLong / (gn < 1 ? 1 : gn), 64);
        h.long_lds = (size_t)(gn + 1) * 4;
    }
    return h;
}

template <typename T, int V, bool BWD>
static void run(const NormParams& p, const NormShape& h, hipStream_t s) {
    NormParams q = p;
    if (h.unit) {
        q.tile_groups = h.tile_groups;
        q.cpr = h.cpr;
        q.slots = h.slots;
        q.lpg = h.lpg;
        const dim3 g((unsigned)h.short_blocks, (unsigned)h.tiles);
        if (h.unit == 64)
            hipLaunchKernelGGL((norm_short<T, V, 64, BWD>), g, dim3(256), h.lds, s, q);
        else if (h.unit == 256)
            hipLaunchKernelGGL((norm_short<T, V, 256, BWD>), g, dim3(256), h.lds, s, q);
        else
            hipLaunchKernelGGL((norm_short<T, V, 1024, BWD>), g, dim3(1024), h.lds, s, q);
    }
    if (!h.unit || h.long_tiles) {
        q.lpg = h.long_lpg;
        const dim3 g((unsigned)h.long_tiles, (unsigned)h.col_tiles);
        if (h.long_tiles)
            hipLaunchKernelGGL((norm_long_stats<T, V, BWD>), g, dim3(kLong), h.long_lds, s, q);
        if (!BWD || q.out) {
            const int gw = pow2_below(p.G, kJoin);
            const int64_t jb = p.S < 4096 ? p.S : 4096;
            hipLaunchKernelGGL((norm_long_join<BWD>), dim3((unsigned)jb), dim3(kJoin), 0, s, q, gw,
                               h.col_tile);
            if (h.long_tiles)
                hipLaunchKernelGGL((norm_long_apply<T, V, BWD>), g, dim3(kLong), 0, s, q);
        }
    }
}

hipError_t launch_norm(NormParams p, const NormShape& h, int dtype, bool backward, float* dgamma,
                       float* dbeta, hipStream_t s) {
    p.lmax = h.lmax;
    p.tile_rows = h.tile_rows;
    p.stat_line = h.stat_line;
    p.short_blocks = h.unit ? h.short_blocks : 0;
#define MP_NORM(T, V)                              \
    if (backward) run<T, V, true>(p, h, s);        \
    else run<T, V, false>(p, h, s)
    if (dtype == MP_BF16) {
        if (h.V == 8) { MP_NORM(BF16, 8); }
        else { MP_NORM(BF16, 1); }
    } else {
        if (h.V == 4) { MP_NORM(F32, 4); }
        else { MP_NORM(F32, 1); }
    }
#undef MP_NORM
    if (backward && p.part)
        hipLaunchKernelGGL(norm_param_grads, dim3((unsigned)ceil_div(2 * p.F, kWave)),
                           dim3(kGradWaves * kWave), 0, s, p, p.short_blocks + h.long_tiles, dgamma,
                           dbeta);
    return hipGetLastError();
}

}  // namespace mp
