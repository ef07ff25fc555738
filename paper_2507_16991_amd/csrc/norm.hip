// Group norm with an activation over segments of consecutive rows, channels
// last, and its gradients (include/mp_layers.h).
//
// Bound by memory (gelu also by its arithmetic), so what counts is how often
// the rows are read.  Segment lengths are on the device; two paths share them
// out by length:
//   * short segments: a unit (a wavefront, or a workgroup) takes a whole
//     segment, statistics and normalisation in one launch; the second read of
//     its rows comes from the caches.  (Rows kept in registers in between were no
//     faster; the kernels take 97 to 128 registers without that.)
//   * long segments (more than lmax rows): tiles of `tile_rows` rows, whatever
//     the segments' lengths, leave partial statistics (norm_long_stats), a
//     workgroup joins those of a segment (norm_long_join), and the tiles
//     are normalised by a second read (norm_long_apply).  The workgroups of the
//     short path leave word whether they met a long segment; these return at
//     once if none did.
// A thread owns a chunk of V = 4 channels and every slots-th row, so
// groups of any width cost nothing in the loops: sums are per channel, and
// channels are added up to groups in LDS.  Rows whose width is no multiple of V
// end with a chunk moved back to end with the row; the channels that it shares
// with the chunk before it are left out of the sums and stored twice, equal.
// Variances are taken about means: batches of a few rows are summed, then their
// squares about the batch's own mean, and (count, mean, M2) of batches joined by
// mean = a + d nb / n,  M2 = M2a + M2b + d^2 na nb / n,  d = b - a.
#include "layers_internal.hpp"

namespace mp {
namespace {

constexpr int kLong = 256;        // threads of the long path's workgroups
constexpr int kPad = 16;          // LDS line of a thread's v-th channel: UNIT + 16 floats,
                                  // so that consecutive channels lie on different banks
constexpr int kJoin = 512;

// Rows of a batch: loads that a thread has in flight.  (Eight spill 8 to 37 registers
// in the short backward of fp32, and 6 in that of bf16 where a chunk has several
// groups; fewer rows there have not been measured.)
constexpr int kShortRows = 8;
constexpr int long_rows(bool bf16, bool backward) { return bf16 || !backward ? 8 : 4; }

// ---- activations ----------------------------------------------------------------------
// The standard normal distribution and density at z.  With a = |z| and t =
// 1 / (1 + 0.29 a), Q(a) = 1 - Phi(a) = exp(-a^2 / 2) t P(t): a least-maximum
// fit of degree 6 made for this file (error 8.4e-8 against Q, 8e-5 of Q out to
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

// f(Act<act>()): the loops over rows are there once for every activation.
template <int A>
struct Act {
    static constexpr int value = A;
};
template <typename Fn>
__device__ inline void by_act(int act, Fn f) {
    if (act == MP_ACT_RELU) f(Act<MP_ACT_RELU>());
    else if (act == MP_ACT_SILU) f(Act<MP_ACT_SILU>());
    else if (act == MP_ACT_GELU) f(Act<MP_ACT_GELU>());
    else f(Act<MP_ACT_NONE>());
}

template <int V, int act>
__device__ inline void activate(float (&z)[V], Act<act>) {
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
template <int V, int act>
__device__ inline void slope(float (&d)[V], const float (&z)[V], Act<act>) {
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

// The first segment s with ptr[s] + s >= key: shares of equal rows plus segments.
__device__ inline int64_t share_begin(const NormParams& P, int64_t key) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = P.S;
    while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        const uint64_t below = __ballot(at < hi && offset_of(P, at) + at < key);
        if (!below) break;
        lo += (63 - __builtin_clzll(below)) * step + 1;
        if (hi > lo - 1 + step) hi = lo - 1 + step;
    }
    return lo;
}

// ---- a thread's chunk of channels ------------------------------------------------------------
// Columns [c0, c0 + W) are cut into cpr chunks of V; thread t of a unit has
// chunk t % cpr and row slot t / cpr (slots of them; threads beyond are idle).
template <int V>
struct Chunk {
    int slot, c;  // c: first column within the tile
    bool on;
    __device__ Chunk(int t, int cpr, int slots, int W) {
        slot = t / cpr;
        on = slot < slots;
        const int c0 = (t - slot * cpr) * V;
        c = c0 + V <= W ? c0 : W - V;
    }
};

// Floats of a unit: ent[v * (UNIT + kPad) + t] is the v-th channel of thread t.
template <int V, int UNIT>
__device__ inline int place(int slot, int c, int cpr, int W) {
    const int k = c / V < cpr - 1 ? c / V : cpr - 1;
    const int v = k == cpr - 1 && cpr * V > W ? c - (W - V) : c - k * V;
    return v * (UNIT + kPad) + slot * cpr + k;
}

// The groups of a chunk's channels: that of the first, and a bit for every channel
// that begins a new one.
template <int V>
struct Groups {
    int first;
    uint32_t next;
    __device__ Groups(int64_t c, int cg) {
        first = (int)(c / cg);
        next = 0;
        int left = (int)((int64_t)(first + 1) * cg - c);  // channels to the next group
#pragma unroll
        for (int v = 1; v < V; ++v)
            if (v == left) {
                next |= 1u << v;
                left += cg;
            }
    }
    __device__ int of(int v) const { return first + __popc(next & ((2u << v) - 1)); }
};

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

// 2^-floor(log2 c) and its inverse, for c >= 1: the squares of c values are added up
// times the first, so that their sum is finite where the variance is.  Products
// by them are exact, and the bits are those of the plain sum.
__device__ inline float down_of(float c) {
    return __uint_as_float((254u << 23) - (__float_as_uint(c) & 0x7F800000u));
}
__device__ inline float up_of(float c) { return __uint_as_float(__float_as_uint(c) & 0x7F800000u); }

__device__ inline int rows_of_slot(int64_t n, int slot, int slots) {
    return n > slot ? (int)((n - slot + slots - 1) / slots) : 0;
}

// ---- a thread's rows -------------------------------------------------------------------------
// `mine` rows from x (and d), step_x (step_f) elements apart.
template <typename T>
struct Rows {
    const typename T::raw* x;
    const typename T::raw* d;
    int64_t step_x, step_f;
    int mine;
};

// A thread's parameters for its V channels; M = 1 where they lie in one group, else V.
template <int V, int M>
struct Param {
    float gamma[V], beta[V], mean[M], rstd[M];
};

// xhat and da of one row.
template <typename T, int V, int M, typename A>
__device__ inline void grads(A act, const Param<V, M>& p, const RawOf<T, V>& a,
                             const RawOf<T, V>& e, float (&xh)[V], float (&da)[V]) {
    float z[V];
    to_floats<T, V>(a, xh);
    to_floats<T, V>(e, da);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        xh[v] = (xh[v] - p.mean[v % M]) * p.rstd[v % M];
        z[v] = __builtin_fmaf(xh[v], p.gamma[v], p.beta[v]);
    }
    slope<V>(da, z, act);
}

// Statistics of the thread's rows, R loads in flight.  Forward: A and B the mean
// and M2 of each channel; backward: the sums of da and da xhat.
template <typename T, int V, int M, int R, bool BWD>
__device__ inline void row_stats(const Rows<T>& rows, const Param<V, M>& p, int act, float (&A)[V],
                                 float (&B)[V]) {
    const auto loop = [&](auto act) {
        const typename T::raw* px = rows.x;
        const typename T::raw* pd = rows.d;
        for (int i0 = 0; i0 < rows.mine; i0 += R) {
            const int nb = rows.mine - i0 < R ? rows.mine - i0 : R;
            RawOf<T, V> xr[R], dr[R];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                // (past the end: the last row again, weighted by nothing)
                xr[i] = load_raw<T, V>(px);
                if (BWD) dr[i] = load_raw<T, V>(pd);
                const bool on = i0 + i + 1 < rows.mine;
                px += on ? rows.step_x : 0;
                pd += on ? rows.step_f : 0;
            }
            if constexpr (!BWD) {
                const float fn = (float)nb, f0 = (float)i0;
                const float share = fn * __builtin_amdgcn_rcpf(f0 + fn);
                float m[V] = {}, q[V] = {};
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    float f[V];
                    to_floats<T, V>(xr[i], f);
#pragma unroll
                    for (int v = 0; v < V; ++v) m[v] += i < nb ? f[v] : 0.f;
                }
#pragma unroll
                for (int v = 0; v < V; ++v)  // (a quotient: the mean is exact where the sum is)
                    m[v] = nb == R ? m[v] * (1.f / R) : m[v] / fn;
#pragma unroll
                for (int i = 0; i < R; ++i) {
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
                    // (the first batch is not joined: u is its mean, whose square may be
                    // infinite, times 0)
                    const float u = i0 ? m[v] - A[v] : 0.f;
                    A[v] = i0 ? __builtin_fmaf(u, share, A[v]) : m[v];
                    B[v] += __builtin_fmaf(u * u, f0 * share, q[v]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    if (i >= nb) break;
                    float xh[V], da[V];
                    grads<T>(act, p, xr[i], dr[i], xh, da);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        A[v] += da[v];
                        B[v] = __builtin_fmaf(da[v], xh[v], B[v]);
                    }
                }
            }
        }
    };
    if constexpr (BWD) by_act(act, loop);
    else loop(Act<MP_ACT_NONE>());
}

// The thread's rows of out (p.rstd times gamma in p.gamma), or of dx.  o: the first
// one's element.
template <typename T, int V, int M, int R, bool BWD>
__device__ inline void row_apply(const Rows<T>& rows, const Param<V, M>& p, const float (&ca)[M],
                                 const float (&cb)[M], int act, void* out, int out_bf16,
                                 int64_t o) {
    by_act(act, [&](auto act) {
        const typename T::raw* px = rows.x;
        const typename T::raw* pd = rows.d;
        for (int i0 = 0; i0 < rows.mine; i0 += R) {
            RawOf<T, V> xr[R], dr[R];
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (i0 + i < rows.mine) {
                    xr[i] = load_raw<T, V>(px);
                    px += rows.step_x;
                    if (BWD) {
                        dr[i] = load_raw<T, V>(pd);
                        pd += rows.step_f;
                    }
                }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                if (i0 + i >= rows.mine) break;
                float f[V];
                if constexpr (!BWD) {
                    to_floats<T, V>(xr[i], f);
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        f[v] = __builtin_fmaf(f[v] - p.mean[v % M], p.gamma[v], p.beta[v]);
                    activate<V>(f, act);
                } else {
                    float xh[V];
                    grads<T>(act, p, xr[i], dr[i], xh, f);
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        f[v] = p.rstd[v % M] *
                               (__builtin_fmaf(p.gamma[v], f[v], -ca[v % M]) - xh[v] * cb[v % M]);
                }
                if (out_bf16) store_floats<BF16, V>(static_cast<uint16_t*>(out) + o, f);
                else store_floats<F32, V>(static_cast<float*>(out) + o, f);
                o += rows.step_f;
            }
        }
    });
}

// Threads of a workgroup of the short path: four wavefronts that are units, or
// one unit.
constexpr int short_block(int unit) { return unit == 64 ? 256 : unit; }

// ---- short segments ----------------------------------------------------------------------
// blockIdx.y: a tile of whole groups (the last one moved back to end with the
// last group).  BWD: workgroup blockIdx.x leaves its sums of da xhat and da in
// line blockIdx.x of P.part.
//
// Units have shares of neighbouring segments, equal by rows and segments together
// (in turn by number, units that met several long ones took twice the average).
//
// WHOLE: a chunk lies within one group (F / G a multiple of V), so a thread has one
// mean and leaves one entry in LDS instead of V.
//
// 190k rows of 128 bf16 channels in 8192 segments, relu: forward 48 us, backward 59
// us, bound by the instructions and latencies of segments of 23 rows (2.0 and 2.5
// TB/s).  Wavefronts as units, with twice the rows a thread: 51 and 88 us.
template <typename T, int V, int UNIT, bool BWD, bool WHOLE>
__global__ __launch_bounds__(short_block(UNIT), 4) void norm_short(NormParams P) {
    typedef typename T::raw raw;
    constexpr int BLOCK = short_block(UNIT), UNITS = BLOCK / UNIT;
    constexpr int ENT = V * (UNIT + kPad);
    constexpr int M = WHOLE ? 1 : V;  // means of a thread
    extern __shared__ float s_mem[];
    const int t = threadIdx.x % UNIT, u = threadIdx.x / UNIT;
    const int cg = P.cg, gt = P.tile_groups;
    const int g0 = (int)blockIdx.y * gt <= (int)P.G - gt ? (int)blockIdx.y * gt : (int)P.G - gt;
    const int own = (int)blockIdx.y * gt * cg - g0 * cg;  // columns of the tile before
    const int W = gt * cg, cpr = P.cpr, slots = P.slots;
    const int64_t c0 = (int64_t)g0 * cg;
    float* ent = s_mem + u * (2 * ENT + 2 * gt);  // means, or sums of gamma da
    float* ent2 = ent + ENT;                      // M2, or sums of gamma da xhat
    float* s_a = ent2 + ENT;
    float* s_b = s_a + gt;
    const Chunk<V> ck(t, cpr, slots, W);
    const Groups<V> lg(ck.c, cg);
    // WHOLE: the entries of a group are its cpg chunks of every slot, lpg threads
    // to them
    const int cpg = WHOLE ? cg / V : 1, l = t & (P.lpg - 1);
    const int e_slot = l / cpg, e_k = l - e_slot * cpg, d_slot = P.lpg / cpg, d_k = P.lpg - d_slot * cpg;
    // f(slot, place of an entry) for the thread's share of group g's entries
    const auto entries = [&](int g, auto f) {
        if constexpr (WHOLE) {
            int i = e_slot, k = e_k;
            while (i < slots) {
                f(i, i * cpr + g * cpg + k);
                i += d_slot;
                k += d_k;
                if (k >= cpg) {
                    k -= cpg;
                    ++i;
                }
            }
        } else {
            int i = l / cg, c = l - i * cg;
            const int di = P.lpg / cg, dc = P.lpg - di * cg;
            while (i < slots) {
                f(i, place<V, UNIT>(i, g * cg + c, cpr, W));
                i += di;
                c += dc;
                if (c >= cg) {
                    c -= cg;
                    ++i;
                }
            }
        }
    };
    const auto over_threads = [&](float a) {
        for (int o = P.lpg >> 1; o > 0; o >>= 1) a += __shfl_xor(a, o);
        return a;
    };

    Param<V, M> p;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        p.gamma[v] = P.gamma ? P.gamma[c0 + ck.c + v] : 1.f;
        p.beta[v] = P.beta ? P.beta[c0 + ck.c + v] : 0.f;
    }
    float sum_g[V] = {}, sum_b[V] = {};  // BWD: over all segments of the unit
    int seen = 0;                        // a long segment

    Rows<T> rows;
    rows.step_x = (int64_t)slots * P.ldx;
    rows.step_f = (int64_t)slots * P.F;
    const raw* x = static_cast<const raw*>(P.x) + c0 + ck.c;
    const raw* d = static_cast<const raw*>(P.dout) + c0 + ck.c;
    const int64_t unit = (int64_t)blockIdx.x * UNITS + u, units = (int64_t)gridDim.x * UNITS;
    const int64_t first = share_begin(P, (P.N + P.S) * unit / units);
    const int64_t last = unit + 1 < units ? share_begin(P, (P.N + P.S) * (unit + 1) / units) : P.S;
    int64_t next = first < last ? offset_of(P, first) : 0;
    for (int64_t s = first; s < last; ++s) {
        const int64_t b = next;
        next = offset_of(P, s + 1);
        const int64_t n64 = next - b;
        if (n64 > P.lmax) {
            seen = 1;
            continue;
        }
        if (n64 <= 0) {
            if (!BWD)
                for (int g = t; g < gt; g += UNIT) {
                    P.mean[s * P.G + g0 + g] = 0.f;
                    P.rstd[s * P.G + g0 + g] = 0.f;
                }
            continue;
        }
        const int n = (int)n64;
        const float count = (float)n * (float)cg, inv = 1.f / count, down = down_of(count);
        rows.mine = ck.on ? rows_of_slot(n, ck.slot, slots) : 0;
        const int64_t r0 = rows.mine ? b + ck.slot : b;
        rows.x = x + r0 * P.ldx;
        rows.d = d + r0 * P.F;
        const int64_t o0 = r0 * P.F + c0 + ck.c;
        float A[V] = {}, B[V] = {};
        if constexpr (BWD) {
#pragma unroll
            for (int m = 0; m < M; ++m) {
                p.mean[m] = P.mean[s * P.G + g0 + lg.of(m)];
                p.rstd[m] = P.rstd[s * P.G + g0 + lg.of(m)];
            }
        }
        row_stats<T, V, M, kShortRows, BWD>(rows, p, P.act, A, B);
        if constexpr (BWD) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                sum_b[v] += A[v];
                sum_g[v] += B[v];
                A[v] *= p.gamma[v];
                B[v] *= p.gamma[v];
            }
            if (!P.out) continue;
        }
        if constexpr (WHOLE) {
            float a = A[0], e = B[0];
#pragma unroll
            for (int v = 1; v < V; ++v) {
                a += A[v];
                e += B[v];
            }
            if (!BWD) {  // one mean of the chunk's channels, and M2 about it
                a *= 1.f / V;
                float q = 0.f;
#pragma unroll
                for (int v = 0; v < V; ++v) q = __builtin_fmaf(A[v] - a, A[v] - a, q);
                e = __builtin_fmaf(q, (float)rows.mine, e);
            }
            ent[t] = a;
            ent2[t] = e;
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                ent[v * (UNIT + kPad) + t] = A[v];
                ent2[v * (UNIT + kPad) + t] = B[v];
            }
        }
        unit_sync<UNIT>();
        for (int gb = 0; gb < gt; gb += UNIT / P.lpg) {
            const int g = gb + t / P.lpg;
            const bool on = g < gt;
            float a = 0.f, e = 0.f;
            if constexpr (BWD) {
                if (on)
                    entries(g, [&](int, int at) {
                        a += ent[at];
                        e += ent2[at];
                    });
                a = over_threads(a) * inv;
                e = over_threads(e) * inv;
                if (on && l == 0) {
                    s_a[g] = a;
                    s_b[g] = e;
                }
            } else {
                constexpr float width = WHOLE ? V : 1;  // channels of an entry
                if (on)
                    entries(g, [&](int i, int at) {
                        a = __builtin_fmaf(width * (float)rows_of_slot(n, i, slots), ent[at], a);
                    });
                a = over_threads(a) / count;
                if (on)
                    entries(g, [&](int i, int at) {
                        const int r = rows_of_slot(n, i, slots);
                        const float q = ent[at] - a;
                        e += r > 0 ? __builtin_fmaf(q * q, width * down * (float)r, ent2[at] * down) : 0.f;
                    });
                e = over_threads(e) * (inv * up_of(count));
                if (on && l == 0) {
                    const float rs = 1.f / sqrtf(e + P.eps);
                    s_a[g] = a;
                    s_b[g] = rs;
                    P.mean[s * P.G + g0 + g] = a;
                    P.rstd[s * P.G + g0 + g] = rs;
                }
            }
        }
        unit_sync<UNIT>();
        float ca[M], cb[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            ca[m] = s_a[lg.of(m)];
            cb[m] = s_b[lg.of(m)];
        }
        if constexpr (BWD) {
            row_apply<T, V, M, kShortRows, true>(rows, p, ca, cb, P.act, P.out, P.out_bf16, o0);
        } else {
            Param<V, M> w = p;
#pragma unroll
            for (int m = 0; m < M; ++m) w.mean[m] = ca[m];
#pragma unroll
            for (int v = 0; v < V; ++v) w.gamma[v] *= cb[v % M];
            row_apply<T, V, M, kShortRows, false>(rows, w, ca, cb, P.act, P.out, P.out_bf16, o0);
        }
    }
    if (P.flags) {
        const int any = __syncthreads_or(seen);
        if (threadIdx.x == 0 && blockIdx.y == 0) P.flags[blockIdx.x] = any;
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
                    const float* q = s_mem + j * (2 * ENT + 2 * gt) + place<V, UNIT>(i, c, cpr, W);
                    a += q[0];
                    e += q[ENT];
                }
            line[c] = a;
            line[P.F + c] = e;
        }
    }
}

// ---- long segments ---------------------------------------------------------------------
// Whether a workgroup of the short path has met a long segment; uniform.
__device__ inline bool any_long(const NormParams& P) {
    if (!P.flags) return true;
    int any = 0;
    for (int i = threadIdx.x; i < P.short_blocks; i += blockDim.x) any |= P.flags[i];
    return __syncthreads_or(any) != 0;
}

// Where the partials of a long segment that begins at row b lie among those of
// the tile at row0: one that has begun has the first place, and the beginnings
// of others lie more than lmax rows apart.
__device__ inline int64_t place_of(const NormParams& P, int64_t b, int64_t row0) {
    return b <= row0 ? 0 : 1 + (b - row0) / (P.lmax + 1);
}

// The long segments of rows [row0, row1) in order: f(segment, first row, end,
// place of its partials).
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
            f(s0 + i, sb > row0 ? sb : row0, se < row1 ? se : row1, place_of(P, sb, row0));
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

// Partials of rows [row0, row1) of a segment: its place among the tile's, then
// blockIdx.y + group: {mean, M2 times down_of(its values)} or {sum gamma da, sum gamma
// da xhat}.  (2.4M x 100
// bf16: forward 125 us, 3.9 TB/s; backward with gelu 318 us, of which its slope's
// vector instructions are about half.)
template <typename T, int V, bool BWD>
__global__ __launch_bounds__(kLong, 4) void norm_long_stats(NormParams P) {
    typedef typename T::raw raw;
    constexpr int UNIT = kLong, ENT = V * (UNIT + kPad);
    __shared__ float ent[ENT], ent2[ENT];
    extern __shared__ float s_a[];  // [groups of a tile]
    const int t = threadIdx.x;
    if (!any_long(P)) return;
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
    Param<V, V> p;
    const Groups<V> lg(cc, P.cg);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        p.gamma[v] = P.gamma ? P.gamma[cc + v] : 1.f;
        p.beta[v] = P.beta ? P.beta[cc + v] : 0.f;
    }
    float sum_g[V] = {}, sum_b[V] = {};
    const raw* x = static_cast<const raw*>(P.x) + cc;
    const raw* d = static_cast<const raw*>(P.dout) + cc;

    long_segments(P, row0, row1, [&](int64_t s, int64_t b, int64_t e, int64_t nth) {
        const int64_t n = e - b;
        Rows<T> rows;
        rows.mine = ck.on ? rows_of_slot(n, ck.slot, lt.slots) : 0;
        const int64_t r0 = rows.mine ? b + ck.slot : b;
        rows.x = x + r0 * P.ldx;
        rows.d = d + r0 * P.F;
        rows.step_x = lt.slots * P.ldx;
        rows.step_f = lt.slots * P.F;
        float A[V] = {}, B[V] = {};
        if (BWD) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                p.mean[v] = P.mean[s * P.G + lg.of(v)];
                p.rstd[v] = P.rstd[s * P.G + lg.of(v)];
            }
        }
        row_stats<T, V, V, long_rows(sizeof(raw) == 2, BWD), BWD>(rows, p, P.act, A, B);
        __syncthreads();  // the segment before has been added up
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ent[v * (UNIT + kPad) + t] = BWD ? p.gamma[v] * A[v] : A[v];
            ent2[v * (UNIT + kPad) + t] = BWD ? p.gamma[v] * B[v] : B[v];
            sum_b[v] += A[v];
            sum_g[v] += B[v];
        }
        __syncthreads();
        float2* out = reinterpret_cast<float2*>(P.stats) +
                      ((int64_t)blockIdx.x * P.places + nth) * P.stat_line + blockIdx.y + lt.ga;
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
                    const float m = s_a[g], down = down_of((float)n * (float)(ge - gb));
                    const int w = ge - gb, ds = P.lpg / w, dc = P.lpg - ds * w;
                    int slot = l / w, c = l - slot * w;
                    while (slot < lt.slots) {
                        const int p = place<V, UNIT>(slot, gb + c, lt.cpr, lt.W);
                        const int rows = rows_of_slot(n, slot, lt.slots);
                        const float u = ent[p] - m;
                        sum += rows > 0 ? __builtin_fmaf(u * u, down * (float)rows, ent2[p] * down) : 0.f;
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
// among 512 at a time; gw (a power of two, at most 64) threads have neighbouring
// groups, and kJoin / gw share a group's partials.
template <bool BWD>
__global__ __launch_bounds__(kJoin) void norm_long_join(NormParams P, int gw, int64_t col_tile) {
    __shared__ float s_sum[kJoin / kWave][kWave];
    __shared__ int64_t s_seg[kJoin];
    __shared__ int s_n;
    const int t = threadIdx.x, gi = t & (gw - 1), q = t / gw, Q = kJoin / gw;
    if (!any_long(P)) return;
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
                const int64_t y0 = cb / col_tile;
                const int ny = ok ? (int)((ce - 1) / col_tile - y0) + 1 : 0;
                const int parts = (int)(t1 - t0 + 1) * ny;
                // (only in its first tile can a segment have another place than 0)
                const int64_t at0 = t0 * P.places + place_of(P, b, t0 * P.tile_rows);
                const auto each = [&](auto f) {
#pragma unroll 8
                    for (int i = q; i < parts; i += Q) {
                        const int dt = ny == 1 ? i : i / ny;
                        const int64_t tile = t0 + dt, y = y0 + (i - dt * ny);
                        const int64_t at = dt ? tile * P.places : at0;
                        const float2 v = reinterpret_cast<const float2*>(P.stats)[at * P.stat_line + y + g];
                        const int64_t ra = dt ? tile * P.tile_rows : b;
                        const int64_t rb = (tile + 1) * P.tile_rows < e ? (tile + 1) * P.tile_rows : e;
                        const int64_t ca = y * col_tile > cb ? y * col_tile : cb;
                        const int64_t cz = (y + 1) * col_tile < ce ? (y + 1) * col_tile : ce;
                        f(v, (float)(int)(rb - ra) * (float)(int)(cz - ca));
                    }
                };
                // over the threads of a group: lanes gw apart, then the wavefronts in order
                const auto total = [&](float v) {
                    for (int o = kWave / 2; o >= gw; o >>= 1) v += __shfl_xor(v, o);
                    __syncthreads();
                    if ((t & 63) < gw) s_sum[t >> 6][gi] = v;
                    __syncthreads();
                    float r = s_sum[0][gi];
                    for (int w = 1; w < kJoin / kWave; ++w) r += s_sum[w][gi];
                    return r;
                };
                const float count = (float)(e - b) * (float)P.cg, inv = 1.f / count;
                if constexpr (BWD) {
                    float A = 0.f, B = 0.f;
                    each([&](float2 v, float) {
                        A += v.x;
                        B += v.y;
                    });
                    A = total(A) * inv;
                    B = total(B) * inv;
                    if (q == 0 && ok) {
                        P.ca[s * P.G + g] = A;
                        P.cb[s * P.G + g] = B;
                    }
                } else {
                    float m = 0.f, M2 = 0.f;
                    each([&](float2 v, float n) { m = __builtin_fmaf(v.x, n, m); });
                    m = total(m) / count;
                    const float down = down_of(count);
                    each([&](float2 v, float n) {
                        const float u = v.x - m;
                        M2 += __builtin_fmaf(u * u, n * down, v.y * (up_of(n) * down));
                    });
                    M2 = total(M2) * (inv * up_of(count));
                    if (q == 0 && ok) {
                        P.mean[s * P.G + g] = m;
                        P.rstd[s * P.G + g] = 1.f / sqrtf(M2 + P.eps);
                    }
                }
            }
        }
    }
}

// The long segments' rows again, in tiles of apply_rows from the last to the first (the
// last rows are still in the caches): out, or dx.  Bound by memory, gelu also by its
// arithmetic (2.4M x 100 bf16: forward 192 us, 5.1 TB/s; backward with gelu 291 us).
template <typename T, int V, bool BWD>
__global__ __launch_bounds__(kLong, 4) void norm_long_apply(NormParams P) {
    typedef typename T::raw raw;
    const int t = threadIdx.x;
    if (!any_long(P)) return;
    const LongTile<V> lt(P);
    const Chunk<V> ck(t, lt.cpr, lt.slots, lt.W);
    const int64_t tile = (int64_t)gridDim.x - 1 - blockIdx.x;
    const int64_t row0 = tile * P.apply_rows;
    const int64_t row1 = row0 + P.apply_rows < P.N ? row0 + P.apply_rows : P.N;
    const int64_t cc = lt.c0 + ck.c;
    const Groups<V> lg(cc, P.cg);
    const raw* x = static_cast<const raw*>(P.x) + cc;
    const raw* d = static_cast<const raw*>(P.dout) + cc;
    long_segments(P, row0, row1, [&](int64_t s, int64_t b, int64_t e, int64_t) {
        Rows<T> rows;
        rows.mine = ck.on ? rows_of_slot(e - b, ck.slot, lt.slots) : 0;
        if (!rows.mine) return;
        const int64_t r0 = b + ck.slot;
        rows.x = x + r0 * P.ldx;
        rows.d = d + r0 * P.F;
        rows.step_x = lt.slots * P.ldx;
        rows.step_f = lt.slots * P.F;
        Param<V, V> p;
        float ca[V], cb[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t g = s * P.G + lg.of(v);
            p.gamma[v] = P.gamma ? P.gamma[cc + v] : 1.f;
            p.beta[v] = P.beta ? P.beta[cc + v] : 0.f;
            p.mean[v] = P.mean[g];
            p.rstd[v] = P.rstd[g];
            ca[v] = BWD ? P.ca[g] : 0.f;
            cb[v] = BWD ? P.cb[g] : 0.f;
            if (!BWD) p.gamma[v] *= p.rstd[v];
        }
        row_apply<T, V, V, long_rows(sizeof(raw) == 2, BWD), BWD>(rows, p, ca, cb, P.act, P.out,
                                                                  P.out_bf16, r0 * P.F + cc);
    });
}

// dgamma and dbeta: the lines of P.part added up in order (those of the tiles only
// if there are long segments).  Bound by the latency of its loads: a workgroup
// has 16 columns, a lane every 64th line of one, eight loads in flight.
constexpr int kGradBlock = 1024, kGradCols = 16, kGradRows = kGradBlock / kGradCols;
__global__ __launch_bounds__(kGradBlock) void norm_param_grads(NormParams P, int64_t long_tiles,
                                                               float* dgamma, float* dbeta) {
    __shared__ float s_sum[kGradRows][kGradCols];
    const int64_t lines = P.short_blocks + (long_tiles && any_long(P) ? long_tiles : 0);
    const int col = threadIdx.x % kGradCols, w = threadIdx.x / kGradCols;
    const int64_t c = (int64_t)blockIdx.x * kGradCols + col, n = 2 * P.F;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < n) {
        for (int64_t i = w; i < lines; i += 8 * kGradRows) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = i + j * kGradRows < lines ? P.part[(i + j * kGradRows) * n + c] : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j & 3] += v[j];
        }
    }
    s_sum[w][col] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    for (int o = kGradRows / 2; o > 0; o >>= 1) {
        if (w < o) s_sum[w][col] += s_sum[w + o][col];
        __syncthreads();
    }
    if (w == 0 && c < n) {
        if (c < P.F) dgamma[c] = s_sum[0][col];
        else dbeta[c - P.F] = s_sum[0][col];
    }
}

// ---- shapes of the launches ------------------------------------------------------------
int pow2_below(int64_t v, int most) {
    int p = 1;
    while (2 * p <= v && 2 * p <= most) p *= 2;
    return p;
}

}  // namespace

// V: 4 channels, or 1 for rows narrower than that.  The
// unit is the smallest that holds a row's chunks and eight rows a
// thread of an average segment, else 256 threads (1024 for rows that need them).
NormShape norm_shape(int64_t N, int64_t S, int64_t F, int64_t G, int dtype, int backward) {
    NormShape h{};
    const int64_t cg = F / G;
    h.V = F >= 4 ? 4 : 1;
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
        for (int u : {64, 128, 256}) {
            if (u < h.cpr) continue;
            if (8 * (u / h.cpr) * S >= N) {
                h.unit = u;
                break;
            }
        }
        if (!h.unit) h.unit = h.cpr <= 256 ? 256 : 1024;
        h.slots = h.unit / h.cpr;
        // Many segments: up to 128 KB of one are its unit's.  Few: at most eight rows of
        // a thread, as longer ones have more of the chip in tiles.  (1M x 64 bf16, forward,
        // by a unit against by tiles: 4,096 segments 74 and 126 us if even, 124 and 166 if
        // ragged; 16,384 ragged 109 and 227.  Below, units have even segments faster, 73
        // and 102 for 1,024, but ragged ones slower: 127 and 126, backward 243 and 202;
        // 64 of them 124 and 99.  128 channels, 4,096 ragged: 216 and 238, backward 394
        // and 365.)
        h.lmax = 8 * (int64_t)h.slots;
        // A call of 64 KB in all has no long ones: one launch instead of four.  (64 KB of 64
        // bf16 channels: 15 us against 21 for one segment and 25 for two.  At 128 KB it is
        // 18 and 21, but backward 28 and 26; at 256 KB 30 and 21.)
        const int64_t bytes = W * (dtype == MP_BF16 ? 2 : 4);
        const int64_t rows = S >= 4096 ? (128 << 10) / bytes : (N * bytes <= (64 << 10) ? N : 0);
        h.lmax = rows > h.lmax ? rows : h.lmax;
        h.lpg = pow2_below(h.unit / h.tile_groups, 64);
        const int64_t units = short_block(h.unit) / h.unit;
        const int64_t cap = 2048;
        const int64_t blocks = ceil_div(S, units);
        h.short_blocks = (int)(blocks < cap ? blocks : cap);
        h.lds = (size_t)units * (2 * h.V * (h.unit + kPad) + 2 * h.tile_groups) * 4;
    }
    h.col_tile = kLong * (int64_t)h.V;
    if (S == 1 && N > h.lmax) h.unit = h.short_blocks = 0;  // (the host knows its length)
    if (N > h.lmax) {
        // Tiles of the statistics: 4096 (2048 leave the forward's last round of workgroups
        // half empty), 2048 backward (two rounds of what the chip holds; half the partials
        // and lines to add: 329 -> 315 us for 2.4M x 100); 8192 for the second read; and
        // of 32 KB at the least (4 KB where the average segment is a long one and the
        // tiles have all the work).
        const int64_t least =
            ceil_div(N > S * h.lmax ? 4 << 10 : 32 << 10, F * (dtype == MP_BF16 ? 2 : 4));
        int64_t r = ceil_div(N, backward ? 2048 : 4096);
        if (r < least) r = least;
        h.tile_rows = r;
        h.apply_rows = ceil_div(N, 8192) < least ? least : ceil_div(N, 8192);
        h.places = 2 + (r - 1) / (h.lmax + 1);
        h.long_tiles = ceil_div(N, r);
        h.col_tiles = (int)ceil_div(F, h.col_tile);
        h.stat_line = h.col_tiles + G;
        // threads of a group: as many as a full column tile's groups leave
        const int64_t gn = h.col_tiles > 1 ? ceil_div(h.col_tile, cg) + 1 : G;
        h.long_lpg = pow2_below(kLong / gn, 64);
        h.long_lds = (size_t)(gn + 1) * 4;
    }
    return h;
}

template <typename T, int V, bool BWD, bool WHOLE>
static void short_path(const NormParams& q, const NormShape& h, dim3 g, hipStream_t s) {
    if (h.unit == 64)
        hipLaunchKernelGGL((norm_short<T, V, 64, BWD, WHOLE>), g, dim3(256), h.lds, s, q);
    else if (h.unit == 128)
        hipLaunchKernelGGL((norm_short<T, V, 128, BWD, WHOLE>), g, dim3(128), h.lds, s, q);
    else if (h.unit == 256)
        hipLaunchKernelGGL((norm_short<T, V, 256, BWD, WHOLE>), g, dim3(256), h.lds, s, q);
    else if constexpr (V > 1)  // (rows of one chunk a channel are narrow)
        hipLaunchKernelGGL((norm_short<T, V, 1024, BWD, WHOLE>), g, dim3(1024), h.lds, s, q);
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
        // (of a width that is a multiple of V no chunk is moved back)
        const bool whole = V > 1 && p.cg % V == 0;
        if constexpr (V > 1)
            if (whole) short_path<T, V, BWD, true>(q, h, g, s);
        if (!whole) short_path<T, V, BWD, false>(q, h, g, s);
    }
    if (!h.unit || h.long_tiles) {
        q.lpg = h.long_lpg;
        const dim3 g((unsigned)h.long_tiles, (unsigned)h.col_tiles);
        if (h.long_tiles)
            hipLaunchKernelGGL((norm_long_stats<T, V, BWD>), g, dim3(kLong), h.long_lds, s, q);
        if (!BWD || q.out) {
            const int gw = pow2_below(p.G, kWave);
            const int64_t jb = p.S < 1024 ? p.S : 1024;
            hipLaunchKernelGGL((norm_long_join<BWD>), dim3((unsigned)jb), dim3(kJoin), 0, s, q, gw,
                               h.col_tile);
            if (h.long_tiles)
                hipLaunchKernelGGL((norm_long_apply<T, V, BWD>),
                                   dim3((unsigned)ceil_div(p.N, h.apply_rows), (unsigned)h.col_tiles),
                                   dim3(kLong), 0, s, q);
        }
    }
}

hipError_t launch_norm(NormParams p, const NormShape& h, int dtype, bool backward, float* dgamma,
                       float* dbeta, hipStream_t s) {
    p.lmax = h.lmax;
    p.tile_rows = h.tile_rows;
    p.stat_line = h.stat_line;
    p.places = h.places;
    p.apply_rows = h.apply_rows;
    if (!h.unit || !h.long_tiles) p.flags = nullptr;
    p.short_blocks = h.unit ? h.short_blocks : 0;
#define MP_NORM(T, V)                              \
    if (backward) run<T, V, true>(p, h, s);        \
    else run<T, V, false>(p, h, s)
    if (dtype == MP_BF16) {
        if (h.V == 4) { MP_NORM(BF16, 4); }
        else { MP_NORM(BF16, 1); }
    } else {
        if (h.V == 4) { MP_NORM(F32, 4); }
        else { MP_NORM(F32, 1); }
    }
#undef MP_NORM
    // (a call without rows may need no workspace, so p.part does not say: zeros are written)
    if (backward && dgamma)
        hipLaunchKernelGGL(norm_param_grads, dim3((unsigned)ceil_div(2 * p.F, kGradCols)),
                           dim3(kGradBlock), 0, s, p, h.long_tiles, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace mp
