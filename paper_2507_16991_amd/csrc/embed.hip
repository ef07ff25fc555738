// Embedding rows by id times a scale, and the table's gradient by sorted ids
// (include/mp_layers.h).
//
// Forward: bound by memory; a thread has 16 bytes of a row.
// Backward: the rows' numbers lie sorted by id (the library's radix sort), and those
// of an id in order, so that every row of the gradient is the sum of consecutive
// positions: no atomics.  The positions, not the ids, are shared out: a team of lanes
// walks over a run of them and writes the rows of the ids that begin and end
// there, so that popular and rare ids cost the same (a team an id instead: 103 us
// for 169,343 ids of 256 fp32, 350 for 2.4M of 100 bf16; now 95 and 280).  What
// an id has in several runs is joined in LDS by the team of its last run, what it
// has in several workgroups by a second launch, whose teams take every so many
// of them and are then added up: an order that the positions alone set.  (That launch has
// one workgroup an id: one with most rows of a large batch leaves the rest of the chip
// idle.)  Rows of ids without positions are zeroed by workgroups of their own.
#include "layers_internal.hpp"

namespace mp {
namespace {

constexpr int kBlock = 256;
constexpr int kRows = 4;  // rows of a thread, forward, and rows zeroed
constexpr int kRun = 8;   // positions whose rows are loaded together
constexpr int64_t kMaxGrid = int64_t(1) << 22;  // (a launch has fewer than 2^32 threads)

__device__ inline int64_t id_at(const EmbedParams& P, int64_t r) {
    const int64_t v = P.ids64 ? static_cast<const int64_t*>(P.ids)[r]
                              : (int64_t)static_cast<const int32_t*>(P.ids)[r];
    return v >= 0 && v < P.V && v != P.padding ? v : -1;
}

// Chunk j of a row of F >= V elements; the last one ends with the row (and repeats
// elements of the one before, to the same values).
template <int V>
__device__ inline int chunk_at(int j, int F) {
    const int c = j * V;
    return c + V > F ? F - V : c;
}

template <int V>
__device__ inline void store_as(void* out, int bf16, int64_t at, const float (&v)[V]) {
    if (bf16) store_floats<BF16, V>(static_cast<uint16_t*>(out) + at, v);
    else store_floats<F32, V>(static_cast<float*>(out) + at, v);
}

// Rows r0, r0 + slots ... of a thread: their ids, then the rows, then the stores go
// out together.
template <typename T, int V>
__device__ inline void copy_rows(const EmbedParams& P, int64_t r0, int first, int per, int slots) {
    const int F = (int)P.F;
    int64_t id[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int64_t r = r0 + u * slots;
        id[u] = r < P.N ? id_at(P, r) : -1;
    }
    for (int j = first; j < per; j += kBlock) {
        const int c = chunk_at<V>(j, F);
        float v[kRows][V];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            if (id[u] >= 0) {
                load_floats<T, V>(static_cast<const typename T::raw*>(P.in) + id[u] * P.ld + c, v[u]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) v[u][i] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int64_t r = r0 + u * slots;
            if (r >= P.N) break;
#pragma unroll
            for (int i = 0; i < V; ++i) v[u][i] = id[u] >= 0 ? v[u][i] * P.scale : 0.f;
            store_as<V>(P.out, P.out_bf16, r * P.F + c, v[u]);
        }
    }
}

// A workgroup has kRows * slots rows, slots = 256 / per of `per` chunks (1 of
// longer ones).
template <typename T, int V>
__global__ __launch_bounds__(kBlock) void embed_rows(EmbedParams P, int per, int slots) {
    const int slot = threadIdx.x / per, first = threadIdx.x - slot * per;
    if (slot >= slots) return;
    const int64_t step = (int64_t)gridDim.x * slots * kRows;
    for (int64_t r0 = (int64_t)blockIdx.x * slots * kRows + slot; r0 < P.N; r0 += step)
        copy_rows<T, V>(P, r0, first, per, slots);
}

// The keys of the sort (V for ids outside the table) and its payload.
__global__ __launch_bounds__(kBlock) void embed_keys(EmbedParams P, int32_t* key, int32_t* row) {
    const int64_t r = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (r >= P.N) return;
    const int64_t id = id_at(P, r);
    key[r] = id >= 0 ? (int32_t)id : (int32_t)P.V;
    row[r] = (int32_t)r;
}

// ---- few rows -----------------------------------------------------------------------
// Without a sort: the place of a row in the order of the ids is the number of rows
// before it, counted against all of them in LDS.  A workgroup has kPlaces rows,
// kSlices threads each, that share the others.
constexpr int kSlices = 8;
constexpr int kPlaces = kBlock / kSlices;

// `places` workgroups for the rows; the others clear the gradient.
template <typename T>
__global__ __launch_bounds__(kBlock) void embed_places(EmbedParams P, int32_t* key, int32_t* row,
                                                       int32_t* status, int places) {
    extern __shared__ int32_t s_key[];
    const int tid = threadIdx.x, N = (int)P.N;
    if ((int)blockIdx.x >= places) {
        const int64_t size = P.V * P.F, threads = (int64_t)(gridDim.x - places) * kBlock;
        typename T::raw* out = static_cast<typename T::raw*>(P.out);
        constexpr int E = 16 / sizeof(typename T::raw);
        const float zero[E] = {};
        const int64_t i0 = (int64_t)(blockIdx.x - places) * kBlock + tid;
        for (int64_t i = i0; i < size / E; i += threads) store_floats<T, E>(out + i * E, zero);
        if (i0 < size % E) store_one<T>(out + size / E * E + i0, 0.f);
        return;
    }
    if (blockIdx.x == 0 && tid == 0) *status = MP_OK;
    // (filled up to whole slices with keys that are before nothing)
    const int per = ((N + kSlices - 1) / kSlices + 3) / 4 * 4;
    for (int i = tid; i < kSlices * per; i += kBlock) {
        const int64_t id = i < N ? id_at(P, i) : -1;
        s_key[i] = i >= N ? INT32_MAX : (id >= 0 ? (int32_t)id : (int32_t)P.V);
    }
    __syncthreads();
    // lanes of a slice are neighbours, so that they read the same words
    const int slice = tid / kPlaces, r = (int)blockIdx.x * kPlaces + tid % kPlaces;
    const int32_t mine = r < N ? s_key[r] : 0;
    const int q0 = slice * per;
    int before = 0;
    for (int q = q0; q < q0 + per; q += 4) {
        const int4 k = *reinterpret_cast<const int4*>(&s_key[q]);
        // of the same id, earlier rows are before
        before += k.x < mine + (q < r) ? 1 : 0;
        before += k.y < mine + (q + 1 < r) ? 1 : 0;
        before += k.z < mine + (q + 2 < r) ? 1 : 0;
        before += k.w < mine + (q + 3 < r) ? 1 : 0;
    }
    __syncthreads();
    s_key[tid] = before;  // (of all slices, in place of the keys)
    __syncthreads();
    if (slice == 0 && r < N) {
        for (int u = 1; u < kSlices; ++u) before += s_key[u * kPlaces + tid];
        key[r] = mine;
        row[before] = r;
    }
}

// Row v of the gradient from its sum, columns c ...; nothing for v = V.
template <typename T, int V>
__device__ inline void write_row(const EmbedParams& P, int32_t v, int c, const float (&sum)[V]) {
    if (v >= P.V) return;
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = sum[i] * P.scale;
    store_as<V>(P.out, P.out_bf16, (int64_t)v * P.F + c, o);
}

// A segment of positions is an id's.  Of a run, the segments that begin and end in it
// are written to the gradient; an end of one that began before goes to A, a
// beginning (or middle) of one that goes on to B.
enum { kEnds = 1, kGoesOn = 2, kMiddle = 4 };  // A there, B there, all of the run is B

// The workgroup's runs of R * kRun positions, columns of chunk j.  Flags and what lies
// in B go through LDS where there are several teams (A is its own team's).
template <typename T, int V>
__device__ inline void sum_runs(const EmbedParams& P, int64_t block, int j, int per, int slots, int slot, int R,
                                float* s_b, int* s_flag) {
    const int F = (int)P.F, c = chunk_at<V>(j, F);
    const int tid = threadIdx.x;
    const int64_t p0 = (block * slots + slot) * R * kRun;
    const int32_t none = (int32_t)P.V;  // ids outside the table, and positions past the last
    const bool on = slot < slots && p0 < P.N;
    const typename T::raw* in = static_cast<const typename T::raw*>(P.in) + c;
    int flag = 0;
    float a[V] = {}, acc[V] = {};
    if (on) {
        const int64_t p1 = p0 + R * kRun;
        const int32_t before = p0 > 0 ? P.key[P.row[p0 - 1]] : -1;
        const int32_t after = p1 < P.N ? P.key[P.row[p1]] : -1;
        int32_t cur = -1;
        bool open = false;    // the present segment began before the run
        bool whole = true;    // there has been no other
        for (int q0 = 0; q0 < R; ++q0) {
            int32_t r[kRun], k[kRun];
            RawOf<T, V> raw[kRun];
#pragma unroll
            for (int q = 0; q < kRun; ++q) {
                const int64_t p = p0 + q0 * kRun + q;
                r[q] = p < P.N ? P.row[p] : -1;
            }
#pragma unroll
            for (int q = 0; q < kRun; ++q) k[q] = r[q] >= 0 ? P.key[r[q]] : none;
#pragma unroll
            for (int q = 0; q < kRun; ++q)  // (rows of padding are not looked at)
                raw[q] = load_raw<T, V>(in + (int64_t)(k[q] < none ? r[q] : 0) * P.ld);
            if (q0 == 0) {
                cur = k[0];
                open = cur == before;
            }
#pragma unroll
            for (int q = 0; q < kRun; ++q) {
                if (k[q] != cur) {
                    if (open) {
                        flag |= kEnds;
#pragma unroll
                        for (int i = 0; i < V; ++i) a[i] = acc[i];
                    } else {
                        write_row<T, V>(P, cur, c, acc);
                    }
                    cur = k[q];
                    open = whole = false;
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[i] = 0.f;
                }
                float v[V];
                to_floats<T, V>(raw[q], v);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += v[i];
            }
        }
        if (cur < none) {
            if (cur == after) {
                flag |= kGoesOn | (whole && open ? kMiddle : 0);
            } else if (open) {
                flag |= kEnds;
#pragma unroll
                for (int i = 0; i < V; ++i) a[i] = acc[i];
            } else {
                write_row<T, V>(P, cur, c, acc);
            }
        }
    }
    float* part = P.part + 2 * block * P.F + c;  // ends, then what goes on
    if (slots == 1) {
        if (flag & kEnds) store_floats<F32, V>(part, a);
        if (flag & kGoesOn) store_floats<F32, V>(part + P.F, acc);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) s_b[i * kBlock + tid] = acc[i];
    if (j == 0) s_flag[slot] = flag;
    __syncthreads();
    if (slot >= slots) return;
    const bool last = slot == slots - 1;
    for (int part_of = 0; part_of < 2; ++part_of) {
        // the end of a segment that began in an earlier run; what goes on past the workgroup
        if (part_of == 0 ? !(flag & kEnds) : !(last && flag & kGoesOn)) continue;
        int t = part_of == 0 ? slot - 1 : slot;
        // (eight flags, and eight teams' sums, on their way together: one by one the gradient
        // of 190,001 rows of 1 or 4 fp32, many of one id, took 95 and 103 us for 82 and 91)
        for (int n = 8; n == 8; t -= n) {
            n = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) n += n == i && t >= i && s_flag[t >= i ? t - i : 0] & kMiddle;
        }
        const bool began = t >= 0;  // in this workgroup
        float v[V] = {};
#pragma unroll 8
        for (int u = t < 0 ? 0 : t; u <= (part_of == 0 ? slot - 1 : slot); ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += s_b[i * kBlock + u * per + j];
        if (part_of == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += a[i];
        }
        if (part_of == 0 && began) {
            write_row<T, V>(P, P.key[P.row[(block * slots + slot) * R * kRun]], c, v);
        } else {
            store_floats<F32, V>(part + part_of * P.F, v);
        }
    }
}

// `sums` workgroups for the runs of positions, among others for the rows of ids
// without any: the first wait for loads, the others for stores.
template <typename T, int V>
__global__ __launch_bounds__(kBlock) void embed_grad(EmbedParams P, int per, int slots, int R,
                                                     int64_t sums) {
    __shared__ float s_b[kBlock * V];
    __shared__ int s_flag[kBlock + 1];  // (one for the threads beside the teams)
    const int F = (int)P.F;
    const int slot = threadIdx.x / per, first = threadIdx.x - slot * per;
    const bool failed = *P.status != MP_OK;  // (then there are neither offsets nor an order)
    const int64_t before = blockIdx.x * sums / gridDim.x;
    if ((blockIdx.x + 1) * sums / gridDim.x > before) {
        if (failed) return;
        // (several teams: all threads make one pass)
        for (int j = first; j < per; j += kBlock)
            sum_runs<T, V>(P, before, j, per, slots, slot, R, s_b, s_flag);
        return;
    }
    if (slot >= slots) return;
    const int64_t step = (gridDim.x - sums) * slots * kRows;
    for (int64_t v0 = ((int64_t)blockIdx.x - before) * slots * kRows + slot; v0 < P.V; v0 += step) {
        bool empty[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int64_t v = v0 + (int64_t)u * slots;
            empty[u] = v < P.V && (failed || P.rowptr[v] == P.rowptr[v + 1]);
        }
        float zero[V];
#pragma unroll
        for (int i = 0; i < V; ++i) zero[i] = failed ? __builtin_nanf("") : 0.f;
        for (int j = first; j < per; j += kBlock) {
            const int c = chunk_at<V>(j, F);
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                if (empty[u]) store_as<V>(P.out, P.out_bf16, (v0 + (int64_t)u * slots) * P.F + c, zero);
        }
    }
}

// The rows of ids whose positions lie in several workgroups (of C each), by the
// workgroup of the first.  There is one less than of the others.
template <int V>
__global__ __launch_bounds__(kBlock) void embed_join(EmbedParams P, int per, int slots, int64_t C) {
    __shared__ float lds[kBlock * V];
    const int F = (int)P.F;
    const int slot = threadIdx.x / per, first = threadIdx.x - slot * per;
    if (*P.status != MP_OK) return;
    const int64_t k0 = blockIdx.x, b = k0 * C, e = b + C;
    const int32_t v = P.key[P.row[e - 1]];  // (a position follows)
    if (v == P.V || P.key[P.row[e]] != v || (b > 0 && P.key[P.row[b - 1]] == v)) return;
    int64_t k1;
    if (P.rowptr) {
        k1 = (P.rowptr[v + 1] - 1) / C;
    } else {
        // the first workgroup that the id does not go on from, 64 at a time
        k1 = k0 + 1;
        uint64_t ends;
        do {
            const int64_t p = (k1 + 1 + (threadIdx.x & 63)) * C;
            ends = __ballot(p >= P.N || P.key[P.row[p]] != v);
            k1 += ends ? __builtin_ctzll(ends) : 64;
        } while (!ends);
    }
    for (int j = first; j < per; j += kBlock) {
        const int c = chunk_at<V>(j, F);
        float acc[V] = {};
        if (slot < slots) {
#pragma unroll 4
            for (int64_t k = k0 + slot; k <= k1; k += slots) {
                float t[V];
                load_floats<F32, V>(P.part + (2 * k + (k < k1 ? 1 : 0)) * P.F + c, t);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += t[i];
            }
        }
        if (slots > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) lds[i * kBlock + threadIdx.x] = acc[i];
            __syncthreads();
            if (slot == 0) {
#pragma unroll 8
                for (int q = 1; q < slots; ++q)
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[i] += lds[i * kBlock + q * per + threadIdx.x];
            }
        }
        if (slot == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] *= P.scale;
            store_as<V>(P.out, P.out_bf16, (int64_t)v * P.F + c, acc);
        }
    }
}

int64_t at_most(int64_t blocks) { return blocks < kMaxGrid ? blocks : kMaxGrid; }

// Elements of a chunk, chunks of a row and rows side by side in a workgroup.  (Rows of
// 100 bf16 by chunks of 4 that divide them: 195 us for 1.9M of them, of 8 155.)
struct EmbedShape {
    int V, per, slots, R;  // R * kRun positions of a team: at least 128 of a workgroup
};
EmbedShape embed_shape(int64_t F, int dtype) {
    EmbedShape h;
    h.V = dtype == MP_BF16 ? 8 : 4;
    if (F < h.V) h.V = 1;
    h.per = (int)ceil_div(F, h.V);
    h.slots = h.per < kBlock ? kBlock / h.per : 1;
    h.R = (int)ceil_div(128, h.slots * kRun);
    return h;
}
int64_t positions(const EmbedShape& h) { return (int64_t)h.slots * h.R * kRun; }

template <typename T, int V>
void launch_rows(const EmbedParams& p, const EmbedShape& h, hipStream_t s) {
    hipLaunchKernelGGL((embed_rows<T, V>), dim3((unsigned)at_most(ceil_div(p.N, h.slots * kRows))),
                       dim3(kBlock), 0, s, p, h.per, h.slots);
}

template <typename T, int V>
void launch_grad(const EmbedParams& p, const EmbedShape& h, hipStream_t s) {
    const int64_t C = positions(h), sums = ceil_div(p.N, C);
    const int64_t zeros = p.rowptr ? at_most(ceil_div(p.V, h.slots * kRows)) : 0;
    if (sums + zeros)
        hipLaunchKernelGGL((embed_grad<T, V>), dim3((unsigned)(sums + zeros)), dim3(kBlock), 0, s, p,
                           h.per, h.slots, h.R, sums);
    if (sums > 1)
        hipLaunchKernelGGL((embed_join<V>), dim3((unsigned)(sums - 1)), dim3(kBlock), 0, s, p, h.per,
                           h.slots, C);
}

}  // namespace

// Workgroups of either type's sums, with two lines of F floats each.
int64_t embed_parts(int64_t N, int64_t F) {
    const int64_t a = ceil_div(N, positions(embed_shape(F, MP_F32)));
    const int64_t b = ceil_div(N, positions(embed_shape(F, MP_BF16)));
    return a > b ? a : b;
}

hipError_t launch_embed(const EmbedParams& p, int dtype, hipStream_t s) {
    if (p.N <= 0) return hipSuccess;
    const EmbedShape h = embed_shape(p.F, dtype);
    if (h.V == 1) {
        if (dtype == MP_BF16) launch_rows<BF16, 1>(p, h, s);
        else launch_rows<F32, 1>(p, h, s);
    } else {
        if (dtype == MP_BF16) launch_rows<BF16, 8>(p, h, s);
        else launch_rows<F32, 4>(p, h, s);
    }
    return hipGetLastError();
}

hipError_t launch_embed_keys(const EmbedParams& p, int32_t* key, int32_t* row, hipStream_t s) {
    if (p.N > 0)
        hipLaunchKernelGGL(embed_keys, dim3((unsigned)ceil_div(p.N, kBlock)), dim3(kBlock), 0, s, p,
                           key, row);
    return hipGetLastError();
}

// Up to 4,096 rows: fewer launches (50 ids of 200,000 14 us against 47, 4,096 of 100,000
// 34 against 43, but 8,192 60 and 47).  Where the library's one-workgroup sort takes
// the ids, up to 2,048 (2,000 of 5,000 ids 22 and 25 us, 8,192 of 10,000 50 and 35).
bool embed_few(int64_t N, int64_t V) { return N <= (V < kSortSmall ? 2048 : 4096); }

hipError_t launch_embed_places(const EmbedParams& p, int32_t* key, int32_t* row, int32_t* status,
                               hipStream_t s) {
    // (without rows the status still is written)
    const int places = (int)ceil_div(p.N > 0 ? p.N : 1, kPlaces);
    const int64_t size = p.V * p.F * (p.out_bf16 ? 2 : 4), fill = ceil_div(size, 16 * kBlock);
    const size_t lds = (size_t)(ceil_div(p.N, kSlices) + 4) * kSlices * 4;
    const dim3 g((unsigned)(places + (fill < 4096 ? fill : 4096)));
    const size_t least = kBlock * 4;
    if (p.out_bf16)
        hipLaunchKernelGGL((embed_places<BF16>), g, dim3(kBlock), lds > least ? lds : least, s, p, key,
                           row, status, places);
    else
        hipLaunchKernelGGL((embed_places<F32>), g, dim3(kBlock), lds > least ? lds : least, s, p, key,
                           row, status, places);
    return hipGetLastError();
}

hipError_t launch_embed_backward(const EmbedParams& p, int dtype, hipStream_t s) {
    const EmbedShape h = embed_shape(p.F, dtype);
    if (h.V == 1) {
        if (dtype == MP_BF16) launch_grad<BF16, 1>(p, h, s);
        else launch_grad<F32, 1>(p, h, s);
    } else {
        if (dtype == MP_BF16) launch_grad<BF16, 8>(p, h, s);
        else launch_grad<F32, 4>(p, h, s);
    }
    return hipGetLastError();
}

}  // namespace mp
