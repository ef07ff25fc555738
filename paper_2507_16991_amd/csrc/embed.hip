// Embedding rows by id times a scale, and the table's gradient by sorted ids
// (include/mp_layers.h).
//
// Forward: bound by memory; a thread has 16 bytes of a row.
// Backward: the rows' numbers lie sorted by id (the library's radix sort), so that
// every row of the gradient is the sum of consecutive positions, in the order of
// the rows: no atomics.  An id of up to C positions is summed by the lanes that
// write its row; the positions of all others, cut into chunks of C, by a workgroup
// a chunk, whose partial sums the workgroup of the id's first chunk adds in
// order.  An id of more than C positions reaches past the chunk that it begins in,
// so that a chunk has parts of two such ids at most.
#include "layers_internal.hpp"

#ifndef MP_ROWS
#define MP_ROWS 4
#endif
namespace mp {
namespace {

constexpr int kBlock = 256;
constexpr int kRows = MP_ROWS;  // rows of a thread
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

// acc += rows row[p], p = b, b + step, ... below e, columns c ...
template <typename T, int V>
__device__ inline void add_rows(const EmbedParams& P, int64_t b, int64_t e, int step, int c,
                                float (&acc)[V]) {
    const typename T::raw* in = static_cast<const typename T::raw*>(P.in) + c;
    int64_t p = b;
    for (; p + 3 * step < e; p += 4 * step) {
        int32_t r[4];
        float v[4][V];
#pragma unroll
        for (int u = 0; u < 4; ++u) r[u] = P.row[p + u * step];
#pragma unroll
        for (int u = 0; u < 4; ++u) load_floats<T, V>(in + (int64_t)r[u] * P.ld, v[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += v[u][i];
    }
    for (; p < e; p += step) {
        float v[V];
        load_floats<T, V>(in + (int64_t)P.row[p] * P.ld, v);
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += v[i];
    }
}

// Rows v0, v0 + slots ... of the gradient, kRows of them, but for ids of more than C
// positions.  Most ids have few: the offsets, the first row's number and the first
// row of all of them go out together.
template <typename T, int V>
__device__ inline void sum_rows(const EmbedParams& P, int64_t v0, int first, int per, int slots,
                                int64_t C, bool failed) {
    const int F = (int)P.F;
    int32_t b[kRows], e[kRows], r[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int64_t v = v0 + (int64_t)u * slots;
        const bool on = v < P.V && !failed;
        b[u] = on ? P.rowptr[v] : 0;
        e[u] = on ? P.rowptr[v + 1] : 0;
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) r[u] = b[u] < e[u] ? P.row[b[u]] : -1;
    for (int j = first; j < per; j += kBlock) {
        const int c = chunk_at<V>(j, F);
        float acc[kRows][V];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            if (r[u] >= 0) {
                load_floats<T, V>(static_cast<const typename T::raw*>(P.in) + r[u] * P.ld + c,
                                  acc[u]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) acc[u][i] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int64_t v = v0 + (int64_t)u * slots;
            if (v >= P.V) break;
            if (e[u] - b[u] > C) continue;
            if (e[u] - b[u] > 1) add_rows<T, V>(P, b[u] + 1, e[u], 1, c, acc[u]);
#pragma unroll
            for (int i = 0; i < V; ++i)
                acc[u][i] = failed ? __builtin_nanf("") : acc[u][i] * P.scale;
            store_as<V>(P.out, P.out_bf16, v * P.F + c, acc[u]);
        }
    }
}

// acc of a workgroup's slots added in order, the result in slot 0.
template <int V>
__device__ inline void add_slots(float (&acc)[V], int per, int slots, int slot, float* lds) {
    if (slots == 1) return;
    __syncthreads();
    if (slot < slots) {
#pragma unroll
        for (int i = 0; i < V; ++i) lds[i * kBlock + threadIdx.x] = acc[i];
    }
    __syncthreads();
    if (slot == 0) {
        for (int q = 1; q < slots; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += lds[i * kBlock + q * per + threadIdx.x];
    }
}

// blockIdx.x < chunks: the partial sums of a chunk of C positions.  Others: rows of
// the gradient whose ids have at most C.
template <typename T, int V>
__global__ __launch_bounds__(kBlock) void embed_grad(EmbedParams P, int per, int slots, int64_t C,
                                                     int64_t chunks) {
    __shared__ float lds[kBlock * V];
    const int F = (int)P.F;
    const int slot = threadIdx.x / per, first = threadIdx.x - slot * per;
    const bool failed = *P.status != MP_OK;  // (then rowptr is not written)
    if ((int64_t)blockIdx.x >= chunks) {
        if (slot >= slots) return;
        const int64_t step = (gridDim.x - chunks) * slots * kRows;
        for (int64_t v0 = ((int64_t)blockIdx.x - chunks) * slots * kRows + slot; v0 < P.V;
             v0 += step)
            sum_rows<T, V>(P, v0, first, per, slots, C, failed);
        return;
    }
    if (failed) return;
    const int64_t inside = P.rowptr[P.V];  // positions of ids of the table
    const int64_t b = (int64_t)blockIdx.x * C, e = b + C < inside ? b + C : inside;
    if (b >= e) return;
    const int32_t va = P.key[P.row[b]], vb = P.key[P.row[e - 1]];
    for (int part = 0; part < (va == vb ? 1 : 2); ++part) {
        const int32_t v = part ? vb : va;
        const int64_t vbeg = P.rowptr[v], vend = P.rowptr[v + 1];
        if (vend - vbeg <= C) continue;
        const int64_t pb = vbeg > b ? vbeg : b, pe = vend < e ? vend : e;
        for (int j = first; j < per; j += kBlock) {
            const int c = chunk_at<V>(j, F);
            float acc[V] = {};
            if (slot < slots) add_rows<T, V>(P, pb + slot, pe, slots, c, acc);
            add_slots<V>(acc, per, slots, slot, lds);
            if (slot == 0)
                store_floats<F32, V>(P.part + (2 * (int64_t)blockIdx.x + part) * P.F + c, acc);
        }
    }
}

// The rows of ids of more than C positions: the workgroup of the chunk that such an
// id begins in (it has the chunk's last position) adds its partial sums.
template <int V>
__global__ __launch_bounds__(kBlock) void embed_join(EmbedParams P, int per, int slots, int64_t C) {
    __shared__ float lds[kBlock * V];
    const int F = (int)P.F;
    const int slot = threadIdx.x / per, first = threadIdx.x - slot * per;
    if (*P.status != MP_OK) return;
    const int64_t inside = P.rowptr[P.V];
    const int64_t k0 = blockIdx.x, b = k0 * C, e = b + C < inside ? b + C : inside;
    if (b >= e) return;
    const int32_t v = P.key[P.row[e - 1]];
    const int64_t vbeg = P.rowptr[v], vend = P.rowptr[v + 1];
    if (vend - vbeg <= C || vbeg < b) return;
    const int64_t k1 = (vend - 1) / C;
    for (int j = first; j < per; j += kBlock) {
        const int c = chunk_at<V>(j, F);
        float acc[V] = {};
        if (slot < slots) {
#pragma unroll 4
            for (int64_t k = k0 + slot; k <= k1; k += slots) {
                // (in its first chunk the id is the second one, unless it begins there)
                float t[V];
                load_floats<F32, V>(P.part + (2 * k + (k == k0 && vbeg > b ? 1 : 0)) * P.F + c, t);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += t[i];
            }
        }
        add_slots<V>(acc, per, slots, slot, lds);
        if (slot == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] *= P.scale;
            store_as<V>(P.out, P.out_bf16, (int64_t)v * P.F + c, acc);
        }
    }
}

int64_t at_most(int64_t blocks) { return blocks < kMaxGrid ? blocks : kMaxGrid; }

// Elements of a chunk, chunks of a row and rows side by side in a workgroup.  bf16
// rows of a multiple of 4 but not of 8 are taken 4 at a time: 
struct EmbedShape {
    int V, per, slots;
};
EmbedShape embed_shape(int64_t F, int dtype) {
    EmbedShape h;
    h.V = dtype == MP_BF16 && (F % 8 == 0 || F % 4 != 0) ? 8 : 4;
    if (F < h.V) h.V = 1;
    h.per = (int)ceil_div(F, h.V);
    h.slots = h.per < kBlock ? kBlock / h.per : 1;
    return h;
}

template <typename T, int V>
void launch_rows(const EmbedParams& p, const EmbedShape& h, hipStream_t s) {
    hipLaunchKernelGGL((embed_rows<T, V>), dim3((unsigned)at_most(ceil_div(p.N, h.slots * kRows))),
                       dim3(kBlock), 0, s, p, h.per, h.slots);
}

template <typename T, int V>
void launch_grad(const EmbedParams& p, const EmbedShape& h, hipStream_t s) {
    const int64_t C = embed_chunk(p.N), chunks = p.N > C ? ceil_div(p.N, C) : 0;
    hipLaunchKernelGGL((embed_grad<T, V>), dim3((unsigned)(chunks + at_most(ceil_div(p.V, h.slots * kRows)))),
                       dim3(kBlock), 0, s, p, h.per, h.slots, C, chunks);
    if (chunks)
        hipLaunchKernelGGL((embed_join<V>), dim3((unsigned)chunks), dim3(kBlock), 0, s, p, h.per,
                           h.slots, C);
}

}  // namespace

// Positions of a chunk.
int64_t embed_chunk(int64_t N) {
    int64_t c = 64;
    while (c < 512 && c * 8192 < N) c *= 2;
    return c;
}

hipError_t launch_embed(const EmbedParams& p, int dtype, hipStream_t s) {
    if (p.N <= 0) return hipSuccess;
    const EmbedShape h = embed_shape(p.F, dtype);
    if (h.V == 1) {
        if (dtype == MP_BF16) launch_rows<BF16, 1>(p, h, s);
        else launch_rows<F32, 1>(p, h, s);
    } else {
        if (dtype == MP_F32) launch_rows<F32, 4>(p, h, s);
        else if (h.V == 8) launch_rows<BF16, 8>(p, h, s);
        else launch_rows<BF16, 4>(p, h, s);
    }
    return hipGetLastError();
}

hipError_t launch_embed_keys(const EmbedParams& p, int32_t* key, int32_t* row, hipStream_t s) {
    if (p.N > 0)
        hipLaunchKernelGGL(embed_keys, dim3((unsigned)ceil_div(p.N, kBlock)), dim3(kBlock), 0, s, p,
                           key, row);
    return hipGetLastError();
}

hipError_t launch_embed_backward(const EmbedParams& p, int dtype, hipStream_t s) {
    const EmbedShape h = embed_shape(p.F, dtype);
    if (h.V == 1) {
        if (dtype == MP_BF16) launch_grad<BF16, 1>(p, h, s);
        else launch_grad<F32, 1>(p, h, s);
    } else {
        if (dtype == MP_F32) launch_grad<F32, 4>(p, h, s);
        else if (h.V == 8) launch_grad<BF16, 8>(p, h, s);
        else launch_grad<BF16, 4>(p, h, s);
    }
    return hipGetLastError();
}

}  // namespace mp
