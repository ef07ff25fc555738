// C ABI of include/mp_layers.h: argument validation, workspace layout and
// launch sequencing of the operators around the aggregation.
#include <cfloat>
#include <climits>
#include <cmath>

#include "layers_internal.hpp"

using namespace mp;

namespace {

inline hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }
inline int hip_status(hipError_t e) { return e == hipSuccess ? MP_OK : MP_ERR_HIP; }

bool valid_dtype(int t) { return t == MP_F32 || t == MP_BF16; }
bool valid_itype(int t) { return t == MP_I32 || t == MP_I64; }
bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
size_t elem(int dtype) { return dtype == MP_BF16 ? 2 : 4; }

constexpr int64_t kMaxF = 65536;


int route_dims(int dtype, int64_t N, int64_t E, int64_t ldl, int64_t k) {
    if (!valid_dtype(dtype)) return MP_ERR_DTYPE;
    if (N < 0 || N > INT32_MAX || E < 1 || E > 1024 || ldl < E || k < 1 || k > 64 || k > E ||
        N * k > INT32_MAX)
        return MP_ERR_SIZE;
    return MP_OK;
}

size_t route_bytes(int64_t N, int64_t E) {
    const int blocks = route_blocks(N, E);
    return blocks > 1 ? (size_t)blocks * (size_t)(2 * E + 2) * 4 : 0;
}

}  // namespace

extern "C" {

int mp_dropout(const void* x, int dtype, int64_t N, int64_t F, int64_t ldx, const void* residual,
               int64_t ldr, const int32_t* ids, int whole_rows, double p, uint64_t seed,
               uint64_t offset, const int64_t* step, void* out, int64_t ldo, void* stream) {
    if (!valid_dtype(dtype)) return MP_ERR_DTYPE;
    if (N < 0 || N > INT32_MAX || F < 1 || F > kMaxF || ldx < F || ldo < F ||
        (residual && ldr < F) || !(p >= 0.0 && p <= 1.0))
        return MP_ERR_SIZE;
    if (N > 0 && (!x || !out)) return MP_ERR_NULL;
    const size_t b = elem(dtype);
    if (!aligned(x, b) || !aligned(out, b) || !aligned(residual, b) || !aligned(ids, 4) ||
        !aligned(step, 8))
        return MP_ERR_ALIGN;
    DropoutParams P{};
    P.x = x;
    P.residual = residual;
    P.ids = ids;
    P.step = step;
    P.out = out;
    P.N = N;
    P.F = F;
    P.ldx = ldx;
    P.ldr = ldr;
    P.ldo = ldo;
    P.limit = (uint32_t)std::floor(65536.0 * p + 0.5);
    P.scale = P.limit < 65536 ? (float)(65536.0 / (65536.0 - P.limit)) : 0.f;
    P.seed = seed;
    P.offset = offset;
    return hip_status(launch_dropout(P, dtype, whole_rows != 0, as_stream(stream)));
}

int mp_route_workspace(int64_t N, int64_t E, size_t* bytes) {
    if (!bytes) return MP_ERR_NULL;
    if (N < 0 || N > INT32_MAX || E < 1 || E > 1024) return MP_ERR_SIZE;
    *bytes = route_bytes(N, E);
    return MP_OK;
}

int mp_route(const void* logits, int dtype, int64_t N, int64_t E, int64_t ldl, int64_t k,
             const uint8_t* mask, int renorm, int32_t* idx, float* weight, int32_t* counts,
             float* loss, void* ws, size_t ws_bytes, void* stream) {
    const int st = route_dims(dtype, N, E, ldl, k);
    if (st != MP_OK) return st;
    const size_t need = route_bytes(N, E);
    if ((N > 0 && (!logits || !idx || !weight)) || !counts || !loss || (need && !ws))
        return MP_ERR_NULL;
    if (!aligned(logits, elem(dtype)) || !aligned(idx, 4) || !aligned(weight, 4) ||
        !aligned(counts, 4) || !aligned(loss, 4) || !aligned(ws, 4))
        return MP_ERR_ALIGN;
    if (ws_bytes < need) return MP_ERR_WORKSPACE;
    RouteParams P{};
    P.logits = logits;
    P.mask = mask;
    P.N = N;
    P.E = E;
    P.ldl = ldl;
    P.k = k;
    P.renorm = renorm;
    P.idx = idx;
    P.weight = weight;
    P.counts = counts;
    P.loss = loss;
    P.part = static_cast<float*>(ws);
    return hip_status(launch_route(P, dtype, as_stream(stream)));
}

int mp_route_backward(const void* logits, int dtype, int64_t N, int64_t E, int64_t ldl,
                      int64_t k, const uint8_t* mask, int renorm, const int32_t* idx,
                      const float* weight, const int32_t* counts, const float* dweight,
                      const float* dloss, void* dlogits, void* stream) {
    const int st = route_dims(dtype, N, E, ldl, k);
    if (st != MP_OK) return st;
    if ((N > 0 && (!logits || !idx || !weight || !dlogits)) || !counts) return MP_ERR_NULL;
    if (!aligned(logits, elem(dtype)) || !aligned(idx, 4) || !aligned(weight, 4) ||
        !aligned(counts, 4) || !aligned(dweight, 4) || !aligned(dloss, 4) ||
        !aligned(dlogits, elem(dtype)))
        return MP_ERR_ALIGN;
    RouteParams P{};
    P.logits = logits;
    P.mask = mask;
    P.N = N;
    P.E = E;
    P.ldl = ldl;
    P.k = k;
    P.renorm = renorm;
    P.idx = const_cast<int32_t*>(idx);
    P.weight = const_cast<float*>(weight);
    P.counts = const_cast<int32_t*>(counts);
    P.dweight = dweight;
    P.dloss = dloss;
    P.dlogits = dlogits;
    return hip_status(launch_route_backward(P, dtype, as_stream(stream)));
}

}  // extern "C"
