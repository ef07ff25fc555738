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

}  // extern "C"
