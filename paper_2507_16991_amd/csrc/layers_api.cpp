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


// Workspace of the group norm, in pieces that start on 256 bytes.
struct NormSpace {
    size_t flags = 0, stats = 0, ca = 0, cb = 0, part = 0, bytes = 0;
};
NormSpace norm_space(const NormShape& h, int64_t S, int64_t F, int64_t G, int backward) {
    NormSpace n;
    const auto take = [&](int64_t floats) {
        const size_t at = n.bytes;
        n.bytes = align_up(at + (size_t)floats * 4, 256);
        return at;
    };
    if (h.long_tiles) {
        n.flags = take(h.short_blocks);
        n.stats = take(h.long_tiles * h.places * h.stat_line * 2);
        if (backward) {
            n.ca = take(S * G);
            n.cb = take(S * G);
        }
    }
    if (backward) n.part = take(((h.unit ? h.short_blocks : 0) + h.long_tiles) * 2 * F);
    return n;
}

int norm_dims(int64_t N, int64_t S, int64_t F, int64_t G, int x_dtype) {
    if (!valid_dtype(x_dtype)) return MP_ERR_DTYPE;
    if (N < 0 || N > INT32_MAX || S < 1 || S > INT32_MAX || F < 1 || F > kMaxF || G < 1 ||
        F % G != 0)
        return MP_ERR_SIZE;
    return MP_OK;
}

int norm_call(const void* ptr, int ptr_itype, int64_t ldx, int64_t F, int act, int out_dtype) {
    if (!valid_itype(ptr_itype) || !valid_dtype(out_dtype)) return MP_ERR_DTYPE;
    if (ldx < F || act < MP_ACT_NONE || act > MP_ACT_GELU) return MP_ERR_SIZE;
    if (!ptr) return MP_ERR_NULL;
    if (!aligned(ptr, ptr_itype == MP_I64 ? 8 : 4)) return MP_ERR_ALIGN;
    return MP_OK;
}

int mx_dims(int64_t T, int64_t N, int64_t K, int64_t Fo) {
    if (N < 0 || N > INT32_MAX || T < 1 || T > 4096 || K < 1 || K > kMaxF || Fo < 1 || Fo > kMaxF)
        return MP_ERR_SIZE;
    return mx_product_fits(T, N, K, Fo) ? MP_OK : MP_ERR_SIZE;
}

// Workspace of the 4-bit product: the rows' codes and scales, and both operands'
// scales in words of four.
struct MxSpace {
    size_t x_scales, x_words, w_words, bytes;
};
MxSpace mx_space(int64_t T, int64_t N, int64_t K, int64_t Fo) {
    const size_t KB = (size_t)ceil_div(K, 32), KS = (KB + 3) / 4;
    MxSpace m;
    m.x_scales = align_up((size_t)N * KB * 16, 256);
    m.x_words = m.x_scales + align_up((size_t)N * KB, 256);
    m.w_words = m.x_words + align_up((size_t)N * KS * 4, 256);
    m.bytes = m.w_words + align_up((size_t)T * (size_t)Fo * KS * 4, 256);
    return m;
}

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

// Workspace of the embedding's gradient, in pieces that start on 256 bytes.
struct EmbedSpace {
    size_t key, row, col, rowptr, status, part, sort, sort_bytes, bytes;
};
int embed_space(int64_t N, int64_t V, int64_t F, EmbedSpace& m) {
    if (N < 0 || N > INT32_MAX || V < 1 || V >= INT32_MAX || F < 1 || F > kMaxF) return MP_ERR_SIZE;
    const int st = mp_coo_to_csr_workspace(N, V + 1, MP_I32, 0, &m.sort_bytes);
    if (st != MP_OK) return st;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t b = at;
        at = align_up(at + bytes, 256);
        return b;
    };
    m.key = take((size_t)N * 4);
    m.row = take((size_t)N * 4);
    m.col = take((size_t)N * 4);
    m.rowptr = take((size_t)(V + 2) * 4);
    m.status = take(4);
    m.part = take((size_t)embed_parts(N, F) * 2 * (size_t)F * 4);
    m.sort = take(m.sort_bytes);
    m.bytes = at;
    return MP_OK;
}

int rms_call(int dtype, int64_t N, int64_t F, int64_t ld) {
    if (!valid_dtype(dtype)) return MP_ERR_DTYPE;
    return N < 0 || N > INT32_MAX || F < 1 || F > kMaxF || ld < F ? MP_ERR_SIZE : MP_OK;
}

size_t rms_bytes(int64_t N, int64_t F, int dtype) {
    const int64_t parts = rms_parts(N, F, dtype);
    return parts > 1 ? (size_t)parts * (size_t)F * 4 : 0;
}

// Workspace of the experts, in pieces that start on 256 bytes.
struct ExpertSpace {
    size_t h, part, arrived, lists, bytes;
};
int expert_space(int64_t N, int64_t k, int64_t E, int64_t H, int64_t Fo, int out_dtype, ExpertSpace& m) {
    if (!valid_dtype(out_dtype)) return MP_ERR_DTYPE;
    if (N < 0 || N > 64 || k < 1 || k > E || E > 1024 || N * k > 1024 || H < 1 || H > kMaxF || Fo < 1 ||
        Fo > kMaxF)
        return MP_ERR_SIZE;
    const size_t tiles = (size_t)ceil_div(Fo, 32), splits = (size_t)expert_splits(Fo);
    m.h = 0;
    m.part = align_up(expert_h_bytes(N * k, (int64_t)align_up((size_t)H, 128)), 256);
    m.arrived = m.part + (splits > 1 ? align_up(tiles * splits * (size_t)N * 32 * 4, 256) : 0);
    m.lists = m.arrived + align_up(tiles * 4, 256);
    m.bytes = m.lists + align_up(expert_list_bytes(E, N * k), 256);
    return MP_OK;
}

// What both forms of the forward check and pass on.
int rms_forward(RmsParams& P, const void* x, int dtype, int64_t N, int64_t F, int64_t ldx,
                const void* residual, int64_t ldr, const float* weight, float eps, void* total,
                float* rstd) {
    const int st = rms_call(dtype, N, F, ldx);
    if (st != MP_OK) return st;
    if ((residual && ldr < F) || !(eps >= FLT_MIN && eps <= 1e30f)) return MP_ERR_SIZE;
    if (total && ((total == x && ldx != F) || (total == residual && ldr != F))) return MP_ERR_SIZE;
    if (N > 0 && !x) return MP_ERR_NULL;
    const size_t b = elem(dtype);
    if (!aligned(x, b) || !aligned(residual, b) || !aligned(total, b) || !aligned(weight, 4) ||
        !aligned(rstd, 4))
        return MP_ERR_ALIGN;
    P.x = x;
    P.residual = residual;
    P.weight = weight;
    P.N = N;
    P.F = F;
    P.ldx = ldx;
    P.ldr = ldr;
    P.eps = eps;
    P.total = total;
    P.rstd = rstd;
    return MP_OK;
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

int mp_group_norm_workspace(int64_t N, int64_t S, int64_t F, int64_t G, int x_dtype,
                            int backward, size_t* bytes) {
    if (!bytes) return MP_ERR_NULL;
    const int st = norm_dims(N, S, F, G, x_dtype);
    if (st != MP_OK) return st;
    *bytes = norm_space(norm_shape(N, S, F, G, x_dtype, backward), S, F, G, backward).bytes;
    return MP_OK;
}

int mp_group_norm(const void* ptr, int ptr_itype, const void* x, int x_dtype, int64_t N,
                  int64_t S, int64_t F, int64_t ldx, int64_t G, const float* gamma,
                  const float* beta, float eps, int act, void* out, int out_dtype, float* mean,
                  float* rstd, void* ws, size_t ws_bytes, void* stream) {
    int st = norm_dims(N, S, F, G, x_dtype);
    if (st == MP_OK) st = norm_call(ptr, ptr_itype, ldx, F, act, out_dtype);
    if (st != MP_OK) return st;
    if (!(eps >= 0.f && eps <= FLT_MAX)) return MP_ERR_SIZE;
    const NormShape h = norm_shape(N, S, F, G, x_dtype, 0);
    const NormSpace n = norm_space(h, S, F, G, 0);
    if ((N > 0 && (!x || !out)) || !mean || !rstd || (n.bytes && !ws)) return MP_ERR_NULL;
    if (!aligned(x, elem(x_dtype)) || !aligned(out, elem(out_dtype)) || !aligned(gamma, 4) ||
        !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(ws, 16))
        return MP_ERR_ALIGN;
    if (ws_bytes < n.bytes) return MP_ERR_WORKSPACE;
    NormParams P{};
    P.ptr = ptr;
    P.rp64 = ptr_itype == MP_I64;
    P.x = x;
    P.N = N;
    P.S = S;
    P.F = F;
    P.ldx = ldx;
    P.G = G;
    P.cg = (int)(F / G);
    P.gamma = gamma;
    P.beta = beta;
    P.eps = eps;
    P.act = act;
    P.out = out;
    P.out_bf16 = out_dtype == MP_BF16;
    P.mean = mean;
    P.rstd = rstd;
    P.flags = reinterpret_cast<int*>(static_cast<char*>(ws) + n.flags);
    P.stats = reinterpret_cast<float*>(static_cast<char*>(ws) + n.stats);
    return hip_status(launch_norm(P, h, x_dtype, false, nullptr, nullptr, as_stream(stream)));
}

int mp_group_norm_backward(const void* ptr, int ptr_itype, const void* x, int x_dtype,
                           const void* dout, int64_t N, int64_t S, int64_t F, int64_t ldx,
                           int64_t G, const float* gamma, const float* beta, const float* mean,
                           const float* rstd, int act, void* dx, int dx_dtype, float* dgamma,
                           float* dbeta, void* ws, size_t ws_bytes, void* stream) {
    int st = norm_dims(N, S, F, G, x_dtype);
    if (st == MP_OK) st = norm_call(ptr, ptr_itype, ldx, F, act, dx_dtype);
    if (st != MP_OK) return st;
    const NormShape h = norm_shape(N, S, F, G, x_dtype, 1);
    const NormSpace n = norm_space(h, S, F, G, 1);
    if ((N > 0 && (!x || !dout)) || !mean || !rstd || !dgamma != !dbeta || (!dx && !dgamma) ||
        (n.bytes && !ws))
        return MP_ERR_NULL;
    if (!aligned(x, elem(x_dtype)) || !aligned(dout, elem(x_dtype)) ||
        !aligned(dx, elem(dx_dtype)) || !aligned(gamma, 4) || !aligned(beta, 4) ||
        !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4) ||
        !aligned(ws, 16))
        return MP_ERR_ALIGN;
    if (ws_bytes < n.bytes) return MP_ERR_WORKSPACE;
    char* w = static_cast<char*>(ws);
    NormParams P{};
    P.ptr = ptr;
    P.rp64 = ptr_itype == MP_I64;
    P.x = x;
    P.dout = dout;
    P.N = N;
    P.S = S;
    P.F = F;
    P.ldx = ldx;
    P.G = G;
    P.cg = (int)(F / G);
    P.gamma = gamma;
    P.beta = beta;
    P.act = act;
    P.out = dx;
    P.out_bf16 = dx_dtype == MP_BF16;
    P.mean = const_cast<float*>(mean);
    P.rstd = const_cast<float*>(rstd);
    P.flags = reinterpret_cast<int*>(w + n.flags);
    P.stats = reinterpret_cast<float*>(w + n.stats);
    P.ca = reinterpret_cast<float*>(w + n.ca);
    P.cb = reinterpret_cast<float*>(w + n.cb);
    P.part = dgamma ? reinterpret_cast<float*>(w + n.part) : nullptr;
    return hip_status(launch_norm(P, h, x_dtype, true, dgamma, dbeta, as_stream(stream)));
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

int mp_mx_quantize(const void* x, int dtype, int64_t N, int64_t K, int64_t ldx, uint8_t* codes,
                   uint8_t* scales, void* values, void* stream) {
    if (!valid_dtype(dtype)) return MP_ERR_DTYPE;
    if (N < 0 || N > INT32_MAX || K < 1 || K > kMaxF || ldx < K) return MP_ERR_SIZE;
    if ((N > 0 && !x) || !codes != !scales || (N > 0 && !codes && !values)) return MP_ERR_NULL;
    if (!aligned(x, elem(dtype)) || !aligned(codes, 16) || !aligned(values, elem(dtype)))
        return MP_ERR_ALIGN;
    return hip_status(
        launch_mx_quantize(x, dtype, N, K, ldx, codes, scales, values, as_stream(stream)));
}

int mp_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t N, int64_t K, void* out,
                     int dtype, void* stream) {
    if (!valid_dtype(dtype)) return MP_ERR_DTYPE;
    if (N < 0 || N > INT32_MAX || K < 1 || K > kMaxF) return MP_ERR_SIZE;
    if (N > 0 && (!codes || !scales || !out)) return MP_ERR_NULL;
    if (!aligned(codes, 16) || !aligned(out, elem(dtype))) return MP_ERR_ALIGN;
    return hip_status(launch_mx_dequantize(codes, scales, N, K, out, dtype, as_stream(stream)));
}

int mp_mx_segment_matmul_workspace(int64_t T, int64_t N, int64_t K, int64_t Fo, size_t* bytes) {
    if (!bytes) return MP_ERR_NULL;
    const int st = mx_dims(T, N, K, Fo);
    if (st != MP_OK) return st;
    *bytes = mx_space(T, N, K, Fo).bytes;
    return MP_OK;
}

int mp_mx_segment_matmul(const void* seg, int seg_itype, int64_t T, const void* x, int x_dtype,
                         int64_t N, int64_t K, int64_t ldx, const uint8_t* w_codes,
                         const uint8_t* w_scales, int64_t Fo, void* out, int out_dtype, void* ws,
                         size_t ws_bytes, void* stream) {
    if (!valid_itype(seg_itype) || !valid_dtype(x_dtype) || !valid_dtype(out_dtype))
        return MP_ERR_DTYPE;
    const int st = mx_dims(T, N, K, Fo);
    if (st != MP_OK) return st;
    if (ldx < K) return MP_ERR_SIZE;
    if (!seg || !w_codes || !w_scales || (N > 0 && (!x || !out || !ws))) return MP_ERR_NULL;
    if (!aligned(seg, seg_itype == MP_I64 ? 8 : 4) || !aligned(x, elem(x_dtype)) ||
        !aligned(w_codes, 16) || !aligned(out, elem(out_dtype)) || !aligned(ws, 16))
        return MP_ERR_ALIGN;
    const MxSpace m = mx_space(T, N, K, Fo);
    if (ws_bytes < m.bytes) return MP_ERR_WORKSPACE;
    uint8_t* w = static_cast<uint8_t*>(ws);
    MxParams P{};
    P.seg = seg;
    P.seg64 = seg_itype == MP_I64;
    P.T = T;
    P.N = N;
    P.x = x;
    P.ldx = ldx;
    P.K = (int)K;
    P.KB = (int)ceil_div(K, 32);
    P.Fo = (int)Fo;
    P.w_codes = w_codes;
    P.w_scales = w_scales;
    P.x_codes = w;
    P.x_scales = w + m.x_scales;
    P.x_words = reinterpret_cast<uint32_t*>(w + m.x_words);
    P.w_words = reinterpret_cast<uint32_t*>(w + m.w_words);
    P.out = out;
    return hip_status(launch_mx_product(P, x_dtype, out_dtype, as_stream(stream)));
}

int mp_embed(const void* ids, int ids_itype, int64_t N, const void* table, int dtype, int64_t V,
             int64_t F, int64_t ldt, int64_t padding, float scale, void* out, int out_dtype,
             void* stream) {
    if (!valid_itype(ids_itype) || !valid_dtype(dtype) || !valid_dtype(out_dtype))
        return MP_ERR_DTYPE;
    if (N < 0 || N > INT32_MAX || V < 1 || V >= INT32_MAX || F < 1 || F > kMaxF || ldt < F)
        return MP_ERR_SIZE;
    if (N > 0 && (!ids || !table || !out)) return MP_ERR_NULL;
    if (!aligned(ids, ids_itype == MP_I64 ? 8 : 4) || !aligned(table, elem(dtype)) ||
        !aligned(out, elem(out_dtype)))
        return MP_ERR_ALIGN;
    EmbedParams P{};
    P.ids = ids;
    P.ids64 = ids_itype == MP_I64;
    P.N = N;
    P.V = V;
    P.F = F;
    P.padding = padding;
    P.scale = scale;
    P.in = table;
    P.ld = ldt;
    P.out = out;
    P.out_bf16 = out_dtype == MP_BF16;
    return hip_status(launch_embed(P, dtype, as_stream(stream)));
}

int mp_embed_backward_workspace(int64_t N, int64_t V, int64_t F, size_t* bytes) {
    if (!bytes) return MP_ERR_NULL;
    EmbedSpace m;
    const int st = embed_space(N, V, F, m);
    if (st != MP_OK) return st;
    *bytes = m.bytes;
    return MP_OK;
}

int mp_embed_backward(const void* ids, int ids_itype, int64_t N, const void* dout, int dtype,
                      int64_t V, int64_t F, int64_t ldd, int64_t padding, float scale,
                      void* dtable, int dtable_dtype, void* ws, size_t ws_bytes, void* stream) {
    if (!valid_itype(ids_itype) || !valid_dtype(dtype) || !valid_dtype(dtable_dtype))
        return MP_ERR_DTYPE;
    EmbedSpace m;
    int st = embed_space(N, V, F, m);
    if (st != MP_OK) return st;
    if (ldd < F) return MP_ERR_SIZE;
    if ((N > 0 && (!ids || !dout)) || !dtable || !ws) return MP_ERR_NULL;
    if (!aligned(ids, ids_itype == MP_I64 ? 8 : 4) || !aligned(dout, elem(dtype)) ||
        !aligned(dtable, elem(dtable_dtype)) || !aligned(ws, 16))
        return MP_ERR_ALIGN;
    if (ws_bytes < m.bytes) return MP_ERR_WORKSPACE;
    char* w = static_cast<char*>(ws);
    int32_t* key = reinterpret_cast<int32_t*>(w + m.key);
    int32_t* row = reinterpret_cast<int32_t*>(w + m.row);
    int32_t* col = reinterpret_cast<int32_t*>(w + m.col);
    int32_t* rowptr = reinterpret_cast<int32_t*>(w + m.rowptr);
    int32_t* status = reinterpret_cast<int32_t*>(w + m.status);
    EmbedParams P{};
    P.ids = ids;
    P.ids64 = ids_itype == MP_I64;
    P.N = N;
    P.V = V;
    P.F = F;
    P.padding = padding;
    P.scale = scale;
    P.in = dout;
    P.ld = ldd;
    P.out = dtable;
    P.out_bf16 = dtable_dtype == MP_BF16;
    P.row = col;
    P.key = key;
    P.status = status;
    P.part = reinterpret_cast<float*>(w + m.part);
    if (embed_few(N, V)) {
        st = hip_status(launch_embed_places(P, key, col, status, as_stream(stream)));
        if (st != MP_OK) return st;
        return hip_status(launch_embed_backward(P, dtype, as_stream(stream)));
    }
    P.rowptr = rowptr;
    st = hip_status(launch_embed_keys(P, key, row, as_stream(stream)));
    if (st == MP_OK)
        st = mp_coo_to_csr(row, key, N, V + 1, rowptr, MP_I32, col, nullptr, nullptr, nullptr,
                           w + m.sort, m.sort_bytes, status, stream);
    if (st != MP_OK) return st;
    return hip_status(launch_embed_backward(P, dtype, as_stream(stream)));
}

int mp_rms_norm(const void* x, int dtype, int64_t N, int64_t F, int64_t ldx, const void* residual,
                int64_t ldr, const float* weight, float eps, void* total, void* out, int out_dtype,
                float* rstd, void* stream) {
    if (!valid_dtype(out_dtype)) return MP_ERR_DTYPE;
    RmsParams P{};
    const int st =
        rms_forward(P, x, dtype, N, F, ldx, residual, ldr, weight, eps, total, rstd);
    if (st != MP_OK) return st;
    if (N > 0 && !out) return MP_ERR_NULL;
    if (!aligned(out, elem(out_dtype))) return MP_ERR_ALIGN;
    P.out = out;
    P.out_bf16 = out_dtype == MP_BF16;
    return hip_status(launch_rms(P, dtype, as_stream(stream)));
}

int mp_rms_norm_mx8(const void* x, int dtype, int64_t N, int64_t F, int64_t ldx,
                    const void* residual, int64_t ldr, const float* weight, float eps, void* total,
                    uint8_t* codes, uint8_t* scales, void* values, float* rstd, void* stream) {
    RmsParams P{};
    const int st =
        rms_forward(P, x, dtype, N, F, ldx, residual, ldr, weight, eps, total, rstd);
    if (st != MP_OK) return st;
    if (N > 0 && (!codes || !scales)) return MP_ERR_NULL;
    if (!aligned(codes, 16) || !aligned(values, elem(dtype))) return MP_ERR_ALIGN;
    P.codes = codes;
    P.scales = scales;
    P.out = values;
    P.out_bf16 = dtype == MP_BF16;
    return hip_status(launch_rms(P, dtype, as_stream(stream)));
}

int mp_mx8_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t N, int64_t K,
                      void* out, int dtype, void* stream) {
    if (!valid_dtype(dtype)) return MP_ERR_DTYPE;
    if (N < 0 || N > INT32_MAX || K < 1 || K > kMaxF) return MP_ERR_SIZE;
    if (N > 0 && (!codes || !scales || !out)) return MP_ERR_NULL;
    if (!aligned(codes, 16) || !aligned(out, elem(dtype))) return MP_ERR_ALIGN;
    return hip_status(launch_mx8_dequantize(codes, scales, N, K, out, dtype, as_stream(stream)));
}

int mp_rms_norm_backward_workspace(int64_t N, int64_t F, int dtype, size_t* bytes) {
    if (!bytes) return MP_ERR_NULL;
    const int st = rms_call(dtype, N, F, F);
    if (st != MP_OK) return st;
    *bytes = rms_bytes(N, F, dtype);
    return MP_OK;
}

int mp_rms_norm_backward(const void* total, int dtype, int64_t N, int64_t F, int64_t ldt,
                         const void* dout, const float* rstd, const float* weight,
                         const void* dtotal, void* dx, int dx_dtype, float* dweight, void* ws,
                         size_t ws_bytes, void* stream) {
    const int st = rms_call(dtype, N, F, ldt);
    if (st != MP_OK) return st;
    if (!valid_dtype(dx_dtype)) return MP_ERR_DTYPE;
    const size_t need = dweight ? rms_bytes(N, F, dtype) : 0;
    if ((N > 0 && (!total || !dout || !rstd)) || (!dx && !dweight) || (need && !ws))
        return MP_ERR_NULL;
    if (!aligned(total, elem(dtype)) || !aligned(dout, elem(dtype)) || !aligned(rstd, 4) ||
        !aligned(weight, 4) || !aligned(dtotal, elem(dtype)) || !aligned(dx, elem(dx_dtype)) ||
        !aligned(dweight, 4) || !aligned(ws, 16))
        return MP_ERR_ALIGN;
    if (ws_bytes < need) return MP_ERR_WORKSPACE;
    RmsParams P{};
    P.x = total;
    P.ldx = ldt;
    P.N = N;
    P.F = F;
    P.dout = dout;
    P.rstd = const_cast<float*>(rstd);
    P.weight = weight;
    P.dtotal = dtotal;
    P.out = dx;
    P.out_bf16 = dx_dtype == MP_BF16;
    P.dweight = dweight;
    P.part = static_cast<float*>(ws);
    return hip_status(launch_rms_backward(P, dtype, as_stream(stream)));
}

int mp_expert_mlp_workspace(int64_t N, int64_t k, int64_t E, int64_t H, int64_t Fo, int out_dtype,
                            size_t* bytes) {
    if (!bytes) return MP_ERR_NULL;
    ExpertSpace m;
    const int st = expert_space(N, k, E, H, Fo, out_dtype, m);
    if (st != MP_OK) return st;
    *bytes = m.bytes;
    return MP_OK;
}

int mp_expert_mlp(const void* x, int x_dtype, const uint8_t* x_scales, int64_t N, int64_t K,
                  int64_t ldx, const int32_t* idx, const float* weight, int64_t k, int64_t E,
                  int64_t H, int64_t Fo, const void* w1, const uint8_t* w1_scales, const void* w2,
                  const uint8_t* w2_scales, int act, int gated, const void* residual, int64_t ldr,
                  void* out, int out_dtype, void* ws, size_t ws_bytes, void* stream) {
    if (!x_scales && !valid_dtype(x_dtype)) return MP_ERR_DTYPE;
    ExpertSpace m;
    const int st = expert_space(N, k, E, H, Fo, out_dtype, m);
    if (st != MP_OK) return st;
    if (K < 1 || K > kMaxF || (!x_scales && ldx < K) ||
        (residual && ldr < Fo) || (residual && residual == out && ldr != Fo) ||
        act < MP_ACT_NONE || act > MP_ACT_GELU)
        return MP_ERR_SIZE;
    if ((N > 0 && (!x || !idx || !weight || !out || !ws)) || !w1 || !w2 || !w1_scales != !w2_scales)
        return MP_ERR_NULL;
    const size_t xa = x_scales ? 16 : elem(x_dtype), wa = w1_scales ? 16 : 2;
    if (!aligned(x, xa) || !aligned(idx, 4) || !aligned(weight, 4) || !aligned(w1, wa) ||
        !aligned(w2, wa) || !aligned(residual, elem(out_dtype)) || !aligned(out, elem(out_dtype)) ||
        !aligned(ws, 16))
        return MP_ERR_ALIGN;
    if (N == 0) return MP_OK;
    if (ws_bytes < m.bytes) return MP_ERR_WORKSPACE;
    char* w = static_cast<char*>(ws);
    ExpertParams P{};
    P.x = x;
    P.x_scales = x_scales;
    P.ldx = ldx;
    P.N = (int)N;
    P.k = (int)k;
    P.P = (int)(N * k);
    P.E = (int)E;
    P.K = (int)K;
    P.H = (int)H;
    P.Fo = (int)Fo;
    P.gated = gated != 0;
    P.act = act;
    P.idx = idx;
    P.weight = weight;
    P.w1 = w1;
    P.w1_scales = w1_scales;
    P.w2 = w2;
    P.w2_scales = w2_scales;
    P.residual = residual;
    P.ldr = ldr;
    P.out = out;
    P.out_bf16 = out_dtype == MP_BF16;
    P.splits = expert_splits(Fo);
    P.h = reinterpret_cast<uint16_t*>(w + m.h);
    P.Hp = (int)align_up((size_t)H, 128);
    P.part = reinterpret_cast<float*>(w + m.part);
    P.arrived = reinterpret_cast<int*>(w + m.arrived);
    P.lists = reinterpret_cast<int*>(w + m.lists);
    const int rows = x_scales ? kRowsMx8 : (x_dtype == MP_BF16 ? kRowsBf16 : kRowsF32);
    return hip_status(launch_experts(P, rows, w1_scales != nullptr, as_stream(stream)));
}

}  // extern "C"
