// Microscaled 4-bit floating point (MXFP4): quantisation, and the product of row
// segments with 4-bit weights (include/mp_layers.h states format and layout).
//
// Products run on v_mfma_scale_f32_*_f8f6f4, whose operands are 32 codes (16
// bytes, along k) and their block's scale exponent from each lane: lane l of
// the 32x32x64 form holds row l % 32 and block l / 32, of the 16x16x128 form
// row l % 16 and block l / 16; the accumulators are those of the bf16 forms.
// Weights are the first operand and rows of x the second, so that a lane's
// accumulators are neighbouring output columns of one row.
//
// Three kernels share the products out; for the last two x is quantised first (a
// quarter of its bytes):
//   * mx_narrow: weights of a segment that fit into LDS, few output columns: x is
//     quantised on the way; bound by reading x and writing out;
//   * mx_thin: segments of few rows: bound by reading the weights, which go
//     straight to registers, k split over the wavefronts of a workgroup;
//   * mx_tiles: tiles staged through LDS by asynchronous loads.
#include "layers_internal.hpp"

namespace mp {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 256;
constexpr int kMxBlock = 32;      // values under one scale
constexpr int kFp4 = 4;           // operand format of the MFMA: E2M1
constexpr uint32_t kNanScale = 255;

// ---- quantisation ------------------------------------------------------------------
// Four neighbouring lanes have the 32 values of a block, eight each.

// Largest over the four lanes of a quad.
__device__ inline uint32_t quad_max(uint32_t x) {
    uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true);
    x = x > y ? x : y;
    y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true);
    return x > y ? x : y;
}

// The scale byte for a block whose largest magnitude has these float bits:
// floor(log2) - 2 with E8M0's bias is the exponent field less two.
__device__ inline uint32_t scale_of(uint32_t bits) {
    const uint32_t e = bits >> 23;
    return e == 255 ? kNanScale : (e > 2 ? e - 2 : 0);
}
// 2^(s - 127) (s = 0 is subnormal); NaN for 255.
__device__ inline float scale_value(uint32_t s) {
    return __uint_as_float(s == kNanScale ? 0x7FC00000u : (s ? s << 23 : 0x00400000u));
}

// Eight values -> their block's scale and eight codes.  The conversion divides by the
// scale, rounds to nearest even and saturates.
template <typename T>
__device__ inline uint32_t quantize8(const RawOf<T, 8>& r, uint32_t& s) {
    uint32_t m = 0, c = 0;
    if constexpr (sizeof(typename T::raw) == 2) {
        u16x2 h = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            h = __builtin_elementwise_max(h, __builtin_bit_cast(u16x2, r.w[i] & 0x7FFF7FFFu));
        m = (uint32_t)(h.x > h.y ? h.x : h.y) << 16;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = r.w[i] & 0x7FFFFFFFu;
            m = m > a ? m : a;
        }
    }
    s = scale_of(quad_max(m));
    const float f = scale_value(s == kNanScale ? 127u : s);
    if constexpr (sizeof(typename T::raw) == 2) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, r.w[0]), f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, r.w[1]), f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, r.w[2]), f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, r.w[3]), f, 3);
    } else {
        float v[8];
        to_floats<T, 8>(r, v);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], f, 3);
    }
    return c;
}

// The value of a code under a scale: magnitude bits e1 e0 m are 0 or 0.5 (e = 0), or
// (1 + m / 2) 2^(e - 1); exact, and exact in bf16.
__device__ inline float value_of(uint32_t code, float scale) {
    const uint32_t e = (code >> 1) & 3, m = code & 1;
    const float a = e ? __uint_as_float(((126 + e) << 23) | (m << 22)) : (m ? 0.5f : 0.f);
    return (code & 8 ? -a : a) * scale;
}

// Values k0 .. k0+7 of a row of K, zero past its end.
template <typename T>
__device__ inline RawOf<T, 8> load8(const typename T::raw* p, int k0, int K) {
    if (k0 + 8 <= K) return load_raw<T, 8>(p + k0);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k0 + i < K ? load_one<T>(p + k0 + i) : 0.f;
    return from_floats<T, 8>(v);
}

template <typename T>
__device__ inline void store8(typename T::raw* p, int k0, int K, const float (&v)[8]) {
    if (k0 + 8 <= K) {
        store_floats<T, 8>(p + k0, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k0 + i < K) store_one<T>(p + k0 + i, v[i]);
}

// A workgroup takes rows_per_block rows, a thread eight values of one.  Bound by
// memory: 32,768 x 4096 bf16 with values 112 us (5.4 TB/s).
template <typename T>
__global__ __launch_bounds__(kBlock) void mx_quantize(const typename T::raw* x, int64_t N, int K,
                                                      int64_t ldx, int rows_per_block,
                                                      uint32_t* codes, uint8_t* scales,
                                                      typename T::raw* values) {
    const int per = 4 * ((K + kMxBlock - 1) / kMxBlock);
    const int64_t groups = (N + rows_per_block - 1) / rows_per_block;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t r0 = g * rows_per_block;
        const uint32_t n = (uint32_t)(N - r0 < rows_per_block ? N - r0 : rows_per_block) * per;
        for (uint32_t l = threadIdx.x; l < n; l += kBlock) {  // (n is a multiple of 4: whole quads)
            const uint32_t dr = l / (uint32_t)per, j = l - dr * per;
            const int64_t r = r0 + dr;
            uint32_t s;
            const uint32_t c = quantize8<T>(load8<T>(x + r * ldx, 8 * j, K), s);
            if (codes) {
                codes[r * per + j] = c;
                if ((j & 3) == 0) scales[r * (per / 4) + j / 4] = (uint8_t)s;
            }
            if (values && 8 * (int)j < K) {
                const float f = scale_value(s);
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = value_of(c >> (4 * i), f);
                store8<T>(values + r * K, 8 * j, K, v);
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void mx_dequantize(const uint32_t* codes,
                                                        const uint8_t* scales, int64_t N, int K,
                                                        int rows_per_block,
                                                        typename T::raw* out) {
    const int per = 4 * ((K + kMxBlock - 1) / kMxBlock);
    const int64_t groups = (N + rows_per_block - 1) / rows_per_block;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t r0 = g * rows_per_block;
        const uint32_t n = (uint32_t)(N - r0 < rows_per_block ? N - r0 : rows_per_block) * per;
        for (uint32_t l = threadIdx.x; l < n; l += kBlock) {
            const uint32_t dr = l / (uint32_t)per, j = l - dr * per;
            if (8 * (int)j >= K) continue;
            const int64_t r = r0 + dr;
            const uint32_t c = codes[r * per + j];
            const float f = scale_value(scales[r * (per / 4) + j / 4]);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = value_of(c >> (4 * i), f);
            store8<T>(out + r * K, 8 * j, K, v);
        }
    }
}

// ---- segments -------------------------------------------------------------------------
__device__ inline int64_t seg_at(const MxParams& P, int64_t t) {
    const int64_t v = P.seg64 ? static_cast<const int64_t*>(P.seg)[t]
                              : (int64_t)static_cast<const int32_t*>(P.seg)[t];
    return v < 0 ? 0 : (v > P.N ? P.N : v);
}

// Tile `tile` of the segments' rows in tiles of BM (no tile has rows of two):
// its segment, rows and the segment's end, or t = -1 past the last.  64 segments a
// step.
struct RowTile {
    int64_t t, r0, r1, end;
};
__device__ inline RowTile row_tile(const MxParams& P, int64_t tile, int BM) {
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int64_t t0 = 0; t0 < P.T; t0 += 64) {
        const int64_t t = t0 + lane;
        const int64_t b = t < P.T ? seg_at(P, t) : 0, e = t < P.T ? seg_at(P, t + 1) : 0;
        const int n = e > b ? (int)((e - b + BM - 1) / BM) : 0;
        int sum = n;  // tiles up to and with this lane's segment
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(sum, o);
            if (lane >= o) sum += v;
        }
        const int64_t end = before + sum;
        const uint64_t hit = __ballot(n > 0 && tile < end);
        if (hit) {
            const int i = __builtin_ctzll(hit);
            // the lane's values, made uniform
            const int64_t ti = t0 + i, bi = seg_at(P, ti), ei = seg_at(P, ti + 1);
            const int ni = __shfl(n, i);
            const int64_t first = before + __shfl(sum, i) - ni;
            const int64_t r0 = bi + (tile - first) * BM;
            return RowTile{ti, r0, r0 + BM < ei ? r0 + BM : ei, ei};
        }
        before += __shfl(sum, 63);
    }
    return RowTile{-1, 0, 0, 0};
}

__device__ inline i32x8 operand(const uint4& c) {
    return i32x8{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};
}

template <bool BF>
__device__ inline void store4(void* out, int64_t at, const float (&v)[4]) {
    if (BF) store_floats<BF16, 4>(static_cast<uint16_t*>(out) + at, v);
    else store_floats<F32, 4>(static_cast<float*>(out) + at, v);
}
template <bool BF>
__device__ inline void store_col(void* out, int64_t at, float v) {
    if (BF) store_one<BF16>(static_cast<uint16_t*>(out) + at, v);
    else store_one<F32>(static_cast<float*>(out) + at, v);
}

// What the lanes of this wavefront have written to LDS is there for the others (the
// LDS operations of one wavefront complete in order: only the compiler waits).
__device__ inline void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ---- tiles ------------------------------------------------------------------------------
// A workgroup of WM x WN wavefronts has 32 FM WM output columns x 32 FN WN rows, a
// wavefront FM x FN products of 32 x 32.  k in steps of 4 blocks (64 bytes a row),
// three buffers: while one is multiplied, asynchronous loads fill the others.  Steps
// are that short so that two workgroups fit into a CU's LDS, and one multiplies
// while the other writes its results.
// In LDS the 16-byte pieces of row r lie at piece ^ (r / 4 % 4), so that the
// lanes of a fragment (32 rows, one piece) spread over the banks.
constexpr int kStep = 4;  // blocks of a step
constexpr int kRowBytes = kStep * 16;

template <int ROWS>
struct TileBuffer {
    uint8_t codes[ROWS * kRowBytes];
    uint32_t scales[ROWS];
};

// A workgroup's asynchronous loads of ROWS rows, blocks 4 k .. 4 k + 3 of step k.  Rows
// past `rows` repeat the last one (their products are not stored), blocks past KB
// the last one, under scales of 0: both factors are then 2^-127, and such products
// vanish.
template <int ROWS, int WAVES>
struct TileLoader {
    static constexpr int PER = ROWS / 16 / WAVES;  // loads of a wavefront, 16 rows each
    static constexpr int LOADS = PER + 1;
    const uint8_t* codes;
    const uint32_t* scales;  // [step][line]: this lane's row of step 0
    int64_t line;
    uint32_t off[PER];
    int KB, piece, first;    // first: row of this wavefront's scales

    __device__ TileLoader(const uint8_t* c, const uint32_t* sc, int64_t sc_line, int rows, int kb) {
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
        codes = c;
        KB = kb;
        line = sc_line;
        piece = (lane & 3) ^ ((lane >> 4) & 3);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = (w * PER + i) * 16 + (lane >> 2);
            off[i] = (uint32_t)((r < rows ? r : rows - 1) * kb) * 16u;
        }
        first = w % (ROWS / 64) * 64;  // (of fewer than 64 rows a wavefront, some load the same)
        const int r = first + lane;
        scales = sc + (r < rows ? r : rows - 1);
    }
    __device__ void fetch(TileBuffer<ROWS>& to, int k) const {
        const int w = threadIdx.x >> 6, kb = k * kStep + piece;
        const uint32_t at = (uint32_t)(kb < KB ? kb : KB - 1) * 16u;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void*)(codes + (off[i] + at)),
                (__attribute__((address_space(3))) void*)(to.codes + (w * PER + i) * 16 * kRowBytes),
                16, 0, 0);
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void*)(scales + k * line),
            (__attribute__((address_space(3))) void*)(to.scales + first), 4, 0, 0);
    }
};

// The scales of R rows, [R, KB] bytes, as a table of words [KS, R]: word (k, r) has those
// of row r in step k, 0 past KB.  Tiles then load a step's scales as whole lines
// (from the format's own layout every row is a request of its own: half of all
// requests to L2: with it 1170 us at 65,536 x 4096 x 4096, without 960 at that time).
struct ScaleTable {
    const uint8_t* in;
    uint32_t* out;
    int64_t R, lines;  // rows; rows to a table of words (the segments' weights have one each)
};
__global__ __launch_bounds__(kBlock) void mx_scale_words(ScaleTable A, ScaleTable B, int KB, int KS,
                                                         int64_t blocks_a) {
    const bool second = (int64_t)blockIdx.x >= blocks_a;
    const ScaleTable t = second ? B : A;
    const int64_t r = ((int64_t)blockIdx.x - (second ? blocks_a : 0)) * kBlock + threadIdx.x;
    if (r >= t.R) return;
    const int64_t table = t.R == t.lines ? 0 : r / t.lines, in_table = r - table * t.lines;
    const uint8_t* p = t.in + r * KB;
    uint32_t* q = t.out + table * KS * t.lines + in_table;
    const int k0 = blockIdx.y * 4;
    uint32_t w[4] = {0, 0, 0, 0};
    if (4 * k0 + 16 <= KB) {
        __builtin_memcpy(w, p + 4 * k0, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (4 * k0 + i < KB) w[i / 4] |= (uint32_t)p[4 * k0 + i] << (8 * (i % 4));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (k0 + i < KS) q[(k0 + i) * t.lines] = w[i];
}

template <int FM, int FN, int BM, int BN>
__device__ inline void multiply(const TileBuffer<BM>& W, const TileBuffer<BN>& X, int wm,
                                int wn, int lane, f32x16 (&acc)[FM][FN]) {
    const int half = lane >> 5, row = lane & 31;
    int sw[FM], sx[FN];  // byte 2 s is the scale of block 2 s + half
#pragma unroll
    for (int i = 0; i < FM; ++i) sw[i] = (int)(W.scales[(wm * FM + i) * 32 + row] >> (8 * half));
#pragma unroll
    for (int j = 0; j < FN; ++j) sx[j] = (int)(X.scales[(wn * FN + j) * 32 + row] >> (8 * half));
    uint4 a[2][FM], b[2][FN];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int at = ((2 * s + half) ^ ((row >> 2) & 3)) * 16;
#pragma unroll
        for (int i = 0; i < FM; ++i)
            a[s][i] = *reinterpret_cast<const uint4*>(
                &W.codes[((wm * FM + i) * 32 + row) * kRowBytes + at]);
#pragma unroll
        for (int j = 0; j < FN; ++j)
            b[s][j] = *reinterpret_cast<const uint4*>(
                &X.codes[((wn * FN + j) * 32 + row) * kRowBytes + at]);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                operand(a[0][i]), operand(b[0][j]), acc[i][j], kFp4, kFp4, 0, sw[i], 0, sx[j]);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                operand(a[1][i]), operand(b[1][j]), acc[i][j], kFp4, kFp4, 2, sw[i], 2, sx[j]);
    // the products stay here: the compiler would sink them past the workgroup's
    // barrier, with all fragments in registers until then
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) asm volatile("" : "+v"(acc[i][j]));
}

// Workgroups go to the XCDs in turn; each XCD has a run of tiles, in bands of
// eight row tiles, so that its L2 serves rows and columns again.  False: none left.
__device__ inline bool pick_tile(int64_t row_tiles, int col_tiles, int64_t& rt, int& ct) {
    const int64_t total = row_tiles * col_tiles, per = (total + 7) / 8;
    const int64_t lin = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if (lin >= total) return false;
    const int64_t band = lin / (8 * col_tiles), in = lin - band * 8 * col_tiles;
    const int64_t high = row_tiles - band * 8 < 8 ? row_tiles - band * 8 : 8;
    rt = band * 8 + in % high;
    ct = (int)(in / high);
    return true;
}

// acc to out: rows r0 .. r0+rows of the tile, columns c0 .. c0+cols.  A lane has four
// columns of a row, so 32 x 32 products go through LDS (the wavefront's own kOut
// floats), to be written by whole lines: 32 bytes at a time, the rows' stores were a
// fifth of all requests to L2 (130 of 960 us at 65,536 x 4096 x 4096; now 850 to 920).
constexpr int kOutLine = 36, kOut = 32 * kOutLine;

template <int FM, int FN, bool BF>
__device__ inline void store_tile(const MxParams& P, const f32x16 (&acc)[FM][FN], int wm, int wn,
                                  int64_t r0, int rows, int c0, int cols, float* lds) {
    constexpr int E = BF ? 8 : 4, PER = 32 / E;  // columns of a 16-byte store, stores of a row
    const int lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            wave_sync();
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<float4*>(&lds[(lane & 31) * kOutLine + 8 * q + 4 * half]) =
                    make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2],
                                acc[i][j][4 * q + 3]);
            wave_sync();
#pragma unroll
            for (int u = 0; u < 32 * PER / kWave; ++u) {
                const int r = (u * kWave + lane) / PER, c = (lane % PER) * E;
                float v[E];
                __builtin_memcpy(v, &lds[r * kOutLine + c], sizeof(v));
                const int row = (wn * FN + j) * 32 + r, col = (wm * FM + i) * 32 + c;
                if (row >= rows) continue;
                const int64_t at = (r0 + row) * P.Fo + c0 + col;
                if (col + E <= cols) {
                    if (BF) store_floats<BF16, E>(static_cast<uint16_t*>(P.out) + at, v);
                    else store_floats<F32, E>(static_cast<float*>(P.out) + at, v);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (col + e < cols) store_col<BF>(P.out, at + e, v[e]);
                }
            }
        }
}

// Three buffers, so that loads have two steps' time to arrive: s_waitcnt of n.
template <int N>
__device__ inline void wait_loads() {
    static_assert(N == 0 || N == 6 || N == 8, "the waits below");
    if constexpr (N == 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else if constexpr (N == 6) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <int FM, int FN, int WM, int WN, bool BF>
__global__ __launch_bounds__(64 * WM * WN, 2) void mx_tiles(MxParams P, int64_t row_tiles,
                                                            int col_tiles) {
    constexpr int BM = 32 * FM * WM, BN = 32 * FN * WN, WAVES = WM * WN;  // columns, rows
    typedef TileLoader<BM, WAVES> LoadW;
    typedef TileLoader<BN, WAVES> LoadX;
    __shared__ __attribute__((aligned(16))) TileBuffer<BM> W0, W1, W2;
    __shared__ __attribute__((aligned(16))) TileBuffer<BN> X0, X1, X2;
    int64_t rt;
    int ct;
    if (!pick_tile(row_tiles, col_tiles, rt, ct)) return;
    const RowTile tile = row_tile(P, rt, BN);
    if (tile.t < 0) return;
    const int KB = P.KB, rows = (int)(tile.r1 - tile.r0), steps = (KB + kStep - 1) / kStep;
    const int c0 = ct * BM, cols = P.Fo - c0 < BM ? P.Fo - c0 : BM;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wm = w % WM, wn = w / WM;

    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    const LoadW lw(P.w_codes + (tile.t * P.Fo + c0) * KB * 16, P.w_words + tile.t * steps * P.Fo + c0,
                   P.Fo, cols, KB);
    const LoadX lx(P.x_codes + tile.r0 * KB * 16, P.x_words + tile.r0, P.N, rows, KB);
    // Step k, from buffer k % 3: its loads have arrived when only those of step k+1 are
    // left; behind the barrier everybody is done with buffer (k+2) % 3.
    const auto step = [&](TileBuffer<BM>& Wb, TileBuffer<BN>& Xb, TileBuffer<BM>& Wn,
                          TileBuffer<BN>& Xn, int k) {
        if (k + 1 < steps) wait_loads<LoadW::LOADS + LoadX::LOADS>();
        else wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        if (k + 2 < steps) {
            lw.fetch(Wn, k + 2);
            lx.fetch(Xn, k + 2);
        }
        multiply<FM, FN, BM, BN>(Wb, Xb, wm, wn, lane, acc);
    };
    lw.fetch(W0, 0);
    lx.fetch(X0, 0);
    if (steps > 1) {
        lw.fetch(W1, 1);
        lx.fetch(X1, 1);
    }
    for (int k = 0; k < steps; k += 3) {
        step(W0, X0, W2, X2, k);
        if (k + 1 < steps) step(W1, X1, W0, X0, k + 1);
        if (k + 2 < steps) step(W2, X2, W1, X1, k + 2);
    }
    __syncthreads();  // everybody is done with the buffers
    uint8_t* const own = w == 0 ? W0.codes : (w == 1 ? W1.codes : (w == 2 ? W2.codes : X0.codes));
    static_assert(WAVES == 4 && sizeof(X0.codes) >= kOut * 4, "a buffer a wavefront");
    store_tile<FM, FN, BF>(P, acc, wm, wn, tile.r0, rows, c0, cols, reinterpret_cast<float*>(own));
}

// ---- few rows ------------------------------------------------------------------------------
// A workgroup has 16 output columns and up to 16 rows of a segment; its four
// wavefronts take steps of four blocks (k = 128) in turn, weights straight from
// memory, kThinDeep loads in flight, and their sums are added in LDS.  (16 rows of 8
// experts of 2048 x 4096, 36 MB of weights: 10.9 us.)
constexpr int kThinRows = 16, kThinCols = 16, kThinDeep = 4;

template <bool BF>
__global__ __launch_bounds__(kBlock) void mx_thin(MxParams P) {
    __shared__ f32x4 s_acc[4][kWave];
    const RowTile tile = row_tile(P, blockIdx.y, kThinRows);
    if (tile.t < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int KB = P.KB, rows = (int)(tile.r1 - tile.r0);
    const int c0 = blockIdx.x * kThinCols, cols = P.Fo - c0 < kThinCols ? P.Fo - c0 : kThinCols;
    const int row = lane & 15, blk = lane >> 4;
    const int64_t wr = tile.t * P.Fo + c0 + (row < cols ? row : cols - 1);
    const int64_t xr = tile.r0 + (row < rows ? row : rows - 1);
    const uint4* wc = reinterpret_cast<const uint4*>(P.w_codes) + wr * KB;
    const uint4* xc = reinterpret_cast<const uint4*>(P.x_codes) + xr * KB;
    const uint8_t* ws = P.w_scales + wr * KB;
    const uint8_t* xs = P.x_scales + xr * KB;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int kb0 = w * 4; kb0 < KB; kb0 += 16 * kThinDeep) {
        uint4 a[kThinDeep], b[kThinDeep];
        int sa[kThinDeep], sb[kThinDeep];
#pragma unroll
        for (int i = 0; i < kThinDeep; ++i) {
            const int kb = kb0 + 16 * i + blk;
            const bool in = kb < KB;
            const int k = in ? kb : KB - 1;
            a[i] = wc[k];
            b[i] = xc[k];
            sa[i] = in ? ws[k] : 0;  // (2^-127 on both sides: products vanish)
            sb[i] = in ? xs[k] : 0;
        }
#pragma unroll
        for (int i = 0; i < kThinDeep; ++i)
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                operand(a[i]), operand(b[i]), acc, kFp4, kFp4, 0, sa[i], 0, sb[i]);
    }
    s_acc[w][lane] = acc;
    __syncthreads();
    if (w) return;
    f32x4 s = s_acc[0][lane];
#pragma unroll
    for (int i = 1; i < 4; ++i) s += s_acc[i][lane];
    if (row >= rows) return;
    const int64_t at = (tile.r0 + row) * P.Fo + c0;
    const int c = 4 * blk;
    const float v[4] = {s[0], s[1], s[2], s[3]};
    if (c + 4 <= cols) {
        store4<BF>(P.out, at + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < cols) store_col<BF>(P.out, at + c + e, v[e]);
    }
}

// ---- few output columns -------------------------------------------------------------------
// The weights of a segment (CT column tiles of 32, KS steps of two blocks) stay in
// LDS while a workgroup goes through a run of the segments' row tiles.  Each
// wavefront has 32 rows to itself: it quantises them into its own part of LDS
// (lanes along the row, so that loads are whole lines), multiplies, and hands the
// results back through the same LDS, to write rows of out in whole pieces.
// No wavefront waits for another but when the segment changes.  (2.6M bf16 rows, 128
// -> 128, calls in a row: 314 us, 4.3 TB/s; quantised in a pass of its own 606 us.)
constexpr int kNarrowRows = 32, kNarrowTile = 32 * 4;  // rows of a wavefront, of a workgroup
constexpr int kNarrowCols = 4;                         // column tiles of a pass (accumulators)
// floats to a row of results in LDS: two rows of a store lie on other banks
constexpr int kNarrowLine = 32 * kNarrowCols + 4;

// Bytes of LDS: weights, their scales, and per wavefront codes and scales of its rows or
// its results.
struct NarrowShape {
    int cols, steps;  // padded: column tiles, steps of 64 along k
    int mask, shift;  // of the order of a row's pieces
    size_t w_codes, w_scales, wave, bytes;
    // Place of a 16-byte piece within row r: exchanged in groups of a power of two that
    // divides the row, so that 16 rows' pieces lie on different banks.
    __device__ int at(int r, int piece) const { return piece ^ ((r >> shift) & mask); }
};
__host__ __device__ inline NarrowShape narrow_shape(int KB, int Fo) {
    NarrowShape h;
    h.cols = (Fo + 31) / 32;
    h.steps = (KB + 1) / 2;
    const int pieces = 2 * h.steps;
    int g = 2;
    h.shift = 3;
    while (g < 16 && pieces % (2 * g) == 0) {
        g *= 2;
        --h.shift;
    }
    h.mask = g - 1;
    h.w_codes = (size_t)h.cols * 32 * h.steps * 32;
    h.w_scales = (size_t)h.cols * 32 * h.steps * 2;
    const size_t in = (size_t)kNarrowRows * h.steps * (32 + 2);
    const size_t out = (size_t)kNarrowRows * kNarrowLine * 4;
    h.wave = in > out ? in : out;
    h.wave = (h.wave + 15) & ~(size_t)15;
    h.bytes = h.w_codes + ((h.w_scales + 15) & ~(size_t)15) + 4 * h.wave;
    return h;
}

template <typename T, bool BF>
__global__ __launch_bounds__(kBlock) void mx_narrow(MxParams P, int64_t row_tiles) {
    extern __shared__ __attribute__((aligned(16))) uint8_t s_mem[];
    const NarrowShape h = narrow_shape(P.KB, P.Fo);
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int pieces = 2 * h.steps;  // 16-byte pieces, blocks, of a row
    uint8_t* s_wc = s_mem;
    uint8_t* s_ws = s_wc + h.w_codes;
    uint8_t* mine = s_ws + ((h.w_scales + 15) & ~(size_t)15) + w * h.wave;
    uint8_t* s_xc = mine;
    uint8_t* s_xs = s_xc + kNarrowRows * pieces * 16;
    float* s_out = reinterpret_cast<float*>(mine);
    const int row = lane & 31, half = lane >> 5;
    const int64_t first = row_tiles * blockIdx.x / gridDim.x;
    const int64_t last = row_tiles * (blockIdx.x + 1) / gridDim.x;
    int64_t have = -1;  // the segment whose weights are in LDS
    RowTile tile{-1, 0, 0, 0};
    for (int64_t rt = first; rt < last; ++rt) {
        if (tile.r1 < tile.end) {  // (the next of the same segment)
            tile.r0 = tile.r1;
            tile.r1 = tile.r0 + kNarrowTile < tile.end ? tile.r0 + kNarrowTile : tile.end;
        } else {
            tile = row_tile(P, rt, kNarrowTile);
        }
        if (tile.t < 0) return;  // (the same for the whole workgroup: no tile follows)
        if (tile.t != have) {
            __syncthreads();  // the others are done with the old weights
            const uint8_t* wc = P.w_codes + tile.t * P.Fo * P.KB * 16;
            const uint8_t* ws = P.w_scales + tile.t * P.Fo * P.KB;
            for (int i = tid; i < h.cols * 32 * pieces; i += kBlock) {
                const int c = i / pieces, k = i - c * pieces;
                const bool in = c < P.Fo && k < P.KB;
                uint4 v = make_uint4(0, 0, 0, 0);
                if (in) v = reinterpret_cast<const uint4*>(wc)[(int64_t)c * P.KB + k];
                reinterpret_cast<uint4*>(s_wc)[c * pieces + h.at(c, k)] = v;
                s_ws[c * pieces + k] = in ? ws[(int64_t)c * P.KB + k] : 0;
            }
            __syncthreads();
            have = tile.t;
        }
        const int64_t r0 = tile.r0 + w * kNarrowRows;
        const int rows = tile.r1 - r0 < kNarrowRows ? (int)(tile.r1 - r0) : kNarrowRows;
        if (rows <= 0) continue;
        // eight values a lane: four lanes a block, `per` lanes a row
        const int per = 4 * pieces, units = kNarrowRows * per;
        const typename T::raw* x = static_cast<const typename T::raw*>(P.x) + r0 * P.ldx;
        for (int i0 = 0; i0 < units; i0 += 4 * kWave) {
            RawOf<T, 8> v[4];
            int r[4], j[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * kWave + lane;
                r[u] = i / per;
                j[u] = i - r[u] * per;
                const int rc = r[u] < rows ? r[u] : rows - 1;  // (rows past the end are not stored)
                v[u] = load8<T>(x + rc * P.ldx, 8 * j[u], P.K);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint32_t sc;
                const uint32_t c = quantize8<T>(v[u], sc);
                if (i0 + u * kWave + lane < units) {
                    const int k = j[u] >> 2;
                    reinterpret_cast<uint32_t*>(s_xc)[(r[u] * pieces + h.at(r[u], k)) * 4 + (j[u] & 3)] = c;
                    if ((j[u] & 3) == 0) s_xs[r[u] * pieces + k] = (uint8_t)sc;
                }
            }
        }
        wave_sync();
        for (int ct0 = 0; ct0 < h.cols; ct0 += kNarrowCols) {
            f32x16 acc[kNarrowCols];
#pragma unroll
            for (int i = 0; i < kNarrowCols; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][v] = 0.f;
            for (int st = 0; st < h.steps; ++st) {
                const int k = 2 * st + half;
                const i32x8 b = operand(
                    reinterpret_cast<const uint4*>(s_xc)[row * pieces + h.at(row, k)]);
                const int sb = s_xs[row * pieces + k];
#pragma unroll
                for (int i = 0; i < kNarrowCols; ++i) {
                    if (ct0 + i < h.cols) {
                        const int c = (ct0 + i) * 32 + row;
                        const i32x8 a = operand(
                            reinterpret_cast<const uint4*>(s_wc)[c * pieces + h.at(c, k)]);
                        acc[i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                            a, b, acc[i], kFp4, kFp4, 0, (int)s_ws[c * pieces + k], 0, sb);
                    }
                }
            }
            const int cols = P.Fo - ct0 * 32 < 32 * kNarrowCols ? P.Fo - ct0 * 32 : 32 * kNarrowCols;
            if (ct0 + kNarrowCols >= h.cols) {
                // the last columns: the rows' codes make room for the results
                wave_sync();
#pragma unroll
                for (int i = 0; i < kNarrowCols; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float4 v = make_float4(acc[i][4 * q], acc[i][4 * q + 1],
                                                     acc[i][4 * q + 2], acc[i][4 * q + 3]);
                        *reinterpret_cast<float4*>(&s_out[row * kNarrowLine + i * 32 + 8 * q + 4 * half]) = v;
                    }
                wave_sync();
                constexpr int E = BF ? 8 : 4;  // columns of a 16-byte store
                const int64_t o0 = r0 * P.Fo + ct0 * 32;
                const int per_row = (cols + E - 1) / E;
                for (int i = lane; i < rows * per_row; i += kWave) {
                    const int rr = i / per_row, c = (i - rr * per_row) * E;
                    float v[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) v[e] = s_out[rr * kNarrowLine + c + e];
                    const int64_t o = o0 + (int64_t)rr * P.Fo + c;
                    if (c + E <= cols) {
                        if (BF) store_floats<BF16, E>(static_cast<uint16_t*>(P.out) + o, v);
                        else store_floats<F32, E>(static_cast<float*>(P.out) + o, v);
                    } else {
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (c + e < cols) store_col<BF>(P.out, o + e, v[e]);
                    }
                }
                wave_sync();
            } else if (row < rows) {
#pragma unroll
                for (int i = 0; i < kNarrowCols; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float v[4] = {acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2],
                                            acc[i][4 * q + 3]};
                        store4<BF>(P.out, (r0 + row) * P.Fo + (ct0 + i) * 32 + 8 * q + 4 * half, v);
                    }
            }
        }
    }
}

}  // namespace

hipError_t launch_mx_quantize(const void* x, int dtype, int64_t N, int64_t K, int64_t ldx,
                              uint8_t* codes, uint8_t* scales, void* values, hipStream_t s) {
    if (N <= 0) return hipSuccess;
    const int64_t per = 4 * ceil_div(K, kMxBlock);
    const int64_t rpb = per >= 4 * kBlock ? 1 : 4 * kBlock / per;
    const int64_t groups = ceil_div(N, rpb);
    const dim3 g((unsigned)(groups < (1 << 22) ? groups : (1 << 22))), b(kBlock);
    if (dtype == MP_BF16)
        hipLaunchKernelGGL(mx_quantize<BF16>, g, b, 0, s, static_cast<const uint16_t*>(x), N, (int)K,
                           ldx, (int)rpb, reinterpret_cast<uint32_t*>(codes), scales,
                           static_cast<uint16_t*>(values));
    else
        hipLaunchKernelGGL(mx_quantize<F32>, g, b, 0, s, static_cast<const float*>(x), N, (int)K,
                           ldx, (int)rpb, reinterpret_cast<uint32_t*>(codes), scales,
                           static_cast<float*>(values));
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t N, int64_t K,
                                void* out, int dtype, hipStream_t s) {
    if (N <= 0) return hipSuccess;
    const int64_t per = 4 * ceil_div(K, kMxBlock);
    const int64_t rpb = per >= 4 * kBlock ? 1 : 4 * kBlock / per;
    const int64_t groups = ceil_div(N, rpb);
    const dim3 g((unsigned)(groups < (1 << 22) ? groups : (1 << 22))), b(kBlock);
    const uint32_t* c = reinterpret_cast<const uint32_t*>(codes);
    if (dtype == MP_BF16)
        hipLaunchKernelGGL(mx_dequantize<BF16>, g, b, 0, s, c, scales, N, (int)K, (int)rpb,
                           static_cast<uint16_t*>(out));
    else
        hipLaunchKernelGGL(mx_dequantize<F32>, g, b, 0, s, c, scales, N, (int)K, (int)rpb,
                           static_cast<float*>(out));
    return hipGetLastError();
}

// Tiles of BM rows that segments of N rows can have at most: every segment that
// has rows may end in a part of one.
static int64_t row_tiles_bound(int64_t T, int64_t N, int64_t BM) {
    return N / BM + (T < N ? T : N);
}
static int64_t row_tiles_bound(const MxParams& p, int64_t BM) {
    return row_tiles_bound(p.T, p.N, BM);
}

template <int FM, int FN, int WM, int WN>
static hipError_t tiles(const MxParams& p, int bf, hipStream_t s) {
    const int64_t rt = row_tiles_bound(p, 32 * FN * WN), ct = ceil_div(p.Fo, 32 * FM * WM);
    const dim3 g((unsigned)(ceil_div(rt * ct, 8) * 8)), b(64 * WM * WN);
    if (bf) hipLaunchKernelGGL((mx_tiles<FM, FN, WM, WN, true>), g, b, 0, s, p, rt, (int)ct);
    else hipLaunchKernelGGL((mx_tiles<FM, FN, WM, WN, false>), g, b, 0, s, p, rt, (int)ct);
    return hipGetLastError();
}

// The smaller tiles are taken for fewer than 512 of these, two to a CU.  (4096 -> 4096, wide
// and smaller: 256 tiles 41 and 38 us, 384 tiles 50 and 50, 512 tiles 58 and 65.)
static int64_t wide_tiles(int64_t T, int64_t N, int64_t Fo) {
    return row_tiles_bound(T, N, 128) * ceil_div(Fo, 256);
}

// At most 256 columns and 96 KB of LDS (weights and four wavefronts' rows): one read
// of x, and no codes in memory.  (1M bf16 rows against tiles: 128 -> 128 127 and 211
// us.  Past 80 KB a CU has one workgroup: 128 -> 256 274 and 224 us, but 16 and 22 for
// 20,000 rows, where one launch instead of three counts.)
static bool is_narrow(const NarrowShape& h, int64_t Fo) {
    return Fo <= 256 && h.bytes <= (96 << 10);
}

// A launch has fewer than 2^32 threads, and a tile 256 of them.
bool mx_product_fits(int64_t T, int64_t N, int64_t K, int64_t Fo) {
    return is_narrow(narrow_shape((int)ceil_div(K, kMxBlock), (int)Fo), Fo) ||
           wide_tiles(T, N, Fo) <= (1 << 24) - 8;
}

hipError_t launch_mx_product(const MxParams& p, int x_dtype, int out_dtype, hipStream_t s) {
    if (p.N <= 0) return hipSuccess;
    const int bf = out_dtype == MP_BF16;
    // Where segments have 16 rows on average each is a thin tile.  (8 types, 4096 -> 4096,
    // thin against tiles: 8 rows each 31 and 32 us, 16 rows 36 and 35, 18 rows 55 and 36.
    // One type: 32 rows 18 and 25, and thin would lead up to 64, 21 and 26.)
    const bool few = p.N <= 16 * p.T + 16;
    const NarrowShape h = narrow_shape(p.KB, p.Fo);
    if (!few && is_narrow(h, p.Fo)) {
        const int64_t rt = row_tiles_bound(p, kNarrowTile);
        // as many workgroups as the CUs hold at once, with 160 KB of LDS each: never more
        // than two (a workgroup has 66 KB for its wavefronts' results alone)
        const int64_t most = 256 * (h.bytes <= (80 << 10) ? 2 : 1);
        const dim3 g((unsigned)(rt < most ? rt : most)), b(kBlock);
        if (x_dtype == MP_BF16) {
            if (bf) hipLaunchKernelGGL((mx_narrow<BF16, true>), g, b, h.bytes, s, p, rt);
            else hipLaunchKernelGGL((mx_narrow<BF16, false>), g, b, h.bytes, s, p, rt);
        } else {
            if (bf) hipLaunchKernelGGL((mx_narrow<F32, true>), g, b, h.bytes, s, p, rt);
            else hipLaunchKernelGGL((mx_narrow<F32, false>), g, b, h.bytes, s, p, rt);
        }
        return hipGetLastError();
    }
    hipError_t e = launch_mx_quantize(p.x, x_dtype, p.N, p.K, p.ldx, p.x_codes, p.x_scales, nullptr,
                                      s);
    if (e != hipSuccess) return e;
    // few rows a segment: the weights are what is read
    if (few) {
        // (at most 8193 row tiles, as T <= 4096)
        const dim3 g((unsigned)ceil_div(p.Fo, kThinCols), (unsigned)row_tiles_bound(p, kThinRows)),
            b(kBlock);
        if (bf) hipLaunchKernelGGL(mx_thin<true>, g, b, 0, s, p);
        else hipLaunchKernelGGL(mx_thin<false>, g, b, 0, s, p);
        return hipGetLastError();
    }
    const int KS = (int)ceil_div(p.KB, kStep);
    const ScaleTable wt{p.w_scales, p.w_words, p.T * p.Fo, p.Fo};
    const ScaleTable xt{p.x_scales, p.x_words, p.N, p.N};
    const int64_t ba = ceil_div(wt.R, kBlock), bb = ceil_div(xt.R, kBlock);
    hipLaunchKernelGGL(mx_scale_words, dim3((unsigned)(ba + bb), (unsigned)ceil_div(KS, 4)),
                       dim3(kBlock), 0, s, wt, xt, p.KB, KS, ba);
    return wide_tiles(p.T, p.N, p.Fo) >= 512 ? tiles<4, 2, 2, 2>(p, bf, s) : tiles<2, 2, 2, 2>(p, bf, s);
}

}  // namespace mp
