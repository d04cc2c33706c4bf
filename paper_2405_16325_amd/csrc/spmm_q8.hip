// The 2:4 sparse product on 8-bit operands,
//
//     Y[b, d_out] = bf16( x_scale[b] w_scale[d_out] sum_k X[b, k] W[d_out, k]  (+ add[b, d_out]) ),
//
// X in e4m3 with a scale per token (what the norm writes), W packed 2:4 in e4m3 with a scale per row, its metadata as it is.
// v_smfmac_f32_16x16x128_fp8_fp8 multiplies 16 rows of W by 16 tokens over 128 logical k; lane l holds
//     of W  row l % 16, packed bytes 16 (l / 16) .. + 15 (logical k 32 (l / 16) ..) and the 4 metadata bytes of that stretch,
//     of X  token l % 16, k 16 (l / 16) .. + 15 and 64 + that,
//     of D  token l % 16, rows 4 (l / 16) .. + 3.
// The instruction adds its 64 products with fewer bits than fp32 has: a sum is off by up to about 2^-14 of its largest
// product (measured), below what rounding the operands to 8 bits costs.  Sums over instructions are fp32.
#include "pipeline.h"
#include "wave.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
union AQ { i32x4 v; u32x4 u; uint32_t w[4]; };
union BQ { i32x8 v; u32x4 u[2]; u32x2 h[4]; };

struct Q8Product {
    const uint8_t* x;          // e4m3[n][K]
    const float* xs;
    int64_t n;
    const uint8_t* a;          // e4m3[m][K / 2]
    const uint8_t* am;         // u8[m][K / 8]
    const float* as;
    int64_t m, K;
    const bf16_t* add;         // or null
    bf16_t* y;
};

constexpr int KSTEP = 128;
constexpr uint32_t META_NONE = 0x44444444u;                    // a legal pair in every group

// Any extents (K % 8 == 0).  Four wavefronts of 32 rows x 32 tokens, operands straight from memory in pieces of 8 logical k,
// each of which is inside its row as a whole.
__global__ void __launch_bounds__(256) q8_generic_kernel(Q8Product p, int64_t tiles_m) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, lq = lane >> 4;
    const int64_t block = flat_block();
    const int64_t m0 = block % tiles_m * 64 + (wave & 1) * 32, n0 = block / tiles_m * 64 + (wave >> 1) * 32;
    if (m0 >= p.m || n0 >= p.n) return;
    f32x4 acc[2][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t k0 = 0; k0 < p.K; k0 += KSTEP) {
        AQ af[2];
        uint32_t meta[2];
        BQ bf[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t row = m0 + i * 16 + l16, k = k0 + 32 * lq;
            meta[i] = META_NONE;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                af[i].w[g] = 0;
                if (row < p.m && k + 8 * g < p.K) {
                    af[i].w[g] = *(const uint32_t*)(p.a + (row * p.K + k) / 2 + 4 * g);
                    meta[i] = (meta[i] & ~(0xFFu << (8 * g))) | (uint32_t)p.am[(row * p.K + k) / 8 + g] << (8 * g);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t tok = n0 + j * 16 + l16;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int64_t k = k0 + 16 * lq + 64 * (g >> 1) + 8 * (g & 1);
                bf[j].h[g] = (u32x2){0, 0};
                if (tok < p.n && k < p.K) bf[j].h[g] = *(const u32x2*)(p.x + tok * p.K + k);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = __builtin_amdgcn_smfmac_f32_16x16x128_fp8_fp8(af[i].v, bf[j].v, acc[i][j], (int)meta[i], 0, 0);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t tok = n0 + j * 16 + l16;
        if (tok >= p.n) continue;
        const float xs = p.xs[tok];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t row = m0 + i * 16 + lq * 4;
            if (row >= p.m) continue;                            // m is a multiple of 8: four rows are inside or outside
            const f32x4 ws = *(const f32x4*)(p.as + row);
            u32x2 add = {0, 0};
            if (p.add) add = *(const u32x2*)(p.add + tok * p.m + row);
            union { __bf16 h[4]; u32x2 u; } o;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t half = add[k >> 1];
                const float t = __uint_as_float((k & 1) ? half & 0xFFFF0000u : half << 16);
                o.h[k] = (__bf16)(p.add ? fmaf(acc[i][j][k] * xs, ws[k], t) : acc[i][j][k] * xs * ws[k]);
            }
            *(u32x2*)(p.y + tok * p.m + row) = o.u;
        }
    }
}

// One wavefront a row: packed bf16 values to e4m3 with the row's scale.  half = d_in / 2, a multiple of 4.
__global__ void __launch_bounds__(256) quantize_packed_kernel(const bf16_t* __restrict__ vals, int64_t rows, int64_t half,
                                                              uint8_t* __restrict__ q, float* __restrict__ scale) {
    const int lane = threadIdx.x & 63;
    const int64_t row = flat_block() * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const bf16_t* const from = vals + row * half;
    float top = 0.0f;
    for (int64_t i = lane * 4; i < half; i += 256) {
        const u32x2 v = *(const u32x2*)(from + i);
#pragma unroll
        for (int k = 0; k < 2; ++k) top = max_abs(max_abs(top, __uint_as_float(v[k] << 16)), __uint_as_float(v[k] & 0xFFFF0000u));
    }
    const Q8Scale s = q8_scale(lanes_max_abs<64>(top));
    if (lane == 0) scale[row] = s.scale;
    for (int64_t i = lane * 4; i < half; i += 256) {
        const u32x2 v = *(const u32x2*)(from + i);
        int o = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(v[0] << 16) * s.inv, __uint_as_float(v[0] & 0xFFFF0000u) * s.inv, 0, false);
        o = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(v[1] << 16) * s.inv, __uint_as_float(v[1] & 0xFFFF0000u) * s.inv, o, true);
        *(uint32_t*)(q + row * half + i) = (uint32_t)o;
    }
}

}  // namespace

hipError_t launch_quantize_packed(const bf16_t* vals, int64_t rows, int64_t cols, uint8_t* q, float* scale, hipStream_t s) {
    quantize_packed_kernel<<<grid_of((rows + 3) / 4), 256, 0, s>>>(vals, rows, cols / 2, q, scale);
    return hipGetLastError();
}

size_t spmm_q8_workspace_bytes(int64_t n, int64_t m, int64_t K) {
    (void)n; (void)m; (void)K;
    return 0;
}

hipError_t launch_spmm_q8(const uint8_t* x, const float* xs, int64_t n, const uint8_t* a, const uint8_t* am, const float* as,
                          int64_t m, int64_t K, const bf16_t* add, bf16_t* y, float* partial_or_null, hipStream_t s) {
    (void)partial_or_null;
    const Q8Product p = {x, xs, n, a, am, as, m, K, add, y};
    const int64_t tiles_m = (m + 63) / 64, tiles = tiles_m * ((n + 63) / 64);
    if (!grid_fits(tiles)) return hipErrorInvalidConfiguration;
    q8_generic_kernel<<<grid_of(tiles), 256, 0, s>>>(p, tiles_m);
    return hipGetLastError();
}
