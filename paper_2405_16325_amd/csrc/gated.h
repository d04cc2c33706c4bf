// What a gated feed-forward layer's kernels share: activations, the order of its weight rows, 8-bit blocks, the tile kernels' epilogue.
//
//     h = act(g) u          g, u = the two halves of a product with a weight of 2 d_ff rows, the gate's first
//
// A tile of a product holds pairs of 16 x 16 fragments, 16 rows of the gate and the same 16 of the up projection (GATE_GROUP): the
// kernel's rows are "virtual" ones, 16 and 16 in turn, which the loads of the weight translate (gated_row), so that a lane has g and u
// of the same four elements in its own registers and h needs no exchange.  m, the number of virtual rows, is 2 d_ff rounded up to
// whole groups.
#pragma once
#include <type_traits>

#include "pipeline.h"
#include "wave.h"

struct GateOut {
    int d_ff, count, act;                                     // elements of a row, those of the launch (a part starts at a multiple of 128)
    bf16_t* gu;                                               // bf16[n][2 d_ff], or null
    uint8_t *q, *bytes;                                       // e4m3[2 n][d_ff] with a scale byte per 32 of a row, or null
    float* sums;                                              // small-batch kernels: [n][2 d_ff] instead of h, or null
    __host__ __device__ bool keeps() const { return gu || q; }
};
constexpr int GATE_GROUP = 16;
inline int64_t gated_rows(int64_t d_ff) { return (d_ff + GATE_GROUP - 1) / GATE_GROUP * (2 * GATE_GROUP); }

// virtual row -> element of h that it belongs to (d_ff or more: none), half (0 gate, 1 up)
__device__ __forceinline__ int gated_element(int row) { return (row >> 5) * GATE_GROUP + (row & (GATE_GROUP - 1)); }
__device__ __forceinline__ int gated_half(int row) { return row >> 4 & 1; }
// row of the weight that is read for a virtual row; d_ff is a multiple of 8, so a group may have eight rows too many: the eight before
__device__ __forceinline__ int gated_row(int row, const GateOut& gate) {
    const int e = gated_element(row);
    return (e < gate.count ? e : e - 8) + (gated_half(row) ? gate.d_ff : 0);
}

// The weight's row for row `row` of a tile, of a plain product (no gate) and of a gated one
__device__ __forceinline__ int weight_row(int row, int m) { return wrap_row(row, m); }
__device__ __forceinline__ int weight_row(int row, int m, const GateOut& gate) { return gated_row(wrap_row(row, m), gate); }
__device__ __forceinline__ int weight_row_near(int row, int m) { return wrap_row_near(row, m); }
__device__ __forceinline__ int weight_row_near(int row, int m, const GateOut& gate) { return gated_row(wrap_row_near(row, m), gate); }

// ---- activations.  sigmoid by the hardware's exponential and reciprocal (each within 1 ulp; the exponent's rounding adds |x| 2^-24):
// results are rounded to bf16 or multiplied by what was.
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }
constexpr float GELU_SCALE = 1.5957691216057308f, GELU_CUBE = 0.044715f;      // 2 sqrt(2 / pi)

// a = act(g), d = act'(g)
//   silu: g s(g)    gelu: g (1 + tanh(z)) / 2 = g s(2 z), z = sqrt(2 / pi) (g + 0.044715 g^3)    relu: max(g, 0)
struct ActValue { float a, d; };
template <int ACT>
__device__ __forceinline__ float act_value(float g) {
    if (ACT == SLOPE_ACT_RELU) return g <= 0.0f ? 0.0f : g;   // NaN stays NaN
    if (ACT == SLOPE_ACT_SILU) return g * sigmoid(g);
    return g * sigmoid(GELU_SCALE * (g + GELU_CUBE * g * g * g));
}
template <int ACT>
__device__ __forceinline__ ActValue act_gradient(float g) {
    if (ACT == SLOPE_ACT_RELU) {
        const float a = g <= 0.0f ? 0.0f : g;
        return {a, g > 0.0f ? 1.0f : a};                      // (NaN for NaN)
    }
    if (ACT == SLOPE_ACT_SILU) {
        const float s = sigmoid(g);
        return {g * s, s * (1.0f + g * (1.0f - s))};
    }
    const float s = sigmoid(GELU_SCALE * (g + GELU_CUBE * g * g * g));
    // s (1 - s) is zero long before 16, where g^2 could begin to pass fp32's range
    const float t = fminf(fabsf(g), 16.0f);
    return {g * s, s + g * (s * (1.0f - s)) * GELU_SCALE * (1.0f + 3.0f * GELU_CUBE * t * t)};
}
// f(std::integral_constant<int, ACT>) for the activation of a call: one branch, which all lanes share
template <class F>
__device__ __forceinline__ void with_act(int act, F f) {
    if (act == SLOPE_ACT_SILU) f(std::integral_constant<int, SLOPE_ACT_SILU>{});
    else if (act == SLOPE_ACT_GELU) f(std::integral_constant<int, SLOPE_ACT_GELU>{});
    else f(std::integral_constant<int, SLOPE_ACT_RELU>{});
}

// ---- 8 bits with a power of two per 32 elements.  The scale is the smallest power of two (from 2^-126 on) that leaves no magnitude
// above 448 = 1.75 2^8, held as exponent + 127; 255: the block has an infinity or NaN and reads as NaN.  Scaling by a power of two is
// exact, so a code is the value rounded once to e4m3 (half a step: 2^-4 of it, 2^-10 of the scale below 2^-6 of it), and what it stands
// for is a bf16 number: under the largest scale, 2^120, values stop at 240, since 256 would be 2^128.
constexpr int Q8_BLOCK = 32;
struct BlockScale {
    uint32_t byte;
    __device__ __forceinline__ float inverse() const { return __uint_as_float((byte == 255u ? 0u : 254u - byte) << 23); }
    __device__ __forceinline__ float clamped(float v) const {
        const float most = byte == 247u ? 240.0f : Q8_MAX;
        return __builtin_amdgcn_fmed3f(v * inverse(), -most, most);
    }
};
__device__ __forceinline__ BlockScale block_scale(uint32_t top) {             // bits of the largest magnitude
    const int e = (int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u);
    return {top >= 0x7F800000u ? 255u : (uint32_t)(e > 1 ? e : 1)};
}
// Bits of the largest magnitude, NaN above all: one instruction for two values
template <int N>
__device__ __forceinline__ uint32_t top_of(const float (&v)[N]) {
    float top = __builtin_elementwise_maximum(__builtin_fabsf(v[0]), __builtin_fabsf(v[1]));
#pragma unroll
    for (int e = 2; e < N; e += 2) top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top, __builtin_fabsf(v[e])), __builtin_fabsf(v[e + 1]));
    return __float_as_uint(top) & 0x7FFFFFFFu;
}
// Codes of N values, four to a word.  The conversion divides by the scale itself; with magnitudes of 448 scale at most it needs no clamp.  Blocks of the
// largest scale, and those that read as NaN, which no lane of a wavefront has as a rule, take the long way.
template <int N>
__device__ __forceinline__ void block_codes(const float (&v)[N], const BlockScale& s, uint32_t (&o)[N / 4]) {
    if (__any(s.byte >= 247u)) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const int p = __builtin_amdgcn_cvt_pk_fp8_f32(s.clamped(v[4 * i]), s.clamped(v[4 * i + 1]), 0, false);
            o[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(s.clamped(v[4 * i + 2]), s.clamped(v[4 * i + 3]), p, true);
        }
        return;
    }
    const float scale = __uint_as_float(s.byte << 23);
    typedef short s16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        s16x2 p = {0, 0};
        p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, v[4 * i], v[4 * i + 1], scale, false);
        p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, v[4 * i + 2], v[4 * i + 3], scale, true);
        o[i] = __builtin_bit_cast(uint32_t, p);
    }
}
// eight codes -> eight bf16 numbers, exactly: one instruction for two of them, which takes the scale's exponent
__device__ __forceinline__ u32x4 restored_bf16(u32x2 codes, uint32_t byte) {
    const float scale = __uint_as_float(byte << 23);
    union { __attribute__((ext_vector_type(2))) __bf16 h[4]; u32x4 u; } o;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        o.h[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], scale, false);
        o.h[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], scale, true);
    }
    return o.u;
}
// an activation in this form, as an operand of the weight gradient
struct BlocksX { const uint8_t *q, *bytes; };

// ---- results.  Four elements e .. e + 3 of token `tok` from their sums; eight neighbouring lanes have a block of 32 of a token (all of
// them make the call, elements from the launch's last on being none).
__device__ __forceinline__ u32x2 four_bf16(const f32x4& v) {
    union { __bf16 h[4]; u32x2 u; } o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o.h[e] = (__bf16)v[e];
    return o.u;
}
__device__ __forceinline__ void finish_gated(const f32x4& g, const f32x4& u, int tok, int e, int n, bf16_t* __restrict__ H, const GateOut& gate) {
    const bool has = tok < n && e < gate.count;
    const size_t at = (size_t)tok * gate.d_ff + e;
    f32x4 h;
    with_act(gate.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = act_value<decltype(act)::value>(g[i]) * u[i];
    });
    if (has) *(u32x2*)(H + at) = four_bf16(h);
    if (gate.gu && has) {
        bf16_t* const row = gate.gu + (size_t)tok * (2 * (size_t)gate.d_ff) + e;
        *(u32x2*)row = four_bf16(g);
        *(u32x2*)(row + gate.d_ff) = four_bf16(u);
    }
    if (gate.q) {
        const float gv[4] = {g[0], g[1], g[2], g[3]}, uv[4] = {u[0], u[1], u[2], u[3]};
        const BlockScale sg = block_scale(lanes_reduce<8>(e < gate.count ? top_of(gv) : 0u, MaxBits()));
        const BlockScale su = block_scale(lanes_reduce<8>(e < gate.count ? top_of(uv) : 0u, MaxBits()));
        uint32_t gq[1], uq[1];
        block_codes(gv, sg, gq);
        block_codes(uv, su, uq);
        if (!has) return;
        uint8_t* const row = gate.q + (size_t)tok * (2 * (size_t)gate.d_ff) + e;
        *(uint32_t*)row = gq[0];
        *(uint32_t*)(row + gate.d_ff) = uq[0];
        if ((e & (Q8_BLOCK - 1)) == 0) {
            const size_t blocks = ((size_t)gate.d_ff + Q8_BLOCK - 1) / Q8_BLOCK;
            uint8_t* const byte = gate.bytes + (size_t)tok * 2 * blocks + e / Q8_BLOCK;
            byte[0] = (uint8_t)sg.byte;
            byte[blocks] = (uint8_t)su.byte;
        }
    }
}

// The largest of the four quarters of 16 lanes, lane by lane: rows of the register exchanged without an LDS round trip
__device__ __forceinline__ uint32_t quarters_max(uint32_t v) {
    const auto far = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = MaxBits()(far[0], far[1]);
    const auto near = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return MaxBits()(near[0], near[1]);
}
// Everybody's LDS accesses are done; stores to memory go on.
__device__ __forceinline__ void lds_barrier() {
    WAIT_HERE(waitcnt_imm(63, 0));
    wg_barrier();
}

// A tile's results, BMT virtual rows (BMT / 2 elements) x BNT tokens, by THREADS threads: like store_rows through LDS, since whole rows
// of a tile leave in whole lines.  h, then the codes, converted while h is on its way (together with h, us: 2048 tokens, 13824 x 2560 108.3 / 105.6, 16384,
// 18432 x 2560 942 / 928), then bf16 projections.  All threads make the call.
// What is kept is for the backward pass, long after, and passes the caches by, but for codes that fit a quarter of the last-level one beside
// others' (us, 16384 tokens, 18432 x 2560, bf16 924 -> 875, codes 931 -> 901; 2048, 13824 x 2560, bf16 111 -> 107, codes 107 -> 105 but, with the
// gradient right behind, 128.5 -> 131).  The tiles of a round end together, so that their results are a burst at the memory's rate, 5 us for the
// projections of 256 tiles of 256 x 256 in bf16; codes are half of it and as long again in conversions (16384, 4096 x 768: h 86, with bf16
// 102, with codes 104).
template <int MF, int NF, int BMT, int BNT, int THREADS>
__device__ __forceinline__ void store_gated(const f32x4 (&acc)[MF][NF], int f0, int t0, int n, int l16, int lq, bf16_t* __restrict__ H,
                                            uint8_t* smem, int tile_f0, int tile_t0, const GateOut& gate) {
    static_assert(MF % 2 == 0, "pairs of fragments");
    constexpr int HALF = BMT / 2;                             // elements of h in the tile
    constexpr int CODES = BNT * (BMT + 16);                   // where the codes are staged, behind h
    const int tile_e0 = tile_f0 / 2, e0 = f0 / 2, d_ff = gate.d_ff, count = gate.count;
    const int le = e0 - tile_e0 + lq * 4, lt = t0 - tile_t0 + l16;        // the lane's first element and token inside the tile
    // rows of BYTES bytes per token at `from` in LDS, piece by piece of 16 bytes, to to(token, piece, its bytes)
    auto leave = [&](auto bytes, const uint8_t* from, auto to) {
        constexpr int BYTES = decltype(bytes)::value, CP = BYTES + 16, PPR = BYTES / 16, PIECES = BNT * PPR;
        constexpr int PER_THREAD = (PIECES + THREADS - 1) / THREADS;
        constexpr bool EVEN = PIECES % THREADS == 0;
        u32x4 piece[PER_THREAD];
#pragma unroll
        for (int u = 0; u < PER_THREAD; ++u) {
            const int idx = (int)threadIdx.x + u * THREADS;
            if (EVEN || idx < PIECES) piece[u] = *(const u32x4*)(from + (idx / PPR) * CP + (idx % PPR) * 16);
        }
#pragma unroll
        for (int u = 0; u < PER_THREAD; ++u) {
            const int idx = (int)threadIdx.x + u * THREADS, tok = tile_t0 + idx / PPR;
            if ((EVEN || idx < PIECES) && tok < n) to(tok, idx % PPR, piece[u]);
        }
    };
    __syncthreads();                                          // every wavefront is done with the rings / the staged factor
    with_act(gate.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int i = 0; i < MF / 2; ++i) {
                f32x4 h;
#pragma unroll
                for (int x = 0; x < 4; ++x) h[x] = act_value<decltype(act)::value>(acc[2 * i][j][x]) * acc[2 * i + 1][j][x];
                *(u32x2*)(smem + (lt + j * 16) * (BMT + 16) + (le + i * 16) * 2) = four_bf16(h);
            }
    });
    lds_barrier();
    leave(std::integral_constant<int, BMT>{}, smem, [&](int tok, int p, const u32x4& v) {
        const int e = tile_e0 + p * 8;
        if (e < count) *(u32x4*)(H + (size_t)tok * d_ff + e) = v;
    });
    const size_t blocks = ((size_t)d_ff + Q8_BLOCK - 1) / Q8_BLOCK;
    if constexpr (MF % 4 == 0) if (gate.q) {                  // whole blocks in a wavefront's rows: no other tile is given codes to write
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int c = 0; c < MF / 4; ++c)                  // blocks: fragments 4 c (gate), 4 c + 2 (gate), and the up projection's
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const f32x4 &a = acc[4 * c + half][j], &b = acc[4 * c + 2 + half][j];
                    const int e = e0 + c * 32;                // the block's first element
                    float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
                    if (tile_e0 + HALF > count)               // uniform: elements past the last are none
#pragma unroll
                        for (int x = 0; x < 8; ++x) v[x] = e + x / 4 * 16 + lq * 4 < count ? v[x] : 0.0f;
                    const BlockScale s = block_scale(quarters_max(top_of(v)));
                    uint32_t codes[2];
                    block_codes(v, s, codes);
                    uint8_t* const at = smem + CODES + (lt + j * 16) * (BMT + 16) + half * HALF + le + c * 32;
                    *(uint32_t*)at = codes[0];
                    *(uint32_t*)(at + 16) = codes[1];
                    const int tok = t0 + j * 16 + l16;
                    if (lq == 0 && tok < n && e < count) gate.bytes[((size_t)tok * 2 + half) * blocks + e / Q8_BLOCK] = (uint8_t)s.byte;
                }
    }
    const bool large = (size_t)n * d_ff > LAST_LEVEL_CACHE_BYTES / 8;
    if constexpr (MF % 4 == 0) if (gate.q) {
        lds_barrier();
        leave(std::integral_constant<int, BMT>{}, smem + CODES, [&](int tok, int p, const u32x4& v) {
            const int half = p * 16 / HALF, e = tile_e0 + p * 16 % HALF;
            uint8_t* const to = gate.q + (size_t)tok * (2 * (size_t)d_ff) + half * (size_t)d_ff + e;
            // d_ff is a multiple of 8: a row's codes may start 8 bytes off, and its last piece may be half a one
            if (e + 8 < count && large) __builtin_nontemporal_store((u32x4_a8)v, (u32x4_a8*)to);
            else if (e + 8 < count) *(u32x4_a8*)to = v;
            else if (e < count) *(u32x2*)to = (u32x2){v[0], v[1]};
        });
    }
    if (gate.gu) {                                            // uniform
        lds_barrier();
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int i = 0; i < MF; ++i)
                *(u32x2*)(smem + (lt + j * 16) * (2 * BMT + 16) + ((i & 1) * HALF + le + (i >> 1) * 16) * 2) = four_bf16(acc[i][j]);
        lds_barrier();
        leave(std::integral_constant<int, 2 * BMT>{}, smem, [&](int tok, int p, const u32x4& v) {
            const int half = p * 8 / HALF, e = tile_e0 + p * 8 % HALF;
            if (e < count) __builtin_nontemporal_store(v, (u32x4*)(gate.gu + (size_t)tok * (2 * (size_t)d_ff) + half * (size_t)d_ff + e));
        });
    }
}
