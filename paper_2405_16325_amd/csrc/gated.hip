// What a gated layer and a backward pass in 8 bits do element by element:
//
//     gated_bwd    a = act(g), d = act'(g):   du = dh a    dg = dh u d    h = a u         from g, u as bf16 or as 8-bit blocks
//     checkpoint   x -> e4m3 codes and a scale byte per 32 elements of a row (gated.h)
//     restore      back; exact, since what a code stands for is a bf16 number
//
// One pass over the data, bound by memory: the lanes of a wavefront have neighbouring pieces of 8 elements, 16 bytes of bf16 or 8 of
// codes.
#include "gated.h"

namespace {

constexpr int THREADS = 256;

// Piece `t` after piece c of row `row`, rows of P pieces
struct Piece { int64_t row; int c; };
__device__ __forceinline__ Piece piece_after(int64_t row, uint32_t c, uint32_t t, uint32_t P) {
    const uint32_t v = c + t, down = v / P;
    return {row + down, (int)(v - down * P)};
}

struct GatedBwd {
    const bf16_t *dh, *gu;                                    // gu: or null
    const uint8_t *q, *bytes;
    bf16_t *dgu, *h;                                          // h: or null
    int64_t n;
    int d_ff, act;
};

template <int ACT, bool Q8>
__device__ __forceinline__ void gated_bwd_piece(const GatedBwd& j, int64_t row, int c) {
    const size_t at = (size_t)row * j.d_ff + c * 8, pair = (size_t)row * (2 * (size_t)j.d_ff) + c * 8;
    F8 g, u;
    const F8 dh = unpack_bf16(*(const u32x4*)(j.dh + at));
    if (Q8) {
        const size_t blocks = ((size_t)j.d_ff + Q8_BLOCK - 1) / Q8_BLOCK;
        const uint8_t* const byte = j.bytes + (size_t)row * 2 * blocks + c / 4;
        g = unpack_e4m3(*(const u32x2*)(j.q + pair), scale_of_byte(byte[0]));
        u = unpack_e4m3(*(const u32x2*)(j.q + pair + j.d_ff), scale_of_byte(byte[blocks]));
    } else {
        g = unpack_bf16(*(const u32x4*)(j.gu + pair));
        u = unpack_bf16(*(const u32x4*)(j.gu + pair + j.d_ff));
    }
    F8 dg, du, h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const ActValue v = act_gradient<ACT>(g.v[i]);
        dg.v[i] = dh.v[i] * u.v[i] * v.d;
        du.v[i] = dh.v[i] * v.a;
        h.v[i] = v.a * u.v[i];
    }
    *(u32x4*)(j.dgu + pair) = pack_bf16(dg);
    *(u32x4*)(j.dgu + pair + j.d_ff) = pack_bf16(du);
    if (j.h) *(u32x4*)(j.h + at) = pack_bf16(h);
}

template <bool Q8>
__global__ void __launch_bounds__(THREADS) gated_bwd_kernel(GatedBwd j) {
    const uint32_t P = (uint32_t)j.d_ff / 8;
    const int64_t first = flat_block() * THREADS, row0 = first / P;
    const Piece p = piece_after(row0, (uint32_t)(first - row0 * P), threadIdx.x, P);
    if (p.row >= j.n) return;
    with_act(j.act, [&](auto act) { gated_bwd_piece<decltype(act)::value, Q8>(j, p.row, p.c); });
}

// rows of P pieces, whole blocks of four: those past the row's end are none
__global__ void __launch_bounds__(THREADS) checkpoint_kernel(const bf16_t* __restrict__ x, int64_t rows, int d, uint8_t* __restrict__ q,
                                                             uint8_t* __restrict__ bytes) {
    const uint32_t blocks = ((uint32_t)d + Q8_BLOCK - 1) / Q8_BLOCK, P = 4 * blocks;
    const int64_t first = flat_block() * THREADS, row0 = first / P;
    const Piece p = piece_after(row0, (uint32_t)(first - row0 * P), threadIdx.x, P);
    const bool has = p.row < rows && p.c * 8 < d;
    const size_t at = (size_t)p.row * d + p.c * 8;
    u32x4 in = {0u, 0u, 0u, 0u};
    if (has) in = *(const u32x4*)(x + at);
    F8 v = unpack_bf16(in);
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max_abs(top, v.v[i]);
    uint32_t bits = __float_as_uint(top);                     // a block is four neighbouring lanes
    bits = MaxBits()(bits, dpp<DPP_XOR1>(bits));
    bits = MaxBits()(bits, dpp<DPP_XOR2>(bits));
    if (!has) return;
    const BlockScale s = block_scale(bits);
#pragma unroll
    for (int i = 0; i < 8; ++i) v.v[i] = s.scaled(v.v[i]);
    *(u32x2*)(q + at) = pack_e4m3(v);
    if ((p.c & 3) == 0) bytes[(size_t)p.row * blocks + p.c / 4] = (uint8_t)s.byte;
}

__global__ void __launch_bounds__(THREADS) restore_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ bytes, int64_t rows, int d,
                                                          bf16_t* __restrict__ x) {
    const uint32_t P = (uint32_t)d / 8;
    const int64_t first = flat_block() * THREADS, row0 = first / P;
    const Piece p = piece_after(row0, (uint32_t)(first - row0 * P), threadIdx.x, P);
    if (p.row >= rows) return;
    const size_t at = (size_t)p.row * d + p.c * 8, blocks = ((size_t)d + Q8_BLOCK - 1) / Q8_BLOCK;
    *(u32x4*)(x + at) = pack_bf16(unpack_e4m3(*(const u32x2*)(q + at), scale_of_byte(bytes[(size_t)p.row * blocks + p.c / 4])));
}

inline int64_t groups(int64_t pieces) { return (pieces + THREADS - 1) / THREADS; }

}  // namespace

// (callers have checked that the pieces' launches fit: ELEMENTS_MAX)
hipError_t launch_gated_bwd(const bf16_t* dh, const bf16_t* gu, const uint8_t* q, const uint8_t* bytes, int64_t n, int64_t d_ff, int act,
                            bf16_t* dgu, bf16_t* h, hipStream_t s) {
    const GatedBwd j = {dh, gu, q, bytes, dgu, h, n, (int)d_ff, act};
    const dim3 grid = grid_of(groups(n * (d_ff / 8)));
    if (gu) gated_bwd_kernel<false><<<grid, dim3(THREADS), 0, s>>>(j);
    else gated_bwd_kernel<true><<<grid, dim3(THREADS), 0, s>>>(j);
    return hipGetLastError();
}

hipError_t launch_checkpoint_q8(const bf16_t* x, int64_t rows, int64_t d, uint8_t* q, uint8_t* bytes, hipStream_t s) {
    checkpoint_kernel<<<grid_of(groups(rows * ((d + Q8_BLOCK - 1) / Q8_BLOCK * 4))), dim3(THREADS), 0, s>>>(x, rows, (int)d, q, bytes);
    return hipGetLastError();
}

hipError_t launch_restore_q8(const uint8_t* q, const uint8_t* bytes, int64_t rows, int64_t d, bf16_t* x, hipStream_t s) {
    restore_kernel<<<grid_of(groups(rows * (d / 8))), dim3(THREADS), 0, s>>>(q, bytes, rows, (int)d, x);
    return hipGetLastError();
}
