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

constexpr int THREADS = 256;      // (of a workgroup, in pieces: one to two per thread)
// STREAM: a call that moves more than the last-level cache holds, of which the next one would find nothing there
template <bool STREAM, class T>
__device__ __forceinline__ T load(const void* p) { return STREAM ? __builtin_nontemporal_load((const T*)p) : *(const T*)p; }
template <bool STREAM, class T>
__device__ __forceinline__ void store(void* p, T v) {
    if (STREAM) __builtin_nontemporal_store(v, (T*)p);
    else *(T*)p = v;
}

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

template <bool Q8, bool STREAM>
__global__ void __launch_bounds__(THREADS) gated_bwd_kernel(GatedBwd j) {
    const uint32_t P = (uint32_t)j.d_ff / 8;
    const int64_t first = flat_block() * THREADS, row0 = first / P;
    const Piece p = piece_after(row0, (uint32_t)(first - row0 * P), threadIdx.x, P);
    if (p.row >= j.n) return;
    const size_t at = (size_t)p.row * j.d_ff + p.c * 8, pair = (size_t)p.row * (2 * (size_t)j.d_ff) + p.c * 8;
    F8 g, u;
    const u32x4 dh_bits = load<STREAM, u32x4>(j.dh + at);
    if (Q8) {
        const size_t blocks = ((size_t)j.d_ff + Q8_BLOCK - 1) / Q8_BLOCK;
        const uint8_t* const byte = j.bytes + (size_t)p.row * 2 * blocks + p.c / 4;
        const uint32_t gb = byte[0], ub = byte[blocks];
        const u32x2 gq = load<STREAM, u32x2>(j.q + pair), uq = load<STREAM, u32x2>(j.q + pair + j.d_ff);
        g = unpack_bf16(restored_bf16(gq, gb));
        u = unpack_bf16(restored_bf16(uq, ub));
    } else {
        const u32x4 gv = load<STREAM, u32x4>(j.gu + pair), uv = load<STREAM, u32x4>(j.gu + pair + j.d_ff);
        g = unpack_bf16(gv);
        u = unpack_bf16(uv);
    }
    const F8 dh = unpack_bf16(dh_bits);
    F8 dg, du, h;
    with_act(j.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const ActValue v = act_gradient<decltype(act)::value>(g.v[i]);
            dg.v[i] = dh.v[i] * u.v[i] * v.d;
            du.v[i] = dh.v[i] * v.a;
            h.v[i] = v.a * u.v[i];
        }
    });
    store<STREAM>(j.dgu + pair, pack_bf16(dg));
    store<STREAM>(j.dgu + pair + j.d_ff, pack_bf16(du));
    if (j.h) store<STREAM>(j.h + at, pack_bf16(h));
}

// rows of P pieces, whole blocks of four: those past the row's end are none.  PER pieces per thread, THREADS apart.
template <int PER, bool STREAM>
__global__ void __launch_bounds__(THREADS) checkpoint_kernel(const bf16_t* __restrict__ x, int64_t rows, int d, uint8_t* __restrict__ q,
                                                             uint8_t* __restrict__ bytes) {
    const uint32_t blocks = ((uint32_t)d + Q8_BLOCK - 1) / Q8_BLOCK, P = 4 * blocks;
    const int64_t first = flat_block() * (THREADS * PER), row0 = first / P;
    u32x4 in[PER];
    Piece p[PER];
    bool has[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        p[i] = piece_after(row0, (uint32_t)(first - row0 * P), threadIdx.x + i * THREADS, P);
        has[i] = p[i].row < rows && p[i].c * 8 < d;
        in[i] = (u32x4){0u, 0u, 0u, 0u};
        if (has[i]) in[i] = load<STREAM, u32x4>(x + (size_t)p[i].row * d + p[i].c * 8);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const F8 v = unpack_bf16(in[i]);
        uint32_t bits = top_of(v.v);                          // a block is four neighbouring lanes
        bits = MaxBits()(bits, dpp<DPP_XOR1>(bits));
        bits = MaxBits()(bits, dpp<DPP_XOR2>(bits));
        const BlockScale s = block_scale(bits);
        uint32_t codes[2];
        block_codes(v.v, s, codes);
        if (has[i]) {
            store<STREAM>(q + (size_t)p[i].row * d + p[i].c * 8, (u32x2){codes[0], codes[1]});
            if ((p[i].c & 3) == 0) bytes[(size_t)p[i].row * blocks + p[i].c / 4] = (uint8_t)s.byte;
        }
    }
}

template <int PER, bool STREAM>
__global__ void __launch_bounds__(THREADS) restore_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ bytes, int64_t rows, int d,
                                                          bf16_t* __restrict__ x) {
    const uint32_t P = (uint32_t)d / 8;
    const int64_t first = flat_block() * (THREADS * PER), row0 = first / P;
    const size_t blocks = ((size_t)d + Q8_BLOCK - 1) / Q8_BLOCK;
    u32x2 in[PER];
    uint32_t byte[PER];
    Piece p[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        p[i] = piece_after(row0, (uint32_t)(first - row0 * P), threadIdx.x + i * THREADS, P);
        if (p[i].row >= rows) continue;
        in[i] = load<STREAM, u32x2>(q + (size_t)p[i].row * d + p[i].c * 8);
        byte[i] = bytes[(size_t)p[i].row * blocks + p[i].c / 4];
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (p[i].row < rows) store<STREAM>(x + (size_t)p[i].row * d + p[i].c * 8, restored_bf16(in[i], byte[i]));
}

inline dim3 grid_for(int64_t pieces, int per) { return grid_of((pieces + THREADS * per - 1) / (THREADS * per)); }
inline bool streams(int64_t bytes) { return bytes > (int64_t)LAST_LEVEL_CACHE_BYTES; }
// Two pieces per thread to and from 8 bits, unless there are few: us, one / two, 777 x 1000 2.7 / 2.9 and 2.5 / 3.0, 2048 x 2560 6.0 / 5.6
// and 5.95 / 5.8, 16384 x 9216 88 / 78 and 84 / 79 (four: 6.4, 6.6; 77, 81).  The gradient, which has three to five loads a piece, is slower
// with two (2048 x 6912 from codes 29.0 / 30.6; 16384 x 24576 694 / 711).
constexpr int64_t PAIRS_FROM = (int64_t)1 << 18;

// Rows of P = Kp / 8 pieces of eight of the contraction: first the tokens' (16 bytes each), then the packed weight's (8 bytes, and a byte of
// metadata).  Past K: zeros, under metadata that names positions 0 and 1, a legal pair.
struct PadJob {
    const bf16_t *x, *vals;
    const uint8_t* meta;
    bf16_t *xp, *vp;
    uint8_t* mp;
    int64_t n, rows;
    int K, Kp;
};
__global__ void __launch_bounds__(THREADS) pad_kernel(PadJob j) {
    const uint32_t P = (uint32_t)j.Kp / 8, have = (uint32_t)j.K / 8;
    const int64_t first = flat_block() * THREADS, row0 = first / P;
    const Piece p = piece_after(row0, (uint32_t)(first - row0 * P), threadIdx.x, P);
    const bool in = (uint32_t)p.c < have;
    if (p.row < j.n) {
        u32x4 v = {0u, 0u, 0u, 0u};
        if (in) v = *(const u32x4*)(j.x + (size_t)p.row * j.K + p.c * 8);
        *(u32x4*)(j.xp + (size_t)p.row * j.Kp + p.c * 8) = v;
        return;
    }
    const int64_t row = p.row - j.n;
    if (row >= j.rows) return;
    u32x2 v = {0u, 0u};
    uint8_t byte = 0x44;
    if (in) {
        v = *(const u32x2*)((const uint8_t*)j.vals + (size_t)row * j.K + p.c * 8);
        byte = j.meta[(size_t)row * have + p.c];
    }
    *(u32x2*)((uint8_t*)j.vp + (size_t)row * j.Kp + p.c * 8) = v;
    j.mp[(size_t)row * P + p.c] = byte;
}

}  // namespace

hipError_t launch_pad_operands(const bf16_t* x, int64_t n, const bf16_t* vals, const uint8_t* meta, int64_t rows, int64_t K, int64_t Kp,
                               bf16_t* xp, bf16_t* vp, uint8_t* mp, hipStream_t s) {
    pad_kernel<<<grid_for((n + rows) * (Kp / 8), 1), dim3(THREADS), 0, s>>>({x, vals, meta, xp, vp, mp, n, rows, (int)K, (int)Kp});
    return hipGetLastError();
}

// (callers have checked that the pieces' launches fit.  16384 x 24576, non-temporal accesses or not: 694 / 698 us from codes, 805 / 844 from bf16)
hipError_t launch_gated_bwd(const bf16_t* dh, const bf16_t* gu, const uint8_t* q, const uint8_t* bytes, int64_t n, int64_t d_ff, int act,
                            bf16_t* dgu, bf16_t* h, hipStream_t s) {
    const GatedBwd j = {dh, gu, q, bytes, dgu, h, n, (int)d_ff, act};
    const bool stream = streams(n * d_ff * (6 + (h ? 2 : 0) + (gu ? 4 : 2)));
    auto kern = gu ? (stream ? gated_bwd_kernel<false, true> : gated_bwd_kernel<false, false>)
                   : (stream ? gated_bwd_kernel<true, true> : gated_bwd_kernel<true, false>);
    kern<<<grid_for(n * (d_ff / 8), 1), dim3(THREADS), 0, s>>>(j);
    return hipGetLastError();
}

hipError_t launch_checkpoint_q8(const bf16_t* x, int64_t rows, int64_t d, uint8_t* q, uint8_t* bytes, hipStream_t s) {
    const int64_t pieces = rows * ((d + Q8_BLOCK - 1) / Q8_BLOCK * 4);
    const int per = pieces < PAIRS_FROM ? 1 : 2;
    auto kern = per == 1 ? checkpoint_kernel<1, false> : streams(3 * rows * d) ? checkpoint_kernel<2, true> : checkpoint_kernel<2, false>;
    kern<<<grid_for(pieces, per), dim3(THREADS), 0, s>>>(x, rows, (int)d, q, bytes);
    return hipGetLastError();
}

hipError_t launch_restore_q8(const uint8_t* q, const uint8_t* bytes, int64_t rows, int64_t d, bf16_t* x, hipStream_t s) {
    const int64_t pieces = rows * (d / 8);
    const int per = pieces < PAIRS_FROM ? 1 : 2;
    auto kern = per == 1 ? restore_kernel<1, false> : streams(3 * rows * d) ? restore_kernel<2, true> : restore_kernel<2, false>;
    kern<<<grid_for(pieces, per), dim3(THREADS), 0, s>>>(q, bytes, rows, (int)d, x);
    return hipGetLastError();
}
