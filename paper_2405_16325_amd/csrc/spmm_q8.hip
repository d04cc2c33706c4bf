// The 2:4 sparse product on 8-bit operands,
//
//     Y[b, d_out] = bf16( x_scale[b] w_scale[d_out] sum_k X[b, k] W[d_out, k]  (+ add[b, d_out]) ),
//
// X in e4m3 with a scale per token (what the norm writes), W packed 2:4 in e4m3 with a scale per row, its metadata as it is.
// v_smfmac_f32_16x16x128_fp8_fp8, in the general kernel below (the others take the 32 x 32 x 64 form; in register loops on Gaussian operands 7.3
// and 5.3 PFLOP/s dense-equivalent), multiplies 16 rows of W by 16 tokens over 128 logical k; lane l holds
//     of W  row l % 16, packed bytes 16 (l / 16) .. + 15 (logical k 32 (l / 16) ..) and the 4 metadata bytes of that stretch,
//     of X  token l % 16, k 16 (l / 16) .. + 15 and 64 + that,
//     of D  token l % 16, rows 4 (l / 16) .. + 3.
// The instruction adds its 64 products with fewer bits than fp32 has: a sum is off by up to about 2^-14 of its largest
// product (measured), below what rounding the operands to 8 bits costs.  Sums over instructions are fp32.
#include <type_traits>

#include "pipeline.h"
#include "wave.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
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
    int64_t ldy;               // of y and add: m, or that of the whole of which this is a part
};

// four rows' sums of a token to Y: scales, the added term, one rounding
__device__ __forceinline__ void store_quad(const Q8Product& p, int64_t tok, int64_t f, f32x4 s) {
    const f32x4 ws = *(const f32x4*)(p.as + f);
    const float xs = p.xs[tok];
    u32x2 add = {0, 0};
    if (p.add) add = *(const u32x2*)(p.add + tok * p.ldy + f);
    union { __bf16 h[4]; u32x2 u; } o;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float t = __uint_as_float((r & 1) ? add[r >> 1] & 0xFFFF0000u : add[r >> 1] << 16);
        o.h[r] = (__bf16)(p.add ? fmaf(s[r] * xs, ws[r], t) : s[r] * xs * ws[r]);
    }
    *(u32x2*)(p.y + tok * p.ldy + f) = o.u;
}

constexpr int KSTEP = 128;
// a raw buffer descriptor over `bytes` bytes; loads at offsets past them give zeros
typedef __amdgpu_buffer_rsrc_t buffer_t;
constexpr uint32_t NOWHERE = 0x80000000u;
__device__ __forceinline__ buffer_t tile_buffer(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
// 64 lanes x 16 bytes: lane l's bytes land at lds_dst + 16 * l; lds_dst and step are the same for all lanes
__device__ __forceinline__ void buffer_dma16(buffer_t from, uint8_t* lds_dst, uint32_t offset, int step) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (void __attribute__((address_space(3)))*)lds_dst, 16, (int)offset, step, 0, 0);
}
constexpr uint32_t META_NONE = 0x44444444u;                    // a legal pair in every group

// Any extents (K % 8 == 0): 32 rows x 32 tokens, whose k-steps four wavefronts take in turn, operands straight from memory in pieces
// of 8 logical k, each of which is inside its row as a whole; the sums are added through LDS, in order.  Latency bounds it where it
// is meant to be used: a wavefront's loads of a k-step are all under way together, and no second launch is needed.
__global__ void __launch_bounds__(256) q8_generic_kernel(Q8Product p, int64_t tiles_m, int64_t tiles) {
    __shared__ f32x4 sums[4][32][9];                            // [wavefront][token][four rows]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, lq = lane >> 4;
    const int64_t block = flat_block();
    if (block >= tiles) return;
    const int64_t m0 = block % tiles_m * 32, n0 = block / tiles_m * 32;
    f32x4 acc[2][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t k0 = wave * KSTEP; k0 < p.K; k0 += 4 * KSTEP) {
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
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) sums[wave][j * 16 + l16][i * 4 + lq] = acc[i][j];
    __syncthreads();
    const int t = threadIdx.x >> 3, q = threadIdx.x & 7;
    if (n0 + t >= p.n || m0 + 4 * q >= p.m) return;             // m is a multiple of 8: four rows are inside or outside
    f32x4 v = sums[0][t][q];
#pragma unroll
    for (int w = 1; w < 4; ++w) v += sums[w][t][q];
    store_quad(p, n0 + t, m0 + 4 * q, v);
}

// ------------------------------------------------------------------------------------------
// q8_tile_kernel: tiles of BM rows x BN tokens, K % 64 == 0 (TAIL: not of 128).  Four wavefronts, one per SIMD, WM along the rows, on
// v_smfmac_f32_32x32x64_fp8_fp8, whose lane l holds
//     of W  row l % 32, packed bytes 16 (l / 32) .. + 15 and the 4 metadata bytes of that stretch,
//     of X  token l % 32, k 16 (l / 32) .. + 15 and 32 + that,
//     of D  token l % 32, rows 8 i + 4 (l / 32) .. + 3, i = 0 .. 3.
// A k-step is 128 logical k: 64 bytes of a packed row, 16 of its metadata, 128 of a token.  Operands come by global -> LDS loads
// of whole 128-byte lines where they can: a compute unit has a fixed number of requests in flight, whatever their size, and that
// bounds the loop (requests of 64 bytes of W and 32 of metadata, in a ring of three k-steps: 1.61 ms for 8192 tokens, 36864 x 9216).
// So W comes by pairs of k-steps and metadata by four, two buffers of each, tokens by k-steps in two stages.  A wavefront reads the
// fragments of half a k-step while it multiplies the half before.  One barrier a k-step, as soon as the fragments of its second half
// are read: then everybody has left its buffers.  After it a wavefront queues, by k mod 4 (k: the k-step in work),
//     the tokens of k-step k + 2 and a quarter of a pair of W, which have landed at the next barrier, and then
//     1, 3: half of the pair of W after next      0: the next metadata block, which have not to.
// What bounds it: 52 KB of operands a k-step, which reach a compute unit at about 30 bytes a cycle in all variants tried (a ring of three
// k-steps with smaller requests, 256 x 192 tiles with two k-steps of look-ahead 13 % slower), at the 1.46 GHz that the power management
// leaves: 1.05 us a k-step, against 0.70 of products; and about 11 us before and after the loop of every tile (8192 tokens, 36864 x 9216:
// 1.52 ms, 3.7 PFLOP/s dense-equivalent, matrix pipes 52 % busy).
template <int BM, int BN>
struct Q8Smem {
    static constexpr int A = BM * 128, B = BN * 128, M = BM * 64;         // a pair of W, a k-step of tokens, a block of metadata
    static constexpr int B_OFF = 2 * A, M_OFF = B_OFF + 2 * B, TOTAL = M_OFF + 2 * M;
    static constexpr int OUT_PITCH = BM * 2 + 16;
    static constexpr int A_LOADS = BM / 32, B_LOADS = BN / 32, M_LOADS = BM / 64;    // a wavefront's
    static constexpr int QUARTER = A_LOADS / 4, HALF = A_LOADS / 2;
    // loads after the barrier of a k-step, k4 = k mod 4, and how many of them, the last, may still be under way at the next barrier
    static constexpr int loads(int k4) { return B_LOADS + QUARTER + late(k4); }
    static constexpr int late(int k4) { return k4 % 2 ? HALF : k4 == 0 ? M_LOADS : 0; }
    static_assert(TOTAL <= 160 * 1024 && BN * OUT_PITCH <= 160 * 1024, "fits");
    static_assert(QUARTER * 4 == A_LOADS && B_LOADS > 0 && M_LOADS > 0, "whole loads");
};

// slabs of `steps` of the `total` k-steps; more than one: fp32 sums to part[slab][token][row]
struct Q8Split { int slabs, steps, total; float* part; };

// A workgroup's tile and slab.  Slabs come one after the other, each XCD takes an equal run of all their tiles (32 tiles of 256 x 256 at
// most, the compute units it has), and so shares the k-steps of one slab or two in its cache.
inline unsigned q8_grid(int tiles_m, int tiles_n, int slabs) {
    return slabs > 1 ? (unsigned)((tiles_m * tiles_n * slabs + XCDS - 1) / XCDS * XCDS) : (unsigned)super_grid(tiles_m, tiles_n);
}
__device__ __forceinline__ bool q8_tile_of_block(int tiles_m, int tiles_n, int slabs, int& tm, int& tn, int& slab) {
    slab = 0;
    if (slabs == 1) return tile_of_block(tiles_m, tiles_n, tm, tn);
    const int tiles = tiles_m * tiles_n, count = tiles * slabs, b = (int)blockIdx.x;
    int t = b % XCDS * ((count + XCDS - 1) / XCDS) + b / XCDS;
    if (t >= count) return false;
    slab = t / tiles;
    t -= slab * tiles;
    if (tiles_m <= tiles_n) { tm = t % tiles_m; tn = t / tiles_m; }
    else { tn = t % tiles_n; tm = t / tiles_n; }
    return true;
}

template <int BM, int BN, int WM, bool TAIL>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, BM * BN > 128 * 128 ? 1 : 2)))
q8_tile_kernel(Q8Product p, int tiles_m, int tiles_n, Q8Split split) {
    using S = Q8Smem<BM, BN>;
    constexpr int WN = 4 / WM, MF = BM / (32 * WM), NF = BN / (32 * WN);
    extern __shared__ __align__(16) uint8_t smem[];
    int tm, tn, slab;
    if (!q8_tile_of_block(tiles_m, tiles_n, split.slabs, tm, tn, slab)) return;
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l32 = lane & 31, lq = lane >> 5, wm = wave % WM, wn = wave / WM;
    const int first = slab * split.steps;
    const int steps = min(split.steps, split.total - first);
    const int K = (int)p.K;

    // loader lanes, through buffer descriptors of the tile's rows: rows past the end read zeros and no memory
    const int rows = (int)min((int64_t)BM, p.m - m0), toks = (int)min((int64_t)BN, p.n - n0);
    const uint32_t a_pitch = (uint32_t)K / 2, b_pitch = (uint32_t)K, m_pitch = (uint32_t)K / 8;
    const buffer_t a_buf = tile_buffer(p.a + m0 * a_pitch, rows * a_pitch);
    const buffer_t b_buf = tile_buffer(p.x + n0 * b_pitch, toks * b_pitch);
    const buffer_t m_buf = tile_buffer(p.am + m0 * m_pitch, rows * m_pitch);
    uint32_t a_off[S::A_LOADS], b_off[S::B_LOADS], m_off[S::M_LOADS];
#pragma unroll
    for (int i = 0; i < S::A_LOADS; ++i) {                      // 8 rows a load, the 16-byte pieces of a row rotated
        const int r = (wave * S::A_LOADS + i) * 8 + (lane >> 3);
        a_off[i] = r < rows ? r * a_pitch + 16 * ((lane & 7) ^ ((r >> 1) & 7)) : NOWHERE;
    }
#pragma unroll
    for (int i = 0; i < S::B_LOADS; ++i) {
        const int r = (wave * S::B_LOADS + i) * 8 + (lane >> 3);
        b_off[i] = r < toks ? r * b_pitch + 16 * ((lane & 7) ^ ((r >> 1) & 7)) : NOWHERE;
    }
#pragma unroll
    for (int i = 0; i < S::M_LOADS; ++i) {                      // 16 rows a load
        const int r = (wave * S::M_LOADS + i) * 16 + (lane >> 2);
        m_off[i] = r < rows ? r * m_pitch + 16 * ((lane & 3) ^ ((r >> 2) & 3)) : NOWHERE;
    }
    // TAIL: the contraction ends inside a k-step; pieces past a row's end read zeros.  Pieces of a row, as its rows give them (rows
    // 16 apart alike): of an even and of an odd load.
    int piece[2];
    if (TAIL)
#pragma unroll
        for (int i = 0; i < 2; ++i) piece[i] = (lane & 7) ^ ((4 * i + (lane >> 4)) & 7);
    // Past the last k-step loads read zeros and no memory: they are counted upon.  The pieces that a last pair or block has too many
    // are the next row's (the last row's: zeros) and not used.
    auto issue_a = [&](int pair, int i) {
        uint32_t off = a_off[i] | (2 * pair >= steps ? NOWHERE : 0);
        if (TAIL) off |= piece[(wave * S::A_LOADS + i) & 1] * 32 >= K - (first + 2 * pair) * KSTEP ? NOWHERE : 0;
        buffer_dma16(a_buf, smem + (pair & 1) * S::A + (wave * S::A_LOADS + i) * 1024, off, first * 64 + pair * 128);
    };
    auto issue_b = [&](int k, int i) {
        uint32_t off = b_off[i] | (k >= steps ? NOWHERE : 0);
        if (TAIL) off |= piece[(wave * S::B_LOADS + i) & 1] * 16 >= K - (first + k) * KSTEP ? NOWHERE : 0;
        buffer_dma16(b_buf, smem + S::B_OFF + (k & 1) * S::B + (wave * S::B_LOADS + i) * 1024, off, (first + k) * KSTEP);
    };
    auto issue_m = [&](int block, int i) {
        buffer_dma16(m_buf, smem + S::M_OFF + (block & 1) * S::M + (wave * S::M_LOADS + i) * 1024, m_off[i] | (4 * block >= steps ? NOWHERE : 0),
                     first * 16 + block * 64);
    };

    // reader lanes
    const int a_row = wm * (BM / WM) + l32, b_row = wn * (BN / WN) + l32, sw = (l32 >> 1) & 7, m_sw = (l32 >> 2) & 3;
    const int a_rd = a_row * 128, b_rd = S::B_OFF + b_row * 128, m_rd = S::M_OFF + a_row * 64 + lq * 4;
    struct Reader { const uint8_t *a, *b[2], *e; };
    auto reader = [&](int k, int h) {                           // half h of k-step k
        const uint8_t *const pa = smem + ((k >> 1) & 1) * S::A + a_rd, *const pb = smem + (k & 1) * S::B + b_rd;
        return Reader{pa + (((4 * (k & 1) + 2 * h + lq) ^ sw) * 16), {pb + (((4 * h + lq) ^ sw) * 16), pb + (((4 * h + 2 + lq) ^ sw) * 16)},
                      smem + m_rd + ((k >> 2) & 1) * S::M + (((k & 3) ^ m_sw) * 16) + 8 * h};
    };
    struct Frags { AQ a[MF]; BQ b[NF]; uint32_t e[MF]; };
    constexpr int READS = 2 * (MF + NF);
    // read i of a half's fragments, in the order in which the products want them
    auto read = [&](Frags& f, const Reader& r, int i) {
        if (i == 0 || i > 2 * NF + 1) {
            const int q = i == 0 ? 0 : (i - 2 * NF) / 2;
            if (i % 2 == 0) f.a[q].u = *(const u32x4*)(r.a + q * 32 * 128);
            else f.e[q] = *(const uint32_t*)(r.e + q * 32 * 64);
        } else if (i == 1) {
            f.e[0] = *(const uint32_t*)r.e;
        } else {
            f.b[(i - 2) / 2].u[i & 1] = *(const u32x4*)(r.b[i & 1] + (i - 2) / 2 * 32 * 128);
        }
    };
    f32x16 acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    // Product i of a half.  With 16 fragments the accumulators fill all accumulation registers; left to itself the compiler keeps
    // some of them in the others and moves them back and forth, two hundred moves a k-step.  (The instruction is written out for
    // that; its wait states: two after a write of an operand by a vector instruction, here in front, and those of a read of the
    // result by one, after the loop.)
    auto multiply = [&](const Frags& f, int i) {
        f32x16& c = acc[i / NF][i % NF];
        if constexpr (MF * NF == 16) {
#ifdef __HIP_DEVICE_COMPILE__
            asm volatile("s_nop 1\n\tv_smfmac_f32_32x32x64_fp8_fp8 %0, %1, %2, %3" : "+a"(c) : "v"(f.a[i / NF].v), "v"(f.b[i % NF].v), "v"(f.e[i / NF]));
#endif
        } else {
            c = __builtin_amdgcn_smfmac_f32_32x32x64_fp8_fp8(f.a[i / NF].v, f.b[i % NF].v, c, (int)f.e[i / NF], 0, 0);
        }
    };
    // The products of a half with a share of n other things after each; the order is kept
    constexpr int PRODUCTS = MF * NF;
    auto share = [&](int i, int n, int over, auto&& f) {
        for (int u = (n * i + over - 1) / over; u < (n * (i + 1) + over - 1) / over && u < n; ++u) f(u);
    };

    constexpr int QUARTER = S::QUARTER, HALF = S::HALF;
    // load u after the barrier of k-step k, k4 = k mod 4
    auto load = [&](int k, int k4, int u) {
        if (u < S::B_LOADS) issue_b(k + 2, u);
        else if (k4 % 2 == 0 && u < S::B_LOADS + QUARTER) issue_a((k >> 1) + 1, QUARTER + HALF + u - S::B_LOADS);
        else if (k4 % 2 == 0) issue_m((k >> 2) + 1, u - S::B_LOADS - QUARTER);
        else issue_a((k >> 1) + 2, u - S::B_LOADS);
    };
    // what the k-steps before the first would have queued
#pragma unroll
    for (int i = 0; i < S::M_LOADS; ++i) issue_m(0, i);
#pragma unroll
    for (int i = 0; i < S::A_LOADS; ++i) issue_a(0, i);
#pragma unroll
    for (int i = 0; i < S::B_LOADS; ++i) issue_b(0, i);
#pragma unroll
    for (int i = 0; i < S::loads(3); ++i) load(-1, 3, i);
    WAIT_HERE(waitcnt_imm(S::loads(3), 15));
    wg_barrier();
    Frags f0, f1;
    {
        const Reader r = reader(0, 0);
#pragma unroll
        for (int i = 0; i < READS; ++i) read(f0, r, i);
    }
    // the barrier comes as soon as the fragments of the second half are read
    constexpr int BARRIER = PRODUCTS > 1 ? PRODUCTS * 5 / 8 : 1;
    auto step = [&](int k, auto mod4) {
        constexpr int K4 = decltype(mod4)::value;
        constexpr int MINE = S::loads(K4), AT_ONCE = PRODUCTS - BARRIER < MINE ? PRODUCTS - BARRIER : MINE;   // one a product, then evenly
        const Reader r1 = reader(k, 1);
#pragma unroll
        for (int i = 0; i < PRODUCTS; ++i) {
            if (i == BARRIER) {
                WAIT_HERE(waitcnt_imm(S::late((K4 + 3) % 4), 0));
                wg_barrier();
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(f0, i);
            if (i < BARRIER) share(i, READS, BARRIER > 2 ? BARRIER - 2 : 1, [&](int u) { read(f1, r1, u); });
            else if (i - BARRIER < AT_ONCE) load(k, K4, i - BARRIER);
        }
        if (BARRIER == PRODUCTS) {
            WAIT_HERE(waitcnt_imm(S::late((K4 + 3) % 4), 0));
            wg_barrier();
        }
        const Reader r0 = reader(k + 1, 0);
#pragma unroll
        for (int i = 0; i < PRODUCTS; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            multiply(f1, i);
            share(i, READS, PRODUCTS - PRODUCTS / 4, [&](int u) { read(f0, r0, u); });
            share(i, MINE - AT_ONCE, PRODUCTS, [&](int u) { load(k, K4, AT_ONCE + u); });
        }
    };
    int k = 0;
    for (; k + 3 < steps; k += 4) {
        step(k, std::integral_constant<int, 0>());
        step(k + 1, std::integral_constant<int, 1>());
        step(k + 2, std::integral_constant<int, 2>());
        step(k + 3, std::integral_constant<int, 3>());
    }
    if (k < steps) step(k, std::integral_constant<int, 0>());
    if (k + 1 < steps) step(k + 1, std::integral_constant<int, 1>());
    if (k + 2 < steps) step(k + 2, std::integral_constant<int, 2>());
#ifdef __HIP_DEVICE_COMPILE__
    if constexpr (MF * NF == 16) {
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j) asm volatile("" : "+a"(acc[i][j]));
    }
#endif

    // ---- results
    const int f_base = wm * (BM / WM) + 4 * lq, t_base = wn * (BN / WN) + l32;
    if (split.part) {
        WAIT_HERE(waitcnt_imm(0, 0));                           // the look-ahead loads
        float* const to = split.part + (int64_t)slab * p.n * p.m;
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t tok = n0 + t_base + 32 * j, f = m0 + f_base + 32 * i + 8 * q;
                    if (tok < p.n && f < p.m)
                        *(f32x4*)(to + tok * p.m + f) = (f32x4){acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                }
        return;
    }
    // The tile leaves in whole rows by way of LDS, and a term that is added comes the same way before.  Everything that is loaded is
    // under way together, from places clamped into the operands: with a branch around each of them the loads of the added term
    // came one after the other (777 tokens, 20480 x 5120: 27 us more than without the term).
    constexpr int PIECES = BN * (BM / 8), PER = PIECES / 256, BATCH = PER < 16 ? PER : 16;
    float xs[NF];
#pragma unroll
    for (int j = 0; j < NF; ++j) xs[j] = p.xs[min(n0 + t_base + 32 * j, p.n - 1)];
    const int piece_f = (int)threadIdx.x % (BM / 8) * 8, piece_tok = (int)threadIdx.x / (BM / 8);       // of the first piece; the next ones:
    constexpr int TOKS_ON = 256 / (BM / 8);                                                             // so many tokens on
    uint8_t* const piece_at = smem + piece_tok * S::OUT_PITCH + piece_f * 2;
    auto barrier = [&] {
        WAIT_HERE(waitcnt_imm(63, 0));
        wg_barrier();
    };
    if (p.add) {
        const bf16_t* const from = p.add + n0 * p.ldy + m0 + (piece_f < rows ? piece_f : 0);
#pragma unroll
        for (int b = 0; b < PER; b += BATCH) {
            u32x4 v[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) v[u] = *(const u32x4*)(from + min(piece_tok + (b + u) * TOKS_ON, toks - 1) * p.ldy);
            if (b == 0) {
                WAIT_HERE(waitcnt_imm(0, 0));                   // the look-ahead loads too
                wg_barrier();
            }
#pragma unroll
            for (int u = 0; u < BATCH; ++u) *(u32x4*)(piece_at + (b + u) * TOKS_ON * S::OUT_PITCH) = v[u];
        }
        barrier();
    } else {
        WAIT_HERE(waitcnt_imm(0, 0));
        wg_barrier();
    }
    // (with and without that term apart: a choice at every value cost 4 us of every tile; all scales of the rows ahead of that, 64 registers
    // more, 2 %)
    auto scale = [&](auto with_add) {
        constexpr bool ADD = decltype(with_add)::value;
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            f32x4 wq[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t f = m0 + f_base + 32 * i + 8 * q;
                wq[q] = *(const f32x4*)(p.as + (f < p.m ? f : 0));
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 ws = wq[q];
#pragma unroll
                for (int j = 0; j < NF; ++j) {
                    u32x2* const at = (u32x2*)(smem + (t_base + 32 * j) * S::OUT_PITCH + (f_base + 32 * i + 8 * q) * 2);
                    const u32x2 add = ADD ? *at : (u32x2){0, 0};
                    union { __bf16 h[4]; u32x2 u; } o;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float t = __uint_as_float((r & 1) ? add[r >> 1] & 0xFFFF0000u : add[r >> 1] << 16);
                        const float v = acc[i][j][4 * q + r] * xs[j];
                        o.h[r] = (__bf16)(ADD ? fmaf(v, ws[r], t) : v * ws[r]);
                    }
                    *at = o.u;
                }
            }
        }
    };
    if (p.add) scale(std::true_type());
    else scale(std::false_type());
    barrier();
    // a Y that the dies' second-level caches would not hold goes past them (777 tokens, 20480 x 5120 110 -> 105 us)
    const bool stream = p.n * p.ldy > ((int64_t)8 << 20);
    bf16_t* const to = p.y + n0 * p.ldy + m0 + piece_f;
#pragma unroll
    for (int b = 0; b < PER; b += BATCH) {
        u32x4 v[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) v[u] = *(const u32x4*)(piece_at + (b + u) * TOKS_ON * S::OUT_PITCH);
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int tok = piece_tok + (b + u) * TOKS_ON;
            if (tok >= toks || piece_f >= rows) continue;
            if (stream) __builtin_nontemporal_store(v[u], (u32x4*)(to + tok * p.ldy));
            else *(u32x4*)(to + tok * p.ldy) = v[u];
        }
    }
}

// ------------------------------------------------------------------------------------------
// q8_stream_kernel: up to TOK (4 or 8) tokens, K % 32 == 0: one pass over the packed weight, bound by memory.  A workgroup owns 32 rows
// and all tokens; its wavefronts take the stretches of 256 logical k in turn, each through a ring of its own in LDS, without a
// barrier, and add their sums through LDS at the end, in order.  Loads are of whole 128-byte lines of W: with operands straight to
// registers, where a load takes 16 bytes from each of 64 places, the address unit is the bound (1 token, 36864 x 9216: 54.6 us).
template <int TOK>
struct Q8Ring {
    static constexpr int M_OFF = 4096, X_OFF = M_OFF + 1024, STAGE = X_OFF + TOK * 256;
    static constexpr int X_LOADS = TOK / 4, LOADS = 5 + X_LOADS;
};
template <int TOK, int WAVES, int STAGES>
__global__ void __launch_bounds__(64 * WAVES) q8_stream_kernel(Q8Product p, Q8Split split) {
    using S = Q8Ring<TOK>;
    extern __shared__ __align__(16) uint8_t smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l32 = lane & 31, lq = lane >> 5;
    const int64_t m0 = (int64_t)blockIdx.x * 32;
    const int rows = (int)min((int64_t)32, p.m - m0), toks = (int)p.n;
    const int K = (int)p.K;
    const buffer_t a_buf = tile_buffer(p.a + m0 * (K / 2), rows * (K / 2));
    const buffer_t m_buf = tile_buffer(p.am + m0 * (K / 8), rows * (K / 8));
    const buffer_t x_buf = tile_buffer(p.x, toks * K);
    uint8_t* const ring = smem + wave * STAGES * S::STAGE;

    // loads: 8 rows of W, 32 rows' metadata, 4 tokens each; pieces of 16 bytes, a row's rotated
    uint32_t a_off[4], x_off[S::X_LOADS];
    int a_piece[2];                                             // of an even load, of an odd one
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 3), c = (lane & 7) ^ ((r >> 1) & 7);
        if (i < 2) a_piece[i] = c;
        a_off[i] = r < rows ? r * (K / 2) + 16 * c : NOWHERE;
    }
    const uint32_t m_off = (lane >> 1) < rows ? (lane >> 1) * (K / 8) + 16 * (lane & 1) : NOWHERE;
#pragma unroll
    for (int i = 0; i < S::X_LOADS; ++i) {
        const int t = 4 * i + (lane >> 4);
        x_off[i] = t < toks ? t * K + 16 * ((lane & 15) ^ (t & 15)) : NOWHERE;
    }
    const int first = (int)blockIdx.y * split.steps, last = min(first + split.steps, split.total);
    auto issue = [&](int s, int stage) {                        // zeros past the row's end and past the last stretch
        uint8_t* const to = ring + stage * S::STAGE;
        const int left = s < last ? K - s * 256 : 0;
        if (left >= 256) {
#pragma unroll
            for (int i = 0; i < 4; ++i) buffer_dma16(a_buf, to + i * 1024, a_off[i], s * 128);
            buffer_dma16(m_buf, to + S::M_OFF, m_off, s * 32);
#pragma unroll
            for (int i = 0; i < S::X_LOADS; ++i) buffer_dma16(x_buf, to + S::X_OFF + i * 1024, x_off[i], s * 256);
        } else {
            const int at = left > 0 ? s : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) buffer_dma16(a_buf, to + i * 1024, a_piece[i & 1] * 32 < left ? a_off[i] : NOWHERE, at * 128);
            buffer_dma16(m_buf, to + S::M_OFF, left > 0 ? m_off : NOWHERE, at * 32);
#pragma unroll
            for (int i = 0; i < S::X_LOADS; ++i) {
                const int c = (lane & 15) ^ ((4 * i + (lane >> 4)) & 15);
                buffer_dma16(x_buf, to + S::X_OFF + i * 1024, c * 16 < left ? x_off[i] : NOWHERE, at * 256);
            }
        }
    };
    const int tok = l32 < TOK ? l32 : TOK - 1;                  // lanes without a token: any one's values, not stored
    const int a_rd = l32 * 128, sw = (l32 >> 1) & 7, m_rd = S::M_OFF + l32 * 32 + 4 * lq, x_rd = S::X_OFF + tok * 256, x_sw = tok & 15;
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.0f;

    int s = first + wave, stage = 0;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) issue(s + i * WAVES, i);
    for (; s < last; s += WAVES) {
        WAIT_HERE(waitcnt_imm((STAGES - 2) * S::LOADS, 15));
        const uint8_t* const at = ring + stage * S::STAGE;
        AQ a[4];
        BQ x[4];
        uint32_t e[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            a[u].u = *(const u32x4*)(at + a_rd + (((2 * u + lq) ^ sw) * 16));
            e[u] = *(const uint32_t*)(at + m_rd + 8 * u);
            x[u].u[0] = *(const u32x4*)(at + x_rd + (((4 * u + lq) ^ x_sw) * 16));
            x[u].u[1] = *(const u32x4*)(at + x_rd + (((4 * u + 2 + lq) ^ x_sw) * 16));
        }
        issue(s + (STAGES - 1) * WAVES, stage == 0 ? STAGES - 1 : stage - 1);    // where the stretch before was
#pragma unroll
        for (int u = 0; u < 4; ++u) acc = __builtin_amdgcn_smfmac_f32_32x32x64_fp8_fp8(a[u].v, x[u].v, acc, (int)e[u], 0, 0);
        stage = stage == STAGES - 1 ? 0 : stage + 1;
        WAIT_HERE(waitcnt_imm(63, 0));                          // read before it is loaded into again
    }
    WAIT_HERE(waitcnt_imm(0, 0));
    __syncthreads();

    // lane: token l32, rows 8 q + 4 lq .. + 3
    constexpr int PITCH = 36;
    float (*const sums)[TOK][PITCH] = (float (*)[TOK][PITCH])smem;
    if (l32 < TOK)
#pragma unroll
        for (int q = 0; q < 4; ++q) *(f32x4*)&sums[wave][l32][8 * q + 4 * lq] = (f32x4){acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    for (int i = threadIdx.x; i < TOK * 8; i += 64 * WAVES) {
        const int t = i >> 3, r = (i & 7) * 4;
        if (t >= toks || r >= rows) continue;
        f32x4 v = *(const f32x4*)&sums[0][t][r];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += *(const f32x4*)&sums[w][t][r];
        if (split.part) *(f32x4*)(split.part + ((int64_t)blockIdx.y * p.n + t) * p.m + m0 + r) = v;
        else store_quad(p, t, m0 + r, v);
    }
}

// Y from the slabs' sums, added in order
__global__ void __launch_bounds__(256) q8_reduce_kernel(Q8Product p, const float* __restrict__ part, int slabs) {
    const int64_t quads = p.m / 4, i = (flat_block() * 256 + threadIdx.x);
    if (i >= p.n * quads) return;
    const int64_t tok = i / quads, f = (i - tok * quads) * 4;
    f32x4 s = *(const f32x4*)(part + tok * p.m + f);
    for (int k = 1; k < slabs; ++k) s += *(const f32x4*)(part + ((int64_t)k * p.n + tok) * p.m + f);
    store_quad(p, tok, f, s);
}

// Operands with rows of whole k-steps' halves: K to Kp = a multiple of 64.  A thread: 8 logical k of a row of W or of a token.
__global__ void __launch_bounds__(256) q8_pad_kernel(Q8Product p, int64_t Kp, uint8_t* __restrict__ a, uint8_t* __restrict__ am, uint8_t* __restrict__ x) {
    const int64_t pieces = Kp / 8, i = flat_block() * 256 + threadIdx.x, row = i / pieces, k = (i - row * pieces) * 8;
    if (row >= p.m + p.n) return;
    const bool in = k < p.K;
    if (row < p.m) {
        *(uint32_t*)(a + (row * Kp + k) / 2) = in ? *(const uint32_t*)(p.a + (row * p.K + k) / 2) : 0u;
        am[(row * Kp + k) / 8] = in ? p.am[(row * p.K + k) / 8] : (uint8_t)META_NONE;
    } else {
        const int64_t t = row - p.m;
        *(u32x2*)(x + t * Kp + k) = in ? *(const u32x2*)(p.x + t * p.K + k) : (u32x2){0, 0};
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

namespace {

// workgroups of 256 along a dimension of a grid, which holds fewer than 2^32 work items
constexpr int64_t GROUPS_END = (int64_t)1 << 24;
// 32-bit offsets inside a tile's rows, and tiles whose number, rounded up to a grid, is an int.  (Of the tiles that a plan may take
// 128 x 32 can be twice as many as are counted here: the plan looks at each one's grid.)
bool tile_fits(int64_t n, int64_t m, int64_t K) {
    return K % 64 == 0 && K < ((int64_t)1 << 23) && (m + 127) / 128 * ((n + 63) / 64) < GROUPS_END / 2;
}

template <int BM, int BN, int WM, bool TAIL>
hipError_t launch_tiles_of(const Q8Product& p, const Q8Split& split, hipStream_t s) {
    using S = Q8Smem<BM, BN>;
    constexpr int LDS = S::TOTAL > BN * S::OUT_PITCH ? S::TOTAL : BN * S::OUT_PITCH;
    const hipError_t e = allow_dynamic_lds<q8_tile_kernel<BM, BN, WM, TAIL>>(LDS);
    if (e != hipSuccess) return e;
    const int tiles_m = (int)((p.m + BM - 1) / BM), tiles_n = (int)((p.n + BN - 1) / BN);
    q8_tile_kernel<BM, BN, WM, TAIL><<<q8_grid(tiles_m, tiles_n, split.slabs), 256, LDS, s>>>(p, tiles_m, tiles_n, split);
    return hipGetLastError();
}
template <int BM, int BN, int WM>
hipError_t launch_tiles(const Q8Product& p, const Q8Split& split, hipStream_t s) {
    return p.K % KSTEP == 0 ? launch_tiles_of<BM, BN, WM, false>(p, split, s) : launch_tiles_of<BM, BN, WM, true>(p, split, s);
}

// below it the general kernel's one launch is faster (us, general / copies and tiles: 200 tokens, 2056 x 2056 15.8 / 17; 600, 1000 x 1000
// 11.8 / 13; 2048, 2056 x 2056 106 / 30)
constexpr int64_t PAD_WORK = (int64_t)1 << 30;
// (us, stream / best of the tiles: 4 tokens, 36864 x 9216 34.8 / 49.1, 5120 x 5120 8.4 / 10.6; 8 tokens 40.7 / 49.4, 9.6 / 10.8)
constexpr int STREAM_WAVES = 4, STREAM_STAGES = 3, STREAM_GROUPS = 1024, STREAM_TOKENS = 8;
bool stream_fits(int64_t n, int64_t m, int64_t K) { return n <= STREAM_TOKENS && K % 32 == 0 && K < ((int64_t)1 << 23) && (m + 31) / 32 < GROUPS_END; }

template <int TOK>
hipError_t launch_stream(const Q8Product& p, const Q8Split& split, hipStream_t s) {
    constexpr int RING = STREAM_WAVES * STREAM_STAGES * Q8Ring<TOK>::STAGE, SUMS = STREAM_WAVES * TOK * 36 * 4, LDS = RING > SUMS ? RING : SUMS;
    const hipError_t e = allow_dynamic_lds<q8_stream_kernel<TOK, STREAM_WAVES, STREAM_STAGES>>(LDS);
    if (e != hipSuccess) return e;
    q8_stream_kernel<TOK, STREAM_WAVES, STREAM_STAGES><<<dim3((unsigned)((p.m + 31) / 32), (unsigned)split.slabs), 64 * STREAM_WAVES, LDS, s>>>(p, split);
    return hipGetLastError();
}

// What a product takes on a tile, us, by constants fitted to the times of 945 products (9 to 8192 tokens, 512 to 36864 rows and
// columns, operands from memory, each on every tile that suits and in 1 to 16 slabs).  On 668 others the least
// estimate's choice takes 1.029 times the best one's time in the geometric mean, 1.49 times at most.  A round that does not fill the chip runs with fewer tiles on a
// compute unit and a higher clock; rounds overlap, so tiles count partly by rounds, partly by their number.  (us, 256 x 256 / 128 x 128 / 128 x 64,
// whole: 793 tokens, 11776 x 3584 34 / 39 / 46; 609, 12800 x 6144 48 / 38 / 52; 972, 12352 x 4416 47 / 62 / 93.  Whole / best number of
// slabs: 60 tokens, 9216 x 9216 34 / 20; 300, 9216 x 36864 145 / 100; 128, 5120 x 5120 16 / 18.)
struct Q8Tile {
    int bm, bn, resident;                                       // resident: on the chip at a time
    double step, full, rest;                                    // of a k-step with one tile on a compute unit, on a full chip; outside of them
};
constexpr Q8Tile Q8_TILES[] = {{256, 256, RESIDENT, 0.73, 1.08, 8.2}, {128, 128, 2 * RESIDENT, 0.45, 0.78, 1.4},
                               {128, 64, 2 * RESIDENT, 0.38, 0.60, 0.6}, {128, 32, 2 * RESIDENT, 0.36, 0.53, 0.0}};
constexpr double BY_NUMBER = 0.4, MEMORY_US = 0.235;            // a MB of operands and result
constexpr double REDUCE_US = 3.5, SUMS_US = 0.27;               // the launch that adds slabs' sums; a MB of them
constexpr double SECOND_US = 4.7, SECOND_STEP_US = 0.35;        // a second launch after whole rounds; and for each of its k-steps
constexpr int SLABS = 16, STEPS_SLAB = 6;                       // most slabs; fewest k-steps of one
int64_t tiles_of(const Q8Tile& t, int64_t n, int64_t m) { return (m + t.bm - 1) / t.bm * ((n + t.bn - 1) / t.bn); }
double tiles_us(const Q8Tile& t, int64_t count, int steps) {
    if (count <= RESIDENT) return t.step * steps + t.rest;
    const double number = (double)count / t.resident, rounds = (double)((count + t.resident - 1) / t.resident);
    return (BY_NUMBER * number + (1.0 - BY_NUMBER) * rounds) * (t.full * steps + t.rest);
}

// kernel of a product: stream (bn: tokens), tiles of bm x bn, or neither (the general one); the contraction in `slabs`
// slabs of `steps` k-steps (stream: stretches)
// rows0: the first rows, on 256 x 256 tiles in whole rounds of the chip, where the others go to bm x bn
struct Q8Plan { bool stream; int bm, bn, slabs, steps, total; int64_t rows0; };
// workgroups along the first dimension of its product's grid (without the whole rounds of rows0)
int64_t q8_groups(const Q8Plan& p, int64_t n, int64_t m) {
    if (p.stream) return (m + 31) / 32;
    if (p.bm == 0) return grid_of((m + 31) / 32 * ((n + 31) / 32)).x;
    return q8_grid((int)((m - p.rows0 + p.bm - 1) / p.bm), (int)((n + p.bn - 1) / p.bn), p.slabs);
}
Q8Plan q8_plan(int64_t n, int64_t m, int64_t K, bool room) {
    if (stream_fits(n, m, K)) {
        Q8Plan plan = {true, 32, n <= 4 ? 4 : 8, 1, 0, (int)((K + 255) / 256), 0};
        plan.steps = plan.total;
        const int64_t groups = (m + 31) / 32;
        int slabs = room ? (int)min((int64_t)STREAM_GROUPS / groups, (int64_t)plan.total / (2 * STREAM_WAVES)) : 1;
        if (slabs > 1) {
            plan.steps = (plan.total + slabs - 1) / slabs;
            plan.slabs = (plan.total + plan.steps - 1) / plan.steps;
        }
        return plan;
    }
    if (!tile_fits(n, m, K)) return {false, 0, 0, 1, 0, 0, 0};
    const int total = (int)((K + KSTEP - 1) / KSTEP);
    const double sums_mb = (double)n * (double)m * 4e-6;
    const double memory = ((double)m * K * 0.625 + (double)n * K + 2.0 * n * m) * 1e-6 * MEMORY_US;
    Q8Plan plan = {false, 0, 0, 1, total, total, 0};
    double best = 0.0;
    auto consider = [&](double us, const Q8Tile& t, int slabs, int steps, int64_t rows0) {
        if (plan.bm != 0 && us >= best) return;
        const Q8Plan p = {false, t.bm, t.bn, slabs, steps, total, rows0};
        if (q8_groups(p, n, m) >= GROUPS_END) return;
        best = us;
        plan = p;
    };
    for (const Q8Tile& t : Q8_TILES) {
        if (t.bn > 32 && t.bn >= 2 * n) continue;                // more than half of it empty
        const int64_t count = tiles_of(t, n, m);
        for (int slabs = 1; slabs == 1 || (room && slabs <= SLABS && total / slabs >= STEPS_SLAB && count * slabs <= t.resident); ++slabs) {
            const int steps = slabs == 1 ? total : ((total + slabs - 1) / slabs + 1) / 2 * 2;        // whole pairs of k-steps
            const int real = (total + steps - 1) / steps;
            if (real != slabs) continue;
            const double us = tiles_us(t, count * slabs, steps) + (slabs > 1 ? REDUCE_US + slabs * sums_mb * SUMS_US : 0.0);
            consider(sqrt(us * us + memory * memory), t, slabs, steps, 0);
        }
    }
    // Whole rounds of 256 x 256 and the rows that are left on tiles of 64 tokens, if these are resident at once, or else of 128.  (us, the best
    // tile / both: 777 tokens, 20480 x 5120 87 / 74; 3418, 7936 x 13312 236 / 258; 1390, 12800 x 5120 82 / 74; with leftover tiles 64 / 128 tokens wide,
    // 416 / 208 of them 74 / 75, 852 / 432 1.13 to 1.  The leftover tiles of the first in four slabs each, whose 64 MB of sums are written and
    // read once more: 21 more than on smaller tiles.)
    const Q8Tile &large = Q8_TILES[0], &wide = Q8_TILES[1], &narrow = Q8_TILES[2];
    const int64_t tn = (n + large.bn - 1) / large.bn, rows0 = tiles_of(large, n, m) / large.resident * large.resident / tn * large.bm;
    if (n > large.bn / 2 && rows0 > 0 && rows0 < m) {
        const Q8Tile& t = tiles_of(narrow, n, m - rows0) <= narrow.resident ? narrow : wide;
        const double us = tiles_us(large, rows0 / large.bm * tn, total) + SECOND_US + SECOND_STEP_US * total + tiles_us(t, tiles_of(t, n, m - rows0), total);
        consider(sqrt(us * us + memory * memory), t, 1, total, rows0);
    }
    return plan;
}

}  // namespace

namespace {

size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

// Copies with longer rows for the kernels above, where rows are no multiple of 64 (nor, for few tokens, of 32) and the product is
// worth two launches
struct Q8Pad { int64_t Kp; size_t a, am, x; };
Q8Pad q8_pad(int64_t n, int64_t m, int64_t K) {
    const int64_t Kp = (K + 63) / 64 * 64;
    if (stream_fits(n, m, K) || K % 64 == 0 || !tile_fits(n, m, Kp) || n * m * K < PAD_WORK) return {0, 0, 0, 0};
    return {Kp, round256((size_t)m * (size_t)(Kp / 2)), round256((size_t)m * (size_t)(Kp / 8)), round256((size_t)n * (size_t)Kp)};
}

}  // namespace

// [ padded copies | slabs' sums ]
size_t spmm_q8_workspace_bytes(int64_t n, int64_t m, int64_t K) {
    const Q8Pad pad = q8_pad(n, m, K);
    const Q8Plan plan = q8_plan(n, m, pad.Kp ? pad.Kp : K, true);
    return pad.a + pad.am + pad.x + (plan.slabs > 1 ? (size_t)plan.slabs * (size_t)n * (size_t)m * 4 : 0);
}

void spmm_q8_plan(int64_t n, int64_t m, int64_t K, bool workspace, int32_t* plan) {
    const Q8Pad pad = workspace ? q8_pad(n, m, K) : Q8Pad{0, 0, 0, 0};
    const Q8Plan p = q8_plan(n, m, pad.Kp ? pad.Kp : K, workspace);
    plan[0] = p.stream ? 0 : p.bm != 0 ? 1 : 2;
    plan[1] = p.bm != 0 ? p.bm : 32;
    plan[2] = p.bm != 0 ? p.bn : 32;
    plan[3] = p.slabs;
    plan[4] = (int32_t)p.rows0;
    plan[5] = (int32_t)pad.Kp;
    plan[6] = (int32_t)q8_groups(p, n, m);
}

hipError_t launch_spmm_q8(const uint8_t* x, const float* xs, int64_t n, const uint8_t* a, const uint8_t* am, const float* as,
                          int64_t m, int64_t K, const bf16_t* add, bf16_t* y, float* workspace_or_null, hipStream_t s) {
    Q8Product p = {x, xs, n, a, am, as, m, K, add, y, m};
    uint8_t* room = (uint8_t*)workspace_or_null;
    const Q8Pad pad = room ? q8_pad(n, m, K) : Q8Pad{0, 0, 0, 0};
    if (pad.Kp) {
        uint8_t *const a2 = room, *const am2 = a2 + pad.a, *const x2 = am2 + pad.am;
        room = x2 + pad.x;
        q8_pad_kernel<<<grid_of(((m + n) * (pad.Kp / 8) + 255) / 256), 256, 0, s>>>(p, pad.Kp, a2, am2, x2);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        p.a = a2;
        p.am = am2;
        p.x = x2;
        p.K = pad.Kp;
    }
    const Q8Plan plan = q8_plan(n, m, p.K, room != nullptr);
    if (plan.bm == 0) {
        const int64_t tiles_m = (m + 31) / 32, tiles = tiles_m * ((n + 31) / 32);
        if (!grid_fits(tiles)) return hipErrorInvalidConfiguration;
        q8_generic_kernel<<<grid_of(tiles), 256, 0, s>>>(p, tiles_m, tiles);
        return hipGetLastError();
    }
    float* const part = plan.slabs > 1 ? (float*)room : nullptr;
    const Q8Split split = {plan.slabs, plan.steps, plan.total, part};
    hipError_t e;
    if (plan.rows0 > 0) {
        Q8Product first = p;
        first.m = plan.rows0;
        e = launch_tiles<256, 256, 2>(first, split, s);
        if (e != hipSuccess) return e;
        p.a += plan.rows0 * (p.K / 2);
        p.am += plan.rows0 * (p.K / 8);
        p.as += plan.rows0;
        p.y += plan.rows0;
        if (p.add) p.add += plan.rows0;
        p.m -= plan.rows0;
    }
    if (plan.stream) e = plan.bn == 4 ? launch_stream<4>(p, split, s) : launch_stream<8>(p, split, s);
    else if (plan.bm == 256) e = launch_tiles<256, 256, 2>(p, split, s);
    else if (plan.bn == 128) e = launch_tiles<128, 128, 2>(p, split, s);
    else if (plan.bn == 64) e = launch_tiles<128, 64, 2>(p, split, s);
    else e = launch_tiles<128, 32, 4>(p, split, s);
    if (e != hipSuccess || plan.slabs == 1) return e;
    q8_reduce_kernel<<<grid_of((n * (m / 4) + 255) / 256), 256, 0, s>>>(p, part, plan.slabs);
    return hipGetLastError();
}
