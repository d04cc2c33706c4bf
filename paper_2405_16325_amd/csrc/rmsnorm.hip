// Root-mean-square norm with the residual's addition, its 8-bit output, and its gradient.
//
//     h = bf16(x + res)      r = 1 / sqrt(mean_j h_j^2 + eps)      y_j = h_j r w_j
//     q = e4m3(y / s), s = max_j |y_j| / 448                        (one scale per token, for the 8-bit product)
//     g_j = dy_j w_j,  c = mean_j g_j h_j r:   dx_j = r (g_j - h_j r c) + dh_j      dw_j = sum over tokens of dy_j h_j r
//
// The statistics are those of the stream as it is stored, rounded: the gradient is taken at that h.  All sums are fp32.
// Memory bounds both directions (16384 x 9216 with the residual: forward 195 us, 6.2 TB/s, gradient 203, 6.0 TB/s), latency a few hundred
// rows (777 x 5120, 28 MB from memory to an 8-bit output: 10.4 to 11.7 us, of which 2.6 are what one row takes; a row has ten
// wavefronts here, a compute unit room for three rows, so nine rows take a second turn).  A row is read once and stays in
// registers: LPR lanes (8 to 64) of a wavefront share a short one, `wpr` wavefronts a longer one; a lane holds VPT pieces of 8 neighbouring elements, so that every load and
// store of a wavefront covers whole 128-byte lines.
#include "pipeline.h"
#include "wave.h"

namespace {

constexpr int MAX_THREADS = 1024;
constexpr int MAX_WAVES = MAX_THREADS / 64;

// The threads of one row: `lane` of `threads`, piece p of the row is lane + p * threads
struct RowThreads { int row, lane, threads; };
template <int LPR>
__device__ __forceinline__ RowThreads row_threads(int wpr) {
    const int t = threadIdx.x;
    if constexpr (LPR < 64) return {t / LPR, t % LPR, LPR};
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6), row = wpr == 1 ? wave : wave / wpr;
    return {row, (wave - row * wpr) * 64 + (t & 63), wpr * 64};
}

// Sum (or largest) over a row's threads.  part: MAX_WAVES floats of LDS that nothing else uses until the next barrier but one.
template <int LPR>
__device__ __forceinline__ float row_sum(float v, int wpr, float* part) {
    v = lanes_sum<LPR>(v);
    if (LPR < 64 || wpr == 1) return v;
    const int wave = threadIdx.x >> 6, first = wave / wpr * wpr;
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    v = part[first];
    for (int i = 1; i < wpr; ++i) v += part[first + i];
    return v;
}
template <int LPR>
__device__ __forceinline__ float row_max(float v, int wpr, float* part) {
    v = lanes_max_abs<LPR>(v);
    if (LPR < 64 || wpr == 1) return v;
    const int wave = threadIdx.x >> 6, first = wave / wpr * wpr;
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    v = part[first];
    for (int i = 1; i < wpr; ++i) v = max_abs(v, part[first + i]);
    return v;
}

// STREAM: a call that moves more than the last-level cache holds, of which nothing would be found there by the next one
// (16384 x 9216, 1.2 GB: forward 205 -> 197 us, gradient 227 -> 201; 4096 x 2560, 84 MB, would take 15.4 -> 17.0 and 22.6 -> 22.9)
template <bool STREAM, class T>
__device__ __forceinline__ T load(const void* p) { return STREAM ? __builtin_nontemporal_load((const T*)p) : *(const T*)p; }
template <bool STREAM, class T>
__device__ __forceinline__ void store(void* p, T v) {
    if (STREAM) __builtin_nontemporal_store(v, (T*)p);
    else *(T*)p = v;
}

struct NormFwd {
    const bf16_t *x, *res, *w;                 // res: or null
    int64_t b;
    int d;
    float eps;
    bf16_t *h, *y;                             // y: or null
    float* rstd;                               // or null
    uint8_t* q;                                // or null
    float* scale;
};

template <int LPR, int VPT, bool STREAM = false>
__global__ void __launch_bounds__(MAX_THREADS) rmsnorm_fwd_kernel(NormFwd a, int wpr) {
    __shared__ float part[2][MAX_WAVES];
    const RowThreads rt = row_threads<LPR>(wpr);
    const int64_t row = flat_block() * (blockDim.x / rt.threads) + rt.row;
    const bool live = row < a.b;
    const int pieces = a.d / 8;
    const size_t at = (size_t)row * a.d;

    F8 h[VPT];
    u32x4 w[VPT];
    float sum = 0.0f;
    u32x4 px[VPT], pr[VPT];
#pragma unroll
    for (int p = 0; p < VPT; ++p) {
        const int i = rt.lane + p * rt.threads;
        px[p] = pr[p] = w[p] = (u32x4){0, 0, 0, 0};
        if (live && i < pieces) {
            px[p] = load<STREAM, u32x4>(a.x + at + 8 * (size_t)i);
            if (a.res) pr[p] = load<STREAM, u32x4>(a.res + at + 8 * (size_t)i);
            w[p] = *(const u32x4*)(a.w + 8 * (size_t)i);
        }
    }
#pragma unroll
    for (int p = 0; p < VPT; ++p) {
        const int i = rt.lane + p * rt.threads;
        if (a.res) {
            F8 s = unpack_bf16(px[p]);
            const F8 r = unpack_bf16(pr[p]);
#pragma unroll
            for (int k = 0; k < 8; ++k) s.v[k] += r.v[k];
            px[p] = pack_bf16(s);
            if (live && i < pieces) store<STREAM>(a.h + at + 8 * (size_t)i, px[p]);
        }
        h[p] = unpack_bf16(px[p]);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = fmaf(h[p].v[k], h[p].v[k], sum);
    }
    sum = row_sum<LPR>(sum, wpr, part[0]);
    const float r = 1.0f / sqrtf(sum / (float)a.d + a.eps);
    if (a.rstd && live && rt.lane == 0) a.rstd[row] = r;

    float top = 0.0f;
#pragma unroll
    for (int p = 0; p < VPT; ++p) {
        const int i = rt.lane + p * rt.threads;
        const F8 f = unpack_bf16(w[p]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            h[p].v[k] = h[p].v[k] * r * f.v[k];
            top = max_abs(top, h[p].v[k]);
        }
        if (a.y && live && i < pieces) store<STREAM>(a.y + at + 8 * (size_t)i, pack_bf16(h[p]));
    }
    if (!a.q) return;
    const Q8Scale s = q8_scale(row_max<LPR>(top, wpr, part[1]));
    if (live && rt.lane == 0) a.scale[row] = s.scale;
#pragma unroll
    for (int p = 0; p < VPT; ++p) {
        const int i = rt.lane + p * rt.threads;
#pragma unroll
        for (int k = 0; k < 8; ++k) h[p].v[k] *= s.inv;
        if (live && i < pieces) store<STREAM>(a.q + at + 8 * (size_t)i, pack_e4m3(h[p]));
    }
}

// Rows too long for registers: the row is read once for the sum and again, from the caches, for the output (twice for an
// 8-bit one).  A thread reads back only what it wrote itself.
__global__ void __launch_bounds__(MAX_THREADS) rmsnorm_fwd_wide_kernel(NormFwd a) {
    __shared__ float part[2][MAX_WAVES];
    const int64_t row = flat_block();
    if (row >= a.b) return;                                     // the whole workgroup
    const int pieces = a.d / 8, t = threadIdx.x;
    const size_t at = (size_t)row * a.d;
    const bf16_t* from = a.res ? a.h : a.x;
    float sum = 0.0f;
    for (int i = t; i < pieces; i += MAX_THREADS) {
        u32x4 p = *(const u32x4*)(a.x + at + 8 * (size_t)i);
        if (a.res) {
            F8 s = unpack_bf16(p);
            const F8 r = unpack_bf16(*(const u32x4*)(a.res + at + 8 * (size_t)i));
#pragma unroll
            for (int k = 0; k < 8; ++k) s.v[k] += r.v[k];
            p = pack_bf16(s);
            *(u32x4*)(a.h + at + 8 * (size_t)i) = p;
        }
        const F8 h = unpack_bf16(p);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = fmaf(h.v[k], h.v[k], sum);
    }
    sum = row_sum<64>(sum, MAX_WAVES, part[0]);
    const float r = 1.0f / sqrtf(sum / (float)a.d + a.eps);
    if (a.rstd && t == 0) a.rstd[row] = r;
    float top = 0.0f, inv = 0.0f;
    for (int pass = 0; pass < (a.q ? 2 : 1); ++pass) {
        for (int i = t; i < pieces; i += MAX_THREADS) {
            F8 y = unpack_bf16(*(const u32x4*)(from + at + 8 * (size_t)i));
            const F8 f = unpack_bf16(*(const u32x4*)(a.w + 8 * (size_t)i));
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                y.v[k] = y.v[k] * r * f.v[k];
                top = max_abs(top, y.v[k]);
            }
            if (pass == 0) {
                if (a.y) *(u32x4*)(a.y + at + 8 * (size_t)i) = pack_bf16(y);
                continue;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) y.v[k] *= inv;
            *(u32x2*)(a.q + at + 8 * (size_t)i) = pack_e4m3(y);
        }
        if (pass == 0 && a.q) {
            const Q8Scale s = q8_scale(row_max<64>(top, MAX_WAVES, part[1]));
            inv = s.inv;
            if (t == 0) a.scale[row] = s.scale;
        }
    }
}

struct NormBwd {
    const bf16_t *dy, *h, *w;
    const float* rstd;
    const bf16_t* dh;                          // or null
    int64_t b;
    int d;
    bf16_t *dx, *dw;
    float* part;                               // fp32[groups][d]: each workgroup's share of dw; one workgroup writes dw itself
};

// Workgroup g takes rows g R .. g R + R - 1, then those `groups` R later, and keeps its share of dw in registers; the R row
// slots' shares are added through LDS.
constexpr int bwd_threads(int vpt) { return vpt == 1 ? MAX_THREADS : 512; }   // more would leave fewer registers than they take

template <int LPR, int VPT, bool STREAM = false>
__global__ void __launch_bounds__(bwd_threads(VPT)) rmsnorm_bwd_kernel(NormBwd a, int wpr) {
    constexpr bool AHEAD = VPT <= 4;                            // longer rows keep enough loads on their way one at a time,
                                                                // and registers only for them and dw
    extern __shared__ float lds[];                              // 2 x MAX_WAVES, then R - 1 rows of d
    const RowThreads rt = row_threads<LPR>(wpr);
    const int slots = blockDim.x / rt.threads, pieces = a.d / 8;
    struct Row { u32x4 dy[VPT], h[VPT], dh[VPT]; float r; };
    auto fetch = [&](Row& o, int64_t row) {
        const bool live = row < a.b;
        const size_t at = (size_t)row * a.d;
        o.r = live ? a.rstd[row] : 0.0f;
#pragma unroll
        for (int p = 0; p < VPT; ++p) {
            const int i = rt.lane + p * rt.threads;
            o.dy[p] = o.h[p] = o.dh[p] = (u32x4){0, 0, 0, 0};
            if (live && i < pieces) {
                o.dy[p] = load<STREAM, u32x4>(a.dy + at + 8 * (size_t)i);
                o.h[p] = load<STREAM, u32x4>(a.h + at + 8 * (size_t)i);
                if (a.dh) o.dh[p] = load<STREAM, u32x4>(a.dh + at + 8 * (size_t)i);
            }
        }
    };
    u32x4 w[AHEAD ? VPT : 1];
    auto weight = [&](int p) {
        const int i = rt.lane + p * rt.threads;
        return i < pieces ? *(const u32x4*)(a.w + 8 * (size_t)i) : (u32x4){0, 0, 0, 0};
    };
    F8 dw[VPT];
#pragma unroll
    for (int p = 0; p < VPT; ++p) {
        if (AHEAD) w[p] = weight(p);
#pragma unroll
        for (int k = 0; k < 8; ++k) dw[p].v[k] = 0.0f;
    }
    int turn = 0;
    const int64_t stride = (int64_t)gridDim.x * slots;
    Row now, next;
    if (AHEAD) fetch(next, (int64_t)blockIdx.x * slots + rt.row);
    for (int64_t first = (int64_t)blockIdx.x * slots; first < a.b; first += stride, turn ^= 1) {
        const int64_t row = first + rt.row;
        const bool live = row < a.b;
        const size_t at = (size_t)row * a.d;
        if (AHEAD) {
            now = next;
            fetch(next, row + stride);                           // on its way while this row is worked on
        } else {
            fetch(now, row);
        }
        float c = 0.0f;
#pragma unroll
        for (int p = 0; p < VPT; ++p) {
            if (!AHEAD) __builtin_amdgcn_sched_barrier(0);      // no pieces of the weight in advance
            const F8 dy = unpack_bf16(now.dy[p]), h = unpack_bf16(now.h[p]), f = unpack_bf16(AHEAD ? w[AHEAD ? p : 0] : weight(p));
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float t = dy.v[k] * (h.v[k] * now.r);
                c = fmaf(t, f.v[k], c);
                dw[p].v[k] += t;
            }
        }
        c = row_sum<LPR>(c, wpr, lds + turn * MAX_WAVES) / (float)a.d;
#pragma unroll
        for (int p = 0; p < VPT; ++p) {
            const int i = rt.lane + p * rt.threads;
            // packed again from here: twice the registers would be taken by the values as they were unpacked above
            if (!AHEAD) __builtin_amdgcn_sched_barrier(0);
            asm volatile("" : "+v"(now.dy[p]), "+v"(now.h[p]));
            const F8 dy = unpack_bf16(now.dy[p]), h = unpack_bf16(now.h[p]), dh = unpack_bf16(now.dh[p]),
                     f = unpack_bf16(AHEAD ? w[AHEAD ? p : 0] : weight(p));
            F8 o;
#pragma unroll
            for (int k = 0; k < 8; ++k) o.v[k] = fmaf(now.r, dy.v[k] * f.v[k] - h.v[k] * now.r * c, dh.v[k]);
            if (live && i < pieces) store<STREAM>(a.dx + at + 8 * (size_t)i, pack_bf16(o));
        }
    }
    float* const sums = lds + 2 * MAX_WAVES;
    if (rt.row > 0)
#pragma unroll
        for (int p = 0; p < VPT; ++p) {
            const int i = rt.lane + p * rt.threads;
            if (i < pieces)
#pragma unroll
                for (int k = 0; k < 8; ++k) sums[(size_t)(rt.row - 1) * a.d + 8 * i + k] = dw[p].v[k];
        }
    __syncthreads();
    if (rt.row > 0) return;
#pragma unroll
    for (int p = 0; p < VPT; ++p) {
        const int i = rt.lane + p * rt.threads;
        if (i >= pieces) continue;
        for (int s = 1; s < slots; ++s)
#pragma unroll
            for (int k = 0; k < 8; ++k) dw[p].v[k] += sums[(size_t)(s - 1) * a.d + 8 * i + k];
        if (gridDim.x == 1) {
            *(u32x4*)(a.dw + 8 * (size_t)i) = pack_bf16(dw[p]);
            continue;
        }
        f32x4* const o = (f32x4*)(a.part + (size_t)blockIdx.x * a.d + 8 * (size_t)i);
        o[0] = (f32x4){dw[p].v[0], dw[p].v[1], dw[p].v[2], dw[p].v[3]};
        o[1] = (f32x4){dw[p].v[4], dw[p].v[5], dw[p].v[6], dw[p].v[7]};
    }
}

// Both gradients in one launch, where dx is not written over dy.  Workgroups below `dw_groups` make dw, 4 pieces (a line of 64 bytes) and all
// rows each, added over the lanes and then, in order, over the wavefronts; the others dx, a row a slot.  dy and h are read twice, the
// second time from the caches.  dw's loads, four rows at a time, bound it (1000 x 1000: 7.5 us).
template <int LPR, int VPT>
__global__ void __launch_bounds__(MAX_THREADS) rmsnorm_bwd_once_kernel(NormBwd a, int wpr, int dw_groups) {
    __shared__ float part[MAX_WAVES];
    __shared__ F8 shares[MAX_WAVES][4];
    const int pieces = a.d / 8;
    if ((int)blockIdx.x < dw_groups) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 4 + (lane & 3), step = blockDim.x / 4;
        F8 s;
#pragma unroll
        for (int k = 0; k < 8; ++k) s.v[k] = 0.0f;
        if (i < pieces)
#pragma unroll 4
            for (int row = threadIdx.x >> 2; row < (int)a.b; row += step) {
                const size_t at = (size_t)row * a.d + 8 * (size_t)i;
                const float r = a.rstd[row];
                const F8 dy = unpack_bf16(*(const u32x4*)(a.dy + at)), h = unpack_bf16(*(const u32x4*)(a.h + at));
#pragma unroll
                for (int k = 0; k < 8; ++k) s.v[k] += dy.v[k] * (h.v[k] * r);
            }
#pragma unroll
        for (int x = 4; x < 64; x *= 2)
#pragma unroll
            for (int k = 0; k < 8; ++k) s.v[k] += __shfl_xor(s.v[k], x);
        if (lane < 4) shares[wave][lane] = s;
        __syncthreads();
        if (threadIdx.x >= 4 || i >= pieces) return;
        for (int w = 1; w < (int)blockDim.x / 64; ++w)
#pragma unroll
            for (int k = 0; k < 8; ++k) s.v[k] += shares[w][lane].v[k];
        *(u32x4*)(a.dw + 8 * (size_t)i) = pack_bf16(s);
        return;
    }
    const RowThreads rt = row_threads<LPR>(wpr);
    const int64_t row = (int64_t)((int)blockIdx.x - dw_groups) * (blockDim.x / rt.threads) + rt.row;
    const size_t at = (size_t)row * a.d;
    const float r = row < a.b ? a.rstd[row] : 0.0f;
    u32x4 pdy[VPT], ph[VPT], pdh[VPT], pw[VPT];
    float c = 0.0f;
#pragma unroll
    for (int p = 0; p < VPT; ++p) {
        const int i = rt.lane + p * rt.threads;
        pdy[p] = ph[p] = pdh[p] = pw[p] = (u32x4){0, 0, 0, 0};
        if (row < a.b && i < pieces) {
            pdy[p] = *(const u32x4*)(a.dy + at + 8 * (size_t)i);
            ph[p] = *(const u32x4*)(a.h + at + 8 * (size_t)i);
            if (a.dh) pdh[p] = *(const u32x4*)(a.dh + at + 8 * (size_t)i);
            pw[p] = *(const u32x4*)(a.w + 8 * (size_t)i);
        }
    }
#pragma unroll
    for (int p = 0; p < VPT; ++p) {
        const F8 dy = unpack_bf16(pdy[p]), h = unpack_bf16(ph[p]), w = unpack_bf16(pw[p]);
#pragma unroll
        for (int k = 0; k < 8; ++k) c = fmaf(dy.v[k] * (h.v[k] * r), w.v[k], c);
    }
    c = row_sum<LPR>(c, wpr, part) / (float)a.d;
#pragma unroll
    for (int p = 0; p < VPT; ++p) {
        const int i = rt.lane + p * rt.threads;
        const F8 dy = unpack_bf16(pdy[p]), h = unpack_bf16(ph[p]), dh = unpack_bf16(pdh[p]), w = unpack_bf16(pw[p]);
        F8 o;
#pragma unroll
        for (int k = 0; k < 8; ++k) o.v[k] = fmaf(r, dy.v[k] * w.v[k] - h.v[k] * r * c, dh.v[k]);
        if (row < a.b && i < pieces) *(u32x4*)(a.dx + at + 8 * (size_t)i) = pack_bf16(o);
    }
}

// Rows too long for registers: dx row by row, reading the row twice, and dw's shares column by column
__global__ void __launch_bounds__(MAX_THREADS) rmsnorm_bwd_wide_kernel(NormBwd a) {
    __shared__ float part[MAX_WAVES];
    const int64_t row = flat_block();
    if (row >= a.b) return;
    const int pieces = a.d / 8;
    const size_t at = (size_t)row * a.d;
    const float r = a.rstd[row];
    float c = 0.0f;
    for (int i = threadIdx.x; i < pieces; i += MAX_THREADS) {
        const F8 dy = unpack_bf16(*(const u32x4*)(a.dy + at + 8 * (size_t)i)), h = unpack_bf16(*(const u32x4*)(a.h + at + 8 * (size_t)i));
        const F8 w = unpack_bf16(*(const u32x4*)(a.w + 8 * (size_t)i));
#pragma unroll
        for (int k = 0; k < 8; ++k) c = fmaf(dy.v[k] * (h.v[k] * r), w.v[k], c);
    }
    c = row_sum<64>(c, MAX_WAVES, part) / (float)a.d;
    for (int i = threadIdx.x; i < pieces; i += MAX_THREADS) {
        const F8 dy = unpack_bf16(*(const u32x4*)(a.dy + at + 8 * (size_t)i)), h = unpack_bf16(*(const u32x4*)(a.h + at + 8 * (size_t)i));
        const F8 w = unpack_bf16(*(const u32x4*)(a.w + 8 * (size_t)i));
        const F8 dh = unpack_bf16(a.dh ? *(const u32x4*)(a.dh + at + 8 * (size_t)i) : (u32x4){0, 0, 0, 0});
        F8 o;
#pragma unroll
        for (int k = 0; k < 8; ++k) o.v[k] = fmaf(r, dy.v[k] * w.v[k] - h.v[k] * r * c, dh.v[k]);
        *(u32x4*)(a.dx + at + 8 * (size_t)i) = pack_bf16(o);
    }
}
// grid: (pieces / 256 rounded up) x groups
__global__ void __launch_bounds__(256) rmsnorm_dw_wide_kernel(NormBwd a) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= a.d / 8) return;
    F8 s;
#pragma unroll
    for (int k = 0; k < 8; ++k) s.v[k] = 0.0f;
    for (int64_t row = blockIdx.y; row < a.b; row += gridDim.y) {
        const size_t at = (size_t)row * a.d + 8 * (size_t)i;
        const float r = a.rstd[row];
        const F8 dy = unpack_bf16(*(const u32x4*)(a.dy + at)), h = unpack_bf16(*(const u32x4*)(a.h + at));
#pragma unroll
        for (int k = 0; k < 8; ++k) s.v[k] += dy.v[k] * (h.v[k] * r);
    }
    f32x4* const o = (f32x4*)(a.part + (size_t)blockIdx.y * a.d + 8 * (size_t)i);
    o[0] = (f32x4){s.v[0], s.v[1], s.v[2], s.v[3]};
    o[1] = (f32x4){s.v[4], s.v[5], s.v[6], s.v[7]};
}

// dw = bf16(sum of the groups' shares), in a fixed order.  A workgroup: 32 columns, 8 lanes of 4 each, 128 shares at a time
__global__ void __launch_bounds__(1024) rmsnorm_dw_kernel(const float* __restrict__ part, int groups, int d, bf16_t* __restrict__ dw) {
    __shared__ f32x4 sums[16][8];
    const int lane = threadIdx.x & 7, wave = threadIdx.x >> 6, col = blockIdx.x * 32 + lane * 4;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < d)
#pragma unroll 4
        for (int g = threadIdx.x >> 3; g < groups; g += 128) s += *(const f32x4*)(part + (size_t)g * d + col);
#pragma unroll
    for (int x = 8; x < 64; x *= 2)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] += __shfl_xor(s[k], x);
    if ((threadIdx.x & 63) < 8) sums[wave][lane] = s;
    __syncthreads();
    if (threadIdx.x >= 8 || col >= d) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += sums[i][lane];
    union { __bf16 h[4]; u32x2 u; } o;
#pragma unroll
    for (int k = 0; k < 4; ++k) o.h[k] = (__bf16)s[k];
    *(u32x2*)(dw + col) = o.u;
}

// How the threads of a workgroup share rows of d elements: `lpr` lanes a row (below 64), or `wpr` wavefronts, vpt pieces a lane
struct RowShape {
    int lpr, wpr, vpt, threads;
    int64_t slots() const { return lpr < 64 ? threads / lpr : threads / (64 * wpr); }
};
RowShape row_shape(int64_t pieces, int vpt) {
    if (pieces <= 32) return {pieces <= 8 ? 8 : pieces <= 16 ? 16 : 32, 1, 1, 256};
    const int wpr = (int)((pieces + 64 * vpt - 1) / (64 * vpt));
    return {64, wpr, vpt, wpr >= 4 ? wpr * 64 : 4 / wpr * wpr * 64};
}
// Few rows: as many threads as there are pieces, up to MAX_THREADS.  Many: two pieces a lane keep enough loads on their way
// (16384 x 9216: 207 us with 2, 3 or 4, with 8, whose registers leave a wavefront per SIMD, 296).  vpt 0: the row stays in memory.
constexpr int64_t MANY_ROWS = 2048;
RowShape fwd_shape(int64_t b, int64_t d) {
    const int64_t pieces = d / 8;
    if (pieces > 4 * MAX_THREADS) return {64, 1, 0, MAX_THREADS};
    return row_shape(pieces, pieces > 2 * MAX_THREADS ? 4 : b >= MANY_ROWS || pieces > MAX_THREADS ? 2 : 1);
}
RowShape bwd_shape(int64_t b, int64_t d) {
    const int64_t pieces = d / 8;
    if (pieces > 6 * 512) return {64, 1, 0, MAX_THREADS};
    if (b < MANY_ROWS && pieces <= MAX_THREADS) return row_shape(pieces, 1);
    return row_shape(pieces, pieces <= 2 * 512 ? 2 : pieces <= 3 * 512 ? 3 : pieces <= 4 * 512 ? 4 : 6);
}

// both gradients in one launch (us in a captured graph, two launches / one: 64 x 768 5.5 / 2.9; 1000 x 1000 9.8 / 7.7; 777 x 5120 14.6 / 12.3;
// 64 x 9216 9.1 / 4.6; 569 x 9216 18.3 / 18.2; 1024 x 5120 15.5 / 15.9; 1400 x 768 8.5 / 8.4; 2000 x 768 9.1 / 11.0; 1000 x 8192 20.6 / 24.3)
bool bwd_once(int64_t b, int64_t d) { return d / 8 <= 2 * MAX_THREADS && b <= 1024 && b * d <= (int64_t)5 << 20; }

// workgroups of the gradient: as many as are resident together (eight wavefronts on a compute unit), so that each makes one share of
// dw; for a few rows one, which saves the second launch
int bwd_groups(int64_t b, int64_t d) {
    const RowShape s = bwd_shape(b, d);
    const int64_t turns = s.vpt == 0 ? b : (b + s.slots() - 1) / s.slots();
    if (s.vpt != 0 && turns <= 4) return 1;
    const int64_t most = RESIDENT * (s.threads >= 8 * 64 ? 1 : 8 * 64 / s.threads);
    return (int)(turns < most ? turns : most);
}

}  // namespace

hipError_t launch_rmsnorm_fwd(const bf16_t* x, const bf16_t* res, const bf16_t* w, int64_t b, int64_t d, float eps, bf16_t* h,
                              bf16_t* y, float* rstd, uint8_t* q, float* scale, hipStream_t s) {
    const NormFwd a = {x, res, w, b, (int)d, eps, h, y, rstd, q, scale};
    const RowShape rs = fwd_shape(b, d);
    const dim3 grid = grid_of((b + rs.slots() - 1) / rs.slots());
    const bool stream = (size_t)b * (size_t)d * (2 + (res ? 4 : 0) + (y ? 2 : 0) + (q ? 1 : 0)) > LAST_LEVEL_CACHE_BYTES;
#define FWD(...) rmsnorm_fwd_kernel<__VA_ARGS__><<<grid, rs.threads, 0, s>>>(a, rs.wpr)
    if (rs.vpt == 0) rmsnorm_fwd_wide_kernel<<<grid_of(b), MAX_THREADS, 0, s>>>(a);
    else if (rs.lpr == 8) FWD(8, 1);
    else if (rs.lpr == 16) FWD(16, 1);
    else if (rs.lpr == 32) FWD(32, 1);
    else if (rs.vpt == 1) FWD(64, 1);
    else if (rs.vpt == 2 && stream) FWD(64, 2, true);
    else if (rs.vpt == 2) FWD(64, 2);
    else if (stream) FWD(64, 4, true);
    else FWD(64, 4);
#undef FWD
    return hipGetLastError();
}

size_t rmsnorm_bwd_workspace_bytes(int64_t b, int64_t d) { return (size_t)bwd_groups(b, d) * (size_t)d * 4; }

hipError_t launch_rmsnorm_bwd(const bf16_t* dy, const bf16_t* h, const bf16_t* w, const float* rstd, const bf16_t* dh, int64_t b,
                              int64_t d, bf16_t* dx, bf16_t* dw, float* part, hipStream_t s) {
    const NormBwd a = {dy, h, w, rstd, dh, b, (int)d, dx, dw, part};
    if (bwd_once(b, d) && (dx + b * d <= dy || dy + b * d <= dx)) {
        const RowShape rs = row_shape(d / 8, d / 8 <= MAX_THREADS ? 1 : 2);
        const int slots = rs.lpr < 64 ? 512 / rs.lpr : rs.wpr < 8 ? 8 / rs.wpr : 1, threads = rs.lpr < 64 ? 512 : slots * rs.wpr * 64;
        const int dw_groups = (int)((d / 8 + 3) / 4);
#define ONCE(...) rmsnorm_bwd_once_kernel<__VA_ARGS__><<<dw_groups + (int)((b + slots - 1) / slots), threads, 0, s>>>(a, rs.wpr, dw_groups)
        if (rs.lpr == 8) ONCE(8, 1);
        else if (rs.lpr == 16) ONCE(16, 1);
        else if (rs.lpr == 32) ONCE(32, 1);
        else if (rs.vpt == 1) ONCE(64, 1);
        else ONCE(64, 2);
#undef ONCE
        return hipGetLastError();
    }
    const RowShape rs = bwd_shape(b, d);
    const int groups = bwd_groups(b, d);
    if (rs.vpt == 0) {
        // dw first: dx may be written over dy
        rmsnorm_dw_wide_kernel<<<dim3((unsigned)((d / 8 + 255) / 256), (unsigned)groups), 256, 0, s>>>(a);
        rmsnorm_bwd_wide_kernel<<<grid_of(b), MAX_THREADS, 0, s>>>(a);
    } else {
        const size_t lds = 2 * MAX_WAVES * 4 + (size_t)(rs.slots() - 1) * d * 4;
        const bool stream = (size_t)b * (size_t)d * (dh ? 8 : 6) > LAST_LEVEL_CACHE_BYTES;
#define BWD(...) rmsnorm_bwd_kernel<__VA_ARGS__><<<groups, rs.threads, lds, s>>>(a, rs.wpr)
        if (rs.lpr == 8) BWD(8, 1);
        else if (rs.lpr == 16) BWD(16, 1);
        else if (rs.lpr == 32) BWD(32, 1);
        else if (rs.vpt == 1) BWD(64, 1);
        else if (rs.vpt == 2 && stream) BWD(64, 2, true);
        else if (rs.vpt == 2) BWD(64, 2);
        else if (rs.vpt == 3 && stream) BWD(64, 3, true);
        else if (rs.vpt == 3) BWD(64, 3);
        else if (rs.vpt == 4 && stream) BWD(64, 4, true);
        else if (rs.vpt == 4) BWD(64, 4);
        else if (stream) BWD(64, 6, true);
        else BWD(64, 6);
#undef BWD
        if (groups == 1) return hipGetLastError();
    }
    rmsnorm_dw_kernel<<<(unsigned)((d + 31) / 32), 1024, 0, s>>>(part, groups, (int)d, dw);
    return hipGetLastError();
}
