// AdamW over many tensors in one launch, and the gradients' global norm.
//
//     g = c grad      m = b1 m + (1 - b1) g      v = b2 v + (1 - b2) g^2
//     p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Memory bounds both: every element is read and written once, 28 bytes of it with 32-bit states and fp32 master weights, 10
// with 8-bit states and bf16 weights alone.  157 M elements with masters take 690 us of 32-bit step, 6.3 TB/s, and 55 + 5 of norm,
// 418 us with 8-bit states, 6.1 TB/s; 531 M with 8-bit states and bf16 weights 930, 5.8 TB/s, where the vector units are as busy.
// The tensors of a set are cut into chunks of CHUNK elements; a table in device memory (laid out once by adamw_fill_table) names
// each chunk's tensor, so that one launch covers hundreds of tensors of any sizes evenly and a workgroup finds its work with two
// scalar loads.
//
// States in 8 bits: m and r = sqrt(v) (its range is half of v's in octaves, and it is what the step divides by) as e4m3
// with an fp32 scale per 128 elements, held as values / scale <= 448.  A moving average of slow decay changes by less than
// half a code's distance per step, so rounded to the nearest it would freeze relative to its block's largest (b2 = 0.999,
// gradients of every other element ten times smaller from step 1500 on, step 3000: median of stored over true r 1.38 for these
// and 0.66 for their neighbours).  So codes are rounded up or down by a threshold u that moves by a fixed fraction of its range
// (the golden ratio's) every step and differs from element to element: as thresholds are evenly spread over any run of steps
// the rounding is unbiased (0.97 and 1.00), and needs no random numbers.  The update itself uses this step's m and v before
// they are rounded.
// An r that is not zero is never stored as zero: m would then be divided by eps alone.
//
// The states' arithmetic (products and sums rounded one by one, no fused forms; square root, reciprocal exactly rounded) is
// part of the format: the codes and scales are the same whatever computes them.  The weights' quotient is no part of it and takes
// the approximate reciprocal (one unit in the last place).
#include "pipeline.h"
#include "wave.h"
#include <math.h>
#include <string.h>

namespace {

constexpr int THREADS = 256;                                    // of the norm's workgroups, and of the step's on large sets
constexpr int CHUNK = 4096;
constexpr int Q8_BLOCK = SLOPE_ADAMW_BLOCK;
constexpr uint32_t DITHER_INDEX = 0x6A09E667u, DITHER_STEP = 0x9E3779B9u;   // 2^32 of sqrt(2) - 1, of the golden ratio - 1

struct Header {
    uint64_t magic;
    int64_t count, chunks, bytes;
    int32_t state_bits, pad[7];
};
static_assert(sizeof(Header) == 64, "the tensors follow aligned");
constexpr uint64_t MAGIC = 0x31574D4144415053ull;
struct Chunk { int32_t tensor, part; };

__device__ __forceinline__ const slope_adamw_tensor* tensors_of(const void* table) {
    return (const slope_adamw_tensor*)((const uint8_t*)table + sizeof(Header));
}
__device__ __forceinline__ const Chunk* chunks_of(const void* table, int64_t count) {
    return (const Chunk*)(tensors_of(table) + count);
}

// W neighbours of a lane, p[0 .. W - 1], of which the first `live` are there (FULL: all).  W is 4 where an array is fp32 and 8 where
// none is, so that no lane has more than 16 bytes of one and every load or store of a wavefront covers whole lines (with 8
// everywhere, 32 bytes a lane in two loads, streaming past the caches made 157 M elements with masters 20 % slower, not faster).
// Values are kept as they are in memory until all of a lane's loads are on their way.
template <int W> struct Vec { float v[W]; };
// The tensors' addresses come out of memory, where the compiler cannot see that they are global: said here.
#define GLOBAL __attribute__((address_space(1)))
template <int BITS, int W> struct Raw { uint32_t u[BITS * W / 32]; };

template <bool STREAM, int DWORDS>
__device__ __forceinline__ void load_dwords(const void* p, uint32_t (&u)[DWORDS]) {
    typedef uint32_t V __attribute__((ext_vector_type(DWORDS == 1 ? 2 : DWORDS)));
    if constexpr (DWORDS == 1) {
        u[0] = STREAM ? __builtin_nontemporal_load((const GLOBAL uint32_t*)p) : *(const GLOBAL uint32_t*)p;
    } else {
        const V x = STREAM ? __builtin_nontemporal_load((const GLOBAL V*)p) : *(const GLOBAL V*)p;
#pragma unroll
        for (int k = 0; k < DWORDS; ++k) u[k] = x[k];
    }
}
template <bool STREAM, int DWORDS>
__device__ __forceinline__ void store_dwords(void* p, const uint32_t (&u)[DWORDS]) {
    typedef uint32_t V __attribute__((ext_vector_type(DWORDS == 1 ? 2 : DWORDS)));
    if constexpr (DWORDS == 1) {
        if (STREAM) __builtin_nontemporal_store(u[0], (GLOBAL uint32_t*)p);
        else *(GLOBAL uint32_t*)p = u[0];
    } else {
        V x;
#pragma unroll
        for (int k = 0; k < DWORDS; ++k) x[k] = u[k];
        if (STREAM) __builtin_nontemporal_store(x, (GLOBAL V*)p);
        else *(GLOBAL V*)p = x;
    }
}
template <int BITS, int W, bool FULL, bool STREAM>
__device__ __forceinline__ Raw<BITS, W> load(const void* base, int64_t i, int live) {
    const uint8_t* const p = (const uint8_t*)base + i * (BITS / 8);
    Raw<BITS, W> o;
    if constexpr (FULL) {
        load_dwords<STREAM>(p, o.u);
    } else {
        constexpr int PER = 32 / BITS;                            // elements of a dword
#pragma unroll
        for (int k = 0; k < BITS * W / 32; ++k) o.u[k] = 0;
#pragma unroll
        for (int k = 0; k < W; ++k)
            if (k < live)
                o.u[k / PER] |= (BITS == 32 ? *(const GLOBAL uint32_t*)(p + 4 * k) : BITS == 16 ? *(const GLOBAL uint16_t*)(p + 2 * k)
                                                                                    : *(const GLOBAL uint8_t*)(p + k)) << (BITS % 32 * (k % PER));
    }
    return o;
}
template <int BITS, int W, bool FULL, bool STREAM>
__device__ __forceinline__ void store(void* base, int64_t i, int live, const Raw<BITS, W>& x) {
    uint8_t* const p = (uint8_t*)base + i * (BITS / 8);
    if constexpr (FULL) {
        store_dwords<STREAM>(p, x.u);
    } else {
        constexpr int PER = 32 / BITS;
#pragma unroll
        for (int k = 0; k < W; ++k)
            if (k < live) {
                const uint32_t v = x.u[k / PER] >> (BITS % 32 * (k % PER));
                if (BITS == 32) *(GLOBAL uint32_t*)(p + 4 * k) = v;
                else if (BITS == 16) *(GLOBAL uint16_t*)(p + 2 * k) = (uint16_t)v;
                else *(GLOBAL uint8_t*)(p + k) = (uint8_t)v;
            }
    }
}
template <int BITS, int W>
__device__ __forceinline__ Vec<W> values(const Raw<BITS, W>& r) {  // fp32, bf16 or e4m3
    Vec<W> o;
    if constexpr (BITS == 8) {
#pragma unroll
        for (int k = 0; k < W / 4; ++k) {
            const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.u[k], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.u[k], true);
            o.v[4 * k] = a[0]; o.v[4 * k + 1] = a[1]; o.v[4 * k + 2] = b[0]; o.v[4 * k + 3] = b[1];
        }
    } else {
#pragma unroll
        for (int k = 0; k < W; ++k)
            o.v[k] = __uint_as_float(BITS == 32 ? r.u[k] : k & 1 ? r.u[k / 2] & 0xFFFF0000u : r.u[k / 2] << 16);
    }
    return o;
}
template <int W>
__device__ __forceinline__ Raw<32, W> raw_f32(const Vec<W>& x) {
    Raw<32, W> o;
#pragma unroll
    for (int k = 0; k < W; ++k) o.u[k] = __float_as_uint(x.v[k]);
    return o;
}
template <int W>
__device__ __forceinline__ Raw<16, W> raw_bf16(const Vec<W>& x) {
    Raw<16, W> o;
#pragma unroll
    for (int k = 0; k < W / 2; ++k) {
        union { __bf16 h[2]; uint32_t u; } t;
        t.h[0] = (__bf16)x.v[2 * k]; t.h[1] = (__bf16)x.v[2 * k + 1];
        o.u[k] = t.u;
    }
    return o;
}

struct StepArgs {
    const void* table;
    int64_t count, chunks;
    float lr, b1, b2, c1, c2, eps, log_b1, log_b2, grad_scale;    // c = 1 - b
    float step;
    const float* control;                                         // or null
};

// The W values of each of 128 / W lanes to codes, with the block's scale to *scale.  The conversion takes a value to one of its e4m3
// neighbours: up where the part of the way from the lower one, in magnitude, plus u (its upper 20 bits, as a fraction) reaches 1.
template <bool ROOT, int W>
__device__ __forceinline__ Raw<8, W> to_codes(const Vec<W>& x, uint32_t u, GLOBAL float* scale, bool writes) {
#pragma clang fp contract(off)
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < W; ++k) top = ROOT ? __uint_as_float(max(__float_as_uint(top), __float_as_uint(x.v[k]))) : max_abs(top, x.v[k]);
    const Q8Scale s = q8_scale(lanes_max_abs<Q8_BLOCK / W>(top));
    if (writes) *scale = s.scale;
    // a root below the smallest code becomes that code, whatever u is
    auto held = [&](float v) {
        const float a = v * s.inv;
        if (ROOT) return a > 0.0f ? __builtin_amdgcn_fmed3f(a, 0.001953125f, Q8_MAX) : 0.0f;
        return __builtin_amdgcn_fmed3f(a, -Q8_MAX, Q8_MAX);
    };
    Raw<8, W> o;
#pragma unroll
    for (int k = 0; k < W; k += 4) {
        int c = __builtin_amdgcn_cvt_sr_fp8_f32(held(x.v[k]), (int)(u + (uint32_t)k * DITHER_INDEX), 0, 0);
        c = __builtin_amdgcn_cvt_sr_fp8_f32(held(x.v[k + 1]), (int)(u + (uint32_t)(k + 1) * DITHER_INDEX), c, 1);
        c = __builtin_amdgcn_cvt_sr_fp8_f32(held(x.v[k + 2]), (int)(u + (uint32_t)(k + 2) * DITHER_INDEX), c, 2);
        c = __builtin_amdgcn_cvt_sr_fp8_f32(held(x.v[k + 3]), (int)(u + (uint32_t)(k + 3) * DITHER_INDEX), c, 3);
        o.u[k / 4] = s.scale < INFINITY ? (uint32_t)c : 0x7F7F7F7Fu;    // else the block holds an infinity or NaN
    }
    return o;
}

// Square roots, exactly rounded: the hardware's is off by one unit at most, and the residuals of its neighbours tell (P. W. Markstein,
// Computation of elementary functions on the IBM RISC System/6000 processor, IBM J. Res. Dev. 34, 1990: the final rounding of a root).  (Zeros, infinities
// and NaN stay as they are: their residuals are no numbers, or zero.)  Below 2^-96 residuals would vanish: the compiler's form for all then.
template <int W>
__device__ __forceinline__ Vec<W> roots(const Vec<W>& x) {
    Vec<W> o;
    bool tiny = false;
#pragma unroll
    for (int k = 0; k < W; ++k) tiny |= x.v[k] < 0x1p-96f && x.v[k] != 0.0f;
    if (__builtin_expect(__any(tiny), 0)) {
#pragma unroll
        for (int k = 0; k < W; ++k) o.v[k] = sqrtf(x.v[k]);
        return o;
    }
#pragma unroll
    for (int k = 0; k < W; ++k) {
        const float s = __builtin_amdgcn_sqrtf(x.v[k]);
        const float down = __uint_as_float(__float_as_uint(s) - 1), up = __uint_as_float(__float_as_uint(s) + 1);
        const float below = fmaf(-down, s, x.v[k]), above = fmaf(-up, s, x.v[k]);
        o.v[k] = above > 0.0f ? up : below <= 0.0f ? down : s;
    }
    return o;
}

struct Rates { float coef, rate, inv_root2, keep, t; };

// One chunk of a tensor, whole (FULL) or its last part
template <int THREADS, bool STATE8, bool MASTER, bool GRAD32, bool FULL, bool STREAM>
__device__ __forceinline__ void adamw_chunk(const StepArgs& a, const slope_adamw_tensor& tensor, int64_t start, const Rates& c) {
#pragma clang fp contract(off)
    constexpr int W = STATE8 && !MASTER && !GRAD32 ? 8 : 4, BLOCK_LANES = Q8_BLOCK / W;
    constexpr int PIECES = CHUNK / (THREADS * W);                 // of a lane
    constexpr int S = STATE8 ? 8 : 32, G = GRAD32 ? 32 : 16, P = MASTER ? 32 : 16;
    const int lane = (int)threadIdx.x & (BLOCK_LANES - 1);
    auto live_at = [&](int64_t i) { return FULL ? W : tensor.n - i >= W ? W : tensor.n - i > 0 ? (int)(tensor.n - i) : 0; };
    auto there = [&](int64_t i) { return FULL || i - lane * W < tensor.n; };     // a block of 128 is there or not as a whole
    const void* const value = MASTER ? tensor.master : tensor.param;
    Raw<G, W> graw[PIECES];
    Raw<P, W> praw[PIECES];
    Raw<S, W> mraw[PIECES], vraw[PIECES];
    float ms[PIECES], vs[PIECES];
#pragma unroll
    for (int t = 0; t < PIECES; ++t) {
        const int64_t i = start + (t * THREADS + (int)threadIdx.x) * W;
        const int live = live_at(i);
        if (!there(i)) continue;
        graw[t] = load<G, W, FULL, STREAM>(tensor.grad, i, live);
        praw[t] = load<P, W, FULL, STREAM>(value, i, live);
        mraw[t] = load<S, W, FULL, STREAM>(tensor.m, i, live);
        vraw[t] = load<S, W, FULL, STREAM>(tensor.v, i, live);
        if (STATE8) {
            ms[t] = ((const GLOBAL float*)tensor.m_scale)[i / Q8_BLOCK];
            vs[t] = ((const GLOBAL float*)tensor.v_scale)[i / Q8_BLOCK];
        }
    }
#pragma unroll
    for (int t = 0; t < PIECES; ++t) {
        const int64_t i = start + (t * THREADS + (int)threadIdx.x) * W;
        const int live = live_at(i);
        if (!there(i)) continue;
        const Vec<W> g = values(graw[t]);
        Vec<W> p = values(praw[t]), m = values(mraw[t]), v = values(vraw[t]), r;
#pragma unroll
        for (int k = 0; k < W; ++k) {
            if (STATE8) {
                m.v[k] *= ms[t];
                v.v[k] *= vs[t];
                v.v[k] *= v.v[k];
            }
            const float x = g.v[k] * c.coef;
            m.v[k] = m.v[k] * a.b1 + x * a.c1;
            v.v[k] = v.v[k] * a.b2 + x * x * a.c2;
        }
        r = roots(v);
#pragma unroll
        for (int k = 0; k < W; ++k)
            p.v[k] = fmaf(-c.rate, m.v[k] * __builtin_amdgcn_rcpf(fmaf(r.v[k], c.inv_root2, a.eps)), p.v[k] * c.keep);
        if constexpr (MASTER) store<32, W, FULL, STREAM>(tensor.master, i, live, raw_f32(p));
        if (!MASTER || tensor.param) store<16, W, FULL, STREAM>(tensor.param, i, live, raw_bf16(p));
        if constexpr (STATE8) {
            const uint32_t u = (uint32_t)i * DITHER_INDEX + (uint32_t)(int)c.t * DITHER_STEP;
            store<8, W, FULL, STREAM>(tensor.m, i, live, to_codes<false>(m, u, (GLOBAL float*)tensor.m_scale + i / Q8_BLOCK, lane == 0));
            store<8, W, FULL, STREAM>(tensor.v, i, live, to_codes<true>(r, u + 0x80000000u, (GLOBAL float*)tensor.v_scale + i / Q8_BLOCK, lane == 0));
        } else {
            store<32, W, FULL, STREAM>(tensor.m, i, live, raw_f32(m));
            store<32, W, FULL, STREAM>(tensor.v, i, live, raw_f32(v));
        }
    }
}

template <int THREADS, bool STATE8, bool STREAM>
__global__ void __launch_bounds__(THREADS) adamw_kernel(StepArgs a) {
    if (flat_block() >= a.chunks) return;
    const Chunk chunk = chunks_of(a.table, a.count)[flat_block()];
    Rates c;
    c.coef = a.grad_scale;
    c.t = a.step;
    if (a.control) {
        if (!(fabsf(a.control[0]) < INFINITY)) return;            // a gradient is not finite: the step is left out
        c.coef = a.control[1];
        c.t = a.control[2];
    }
    const slope_adamw_tensor tensor = tensors_of(a.table)[chunk.tensor];
    c.rate = a.lr / -expm1f(c.t * a.log_b1);
    c.inv_root2 = 1.0f / sqrtf(-expm1f(c.t * a.log_b2));
    c.keep = 1.0f - a.lr * tensor.weight_decay;
    const int64_t start = (int64_t)chunk.part * CHUNK;
    const bool full = tensor.n - start >= CHUNK;
#define CHUNK_OF(M, G) full ? adamw_chunk<THREADS, STATE8, M, G, true, STREAM>(a, tensor, start, c) : adamw_chunk<THREADS, STATE8, M, G, false, false>(a, tensor, start, c)
    if (tensor.master) {
        if (tensor.grad_bits == 32) CHUNK_OF(true, true);
        else CHUNK_OF(true, false);
    } else {
        if (tensor.grad_bits == 32) CHUNK_OF(false, true);
        else CHUNK_OF(false, false);
    }
#undef CHUNK_OF
}

// Sum of squares of a workgroup's run of chunks, one partial sum a workgroup.  (157 M elements, us: chunk w, w + 2048, ... 96; runs of
// neighbours, whose table entries come together, 55; 8192 shorter runs 50, and 11 for the sum of that many.  The last workgroup to be
// done as the one that adds them, in one launch: 244, the release of 4096 partial sums to all dies one after the other.)
constexpr int NORM_GROUPS = 4096, FINISH_THREADS = 1024;
__device__ __forceinline__ float block_sum(float v) {
    __shared__ float part[THREADS / 64];
    v = lanes_sum<64>(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
    for (int i = 1; i < THREADS / 64; ++i) v += part[i];
    return v;
}
template <int BITS, bool FULL>
__device__ __forceinline__ float chunk_squares(const void* grad, int64_t n, int64_t start, float sum) {
    constexpr int W = 128 / BITS, PIECES = CHUNK / (THREADS * W);
    Raw<BITS, W> raw[PIECES];
#pragma unroll
    for (int piece = 0; piece < PIECES; ++piece) {
        const int64_t i = start + (piece * THREADS + (int)threadIdx.x) * W;
        raw[piece] = load<BITS, W, FULL, false>(grad, i, n - i >= W ? W : n - i > 0 ? (int)(n - i) : 0);
    }
#pragma unroll
    for (int piece = 0; piece < PIECES; ++piece) {
        const Vec<W> g = values(raw[piece]);
#pragma unroll
        for (int k = 0; k < W; ++k) sum = fmaf(g.v[k], g.v[k], sum);
    }
    return sum;
}
__global__ void __launch_bounds__(THREADS) grad_norm_kernel(const void* table, int64_t count, int64_t chunks, float* part) {
    float sum = 0.0f;
    const int64_t each = (chunks + gridDim.x - 1) / gridDim.x, first = blockIdx.x * each, last = min(chunks, first + each);
    for (int64_t w = first; w < last; ++w) {
        const Chunk c = chunks_of(table, count)[w];
        const slope_adamw_tensor& tensor = tensors_of(table)[c.tensor];
        const int64_t start = (int64_t)c.part * CHUNK;
        const bool full = tensor.n - start >= CHUNK;
        if (tensor.grad_bits == 32)
            sum = full ? chunk_squares<32, true>(tensor.grad, tensor.n, start, sum) : chunk_squares<32, false>(tensor.grad, tensor.n, start, sum);
        else
            sum = full ? chunk_squares<16, true>(tensor.grad, tensor.n, start, sum) : chunk_squares<16, false>(tensor.grad, tensor.n, start, sum);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}
// control = {norm, factor for the gradients, steps taken, 0}
__global__ void __launch_bounds__(FINISH_THREADS) grad_norm_finish_kernel(const float* part, int groups, float inv_scale, float max_norm, float* control) {
    __shared__ double sums[FINISH_THREADS / 64];
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < NORM_GROUPS / FINISH_THREADS; ++i) {
        const int at = i * FINISH_THREADS + threadIdx.x;
        s += at < groups ? (double)part[at] : 0.0;
    }
#pragma unroll
    for (int x = 1; x < 64; x *= 2) s += __shfl_xor(s, x);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int i = 1; i < FINISH_THREADS / 64; ++i) sums[0] += sums[i];
    const float norm = (float)(sqrt(sums[0]) * (double)inv_scale);
    const bool fine = fabsf(norm) < INFINITY;
    control[0] = norm;
    control[1] = fine ? inv_scale * fminf(max_norm / (norm + 1e-6f), 1.0f) : 0.0f;
    if (fine) control[2] += 1.0f;
}

const Header* header_of(const void* table) {
    const Header* h = (const Header*)table;
    return h->magic == MAGIC ? h : nullptr;
}

int64_t chunks_of_tensor(int64_t n) { return (n + CHUNK - 1) / CHUNK; }

int norm_groups(int64_t chunks) { return (int)(chunks < NORM_GROUPS ? chunks : NORM_GROUPS); }

}  // namespace

int64_t adamw_chunks(const slope_adamw_tensor* tensors, int64_t count) {
    int64_t chunks = 0;
    for (int64_t i = 0; i < count; ++i) chunks += chunks_of_tensor(tensors[i].n);
    return chunks;
}

size_t adamw_table_bytes(int64_t count, int64_t chunks) {
    return sizeof(Header) + (size_t)count * sizeof(slope_adamw_tensor) + (size_t)chunks * sizeof(Chunk);
}

void adamw_fill_table(const slope_adamw_tensor* tensors, int64_t count, int state_bits, void* table) {
    const int64_t chunks = adamw_chunks(tensors, count);
    Header h = {};
    h.magic = MAGIC;
    h.count = count;
    h.chunks = chunks;
    h.bytes = (int64_t)adamw_table_bytes(count, chunks);
    h.state_bits = state_bits;
    memcpy(table, &h, sizeof h);
    uint8_t* at = (uint8_t*)table + sizeof h;
    memcpy(at, tensors, (size_t)count * sizeof *tensors);
    Chunk* c = (Chunk*)(at + (size_t)count * sizeof *tensors);
    for (int64_t i = 0; i < count; ++i)
        for (int64_t k = 0; k < chunks_of_tensor(tensors[i].n); ++k) *c++ = {(int32_t)i, (int32_t)k};
}

bool adamw_table_ok(const void* table) { return header_of(table) != nullptr; }

size_t grad_norm_workspace_bytes(const void* table) {
    const Header* h = header_of(table);
    return h ? (size_t)(norm_groups(h->chunks) > 0 ? norm_groups(h->chunks) : 1) * 4 : 0;
}

hipError_t launch_grad_norm(const void* table, const void* device_table, float inv_scale, float max_norm, float* control,
                            float* part, hipStream_t s) {
    const Header* h = header_of(table);
    const int groups = norm_groups(h->chunks);
    if (groups > 0) grad_norm_kernel<<<groups, THREADS, 0, s>>>(device_table, h->count, h->chunks, part);
    grad_norm_finish_kernel<<<1, FINISH_THREADS, 0, s>>>(part, groups, inv_scale, max_norm, control);
    return hipGetLastError();
}

hipError_t launch_adamw(const void* table, const void* device_table, double lr, double beta1, double beta2, double eps,
                        double grad_scale, int64_t step, const float* control, hipStream_t s) {
    const Header* h = header_of(table);
    if (h->chunks == 0) return hipSuccess;
    const StepArgs a = {device_table, h->count, h->chunks, (float)lr, (float)beta1, (float)beta2, (float)(1.0 - beta1), (float)(1.0 - beta2),
                        (float)eps, (float)log(beta1), (float)log(beta2), (float)grad_scale, (float)step, control};
    const dim3 grid = grid_of(h->chunks);
    // a set that the last-level cache does not hold goes past it (us, through it / past it: 157 M elements with masters, 32-bit states
    // and the norm 897 / 771, 8-bit states 473 / 427; 531 M, 8-bit states, bf16 weights 959 / 911 to 947)
    const bool stream = (size_t)h->chunks * CHUNK * (h->state_bits == 8 ? 8 : 16) > LAST_LEVEL_CACHE_BYTES;
    // few chunks: more wavefronts on each, so that all of its loads are under way at once (0.9 M elements with masters,
    // us, 256 / 512: with the norm 17.1 / 15.7; 8-bit states 11.1 / 10.0)
    const bool few = h->chunks < 4 * RESIDENT;
    if (h->state_bits == 8 && stream) adamw_kernel<THREADS, true, true><<<grid, THREADS, 0, s>>>(a);
    else if (h->state_bits == 8 && few) adamw_kernel<512, true, false><<<grid, 512, 0, s>>>(a);
    else if (h->state_bits == 8) adamw_kernel<THREADS, true, false><<<grid, THREADS, 0, s>>>(a);
    else if (stream) adamw_kernel<THREADS, false, true><<<grid, THREADS, 0, s>>>(a);
    else if (few) adamw_kernel<512, false, false><<<grid, 512, 0, s>>>(a);
    else adamw_kernel<THREADS, false, false><<<grid, THREADS, 0, s>>>(a);
    return hipGetLastError();
}
