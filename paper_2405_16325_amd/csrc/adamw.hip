// AdamW over many tensors in one launch, and the gradients' global norm.
//
//     g = c grad      m = b1 m + (1 - b1) g      v = b2 v + (1 - b2) g^2
//     p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Memory bounds both: every element is read and written once, 28 bytes of it with 32-bit states and fp32 master weights, 10
// with 8-bit states and bf16 weights alone.  The tensors of a set are cut into chunks of CHUNK elements; a table in device
// memory (laid out once by adamw_fill_table) names each chunk's tensor, so that one launch covers hundreds of tensors of
// any sizes evenly and a workgroup finds its work with two scalar loads.
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
// part of the format: the codes and scales are the same whatever computes them.
#include "wave.h"
#include <math.h>
#include <string.h>

namespace {

constexpr int THREADS = 256, PER_LANE = 8;
constexpr int TURNS = 2;                                        // pieces of THREADS x PER_LANE elements per chunk
constexpr int CHUNK = THREADS * PER_LANE * TURNS;
constexpr int Q8_BLOCK = SLOPE_ADAMW_BLOCK;
static_assert(Q8_BLOCK == 16 * PER_LANE, "sixteen lanes hold a block");
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

// eight neighbours from element i of n on: all of them, or the last few
__device__ __forceinline__ F8 load_f32(const float* p, int64_t i, int live) {
    F8 o;
    if (live == 8) {
        const f32x4 a = *(const f32x4*)(p + i), b = *(const f32x4*)(p + i + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) o.v[k] = a[k], o.v[4 + k] = b[k];
        return o;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) o.v[k] = k < live ? p[i + k] : 0.0f;
    return o;
}
__device__ __forceinline__ F8 load_bf16(const bf16_t* p, int64_t i, int live) {
    if (live == 8) return unpack_bf16(*(const u32x4*)(p + i));
    F8 o;
#pragma unroll
    for (int k = 0; k < 8; ++k) o.v[k] = k < live ? __uint_as_float((uint32_t)p[i + k] << 16) : 0.0f;
    return o;
}
__device__ __forceinline__ u32x2 load_codes(const uint8_t* p, int64_t i, int live) {
    if (live == 8) return *(const u32x2*)(p + i);
    u32x2 o = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < live) o[k >> 2] |= (uint32_t)p[i + k] << (8 * (k & 3));
    return o;
}
__device__ __forceinline__ void store_f32(float* p, int64_t i, int live, const F8& x) {
    if (live == 8) {
        *(f32x4*)(p + i) = (f32x4){x.v[0], x.v[1], x.v[2], x.v[3]};
        *(f32x4*)(p + i + 4) = (f32x4){x.v[4], x.v[5], x.v[6], x.v[7]};
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < live) p[i + k] = x.v[k];
}
__device__ __forceinline__ void store_bf16(bf16_t* p, int64_t i, int live, const F8& x) {
    const u32x4 o = pack_bf16(x);
    if (live == 8) {
        *(u32x4*)(p + i) = o;
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < live) p[i + k] = (bf16_t)(o[k >> 1] >> (16 * (k & 1)));
}
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t i, int live, u32x2 o) {
    if (live == 8) {
        *(u32x2*)(p + i) = o;
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < live) p[i + k] = (uint8_t)(o[k >> 2] >> (8 * (k & 3)));
}

// |x| <= 448 to one of its e4m3 neighbours: up where the part of the distance that x is above the lower one, plus u, reaches 1
// (u: its upper 20 bits, as a fraction).  Below 2^-6 the codes are 2^-9 apart throughout: 2^-6 is added first, so that the
// sum's lowest kept mantissa bit is worth that much, and taken off again.
__device__ __forceinline__ float dithered(float x, uint32_t u) {
    const float low = x < 0.015625f ? 0.015625f : 0.0f;
    return __uint_as_float((__float_as_uint(x + low) + (u >> 12)) & 0xFFF00000u) - low;
}

struct StepArgs {
    const void* table;
    int64_t count, chunks;
    float lr, b1, b2, c1, c2, eps, log_b1, log_b2, grad_scale;    // c = 1 - b
    float step;
    const float* control;                                         // or null
};

// sixteen lanes' eight values each to codes; x's block scale goes to scales[block]
template <bool ROOT>
__device__ __forceinline__ u32x2 to_codes(F8& x, uint32_t u, float* scale, bool writes) {
#pragma clang fp contract(off)
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max_abs(top, x.v[k]);
    const Q8Scale s = q8_scale(lanes_max_abs<16>(top));
    if (writes) *scale = s.scale;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float a = fminf(fabsf(x.v[k]) * s.inv, Q8_MAX);
        float q = dithered(a, u + (uint32_t)k * DITHER_INDEX);
        if (ROOT) {
            if (a > 0.0f) q = fmaxf(q, 0.001953125f);
            x.v[k] = q;
        } else {
            x.v[k] = copysignf(q, x.v[k]);
        }
        if (!(s.scale < INFINITY)) x.v[k] = NAN;                  // the block holds an infinity or NaN
    }
    return pack_e4m3(x);
}

template <bool STATE8>
__global__ void __launch_bounds__(THREADS) adamw_kernel(StepArgs a) {
#pragma clang fp contract(off)
    float coef = a.grad_scale, t = a.step;
    if (a.control) {
        if (!(fabsf(a.control[0]) < INFINITY)) return;            // a gradient is not finite: the step is left out
        coef = a.control[1];
        t = a.control[2];
    }
    if (flat_block() >= a.chunks) return;
    const Chunk c = chunks_of(a.table, a.count)[flat_block()];
    const slope_adamw_tensor tensor = tensors_of(a.table)[c.tensor];
    const float rate = a.lr / -expm1f(t * a.log_b1), inv_root2 = 1.0f / sqrtf(-expm1f(t * a.log_b2));
    const float keep = 1.0f - a.lr * tensor.weight_decay;
#pragma unroll
    for (int turn = 0; turn < TURNS; ++turn) {
        const int64_t i = (int64_t)c.part * CHUNK + (turn * THREADS + (int)threadIdx.x) * PER_LANE;
        if (i - (int64_t)(threadIdx.x & 15) * PER_LANE >= tensor.n) continue;     // the block of 128 as a whole
        const int live = tensor.n - i >= 8 ? 8 : tensor.n - i > 0 ? (int)(tensor.n - i) : 0;
        const F8 g = tensor.grad_bits == 32 ? load_f32((const float*)tensor.grad, i, live) : load_bf16((const bf16_t*)tensor.grad, i, live);
        F8 p = tensor.master ? load_f32((const float*)tensor.master, i, live) : load_bf16((const bf16_t*)tensor.param, i, live);
        F8 m, v;
        if constexpr (STATE8) {
            m = unpack_e4m3(load_codes((const uint8_t*)tensor.m, i, live));
            v = unpack_e4m3(load_codes((const uint8_t*)tensor.v, i, live));
            const float ms = tensor.m_scale[i / Q8_BLOCK], vs = tensor.v_scale[i / Q8_BLOCK];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                m.v[k] *= ms;
                v.v[k] *= vs;
                v.v[k] *= v.v[k];
            }
        } else {
            m = load_f32((const float*)tensor.m, i, live);
            v = load_f32((const float*)tensor.v, i, live);
        }
        F8 r;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float x = g.v[k] * coef;
            m.v[k] = m.v[k] * a.b1 + x * a.c1;
            v.v[k] = v.v[k] * a.b2 + x * x * a.c2;
            r.v[k] = sqrtf(v.v[k]);
            p.v[k] = p.v[k] * keep - rate * (m.v[k] / (r.v[k] * inv_root2 + a.eps));
        }
        if (tensor.master) store_f32((float*)tensor.master, i, live, p);
        if (tensor.param) store_bf16((bf16_t*)tensor.param, i, live, p);
        if constexpr (STATE8) {
            const uint32_t u = (uint32_t)i * DITHER_INDEX + (uint32_t)(int)t * DITHER_STEP;
            const bool first = (threadIdx.x & 15) == 0;
            store_codes((uint8_t*)tensor.m, i, live, to_codes<false>(m, u, tensor.m_scale + i / Q8_BLOCK, first));
            store_codes((uint8_t*)tensor.v, i, live, to_codes<true>(r, u + 0x80000000u, tensor.v_scale + i / Q8_BLOCK, first));
        } else {
            store_f32((float*)tensor.m, i, live, m);
            store_f32((float*)tensor.v, i, live, v);
        }
    }
}

// Sum of squares of a workgroup's chunks: chunk w, w + grid, ...  One partial sum a workgroup.
constexpr int NORM_GROUPS = 2048;
__device__ __forceinline__ float block_sum(float v) {
    __shared__ float part[THREADS / 64];
    v = lanes_sum<64>(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
    for (int i = 1; i < THREADS / 64; ++i) v += part[i];
    return v;
}
__global__ void __launch_bounds__(THREADS) grad_norm_kernel(const void* table, int64_t count, int64_t chunks, float* part) {
    float sum = 0.0f;
    for (int64_t w = blockIdx.x; w < chunks; w += gridDim.x) {
        const Chunk c = chunks_of(table, count)[w];
        const slope_adamw_tensor& tensor = tensors_of(table)[c.tensor];
#pragma unroll
        for (int turn = 0; turn < TURNS; ++turn) {
            const int64_t i = (int64_t)c.part * CHUNK + (turn * THREADS + (int)threadIdx.x) * PER_LANE;
            const int live = tensor.n - i >= 8 ? 8 : tensor.n - i > 0 ? (int)(tensor.n - i) : 0;
            if (live == 0) continue;
            const F8 g = tensor.grad_bits == 32 ? load_f32((const float*)tensor.grad, i, live) : load_bf16((const bf16_t*)tensor.grad, i, live);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum = fmaf(g.v[k], g.v[k], sum);
        }
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}
// control = {norm, factor for the gradients, steps taken, 0}
__global__ void __launch_bounds__(THREADS) grad_norm_finish_kernel(const float* part, int groups, float inv_scale, float max_norm, float* control) {
    __shared__ double sums[THREADS];
    double s = 0.0;
    for (int i = threadIdx.x; i < groups; i += THREADS) s += (double)part[i];
    sums[threadIdx.x] = s;
    __syncthreads();
    for (int half = THREADS / 2; half > 0; half /= 2) {
        if ((int)threadIdx.x < half) sums[threadIdx.x] += sums[threadIdx.x + half];
        __syncthreads();
    }
    if (threadIdx.x != 0) return;
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
    grad_norm_finish_kernel<<<1, THREADS, 0, s>>>(part, groups, inv_scale, max_norm, control);
    return hipGetLastError();
}

hipError_t launch_adamw(const void* table, const void* device_table, double lr, double beta1, double beta2, double eps,
                        double grad_scale, int64_t step, const float* control, hipStream_t s) {
    const Header* h = header_of(table);
    if (h->chunks == 0) return hipSuccess;
    const StepArgs a = {device_table, h->count, h->chunks, (float)lr, (float)beta1, (float)beta2, (float)(1.0 - beta1), (float)(1.0 - beta2),
                        (float)eps, (float)log(beta1), (float)log(beta2), (float)grad_scale, (float)step, control};
    const dim3 grid = grid_of(h->chunks);
    if (h->state_bits == 8) adamw_kernel<true><<<grid, THREADS, 0, s>>>(a);
    else adamw_kernel<false><<<grid, THREADS, 0, s>>>(a);
    return hipGetLastError();
}
