// The description of a matrix product that the host hands to the product kernels, and the elementwise pieces that
// products and passes share.
#pragma once

#include "ssd_layers_common.cuh"

#include <cuda_bf16.h>

#include <cmath>
#include <cstdint>

namespace ssd_layers {

// ---------------------------------------------------------------------------------------------------------
// A product: C[m, n] = sum over segments s, over k, of A_s[m, k] * B_s[n, k], summed in float32.
//
// Operands are bfloat16 planes of row-major matrices.  A segment names one plane of A and one of B; one segment is a plain
// bfloat16 product, several are the partial products of operands in parts, or the two halves of the gated
// dx = dgate w_gate + dup w_up.  Segments are ordered from the smallest contribution to the largest, so that the
// running sum is small while the small terms arrive.

struct Planes {
    const __nv_bfloat16 *p;
    int64_t ld;            // elements between rows
    int64_t zstride;       // elements between planes
    int rows, cols, nz;    // as stored
};

struct Segment {
    int8_t az, b, bz;      // plane of A, which B operand, its plane
};

constexpr int kMaxSegments = 12;

struct Epilogue {
    // out = act(acc + bias) (* (acc2 + bias2)) + residual; z receives acc + bias before the activation.
    // Index 0 / 1: the gate and up halves of a gated product, or the groups of a grouped one.
    const float *bias[2];
    const void *residual;
    int64_t ldr;
    void *out[2];
    int64_t ldo[2];
    void *z[2];
    int64_t ldz[2];
    int act;
    int f32;               // type of residual, out and z: float32, else bfloat16
    int vec;               // bytes that every row of residual, out and z is aligned to: 32, 16, or less (0)
};

struct Product {
    Planes a, b[2];
    int a_mn, b_mn;        // operand stored with the product's row index along its rows (contraction runs down the rows)
    int nseg, nmain;       // the last nmain segments carry the leading terms
    Segment seg[kMaxSegments];
    int m, n, k;           // sizes of one group, k per segment
    int groups;            // > 1: group g uses plane az + g of A and out[g]
    int gated;             // two B operands side by side, combined in the epilogue
    Epilogue e;
};

// Enqueues the product (csrc/ssd_product.cu) and counts its launches.  partial: workspace of product_partial_floats() floats, which depends on the
// sizes and on e.vec alone.
int64_t product_partial_floats(const Product &p);
cudaError_t launch_product(const Product &p, float *partial, cudaStream_t stream);
double product_us(const Product &p);      // its estimated time: of p the sizes, groups, gated, nseg and e.vec

// A few rows (csrc/ssd_rows.cu).

struct RowsForward {
    const void *x, *w[2];
    int64_t ldx, ldw[2];
    int rows, in, out, gated;
    int slices, across;                  // set by the launcher: warps that share a contraction, blocks over the weight rows
    Epilogue e;
};

struct RowsBackward {
    const void *dy, *x, *w[2], *z[2];
    int64_t lddy, ldx, ldw[2], ldz[2];
    void *dx, *dw[2], *db[2];            // NULL: not wanted
    int64_t lddx, lddw[2];
    float *partial;                      // rows_partial_floats() of workspace if dx is wanted, else NULL
    int rows, in, out, act, mats, f32, grad_f32, strip;
};

cudaError_t launch_rows_forward(RowsForward p, cudaStream_t stream);        // these count their launches themselves
double rows_forward_f32_us(const RowsForward &p);                           // the estimated time for float32 and more than four rows
bool rows_mma_pays(const RowsForward &p);                                   // bfloat16 in aligned rows, two of them or more: whether these kernels are the faster ones
int64_t rows_partial_floats(int rows, int out, int in);
cudaError_t launch_rows_backward(RowsBackward p, cudaStream_t stream);

// Whether a bounded wait of a product kernel ever ran out.
cudaError_t read_product_error(int *flag);

// ---------------------------------------------------------------------------------------------------------
// Elementwise pieces.

template <typename T> __device__ __forceinline__ float load_as_float(const T *p);
template <> __device__ __forceinline__ float load_as_float<float>(const float *p) { return *p; }
template <> __device__ __forceinline__ float load_as_float<__nv_bfloat16>(const __nv_bfloat16 *p) { return __bfloat162float(*p); }

__device__ __forceinline__ float load_at(const void *p, int64_t i, int f32)
{
    return f32 ? static_cast<const float *>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}
__device__ __forceinline__ void store_at(void *p, int64_t i, int f32, float v)
{
    if (f32) static_cast<float *>(p)[i] = v;
    else static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
}

__device__ __forceinline__ float activate(float v, int act);

// One element of the result from its sum (and, gated, the second one).  `residual`: its value there, loaded before the stores of other elements
// so that the loads of several elements are under way together.
template <bool GATED> __device__ __forceinline__ void finish(const Epilogue &e, int group, int64_t m, int n, float v, float u, float residual)
{
    if (e.z[0]) store_at(e.z[0], m * e.ldz[0] + n, e.f32, v);
    v = activate(v, e.act);
    if (GATED) {
        if (e.z[1]) store_at(e.z[1], m * e.ldz[1] + n, e.f32, u);
        v *= u;
    }
    if (e.residual) v += residual;
    store_at(e.out[group], m * e.ldo[group] + n, e.f32, v);
}
__device__ __forceinline__ float residual_at(const Epilogue &e, int64_t m, int n) { return e.residual ? load_at(e.residual, m * e.ldr + n, e.f32) : 0.0f; }

// The passes over dz are long enough that these decide between memory and arithmetic as their bound, so each
// function takes one exponential and one reciprocal.
// The normal distribution function and density: the rational form 7.1.26 of Abramowitz and Stegun for erf(v / sqrt(2)), which
// is off by at most 1.5e-7 absolutely (Phi by half of that), and shares its exponential with the density.
__device__ __forceinline__ float normal_cdf(float v, float *density)
{
    const float x = fabsf(v) * 0.70710678f;
    const float g = __expf(-x * x);
    const float t = __fdividef(1.0f, fmaf(0.3275911f, x, 1.0f));
    const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    const float tail = 0.5f * poly * g;             // 1 - Phi(|v|)
    *density = 0.39894228f * g;
    return v < 0.0f ? tail : 1.0f - tail;           // a NaN stays one
}
// 1 / (1 + exp(-v)); 0 and 1 at the ends.
__device__ __forceinline__ float sigmoid(float v) { return __fdividef(1.0f, 1.0f + __expf(-v)); }

__device__ __forceinline__ float activate(float v, int act)
{
    if (act == SSD_ACT_RELU) return v < 0.0f ? 0.0f : v;              // a NaN stays one
    float density;
    if (act == SSD_ACT_GELU) return v * normal_cdf(v, &density);
    if (act == SSD_ACT_SILU) return v * sigmoid(v);
    return v;
}

// act(v) and act'(v).
__device__ __forceinline__ void activate_both(float v, int act, float *value, float *slope)
{
    if (act == SSD_ACT_RELU) {
        *value = v < 0.0f ? 0.0f : v;
        *slope = v > 0.0f ? 1.0f : 0.0f;
    } else if (act == SSD_ACT_GELU) {
        float density;
        const float cdf = normal_cdf(v, &density);
        *value = v * cdf;
        *slope = fmaf(v, density, cdf);
    } else if (act == SSD_ACT_SILU) {
        const float s = sigmoid(v);
        *value = v * s;
        *slope = s * fmaf(v, 1.0f - s, 1.0f);
    } else {
        *value = v;
        *slope = 1.0f;
    }
}

// ---------------------------------------------------------------------------------------------------------
// Epilogue of 32 columns of a row that a thread holds in registers, for rows aligned to 16 or 32 bytes: whole sectors go out
// with each 256-bit store, and nothing passes through shared memory.

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <bool F32> __device__ __forceinline__ void store_row(void *out, int64_t at, const float (&v)[32], int vec)
{
    constexpr int kWords = F32 ? 32 : 16;
    uint32_t w[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = F32 ? __float_as_uint(v[i]) : pack_bf16(v[2 * i % 32], v[(2 * i + 1) % 32]);
    uint32_t *o = reinterpret_cast<uint32_t *>(static_cast<char *>(out) + at * (F32 ? 4 : 2));
    if (vec == 32) {
#pragma unroll
        for (int i = 0; i < kWords; i += 8)
            asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(o + i), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]),
                         "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7]) : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < kWords; i += 4) *reinterpret_cast<uint4 *>(o + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    }
}

template <bool F32> __device__ __forceinline__ void add_row(const void *in, int64_t at, float (&v)[32])
{
    constexpr int kWords = F32 ? 32 : 16;
    const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const char *>(in) + at * (F32 ? 4 : 2));
    uint4 w[kWords / 4];
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) w[i] = p[i];
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) {
        const uint32_t q[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (F32) {
                v[i * 4 + j] += __uint_as_float(q[j]);
            } else {
                v[(i * 8 + 2 * j) % 32] += __uint_as_float(q[j] << 16);
                v[(i * 8 + 2 * j + 1) % 32] += __uint_as_float(q[j] & 0xffff0000u);
            }
        }
    }
}

template <int ACT> __device__ __forceinline__ void activate_row(float (&v)[32])
{
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = activate(v[j], ACT);
}
__device__ __forceinline__ void activate_row(float (&v)[32], int act)
{
    if (act == SSD_ACT_RELU) activate_row<SSD_ACT_RELU>(v);
    else if (act == SSD_ACT_GELU) activate_row<SSD_ACT_GELU>(v);
    else if (act == SSD_ACT_SILU) activate_row<SSD_ACT_SILU>(v);
}

// By a whole warp, lane l with row m of its own (`in`: whether there is one); columns n .. n + 31 exist.
__device__ __forceinline__ void add_bias_row(const float *bias, int n, float (&v)[32])
{
    if (!bias) return;
    const float b = bias[n + (threadIdx.x & 31)];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(0xffffffffu, b, j);
}

template <bool GATED, bool F32> __device__ __forceinline__ void finish_row(const Epilogue &e, int group, bool in, int64_t m, int n, float (&v)[32], float (&u)[32])
{
    add_bias_row(e.bias[0], n, v);
    if (e.z[0] && in) store_row<F32>(e.z[0], m * e.ldz[0] + n, v, e.vec);
    activate_row(v, e.act);
    if (GATED) {
        add_bias_row(e.bias[1], n, u);
        if (e.z[1] && in) store_row<F32>(e.z[1], m * e.ldz[1] + n, u, e.vec);
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] *= u[j];
    }
    if (!in) return;
    if (e.residual) add_row<F32>(e.residual, m * e.ldr + n, v);
    store_row<F32>(e.out[group], m * e.ldo[group] + n, v, e.vec);
}

// Four columns of ROWS rows, `step` apart, from n on (columns 4 lanes apart each where CONTIGUOUS is false, so that neighbouring lanes store
// neighbouring elements of rows that no vector fits).  rows: those that exist; cols: columns of the result.
template <bool F32> __device__ __forceinline__ void store_four(void *out, int64_t at, const float (&v)[4])
{
    if (F32) *reinterpret_cast<float4 *>(static_cast<float *>(out) + at) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(out) + at) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
}

template <bool GATED, bool F32, int ROWS, int APART>
__device__ __forceinline__ void finish_fours(const Epilogue &e, int group, int64_t m, int step, int rows, int n, int cols, float (&v)[ROWS][4], float (&u)[ROWS][4])
{
    float r[ROWS][4];
#pragma unroll
    for (int q = 0; q < ROWS; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) r[q][j] = q < rows && n + j * APART < cols ? residual_at(e, m + q * step, n + j * APART) : 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool in = n + j * APART < cols;
        const float b0 = e.bias[0] && in ? e.bias[0][n + j * APART] : 0.0f, b1 = GATED && e.bias[1] && in ? e.bias[1][n + j * APART] : 0.0f;
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
            v[q][j] += b0;
            if (GATED) u[q][j] += b1;
        }
    }
    const bool vector = APART == 1 && e.vec && n + 4 <= cols;
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
        if (q >= rows) break;
        const int64_t row = m + q * step;
        if (!vector) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (n + j * APART < cols) finish<GATED>(e, group, row, n + j * APART, v[q][j], u[q][j], r[q][j]);
            continue;
        }
        if (e.z[0]) store_four<F32>(e.z[0], row * e.ldz[0] + n, v[q]);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[q][j] = activate(v[q][j], e.act);
        if (GATED) {
            if (e.z[1]) store_four<F32>(e.z[1], row * e.ldz[1] + n, u[q]);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[q][j] *= u[q][j];
        }
        if (e.residual) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[q][j] += r[q][j];
        }
        store_four<F32>(e.out[group], row * e.ldo[group] + n, v[q]);
    }
}

// Two values as three bfloat16 parts each, packed: 8 bits a part, nothing of a float32 is left over (except below bfloat16's smallest
// step).  A value that would round up to infinity is cut instead; an infinity or NaN has no further parts.  Only the first part can
// meet those: what it leaves is at most 2^-8 of the value.
__device__ __forceinline__ void split_parts(float x, float y, uint32_t (&h)[3])
{
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(h[0]) : "f"(y), "f"(x));
    float rx = x - __uint_as_float(h[0] << 16), ry = y - __uint_as_float(h[0] & 0xffff0000u);
    if (!(fabsf(rx) + fabsf(ry) < INFINITY)) {
        uint32_t hx = h[0] & 0xffffu, hy = h[0] >> 16;
        if (!(fabsf(rx) < INFINITY)) {
            if (fabsf(x) < INFINITY) hx = __float_as_uint(x) >> 16;
            rx = fabsf(x) < INFINITY ? x - __uint_as_float(hx << 16) : 0.0f;
        }
        if (!(fabsf(ry) < INFINITY)) {
            if (fabsf(y) < INFINITY) hy = __float_as_uint(y) >> 16;
            ry = fabsf(y) < INFINITY ? y - __uint_as_float(hy << 16) : 0.0f;
        }
        h[0] = hx | (hy << 16);
    }
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(h[1]) : "f"(ry), "f"(rx));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(h[2]) : "f"(ry - __uint_as_float(h[1] & 0xffff0000u)), "f"(rx - __uint_as_float(h[1] << 16)));
}

}  // namespace ssd_layers
