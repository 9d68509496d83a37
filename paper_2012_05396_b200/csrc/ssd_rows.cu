// The layers for a few rows: one token, or a handful.
//
// The weights are read once (and their gradients written once), which is all the time such a call should take; a tile of 128
// rows would be nearly empty.  The products are float32 fused multiply-adds on the weights as they come: no passes over operands, and any type, pitch and
// alignment in one launch (two with dx).
//
// Forward: a warp holds the sums of kWarpRows weight rows times all rows of x, its lanes along the contraction; `slices` warps of a block share
// the contraction so that enough loads are under way, and are added up in their order.
// Backward: a block takes a strip of weight rows and kCols columns, four a thread.  dz of the strip is computed first, into shared
// memory; then one sweep down the strip reads W and writes dW, x staying in registers, and adds up the strip's part of dx, which a
// second kernel joins over the strips in their order.
// Measured, 4096 x 4096, weights from HBM: forward of 1 row 8.0 us bfloat16 (33.6 MB: 5.1 at the copy rate) and 13.7 float32 (10.3), of 8 rows 11.7 and 26;
// backward with float32 gradients, 1 row 24 us bfloat16 (15.4), 8 rows 35.
#include "ssd_layers.cuh"

namespace ssd_layers {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kWarpRows = 4;                 // weight rows of a warp (gated: half of the gate's, half of up's)

// Eight consecutive values of a row from column c on, zero beyond the last.
template <typename T, bool VEC> struct Eight {
    uint32_t w[VEC ? 2 * sizeof(T) : 8];

    __device__ __forceinline__ void load(const T *row, int c, int cols, bool in)
    {
        if (VEC) {
#pragma unroll
            for (int i = 0; i < int(2 * sizeof(T)); i += 4) {
                const uint4 t = in && c < cols ? *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint32_t *>(row + c) + i) : make_uint4(0, 0, 0, 0);
                w[i] = t.x;
                w[i + 1] = t.y;
                w[i + 2] = t.z;
                w[i + 3] = t.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = in && c + j < cols ? __float_as_uint(load_as_float<T>(row + c + j)) : 0u;
        }
    }
    __device__ __forceinline__ float operator[](int j) const
    {
        if (VEC && sizeof(T) == 2) return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
        return __uint_as_float(w[j % (VEC ? 2 * sizeof(T) : 8)]);
    }
};

// V sums over the lanes, V a power of two up to 32: afterwards v[0] of lane l is sum number l / (32 / V).
template <int V> __device__ __forceinline__ void reduce_lanes(float (&v)[V])
{
    int c = V;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        if (c > 1) {
            c /= 2;
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                if (i >= c) break;
                const float give = threadIdx.x & o ? v[i] : v[i + c], keep = threadIdx.x & o ? v[i + c] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        }
    }
}

// VEC: x and the weights in rows of aligned groups of eight.
template <typename T, bool VEC, int R, bool GATED> __global__ void __launch_bounds__(kThreads) rows_forward_kernel(const __grid_constant__ RowsForward p)
{
    constexpr int kOuts = GATED ? kWarpRows / 2 : kWarpRows, V = kWarpRows * R;
    __shared__ float sums[kWarps][V];
    dependents_may_start();
    wait_for_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per_block = kWarps / p.slices, slice = warp % p.slices, across = int(blockIdx.x % unsigned(p.across));
    const int n0 = (across * per_block + warp / p.slices) * kOuts;
    const T *wrow[kWarpRows];
    bool in[kWarpRows];
#pragma unroll
    for (int i = 0; i < kWarpRows; ++i) {
        const int mat = GATED ? i / kOuts : 0, n = n0 + i % kOuts;
        in[i] = n < p.out;
        wrow[i] = static_cast<const T *>(p.w[mat]) + int64_t(in[i] ? n : 0) * p.ldw[mat];
    }
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    // R rows of x for every `across` blocks
    const int r0 = int(blockIdx.x / unsigned(p.across)) * R, rows = p.rows - r0 < R ? p.rows - r0 : R;
    const T *x = static_cast<const T *>(p.x) + r0 * p.ldx;
    // two steps of 256 of the contraction under way at a time (one where the registers are wanted for the sums)
    constexpr int kSteps = R <= 4 ? 2 : 1;
    const int stride = 256 * p.slices;
    for (int c = slice * 256 + lane * 8; c - lane * 8 < p.in; c += kSteps * stride) {
        Eight<T, VEC> w[kSteps][kWarpRows];
#pragma unroll
        for (int h = 0; h < kSteps; ++h)
#pragma unroll
            for (int i = 0; i < kWarpRows; ++i) w[h][i].load(wrow[i], c + h * stride, p.in, in[i]);
#pragma unroll
        for (int h = 0; h < kSteps; ++h) {
            if (c - lane * 8 + h * stride >= p.in) break;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                Eight<T, VEC> v;
                v.load(x + r * p.ldx, c + h * stride, p.in, r < rows);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float xf = v[j];
#pragma unroll
                    for (int i = 0; i < kWarpRows; ++i) acc[i * R + r] = fmaf(w[h][i][j], xf, acc[i * R + r]);
                }
            }
        }
    }
    reduce_lanes<V>(acc);
    if (lane % (32 / V) == 0) sums[warp][lane / (32 / V)] = acc[0];
    __syncthreads();
    // one thread for each output of the block
    for (int t = threadIdx.x; t < per_block * kOuts * R; t += kThreads) {
        const int g = t / (kOuts * R), i = t / R % kOuts, r = t % R;
        const int n = (across * per_block + g) * kOuts + i;
        if (n >= p.out || r >= rows) continue;
        float v = 0.0f, u = 0.0f;
        for (int s = 0; s < p.slices; ++s) {
            v += sums[g * p.slices + s][i * R + r];
            if (GATED) u += sums[g * p.slices + s][((kOuts + i) * R + r) % V];
        }
        finish<GATED>(p.e, 0, r0 + r, n, v + (p.e.bias[0] ? p.e.bias[0][n] : 0.0f), GATED && p.e.bias[1] ? u + p.e.bias[1][n] : u, residual_at(p.e, r0 + r, n));
    }
}

// bfloat16 forward on aligned rows, up to 16 rows: the same reading, the products on mma.sync.  What bounds the call is reading the weights, which these small
// matrix instructions leave time for (eight rows of fused multiply-adds do not).
// A warp multiplies 16 weight rows (gated: 8 of each matrix) with 8 or 16 rows of x.  The order of the contraction is free as long as both
// operands agree on it, so a thread loads eight consecutive values of its rows and hands them to two instructions as they are.  A step
// takes 512 bytes of each row, 256 where the contraction is short and more warps have to share it (gated 8 x 2048 x 8192: 14.3 us with 512
// bytes, 17.4 with 256; 8 x 1024 x 1024: 3.6 and 2.8).  For up to eight rows both are compiled to 46 registers, so a step's loads are not all under
// way at once, and a step takes about 4 us from HBM: long contractions are left to the tensor cores (rows_mma_pays).
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NX: eights of rows of x, 1 or 2.  LOADS: 64-byte pieces of a row in a step.
template <int NX, bool GATED, int LOADS> __global__ void __launch_bounds__(kThreads) rows_mma_kernel(const __grid_constant__ RowsForward p)
{
    constexpr int kOuts = GATED ? 8 : 16, kStep = 32 * LOADS;      // columns of the result; contraction of a step
    __shared__ float sums[kWarps][NX * 4][33];
    dependents_may_start();
    wait_for_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int per_block = kWarps / p.slices, slice = warp % p.slices;
    const int n0 = (int(blockIdx.x) * per_block + warp / p.slices) * kOuts;
    const __nv_bfloat16 *wrow[2], *xrow[NX];
    bool win[2], xin[NX];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int n = n0 + g + (GATED ? 0 : 8 * h), mat = GATED ? h : 0;
        win[h] = n < p.out;
        wrow[h] = static_cast<const __nv_bfloat16 *>(p.w[mat]) + int64_t(win[h] ? n : 0) * p.ldw[mat];
    }
#pragma unroll
    for (int x = 0; x < NX; ++x) {
        xin[x] = g + 8 * x < p.rows;
        xrow[x] = static_cast<const __nv_bfloat16 *>(p.x) + int64_t(xin[x] ? g + 8 * x : 0) * p.ldx;
    }
    auto load = [&](const __nv_bfloat16 *row, int c, bool in) { return in && c < p.in ? *reinterpret_cast<const uint4 *>(row + c) : make_uint4(0, 0, 0, 0); };
    float acc[NX][4] = {};
    for (int c = slice * kStep + t * 8; c - t * 8 < p.in; c += kStep * p.slices) {
        uint4 w[2][LOADS];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < LOADS; ++i) w[h][i] = load(wrow[h], c + 32 * i, win[h]);
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                const uint4 b = load(xrow[x], c + 32 * i, xin[x]), lo = w[0][i], hi = w[1][i];
                mma_16x8x16(acc[x], lo.x, hi.x, lo.y, hi.y, b.x, b.y);
                mma_16x8x16(acc[x], lo.z, hi.z, lo.w, hi.w, b.z, b.w);
            }
    }
#pragma unroll
    for (int x = 0; x < NX; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[warp][x * 4 + i][lane] = acc[x][i];
    __syncthreads();
    // accumulator i of lane (g, t): weight row g + 8 (i / 2), row of x 2 t + i % 2; a thread an output, neighbours along the weight rows
    for (int o = threadIdx.x; o < per_block * kOuts * 8 * NX; o += kThreads) {
        const int f = o % kOuts, group = o / kOuts % per_block, r = o / (kOuts * per_block);
        const int n = (int(blockIdx.x) * per_block + group) * kOuts + f;
        if (n >= p.out || r >= p.rows) continue;
        const int from = (f & 7) * 4 + (r & 7) / 2, i = (r >> 3) * 4 + f / 8 * 2 + (r & 1);
        float v = 0.0f, u = 0.0f;
        for (int q = 0; q < p.slices; ++q) {
            v += sums[group * p.slices + q][i][from];
            if (GATED) u += sums[group * p.slices + q][i + 2][from];
        }
        finish<GATED>(p.e, 0, r, n, v + (p.e.bias[0] ? p.e.bias[0][n] : 0.0f), GATED && p.e.bias[1] ? u + p.e.bias[1][n] : u, residual_at(p.e, r, n));
    }
}

constexpr int kCols = 4 * kThreads;          // columns of a block in the backward pass
constexpr int kStripMax = 64;                // weight rows of a strip

// Four consecutive values of a row from column c on, zero beyond the last or where there is no row.
template <typename T, bool VEC> struct Four {
    static constexpr int kWords = VEC ? int(sizeof(T)) : 4;
    uint32_t w[kWords];

    __device__ __forceinline__ void load(const T *row, int c, int cols, bool in)
    {
        if (VEC) {          // cols is a multiple of four
            in = in && c < cols;
            if (sizeof(T) == 4) {
                const uint4 t = in ? *reinterpret_cast<const uint4 *>(row + c) : make_uint4(0, 0, 0, 0);
                w[0] = t.x; w[1] = t.y; w[2 % kWords] = t.z; w[3 % kWords] = t.w;
            } else {
                const uint2 t = in ? *reinterpret_cast<const uint2 *>(row + c) : make_uint2(0, 0);
                w[0] = t.x; w[1] = t.y;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j % kWords] = in && c + j < cols ? __float_as_uint(load_as_float<T>(row + c + j)) : 0u;
        }
    }
    __device__ __forceinline__ float operator[](int j) const
    {
        if (VEC && sizeof(T) == 2) return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
        return __uint_as_float(w[j % kWords]);
    }
};

// VEC: x, weights and weight gradients in rows of aligned groups of four.
template <typename T, bool VEC, int R> __global__ void __launch_bounds__(kThreads, R <= 4 ? 3 : (R == 8 ? 2 : 1)) rows_backward_kernel(const __grid_constant__ RowsBackward p)
{
    __shared__ __align__(16) float dz[2][kStripMax][R];
    dependents_may_start();
    wait_for_previous();
    const int strips = (p.out + p.strip - 1) / p.strip;
    const int strip = int(blockIdx.x) % strips, c = int(blockIdx.x) / strips * kCols + int(threadIdx.x) * 4;
    const int n0 = strip * p.strip, count = p.out - n0 < p.strip ? p.out - n0 : p.strip;
    for (int t = threadIdx.x; t < count * R; t += kThreads) {
        const int i = t % count, r = t / count;
        float v = 0.0f, u = 0.0f;
        if (r < p.rows) {
            const float g = load_as_float<T>(static_cast<const T *>(p.dy) + r * p.lddy + n0 + i);
            if (p.mats == 2) {
                float value, slope;
                activate_both(load_as_float<T>(static_cast<const T *>(p.z[0]) + r * p.ldz[0] + n0 + i), p.act, &value, &slope);
                v = __fmul_rn(__fmul_rn(g, load_as_float<T>(static_cast<const T *>(p.z[1]) + r * p.ldz[1] + n0 + i)), slope);
                u = __fmul_rn(g, value);
            } else if (p.act != SSD_ACT_NONE) {
                float value, slope;
                activate_both(load_as_float<T>(static_cast<const T *>(p.z[0]) + r * p.ldz[0] + n0 + i), p.act, &value, &slope);
                v = __fmul_rn(g, slope);
            } else {
                v = g;
            }
        }
        dz[0][i][r] = v;
        dz[1][i][r] = u;
    }
    __syncthreads();
    if (int(blockIdx.x) < strips)      // the first columns' blocks add up the bias gradients
        for (int t = threadIdx.x; t < count * p.mats; t += kThreads) {
            const int i = t % count, mat = t / count;
            float s = 0.0f;
            for (int r = 0; r < R; ++r) s += dz[mat][i][r];
            if (p.db[mat]) store_at(p.db[mat], n0 + i, p.grad_f32, s);
        }
    if (c >= p.in || (!p.partial && !p.dw[0])) return;
    float x[R][4], dx[R][4];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        Four<T, VEC> v;
        v.load(static_cast<const T *>(p.x) + r * p.ldx, c, p.in, p.dw[0] && r < p.rows);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[r][j] = v[j];
            dx[r][j] = 0.0f;
        }
    }
    const bool whole = c + 4 <= p.in;
    for (int mat = 0; mat < p.mats; ++mat) {
        const T *w = static_cast<const T *>(p.w[mat]) + int64_t(n0) * p.ldw[mat];
        const int64_t ldw = p.ldw[mat], lddw = p.lddw[mat];
        void *const dw = p.dw[mat];
        constexpr int kAtOnce = R <= 4 ? 8 : 4;
        Four<T, VEC> next[kAtOnce];           // the next rows of W are on their way while these are used
        auto fetch = [&](int i) {
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) next[q].load(w + (i + q) * ldw, c, p.in, p.partial && i + q < count);
        };
        fetch(0);
        for (int i = 0; i < count; i += kAtOnce) {
            Four<T, VEC> now[kAtOnce];
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) now[q] = next[q];
            fetch(i + kAtOnce);
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                if (i + q >= count) break;
                float g[4] = {0.0f, 0.0f, 0.0f, 0.0f}, d[R];
#pragma unroll
                for (int r = 0; r < R; ++r) d[r] = dz[mat][i + q][r];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float wf = now[q][j];
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        dx[r][j] = fmaf(d[r], wf, dx[r][j]);
                        g[j] = fmaf(d[r], x[r][j], g[j]);
                    }
                }
                if (dw) {
                    const int64_t at = int64_t(n0 + i + q) * lddw + c;
                    if (VEC && whole) {
                        if (p.grad_f32) store_four<true>(dw, at, g);
                        else store_four<false>(dw, at, g);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (c + j < p.in) store_at(dw, at + j, p.grad_f32, g[j]);
                    }
                }
            }
        }
    }
    if (p.partial) {
        const int pitch = (p.in + 3) / 4 * 4;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < p.rows) *reinterpret_cast<float4 *>(p.partial + (int64_t(strip) * p.rows + r) * pitch + c) = make_float4(dx[r][0], dx[r][1], dx[r][2], dx[r][3]);
    }
}

// dx from the strips' parts: eight warps take every eighth strip each, and are added up in their order.
__global__ void __launch_bounds__(kThreads) rows_join_kernel(const float *partial, int strips, int rows, int cols, void *dx, int64_t lddx, int f32)
{
    __shared__ float4 part[kWarps][32];
    dependents_may_start();
    wait_for_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pitch = (cols + 3) / 4 * 4;
    const int c = (int(blockIdx.x) * 32 + lane) * 4, r = blockIdx.y;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c < cols) {
#pragma unroll 4
        for (int i = warp; i < strips; i += kWarps) {
            const float4 v = *reinterpret_cast<const float4 *>(partial + (int64_t(i) * rows + r) * pitch + c);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp || c >= cols) return;
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
        const float4 v = part[w][lane];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const float v[4] = {s.x, s.y, s.z, s.w};
    for (int j = 0; j < 4; ++j)
        if (c + j < cols) store_at(dx, r * lddx + c + j, f32, v[j]);
}

bool aligned(const void *p, int64_t ld, int rows, int size, int to) { return reinterpret_cast<uintptr_t>(p) % to == 0 && (rows == 1 || ld * size % to == 0); }

// Whether x and the weights have rows of aligned groups of eight.
bool eights(const RowsForward &p)
{
    const int size = p.e.f32 ? 4 : 2;
    bool vec = p.in % 8 == 0 && aligned(p.x, p.ldx, p.rows, size, 16);
    for (int i = 0; i < (p.gated ? 2 : 1); ++i) vec = vec && aligned(p.w[i], p.ldw[i], p.out, size, 16);
    return vec;
}

// How a call is cut into blocks.  The contraction is shared by as many warps as still fit the chip in one go: too few leave its memory idle, and what
// does not fit runs after the rest.
// `rows`: rows of x of a block; `group`: weight rows of a warp, over both matrices; `step`: contraction that a warp takes at a time; `resident`:
// blocks that fit the chip.
struct RowsCut {
    int slices;
    int64_t times, across;      // blocks over the rows of x, and over the weight rows
};

RowsCut cut_rows(const RowsForward &p, int rows, int group, int step, int resident)
{
    const int64_t groups = (int64_t(p.out) * (p.gated ? 2 : 1) + group - 1) / group;
    const int64_t times = (int64_t(p.rows) + rows - 1) / rows;
    auto across = [=](int slices) { return (groups * slices + kWarps - 1) / kWarps; };
    int slices = 1;
    while (slices < kWarps && across(2 * slices) * times <= resident && p.in > step * slices) slices *= 2;
    return RowsCut{slices, times, across(slices)};
}

// rows_mma_kernel: weight rows of a warp, blocks that fit the chip (up to eight rows of x: 46 registers a thread), contraction of a step.
constexpr int kMmaGroup = 16, kMmaResident = 5 * 148;
int mma_step(const RowsForward &p) { return p.in > 1024 ? 256 : 128; }

// The kernel is a template argument, not a function argument: all of them have one type, and each has to be asked for its own occupancy, so that
// the split, and with it the order of the sums, follows from the call alone.  (It is the same on every device that this code runs on.)
template <void (*KERNEL)(RowsForward)> cudaError_t launch_slices(RowsForward p, int rows, int group, int step, cudaStream_t stream)
{
    static std::atomic<int> known{0};
    int resident = known;
    if (!resident) {
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, KERNEL, kThreads, 0);
        if (e != cudaSuccess) return e;
        known = resident *= 148;
    }
    const RowsCut cut = cut_rows(p, rows, group, step, resident);
    if (cut.across * cut.times > INT32_MAX) return cudaErrorInvalidConfiguration;
    p.slices = cut.slices;
    p.across = int(cut.across);
    return launch(KERNEL, dim3(unsigned(cut.across * cut.times)), kThreads, 0, 1, stream, p);      // in one dimension: the others end at 65535 blocks
}

template <typename T, bool VEC, int R> cudaError_t launch_forward(const RowsForward &p, cudaStream_t stream)
{
    if (p.gated) return launch_slices<rows_forward_kernel<T, VEC, R, true>>(p, R, kWarpRows, 256, stream);
    return launch_slices<rows_forward_kernel<T, VEC, R, false>>(p, R, kWarpRows, 256, stream);
}

template <int LOADS> cudaError_t launch_mma(const RowsForward &p, cudaStream_t stream)
{
    if (p.rows <= 8) return p.gated ? launch_slices<rows_mma_kernel<1, true, LOADS>>(p, 16, kMmaGroup, 32 * LOADS, stream) : launch_slices<rows_mma_kernel<1, false, LOADS>>(p, 16, kMmaGroup, 32 * LOADS, stream);
    return p.gated ? launch_slices<rows_mma_kernel<2, true, LOADS>>(p, 16, kMmaGroup, 32 * LOADS, stream) : launch_slices<rows_mma_kernel<2, false, LOADS>>(p, 16, kMmaGroup, 32 * LOADS, stream);
}

template <typename T, bool VEC> cudaError_t launch_forward_rows(const RowsForward &p, cudaStream_t stream)
{
    if (p.rows == 1) return launch_forward<T, VEC, 1>(p, stream);
    if (p.rows == 2) return launch_forward<T, VEC, 2>(p, stream);
    if (p.rows <= 4) return launch_forward<T, VEC, 4>(p, stream);
    return launch_forward<T, VEC, 8>(p, stream);
}

template <typename T, bool VEC> cudaError_t launch_backward_rows(const RowsBackward &p, int blocks, cudaStream_t stream)
{
    if (p.rows == 1) return launch(rows_backward_kernel<T, VEC, 1>, dim3(unsigned(blocks)), kThreads, 0, 1, stream, p);
    if (p.rows == 2) return launch(rows_backward_kernel<T, VEC, 2>, dim3(unsigned(blocks)), kThreads, 0, 1, stream, p);
    if (p.rows <= 4) return launch(rows_backward_kernel<T, VEC, 4>, dim3(unsigned(blocks)), kThreads, 0, 1, stream, p);
    if (p.rows <= 8) return launch(rows_backward_kernel<T, VEC, 8>, dim3(unsigned(blocks)), kThreads, 0, 1, stream, p);
    return launch(rows_backward_kernel<T, VEC, 16>, dim3(unsigned(blocks)), kThreads, 0, 1, stream, p);
}

}  // namespace

cudaError_t launch_rows_forward(RowsForward p, cudaStream_t stream)
{
    const bool vec = eights(p);
    if (!p.e.f32 && vec && p.rows > 1) {
        count_launches(1);
        return mma_step(p) == 256 ? launch_mma<8>(p, stream) : launch_mma<4>(p, stream);
    }
    count_launches(1);
    if (p.e.f32) return vec ? launch_forward_rows<float, true>(p, stream) : launch_forward_rows<float, false>(p, stream);
    return vec ? launch_forward<__nv_bfloat16, true, 1>(p, stream) : launch_forward_rows<__nv_bfloat16, false>(p, stream);
}

// An SM has arithmetic for one block of eight rows of x at a time (its registers hold two), so what counts is how often the chip is filled with those and how
// many steps of 256 a warp takes each time; rows without vectors load value by value, for as many lanes as there are columns.  Within a third of the measured times of 300
// calls of 17 to 157 000 rows, widths 1 to 2048 and up to 3e7 weights, counted once for every eight rows.
double rows_forward_f32_us(const RowsForward &p)
{
    const RowsCut cut = cut_rows(p, 8, kWarpRows, 256, 148);
    const double fills = double((cut.across * cut.times + 147) / 148), steps = double((int64_t(p.in) + 256 * cut.slices - 1) / (256 * cut.slices));
    return 2.2 + fills * (0.45 + steps * (eights(p) ? 0.8 : 1.0 + 2.2 * std::min(1.0, p.in / 256.0)));
}

// A step of rows_mma_kernel does not hide the way to memory, so few may follow each other: three at most, or any number of them where up to eight
// rows of x fill two thirds of the chip with blocks.
bool rows_mma_pays(const RowsForward &p)
{
    const RowsCut cut = cut_rows(p, 16, kMmaGroup, mma_step(p), kMmaResident);
    const int64_t taken = int64_t(mma_step(p)) * cut.slices;
    return (p.in + taken - 1) / taken <= 3 || (p.rows <= 8 && cut.across >= kMmaResident * 2 / 3);
}

// Weight rows of a strip: about three blocks for every SM, so that the parts of dx stay few.
int rows_strip(int out, int in)
{
    const int64_t across = (int64_t(in) + kCols - 1) / kCols;
    int64_t strips = 3 * 148 / across;
    if (strips < 1) strips = 1;
    int64_t strip = (out + strips - 1) / strips;
    if (strip < 4) strip = 4;
    return int(strip > kStripMax ? kStripMax : strip);
}

int64_t rows_partial_floats(int rows, int out, int in)
{
    const int64_t strip = rows_strip(out, in);
    return (out + strip - 1) / strip * rows * ((in + 3) / 4 * 4);
}

cudaError_t launch_rows_backward(RowsBackward p, cudaStream_t stream)
{
    const int size = p.f32 ? 4 : 2, grad = p.grad_f32 ? 4 : 2;
    bool vec = p.in % 4 == 0 && (!p.dw[0] || aligned(p.x, p.ldx, p.rows, size, 4 * size));
    for (int i = 0; i < p.mats; ++i) {
        if (p.partial) vec = vec && aligned(p.w[i], p.ldw[i], p.out, size, 4 * size);
        if (p.dw[i]) vec = vec && aligned(p.dw[i], p.lddw[i], p.out, grad, 4 * grad);
    }
    p.strip = rows_strip(p.out, p.in);
    const int64_t strips = (int64_t(p.out) + p.strip - 1) / p.strip, across = p.partial || p.dw[0] ? (int64_t(p.in) + kCols - 1) / kCols : 1;
    if (strips * across > INT32_MAX) return cudaErrorInvalidConfiguration;
    const int blocks = int(strips * across);
    cudaError_t e;
    if (p.f32) e = vec ? launch_backward_rows<float, true>(p, blocks, stream) : launch_backward_rows<float, false>(p, blocks, stream);
    else e = vec ? launch_backward_rows<__nv_bfloat16, true>(p, blocks, stream) : launch_backward_rows<__nv_bfloat16, false>(p, blocks, stream);
    count_launches(1);
    if (e != cudaSuccess || !p.partial) return e;
    count_launches(1);
    return launch(rows_join_kernel, dim3(unsigned((int64_t(p.in) + 127) / 128), unsigned(p.rows)), kThreads, 0, 1, stream, static_cast<const float *>(p.partial), int(strips),
                  p.rows, p.in, p.dx, p.lddx, p.f32);
}

}  // namespace ssd_layers
