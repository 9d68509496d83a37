// Gradient norms over groups of tensors, and clipping (contract: include/ssd_layers.h).
//
//   norm_G = sqrt(sum g^2),  c_G = min(1, max_norm / (norm_G + 1e-6)),  out = c_G * g
//
// Two sweeps over the gradients, because every output needs the whole sum: what bounds both is HBM
// (read + read + write; the second read comes out of the 126 MB L2 as far as it fits).  The tensors are
// cut into chunks of one thread block each, listed in a device table, so that 1 tensor of 10^9 elements and
// 6000 small ones make the same kind of launch.
// Measured: 8 arenas of 25.6 M float32 into bfloat16 313 us (reading twice and writing once at the copy rate is 312); 16 of 138 M
// bfloat16 2.07 ms (2.03); 4 of 0.27 M 7.1 us, two launches whose start overlaps, in place with nothing to scale 6.0, the norms alone 4.2.
#include "ssd_layers.h"
#include "ssd_layers_common.cuh"

#include <cuda_bf16.h>

#include <cmath>
#include <cstring>
#include <iterator>
#include <memory>
#include <new>
#include <utility>
#include <vector>

namespace {

using namespace ssd_layers;

// One thread block's share of a tensor.
struct __align__(16) Chunk {
    uint64_t src, dst;
    int32_t count, group;
    int32_t pad[2];
};

// Chunks are cut so that a long list makes about kChunkTarget of them (32 per SM) and none is shorter than
// kChunkMin elements, unless its tensor is.
constexpr int64_t kChunkTarget = 148 * 32;
constexpr int64_t kChunkMin = 4096;
constexpr int kThreads = 256;

int64_t chunk_elems(int64_t total)
{
    const int64_t c = ((total + kChunkTarget - 1) / kChunkTarget + kChunkMin - 1) / kChunkMin * kChunkMin;
    return c < kChunkMin ? kChunkMin : (c > (int64_t(1) << 30) ? (int64_t(1) << 30) : c);
}

// The table: chunks, one partial sum each, then for every group its chunk count, arrivals and factor.
struct TableLayout {
    int64_t chunks, partial, group_first, arrived, factor, bytes;
};

TableLayout table_layout(int64_t chunks, int32_t groups)
{
    auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
    TableLayout t{};
    t.chunks = 0;
    t.partial = up(chunks * int64_t(sizeof(Chunk)));
    t.group_first = t.partial + up(chunks * 8);
    t.arrived = t.group_first + up((int64_t(groups) + 1) * 4);
    t.factor = t.arrived + up(int64_t(groups) * 4);
    t.bytes = t.factor + up(int64_t(groups) * 4);
    return t;
}

ssd_status count_chunks(int32_t T, const int64_t *numel, int32_t groups, int64_t *elems, int64_t *chunks)
{
    if (!numel || T < 1 || groups < 1) return SSD_ERR_ARG;
    int64_t total = 0;
    for (int32_t t = 0; t < T; ++t) {
        if (numel[t] < 0 || numel[t] >= (int64_t(1) << 40)) return SSD_ERR_LAYOUT;
        total += numel[t];
        if (total >= (int64_t(1) << 42)) return SSD_ERR_LAYOUT;
    }
    const int64_t c = chunk_elems(total);
    int64_t n = 0;
    for (int32_t t = 0; t < T; ++t) n += (numel[t] + c - 1) / c;
    *elems = c;
    *chunks = n;
    return SSD_OK;
}

struct ClipParams {
    const Chunk *chunks;
    double *partial;
    const int32_t *group_first;   // chunks of group g: [group_first[g], group_first[g + 1])
    int32_t *arrived;
    float *factor;
    float *norms;
    float max_norm;
    int32_t zero_nonfinite;
    int32_t num_chunks;
    int32_t captured;             // the table's copy is part of a graph, as this kernel is
};

// A block's share.  The table is in place before the list is handed out, so it is read while the kernel before this one still runs; gradients and
// whatever else kernels write are read after wait_for_previous only, which is what makes their stores visible.
__device__ __forceinline__ Chunk chunk_at(const ClipParams &p, unsigned i)
{
    if (p.captured) wait_for_previous();
    return p.chunks[i];
}

template <typename T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen<uint16_t>(uint16_t v) { return __uint_as_float(uint32_t(v) << 16); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t narrow<uint16_t>(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

template <typename T, int V> struct __align__(sizeof(T) * V) Pack { T v[V]; };

__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double part[kThreads / 32];
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    for (int i = 0; i < kThreads / 32; ++i) s += part[i];
    __syncthreads();
    return s;
}

// Sum of squares of every chunk; the block that arrives last in a group adds the group's partial sums in
// their order (so the result does not depend on which block that is), writes the norm and the factor and
// puts the counter back to zero for the next call.
template <typename T> __global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ ClipParams p)
{
    constexpr int V = 16 / sizeof(T);
    const Chunk c = chunk_at(p, blockIdx.x);
    wait_for_previous();
    dependents_may_start();                     // not before: scale_kernel's blocks, come up this early, would only be in the way (4 x ResNet-20: 8.9 us for 7.1)
    const T *g = reinterpret_cast<const T *>(c.src);
    // elements before the first 16-byte boundary, whole vectors, rest
    int head = int(((16 - (c.src & 15)) & 15) / sizeof(T));
    if (head > c.count) head = c.count;
    const int nvec = (c.count - head) / V;
    const Pack<T, V> *gv = reinterpret_cast<const Pack<T, V> *>(g + head);
    double s0 = 0.0, s1 = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < nvec; i += kThreads) {
        const Pack<T, V> x = gv[i];
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const double a = widen<T>(x.v[j]), b = widen<T>(x.v[j + 1]);
            s0 = fma(a, a, s0);
            s1 = fma(b, b, s1);
        }
    }
    const int tail = head + nvec * V;
    if (int(threadIdx.x) < head) { const double a = widen<T>(g[threadIdx.x]); s0 = fma(a, a, s0); }
    if (tail + int(threadIdx.x) < c.count) { const double a = widen<T>(g[tail + threadIdx.x]); s1 = fma(a, a, s1); }
    const double sum = block_sum(s0 + s1);

    __shared__ int last;
    const int first = p.group_first[c.group], count = p.group_first[c.group + 1] - first;
    if (threadIdx.x == 0) {
        p.partial[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(&p.arrived[c.group], 1) == count - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += kThreads) s += __ldcg(&p.partial[first + i]);
    s = block_sum(s);
    if (threadIdx.x == 0) {
        const double norm = sqrt(s);
        p.norms[c.group] = float(norm);
        float f = 1.0f;
        if (!(float(norm) <= 3.402823466e38f)) f = p.zero_nonfinite ? 0.0f : 1.0f;
        else if (double(p.max_norm) < norm + 1e-6) f = float(double(p.max_norm) / (norm + 1e-6));
        p.factor[c.group] = f;
        p.arrived[c.group] = 0;
    }
}

// Groups without elements have no block in norm_kernel.
__global__ void empty_groups_kernel(const __grid_constant__ ClipParams p, int groups)
{
    dependents_may_start();
    wait_for_previous();
    const int g = blockIdx.x * blockDim.x + threadIdx.x;
    if (g < groups && p.group_first[g] == p.group_first[g + 1]) p.norms[g] = 0.0f;
}

// out = factor * g, the chunks from the last one on: their gradients are the ones that L2 still holds.
template <typename S, typename D> __global__ void __launch_bounds__(kThreads) scale_kernel(const __grid_constant__ ClipParams p)
{
    constexpr int V = 16 / (sizeof(S) > sizeof(D) ? sizeof(S) : sizeof(D));
    dependents_may_start();
    const Chunk c = chunk_at(p, p.num_chunks - 1 - blockIdx.x);
    const S *g = reinterpret_cast<const S *>(c.src);
    D *o = reinterpret_cast<D *>(c.dst);
    // vectors where source and destination reach a vector boundary at the same element
    const int hs = int(((sizeof(S) * V - (c.src & (sizeof(S) * V - 1))) & (sizeof(S) * V - 1)) / sizeof(S));
    const int hd = int(((sizeof(D) * V - (c.dst & (sizeof(D) * V - 1))) & (sizeof(D) * V - 1)) / sizeof(D));
    int head = hs, nvec = 0;
    if (hs == hd && hs < c.count) nvec = (c.count - hs) / V;
    else head = 0;
    const Pack<S, V> *gv = reinterpret_cast<const Pack<S, V> *>(g + head);
    Pack<D, V> *ov = reinterpret_cast<Pack<D, V> *>(o + head);
    constexpr int kAtOnce = 4;
    Pack<S, V> x[kAtOnce];
    auto fetch = [&](int i) {
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q)
            if (i + q * kThreads < nvec) x[q] = gv[i + q * kThreads];
    };
    wait_for_previous();
    fetch(threadIdx.x);                         // on their way together with the factor
    const float f = __ldcg(&p.factor[c.group]);
    if (f == 1.0f && c.src == c.dst) return;
    const bool zero = f == 0.0f && p.zero_nonfinite;      // nothing of an infinity or NaN may stay
    auto scaled = [&](S v) { return narrow<D>(zero ? 0.0f : __fmul_rn(f, widen<S>(v))); };
    for (int i = threadIdx.x; i < nvec; i += kAtOnce * kThreads) {
        if (i != int(threadIdx.x)) fetch(i);
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            if (i + q * kThreads >= nvec) break;
            Pack<D, V> y;
#pragma unroll
            for (int j = 0; j < V; ++j) y.v[j] = scaled(x[q].v[j]);
            ov[i + q * kThreads] = y;
        }
    }
    if (int(threadIdx.x) < head) o[threadIdx.x] = scaled(g[threadIdx.x]);
    for (int i = head + nvec * V + threadIdx.x; i < c.count; i += kThreads) o[i] = scaled(g[i]);
}

}  // namespace

struct ssd_grad_list {
    int32_t groups = 0;
    int32_t chunks = 0;
    int32_t src_dtype = 0, dst_dtype = 0;
    bool has_empty_group = false;
    bool writes = false;              // some destination is not its source
    bool captured = false;            // created while its stream was captured
    TableLayout at{};
    unsigned char *table = nullptr;   // the caller's device memory
    std::vector<unsigned char> image;
    std::vector<std::pair<uintptr_t, uintptr_t>> taken;      // address ranges of gradients, destinations and table: ascending, apart from each other
};

extern "C" {

ssd_status ssd_grad_list_bytes(int32_t T, const int64_t *numel, int32_t groups, int64_t *bytes)
{
    if (!bytes) return SSD_ERR_ARG;
    int64_t elems = 0, chunks = 0;
    const ssd_status st = count_chunks(T, numel, groups, &elems, &chunks);
    if (st != SSD_OK) return st;
    *bytes = table_layout(chunks, groups).bytes;
    return SSD_OK;
}

ssd_status ssd_grad_list_create(ssd_grad_list **out, int32_t T, const int64_t *numel, const int32_t *group, int32_t groups,
                                const void *const *src, int32_t src_dtype, void *const *dst, int32_t dst_dtype,
                                void *device_table, int64_t table_bytes, void *cuda_stream)
try {
    if (!out) return SSD_ERR_ARG;
    *out = nullptr;
    if (!src || !dst || !device_table || !valid_dtype(src_dtype) || !valid_dtype(dst_dtype)) return SSD_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(device_table) & 15) return SSD_ERR_ALIGN;
    int64_t elems = 0, nchunks = 0;
    ssd_status st = count_chunks(T, numel, groups, &elems, &nchunks);
    if (st != SSD_OK) return st;
    if (nchunks > (int64_t(1) << 30)) return SSD_ERR_LAYOUT;
    const TableLayout at = table_layout(nchunks, groups);
    if (table_bytes < at.bytes) return SSD_ERR_ARG;
    const uint64_t ss = src_dtype == SSD_BF16 ? 2 : 4, ds = dst_dtype == SSD_BF16 ? 2 : 4;

    // address ranges of every tensor, sources and destinations: a destination meets nothing but its own source
    struct Span { uintptr_t lo, hi; int32_t t; bool write; };
    std::vector<Span> spans;
    spans.reserve(size_t(T) * 2 + 1);
    bool writes = false;
    for (int32_t t = 0; t < T; ++t) {
        const int32_t g = group ? group[t] : 0;
        if (g < 0 || g >= groups || (t > 0 && group && g < group[t - 1])) return SSD_ERR_ARG;
        if (numel[t] == 0) continue;
        if (!src[t] || !dst[t]) return SSD_ERR_ARG;
        const uintptr_t s = reinterpret_cast<uintptr_t>(src[t]), d = reinterpret_cast<uintptr_t>(dst[t]);
        if (s % ss || d % ds) return SSD_ERR_ALIGN;
        if (s == d && src_dtype != dst_dtype) return SSD_ERR_ARG;
        if (s != d) {
            writes = true;
            spans.push_back({s, s + uintptr_t(numel[t]) * ss, t, false});
        }
        spans.push_back({d, d + uintptr_t(numel[t]) * ds, t, true});
    }
    const uintptr_t tab = reinterpret_cast<uintptr_t>(device_table);
    spans.push_back({tab, tab + uintptr_t(at.bytes), -1, true});
    std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.lo < b.lo; });
    uintptr_t written = 0, read = 0;                        // ends of the spans seen so far
    for (const Span &s : spans) {
        if (s.lo < written || (s.write && s.lo < read)) return SSD_ERR_ARG;
        if (s.write) written = s.hi > written ? s.hi : written;
        else read = s.hi > read ? s.hi : read;
    }

    std::unique_ptr<ssd_grad_list> owned(new ssd_grad_list);       // until it is handed out
    ssd_grad_list *const l = owned.get();
    l->groups = groups;
    l->chunks = int32_t(nchunks);
    l->src_dtype = src_dtype;
    l->dst_dtype = dst_dtype;
    l->writes = writes;
    l->at = at;
    l->table = static_cast<unsigned char *>(device_table);
    l->image.assign(size_t(at.bytes), 0);
    for (const Span &s : spans) {
        if (l->taken.empty() || s.lo > l->taken.back().second) l->taken.emplace_back(s.lo, s.hi);
        else l->taken.back().second = std::max(l->taken.back().second, s.hi);
    }
    Chunk *c = reinterpret_cast<Chunk *>(l->image.data() + at.chunks);
    int32_t *first = reinterpret_cast<int32_t *>(l->image.data() + at.group_first);
    int32_t n = 0, g_at = 0;
    for (int32_t t = 0; t < T; ++t) {
        const int32_t g = group ? group[t] : 0;
        while (g_at < g) first[++g_at] = n;
        for (int64_t o = 0; o < numel[t]; o += elems) {
            c[n].src = reinterpret_cast<uint64_t>(src[t]) + uint64_t(o) * ss;
            c[n].dst = reinterpret_cast<uint64_t>(dst[t]) + uint64_t(o) * ds;
            c[n].count = int32_t(numel[t] - o < elems ? numel[t] - o : elems);
            c[n].group = g;
            ++n;
        }
    }
    while (g_at < groups) first[++g_at] = n;
    for (int32_t g = 0; g < groups; ++g) l->has_empty_group = l->has_empty_group || first[g] == first[g + 1];
    // The table holds addresses that kernels read and write by, so it is in place before the list is handed out: calls may come on any stream, and
    // their kernels read it before they wait for their predecessors (not where the copy is captured: it then runs with its graph).
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(stream, &capture);
    if (e == cudaSuccess) e = cudaMemcpyAsync(l->table, l->image.data(), l->image.size(), cudaMemcpyHostToDevice, stream);
    l->captured = capture != cudaStreamCaptureStatusNone;
    if (e == cudaSuccess && !l->captured) e = cudaStreamSynchronize(stream);
    if (e != cudaSuccess) return layer_cuda_fail(e);
    *out = owned.release();
    return SSD_OK;
} catch (const std::bad_alloc &) {
    return SSD_ERR_NOMEM;
}

void ssd_grad_list_destroy(ssd_grad_list *list) { delete list; }

static ssd_status clip_call(ssd_grad_list *l, float max_norm, int32_t nonfinite, float *norms, bool scale, void *cuda_stream)
{
    if (!l || !norms || !(max_norm >= 0.0f)) return SSD_ERR_ARG;
    if (nonfinite != SSD_NONFINITE_KEEP && nonfinite != SSD_NONFINITE_ZERO) return SSD_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(norms) & 3) return SSD_ERR_ALIGN;
    // the norms lie over nothing that the call reads or writes: the last range that starts before their end ends before them
    const uintptr_t lo = reinterpret_cast<uintptr_t>(norms), hi = lo + uintptr_t(l->groups) * 4;
    const auto after = std::partition_point(l->taken.begin(), l->taken.end(), [&](const auto &range) { return range.first < hi; });
    if (after != l->taken.begin() && std::prev(after)->second > lo) return SSD_ERR_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    ClipParams p{};
    p.chunks = reinterpret_cast<const Chunk *>(l->table + l->at.chunks);
    p.partial = reinterpret_cast<double *>(l->table + l->at.partial);
    p.group_first = reinterpret_cast<const int32_t *>(l->table + l->at.group_first);
    p.arrived = reinterpret_cast<int32_t *>(l->table + l->at.arrived);
    p.factor = reinterpret_cast<float *>(l->table + l->at.factor);
    p.norms = norms;
    p.max_norm = max_norm;
    p.zero_nonfinite = nonfinite == SSD_NONFINITE_ZERO;
    p.num_chunks = l->chunks;
    p.captured = l->captured;
    cudaError_t e = cudaSuccess;
    auto run = [&](auto kernel, int blocks, auto... args) {
        if (e != cudaSuccess) return;
        e = launch(kernel, dim3(unsigned(blocks)), kThreads, 0, 1, stream, args...);
        count_launches(1);
    };
    if (l->has_empty_group) run(empty_groups_kernel, (l->groups + kThreads - 1) / kThreads, p, l->groups);
    if (l->chunks > 0) {
        const bool s32 = l->src_dtype == SSD_F32, d32 = l->dst_dtype == SSD_F32;
        run(s32 ? norm_kernel<float> : norm_kernel<uint16_t>, l->chunks, p);
        // in place, an infinite limit leaves everything as it is (unless a group is to be zeroed)
        const bool nothing = !l->writes && std::isinf(max_norm) && !p.zero_nonfinite;
        if (scale && !nothing)
            run(s32 ? (d32 ? scale_kernel<float, float> : scale_kernel<float, uint16_t>) : (d32 ? scale_kernel<uint16_t, float> : scale_kernel<uint16_t, uint16_t>),
                l->chunks, p);
    }
    return e == cudaSuccess ? SSD_OK : layer_cuda_fail(e);
}

ssd_status ssd_clip_grad_norm(ssd_grad_list *list, float max_norm, int32_t nonfinite, float *norms, void *cuda_stream)
{
    return clip_call(list, max_norm, nonfinite, norms, true, cuda_stream);
}

ssd_status ssd_grad_norm(ssd_grad_list *list, float *norms, void *cuda_stream)
{
    return clip_call(list, INFINITY, SSD_NONFINITE_KEEP, norms, false, cuda_stream);
}

}  // extern "C"
