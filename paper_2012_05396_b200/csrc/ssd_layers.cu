// Host side of the layer operators: argument checks, workspace, and the launches of a call.
// The contract of every entry point is stated in include/ssd_layers.h.
#include "ssd_layers.cuh"
#include "ssd_prep.cuh"

#include <string>

namespace ssd_layers {

namespace {
thread_local std::string g_cuda_error;
std::atomic<int64_t> g_launches{0};
}  // namespace

ssd_status layer_cuda_fail(cudaError_t e)
{
    try {
        g_cuda_error = cudaGetErrorString(e);
    } catch (...) {
    }
    return SSD_ERR_CUDA;
}

void count_launches(int n) { g_launches += n; }

}  // namespace ssd_layers

namespace {

using namespace ssd_layers;

constexpr int64_t kMaxDim = (int64_t(1) << 31) - (int64_t(1) << 16);

// ---------------------------------------------------------------------------------------------------------
// Arguments.  Both layers are brought into one form: `mats` weight matrices (1 linear, 2 gated).

struct Matrix {
    void *p;
    int64_t ld, rows, cols;
    int esize;
    bool write;
};

uintptr_t addr(const void *p) { return reinterpret_cast<uintptr_t>(p); }
uintptr_t end_of(const Matrix &m) { return addr(m.p) + uintptr_t(((m.rows - 1) * m.ld + m.cols) * m.esize); }

bool overlap(const Matrix &a, const Matrix &b)
{
    if (!a.p || !b.p || a.rows == 0 || b.rows == 0) return false;
    if (end_of(a) <= addr(b.p) || end_of(b) <= addr(a.p)) return false;
    // side by side in rows of the same pitch
    const int64_t pitch = a.ld * a.esize;
    if (a.rows > 1 && b.rows > 1 && pitch == b.ld * b.esize) {
        const int64_t d = int64_t(addr(b.p)) - int64_t(addr(a.p));
        const int64_t off = ((d % pitch) + pitch) % pitch;
        if (off >= a.cols * a.esize && off + b.cols * b.esize <= pitch) return false;
    }
    return true;
}

struct Checker {
    Matrix m[16];
    int n = 0;
    int twin_in = -1, twin_out = -1;      // places of an input and of the output that may coincide with it exactly
    ssd_status st = SSD_OK;

    // The argument's place in `m`, or -1 where there is none.
    int add(const void *p, int64_t ld, int64_t rows, int64_t cols, int esize, bool write, bool needed)
    {
        if (!p && rows > 0 && needed) st = SSD_ERR_ARG;
        if (!p || rows == 0) return -1;
        if (rows > 1 && (ld < cols || ld >= (int64_t(1) << 36))) {
            st = SSD_ERR_ARG;
            return -1;
        }
        if (st == SSD_OK && addr(p) % esize) st = SSD_ERR_ALIGN;
        m[n] = Matrix{const_cast<void *>(p), ld, rows, cols, esize, write};
        return n++;
    }
    ssd_status overlaps(const void *workspace, int64_t bytes) const
    {
        for (int i = 0; i < n; ++i) {
            if (bytes > 0 && overlap(m[i], Matrix{const_cast<void *>(workspace), bytes, 1, bytes, 1, true})) return SSD_ERR_ARG;
            for (int j = 0; j < i; ++j) {
                if (!m[i].write && !m[j].write) continue;
                if (!overlap(m[i], m[j])) continue;
                // by their places: another argument may have the same address and pitch
                const bool twins = (i == twin_out && j == twin_in) || (i == twin_in && j == twin_out);
                if (twins && m[i].p == m[j].p && (m[i].ld == m[j].ld || m[i].rows == 1)) continue;
                return SSD_ERR_ARG;
            }
        }
        return SSD_OK;
    }
};

int esize(int32_t dtype) { return dtype == SSD_BF16 ? 2 : 4; }

bool bad_sizes(int64_t rows, int64_t in, int64_t out)
{
    return rows < 0 || in < 1 || out < 1 || rows > kMaxDim || in > kMaxDim || out > kMaxDim;
}

bool bad_act(int32_t act) { return act < SSD_ACT_NONE || act > SSD_ACT_SILU; }

struct Forward {
    int64_t rows, in, out;
    int dtype, act, mats;
    const void *x, *w[2];
    int64_t ldx, ldw[2];
    Epilogue e;
};

struct Backward {
    int64_t rows, in, out;
    int dtype, act, grad_dtype, mats;
    const void *dy, *x, *w[2], *z[2];
    int64_t lddy, ldx, ldw[2], ldz[2];
    void *dx, *dw[2], *db[2];
    int64_t lddx, lddw[2];
};

// ---------------------------------------------------------------------------------------------------------
// Work of a call.  The same code runs twice: once without a workspace, to count the bytes it takes from it, and once
// in earnest.

// What a call takes from its workspace starts on 32 bytes (sums of split products go out by 256-bit stores), the workspace itself on 16: the
// room to round it up is counted with the rest.
constexpr int64_t kWorkspaceAlign = 16, kTakeAlign = 32;
int64_t workspace_bytes_of(int64_t used) { return used ? used + (kTakeAlign - kWorkspaceAlign) : 0; }

struct Call {
    unsigned char *base = nullptr;      // a multiple of kTakeAlign; NULL: count only
    int64_t used = 0;
    cudaStream_t stream = nullptr;
    cudaError_t err = cudaSuccess;

    void *take(int64_t bytes)
    {
        void *p = base ? base + used : nullptr;
        used += (bytes + 255) / 256 * 256;
        return p;
    }
    bool live() const { return base != nullptr && err == cudaSuccess; }
    void launched(cudaError_t e)
    {
        if (err == cudaSuccess) err = e;
        count_launches(1);
    }
};

int64_t round8(int64_t v) { return (v + 7) / 8 * 8; }

struct PrepResult {
    Planes planes;
    float *sums = nullptr;
    int chunks = 0;
};

// Rows of a chunk: 16, the fewest that give each warp two, or as many more as keep the blocks at about eight per SM and the
// chunks, whose column sums are added up again, at 256.
int prep_rows_per_chunk(int64_t rows, int64_t cols)
{
    const int64_t strips = (cols + kPrepCols - 1) / kPrepCols;
    int64_t r = 16;
    while ((rows + r - 1) / r > 256 || (rows + r - 1) / r * strips > 8 * 148) {
        if ((rows + r - 1) / r <= 1) break;
        r *= 2;
    }
    return int(r);
}

template <typename T, int MATS, int ACT> cudaError_t launch_prep_parts(const PrepJobs &jobs, int blocks, cudaStream_t stream)
{
    if (jobs.job[0].parts == 3) return launch(prep_kernel<T, MATS, ACT, 3>, dim3(unsigned(blocks)), kPrepWarps * 32, 0, 1, stream, jobs);
    return launch(prep_kernel<T, MATS, ACT, 1>, dim3(unsigned(blocks)), kPrepWarps * 32, 0, 1, stream, jobs);
}

template <typename T, int MATS> cudaError_t launch_prep_act(const PrepJobs &jobs, int blocks, cudaStream_t stream)
{
    const int act = jobs.job[0].act;
    if (act == SSD_ACT_RELU) return launch_prep_parts<T, MATS, SSD_ACT_RELU>(jobs, blocks, stream);
    if (act == SSD_ACT_GELU) return launch_prep_parts<T, MATS, SSD_ACT_GELU>(jobs, blocks, stream);
    if (act == SSD_ACT_SILU) return launch_prep_parts<T, MATS, SSD_ACT_SILU>(jobs, blocks, stream);
    return launch_prep_parts<T, MATS, SSD_ACT_NONE>(jobs, blocks, stream);
}

template <typename T> cudaError_t launch_prep(const PrepJobs &jobs, int blocks, cudaStream_t stream)
{
    return jobs.job[0].mats == 2 ? launch_prep_act<T, 2>(jobs, blocks, stream) : launch_prep_act<T, 1>(jobs, blocks, stream);
}

// The passes of a call.  Matrices that are only brought into planes are collected and go in one launch.
struct Passes {
    PrepJobs jobs{};
    int count = 0;

    // Takes the pass's room in the workspace and its place in the launch.
    PrepResult add(Call &c, PrepParams p, int dtype, bool want_sums)
    {
        PrepResult r;
        const int es = esize(dtype);
        p.rows_per_chunk = prep_rows_per_chunk(p.rows, p.cols);
        p.strips = (p.cols + kPrepCols - 1) / kPrepCols;
        r.chunks = int((p.rows + p.rows_per_chunk - 1) / p.rows_per_chunk);
        p.ldp = round8(p.cols);
        p.zstride = p.rows * p.ldp;
        p.planes = static_cast<__nv_bfloat16 *>(c.take(int64_t(p.parts) * p.mats * p.zstride * 2));
        p.sums = want_sums ? static_cast<float *>(c.take(int64_t(r.chunks) * p.mats * p.cols * 4)) : nullptr;
        r.planes = Planes{p.planes, p.ldp, p.zstride, int(p.rows), p.cols, p.parts * p.mats};
        r.sums = p.sums;
        auto vec = [&](const void *q, int64_t ld) { return addr(q) % 16 == 0 && (ld * es % 16 == 0 || p.rows == 1); };
        const bool use_z0 = p.act != SSD_ACT_NONE || p.mats == 2;
        p.vec = p.cols % kLane == 0 && vec(p.src, p.ld) && (!use_z0 || vec(p.z0, p.ldz0)) && (p.mats == 1 || vec(p.z1, p.ldz1));
        jobs.job[count] = p;
        jobs.end[count] = (count ? jobs.end[count - 1] : 0) + p.strips * r.chunks;
        ++count;
        return r;
    }
    void run(Call &c, int dtype)
    {
        if (count == 0) return;
        const int blocks = jobs.end[count - 1];
        for (int i = count; i < kMaxJobs; ++i) jobs.end[i] = blocks;
        if (c.live()) c.launched(dtype == SSD_F32 ? launch_prep<float>(jobs, blocks, c.stream) : launch_prep<__nv_bfloat16>(jobs, blocks, c.stream));
        count = 0;
    }
};

bool tma_can_read(const void *src, int64_t ld, int64_t rows, int dtype) { return dtype == SSD_BF16 && addr(src) % 16 == 0 && (ld % 8 == 0 || rows == 1); }

// A matrix as the product kernels read it: in place where it is bfloat16 with 16-byte rows, else as planes that a pass makes.
Planes operand(Call &c, Passes &passes, const void *src, int64_t ld, int64_t rows, int64_t cols, int dtype, int parts)
{
    if (tma_can_read(src, ld, rows, dtype))
        return Planes{static_cast<const __nv_bfloat16 *>(src), rows == 1 ? round8(cols) : ld, 0, int(rows), int(cols), 1};
    PrepParams p{};
    p.src = src;
    p.ld = ld;
    p.rows = rows;
    p.cols = int(cols);
    p.act = SSD_ACT_NONE;
    p.mats = 1;
    p.parts = parts;
    return passes.add(c, p, dtype, false).planes;
}

// Partial products kept of operands in pa and pb parts (part i is at most 2^-8i of the value): orders 0 to 2, the
// smallest first; what is left out is 2e-8 of the result's norm, a thirtieth of the rounding of the sums, for six products in place of nine.
// `half`: orders 0 and 1, for results that are rounded to bfloat16: 3e-6 left out of a result that is rounded to 1.7e-3, for half the products.
int segments_of(Segment *out, int pa, int pb, int a_step, int b, bool half)
{
    int n = 0;
    for (int order = 2; order >= 0; --order) {
        if (half && order == 2 && pa + pb > 2) continue;
        for (int i = 0; i <= order; ++i) {
            const int ia = order - i, ib = i;
            if (ia < pa && ib < pb) out[n++] = Segment{int8_t(ia * a_step), int8_t(b), int8_t(ib)};
        }
    }
    return n;
}

// What the rows of residual, out and z are all aligned to, for the epilogue.
int row_alignment(const Product &p)
{
    const Epilogue &e = p.e;
    uintptr_t bits = 0;
    const int es = e.f32 ? 4 : 2;
    auto add = [&](const void *q, int64_t ld) { bits |= q ? addr(q) | (p.m > 1 ? uintptr_t(ld) * es : 0) : 0; };
    add(e.residual, e.ldr);
    for (int i = 0; i < 2; ++i) {
        add(e.out[i], e.ldo[i]);
        add(e.z[i], e.ldz[i]);
    }
    return bits % 32 == 0 ? 32 : (bits % 16 == 0 ? 16 : 0);
}

void product(Call &c, Product &p)
{
    p.e.vec = row_alignment(p);
    float *partial = static_cast<float *>(c.take(product_partial_floats(p) * 4));
    if (!c.live()) return;
    const cudaError_t e = launch_product(p, partial, c.stream);
    if (c.err == cudaSuccess) c.err = e;
}

// Which calls go to the kernels for a few rows.  Measured, microseconds there and on the tensor cores, weights from HBM (where they are many enough):
//   float32 forward  4096 x 4096, 1 row 13.9 / 60, 8 rows 26 / 61, 16 rows 46 / 61; 1024 x 1024, 16 rows 4.8 / 14; 2048 x 128256, 16 rows 514 / 961
//   float32 forward of more rows, eight at a time: 64 x 512 x 512 4.4 / 9.5, 24 x 1024 x 1024 7.1 / 13.6 (gated 12.2 / 15.4), 1024 x 64 x 10 3.4 / 9.5,
//                    7000 x 1000 x 8 24 / 30; but 1000 x 64 x 1000 38 / 9.7, 8000 x 8 x 1000 289 / 32, 250 x 500 x 500 30 / 16, 100000 x 1 x 64 240 / 99
//   bfloat16 forward 4096 x 4096, 1 row 8.3 / 10.4, 8 rows 11.4 / 11.0, 16 rows 10.3 / 11.1; 1024 x 1024, 8 rows 2.7 / 5.2;
//                    gated 2048 x 8192, 8 rows 14.5 / 16.2, 16 rows 16.5 / 16.8;
//                    a long contraction or many weights: 8192 x 2048, 8 rows 19 / 14; 32768 x 2048, 8 rows 67 / 29; 2048 x 128256, 16 rows 136 / 103
//   ... of rows that lie anywhere (weights in L2): 1001 x 2003, 4 rows 5.7 / 9.9, 8 rows 13 / 9.9; 301 x 200, 30 rows 6.9 / 5.9
//   backward (float32 weight gradients) 4096 x 4096, 8 rows 35 / 52 bfloat16, 38 / 106 float32; 16 rows 51 / 53, 54 / 108;
//                    256 x 256, 16 rows 6.6 / 17 bfloat16; 2048 x 128256, 16 rows 717 / 463 bfloat16, 726 / 1302 float32
//   backward (bfloat16 gradients, 16 rows) 1024 x 1024 17 / 16, 4096 x 4096 50 / 36, 2048 x 128256 722 / 300; 9900 x 7634 (rows off 16 bytes) 370 / 914
// so multiply-adds take float32 of up to 16 rows, and of more where both sides' estimates say so (over 300 drawn calls 0.4 % slower than the better side of
// each, 1.4 times at worst); bfloat16 in aligned rows goes by what a warp has to do (rows_mma_pays: 0.2 % over 110 drawn calls), rows that lie anywhere
// by the number of weights, counted once for every eight rows.  Backward, nine to sixteen bfloat16 rows go to the tensor cores from a number of weights on.
constexpr int kFewRowsMost = 16;
constexpr double kFewEightsAnywhere = 2.5e6;

// Estimated time of a float32 forward on the tensor cores: the pass that brings the operands into parts (2 us for each time a warp goes
// through its rows of them, 5 TB/s where there is much of it), and the product.
double parts_forward_us(const Forward &f)
{
    Product p{};
    p.m = int(f.rows);
    p.n = int(f.out);
    p.k = int(f.in);
    p.nseg = 6;
    p.nmain = p.groups = 1;
    p.gated = f.mats == 2;
    p.e = f.e;
    p.e.vec = row_alignment(p);
    auto turns = [&](int64_t rows) { return double((std::min<int64_t>(prep_rows_per_chunk(rows, f.in), rows) + 2 * kPrepWarps - 1) / (2 * kPrepWarps)); };
    const double bytes = 10.0 * double(f.in) * (double(f.rows) + double(f.mats) * double(f.out));
    return 2.0 + std::max(2.0 * std::max(turns(f.rows), turns(f.out)), bytes / 5e6) + product_us(p);
}

RowsForward rows_of(const Forward &f)
{
    return RowsForward{f.x, {f.w[0], f.w[1]}, f.ldx, {f.ldw[0], f.ldw[1]}, int(f.rows), int(f.in), int(f.out), f.mats == 2, 0, 0, f.e};
}

bool few_rows(const Forward &f)
{
    if (f.dtype == SSD_F32) return f.rows <= kFewRowsMost || rows_forward_f32_us(rows_of(f)) <= parts_forward_us(f);
    const double eights = double((f.rows + 7) / 8) * double(f.out) * double(f.in) * f.mats;      // weights read by eight rows at a time
    bool aligned = tma_can_read(f.x, f.ldx, f.rows, f.dtype) && f.in % 8 == 0;
    for (int i = 0; i < f.mats; ++i) aligned = aligned && tma_can_read(f.w[i], f.ldw[i], f.out, f.dtype);
    if (aligned) return f.rows == 1 || (f.rows <= kFewRowsMost && rows_mma_pays(rows_of(f)));
    return f.rows <= 4 ? eights <= kFewEightsAnywhere : f.rows <= 8 && eights <= kFewEightsAnywhere / 8;
}

bool few_rows(const Backward &b)
{
    if (b.rows <= 8 || b.rows > kFewRowsMost || b.dtype == SSD_F32) return b.rows <= kFewRowsMost;
    bool aligned = b.in % 8 == 0 && (!b.dw[0] || tma_can_read(b.x, b.ldx, b.rows, b.dtype));
    for (int i = 0; i < b.mats; ++i) aligned = aligned && (!b.dx || tma_can_read(b.w[i], b.ldw[i], b.out, b.dtype));
    return !aligned || double(b.out) * double(b.in) * b.mats <= (b.grad_dtype == SSD_F32 ? 5e7 : 5e6);
}

void run_forward(Call &c, const Forward &f)
{
    if (f.rows == 0) return;
    if (few_rows(f)) {
        if (c.live()) {
            const cudaError_t e = launch_rows_forward(rows_of(f), c.stream);
            if (c.err == cudaSuccess) c.err = e;
        }
        return;
    }
    const int parts = f.dtype == SSD_F32 ? 3 : 1;
    Product p{};
    Passes passes;
    p.a = operand(c, passes, f.x, f.ldx, f.rows, f.in, f.dtype, parts);
    for (int i = 0; i < f.mats; ++i) p.b[i] = operand(c, passes, f.w[i], f.ldw[i], f.out, f.in, f.dtype, parts);
    passes.run(c, f.dtype);
    p.nseg = segments_of(p.seg, parts, parts, 1, 0, false);
    p.nmain = 1;
    p.m = int(f.rows);
    p.n = int(f.out);
    p.k = int(f.in);
    p.groups = 1;
    p.gated = f.mats == 2;
    p.e = f.e;
    product(c, p);
}

void run_backward(Call &c, const Backward &b)
{
    const bool want_dw = b.dw[0] != nullptr, want_db = b.db[0] != nullptr, want_dx = b.dx != nullptr;
    const int gs = esize(b.grad_dtype);
    if (b.rows == 0) {
        if (!c.live()) return;
        for (int i = 0; i < b.mats; ++i) {
            if (want_dw) c.err = cudaMemset2DAsync(b.dw[i], size_t(b.out == 1 ? b.in : b.lddw[i]) * gs, 0, size_t(b.in) * gs, size_t(b.out), c.stream);
            if (want_db && c.err == cudaSuccess) c.err = cudaMemsetAsync(b.db[i], 0, size_t(b.out) * gs, c.stream);
        }
        return;
    }
    const bool f32 = b.dtype == SSD_F32;
    if (few_rows(b)) {
        RowsBackward q{};
        q.dy = b.dy;
        q.lddy = b.lddy;
        q.x = b.x;
        q.ldx = b.ldx;
        q.dx = b.dx;
        q.lddx = b.lddx;
        for (int i = 0; i < b.mats; ++i) {
            q.w[i] = b.w[i];
            q.ldw[i] = b.ldw[i];
            q.z[i] = b.z[i];
            q.ldz[i] = b.ldz[i];
            q.dw[i] = b.dw[i];
            q.lddw[i] = b.lddw[i];
            q.db[i] = b.db[i];
        }
        if (want_dx) q.partial = static_cast<float *>(c.take(rows_partial_floats(int(b.rows), int(b.out), int(b.in)) * 4));
        q.rows = int(b.rows);
        q.in = int(b.in);
        q.out = int(b.out);
        q.act = b.act;
        q.mats = b.mats;
        q.f32 = f32;
        q.grad_f32 = b.grad_dtype == SSD_F32;
        if (c.live() && (want_dx || want_dw || want_db)) {
            const cudaError_t e = launch_rows_backward(q, c.stream);
            if (c.err == cudaSuccess) c.err = e;
        }
        return;
    }
    const bool plain = b.act == SSD_ACT_NONE && b.mats == 1;      // dz is dy
    // dz in as many parts as its most exact use asks for: float32 operands, or float32 weight gradients of a dz that bfloat16 does not hold exactly.
    // For bfloat16 results one part, a rounding to the type that the results have themselves: two or three parts would take that many times the
    // products, for an error of 1.7e-3 of the result's norm instead of 2.3e-3 (of which 1.7e-3 is the rounding of the result).
    const int dw_parts = f32 ? 3 : (plain || b.grad_dtype == SSD_BF16 ? 1 : 3);
    const int dx_parts = f32 ? 3 : 1, op_parts = f32 ? 3 : 1;
    const bool dy_ready = plain && tma_can_read(b.dy, b.lddy, b.rows, b.dtype);

    // dz, the bias gradients' chunks
    PrepParams q{};
    q.src = b.dy;
    q.ld = b.lddy;
    q.z0 = b.z[0];
    q.ldz0 = b.ldz[0];
    q.z1 = b.z[1];
    q.ldz1 = b.ldz[1];
    q.rows = b.rows;
    q.cols = int(b.out);
    q.act = b.act;
    q.mats = b.mats;
    q.parts = dy_ready || !(want_dx || want_dw) ? 0 : (want_dw && dw_parts > dx_parts ? dw_parts : dx_parts);
    Passes passes;
    PrepResult r;
    if (q.parts || want_db) {
        r = passes.add(c, q, b.dtype, want_db);
        // a dz that is more than dy in parts takes a launch of its own
        if (!plain || q.parts != op_parts) passes.run(c, b.dtype);
    }
    const Planes dz = dy_ready ? operand(c, passes, b.dy, b.lddy, b.rows, b.out, b.dtype, 1) : r.planes;

    // dx: by order of magnitude over both halves of a gated sum
    Product x{};
    if (want_dx) {
        Segment half[kMaxSegments];
        const int n = segments_of(half, dx_parts, op_parts, b.mats, 0, false);
        for (int s = 0; s < n; ++s)
            for (int i = 0; i < b.mats; ++i) x.seg[x.nseg++] = Segment{int8_t(half[s].az + i), int8_t(i), half[s].bz};
        x.nmain = b.mats;
        x.a = dz;
        for (int i = 0; i < b.mats; ++i) x.b[i] = operand(c, passes, b.w[i], b.ldw[i], b.out, b.in, b.dtype, op_parts);
        x.b_mn = 1;
        x.m = int(b.rows);
        x.n = int(b.in);
        x.k = int(b.out);
        x.groups = 1;
        x.e.out[0] = b.dx;
        x.e.ldo[0] = b.lddx;
        x.e.f32 = f32;
        if (passes.count == kMaxJobs) passes.run(c, b.dtype);
    }
    Product w{};
    if (want_dw) {
        w.a = dz;
        w.a_mn = 1;
        w.b[0] = operand(c, passes, b.x, b.ldx, b.rows, b.in, b.dtype, op_parts);
        w.b_mn = 1;
        w.nseg = segments_of(w.seg, dw_parts, op_parts, b.mats, 0, b.grad_dtype == SSD_BF16);
        w.nmain = 1;
        w.m = int(b.out);
        w.n = int(b.in);
        w.k = int(b.rows);
        w.groups = b.mats;
        for (int i = 0; i < b.mats; ++i) {
            w.e.out[i] = b.dw[i];
            w.e.ldo[i] = b.lddw[i];
        }
        w.e.f32 = b.grad_dtype == SSD_F32;
    }
    passes.run(c, b.dtype);
    if (want_db && c.live())
        c.launched(launch(sums_kernel, dim3(unsigned((b.out + 31) / 32), unsigned(b.mats)), 256, 0, 1, c.stream, static_cast<const float *>(r.sums), r.chunks, b.mats,
                          int(b.out), b.db[0], b.db[1], int(b.grad_dtype == SSD_F32)));
    if (want_dx) product(c, x);
    if (want_dw) product(c, w);
}

ssd_status check(const ssd_linear_fwd *a, Forward *f, Checker *k)
{
    if (!a || bad_sizes(a->rows, a->in_features, a->out_features) || !valid_dtype(a->dtype) || bad_act(a->act)) return SSD_ERR_ARG;
    const int es = esize(a->dtype);
    *f = Forward{a->rows, a->in_features, a->out_features, a->dtype, a->act, 1, a->x, {a->weight, nullptr}, a->ldx, {a->ldw, 0}, {}};
    k->add(a->x, a->ldx, f->rows, f->in, es, false, true);
    k->add(a->weight, a->ldw, f->out, f->in, es, false, true);
    k->add(a->bias, f->out, 1, f->out, 4, false, false);
    k->twin_in = k->add(a->residual, a->ldr, f->rows, f->out, es, false, false);
    k->twin_out = k->add(a->y, a->ldy, f->rows, f->out, es, true, true);
    k->add(a->z, a->ldz, f->rows, f->out, es, true, false);
    f->e.bias[0] = a->bias;
    f->e.residual = a->residual;
    f->e.ldr = a->ldr;
    f->e.out[0] = a->y;
    f->e.ldo[0] = a->ldy;
    f->e.z[0] = a->z;
    f->e.ldz[0] = a->ldz;
    f->e.act = a->act;
    f->e.f32 = a->dtype == SSD_F32;
    return k->st;
}

ssd_status check(const ssd_gated_fwd *a, Forward *f, Checker *k)
{
    if (!a || bad_sizes(a->rows, a->in_features, a->out_features) || !valid_dtype(a->dtype) || bad_act(a->act)) return SSD_ERR_ARG;
    const int es = esize(a->dtype);
    *f = Forward{a->rows, a->in_features, a->out_features, a->dtype, a->act, 2, a->x, {a->w_gate, a->w_up}, a->ldx, {a->ldwg, a->ldwu}, {}};
    k->add(a->x, a->ldx, f->rows, f->in, es, false, true);
    k->add(a->w_gate, a->ldwg, f->out, f->in, es, false, true);
    k->add(a->w_up, a->ldwu, f->out, f->in, es, false, true);
    k->add(a->b_gate, f->out, 1, f->out, 4, false, false);
    k->add(a->b_up, f->out, 1, f->out, 4, false, false);
    k->add(a->h, a->ldh, f->rows, f->out, es, true, true);
    k->add(a->gate, a->ldgate, f->rows, f->out, es, true, false);
    k->add(a->up, a->ldup, f->rows, f->out, es, true, false);
    f->e.bias[0] = a->b_gate;
    f->e.bias[1] = a->b_up;
    f->e.out[0] = a->h;
    f->e.ldo[0] = a->ldh;
    f->e.z[0] = a->gate;
    f->e.ldz[0] = a->ldgate;
    f->e.z[1] = a->up;
    f->e.ldz[1] = a->ldup;
    f->e.act = a->act;
    f->e.f32 = a->dtype == SSD_F32;
    return k->st;
}

ssd_status check(const ssd_linear_bwd *a, Backward *b, Checker *k)
{
    if (!a || bad_sizes(a->rows, a->in_features, a->out_features) || !valid_dtype(a->dtype) || !valid_dtype(a->grad_dtype) || bad_act(a->act) || a->reserved)
        return SSD_ERR_ARG;
    const int es = esize(a->dtype), gs = esize(a->grad_dtype);
    *b = Backward{a->rows, a->in_features, a->out_features, a->dtype, a->act, a->grad_dtype, 1, a->dy, a->x, {a->weight, nullptr}, {a->z, nullptr},
                  a->lddy, a->ldx, {a->ldw, 0}, {a->ldz, 0}, a->dx, {a->dweight, nullptr}, {a->dbias, nullptr}, a->lddx, {a->lddw, 0}};
    k->add(a->dy, a->lddy, b->rows, b->out, es, false, true);
    if (a->dweight) k->add(a->x, a->ldx, b->rows, b->in, es, false, true);
    if (a->dx) k->add(a->weight, a->ldw, b->out, b->in, es, false, b->rows > 0);
    if (a->act != SSD_ACT_NONE) k->add(a->z, a->ldz, b->rows, b->out, es, false, true);
    k->add(a->dx, a->lddx, b->rows, b->in, es, true, false);
    k->add(a->dweight, a->lddw, b->out, b->in, gs, true, false);
    k->add(a->dbias, b->out, 1, b->out, gs, true, false);
    return k->st;
}

ssd_status check(const ssd_gated_bwd *a, Backward *b, Checker *k)
{
    if (!a || bad_sizes(a->rows, a->in_features, a->out_features) || !valid_dtype(a->dtype) || !valid_dtype(a->grad_dtype) || bad_act(a->act) || a->reserved)
        return SSD_ERR_ARG;
    if (!a->dw_gate != !a->dw_up || !a->db_gate != !a->db_up) return SSD_ERR_ARG;
    const int es = esize(a->dtype), gs = esize(a->grad_dtype);
    *b = Backward{a->rows, a->in_features, a->out_features, a->dtype, a->act, a->grad_dtype, 2, a->dh, a->x, {a->w_gate, a->w_up}, {a->gate, a->up},
                  a->lddh, a->ldx, {a->ldwg, a->ldwu}, {a->ldgate, a->ldup}, a->dx, {a->dw_gate, a->dw_up}, {a->db_gate, a->db_up}, a->lddx,
                  {a->lddwg, a->lddwu}};
    k->add(a->dh, a->lddh, b->rows, b->out, es, false, true);
    if (a->dw_gate) k->add(a->x, a->ldx, b->rows, b->in, es, false, true);
    if (a->dx) {
        k->add(a->w_gate, a->ldwg, b->out, b->in, es, false, b->rows > 0);
        k->add(a->w_up, a->ldwu, b->out, b->in, es, false, b->rows > 0);
    }
    k->add(a->gate, a->ldgate, b->rows, b->out, es, false, true);
    k->add(a->up, a->ldup, b->rows, b->out, es, false, true);
    k->add(a->dx, a->lddx, b->rows, b->in, es, true, false);
    k->add(a->dw_gate, a->lddwg, b->out, b->in, gs, true, false);
    k->add(a->dw_up, a->lddwu, b->out, b->in, gs, true, false);
    k->add(a->db_gate, b->out, 1, b->out, gs, true, false);
    k->add(a->db_up, b->out, 1, b->out, gs, true, false);
    return k->st;
}

void run(Call &c, const Forward &f) { run_forward(c, f); }
void run(Call &c, const Backward &b) { run_backward(c, b); }

template <typename Work, typename Args> ssd_status workspace_of(const Args *args, int64_t *bytes)
{
    if (!bytes) return SSD_ERR_ARG;
    Work w;
    Checker k;
    const ssd_status st = check(args, &w, &k);
    if (st != SSD_OK) return st;
    Call c;
    run(c, w);
    *bytes = workspace_bytes_of(c.used);
    return SSD_OK;
}

template <typename Work, typename Args>
ssd_status run_call(const Args *args, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    Work w;
    Checker k;
    ssd_status st = check(args, &w, &k);
    if (st != SSD_OK) return st;
    Call count;
    run(count, w);
    const int64_t need = workspace_bytes_of(count.used);
    if (need > 0 && (!workspace || workspace_bytes < need)) return SSD_ERR_ARG;
    if (need > 0 && addr(workspace) % kWorkspaceAlign) return SSD_ERR_ALIGN;
    st = k.overlaps(workspace, need);
    if (st != SSD_OK) return st;
    Call c;
    alignas(kTakeAlign) static unsigned char none;
    c.base = need > 0 ? static_cast<unsigned char *>(workspace) + (addr(workspace) % kTakeAlign ? kTakeAlign - kWorkspaceAlign : 0) : &none;
    c.stream = static_cast<cudaStream_t>(cuda_stream);
    run(c, w);
    return c.err == cudaSuccess ? SSD_OK : layer_cuda_fail(c.err);
}

}  // namespace

extern "C" {

ssd_status ssd_linear_forward_workspace(const ssd_linear_fwd *args, int64_t *bytes) { return workspace_of<Forward>(args, bytes); }
ssd_status ssd_linear_backward_workspace(const ssd_linear_bwd *args, int64_t *bytes) { return workspace_of<Backward>(args, bytes); }
ssd_status ssd_gated_forward_workspace(const ssd_gated_fwd *args, int64_t *bytes) { return workspace_of<Forward>(args, bytes); }
ssd_status ssd_gated_backward_workspace(const ssd_gated_bwd *args, int64_t *bytes) { return workspace_of<Backward>(args, bytes); }

ssd_status ssd_linear_forward(const ssd_linear_fwd *args, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    return run_call<Forward>(args, workspace, workspace_bytes, cuda_stream);
}
ssd_status ssd_linear_backward(const ssd_linear_bwd *args, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    return run_call<Backward>(args, workspace, workspace_bytes, cuda_stream);
}
ssd_status ssd_gated_forward(const ssd_gated_fwd *args, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    return run_call<Forward>(args, workspace, workspace_bytes, cuda_stream);
}
ssd_status ssd_gated_backward(const ssd_gated_bwd *args, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    return run_call<Backward>(args, workspace, workspace_bytes, cuda_stream);
}

ssd_status ssd_layer_error(int32_t *flag)
{
    if (!flag) return SSD_ERR_ARG;
    int value = 0;
    const cudaError_t e = read_product_error(&value);
    if (e != cudaSuccess) return layer_cuda_fail(e);
    *flag = value;
    return SSD_OK;
}

const char *ssd_layer_cuda_error(void) { return g_cuda_error.c_str(); }

int64_t ssd_layer_launches(void) { return g_launches; }

}  // extern "C"
