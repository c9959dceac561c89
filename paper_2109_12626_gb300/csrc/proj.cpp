// proj.cpp -- host side of the projections: plans, argument checks, scratch
// and the sequence of kernels of each call.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <mutex>
#include <new>
#include <utility>

#include "proj.h"

namespace dpdr {
namespace proj {

namespace {

constexpr int64_t kMost = (int64_t(1) << 31) - 1;

// A refusal as "who: what", without allocating.
int refuse(const char* who, const char* what, const char* more = "")
{
    char msg[200];
    std::snprintf(msg, sizeof msg, "%s: %s%s%s", who, what, *more ? " " : "", more);
    return fail_c(DPDR_ERR_INVALID, msg);
}

bool is_half_kind(int t) { return t == DPDR_BFLOAT16 || t == DPDR_FLOAT16; }

// Error words of all plans: page-locked host memory that kernels write to and
// the host reads, allocated for many plans at a time and kept for the process
// (a device allocation and its clearing made a plan 60 us longer to build).
class ErrorWords {
public:
    uint32_t* take(const char* who)
    {
        std::lock_guard<std::mutex> hold(m_);
        if (!free_) {
            void* p = nullptr;
            const cudaError_t e = cudaHostAlloc(&p, kSlots * sizeof(Slot), cudaHostAllocPortable | cudaHostAllocMapped);
            if (e != cudaSuccess) {
                cuda_fail_c(e, who);
                return nullptr;
            }
            Slot* slots = static_cast<Slot*>(p);
            for (int i = 0; i < kSlots; i++) slots[i].next = i + 1 < kSlots ? slots + i + 1 : nullptr;
            free_ = slots;
        }
        Slot* s = free_;
        free_ = s->next;
        s->word = 0;
        return &s->word;
    }
    void give(uint32_t* w)
    {
        if (!w) return;
        std::lock_guard<std::mutex> hold(m_);
        Slot* s = reinterpret_cast<Slot*>(w);   // its first member
        s->next = free_;
        free_ = s;
    }

private:
    struct alignas(32) Slot {
        uint32_t word;
        Slot* next;   // of a slot that no plan has
    };
    static constexpr int kSlots = 1024;
    std::mutex m_;
    Slot* free_ = nullptr;
};
ErrorWords g_errors;

Proj* make(bool gated, int64_t max_rows, int64_t n_in, int64_t n_out, int operands, int result, int gradients,
           int act, const char* who)
{
    auto bad = [&](const char* what) {
        refuse(who, what);
        return nullptr;
    };
    if (max_rows < 0 || max_rows > kMost || n_in < 1 || n_in > kMost || n_out < 1 || n_out > kMost)
        return bad("need 0 <= max_rows and 1 <= sizes, below 2^31");
    if (!is_half_kind(operands)) return bad("operands are bfloat16 or float16");
    if ((result != operands && result != DPDR_FLOAT32) || (gradients != operands && gradients != DPDR_FLOAT32))
        return bad("result and gradients have the operands' type or float32");
    if (act < DPDR_ACT_NONE || act > DPDR_ACT_SIGMOID) return bad("unknown activation");
    Proj* P = new (std::nothrow) Proj;
    if (!P) {
        fail_c(DPDR_ERR_OOM, "projection plan: host allocation");
        return nullptr;
    }
    P->gated = gated;
    P->max_rows = max_rows;
    P->n_in = n_in;
    P->n_out = n_out;
    P->half = operands == DPDR_FLOAT16;
    P->out_f32 = result == DPDR_FLOAT32;
    P->grad_f32 = gradients == DPDR_FLOAT32;
    P->act = act;
    cudaError_t e = cudaGetDevice(&P->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&P->num_sms, cudaDevAttrMultiProcessorCount, P->device);
    if (e != cudaSuccess) {
        cuda_fail_c(e, who);
        delete P;
        return nullptr;
    }
    P->err = g_errors.take(who);
    if (!P->err) {
        delete P;
        return nullptr;
    }
    return P;
}

// A matrix argument in bytes: which range of memory it touches, and which
// part of each row of its pitch.
struct Span {
    uintptr_t lo = 0, hi = 0, pitch = 0, width = 0;
};

Span span_of(const dpdr_matrix& m, int64_t rows, int64_t cols, int esize)
{
    Span s;
    if (rows == 0 || cols == 0) return s;
    s.lo = reinterpret_cast<uintptr_t>(m.data);
    const uintptr_t last = uintptr_t(rows - 1) * uintptr_t(m.row_stride) + uintptr_t(cols - 1) * uintptr_t(m.col_stride);
    s.hi = s.lo + (last + 1) * esize;
    s.pitch = uintptr_t(m.row_stride) * esize;
    s.width = m.col_stride == 1 ? uintptr_t(cols) * esize : s.pitch;
    return s;
}

// Whether two arguments may share a byte.  Column slices of one wider array
// (equal pitch, disjoint parts of it) do not.
bool overlap(const Span& a, const Span& b)
{
    if (a.lo == a.hi || b.lo == b.hi || a.hi <= b.lo || b.hi <= a.lo) return false;
    if (a.pitch == b.pitch && a.pitch > 0 && a.width <= a.pitch && b.width <= b.pitch) {
        const uintptr_t d = b.lo >= a.lo ? (b.lo - a.lo) % a.pitch : (a.pitch - (a.lo - b.lo) % a.pitch) % a.pitch;
        if (d >= a.width && d + b.width <= a.pitch) return false;
    }
    return true;
}

// The arguments of one call, checked as they are added.
struct Args {
    const char* who;
    Span in[6], out[4];
    int nin = 0, nout = 0;
    int rc = DPDR_OK;

    void refuse(const char* name, const char* what)
    {
        if (rc == DPDR_OK) rc = proj::refuse(who, name, what);
    }
    void input(const char* name, const dpdr_matrix* m, int64_t rows, int64_t cols, int esize)
    {
        if (!m) return refuse(name, "is NULL");
        check(name, *m, rows, cols, esize);
        if (m->row_stride < 0 || m->col_stride < 0) return refuse(name, "has a negative stride");
        in[nin++] = span_of(*m, rows, cols, esize);
    }
    void output(const char* name, const dpdr_matrix* m, int64_t rows, int64_t cols, int esize)
    {
        if (!m) return refuse(name, "is NULL");
        check(name, *m, rows, cols, esize);
        if (cols > 1 && m->col_stride != 1) return refuse(name, "needs col_stride 1");
        if (rows > 1 && m->row_stride < cols) return refuse(name, "has rows that overlap");
        dpdr_matrix unit = *m;
        unit.col_stride = 1;
        out[nout++] = span_of(unit, rows, cols, esize);
    }
    void check(const char* name, const dpdr_matrix& m, int64_t rows, int64_t cols, int esize)
    {
        if (rows == 0 || cols == 0) return;
        if (!m.data) return refuse(name, "has no address");
        if (reinterpret_cast<uintptr_t>(m.data) % uintptr_t(esize)) refuse(name, "is not aligned to its element");
        // byte offsets stay within 2^62
        const __int128 far = (__int128)(rows - 1) * m.row_stride + (__int128)(cols - 1) * m.col_stride;
        if (far > (__int128(1) << 59)) refuse(name, "reaches too far");
    }
    void vector(const char* name, const void* p, int64_t n, int esize, bool result)
    {
        const dpdr_matrix m{const_cast<void*>(p), n, 1};
        if (result) output(name, &m, 1, n, esize);
        else input(name, &m, 1, n, esize);
    }
    // no result may touch another argument (but the residual, which is checked
    // on its own)
    int done()
    {
        for (int i = 0; i < nout && rc == DPDR_OK; i++) {
            for (int k = 0; k < nin; k++)
                if (overlap(out[i], in[k])) return rc = proj::refuse(who, "a result overlaps an input");
            for (int k = 0; k < i; k++)
                if (overlap(out[i], out[k])) return rc = proj::refuse(who, "two results overlap");
        }
        return rc;
    }
};

int check_plan(const Proj* P, bool gated, int64_t rows, const char* who)
{
    if (!P) return refuse(who, "NULL plan");
    if (P->gated != gated) return refuse(who, "a plan of the other operator");
    if (rows < 0 || rows > P->max_rows) return refuse(who, "need 0 <= rows <= max_rows");
    // the plan's scratch, its kernels' attributes and the arrays belong to its device
    int current = -1;
    const cudaError_t e = cudaGetDevice(&current);
    if (e != cudaSuccess) return cuda_fail_c(e, who);
    if (current != P->device) return refuse(who, "the plan's device is not the current one");
    return DPDR_OK;
}

// Device memory of the plan's, made by the first call that needs it at the
// size of the largest use that any later call can have for it: a captured call
// may be replayed after others, so nothing is moved before the plan goes.
int hold(char*& at, size_t bytes, const char* what)
{
    if (at || bytes == 0) return DPDR_OK;
    const cudaError_t e = cudaMalloc(&at, bytes);
    return e == cudaSuccess ? DPDR_OK : cuda_fail_c(e, what);
}

Operand rows_of(const dpdr_matrix& m) { return {static_cast<const char*>(m.data), m.row_stride, m.col_stride}; }
Operand cols_of(const dpdr_matrix& m) { return {static_cast<const char*>(m.data), m.col_stride, m.row_stride}; }

Epilogue epilogue_of(const Proj* P)
{
    Epilogue e;
    e.act = P->act;
    e.half = P->half;
    return e;
}

void set_other(Epilogue& e, const dpdr_matrix& m, int f32)
{
    e.other = static_cast<const char*>(m.data);
    e.other_rs = m.row_stride;
    e.other_cs = m.col_stride;
    e.other_f32 = f32;
}

// A driver call by name: the library links no libcuda.
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return fn;
}

int64_t padded(int64_t n) { return (n + 7) / 8 * 8; }
// TMA's strides are below 2^40 bytes
constexpr int64_t kFarthest = int64_t(1) << 39;
// rows of column sums that join_launch takes: as many as column_sum_parts gives
constexpr int64_t kJoined = 512;
size_t upto256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

bool by_fours(const Epilogue& e)
{
    auto fits = [](const void* q, int64_t rs, int esize) {
        return reinterpret_cast<uintptr_t>(q) % uintptr_t(4 * esize) == 0 && rs % 4 == 0;
    };
    const int os = e.out_f32 ? 4 : 2;
    return fits(e.out, e.out_rs, os) && fits(e.out2, e.out2_rs, os) &&
           (!e.other || (e.other_cs == 1 && fits(e.other, e.other_rs, e.other_f32 ? 4 : 2))) &&
           (!e.pre || (fits(e.pre, e.pre_rs, 4) && e.pre_up % 4 == 0)) && fits(e.bias, 0, 2);
}

int tensor_map(CUtensorMap* map, const Operand& o, int64_t n, int64_t k, int half, int rows, int step)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return fail_c(DPDR_ERR_CUDA, "projection: the driver has no cuTensorMapEncodeTiled");
    const bool inner_k = o.ks == 1;
    const cuuint64_t dims[2] = {cuuint64_t(inner_k ? k : n), cuuint64_t(inner_k ? n : k)};
    const cuuint64_t pitch[1] = {cuuint64_t(inner_k ? o.is : o.ks) * 2};
    const cuuint32_t box[2] = {cuuint32_t(inner_k ? step : 64), cuuint32_t(inner_k ? rows : step)};
    const cuuint32_t one[2] = {1, 1};
    const CUresult r = encode(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
                              const_cast<char*>(o.p), dims, pitch, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? DPDR_OK : fail_c(DPDR_ERR_CUDA, "projection: tensor map refused");
}

// A packed copy in the plan's slot, made m's place: by rows, or by columns
// where `turned` (whichever index is contiguous stays so).
static int pack(Proj* P, dpdr_matrix& m, int64_t rows, int64_t cols, int64_t most_rows, int slot, bool turned,
                Copies& c)
{
    const int64_t ld = padded(turned ? rows : cols);
    // either way round
    const size_t most = std::max(size_t(most_rows) * size_t(padded(cols)), size_t(cols) * size_t(padded(most_rows)));
    const int rc = hold(P->packed[slot], most * 2, "projection operand copy");
    if (rc) return rc;
    int at = 0;
    while (at < c.n && c.slot[at] != slot) at++;
    if (at == c.n) c.n++;
    c.slot[at] = slot;
    const char* from = static_cast<const char*>(m.data);
    char* to = P->packed[slot];
    c.job[at] = turned ? Copies::Job{from, to, m.col_stride, m.row_stride, cols, rows, ld}
                       : Copies::Job{from, to, m.row_stride, m.col_stride, rows, cols, ld};
    m = turned ? dpdr_matrix{to, 1, ld} : dpdr_matrix{to, ld, 1};
    return DPDR_OK;
}

// The matrix as TMA can load it: as it lies where one stride is 1, the other a
// multiple of 8 that is no shorter than a row (column), and the address a
// multiple of 16 bytes; else a packed copy in the plan's slot.
static int loadable(Proj* P, dpdr_matrix& m, int64_t rows, int64_t cols, int64_t most_rows, int slot, Copies& c)
{
    if (rows == 0 || cols == 0) return DPDR_OK;
    const bool placed = reinterpret_cast<uintptr_t>(m.data) % 16 == 0;
    dpdr_matrix as = m;
    if (rows == 1) as.row_stride = padded(cols);   // never stepped over
    if (placed && (as.col_stride == 1 || cols == 1) && as.row_stride % 8 == 0 && as.row_stride >= cols &&
        as.row_stride < kFarthest) {
        as.col_stride = 1;
        m = as;
        return DPDR_OK;
    }
    as = m;
    if (cols == 1) as.col_stride = padded(rows);
    if (placed && (as.row_stride == 1 || rows == 1) && as.col_stride % 8 == 0 && as.col_stride >= rows &&
        as.col_stride < kFarthest) {
        as.row_stride = 1;
        m = as;
        return DPDR_OK;
    }
    return pack(P, m, rows, cols, most_rows, slot, m.row_stride == 1 && m.col_stride != 1, c);
}

// Few rows take row_kernel, which reads the weights once for up to 128 rows
// and splits the sum over k; so do products whose tiles of 128 x 128 (of a
// pair 64 x 128) are no more than two thirds of the SMs, most of which the 256 x
// 256 tiles of tile_kernel would leave idle.  us with row_kernel and
// tile_kernel, 4096 x 4096 weights: 64 rows 11.0 and 17.8, 256 rows 15.5 and 18.4,
// 384 rows (96 tiles) 17.0 and 18.6, 512 rows 20.2 and 18.6, 1024 rows 32.3 and
// 25.2; 1024 x 1024 weights: 1024 rows (64 tiles) 7.7 and 8.6, 2048 rows 10.3 and
// 9.0; a pair of 8192 x 4096: 128 rows 28.0 and 30.0, 192 rows 33.7 and 30.1.
static int product_launch(Proj* P, const Product& p, cudaStream_t s)
{
    const int64_t width = p.kind == kPair ? 64 : 128;
    const bool few = p.M <= 128 || 3 * ((p.M + 127) / 128) * ((p.N + width - 1) / width) <= 2 * P->num_sms;
    return p.kind != kTwin && few ? row_launch(P, p, s) : tile_launch(P, p, s);
}

// Whether a forward call goes to token_kernel as its operands lie
static bool for_token(int64_t rows, const dpdr_matrix& x, const dpdr_matrix& w0, const dpdr_matrix* w1)
{
    return rows == 1 && x.col_stride == 1 && w0.col_stride == 1 && (!w1 || w1->col_stride == 1);
}

// The forward product, or with slope the same product finished as dz (dg, du).
static int forward(Proj* P, int64_t rows, const dpdr_matrix& x, const dpdr_matrix& w0, const dpdr_matrix& w1,
                   const void* bias, const Epilogue& e, cudaStream_t s, bool token = false,
                   int64_t* sum_parts = nullptr)
{
    Product p;
    p.sum_parts = sum_parts;
    p.kind = P->gated ? kPair : kSingle;
    p.M = rows;
    p.N = P->n_out;
    p.K = P->n_in;
    p.a[0] = rows_of(x);
    p.b[0] = rows_of(w0);
    p.b[1] = rows_of(w1);
    p.e = e;
    p.e.bias = bias;
    return token ? token_launch(P, p, s) : product_launch(P, p, s);
}

// The operands as loadable matrices: x, each weight and dy, those that a call
// reads, the copies that this takes in one launch.  Both weights of a pair have
// to lie the same way (one tile layout); otherwise one is copied too.
struct Operands {
    dpdr_matrix x{}, w[2] = {}, dy{};
};

static int operands(Proj* P, int64_t rows, const dpdr_matrix* x, const dpdr_matrix* w0, const dpdr_matrix* w1,
                    const dpdr_matrix* dy, Operands& o, cudaStream_t s)
{
    int rc = DPDR_OK;
    Copies c;
    if (x) {
        o.x = *x;
        rc = loadable(P, o.x, rows, P->n_in, P->max_rows, 0, c);
    }
    const dpdr_matrix* w[2] = {w0, w1};
    for (int i = 0; i < 2 && !rc; i++) {
        if (!w[i]) continue;
        o.w[i] = *w[i];
        rc = loadable(P, o.w[i], P->n_out, P->n_in, P->n_out, 1 + i, c);
    }
    if (!rc && w0 && w1 && (o.w[0].col_stride == 1) != (o.w[1].col_stride == 1)) {
        // one lies by rows, the other by columns: the latter is copied by rows
        const int i = o.w[0].col_stride == 1 ? 1 : 0;
        o.w[i] = *w[i];
        rc = pack(P, o.w[i], P->n_out, P->n_in, P->n_out, 1 + i, false, c);
    }
    if (dy && !rc) {
        o.dy = *dy;
        rc = loadable(P, o.dy, rows, P->n_out, P->max_rows, 3, c);
    }
    if (!rc && c.n) rc = copies_launch(P, c, s);
    return rc;
}

struct Backward {
    const dpdr_matrix *x, *w0, *w1, *dy, *pre, *dx, *dw0, *dw1;
    const void* bias;
    void* dbias;
};

static int backward(Proj* P, int64_t rows, const Backward& c, cudaStream_t s)
{
    const int n = P->gated ? 2 : 1;
    const int64_t N = P->n_out, K = P->n_in;
    if (!c.dx && !c.dw0 && !c.dbias) return DPDR_OK;
    if (rows == 0) {
        const size_t qs = P->grad_f32 ? 4 : 2;
        cudaError_t e = cudaSuccess;
        for (const dpdr_matrix* d : {c.dw0, c.dw1})
            if (d && e == cudaSuccess)
                e = cudaMemset2DAsync(d->data, size_t(N > 1 ? d->row_stride : K) * qs, 0, size_t(K) * qs, size_t(N), s);
        if (c.dbias && e == cudaSuccess) e = cudaMemsetAsync(c.dbias, 0, size_t(N) * qs, s);
        return e == cudaSuccess ? DPDR_OK : cuda_fail_c(e, "zero gradients");
    }
    // dz as operands: dy itself where it already is (no activation, 16 bits)
    const bool as_is = !P->gated && P->act == DPDR_ACT_NONE && !P->out_f32;
    const int64_t ld = padded(N);
    const size_t dz_bytes = as_is ? 0 : upto256(size_t(P->max_rows) * size_t(ld) * 2);
    const bool again = !as_is && !c.pre && (P->gated || P->act != DPDR_ACT_NONE);
    // column sums for the bias: as many rows of them as max_rows rows may come in,
    // and where those are too many to join at once, their own column sums
    const int64_t most = std::max<int64_t>(P->act == DPDR_ACT_NONE ? 0 : product_sum_parts(P->max_rows, P->num_sms),
                                           column_sum_parts(P->max_rows));
    const size_t sum_bytes = P->gated ? 0 : upto256(size_t(most) * size_t(N) * 4);
    const size_t more_bytes = P->gated || most <= kJoined ? 0 : upto256(size_t(column_sum_parts(most)) * size_t(N) * 4);
    int rc = DPDR_OK;
    if (!as_is || c.dbias) rc = hold(P->scratch, n * dz_bytes + sum_bytes + more_bytes, "projection scratch");
    if (rc) return rc;
    Operands o;
    const bool need_w = again || c.dx;
    const bool products = c.dx || c.dw0;
    rc = operands(P, rows, again || c.dw0 ? c.x : nullptr, need_w ? c.w0 : nullptr, need_w ? c.w1 : nullptr,
                  as_is && products ? c.dy : nullptr, o, s);
    if (rc) return rc;
    dpdr_matrix dz[2] = {{P->scratch, ld, 1}, {P->scratch + dz_bytes, ld, 1}};
    float* sums = reinterpret_cast<float*>(P->scratch + n * dz_bytes);
    int64_t parts = column_sum_parts(rows);
    Epilogue e = epilogue_of(P);
    if (as_is) {
        dz[0] = products ? o.dy : *c.dy;
    } else {
        e.finish = kSlope;
        set_other(e, *c.dy, P->out_f32);
        e.out = static_cast<char*>(dz[0].data);
        e.out2 = static_cast<char*>(dz[1].data);
        e.out_rs = e.out2_rs = ld;
        if (again) {
            if (c.dbias) e.sums = sums;
            rc = forward(P, rows, o.x, o.w[0], o.w[1], c.bias, e, s, false, &parts);
        } else {
            if (c.pre) {   // without: no activation, dy is rounded to the operand type
                e.pre = static_cast<float*>(c.pre->data);
                e.pre_rs = c.pre->row_stride;
                e.pre_up = N;
            }
            if (!products) e.out = e.out2 = nullptr;
            rc = slope_launch(e, P->gated, rows, N, c.dbias ? sums : nullptr, s);
        }
        if (rc) return rc;
    }
    if (c.dx) {
        Product p;
        p.kind = P->gated ? kChain : kSingle;
        p.M = rows;
        p.N = K;
        p.K = N;
        for (int i = 0; i < n; i++) {
            p.a[i] = rows_of(dz[i]);
            p.b[i] = cols_of(o.w[i]);
        }
        p.e.half = P->half;
        p.e.out = static_cast<char*>(c.dx->data);
        p.e.out_rs = c.dx->row_stride;
        p.e.out_f32 = P->grad_f32;
        rc = product_launch(P, p, s);
        if (rc) return rc;
    }
    if (c.dw0) {
        Product p;
        p.kind = P->gated ? kTwin : kSingle;
        p.M = N;
        p.N = K;
        p.K = rows;
        for (int i = 0; i < n; i++) p.a[i] = cols_of(dz[i]);
        p.b[0] = cols_of(o.x);
        p.e.half = P->half;
        p.e.out = static_cast<char*>(c.dw0->data);
        p.e.out_rs = c.dw0->row_stride;
        p.e.out_f32 = P->grad_f32;
        if (P->gated) {
            p.e.out2 = static_cast<char*>(c.dw1->data);
            p.e.out2_rs = c.dw1->row_stride;
        }
        rc = product_launch(P, p, s);
        if (rc) return rc;
    }
    if (c.dbias) {
        auto sum_columns = [&](const dpdr_matrix& of, int f32, int64_t height, float* into) {
            Epilogue d = epilogue_of(P);
            d.act = DPDR_ACT_NONE;
            set_other(d, of, f32);
            return slope_launch(d, false, height, N, into, s);
        };
        if (as_is) rc = sum_columns(dz[0], 0, rows, sums);
        if (!rc && parts > kJoined) {
            float* more = sums + sum_bytes / 4;
            rc = sum_columns(dpdr_matrix{sums, N, 1}, 1, parts, more);
            sums = more;
            parts = column_sum_parts(parts);
        }
        if (!rc) rc = join_launch(sums, int(parts), N, c.dbias, P->grad_f32, P->half, s);
    }
    return rc;
}

}  // namespace proj
}  // namespace dpdr

using namespace dpdr;
using namespace dpdr::proj;

static Proj* plan_of(dpdr_proj_t h) { return reinterpret_cast<Proj*>(h); }

extern "C" dpdr_proj_t dpdr_linear_plan(int64_t max_rows, int64_t n_in, int64_t n_out, dpdr_dtype operands,
                                        dpdr_dtype result, dpdr_dtype gradients, dpdr_act act)
{
    return reinterpret_cast<dpdr_proj_t>(
        make(false, max_rows, n_in, n_out, operands, result, gradients, act, "dpdr_linear_plan"));
}

extern "C" dpdr_proj_t dpdr_gated_plan(int64_t max_rows, int64_t n_in, int64_t n_hidden, dpdr_dtype operands,
                                       dpdr_dtype result, dpdr_dtype gradients, dpdr_act act)
{
    return reinterpret_cast<dpdr_proj_t>(
        make(true, max_rows, n_in, n_hidden, operands, result, gradients, act, "dpdr_gated_plan"));
}

extern "C" int dpdr_linear(dpdr_proj_t h, int64_t rows, const dpdr_matrix* x, const dpdr_matrix* w, const void* bias,
                           const dpdr_matrix* residual, const dpdr_matrix* y, const dpdr_matrix* pre,
                           dpdr_stream_t stream)
{
    Proj* P = plan_of(h);
    int rc = check_plan(P, false, rows, "dpdr_linear");
    if (rc) return rc;
    const int es = P->out_f32 ? 4 : 2;
    Args a{"dpdr_linear"};
    a.input("x", x, rows, P->n_in, 2);
    a.input("w", w, P->n_out, P->n_in, 2);
    if (bias) a.vector("bias", bias, P->n_out, 2, false);
    // y may be the residual itself: each element is read by the thread that
    // then writes it
    const bool same = residual && y && residual->data == y->data && (rows < 2 || residual->row_stride == y->row_stride) &&
                      (P->n_out < 2 || residual->col_stride == y->col_stride);
    if (residual && !same) a.input("residual", residual, rows, P->n_out, es);
    a.output("y", y, rows, P->n_out, es);
    if (pre) a.output("pre", pre, rows, P->n_out, 4);
    if (a.done()) return a.rc;
    if (rows == 0) return DPDR_OK;
    Epilogue e = epilogue_of(P);
    if (residual) set_other(e, *residual, P->out_f32);
    e.out = static_cast<char*>(y->data);
    e.out_rs = y->row_stride;
    e.out_f32 = P->out_f32;
    if (pre) {
        e.pre = static_cast<float*>(pre->data);
        e.pre_rs = pre->row_stride;
    }
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (for_token(rows, *x, *w, nullptr)) return forward(P, rows, *x, *w, dpdr_matrix{}, bias, e, s, true);
    Operands o;
    rc = operands(P, rows, x, w, nullptr, nullptr, o, s);
    return rc ? rc : forward(P, rows, o.x, o.w[0], o.w[1], bias, e, s);
}

extern "C" int dpdr_gated(dpdr_proj_t h, int64_t rows, const dpdr_matrix* x, const dpdr_matrix* w_gate,
                          const dpdr_matrix* w_up, const dpdr_matrix* out, const dpdr_matrix* pre, dpdr_stream_t stream)
{
    Proj* P = plan_of(h);
    int rc = check_plan(P, true, rows, "dpdr_gated");
    if (rc) return rc;
    Args a{"dpdr_gated"};
    a.input("x", x, rows, P->n_in, 2);
    a.input("w_gate", w_gate, P->n_out, P->n_in, 2);
    a.input("w_up", w_up, P->n_out, P->n_in, 2);
    a.output("h", out, rows, P->n_out, P->out_f32 ? 4 : 2);
    if (pre) a.output("pre", pre, rows, 2 * P->n_out, 4);
    if (a.done()) return a.rc;
    if (rows == 0) return DPDR_OK;
    Epilogue e = epilogue_of(P);
    e.out = static_cast<char*>(out->data);
    e.out_rs = out->row_stride;
    e.out_f32 = P->out_f32;
    if (pre) {
        e.pre = static_cast<float*>(pre->data);
        e.pre_rs = pre->row_stride;
        e.pre_up = P->n_out;
    }
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (for_token(rows, *x, *w_gate, w_up)) return forward(P, rows, *x, *w_gate, *w_up, nullptr, e, s, true);
    Operands o;
    rc = operands(P, rows, x, w_gate, w_up, nullptr, o, s);
    return rc ? rc : forward(P, rows, o.x, o.w[0], o.w[1], nullptr, e, s);
}

extern "C" int dpdr_linear_backward(dpdr_proj_t h, int64_t rows, const dpdr_matrix* x, const dpdr_matrix* w,
                                    const void* bias, const dpdr_matrix* dy, const dpdr_matrix* pre,
                                    const dpdr_matrix* dx, const dpdr_matrix* dw, void* dbias, dpdr_stream_t stream)
{
    Proj* P = plan_of(h);
    int rc = check_plan(P, false, rows, "dpdr_linear_backward");
    if (rc) return rc;
    const int qs = P->grad_f32 ? 4 : 2;
    Args a{"dpdr_linear_backward"};
    a.input("x", x, rows, P->n_in, 2);
    a.input("w", w, P->n_out, P->n_in, 2);
    if (bias) a.vector("bias", bias, P->n_out, 2, false);
    a.input("dy", dy, rows, P->n_out, P->out_f32 ? 4 : 2);
    if (pre) a.input("pre", pre, rows, P->n_out, 4);
    if (pre && P->n_out > 1 && pre->col_stride != 1) a.refuse("pre", "needs col_stride 1");
    if (dx) a.output("dx", dx, rows, P->n_in, qs);
    if (dw) a.output("dw", dw, P->n_out, P->n_in, qs);
    if (dbias) a.vector("dbias", dbias, P->n_out, qs, true);
    if (a.done()) return a.rc;
    return backward(P, rows, Backward{x, w, nullptr, dy, pre, dx, dw, nullptr, bias, dbias},
                    reinterpret_cast<cudaStream_t>(stream));
}

extern "C" int dpdr_gated_backward(dpdr_proj_t h, int64_t rows, const dpdr_matrix* x, const dpdr_matrix* w_gate,
                                   const dpdr_matrix* w_up, const dpdr_matrix* dh, const dpdr_matrix* pre,
                                   const dpdr_matrix* dx, const dpdr_matrix* dw_gate, const dpdr_matrix* dw_up,
                                   dpdr_stream_t stream)
{
    Proj* P = plan_of(h);
    int rc = check_plan(P, true, rows, "dpdr_gated_backward");
    if (rc) return rc;
    const int qs = P->grad_f32 ? 4 : 2;
    Args a{"dpdr_gated_backward"};
    a.input("x", x, rows, P->n_in, 2);
    a.input("w_gate", w_gate, P->n_out, P->n_in, 2);
    a.input("w_up", w_up, P->n_out, P->n_in, 2);
    a.input("dh", dh, rows, P->n_out, P->out_f32 ? 4 : 2);
    if (pre) a.input("pre", pre, rows, 2 * P->n_out, 4);
    if (pre && pre->col_stride != 1) a.refuse("pre", "needs col_stride 1");
    if (dx) a.output("dx", dx, rows, P->n_in, qs);
    if (!dw_gate != !dw_up) a.refuse("dw_gate and dw_up", "go together");
    if (dw_gate) a.output("dw_gate", dw_gate, P->n_out, P->n_in, qs);
    if (dw_up) a.output("dw_up", dw_up, P->n_out, P->n_in, qs);
    if (a.done()) return a.rc;
    return backward(P, rows, Backward{x, w_gate, w_up, dh, pre, dx, dw_gate, dw_up, nullptr, nullptr},
                    reinterpret_cast<cudaStream_t>(stream));
}

extern "C" int dpdr_proj_sync(dpdr_proj_t h, dpdr_stream_t stream)
{
    Proj* P = plan_of(h);
    if (!P) return refuse("dpdr_proj_sync", "NULL plan");
    cudaError_t e = cudaStreamSynchronize(reinterpret_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail_c(e, "stream synchronize");
    volatile uint32_t* err = P->err;   // the stream has passed its writers
    if (*err == 0) return DPDR_OK;
    *err = 0;
    return fail_c(DPDR_ERR_TIMEOUT, "projection: a bounded wait expired");
}

extern "C" void dpdr_proj_destroy(dpdr_proj_t h)
{
    Proj* P = plan_of(h);
    if (!P) return;
    cudaFree(P->scratch);
    for (char* p : P->packed) cudaFree(p);
    g_errors.give(P->err);
    delete P;
}
