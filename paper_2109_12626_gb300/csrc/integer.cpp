// integer.cpp -- host side of the products of 8-bit integers: plan, argument
// checks, scratch, and which kernels a call takes.
#include <algorithm>
#include <new>

#include "args.h"
#include "integer.h"

namespace dpdr {
namespace integer {

namespace {

// the plan behind dpdr_integer_t
struct Integer {
    // its device, its error word and the tiles' kernels
    dpdr_proj_t tiles = nullptr;
    int64_t max_rows = 0, n_in = 0, n_out = 0;
    int out_f32 = 0, half = 0;
    char* x_copy = nullptr;     // x of few rows, padded
    int32_t* parts = nullptr;   // of their sums, and counters
    char* wide[2] = {};         // x and w in 16 bits
    bool set[3][2] = {}, wide_set[2] = {};   // kernels' attributes set
    proj::Proj* base() const { return reinterpret_cast<proj::Proj*>(tiles); }
};

int64_t upto(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }

// Device memory of the plan's, made once
template <typename T>
int hold(T*& at, int64_t bytes, const char* what)
{
    if (at) return DPDR_OK;
    const cudaError_t e = cudaMalloc(reinterpret_cast<void**>(&at), size_t(bytes));
    return e == cudaSuccess ? DPDR_OK : cuda_fail_c(e, what);
}

int few(Integer* P, int64_t rows, const dpdr_matrix& x, const dpdr_matrix& w, const Finish& f, cudaStream_t s)
{
    const int num_sms = P->base()->num_sms;
    const int64_t pad = upto(P->n_in, kRowsPad), most = std::min<int64_t>(P->max_rows, kFewRows);
    Rows r{};
    r.rows = int(rows);
    r.k = int(P->n_in);
    r.n = P->n_out;
    r.w = static_cast<const char*>(w.data);
    r.w_rs = P->n_out > 1 ? w.row_stride : P->n_in;
    r.f = f;
    r.set = P->set;
    const bool token = for_tokens(r);
    r.parts = P->parts;
    r.count = reinterpret_cast<uint32_t*>(P->parts + parts_ints(num_sms));
    // x as it lies where its rows are whole pieces at multiples of 16 bytes, and wherever
    // they are for tokens and weights at any address
    const bool at_16 = reinterpret_cast<uintptr_t>(x.data) % 16 == 0 && (rows == 1 || x.row_stride % 16 == 0);
    if (x.col_stride == 1 && (P->n_in == pad || token) && (at_16 || (token && !aligned_weights(r)))) {
        r.x = static_cast<const char*>(x.data);
        r.x_rs = x.row_stride;
    } else {
        int rc = hold(P->x_copy, most * pad, "integer product: operand copy");
        if (rc) return rc;
        Relay c;
        c.job[c.n++] = {static_cast<const int8_t*>(x.data), P->x_copy, x.row_stride, x.col_stride, rows, P->n_in,
                        pad, pad};
        rc = relay_launch(c, num_sms, s);
        if (rc) return rc;
        r.x = P->x_copy;
        r.x_rs = pad;
    }
    return rows_launch(r, num_sms, s);
}

int some(Integer* P, int64_t rows, const dpdr_matrix& x, const dpdr_matrix& w, const Finish& f, cudaStream_t s)
{
    Wide q;
    q.rows = int(rows);
    q.k = int(P->n_in);
    q.n = P->n_out;
    q.x = static_cast<const char*>(x.data);
    q.x_rs = x.row_stride;
    q.w = static_cast<const char*>(w.data);
    q.w_rs = w.row_stride;
    q.f = f;
    q.set = P->wide_set;
    q.err = P->base()->err;
    return wide_launch(q, P->base()->num_sms, s);
}

int many(Integer* P, int64_t rows, const dpdr_matrix& x, const dpdr_matrix& w, const Finish& f, cudaStream_t s)
{
    proj::Proj* B = P->base();
    const int64_t ld = upto(P->n_in, 8);
    int rc = hold(P->wide[0], P->max_rows * ld * 2, "integer product: widened x");
    if (!rc) rc = hold(P->wide[1], P->n_out * ld * 2, "integer product: widened w");
    if (rc) return rc;
    Relay c;
    c.wide = 1 + P->half;
    const int64_t k = P->n_in;
    c.job[c.n++] = {static_cast<const int8_t*>(x.data), P->wide[0], x.row_stride, x.col_stride, rows, k, ld, k};
    c.job[c.n++] = {static_cast<const int8_t*>(w.data), P->wide[1], w.row_stride, w.col_stride, P->n_out, k, ld, k};
    rc = relay_launch(c, B->num_sms, s);
    if (rc) return rc;
    proj::Product p;
    p.kind = proj::kSingle;
    p.M = rows;
    p.N = P->n_out;
    p.K = P->n_in;
    p.a[0] = {P->wide[0], ld, 1};
    p.b[0] = {P->wide[1], ld, 1};
    p.e.finish = proj::kScaled;
    p.e.half = P->half;
    p.e.other = f.residual;
    p.e.other_rs = f.residual_rs;
    p.e.other_cs = f.residual_cs;
    p.e.other_f32 = P->out_f32;
    p.e.out = f.y;
    p.e.out_rs = f.y_rs;
    p.e.out_f32 = P->out_f32;
    p.e.row_scale = f.x_scale;
    p.e.col_scale = f.w_scale;
    p.e.bias32 = f.bias;
    return proj::tile_launch(B, p, s);
}

}  // namespace

}  // namespace integer
}  // namespace dpdr

using namespace dpdr;
using namespace dpdr::integer;
using dpdr::proj::Args;
using dpdr::proj::refuse;

static Integer* plan_of(dpdr_integer_t h) { return reinterpret_cast<Integer*>(h); }

extern "C" int dpdr_quantise(int64_t rows, int64_t n, dpdr_dtype dtype, const dpdr_matrix* x, const dpdr_matrix* q,
                             float* scale, dpdr_stream_t stream)
{
    const char* who = "dpdr_quantise";
    const int64_t most = (int64_t(1) << 31) - 1;
    if (rows < 0 || rows > most || n < 1 || n > most) return refuse(who, "need 0 <= rows and 1 <= n, below 2^31");
    if (dtype != DPDR_BFLOAT16 && dtype != DPDR_FLOAT16 && dtype != DPDR_FLOAT32)
        return refuse(who, "x is bfloat16, float16 or float32");
    Args a{who};
    a.input("x", x, rows, n, dtype == DPDR_FLOAT32 ? 4 : 2);
    a.output("q", q, rows, n, 1);
    a.vector("scale", scale, rows, 4, true);
    if (a.done()) return a.rc;
    if (rows == 0) return DPDR_OK;
    return quantise_launch(dtype, rows, n, *x, *q, scale, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" dpdr_integer_t dpdr_integer_plan(int64_t max_rows, int64_t n_in, int64_t n_out, dpdr_dtype result)
{
    const char* who = "dpdr_integer_plan";
    auto bad = [&](const char* what) {
        refuse(who, what);
        return dpdr_integer_t(nullptr);
    };
    const int64_t most = (int64_t(1) << 31) - 1;
    if (max_rows < 0 || max_rows > most || n_out < 1 || n_out > most)
        return bad("need 0 <= max_rows and 1 <= n_out, below 2^31");
    if (n_in < 1 || n_in > kMostSummed) return bad("need 1 <= n_in < 2^17, so that sums stay below 2^31");
    if (result != DPDR_BFLOAT16 && result != DPDR_FLOAT16 && result != DPDR_FLOAT32)
        return bad("the result is bfloat16, float16 or float32");
    Integer* P = new (std::nothrow) Integer;
    if (!P) {
        fail_c(DPDR_ERR_OOM, "integer plan: host allocation");
        return nullptr;
    }
    P->half = result == DPDR_FLOAT16;
    P->out_f32 = result == DPDR_FLOAT32;
    const dpdr_dtype wide = P->half ? DPDR_FLOAT16 : DPDR_BFLOAT16;
    P->max_rows = max_rows;
    P->n_in = n_in;
    P->n_out = n_out;
    P->tiles = dpdr_linear_plan(max_rows, n_in, n_out, wide, result, wide, DPDR_ACT_NONE);
    if (!P->tiles) {
        delete P;
        return nullptr;
    }
    // counters at zero before any call: a call's own clearing, captured, would wait for its replay
    const int num_sms = P->base()->num_sms;
    const int64_t ints = parts_ints(num_sms), counters = 2 * num_sms * 4;
    int rc = hold(P->parts, ints * 4 + counters, who);
    if (!rc) {
        cudaError_t e = cudaMemset(P->parts + ints, 0, size_t(counters));
        if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
        if (e != cudaSuccess) rc = cuda_fail_c(e, who);
    }
    if (rc) {
        dpdr_integer_destroy(reinterpret_cast<dpdr_integer_t>(P));
        return nullptr;
    }
    return reinterpret_cast<dpdr_integer_t>(P);
}

extern "C" int dpdr_integer_linear(dpdr_integer_t h, int64_t rows, const dpdr_matrix* x, const float* x_scale,
                                   const dpdr_matrix* w, const float* w_scale, const float* bias,
                                   const dpdr_matrix* residual, const dpdr_matrix* y, dpdr_stream_t stream)
{
    const char* who = "dpdr_integer_linear";
    Integer* P = plan_of(h);
    if (!P) return refuse(who, "NULL plan");
    if (rows < 0 || rows > P->max_rows) return refuse(who, "need 0 <= rows <= max_rows");
    int current = -1;
    const cudaError_t e = cudaGetDevice(&current);
    if (e != cudaSuccess) return cuda_fail_c(e, who);
    if (current != P->base()->device) return refuse(who, "the plan's device is not the current one");
    const int es = P->out_f32 ? 4 : 2;
    Args a{who};
    a.input("x", x, rows, P->n_in, 1);
    a.vector("x_scale", x_scale, rows, 4, false);
    a.input("w", w, P->n_out, P->n_in, 1);
    a.vector("w_scale", w_scale, P->n_out, 4, false);
    if (bias) a.vector("bias", bias, P->n_out, 4, false);
    // y may be the residual itself: each element is read by the thread that
    // then writes it
    const bool same = residual && y && residual->data == y->data &&
                      (rows < 2 || residual->row_stride == y->row_stride) &&
                      (P->n_out < 2 || residual->col_stride == y->col_stride);
    if (residual && !same) a.input("residual", residual, rows, P->n_out, es);
    a.output("y", y, rows, P->n_out, es);
    if (a.done()) return a.rc;
    if (rows == 0) return DPDR_OK;
    Finish f{};
    f.x_scale = x_scale;
    f.w_scale = w_scale;
    f.bias = bias;
    if (residual) {
        f.residual = static_cast<const char*>(residual->data);
        f.residual_rs = residual->row_stride;
        f.residual_cs = residual->col_stride;
    }
    f.y = static_cast<char*>(y->data);
    f.y_rs = y->row_stride;
    f.out_f32 = P->out_f32;
    f.half = P->half;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const bool in_place = w->col_stride == 1 || P->n_in == 1;
    if (rows > kStreamRows && in_place && (x->col_stride == 1 || P->n_in == 1) &&
        wide_takes(rows, P->n_out, P->n_in, P->base()->num_sms))
        return some(P, rows, *x, *w, f, s);
    return rows <= kFewRows && in_place ? few(P, rows, *x, *w, f, s) : many(P, rows, *x, *w, f, s);
}

extern "C" int dpdr_integer_sync(dpdr_integer_t h, dpdr_stream_t stream)
{
    Integer* P = plan_of(h);
    if (!P) return refuse("dpdr_integer_sync", "NULL plan");
    return dpdr_proj_sync(P->tiles, stream);
}

extern "C" void dpdr_integer_destroy(dpdr_integer_t h)
{
    Integer* P = plan_of(h);
    if (!P) return;
    dpdr_proj_destroy(P->tiles);
    cudaFree(P->x_copy);
    cudaFree(P->parts);
    for (char* p : P->wide) cudaFree(p);
    delete P;
}
