// experts.cpp -- host side of a layer of experts: plan, argument checks.
#include <algorithm>
#include <new>

#include "args.h"
#include "experts.h"

namespace dpdr {
namespace experts {

namespace {

// the plan behind dpdr_experts_t
struct Experts {
    Layer l;            // sizes, types and scratch of every call; rows is max_rows
    int device = 0, num_sms = 0;
    char* scratch = nullptr;
};

int64_t upto(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }

}  // namespace

}  // namespace experts
}  // namespace dpdr

using namespace dpdr;
using namespace dpdr::experts;
using dpdr::proj::Args;
using dpdr::proj::refuse;

static Experts* plan_of(dpdr_experts_t h) { return reinterpret_cast<Experts*>(h); }

extern "C" dpdr_experts_t dpdr_experts_plan(int64_t max_rows, int64_t n_model, int64_t n_hidden, int experts, int top,
                                            int first, int local, dpdr_dtype operands, dpdr_dtype weights,
                                            dpdr_dtype result, dpdr_act act, int normalise)
{
    const char* who = "dpdr_experts_plan";
    auto bad = [&](const char* what) {
        refuse(who, what);
        return dpdr_experts_t(nullptr);
    };
    if (max_rows < 1 || max_rows > kMostRows) return bad("need 1 <= max_rows <= 64");
    if (n_model < 1 || n_model > kMostSize || n_hidden < 1 || n_hidden > kMostSize)
        return bad("need 1 <= n_model, n_hidden <= 2^20");
    if (experts < 1 || experts > kMostExperts || top < 1 || top > kMostTop || top > experts)
        return bad("need 1 <= top <= 16 and top <= experts <= 512");
    if (first < 0 || local < 1 || first > experts - local)
        return bad("need 0 <= first, 1 <= local, first + local <= experts");
    if (operands != DPDR_BFLOAT16 && operands != DPDR_FLOAT16) return bad("operands are bfloat16 or float16");
    if (weights != operands && weights != DPDR_INT8) return bad("weights have the operands' type or int8");
    if (result != operands && result != DPDR_FLOAT32) return bad("the result has the operands' type or float32");
    if (act < DPDR_ACT_NONE || act > DPDR_ACT_SIGMOID) return bad("unknown activation");
    // pieces of 64 bytes that the warps share, counted in 32 bits
    const int64_t pairs_most = max_rows * top, entries = std::min<int64_t>(local, pairs_most) + pairs_most / 8;
    if (entries * ((n_hidden + 15) / 16) * (n_model / 32 + 1) > (int64_t(1) << 30) ||
        entries * ((n_model + 31) / 32) * (n_hidden / 32 + 1) > (int64_t(1) << 30))
        return bad("more than 2^30 pieces of weights");
    Experts* P = new (std::nothrow) Experts;
    if (!P) {
        fail_c(DPDR_ERR_OOM, "experts plan: host allocation");
        return nullptr;
    }
    Layer& l = P->l;
    l = Layer{};
    l.rows = int(max_rows);
    l.top = top;
    l.total = experts;
    l.first = first;
    l.local = local;
    l.d = int(n_model);
    l.h = int(n_hidden);
    l.half = operands == DPDR_FLOAT16;
    l.w_int8 = weights == DPDR_INT8;
    l.d_pad = upto(n_model, l.w_int8 ? kPad8 : kPad);
    l.h_pad = upto(n_hidden, kPad);
    l.act = act;
    l.terms = l.half && !l.w_int8 ? 1 : 3;
    l.pairs = l.rows * top;
    l.normalise = normalise != 0;
    l.out_f32 = result == DPDR_FLOAT32;
    cudaError_t e = cudaGetDevice(&P->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&P->num_sms, cudaDevAttrMultiProcessorCount, P->device);
    int rc = e == cudaSuccess ? product_ctas(l, P->num_sms) : cuda_fail_c(e, who);
    if (!rc) {
        const int64_t pairs = max_rows * top;
        const int64_t warps = 8 * int64_t(l.ctas);
        // two places a warp, of 32 rows by as many columns as an entry may have
        const int64_t places = 2 * warps * 32 * (max_rows <= 8 ? 8 : max_rows <= 16 ? 16 : 32);
        int64_t size = 0;
        auto take = [&](int64_t bytes) {
            const int64_t at = size;
            size += upto(bytes, 256);
            return at;
        };
        const int64_t logits = take(max_rows * experts * 4), x = take(max_rows * l.d_pad * 2),
                      hidden = take(pairs * l.h_pad * (l.terms == 1 ? 4 : 2 * l.terms)),
                      some = take(places * 4),
                      z = take(max_rows <= kWholeRows ? 0 : pairs * n_model * 4), expert = take(pairs * 4), shares = take(pairs * 4),
                      scores = take(max_rows * 4),
                      up = take(warps * 4), down = take(warps * 4);
        e = cudaMalloc(&P->scratch, size_t(size));
        // counters at zero, and what lies behind the rows of x and of hidden values
        if (e == cudaSuccess) e = cudaMemset(P->scratch, 0, size_t(size));
        if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
        if (e != cudaSuccess) rc = cuda_fail_c(e, who);
        l.logits = reinterpret_cast<float*>(P->scratch + logits);
        l.x_copy = P->scratch + x;
        l.hidden = P->scratch + hidden;
        l.parts = reinterpret_cast<float*>(P->scratch + some);
        l.z = reinterpret_cast<float*>(P->scratch + z);
        l.expert = reinterpret_cast<int32_t*>(P->scratch + expert);
        l.shares = reinterpret_cast<float*>(P->scratch + shares);
        l.score_count = reinterpret_cast<uint32_t*>(P->scratch + scores);
        l.up_count = reinterpret_cast<uint32_t*>(P->scratch + up);
        l.down_count = reinterpret_cast<uint32_t*>(P->scratch + down);
    }
    if (rc) {
        cudaFree(P->scratch);
        delete P;
        return nullptr;
    }
    return reinterpret_cast<dpdr_experts_t>(P);
}

extern "C" int dpdr_experts(dpdr_experts_t h, int64_t rows, const dpdr_matrix* x, const dpdr_matrix* router,
                            const dpdr_matrices* w_gate, const dpdr_matrices* w_up, const dpdr_matrices* w_down,
                            const float* gate_scale, const float* up_scale, const float* down_scale,
                            const dpdr_matrix* y, int32_t* chosen, float* share, dpdr_stream_t stream)
{
    const char* who = "dpdr_experts";
    Experts* P = plan_of(h);
    if (!P) return refuse(who, "NULL plan");
    Layer l = P->l;
    if (rows < 0 || rows > l.rows) return refuse(who, "need 0 <= rows <= max_rows");
    int current = -1;
    const cudaError_t e = cudaGetDevice(&current);
    if (e != cudaSuccess) return cuda_fail_c(e, who);
    if (current != P->device) return refuse(who, "the plan's device is not the current one");
    const int es = l.w_int8 ? 1 : 2;
    Args a{who};
    a.input("x", x, rows, l.d, 2);
    a.input("router", router, l.total, l.d, 2);
    a.stack("w_gate", w_gate, l.local, l.h, l.d, es);
    a.stack("w_up", w_up, l.local, l.h, l.d, es);
    a.stack("w_down", w_down, l.local, l.d, l.h, es);
    const float* scale[3] = {gate_scale, up_scale, down_scale};
    const char* names[3] = {"gate_scale", "up_scale", "down_scale"};
    for (int i = 0; i < 3; i++) {
        if (l.w_int8) a.vector(names[i], scale[i], int64_t(l.local) * (i < 2 ? l.h : l.d), 4, false);
        else if (scale[i]) a.refuse(names[i], "goes with 8-bit weights");
    }
    a.output("y", y, rows, l.d, l.out_f32 ? 4 : 2);
    if (chosen) a.vector("chosen", chosen, rows * l.top, 4, true);
    if (share) a.vector("share", share, rows * l.top, 4, true);
    if (a.done()) return a.rc;
    if (rows == 0) return DPDR_OK;
    l.rows = int(rows);
    l.x = static_cast<const char*>(x->data);
    l.x_rs = x->row_stride;
    l.x_cs = x->col_stride;
    l.router = static_cast<const char*>(router->data);
    l.router_rs = router->row_stride;
    l.router_cs = router->col_stride;
    l.w[0] = *w_gate;
    l.w[1] = *w_up;
    l.w[2] = *w_down;
    for (int i = 0; i < 3; i++) l.scale[i] = scale[i];
    l.y = static_cast<char*>(y->data);
    l.y_rs = y->row_stride;
    l.chosen = chosen;
    l.share = share;
    return launch(l, P->num_sms, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" int dpdr_experts_sync(dpdr_experts_t h, dpdr_stream_t stream)
{
    if (!h) return refuse("dpdr_experts_sync", "NULL plan");
    const cudaError_t e = cudaStreamSynchronize(reinterpret_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? DPDR_OK : cuda_fail_c(e, "stream synchronize");
}

extern "C" void dpdr_experts_destroy(dpdr_experts_t h)
{
    Experts* P = plan_of(h);
    if (!P) return;
    cudaFree(P->scratch);
    delete P;
}
