// serving_fake.cpp -- the host code of the 8-bit products and the experts
// (integer.cpp, experts.cpp) over the CUDA runtime of proj_fake.cpp, which keeps
// books, with kernels that only check the places that they get (test
// infrastructure only).
#include "proj_fake.cpp"

#include "experts.h"
#include "integer.h"

namespace {

long streamed = 0, widened = 0, tiled = 0, layers = 0, copies = 0;
int ctas_an_sm = 2;

}  // namespace

extern "C" {
cudaError_t cudaMemset(void*, int, size_t) { return cudaSuccess; }
}

namespace dpdr {
namespace integer {
int rows_launch(const Rows& r, int num_sms, cudaStream_t)
{
    B.launches++;
    streamed++;
    const bool aligned = reinterpret_cast<uintptr_t>(r.w) % 16 == 0 && (r.n == 1 || r.w_rs % 16 == 0);
    const bool token = aligned ? r.rows <= 4 : r.rows <= 2 && r.n * r.k <= 1 << 25;
    if (r.rows < 1 || r.rows > kFewRows) wrong("rows", nullptr, r.rows);
    // whole pieces of 64 values, but for up to four rows
    holds("x", r.x, size_t(r.rows - 1) * r.x_rs + (token ? r.k : (r.k + 63) / 64 * 64));
    if ((aligned || !token) && (reinterpret_cast<uintptr_t>(r.x) % 16 || (r.rows > 1 && r.x_rs % 16))) wrong("x at", r.x, 0);
    if (token) return DPDR_OK;
    if (!r.parts || !r.count) wrong("no parts", nullptr, 0);
    holds("parts", r.parts, size_t(parts_ints(num_sms)) * 4);
    holds("counters", r.count, size_t(2 * num_sms) * 4);
    if (reinterpret_cast<char*>(r.count) < reinterpret_cast<char*>(r.parts + parts_ints(num_sms)))
        wrong("counters over parts", r.count, 0);
    return DPDR_OK;
}
bool wide_takes(int64_t rows, int64_t n, int64_t, int num_sms) { return (rows + 127) / 128 * ((n + 127) / 128) <= num_sms / 2; }
int wide_launch(const Wide&, int, cudaStream_t)
{
    B.launches++;
    widened++;
    return DPDR_OK;
}
int relay_launch(const Relay& r, int, cudaStream_t)
{
    B.launches++;
    copies++;
    for (int i = 0; i < r.n; i++) {
        const auto& j = r.job[i];
        // written by 16 values (of 16-bit ones, eight where the row ends there)
        rows_hold("copy", j.dst, j.ld, j.rows, r.wide ? j.ld : j.to, r.wide ? 2 : 1);
        if (r.wide ? j.ld % 8 : j.to % 16 || j.to > j.ld) wrong("row of a copy", j.dst, j.ld);
    }
    return DPDR_OK;
}
int quantise_launch(int, int64_t, int64_t, const dpdr_matrix&, const dpdr_matrix&, float*, cudaStream_t)
{
    B.launches++;
    return DPDR_OK;
}
}  // namespace integer
namespace experts {
int product_ctas(Layer& l, int num_sms)
{
    l.ctas = ctas_an_sm * num_sms;
    return DPDR_OK;
}
int launch(const Layer& l, int, cudaStream_t)
{
    B.launches++;
    layers++;
    const int64_t pairs = int64_t(l.rows) * l.top, warps = 8 * int64_t(l.ctas);
    const int64_t columns = l.rows <= 8 ? 8 : l.rows <= 16 ? 16 : 32;
    if (pairs > l.pairs) wrong("pairs", nullptr, pairs);
    holds("scores", l.logits, size_t(l.rows) * l.total * 4);
    holds("x", l.x_copy, size_t(l.rows) * l.d_pad * 2);
    holds("hidden", l.hidden, size_t(l.terms == 1 ? pairs * l.h_pad * 4 : ((l.terms - 1) * int64_t(l.pairs) + pairs) * l.h_pad * 2));
    holds("parts", l.parts, size_t(2 * warps * 32 * columns) * 4);
    if (l.rows > kWholeRows) holds("results", l.z, size_t(pairs) * l.d * 4);
    holds("chosen", l.expert, size_t(pairs) * 4);
    holds("shares", l.shares, size_t(pairs) * 4);
    holds("counters of scores", l.score_count, size_t(l.rows) * 4);
    holds("counters", l.up_count, size_t(warps) * 4);
    holds("counters", l.down_count, size_t(warps) * 4);
    if (l.d_pad % 64 || l.h_pad % 64 || l.d_pad < l.d || l.h_pad < l.h) wrong("padding", nullptr, 0);
    // no two of them overlap
    const std::map<uintptr_t, size_t> at = {
        {reinterpret_cast<uintptr_t>(l.logits), size_t(l.rows) * l.total * 4},
        {reinterpret_cast<uintptr_t>(l.x_copy), size_t(l.rows) * l.d_pad * 2},
        {reinterpret_cast<uintptr_t>(l.hidden), size_t(l.pairs) * l.h_pad * (l.terms == 1 ? 4 : 2 * l.terms)},
        {reinterpret_cast<uintptr_t>(l.parts), size_t(2 * warps * 32 * columns) * 4},
        {reinterpret_cast<uintptr_t>(l.expert), size_t(pairs) * 4},
        {reinterpret_cast<uintptr_t>(l.shares), size_t(pairs) * 4},
        {reinterpret_cast<uintptr_t>(l.score_count), size_t(l.rows) * 4},
        {reinterpret_cast<uintptr_t>(l.up_count), size_t(warps) * 4},
        {reinterpret_cast<uintptr_t>(l.down_count), size_t(warps) * 4}};
    uintptr_t end = 0;
    for (const auto& a : at) {
        if (a.first < end) wrong("scratch overlaps", reinterpret_cast<void*>(a.first), a.second);
        end = a.first + a.second;
    }
    return DPDR_OK;
}
}  // namespace experts
}  // namespace dpdr

extern "C" {
long fake_streamed(void) { return streamed; }
long fake_widened(void) { return widened; }
long fake_layers(void) { return layers; }
long fake_copies(void) { return copies; }
void fake_counts_reset(void) { streamed = widened = tiled = layers = copies = 0; }
}
