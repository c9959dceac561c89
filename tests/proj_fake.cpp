// proj_fake.cpp -- the projections' host code (proj.cpp) over a CUDA runtime
// that only keeps books (test infrastructure only): which device allocations
// live, what was freed, which device is current, which kernels a call asked
// for, and whether the scratch that they get holds what they put there.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <set>

#include "proj.h"

namespace {

struct Books {
    int device = 0;
    long frees = 0, host_allocs = 0, syncs = 0, launches = 0, tiles = 0, rows = 0;
    int refuse_mallocs = 0;            // as many allocations fail
    cudaError_t last = cudaSuccess;    // what cudaGetLastError gives
    std::map<uintptr_t, size_t> live;  // device allocations
    char wrong[200] = "";
};
Books B;

void wrong(const char* what, const void* p, size_t bytes)
{
    if (!*B.wrong) std::snprintf(B.wrong, sizeof B.wrong, "%s: %zu bytes at %p", what, bytes, p);
}

// Addresses from here on are the library's own allocations.
constexpr uintptr_t kOwn = uintptr_t(1) << 44;
uintptr_t next_at = kOwn;

// Whether [p, p + bytes) lies in one live allocation, if it is the library's.
void holds(const char* what, const void* p, size_t bytes)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    if (a < kOwn || bytes == 0) return;
    auto it = B.live.upper_bound(a);
    if (it == B.live.begin()) return wrong(what, p, bytes);
    --it;
    if (a + bytes > it->first + it->second) wrong(what, p, bytes);
}

void rows_hold(const char* what, const void* p, int64_t rs, int64_t rows, int64_t cols, int64_t esize)
{
    if (p && rows && cols) holds(what, p, size_t((rows - 1) * rs + cols) * esize);
}

void operand_holds(const char* what, const dpdr::proj::Operand& o, int64_t n, int64_t k)
{
    if (o.p && n && k) holds(what, o.p, size_t((n - 1) * o.is + (k - 1) * o.ks + 1) * 2);
}

int product(const dpdr::proj::Product& p)
{
    using namespace dpdr::proj;
    B.launches++;
    const int two_a = p.kind == kChain || p.kind == kTwin, two_b = p.kind == kChain || p.kind == kPair;
    for (int i = 0; i <= two_a; i++) operand_holds("operand a", p.a[i], p.M, p.K);
    for (int i = 0; i <= two_b; i++) operand_holds("operand b", p.b[i], p.N, p.K);
    const int es = p.e.out_f32 ? 4 : 2;
    rows_hold("out", p.e.out, p.e.out_rs, p.M, p.N, es);
    if (p.kind == kTwin || (p.kind == kPair && p.e.finish == kSlope))
        rows_hold("out2", p.e.out2, p.e.out2_rs, p.M, p.N, es);
    if (p.e.sums) {   // as many rows of sums as the kernels may fill
        const int64_t parts = product_sum_parts(p.M, 152);
        if (!p.sum_parts) return wrong("sums, but no count", p.e.sums, 0), DPDR_OK;
        *p.sum_parts = parts;
        rows_hold("column sums", p.e.sums, p.N, parts, p.N, 4);
        const uintptr_t at = reinterpret_cast<uintptr_t>(p.e.sums), z = reinterpret_cast<uintptr_t>(p.e.out);
        if (at < z + size_t((p.M - 1) * p.e.out_rs + p.N) * es) wrong("sums over dz", p.e.sums, 0);
    }
    return DPDR_OK;
}

}  // namespace

// ------------------------------------------------------ the CUDA runtime
extern "C" {
cudaError_t cudaGetDevice(int* d)
{
    *d = B.device;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int)
{
    *v = 152;
    return cudaSuccess;
}
cudaError_t cudaHostAlloc(void** p, size_t n, unsigned)
{
    B.host_allocs++;
    *p = std::calloc(1, n);
    return cudaSuccess;
}
cudaError_t cudaMalloc(void** p, size_t n)
{
    if (B.refuse_mallocs > 0) {
        B.refuse_mallocs--;
        return B.last = cudaErrorMemoryAllocation;
    }
    *p = reinterpret_cast<void*>(next_at);
    B.live[next_at] = n;
    next_at += (n + 511) / 256 * 256;
    return cudaSuccess;
}
cudaError_t cudaFree(void* p)
{
    if (!p) return cudaSuccess;
    B.frees++;
    if (!B.live.erase(reinterpret_cast<uintptr_t>(p))) wrong("freed twice", p, 0);
    return cudaSuccess;
}
cudaError_t cudaMemset2DAsync(void*, size_t, int, size_t, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t)
{
    B.syncs++;
    return cudaSuccess;
}
cudaError_t cudaGetDriverEntryPointByVersion(const char*, void** f, unsigned, unsigned long long,
                                             cudaDriverEntryPointQueryResult*)
{
    *f = nullptr;
    return cudaErrorUnknown;
}
cudaError_t cudaGetLastError(void)
{
    const cudaError_t e = B.last;
    B.last = cudaSuccess;
    return e;
}
}

// ------------------------------------------------------- the library's rest
namespace dpdr {
static char message[256];
int fail_c(int status, const char* msg)
{
    std::snprintf(message, sizeof message, "%s", msg);
    return status;
}
int cuda_fail_c(cudaError_t e, const char* what)
{
    return fail_c(e == cudaErrorMemoryAllocation ? DPDR_ERR_OOM : DPDR_ERR_CUDA, what);
}
namespace proj {
int tile_launch(Proj*, const Product& p, cudaStream_t)
{
    B.tiles++;
    return product(p);
}
int row_launch(Proj*, const Product& p, cudaStream_t)
{
    B.rows++;
    return product(p);
}
int token_launch(Proj*, const Product& p, cudaStream_t) { return product(p); }
int column_sum_parts(int64_t rows)
{
    return int(std::min<int64_t>(std::max<int64_t>((rows + 15) / 16, std::min<int64_t>(rows, 64)), 512));
}
int slope_launch(const Epilogue& e, bool pair, int64_t rows, int64_t cols, float* sums, cudaStream_t)
{
    B.launches++;
    rows_hold("dz", e.out, e.out_rs, rows, cols, 2);
    if (pair) rows_hold("du", e.out2, e.out2_rs, rows, cols, 2);
    if (sums) rows_hold("sums", sums, cols, column_sum_parts(rows), cols, 4);
    rows_hold("summed", e.other, e.other_rs, rows, cols, e.other_f32 ? 4 : 2);
    if (e.other_f32 && reinterpret_cast<uintptr_t>(e.other) >= kOwn) {   // sums of sums
        const uintptr_t a = reinterpret_cast<uintptr_t>(e.other), b = reinterpret_cast<uintptr_t>(sums);
        if (b < a + size_t(rows) * cols * 4) wrong("sums over those they add up", sums, 0);
    }
    return DPDR_OK;
}
int join_launch(const float* sums, int parts, int64_t cols, void*, int, int, cudaStream_t)
{
    B.launches++;
    if (parts < 1 || parts > 512) wrong("joined parts", nullptr, parts);
    rows_hold("joined sums", sums, cols, parts, cols, 4);
    return DPDR_OK;
}
int copies_launch(Proj*, const Copies& c, cudaStream_t)
{
    B.launches++;
    for (int i = 0; i < c.n; i++) rows_hold("copy", c.job[i].dst, c.job[i].ld, c.job[i].rows, c.job[i].cols, 2);
    return DPDR_OK;
}
}  // namespace proj
}  // namespace dpdr

// ------------------------------------------------------------- for the tests
extern "C" {
void fake_reset(void) { B = Books(); }
void fake_device(int d) { B.device = d; }
void fake_refuse_mallocs(int n) { B.refuse_mallocs = n; }
long fake_frees(void) { return B.frees; }
long fake_launches(void) { return B.launches; }
long fake_syncs(void) { return B.syncs; }
long fake_tiles(void) { return B.tiles; }   // products of tile_launch, row_launch
long fake_rows(void) { return B.rows; }
int fake_live(void) { return int(B.live.size()); }
int fake_last_error(void) { return int(B.last); }
const char* fake_wrong(void) { return B.wrong; }
const char* fake_message(void) { return dpdr::message; }
// Whether the runs of a sum of `steps` steps, at most `most` a run, are all of
// 1 to `most` steps, one behind the other, and end with the sum
int fake_runs_fit(int steps, int most)
{
    const int runs = int((int64_t(steps) + most - 1) / most);
    int k = 0;
    dpdr::proj::RunEnds ends(steps, runs);
    for (int run = 0; run < runs; run++) {
        const int end = ends.next();
        if (end != int(int64_t(steps) * (run + 1) / runs) || end <= k || end - k > most) return 0;
        k = end;
    }
    return k == steps;
}
// how many different error words the plans have
int fake_error_words(void** plans, int n)
{
    std::set<uint32_t*> words;
    for (int i = 0; i < n; i++) words.insert(static_cast<dpdr::proj::Proj*>(plans[i])->err);
    return int(words.size());
}
}
