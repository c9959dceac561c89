// integer.cu -- products of 8-bit integers with a scale for each row and each
// feature, for few rows, and what goes with them: rows rounded to such integers,
// matrices laid out anew for the products.
//
//   y = (sum_k x w) sx sw + bias + residual
//
// Up to four rows take four products at a time on the integer units.  Some more
// stream the weights past once (stream.cuh): a unit is 32 features and up to 32 rows, a
// CTA a unit, its sum over eight warps and, where there are fewer units than CTAs,
// several CTAs; the sums are whole numbers, so their order does not matter.  More rows
// are widened on their way to the tensor cores (integer_rows.cu), and many go to the
// tensor cores' tiles (proj_tile.cuh) as copies in 16 bits, which hold 8-bit integers
// exactly: the 8-bit integer instructions of this GPU reach 150 TOP/s, the 16-bit ones
// twelve times that.
//
// One row of 4096 x 4096 5.5 us from memory (3.1 TB/s), 16 rows 9.3; 8192 rows of 4096 x
// 8192 with bias and residual 380 to 397 (1.4 PFLOP/s), 32 of them the copies.
#include <algorithm>

#include "integer.h"
#include "stream.cuh"

namespace dpdr {
namespace integer {

using namespace stream;

namespace {

// ------------------------------------------------------------- few rows

constexpr int kPiece = 64;

struct RowsArgs {
    Rows r;
    int passes, parts, pieces, units;
};

__device__ __forceinline__ void put(const Finish& f, int64_t m, int64_t n, int sum, float w_scale, float bias)
{
    float v = float(sum) * (f.x_scale[m] * w_scale) + bias;
    if (f.residual) v += proj::load1(f.residual, m * f.residual_rs + n * f.residual_cs, f.out_f32, f.half);
    proj::store1(f.y, m * f.y_rs + n, v, f.out_f32, f.half);
}

template <int NT, bool SHIFT>
__global__ void __launch_bounds__(kThreads, 2) rows_kernel(const __grid_constant__ RowsArgs a)
{
    extern __shared__ __align__(128) char raw[];
    using S = Stream<kI8, kI8, NT, SHIFT, 1, kPiece, kWarps>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Rows& r = a.r;
    S st(shared_at(raw), warp, lane);
    float* room = reinterpret_cast<float*>(raw + kWarps * S::kWarpBytes);
    wait_previous();
    allow_next();
    const int all = a.units * a.parts;
    auto unit = [&](int u, int64_t& n0, int& m0) {
        const int part = u % a.parts, b = u / a.parts;
        n0 = int64_t(b / a.passes) * 32;
        m0 = b % a.passes * (8 * NT);
        Unit q;
        q.a[0] = r.w + n0 * r.w_rs;
        q.a[1] = q.a[0] + 16 * r.w_rs;
        q.a_stride[0] = q.a_stride[1] = r.w_rs;
        q.rows_left[0] = int(min(int64_t(16), r.n - n0));
        q.rows_left[1] = int(max(int64_t(0), min(int64_t(16), r.n - n0 - 16)));
        q.row_bytes = r.k;
        q.first = int(int64_t(a.pieces) * part / a.parts) + warp;
        q.last = int(int64_t(a.pieces) * (part + 1) / a.parts);
        return q;
    };
    int loading = int(blockIdx.x) - int(gridDim.x);
    auto next = [&]() {
        while (!st.more() && loading + int(gridDim.x) < all) {
            loading += gridDim.x;
            int64_t n0;
            int m0;
            const Unit q = unit(loading, n0, m0);
            // columns past the last repeat it, for nothing
            st.load_from(q, [&](int col) { return r.x + min(m0 + col, r.rows - 1) * r.x_rs; });
        }
    };
    st.begin(next);
    for (int u = blockIdx.x; u < all; u += gridDim.x) {
        int64_t n0;
        int m0;
        const Unit q = unit(u, n0, m0);
        float sum[2][NT][4];
        int v[NT];
        S::clear(sum);
        st.sums(q, sum, next);
#pragma unroll
        for (int n = 0; n < NT; n++) v[n] = join_columns(room, sum[0][n], sum[1][n], warp, lane);
        if (a.parts > 1) {
            int32_t* mine = r.parts + int64_t(u) * NT * kThreads + threadIdx.x;
#pragma unroll
            for (int n = 0; n < NT; n++) mine[n * kThreads] = v[n];
            if (!last_to_come(r.count + u / a.parts, a.parts)) continue;
            const int32_t* from = r.parts + int64_t(u / a.parts) * a.parts * NT * kThreads + threadIdx.x;
#pragma unroll
            for (int n = 0; n < NT; n++) v[n] = 0;
#pragma unroll 4
            for (int p = 0; p < a.parts; p++)
#pragma unroll
                for (int n = 0; n < NT; n++) v[n] += __ldcg(from + (p * NT + n) * kThreads);
        }
        const int64_t feature = n0 + lane;
        if (feature >= r.n) continue;
        const float w_scale = r.f.w_scale[feature], bias = r.f.bias ? r.f.bias[feature] : 0.0f;
#pragma unroll
        for (int n = 0; n < NT; n++) {
            const int m = m0 + n * 8 + warp;
            if (m < r.rows) put(r.f, m, feature, v[n], w_scale, bias);
        }
    }
}

// -------------------------------------------------------- up to four rows

constexpr int kTokenWarps = 8, kTokenDeep = 4;

// A group of `share` warps takes two features, each lane 16 bytes of both rows of
// w four times over before it uses the first, and four products at a time on the
// integer units, which hold whole sums of 32 bits: nothing to widen, and nothing to
// join beyond the group.  x comes from L1.  From five rows on the reads of x and the
// products take longer than the weights.
// ALIGNED: rows of w and x at multiples of 16 bytes.  Others are loaded by the aligned 16
// bytes that what is wanted begins and ends in, and shifted, which binds: one row of 4001 x
// 4003 9.0 us (1.8 TB/s), aligned of 4096 x 4096 5.2.
template <int ROWS, bool ALIGNED>
__global__ void __launch_bounds__(32 * kTokenWarps) token_kernel(const __grid_constant__ Rows r, int share)
{
    constexpr int kDeep = ALIGNED ? kTokenDeep : 2, kParts = ALIGNED ? 1 : 2;
    __shared__ int parts[kTokenWarps][2 * ROWS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = warp / share, mine = warp % share;
    const int64_t first = (int64_t(blockIdx.x) * (kTokenWarps / share) + group) * 2;
    const int64_t second = first + 1 >= r.n ? first : first + 1;   // a last odd feature is taken twice
    const char *w0 = r.w + first * r.w_rs, *w1 = r.w + second * r.w_rs;
    // the first loads' lines are asked into L2 while the kernel before drains
    if (first < r.n)
        for (int at = 128 * (mine * 32 + lane); at < r.k && at < 16 * 32 * kTokenDeep * share; at += 128 * 32 * share) {
            asm volatile("prefetch.global.L2 [%0];" ::"l"(w0 + at));
            asm volatile("prefetch.global.L2 [%0];" ::"l"(w1 + at));
        }
    wait_previous();
    allow_next();
    int acc[2][ROWS] = {};
    if (first < r.n) {
        const int units = r.k / 16, step = 32 * share;
        // 16 bytes from p on, all of them of one row, as they are loaded and as they are meant
        auto load = [](const char* p, uint4 (&v)[kParts]) {
            const int o = ALIGNED ? 0 : int(reinterpret_cast<uintptr_t>(p) & 15);
            const uint4* q = reinterpret_cast<const uint4*>(p - o);
            v[0] = __ldcs(q);
            if (!ALIGNED) v[kParts - 1] = o ? __ldcs(q + 1) : v[0];
        };
        auto meant = [](const char* p, const uint4 (&v)[kParts]) {
            return ALIGNED ? v[0] : shifted(v[0], v[kParts - 1], int(reinterpret_cast<uintptr_t>(p) & 15));
        };
        auto sum = [&](const uint4& a, const uint4& b, int u) {
#pragma unroll
            for (int m = 0; m < ROWS; m++) {
                const char* p = r.x + min(m, r.rows - 1) * r.x_rs + 16 * u;
                uint4 v[kParts];
                const int o = ALIGNED ? 0 : int(reinterpret_cast<uintptr_t>(p) & 15);
                const uint4* q = reinterpret_cast<const uint4*>(p - o);
                v[0] = q[0];
                if (!ALIGNED) v[kParts - 1] = o ? q[1] : v[0];
                const uint4 x = meant(p, v);
                acc[0][m] = __dp4a(int(a.x), int(x.x), __dp4a(int(a.y), int(x.y), acc[0][m]));
                acc[1][m] = __dp4a(int(b.x), int(x.x), __dp4a(int(b.y), int(x.y), acc[1][m]));
                acc[0][m] = __dp4a(int(a.z), int(x.z), __dp4a(int(a.w), int(x.w), acc[0][m]));
                acc[1][m] = __dp4a(int(b.z), int(x.z), __dp4a(int(b.w), int(x.w), acc[1][m]));
            }
        };
        for (int u0 = mine * 32 + lane; u0 < units; u0 += kDeep * step) {
            uint4 a[kDeep][kParts], b[kDeep][kParts];
#pragma unroll
            for (int d = 0; d < kDeep; d++)
                if (u0 + d * step < units) {
                    load(w0 + 16 * (u0 + d * step), a[d]);
                    load(w1 + 16 * (u0 + d * step), b[d]);
                }
#pragma unroll
            for (int d = 0; d < kDeep; d++) {
                const int u = u0 + d * step;
                if (u < units) sum(meant(w0 + 16 * u, a[d]), meant(w1 + 16 * u, b[d]), u);
            }
        }
        const int k = units * 16 + lane;   // fewer than 16 are left
        if (mine == 0 && k < r.k) {
#pragma unroll
            for (int m = 0; m < ROWS; m++) {
                const int x = reinterpret_cast<const int8_t*>(r.x)[min(m, r.rows - 1) * r.x_rs + k];
                acc[0][m] += x * reinterpret_cast<const int8_t*>(w0)[k];
                acc[1][m] += x * reinterpret_cast<const int8_t*>(w1)[k];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int m = 0; m < ROWS; m++) acc[i][m] = __reduce_add_sync(0xFFFFFFFFu, acc[i][m]);
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int m = 0; m < ROWS; m++) parts[warp][2 * m + i] = acc[i][m];
    if (share > 1) __syncthreads();
    else __syncwarp();
    // lane i finishes feature i % 2 of row i / 2
    const int m = lane / 2;
    const int64_t n = first + lane % 2;
    if (mine != 0 || m >= r.rows || n >= r.n) return;
    int v = 0;
    for (int w = 0; w < share; w++) v += parts[warp + w][lane];
    put(r.f, m, n, v, r.f.w_scale[n], r.f.bias ? r.f.bias[n] : 0.0f);
}

int token_launch(const Rows& r, int num_sms, cudaStream_t s)
{
    // More warps a group where the features alone are too few to keep the memory
    // busy and each warp keeps four loads a lane
    const int64_t groups = (r.n + 1) / 2;
    int share = 1;
    while (share < 8 && groups * share < 8 * num_sms && r.k >= 4096 * share) share *= 2;
    const int64_t per = kTokenWarps / share;
    const bool aligned = aligned_weights(r);
    auto* kernel = r.rows == 1   ? (aligned ? token_kernel<1, true> : token_kernel<1, false>)
                   : r.rows == 2 ? (aligned ? token_kernel<2, true> : token_kernel<2, false>)
                                 : token_kernel<4, true>;
    return proj::launch(kernel, dim3(unsigned((groups + per - 1) / per)), dim3(32 * kTokenWarps), 0, 1, s,
                        "integer token kernel", r, share);
}

// --------------------------------------------------------- laid out anew

// Sixteen elements a thread at a time.  Bound by the bytes: 8192 x 4096 twice to 16
// bits, 201 MB, in 32 us (6.2 TB/s).
template <int WIDE>
__global__ void __launch_bounds__(256) relay_kernel(const __grid_constant__ Relay r)
{
    wait_previous();
    allow_next();
    const Relay::Job& j = r.job[blockIdx.y];
    const int64_t across = (j.to + 15) / 16, all = across * j.rows, apart = int64_t(gridDim.x) * 256;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += apart) {
        const int64_t m = i / across, n = (i - m * across) * 16;
        const int8_t* p = j.src + m * j.rs + n * j.cs;
        uint32_t w[4] = {0, 0, 0, 0};
        if (j.cs == 1 && n + 16 <= j.cols) {
            // the aligned words around them
            const int o = int(reinterpret_cast<uintptr_t>(p) & 3);
            const uint32_t* q = reinterpret_cast<const uint32_t*>(p - o);
            if (reinterpret_cast<uintptr_t>(p) % 16 == 0) {
                const uint4 v = *reinterpret_cast<const uint4*>(p);
                w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
            } else {
                uint32_t v[5];
#pragma unroll
                for (int k = 0; k < 4; k++) v[k] = q[k];
                v[4] = o ? q[4] : 0u;
#pragma unroll
                for (int k = 0; k < 4; k++) w[k] = __funnelshift_r(v[k], v[k + 1], 8 * o);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 16; k++)
                if (n + k < j.cols) w[k / 4] |= uint32_t(uint8_t(p[k * j.cs])) << 8 * (k % 4);
        }
        if (WIDE == 0) {
            *reinterpret_cast<uint4*>(j.dst + m * j.ld + n) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            uint32_t v[8];
#pragma unroll
            for (int k = 0; k < 4; k++) {
                if (WIDE == 1) bytes_to_bf16(w[k], v[2 * k], v[2 * k + 1]);
                else bytes_to_f16(w[k], v[2 * k], v[2 * k + 1]);
            }
            char* to = j.dst + (m * j.ld + n) * 2;
            *reinterpret_cast<uint4*>(to) = make_uint4(v[0], v[1], v[2], v[3]);
            if (n + 8 < j.ld) *reinterpret_cast<uint4*>(to + 16) = make_uint4(v[4], v[5], v[6], v[7]);
        }
    }
}

// -------------------------------------------------------------- rounding

__device__ __forceinline__ float value_of(const void* p, int64_t i, int dtype)
{
    if (dtype == DPDR_FLOAT32) return static_cast<const float*>(p)[i];
    return proj::widen(static_cast<const uint16_t*>(p)[i], dtype == DPDR_FLOAT16);
}

// A row's numbers: what its values are multiplied by before they are rounded,
// and by what power of two values and largest size are scaled so that nothing in
// the arithmetic below overflows or loses places.
struct Rounding {
    float most, power, by;
    __device__ __forceinline__ explicit Rounding(float a)
    {
        // 2^-64 above 2^100, 2^64 below 2^-60
        power = a > 1.2676506e30f ? 5.421010862427522e-20f : a < 8.6736174e-19f ? 1.8446744073709552e19f : 1.0f;
        most = a * power;
        by = 127.0f / most;
    }
};

// 127 v / most, rounded to the nearest whole number, halves to even, exactly.
// v times the float32 quotient 127 / most is off by 1.6e-5 at most, so it decides unless
// it is near a half (the caller's fast way); there 254 |v| and (2 k + 1) most are
// compared, each as a float and what that leaves of the product, eight bits more, whose
// differences are exact.
__device__ __forceinline__ int rounded(float v, const Rounding& r)
{
    const float size = fabsf(v) * r.power, t = size * r.by, low = floorf(t), part = t - low;
    int q = part > 0.5f ? int(low) + 1 : int(low);
    if (fabsf(part - 0.5f) < 1e-4f) {
        const float odd = 2.0f * low + 1.0f;
        const float a = 254.0f * size, a_rest = fmaf(254.0f, size, -a);
        const float b = odd * r.most, b_rest = fmaf(odd, r.most, -b);
        const float d = (a - b) + (a_rest - b_rest);
        q = d > 0.0f || (d == 0.0f && (int(low) & 1)) ? int(low) + 1 : int(low);
    }
    return v < 0.0f ? -q : q;
}

// What a row's largest size makes of its values: `plain` rounding, or none (zeros,
// infinities, NaN)
struct Row {
    uint32_t high;   // the size's bits
    Rounding r;
    bool plain;
    __device__ __forceinline__ Row(uint32_t bits, float size)
        : high(bits), r(size), plain(bits > 0 && bits < 0x7F800000u)
    {
    }
};

// four values of it, each by itself
__device__ __noinline__ uint32_t round4_apart(float f0, float f1, float f2, float f3, uint32_t high, float size)
{
    const Row w(high, size);
    auto one = [&](float f) {
        if (w.plain) return uint32_t(rounded(f, w.r) & 255);
        if (w.high == 0x7F800000u && isinf(f)) return f < 0.0f ? 129u : 127u;
        return 0u;
    };
    return one(f0) | one(f1) << 8 | one(f2) << 16 | one(f3) << 24;
}

// t + 1.5 2^23 is t rounded in the low bits; what it was off by tells whether a half
// is near
__device__ __forceinline__ uint32_t round4(const float (&f)[4], const Row& w)
{
    uint32_t v[4];
    float off = w.plain && w.r.power == 1.0f ? 0.0f : 1.0f;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const float y = fmaf(f[k], w.r.by, 12582912.0f);
        off = fmaxf(off, fabsf(fmaf(f[k], w.r.by, 12582912.0f - y)));
        v[k] = __float_as_uint(y);
    }
    if (off > 0.4999f) return round4_apart(f[0], f[1], f[2], f[3], w.high, __uint_as_float(w.high));
    return __byte_perm(__byte_perm(v[0], v[1], 0x0040), __byte_perm(v[2], v[3], 0x0040), 0x5410);
}

// The largest of a row's threads' `high`; all threads of the CTA come here
template <int SHARE, int THREADS>
__device__ __forceinline__ uint32_t row_high(uint32_t high)
{
    __shared__ uint32_t most[THREADS / 32];
    high = __reduce_max_sync(0xFFFFFFFFu, high);
    if (SHARE > 32) {
        if (threadIdx.x % 32 == 0) most[threadIdx.x / 32] = high;
        __syncthreads();
        const int first = threadIdx.x / SHARE * (SHARE / 32);
#pragma unroll
        for (int w = 0; w < SHARE / 32; w++) high = max(high, most[first + w]);
    }
    return high;
}

// Rows that lie at multiples of 16 bytes, and are such long: SHARE threads a row, one
// pass.  The values stay in registers, HELD groups of 16 bytes a thread, kept as they
// came (as few as let several rows an SM be under way); longer rows are read twice, from
// L2 the second time.  Bound by the bytes, and by some ten instructions a value: 8192 x
// 8192 float32, 336 MB, in 52 us (6.4 TB/s; with 256 threads a row 60, with the exact
// comparison for every value 79), 4096 x 4096 bfloat16, 50 MB, in 13.3.
template <int DT, int HELD, int SHARE>
__global__ void __launch_bounds__(SHARE < 256 ? 256 : SHARE)
    quantise_kernel(const char* x, int64_t x_bytes, int8_t* q, int64_t q_rs, float* scale, int64_t rows, int units)
{
    constexpr int kThreads = SHARE < 256 ? 256 : SHARE, kEach = DT == DPDR_FLOAT32 ? 4 : 8;   // values of a group
    wait_previous();
    allow_next();
    const int at = int(threadIdx.x) % SHARE;
    const int64_t m = int64_t(blockIdx.x) * (kThreads / SHARE) + threadIdx.x / SHARE;
    const bool there = m < rows;
    const uint4* from = reinterpret_cast<const uint4*>(x + m * x_bytes) + at;
    // Sizes as whole numbers, whose order puts NaN above infinity: of 16-bit types two at a
    // time
    uint32_t high = 0;
    auto look = [&](const uint4& h) {
        const uint32_t w[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
        for (int k = 0; k < 4; k++) {
            if (DT == DPDR_FLOAT32) high = max(high, w[k] & 0x7FFFFFFFu);
            else high = __vmaxu2(high, w[k] & 0x7FFF7FFFu);
        }
    };
    uint4 held[HELD];
    const bool whole = units <= HELD * SHARE;
    if (there) {
        if (whole) {
#pragma unroll
            for (int k = 0; k < HELD; k++)
                if (at + k * SHARE < units) held[k] = from[k * SHARE];
#pragma unroll
            for (int k = 0; k < HELD; k++)
                if (at + k * SHARE < units) look(held[k]);
        } else {
#pragma unroll 4
            for (int u = 0; u < units - at; u += SHARE) look(from[u]);
        }
    }
    if (DT != DPDR_FLOAT32) {
        high = max(high >> 16, high & 0xFFFFu);
        high = __float_as_uint(proj::widen(uint16_t(high), DT == DPDR_FLOAT16));
    }
    high = row_high<SHARE, kThreads>(high);
    const Row w(high, __uint_as_float(high));
    if (!there) return;
    if (at == 0) scale[m] = __uint_as_float(w.high) / 127.0f;
    int8_t* to = q + m * q_rs + at * kEach;
    auto put = [&](int u, const uint4& h) {
        float f[4];
        if (DT == DPDR_FLOAT32) {
            proj::widen4(h, 1, 0, f);
            *reinterpret_cast<uint32_t*>(to + u * kEach) = round4(f, w);
        } else {
            uint2 v;
            proj::widen4(make_uint4(h.x, h.y, 0, 0), 0, DT == DPDR_FLOAT16, f);
            v.x = round4(f, w);
            proj::widen4(make_uint4(h.z, h.w, 0, 0), 0, DT == DPDR_FLOAT16, f);
            v.y = round4(f, w);
            *reinterpret_cast<uint2*>(to + u * kEach) = v;
        }
    };
    if (whole) {
#pragma unroll
        for (int k = 0; k < HELD; k++)
            if (at + k * SHARE < units) put(k * SHARE, held[k]);
    } else {
#pragma unroll 2
        for (int u = 0; u < units - at; u += SHARE) put(u, from[u]);
    }
}

// Rows that lie otherwise: a CTA a row, value by value, read twice: 8192 x 8191 float32 in
// 100 us (of 8192 values 52), 4096 x 4095 bfloat16 in 32 (15)
template <int DT>
__global__ void __launch_bounds__(256)
    quantise_any_kernel(const void* x, int64_t rs, int64_t cs, int8_t* q, int64_t q_rs, float* scale, int64_t n)
{
    constexpr int kDeep = 8;   // values of a thread under way
    wait_previous();
    allow_next();
    const int64_t m = blockIdx.x, from = m * rs;
    auto get = [&](int64_t k) {
        if (DT == DPDR_FLOAT32) return static_cast<const float*>(x)[from + k * cs];
        return proj::widen(static_cast<const uint16_t*>(x)[from + k * cs], DT == DPDR_FLOAT16);
    };
    uint32_t high = 0;
    for (int64_t k0 = threadIdx.x; k0 < n; k0 += kDeep * 256) {
        float f[kDeep];
#pragma unroll
        for (int d = 0; d < kDeep; d++) f[d] = k0 + d * 256 < n ? get(k0 + d * 256) : 0.0f;
#pragma unroll
        for (int d = 0; d < kDeep; d++) high = max(high, __float_as_uint(f[d]) & 0x7FFFFFFFu);
    }
    high = row_high<256, 256>(high);
    const Row w(high, __uint_as_float(high));
    if (threadIdx.x == 0) scale[m] = __uint_as_float(w.high) / 127.0f;
    int8_t* to = q + m * q_rs;
    for (int64_t k0 = threadIdx.x; k0 < n; k0 += kDeep * 256) {
        float f[kDeep];
#pragma unroll
        for (int d = 0; d < kDeep; d++) f[d] = k0 + d * 256 < n ? get(k0 + d * 256) : 0.0f;
#pragma unroll
        for (int d = 0; d < kDeep; d += 4) {
            const uint32_t v = round4(reinterpret_cast<const float(&)[4]>(f[d]), w);
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (k0 + (d + i) * 256 < n) to[k0 + (d + i) * 256] = int8_t(v >> 8 * i);
        }
    }
}

template <int DT>
int quantise(int64_t rows, int64_t n, const dpdr_matrix& x, const dpdr_matrix& q, float* scale, cudaStream_t s)
{
    const char* what = "quantise kernel";
    const int es = DT == DPDR_FLOAT32 ? 4 : 2, each = 16 / es;
    auto fits = [&](const void* p, int64_t bytes, int unit) {
        return reinterpret_cast<uintptr_t>(p) % unit == 0 && (rows == 1 || bytes % unit == 0);
    };
    if ((x.col_stride != 1 && n > 1) || n % each || !fits(x.data, x.row_stride * es, 16) ||
        !fits(q.data, q.row_stride, each))
        return proj::launch(quantise_any_kernel<DT>, dim3(unsigned(rows)), dim3(256), 0, 1, s, what,
                            (const void*)x.data, x.row_stride, x.col_stride, static_cast<int8_t*>(q.data), q.row_stride,
                            scale, n);
    const int units = int(n / each);
    auto run = [&](auto* kernel, int share) {
        const int threads = share < 256 ? 256 : share, per = threads / share;
        return proj::launch(kernel, dim3(unsigned((rows + per - 1) / per)), dim3(unsigned(threads)), 0, 1, s, what,
                            (const char*)x.data, x.row_stride * es, static_cast<int8_t*>(q.data), q.row_stride, scale,
                            rows, units);
    };
    if (units <= 4 * 32) return run(quantise_kernel<DT, 4, 32>, 32);
    if (units <= 4 * 128) return run(quantise_kernel<DT, 4, 128>, 128);
    if (units <= 4 * 256) return run(quantise_kernel<DT, 4, 256>, 256);
    if (units <= 4 * 512) return run(quantise_kernel<DT, 4, 512>, 512);
    if (units <= 8 * 512) return run(quantise_kernel<DT, 8, 512>, 512);
    return run(quantise_kernel<DT, 8, 1024>, 1024);
}

template <int NT>
int rows_launch_of(const RowsArgs& a, bool shift, int ctas, cudaStream_t s)
{
    auto* kernel = shift ? rows_kernel<NT, true> : rows_kernel<NT, false>;
    using S = Stream<kI8, kI8, NT, true, 1, kPiece, kWarps>;
    using T = Stream<kI8, kI8, NT, false, 1, kPiece, kWarps>;
    const int bytes = kWarps * (shift ? S::kWarpBytes : T::kWarpBytes) + kJoin * 4;
    bool& set = a.r.set[NT == 1 ? 0 : NT == 2 ? 1 : 2][shift];
    if (!set) {
        const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                   cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess) return cuda_fail_c(e, "integer rows kernel");
        set = true;
    }
    return proj::launch(kernel, dim3(unsigned(ctas)), dim3(kThreads), size_t(bytes), 1, s, "integer rows kernel", a);
}

}  // namespace

int rows_launch(const Rows& r, int num_sms, cudaStream_t s)
{
    if (for_tokens(r)) return token_launch(r, num_sms, s);
    const bool shift = !aligned_weights(r);
    RowsArgs a;
    a.r = r;
    const int nt = r.rows <= 8 ? 1 : r.rows <= 16 ? 2 : 4;
    a.passes = (r.rows + 8 * nt - 1) / (8 * nt);
    const int64_t units = (r.n + 31) / 32 * a.passes;
    a.units = int(units);
    a.pieces = (r.k + kPiece - 1) / kPiece;
    const int slots = 2 * num_sms;
    // as many parts as there are CTAs for, while a warp keeps two pieces
    a.parts = int(std::max<int64_t>(1, std::min<int64_t>(slots / units, a.pieces / (2 * kWarps))));
    const int ctas = int(std::min<int64_t>(units * a.parts, slots));
    return nt == 1   ? rows_launch_of<1>(a, shift, ctas, s)
           : nt == 2 ? rows_launch_of<2>(a, shift, ctas, s)
                     : rows_launch_of<4>(a, shift, ctas, s);
}

int relay_launch(const Relay& r, int num_sms, cudaStream_t s)
{
    int64_t most = 0;
    for (int i = 0; i < r.n; i++) most = std::max(most, r.job[i].rows * ((r.job[i].to + 15) / 16));
    const unsigned blocks = unsigned(std::min<int64_t>((most + 255) / 256, int64_t(num_sms) * 16));
    auto* kernel = r.wide == 0 ? relay_kernel<0> : r.wide == 1 ? relay_kernel<1> : relay_kernel<2>;
    return proj::launch(kernel, dim3(blocks, unsigned(r.n)), dim3(256), 0, 1, s, "integer operand copy", r);
}

int quantise_launch(int dtype, int64_t rows, int64_t n, const dpdr_matrix& x, const dpdr_matrix& q, float* scale,
                    cudaStream_t s)
{
    if (dtype == DPDR_FLOAT32) return quantise<DPDR_FLOAT32>(rows, n, x, q, scale, s);
    if (dtype == DPDR_FLOAT16) return quantise<DPDR_FLOAT16>(rows, n, x, q, scale, s);
    return quantise<DPDR_BFLOAT16>(rows, n, x, q, scale, s);
}

}  // namespace integer
}  // namespace dpdr
