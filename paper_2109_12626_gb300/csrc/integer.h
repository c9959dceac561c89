// integer.h -- what the host side of the products of 8-bit integers
// (integer.cpp) hands to their kernels (integer.cu).  Not part of the public ABI.
#pragma once

#include "proj.h"

namespace dpdr {
namespace integer {

// Sums of products of 8-bit integers stay below 2^31
constexpr int64_t kMostSummed = (int64_t(1) << 17) - 1;

// rows that rows_launch takes
constexpr int kFewRows = 64;
// and of these the ones that its kernel for tokens takes: of w and x at multiples of 16
// bytes, and of both at any address
constexpr int kTokenRows = 4, kAnyTokenRows = 2;
// Weights up to which it is faster than the streams for rows at any address.  us of it
// and of them, one or two rows: 4001 x 4003 9.0 and 12.5, 14,336 x 4096 29 and 23; three
// rows of 4001 x 4003 12.5 and 12.4.
constexpr int64_t kAnyTokenMost = int64_t(1) << 25;
// Rows past which wide_launch is faster where it takes the product.  us of
// rows_launch and of it, 4096 x 4096 weights: 16 rows 9.3 and 10.2, 32 rows 12.0
// and 10.6; 24 rows of 1024 x 8192 11.6 and 7.9.
constexpr int kStreamRows = 16;
// what their elements are a multiple of
constexpr int kRowsPad = 64;

struct Finish {
    const float* x_scale;    // of a row, of a feature
    const float* w_scale;
    const float* bias;       // or NULL
    const char* residual;    // result type, or NULL
    int64_t residual_rs, residual_cs;
    char* y;
    int64_t y_rs;
    int out_f32, half;       // result: float32, or 0 bfloat16, 1 float16
};

// Few rows: x by rows of whole 64 bytes at multiples of 16 (zero or not there
// behind k), w with the summed index contiguous at any address and row stride.
struct Rows {
    int rows, k;
    int64_t n;
    const char* x;
    int64_t x_rs;
    const char* w;
    int64_t w_rs;
    Finish f;
    int32_t* parts;          // of units whose sum is split
    uint32_t* count;
    bool (*set)[2];          // of the plan: kernels' attributes set
};
// (that kernel needs neither parts nor padded rows of x)
int rows_launch(const Rows& r, int num_sms, cudaStream_t s);
inline bool aligned_weights(const Rows& r)
{
    return reinterpret_cast<uintptr_t>(r.w) % 16 == 0 && (r.n == 1 || r.w_rs % 16 == 0);
}
inline bool for_tokens(const Rows& r)
{
    return aligned_weights(r) ? r.rows <= kTokenRows : r.rows <= kAnyTokenRows && r.n <= kAnyTokenMost / r.k;
}
constexpr int64_t parts_ints(int num_sms) { return int64_t(2 * num_sms) * 32 * 32; }

// Some rows, both operands widened on their way to the tensor cores: rows of x and w
// contiguous, at any address and row stride.
struct Wide {
    int rows, k;
    int64_t n;
    const char* x;
    int64_t x_rs;
    const char* w;
    int64_t w_rs;
    Finish f;
    bool* set;               // of the plan: kernels' attributes set
    uint32_t* err;
};
// whether the product's tiles leave SMs for parts of its sum, and tensor memory holds its runs
bool wide_takes(int64_t rows, int64_t n, int64_t k, int num_sms);
int wide_launch(const Wide& q, int num_sms, cudaStream_t s);

// 8-bit matrices laid out anew: by rows ld apart, zero from cols up to `to`, as
// 8-bit integers (wide 0), bfloat16 (1) or float16 (2)
struct Relay {
    struct Job {
        const int8_t* src;
        char* dst;
        int64_t rs, cs, rows, cols, ld, to;
    };
    Job job[2];
    int n = 0, wide = 0;
};
int relay_launch(const Relay& r, int num_sms, cudaStream_t s);

// a row's largest size over 127, and the row in units of that, rounded
int quantise_launch(int dtype, int64_t rows, int64_t n, const dpdr_matrix& x, const dpdr_matrix& q, float* scale,
                    cudaStream_t s);

}  // namespace integer
}  // namespace dpdr
