// proj.h -- what the host side of the projections (proj.cpp) hands to their
// kernels: operands by address and strides, and what becomes of a finished
// sum.  Not part of the public ABI.
#pragma once

#include <cstdint>

#include <cuda.h>

#include "dpdr_internal.h"

namespace dpdr {
namespace proj {

// An operand, indexed [i][k], k the index that is summed over.
struct Operand {
    const char* p;
    int64_t is, ks;   // strides in elements
};

// What a product is: D = A B^T and its bookkeeping.
//   kSingle  sum_k a0[m][k] b0[n][k]
//   kPair    the same a0 with b0 and b1: two sums of one output (gated forward)
//   kChain   sum_k a0 b0 + sum_k a1 b1 (the gated operator's dx)
//   kTwin    two products of one shape, a0 b0 -> out and a1 b0 -> out2 (its
//            weight gradients)
enum Kind { kSingle, kPair, kChain, kTwin };

// What becomes of z = sum (+ bias), or of the pair g, u:
//   kValue   act(z) + other, or act(g) * u
//   kSlope   other * act'(z), or other * u * act'(g) -> out and
//            other * act(g) -> out2
enum Finish { kValue, kSlope };

struct Epilogue {
    int finish = kValue;
    int act = DPDR_ACT_NONE;
    int half = 0;                  // operand type: 0 bfloat16, 1 float16
    const void* bias = nullptr;    // operand type
    const char* other = nullptr;   // residual, dy or dh
    int64_t other_rs = 0, other_cs = 0;
    int other_f32 = 0;
    char* out = nullptr;
    char* out2 = nullptr;
    int64_t out_rs = 0, out2_rs = 0;
    int out_f32 = 0;
    float* pre = nullptr;          // z, or g and, pre_up columns on, u
    int64_t pre_rs = 0, pre_up = 0;
    // Where the product is finished as a single dz, its column sums before it is
    // rounded: rows of one float a column, each over some of the rows
    float* sums = nullptr;
};

// The tensor cores add to a float32 sum by cutting off, not by rounding, so a
// long sum comes out too small.  Positive products (of 0.5 to 1.5 each) of
// bfloat16 lose 4.5e-7 of a sum of 640, 2.5e-5 of 8192 and 6.5e-5 of 16,384, of
// float16, whose products have more places, 3.4e-6 of 640 and 4.5e-5 of 8192;
// products of random sign a fraction of that.  Longer sums are taken in runs,
// which are added up rounded: of at most 10 steps (640 products) for float32
// results, for 16-bit ones as long as the loss is below a tenth of what the
// result's rounding may be off by.
constexpr int kSumStep = 64;   // products a step
constexpr int most_run_steps(int out_f32, int half) { return out_f32 ? 10 : half ? 128 : 256; }

// The runs of a sum, of nearly equal length: next() gives the step behind each,
// steps * (run + 1) / runs, without the product, which can pass 32 bits, or a
// division.
struct RunEnds {
    int whole, rest, runs, end, carry;
    constexpr RunEnds(int steps, int n, int from = 0)
        : whole(steps / n), rest(steps % n), runs(n), end(from), carry(0)
    {
    }
    constexpr int next()
    {
        end += whole;
        carry += rest;
        if (carry >= runs) carry -= runs, end++;
        return end;
    }
};

struct Product {
    Kind kind = kSingle;
    int64_t M = 0, N = 0, K = 0;
    Operand a[2] = {}, b[2] = {};
    Epilogue e;
    int64_t* sum_parts = nullptr;   // given how many rows of e.sums the product fills
};

constexpr int kPacked = 4;   // x, the weights, dy

// the plan behind dpdr_proj_t
struct Proj {
    bool gated = false;
    int64_t max_rows = 0, n_in = 0, n_out = 0;
    int half = 0, out_f32 = 0, grad_f32 = 0, act = 0;
    int device = 0, num_sms = 0;
    char* scratch = nullptr;       // dz (dg, du) and column sums
    // copies of operands that the tensor cores' loads cannot take as they lie
    char* packed[kPacked] = {};
    uint32_t* err = nullptr;       // error word, in host memory that kernels write to
    bool tile_set[2][2][2][2] = {}, row_set[2][2][2][3] = {};   // kernel attributes set
};

// Tensor-core product of operands that TMA can load: one stride 1, the other
// a multiple of 8, addresses multiples of 16 bytes (proj_tile.cu).  K >= 1.
int tile_launch(Proj* P, const Product& p, cudaStream_t s);

// The same for few rows (proj_rows.cu); not for kTwin.
int row_launch(Proj* P, const Product& p, cudaStream_t s);

// The same for one row, forward only (proj_token.cu): the summed index of all
// operands contiguous, any alignment and row stride.
int token_launch(Proj* P, const Product& p, cudaStream_t s);

// Whether the results and what else an epilogue reads allow four elements at
// a time: addresses and row strides of four elements, unit column strides
bool by_fours(const Epilogue& e);

// Tensor map of operand o, n x k elements, for boxes of `rows` x `step` (n by
// summed index), or of 64 x `step` where the summed index is the outer one
int tensor_map(CUtensorMap* map, const Operand& o, int64_t n, int64_t k, int half, int rows, int step);

// dz (or dg and du) of at least one row from the kept projections: e.pre and
// e.other in, e.out (and out2), where given, out.  With `sums` also dz's column
// sums over column_sum_parts(rows) runs of rows, cols floats each.  No e.pre: z
// is 0 (of use without an activation).
int slope_launch(const Epilogue& e, bool pair, int64_t rows, int64_t cols, float* sums, cudaStream_t s);
int column_sum_parts(int64_t rows);

// `parts` rows of column sums added up to the gradient of the bias
int join_launch(const float* sums, int parts, int64_t cols, void* out, int out_f32, int half, cudaStream_t s);

// Rows of column sums that a product of up to `rows` rows may fill: one for every 32
// rows (tile_launch); one for each CTA down the rows, of 64 rows at least, and of
// its cluster, of at most eight, with more than one no more in all than two an SM
// (row_launch).
constexpr int64_t product_sum_parts(int64_t rows, int num_sms)
{
    const int64_t tiles = (rows + 31) / 32, down = (rows + 63) / 64;
    const int64_t split = 8 * down < 2 * num_sms ? 8 * down : 2 * num_sms;
    return split > tiles ? split : tiles;
}

// Copies of 16-bit matrices with unit column stride and rows ld apart, each
// into a slot of the plan's
struct Copies {
    struct Job {
        const char* src;
        char* dst;
        int64_t rs, cs, rows, cols, ld;
    };
    Job job[kPacked];
    int slot[kPacked];
    int n = 0;
};
int copies_launch(Proj* P, const Copies& c, cudaStream_t s);

}  // namespace proj
}  // namespace dpdr
