// experts.h -- what the host side of a layer of experts (experts.cpp) hands to
// its kernels (experts.cu).  Not part of the public ABI.
#pragma once

#include "dpdr_internal.h"

namespace dpdr {
namespace experts {

constexpr int kMostRows = 64;       // tokens: a bit each in an expert's mask
constexpr int kMostTop = 16;        // of them chosen, a lane each
constexpr int kMostExperts = 512;   // 16 a lane of a warp
constexpr int64_t kMostSize = 1 << 20;
constexpr int kWholeRows = 8;       // of which each has a column of its own in the last product
// Columns of the products (x, hidden values) are read by whole pieces of the rows of
// weights, so a row of them is a multiple of the elements that a piece has at most: in
// the up products of 8-bit weights 128, else 64 (checked where the pieces are chosen).
constexpr int kPad = 64, kPad8 = 128;

struct Layer {
    int rows, top, total, first, local;
    int d, h;                      // n_model, n_hidden
    int64_t d_pad, h_pad;          // a row of the copy of x, of the hidden values (kPad)
    int half;                      // operand type: 0 bfloat16, 1 float16
    int w_int8, act, normalise, out_f32;
    const char* x;
    int64_t x_rs, x_cs;
    const char* router;
    int64_t router_rs, router_cs;
    dpdr_matrices w[3];            // gate, up, down
    const float* scale[3];         // contiguous, channels of an expert after another
    char* y;
    int64_t y_rs;
    int32_t* chosen;               // rows by top, or NULL
    float* share;
    // scratch of the plan
    float* logits;                 // rows by total
    char* x_copy;                  // rows by d_pad, zero behind d
    // rows top by h_pad, zero behind h: three terms of bfloat16, an array each of `pairs`
    // rows (the most that the plan takes), or with terms 1 float32
    char* hidden;
    int terms, pairs;
    float* parts;                  // sums of units that several warps share
    float* z;                      // of more than 8 rows, the experts' results by pair
    int32_t* expert;               // of a pair, and its share
    float* shares;
    uint32_t* score_count;         // a counter for some tokens
    uint32_t* up_count;            // a counter a warp
    uint32_t* down_count;
    int ctas;                      // of either product kernel
};

// makes the product kernels ready and sets how many CTAs each has, of l's rows and top
int product_ctas(Layer& l, int num_sms);
// the whole layer, at least one row
int launch(const Layer& l, int num_sms, cudaStream_t s);

}  // namespace experts
}  // namespace dpdr
