// proj_token.cu -- launch of the kernels of proj_token.cuh.
#include "proj_token.cuh"

namespace dpdr {
namespace proj {

int token_launch(Proj* P, const Product& p, cudaStream_t s)
{
    const bool pair = p.kind == kPair;
    TokenArgs t;
    t.x = p.a[0];
    t.w[0] = p.b[0];
    t.w[1] = p.b[pair ? 1 : 0];
    t.K = p.K;
    t.N = p.N;
    t.e = p.e;
    auto fits = [&](const Operand& o) {
        return reinterpret_cast<uintptr_t>(o.p) % 16 == 0 && (p.N == 1 || o.is % 8 == 0);
    };
    t.aligned = reinterpret_cast<uintptr_t>(t.x.p) % 16 == 0 && fits(t.w[0]) && fits(t.w[1]);
    // More warps a feature where the features alone are too few to keep the
    // memory busy and each warp keeps four loads a lane: 512 x 8192 weights
    // with 1, 2, 4 and 8: 8.4, 5.2, 4.1 and 3.4 us; 4096 x 4096, which has
    // enough: 7.5, 9.9, 8.9 and 11.4.
    const int64_t groups = pair ? p.N : (p.N + 1) / 2;
    t.share = 1;
    while (t.share < 8 && groups * t.share < 8 * P->num_sms && p.K >= 2048 * t.share) t.share *= 2;
    const int64_t per = kTokenWarps / t.share;
    const TokenKernel kernel = pair ? token_kernel_of<true>(p.e.act) : token_kernel_of<false>(p.e.act);
    return launch(kernel, dim3(unsigned((groups + per - 1) / per)), dim3(32 * kTokenWarps), 0, 1, s,
                  "projection token kernel", t);
}

}  // namespace proj
}  // namespace dpdr
