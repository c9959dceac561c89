// stream.cuh -- products of a few columns with weights that stream past once:
// what the kernels for a few tokens (experts.cu, integer.cu) share.
//
// D[row][column] = sum_k A[row][k] B[column][k] for 32 rows of A (weights: 32 of
// one matrix, or 16 of either of two) and 8 NT columns (tokens).  With so few
// columns the weights' bytes are the bound, and what matters is that some 100 KB
// an SM are always under way.  Each warp of a CTA takes every eighth piece of 64
// bytes along k and loads it into a ring of its own by cp.async, four bytes of
// A's rows beside the columns that go with them, several pieces ahead, across
// the CTA's units of work; no warp waits for another until a unit's eight partial
// sums are joined, in the order of the warps.  (Rows copied by cp.async.bulk
// instead reached 4.1 TB/s with 1 KB a copy, an issuing warp making one in 70
// cycles.)
//
// The products are legacy matrix instructions (m16n8k16 of 16-bit operands,
// m16n8k8 of tf32), which at 600 and 300 TFLOP/s are far from the bound for up
// to 32 columns.  Which k goes to which place of an instruction is free, as long as
// A and B agree, so a lane takes 16 bytes side by side of each row.
//   16-bit weights, columns of their type: as they are.
//   8-bit weights: widened in registers, exactly, to the columns' type.  (The
//     8-bit integer instruction reaches 150 TOP/s, a quarter of what the widened
//     operands do.)
//   8-bit weights and 8-bit columns: both widened to float16; products and sums
//     below 2^24 are whole numbers that float32 holds exactly, so the sums of 1024
//     products are added up as integers.
//   float32 columns: A widened to tf32, exactly, and each column value split into
//     two of 11 bits (the second cut off, 2^-21 of the value), two products.
// SHIFT: rows of A at any address.  The aligned 16 bytes around what a lane needs
// are loaded, and shifted in registers.  What lies behind the end of a row is
// never read (cp.async fills up with zeros).
#pragma once

#include "proj_common.cuh"
#include "proj_launch.cuh"

namespace dpdr {
namespace stream {

using proj::wait_previous;
using proj::allow_next;

enum Kind { kBf16, kF16, kI8, kF32 };   // of weights (not kF32) and columns

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kRows = 32;               // of A, a unit
constexpr int kPiece = 64;              // bytes of a row of A, a stage
// bytes of a warp's ring: rooms of two CTAs an SM, where the shifted rows of A do
// not make two stages larger
constexpr int ring_bytes(bool shift) { return shift ? 13312 : 12288; }

constexpr int size_of(int kind) { return kind == kI8 ? 1 : kind == kF32 ? 4 : 2; }
constexpr int elements(int wt) { return kPiece / size_of(wt); }   // of a piece

__device__ __forceinline__ uint32_t shared_at(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }

// 16 bytes, of which the first `bytes` are read and the others are zero
__device__ __forceinline__ void copy16(uint32_t to, const char* from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

__device__ __forceinline__ uint4 load16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}

// bytes o .. o + 15 of the 32 in lo and hi, 0 <= o < 16
__device__ __forceinline__ uint4 shifted(const uint4& lo, const uint4& hi, int o)
{
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    if (o & 8)
#pragma unroll
        for (int i = 0; i < 6; i++) w[i] = w[i + 2];
    if (o & 4)
#pragma unroll
        for (int i = 0; i < 5; i++) w[i] = w[i + 1];
    const int b = 8 * (o & 3);
    return make_uint4(__funnelshift_r(w[0], w[1], b), __funnelshift_r(w[1], w[2], b), __funnelshift_r(w[2], w[3], b),
                      __funnelshift_r(w[3], w[4], b));
}

// ------------------------------------------------------- 8 bits widened

// Four 8-bit integers as float16: 1024 + (v + 128) has v + 128 in its low bits
__device__ __forceinline__ void bytes_to_f16(uint32_t v, uint32_t& a, uint32_t& b)
{
    v ^= 0x80808080u;
    const uint32_t lo = __byte_perm(v, 0x64646464u, 0x4140), hi = __byte_perm(v, 0x64646464u, 0x4342);
    const __half2 off = __half2half2(__ushort_as_half(0x6480));   // 1152
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&lo), off),
                  y = __hsub2(*reinterpret_cast<const __half2*>(&hi), off);
    a = *reinterpret_cast<const uint32_t*>(&x);
    b = *reinterpret_cast<const uint32_t*>(&y);
}

// and as bfloat16, whose 7 bits behind the first hold the lower seven at 128:
// (128 + v mod 128) - (256 for a negative v, else 128)
__device__ __forceinline__ void bytes_to_bf16(uint32_t v, uint32_t& a, uint32_t& b)
{
    const uint32_t lo = __byte_perm(v, 0x43434343u, 0x4140), hi = __byte_perm(v, 0x43434343u, 0x4342);
    auto part = [](uint32_t w) {
        const uint32_t low = w & 0xFF7FFF7Fu, sign = w & 0xFF80FF80u;
        const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&low),
                                         *reinterpret_cast<const __nv_bfloat162*>(&sign));
        return *reinterpret_cast<const uint32_t*>(&d);
    };
    a = part(lo);
    b = part(hi);
}

// and as float32, 2^23 + (v + 128)
__device__ __forceinline__ void bytes_to_f32(uint32_t v, float (&f)[4])
{
    v ^= 0x80808080u;
    constexpr float off = 8388608.0f + 128.0f;
    f[0] = __uint_as_float(__byte_perm(v, 0x4B000000u, 0x7650)) - off;
    f[1] = __uint_as_float(__byte_perm(v, 0x4B000000u, 0x7651)) - off;
    f[2] = __uint_as_float(__byte_perm(v, 0x4B000000u, 0x7652)) - off;
    f[3] = __uint_as_float(__byte_perm(v, 0x4B000000u, 0x7653)) - off;
}

// ---------------------------------------------------- matrix instructions

template <int XT>
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                      uint32_t b1)
{
    if (XT == kBf16)
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma_tf32(float (&c)[4], float a0, float a1, float a2, float a3, float b0, float b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(__float_as_uint(a0)), "r"(__float_as_uint(a1)), "r"(__float_as_uint(a2)), "r"(__float_as_uint(a3)),
          "r"(__float_as_uint(b0)), "r"(__float_as_uint(b1)));
}

// h as a value of 11 bits and the rest of it, none of infinities and NaN
__device__ __forceinline__ void split_tf32(float h, float& hi, float& lo)
{
    const uint32_t top = __float_as_uint(h) & 0xFFFFE000u;
    hi = __uint_as_float(top);
    lo = (top & 0x7F800000u) == 0x7F800000u ? 0.0f : h - hi;
}

// ---------------------------------------------------------------- a unit

// Where a unit's operands lie.  A's row r (0 .. 31) is row r of the first 16 at
// a[0], the others at a[1]; rows past rows_left[.] are zero.
struct Unit {
    const char* a[2];
    int64_t a_stride[2];     // bytes from row to row
    int rows_left[2];        // rows that there are, of 16
    int row_bytes;
    int first, last;         // pieces along k
};

template <int WT, int XT, int NT, bool SHIFT>
struct Stream {
    static constexpr int kK = elements(WT);              // of a piece
    static constexpr int kAPitch = SHIFT ? kPiece + 16 : kPiece;
    static constexpr int kABytes = kRows * kAPitch;
    static constexpr int kB = kK * size_of(XT);          // bytes of a column, a piece
    static constexpr int kChunks = kB / 16;              // 16-byte pieces of it
    static constexpr int kBLoads = 8 * kChunks / 32;     // of a lane, for 8 columns
    static constexpr int kALoads = SHIFT ? 5 : 4;
    static constexpr int kStage = kABytes + NT * 8 * kB;
    static constexpr int kStages = ring_bytes(SHIFT) / kStage > 5 ? 5 : ring_bytes(SHIFT) / kStage;
    static constexpr int kWarpBytes = kStages * kStage;
    static_assert(kStages >= 2, "the ring holds two stages");
    static constexpr bool kWhole = XT == kI8;            // sums are integers
    static constexpr int kRun = 1024 / kK;               // pieces whose products float32 sums exactly

    const int lane, warp;
    const uint32_t ring;
    // loading side
    const char* a_at[kALoads];
    int a_left[kALoads];     // bytes of the row from there on; 0: no such row
    const char* b_at[NT][kBLoads];
    uint32_t b_there;        // which of them there are
    int load_piece, load_last, load_stage;
    // using side
    int use_stage;
    int shift[2][2];         // of this lane's rows

    __device__ __forceinline__ Stream(uint32_t ring_of_cta, int w, int l)
        : lane(l), warp(w), ring(ring_of_cta + w * kWarpBytes), load_piece(0), load_last(0), load_stage(0), use_stage(0)
    {
    }

    // The loading side turns to a unit.  column(c): address of column c's values,
    // nullptr for none; whole pieces of it can be read.
    template <typename Column>
    __device__ __forceinline__ void load_from(const Unit& u, Column column)
    {
#pragma unroll
        for (int i = 0; i < kALoads; i++) {
            const int id = lane + 32 * i, row = SHIFT ? id / 5 : id >> 2, c = SHIFT ? id % 5 : id & 3;
            const bool second = row >= 16;
            const int in = row & 15;
            const char* p = (second ? u.a[1] : u.a[0]) + in * (second ? u.a_stride[1] : u.a_stride[0]);
            const int o = SHIFT ? int(reinterpret_cast<uintptr_t>(p) & 15) : 0;
            const bool there = in < (second ? u.rows_left[1] : u.rows_left[0]);
            a_at[i] = there ? p - o + 16 * c : nullptr;
            a_left[i] = there ? u.row_bytes - 16 * c + o : 0;
        }
        b_there = 0;
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
            for (int j = 0; j < kBLoads; j++) {
                const int id = lane + 32 * j;
                const char* p = column(n * 8 + id / kChunks);
                b_at[n][j] = p + 16 * (id % kChunks);
                if (p) b_there |= 1u << (n * kBLoads + j);
            }
        load_piece = u.first + warp;
        load_last = u.last;
    }

    __device__ __forceinline__ bool more() const { return load_piece < load_last; }

    // where chunk c of column row r lies: no bank is met twice by the eight lanes
    // that a 16-byte access takes together
    static __device__ __forceinline__ int b_place(int r, int c)
    {
        if (kChunks == 4) return r * kB + 16 * c;
        if (kChunks == 8) return r * kB + 16 * (c ^ (r & 1));
        return r * kB + 16 * (c ^ ((c >> 3) & 1) ^ ((r & 1) << 1));
    }

    // `any`: an address that can be read, for copies of nothing
    __device__ __forceinline__ void load(const char* any)
    {
        const uint32_t to = ring + load_stage * kStage;
        const int off = load_piece * kPiece;
#pragma unroll
        for (int i = 0; i < kALoads; i++) {
            const int id = lane + 32 * i, row = SHIFT ? id / 5 : id >> 2, c = SHIFT ? id % 5 : id & 3;
            const int bytes = max(0, min(16, a_left[i] - off));
            copy16(to + row * kAPitch + 16 * c, bytes > 0 ? a_at[i] + off : any, bytes);
        }
        const int64_t b_off = int64_t(load_piece) * kB;
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
            for (int j = 0; j < kBLoads; j++) {
                const int id = lane + 32 * j;
                const bool there = b_there >> (n * kBLoads + j) & 1;
                copy16(to + kABytes + b_place(n * 8 + id / kChunks, id % kChunks), there ? b_at[n][j] + b_off : any,
                       there ? 16 : 0);
            }
        load_piece += kWarps;
        if (++load_stage == kStages) load_stage = 0;
    }

    __device__ __forceinline__ void use_from(const Unit& u)
    {
        if (SHIFT)
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int h = 0; h < 2; h++)
                    shift[i][h] = int((reinterpret_cast<uintptr_t>(u.a[i]) + (lane / 4 + 8 * h) * u.a_stride[i]) & 15);
    }

    __device__ __forceinline__ uint4 a_lane(uint32_t at, int i, int h) const
    {
        const uint32_t p = at + (i * 16 + h * 8 + lane / 4) * kAPitch + 16 * (lane & 3);
        return SHIFT ? shifted(load16(p), load16(p + 16), shift[i][h]) : load16(p);
    }

    // One piece's products
    __device__ __forceinline__ void use(float (&acc)[2][NT][4])
    {
        const uint32_t at = ring + use_stage * kStage, b0 = at + kABytes;
        const int g = lane / 4, t = lane & 3;
        if (++use_stage == kStages) use_stage = 0;
        if constexpr (XT == kF32) {
            constexpr int kEach = kK / 4;   // elements of a lane
#pragma unroll
            for (int part = 0; part < kEach / 8; part++) {   // eight elements at a time
                float a[2][2][8];
#pragma unroll
                for (int i = 0; i < 2; i++)
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        const uint4 v = a_lane(at, i, h);
                        if (WT == kI8) {
                            float f[4];
                            bytes_to_f32(part ? v.z : v.x, f);
#pragma unroll
                            for (int k = 0; k < 4; k++) a[i][h][k] = f[k];
                            bytes_to_f32(part ? v.w : v.y, f);
#pragma unroll
                            for (int k = 0; k < 4; k++) a[i][h][4 + k] = f[k];
                        } else {
                            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int k = 0; k < 4; k++) {
                                if (WT == kF16) {
                                    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
                                    a[i][h][2 * k] = p.x, a[i][h][2 * k + 1] = p.y;
                                } else {
                                    a[i][h][2 * k] = __uint_as_float(w[k] << 16);
                                    a[i][h][2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
                                }
                            }
                        }
                    }
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    float hi[8], lo[8];
#pragma unroll
                    for (int q = 0; q < 2; q++) {
                        const uint4 v = load16(b0 + b_place(n * 8 + g, kEach / 4 * t + 2 * part + q));
                        split_tf32(__uint_as_float(v.x), hi[4 * q], lo[4 * q]);
                        split_tf32(__uint_as_float(v.y), hi[4 * q + 1], lo[4 * q + 1]);
                        split_tf32(__uint_as_float(v.z), hi[4 * q + 2], lo[4 * q + 2]);
                        split_tf32(__uint_as_float(v.w), hi[4 * q + 3], lo[4 * q + 3]);
                    }
#pragma unroll
                    for (int i = 0; i < 2; i++)
#pragma unroll
                        for (int s = 0; s < 4; s++) {
                            mma_tf32(acc[i][n], a[i][0][2 * s], a[i][1][2 * s], a[i][0][2 * s + 1], a[i][1][2 * s + 1],
                                     lo[2 * s], lo[2 * s + 1]);
                            mma_tf32(acc[i][n], a[i][0][2 * s], a[i][1][2 * s], a[i][0][2 * s + 1], a[i][1][2 * s + 1],
                                     hi[2 * s], hi[2 * s + 1]);
                        }
                }
            }
        } else {
            // words of two elements: four a lane and row, of 8-bit weights eight
            constexpr int kWords = kK / 8;
            uint32_t a[2][2][kWords];
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const uint4 v = a_lane(at, i, h);
                    if constexpr (WT == kI8) {
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            if (XT == kBf16) bytes_to_bf16(w[k], a[i][h][2 * k], a[i][h][2 * k + 1]);
                            else bytes_to_f16(w[k], a[i][h][2 * k], a[i][h][2 * k + 1]);
                        }
                    } else {
                        a[i][h][0] = v.x, a[i][h][1] = v.y, a[i][h][2] = v.z, a[i][h][3] = v.w;
                    }
                }
#pragma unroll
            for (int n = 0; n < NT; n++) {
                uint32_t b[kWords];
                if constexpr (XT == kI8) {
                    const uint4 v = load16(b0 + b_place(n * 8 + g, t));
                    bytes_to_f16(v.x, b[0], b[1]);
                    bytes_to_f16(v.y, b[2], b[3]);
                    bytes_to_f16(v.z, b[4], b[5]);
                    bytes_to_f16(v.w, b[6], b[7]);
                } else {
#pragma unroll
                    for (int q = 0; q < kWords / 4; q++) {
                        const uint4 v = load16(b0 + b_place(n * 8 + g, kWords / 4 * t + q));
                        b[4 * q] = v.x, b[4 * q + 1] = v.y, b[4 * q + 2] = v.z, b[4 * q + 3] = v.w;
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; i++)
#pragma unroll
                    for (int s = 0; s < kWords / 2; s++)
                        mma16<XT>(acc[i][n], a[i][0][2 * s], a[i][1][2 * s], a[i][0][2 * s + 1], a[i][1][2 * s + 1],
                                  b[2 * s], b[2 * s + 1]);
            }
        }
    }

    // This warp's sums over its pieces of unit u.  next(): the loading side turns
    // to the unit behind the one that it is at, if there is one.
    template <typename Next>
    __device__ __forceinline__ void sums(const Unit& u, float (&total)[2][NT][4], const char* any, Next next)
    {
        use_from(u);
        float acc[2][NT][4];
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int q = 0; q < 4; q++) acc[i][n][q] = total[i][n][q] = 0.0f;
        int run = 0;
        for (int piece = u.first + warp; piece < u.last; piece += kWarps) {
            copies_wait<kStages - 2>();
            __syncwarp();   // every lane's copies are there, and the stage before is free
            if (!more()) next();
            if (more()) load(any);
            copies_group();
            use(acc);
            if (kWhole && ++run == kRun) run = 0, take(acc, total);
        }
        take(acc, total);
    }

    // sums of a run to the total
    static __device__ __forceinline__ void take(float (&acc)[2][NT][4], float (&total)[2][NT][4])
    {
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    if (kWhole)
                        total[i][n][q] =
                            __int_as_float(__float_as_int(total[i][n][q]) + __float2int_rn(acc[i][n][q]));
                    else
                        total[i][n][q] += acc[i][n][q];
                    acc[i][n][q] = 0.0f;
                }
    }

    // fills the ring ahead of the first unit
    template <typename Next>
    __device__ __forceinline__ void begin(const char* any, Next next)
    {
#pragma unroll
        for (int i = 0; i < kStages - 1; i++) {
            if (!more()) next();
            if (more()) load(any);
            copies_group();
        }
    }
};

// The eight warps' sums of 8 columns, joined in the order of the warps: thread
// `threadIdx.x` gets those of row threadIdx.x % 32, column threadIdx.x / 32.  `room`:
// kJoin floats of shared memory.
constexpr int kJoinPitch = kRows + 4;                     // floats of a column
constexpr int kJoin = kWarps * 8 * kJoinPitch;

template <bool WHOLE>
__device__ __forceinline__ float join_columns(float* room, const float (&first)[4], const float (&second)[4], int warp,
                                              int lane)
{
    const int g = lane / 4, t = lane & 3;
    float* mine = room + warp * 8 * kJoinPitch;
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const int row = g + 8 * (q >> 1), column = 2 * t + (q & 1);
        mine[column * kJoinPitch + row] = first[q];
        mine[column * kJoinPitch + 16 + row] = second[q];
    }
    __syncthreads();
    const float* at = room + (threadIdx.x / kRows) * kJoinPitch + threadIdx.x % kRows;
    float v[kWarps];
#pragma unroll
    for (int w = 0; w < kWarps; w++) v[w] = at[w * 8 * kJoinPitch];
    __syncthreads();
    if (WHOLE) {
        int s = __float_as_int(v[0]);
#pragma unroll
        for (int w = 1; w < kWarps; w++) s += __float_as_int(v[w]);
        return __int_as_float(s);
    }
    float s = v[0];
#pragma unroll
    for (int w = 1; w < kWarps; w++) s += v[w];
    return s;
}

// Whether this CTA is the last of `all` to come to a counter, which it then sets
// back to zero; what the others wrote before they came is visible to it.
__device__ __forceinline__ bool last_to_come(uint32_t* counter, uint32_t all)
{
    __shared__ uint32_t came;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        came = atomicAdd(counter, 1u) + 1u;
        if (came == all) *counter = 0u;
        __threadfence();
    }
    __syncthreads();
    return came == all;
}

}  // namespace stream
}  // namespace dpdr
