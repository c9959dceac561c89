// stream.cuh -- products of a few columns with weights that stream past once:
// what the kernels for a few tokens (experts.cu, integer.cu) share.
//
// D[row][column] = sum_k A[row][k] B[column][k] for 32 rows of A (weights: 32 of
// one matrix, or 16 of either of two) and 8 NT columns (tokens).  With so few
// columns the weights' bytes are the bound, and what matters is that some 100 KB
// an SM are always under way.  Each warp loads pieces of 64 bytes along k of its rows,
// beside the columns that go with them, into a ring of its own by cp.async, several
// pieces ahead and across the ends of units, and no warp waits for another until its
// sums are done.  (Rows copied by cp.async.bulk instead reached 4.1 TB/s with 1 KB a
// copy, an issuing warp making one in 70 cycles.)
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
//   columns as terms of bfloat16 that add up to a float32 value: a product each.
//   float32 columns with float16 weights, which such terms cannot meet: A widened to
//     tf32, exactly, and each column value split into two of 11 bits (the second
//     cut off, 2^-21 of the value), two products.
// SHIFT: rows of A at any address.  The aligned 16 bytes around what a lane needs
// are copied, read by words and shifted in registers (8 rows of 64 experts of 2001 x
// 1003 96 us; two reads of 16 bytes and a choice among their words 100).  What lies
// behind the end of a row is never read (cp.async fills up with zeros).
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
constexpr int kRing = 12288;            // bytes, a warp: two CTAs an SM

constexpr int size_of(int kind) { return kind == kI8 ? 1 : kind == kF32 ? 4 : 2; }

__device__ __forceinline__ uint32_t shared_at(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }

// 16 bytes, of which the first `bytes` are read and the others are zero
__device__ __forceinline__ void copy16(uint32_t to, const char* from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t to, const char* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
// The same of a row that is read on from there: what lies beside it goes to L2 too, 256
// bytes, which DRAM serves at a better rate than 64 (8 rows of 64 experts 113 to 106 us).
__device__ __forceinline__ void copy16_on(uint32_t to, const char* from)
{
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
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

// 16 bytes at any place
__device__ __forceinline__ uint4 load16_at(uint32_t at)
{
    const uint32_t p = at & ~3u, b = 8 * (at & 3u);
    uint32_t w[5];
#pragma unroll
    for (int i = 0; i < 5; i++) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[i]) : "r"(p + 4 * i));
    return make_uint4(__funnelshift_r(w[0], w[1], b), __funnelshift_r(w[1], w[2], b), __funnelshift_r(w[2], w[3], b),
                      __funnelshift_r(w[3], w[4], b));
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

// Four 8-bit integers as float16, by the known way of putting a whole number into the
// low bits of a float whose last bit counts one: 1024 + (v + 128) has v + 128 there
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

// ---------------------------------------------------- matrix instructions

// d = a b + c
template <int XT>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                      uint32_t b1, float c0, float c1, float c2, float c3)
{
    if (XT == kBf16)
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%10, %11, %12, %13};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
    else
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%10, %11, %12, %13};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
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

// h as three bfloat16 values of 8 bits each that add up to it.  Infinities and NaN
// have one.
__device__ __forceinline__ void split_bf16(float h, uint16_t (&t)[3])
{
    const uint32_t b = __float_as_uint(h);
    t[0] = uint16_t(b >> 16);
    t[1] = t[2] = 0;
    if ((b & 0x7F800000u) == 0x7F800000u) {
        if (h != h) t[0] |= 0x40;   // the bit that tells may be among those cut off
        return;
    }
    const float r = h - __uint_as_float(b & 0xFFFF0000u);
    const uint32_t c = __float_as_uint(r);
    t[1] = uint16_t(c >> 16);
    t[2] = uint16_t(__float_as_uint(r - __uint_as_float(c & 0xFFFF0000u)) >> 16);
}

// ---------------------------------------------------------------- a unit

// Where a unit's operands lie.  A's row r (0 .. 31) is row r of the first 16 at
// a[0], the others at a[1].  Rows past rows_left[.] repeat the last, for nothing
// that is used; of none the others are taken.
struct Unit {
    const char* a[2];
    int64_t a_stride[2];     // bytes from row to row
    int rows_left[2];        // rows that there are, of 16; rows_left[0] >= 1
    int row_bytes;
    int first, last;         // pieces along k
    uint32_t counts = 0;     // with ZEROS: bits of the columns whose sums are wanted
    __device__ __forceinline__ const char* row(int r) const
    {
        const int in = r & 15;
        if (r >= 16 && rows_left[1] > 0) return a[1] + min(in, rows_left[1] - 1) * a_stride[1];
        return a[0] + min(in, rows_left[0] - 1) * a_stride[0];
    }
};

// TERMS: a column's values are the sums of so many, whose arrays lie `apart`
// bytes from each other.  PIECE: bytes of a row of A, a stage.  STEP: a warp takes
// every STEP-th piece of a unit.  ZEROS: some columns are zeros, whose sums with
// infinities and NaN among the weights are left out.
template <int WT, int XT, int NT, bool SHIFT, int TERMS, int PIECE, int STEP, bool ZEROS = false>
struct Stream {
    static constexpr int kPiece = PIECE;
    static constexpr bool kZeros = ZEROS;
    static constexpr int kParts = kPiece / 64;           // a lane has 16 bytes of a row in each
    static constexpr int kK = 64 / size_of(WT);          // elements of a part
    static constexpr int kAChunks = kPiece / 16 + SHIFT; // 16-byte chunks of a row
    static constexpr int kAPitch = 16 * kAChunks;
    static constexpr int kABytes = kRows * kAPitch;
    static constexpr int kB = kParts * kK * size_of(XT); // bytes of a column, a piece
    static constexpr int kBChunks = kB / 16;
    static constexpr int kBLoads = 8 * kBChunks / 32;    // of a lane, for 8 columns
    static constexpr int kALoads = kAChunks;
    static constexpr int kBTerm = NT * 8 * kB;
    static constexpr int kStage = kABytes + TERMS * kBTerm;
    static constexpr int kStages = kRing / kStage > 5 ? 5 : kRing / kStage;
    static constexpr int kWarpBytes = kStages * kStage;
    static_assert(kStages >= 2, "the ring holds two stages");
    static_assert(!SHIFT || kALoads <= 8, "four bits a load");
    static constexpr bool kWhole = XT == kI8;            // sums are integers
    static constexpr int kRun = 1024 / (kParts * kK);    // pieces whose products float32 sums exactly

    const int lane, warp;
    const uint32_t ring;
    // loading side
    const char* a_at[kALoads];
    const char* b_at[NT * kBLoads];
    int b_bytes[NT * kBLoads];   // 0: a column of zeros
    int64_t apart;
    int load_piece, load_last, load_whole;   // pieces before load_whole are inside every row
    int load_bytes, load_shift;              // of a row; of the loads, four bits each
    uint32_t load_to, load_end;
    // using side
    uint32_t use_from_here;
    int shift[2][2];         // of this lane's rows
    bool counts[2];          // this lane's columns

    __device__ __forceinline__ Stream(uint32_t ring_of_cta, int w, int l, int64_t terms_apart = 0)
        : lane(l),
          warp(w),
          ring(ring_of_cta + w * kWarpBytes),
          apart(terms_apart),
          load_piece(0),
          load_last(0),
          load_to(ring),
          load_end(ring + kWarpBytes),
          use_from_here(ring)
    {
    }

    // the row and chunk of a lane's i-th 16 bytes of A, and where they go
    __device__ __forceinline__ int a_row(int i) const { return int((unsigned(lane) + 32 * i) / kAChunks); }
    __device__ __forceinline__ int a_chunk(int i) const { return int((unsigned(lane) + 32 * i) % kAChunks); }
    __device__ __forceinline__ uint32_t a_to(int i) const
    {
        if (SHIFT || kParts == 1) return 16 * lane + 512 * i;
        return (16 * lane ^ (lane & 8) << 3) + 512 * i;
    }

    // The loading side turns to pieces u.first (to u.last) of a unit.  column(c):
    // address of column c's values, for any c; whole pieces of it can be read.  With
    // ZEROS nullptr: a column of zeros.
    template <typename Column>
    __device__ __forceinline__ void load_from(const Unit& u, Column column)
    {
        load_piece = u.first;
        load_last = u.last;
        load_bytes = u.row_bytes;
        load_whole = (u.row_bytes - (SHIFT ? 16 : 0)) / kPiece;
#pragma unroll
        for (int i = 0; i < kALoads; i++) {
            const char* p = u.row(a_row(i)) + load_piece * kPiece + 16 * a_chunk(i);
            a_at[i] = SHIFT ? p - int(reinterpret_cast<uintptr_t>(p) & 15) : p;
        }
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
            for (int j = 0; j < kBLoads; j++) {
                const unsigned id = lane + 32 * j;
                const char* p = column(n * 8 + id / kBChunks);
                if (ZEROS) {
                    b_bytes[n * kBLoads + j] = p ? 16 : 0;
                    if (!p) p = u.a[0] - int(reinterpret_cast<uintptr_t>(u.a[0]) & 15);   // any address
                }
                b_at[n * kBLoads + j] = p + load_piece * kB + 16 * (id % kBChunks);
            }
        if (SHIFT) {   // what the last pieces have to know of each row
            load_shift = 0;
#pragma unroll
            for (int i = 0; i < kALoads; i++)
                load_shift |= int(reinterpret_cast<uintptr_t>(u.row(a_row(i))) & 15) << 4 * i;
        }
    }

    __device__ __forceinline__ bool more() const { return load_piece < load_last; }

    // Where chunk c of column r's piece lies: no bank is met twice by the eight lanes
    // that a 16-byte access takes together, which have two columns next to each other
    // and chunks kBChunks / 4 / kParts apart.
    static __device__ __forceinline__ int b_place(int r, int c)
    {
        constexpr int kApart = kBChunks / kParts / 4;   // chunks of a lane in a part
        static_assert(kApart == 1 || kApart == 2, "one or two");
        if (kApart == 1) return r * kB + 16 * (kParts == 1 ? c : c ^ ((r & 1) << 2));
        return r * kB + 16 * (c ^ (r & 1));
    }
    static __device__ __forceinline__ int a_place(int r, int c)
    {
        return r * kAPitch + 16 * (SHIFT || kParts == 1 ? c : c ^ ((r & 1) << 2));
    }

    __device__ __forceinline__ void load()
    {
        if (load_piece < load_whole) {
#pragma unroll
            for (int i = 0; i < kALoads; i++) copy16_on(load_to + a_to(i), a_at[i]);
        } else {
            const int left = load_bytes - load_piece * kPiece;
#pragma unroll
            for (int i = 0; i < kALoads; i++) {
                const int o = SHIFT ? load_shift >> 4 * i & 15 : 0;
                const int bytes = max(0, min(16, left + o - 16 * a_chunk(i)));
                // of none, the address of the row's first bytes in this piece
                copy16(load_to + a_to(i), a_at[i] - (bytes > 0 ? 0 : 16 * a_chunk(i)), bytes);
            }
        }
#pragma unroll
        for (int i = 0; i < kALoads; i++) a_at[i] += STEP * kPiece;
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
            for (int j = 0; j < kBLoads; j++) {
                const unsigned id = lane + 32 * j;
                const uint32_t to = load_to + kABytes + b_place(n * 8 + id / kBChunks, id % kBChunks);
#pragma unroll
                for (int t = 0; t < TERMS; t++) {
                    const char* from = b_at[n * kBLoads + j] + t * apart;
                    if (ZEROS) copy16(to + t * kBTerm, from, b_bytes[n * kBLoads + j]);
                    else copy16(to + t * kBTerm, from);
                }
                b_at[n * kBLoads + j] += STEP * kB;
            }
        load_piece += STEP;
        load_to += kStage;
        if (load_to == load_end) load_to = ring;
    }

    __device__ __forceinline__ void use_from(const Unit& u)
    {
        if (ZEROS) {
            static_assert(!ZEROS || NT == 1, "a bit a column");
            counts[0] = u.counts >> 2 * (lane & 3) & 1u;
            counts[1] = u.counts >> 2 * (lane & 3) & 2u;
        }
        if (SHIFT)
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int h = 0; h < 2; h++)
                    shift[i][h] = int(reinterpret_cast<uintptr_t>(u.row(16 * i + lane / 4 + 8 * h)) & 15);
    }

    __device__ __forceinline__ uint4 a_lane(uint32_t at, int part, int i, int h) const
    {
        const int r = i * 16 + h * 8 + lane / 4, c = 4 * part + (lane & 3);
        if (SHIFT) return load16_at(at + a_place(r, c) + shift[i][h]);
        return load16(at + a_place(r, c));
    }

    // One piece's products, added to the sums; of whole numbers to the run's
    __device__ __forceinline__ void use(float (&sum)[2][NT][4])
    {
        const uint32_t at = use_from_here, b0 = at + kABytes;
        const int g = lane / 4, t = lane & 3;
        use_from_here += kStage;
        if (use_from_here == load_end) use_from_here = ring;
        if constexpr (XT == kF32) {
            // 11 and 11 bits of a column's values, each with sums of its own
            static_assert(WT == kF16, "other weights take terms of bfloat16");
            float high[2][NT][4], low[2][NT][4];
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int n = 0; n < NT; n++)
#pragma unroll
                    for (int q = 0; q < 4; q++) high[i][n][q] = low[i][n][q] = 0.0f;
#pragma unroll
            for (int part = 0; part < kParts; part++) {
                float a[2][2][8];
#pragma unroll
                for (int i = 0; i < 2; i++)
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        const uint4 v = a_lane(at, part, i, h);
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
                            a[i][h][2 * k] = p.x, a[i][h][2 * k + 1] = p.y;
                        }
                    }
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    float hi[8], lo[8];
#pragma unroll
                    for (int q = 0; q < 2; q++) {
                        const uint4 v = load16(b0 + b_place(n * 8 + g, 8 * part + 2 * t + q));
                        split_tf32(__uint_as_float(v.x), hi[4 * q], lo[4 * q]);
                        split_tf32(__uint_as_float(v.y), hi[4 * q + 1], lo[4 * q + 1]);
                        split_tf32(__uint_as_float(v.z), hi[4 * q + 2], lo[4 * q + 2]);
                        split_tf32(__uint_as_float(v.w), hi[4 * q + 3], lo[4 * q + 3]);
                    }
#pragma unroll
                    for (int s = 0; s < 4; s++)
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            mma_tf32(low[i][n], a[i][0][2 * s], a[i][1][2 * s], a[i][0][2 * s + 1], a[i][1][2 * s + 1],
                                     lo[2 * s], lo[2 * s + 1]);
                            mma_tf32(high[i][n], a[i][0][2 * s], a[i][1][2 * s], a[i][0][2 * s + 1], a[i][1][2 * s + 1],
                                     hi[2 * s], hi[2 * s + 1]);
                        }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int n = 0; n < NT; n++)
#pragma unroll
                    for (int q = 0; q < 4; q++)
                        if (!ZEROS || counts[q & 1]) sum[i][n][q] += high[i][n][q] + low[i][n][q];
        } else {
            // words of two elements: four a lane and row, of 8-bit weights eight
            constexpr int kWords = kK / 8;
#pragma unroll
            for (int part = 0; part < kParts; part++) {
                uint32_t a[2][2][kWords];
#pragma unroll
                for (int i = 0; i < 2; i++)
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        const uint4 v = a_lane(at, part, i, h);
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
                    // a chain of products for each of the two groups of rows
                    float d[2][4];
                    bool first = !kWhole;
#pragma unroll
                    for (int term = TERMS - 1; term >= 0; term--) {   // the smallest first
                        uint32_t b[kWords];
                        if constexpr (XT == kI8) {
                            const uint4 v = load16(b0 + b_place(n * 8 + g, 4 * part + t));
                            bytes_to_f16(v.x, b[0], b[1]);
                            bytes_to_f16(v.y, b[2], b[3]);
                            bytes_to_f16(v.z, b[4], b[5]);
                            bytes_to_f16(v.w, b[6], b[7]);
                        } else {
#pragma unroll
                            for (int q = 0; q < kWords / 4; q++) {
                                const uint4 v =
                                    load16(b0 + term * kBTerm + b_place(n * 8 + g, kWords * part + kWords / 4 * t + q));
                                b[4 * q] = v.x, b[4 * q + 1] = v.y, b[4 * q + 2] = v.z, b[4 * q + 3] = v.w;
                            }
                        }
#pragma unroll
                        for (int s = 0; s < kWords / 2; s++)
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                float(&c)[4] = kWhole ? sum[i][n] : d[i];
                                const bool zero = first && s == 0;
                                mma16<XT>(c, a[i][0][2 * s], a[i][1][2 * s], a[i][0][2 * s + 1], a[i][1][2 * s + 1],
                                          b[2 * s], b[2 * s + 1], zero ? 0.0f : c[0], zero ? 0.0f : c[1],
                                          zero ? 0.0f : c[2], zero ? 0.0f : c[3]);
                            }
                        first = false;
                    }
                    if (!kWhole)
#pragma unroll
                        for (int i = 0; i < 2; i++)
#pragma unroll
                            for (int q = 0; q < 4; q++)
                                if (!ZEROS || counts[q & 1]) sum[i][n][q] += d[i][q];
                }
            }
        }
    }

    // The products of the next pieces of a unit, added to `total`.  next(): the
    // loading side turns to what comes behind the pieces that it is at, if anything.
    // The instructions cut sums off, so each part's products are summed by
    // themselves and added up rounded; whole numbers in `run` first.
    template <typename Next>
    __device__ __forceinline__ void sums(const Unit& u, float (&total)[2][NT][4], Next next)
    {
        use_from(u);
        float run[2][NT][4];
        if (kWhole) clear(run);
        int done = 0;
        for (int piece = u.first; piece < u.last; piece += STEP) {
            copies_wait<kStages - 2>();
            __syncwarp();   // every lane's copies are there, and the stage before is free
            if (!more()) next();
            if (more()) load();
            copies_group();
            if (kWhole) {
                use(run);
                if (++done == kRun) done = 0, take(run, total);
            } else {
                use(total);
            }
        }
        if (kWhole) take(run, total);
    }

    static __device__ __forceinline__ void clear(float (&v)[2][NT][4])
    {
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int q = 0; q < 4; q++) v[i][n][q] = 0.0f;
    }

    // whole numbers of a run to the total, which is held as integers
    static __device__ __forceinline__ void take(float (&run)[2][NT][4], float (&total)[2][NT][4])
    {
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    total[i][n][q] = __int_as_float(__float_as_int(total[i][n][q]) + __float2int_rn(run[i][n][q]));
                    run[i][n][q] = 0.0f;
                }
    }

    // fills the ring ahead of the first unit
    template <typename Next>
    __device__ __forceinline__ void begin(Next next)
    {
#pragma unroll
        for (int i = 0; i < kStages - 1; i++) {
            if (!more()) next();
            if (more()) load();
            copies_group();
        }
    }
};

constexpr int kJoinPitch = kRows + 4;                     // floats of a column
constexpr int kTile = 8 * kJoinPitch;                     // of a warp
constexpr int kJoin = kWarps * kTile;

// A warp's sums of 8 columns to its tile, column by column
__device__ __forceinline__ void put_tile(float* tile, const float (&first)[4], const float (&second)[4], int lane)
{
    const int g = lane / 4, t = lane & 3;
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const int row = g + 8 * (q >> 1), column = 2 * t + (q & 1);
        tile[column * kJoinPitch + row] = first[q];
        tile[column * kJoinPitch + 16 + row] = second[q];
    }
}

// and those of a tile added to a warp's
__device__ __forceinline__ void add_tile(const float* tile, float (&first)[4], float (&second)[4], int lane)
{
    const int g = lane / 4, t = lane & 3;
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const int row = g + 8 * (q >> 1), column = 2 * t + (q & 1);
        first[q] += tile[column * kJoinPitch + row];
        second[q] += tile[column * kJoinPitch + 16 + row];
    }
}

// The eight warps' sums of 8 columns, held as integers, added up: thread `threadIdx.x` gets
// those of row threadIdx.x % 32, column threadIdx.x / 32.  `room`: kJoin floats of shared
// memory.
__device__ __forceinline__ int join_columns(float* room, const float (&first)[4], const float (&second)[4], int warp,
                                            int lane)
{
    put_tile(room + warp * kTile, first, second, lane);
    __syncthreads();
    const float* at = room + (threadIdx.x / kRows) * kJoinPitch + threadIdx.x % kRows;
    float v[kWarps];
#pragma unroll
    for (int w = 0; w < kWarps; w++) v[w] = at[w * kTile];
    __syncthreads();
    int s = __float_as_int(v[0]);
#pragma unroll
    for (int w = 1; w < kWarps; w++) s += __float_as_int(v[w]);
    return s;
}

// One more on a counter, and what it was: what the thread knows to be written is
// visible to whoever adds later, and what was written before earlier ones to it.
__device__ __forceinline__ uint32_t add_in_order(uint32_t* counter)
{
    uint32_t was;
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(was) : "l"(counter) : "memory");
    return was;
}

// Whether this CTA is the last of `all` to come to a counter, which it then sets
// back to zero; what the others wrote before they came is visible to it.
__device__ __forceinline__ bool last_to_come(uint32_t* counter, uint32_t all)
{
    __shared__ uint32_t came;
    __syncthreads();
    if (threadIdx.x == 0) {
        came = add_in_order(counter) + 1u;
        if (came == all) *counter = 0u;
    }
    __syncthreads();
    return came == all;
}

// ------------------------------------------------------------ equal shares

// `total` pieces dealt out to `of` warps, each a contiguous share; units of `each`
// pieces may lie in several.
constexpr int kLeast = 4;   // pieces a warp, where there are fewer than warps
struct Shares {
    int total, of, each;
    int most, long_ones, behind;   // the first long_ones warps have one more than most, up to piece `behind`
    __device__ __forceinline__ Shares(int all, int warps, int unit)
        : total(all),
          of(warps),
          each(unit),
          most(all / warps),
          long_ones(all - most * warps),
          behind(long_ones * (most + 1))
    {
    }
    __device__ __forceinline__ int start(int w) const { return w * most + min(w, long_ones); }
    __device__ __forceinline__ int owner(int piece) const
    {
        return piece < behind ? piece / (most + 1) : long_ones + (piece - behind) / most;
    }
};

// Fewer units than warps: a team of warps a unit, one after another, teams of equal
// size (or one more), of no more warps than have a few pieces each.
struct Teams {
    int units, of, each;   // units, warps, pieces a unit
    __device__ __forceinline__ int start(int u) const { return u * of / units; }
    __device__ __forceinline__ int unit(int w) const { return ((w + 1) * units - 1) / of; }
    __device__ __forceinline__ int size(int u) const { return min(start(u + 1) - start(u), max(1, each / kLeast)); }
};

// Sums of a unit that several contributors have parts of -- warps, or CTAs -- added up
// in the order of these by the last of them to come, which gets true.  Each has two
// places: place(c) is contributor c's for this unit.  count: the unit's counter,
// zero.
template <int NT, typename Place>
__device__ __forceinline__ bool join_parts(float (&v)[2][NT][4], int me, int first, int last, Place place,
                                           uint32_t* count, int lane)
{
    float4* mine = reinterpret_cast<float4*>(place(me)) + lane;
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int n = 0; n < NT; n++)
            mine[(i * NT + n) * 32] = make_float4(v[i][n][0], v[i][n][1], v[i][n][2], v[i][n][3]);
    __syncwarp();
    uint32_t came = 0;
    if (lane == 0) {
        came = add_in_order(count) + 1u;
        if (came == uint32_t(last - first + 1)) *count = 0u;
    }
    came = __shfl_sync(0xFFFFFFFFu, came, 0);
    if (came != uint32_t(last - first + 1)) return false;
    constexpr int kAhead = NT == 1 ? 6 : NT == 2 ? 2 : 1;   // contributors whose sums are asked for together
#pragma unroll 1
    for (int c = first; c <= last; c += kAhead) {
        float4 p[kAhead][2 * NT];
#pragma unroll
        for (int k = 0; k < kAhead; k++) {
            const float4* at = reinterpret_cast<const float4*>(place(min(c + k, last))) + lane;
#pragma unroll
            for (int i = 0; i < 2 * NT; i++)
                p[k][i] = c + k <= last ? __ldcg(at + i * 32) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
#pragma unroll
        for (int k = 0; k < kAhead; k++)
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    const float4 q = p[k][i * NT + n];
                    if (k == 0 && c == first)
                        v[i][n][0] = q.x, v[i][n][1] = q.y, v[i][n][2] = q.z, v[i][n][3] = q.w;
                    else
                        v[i][n][0] += q.x, v[i][n][1] += q.y, v[i][n][2] += q.z, v[i][n][3] += q.w;
                }
    }
    return true;
}

}  // namespace stream
}  // namespace dpdr
