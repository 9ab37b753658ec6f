// The 4-bit form of the block cache, shared by the kernels that write and read it.  Internal to the library.
//
// For every row and every 32 dimensions ("group") a step s = bf16(max|x| / 7) and codes u = round(x / s), halves away from
// zero, so -7 <= u <= 7; the value held is s u.  A step that would be below 2^-126 is 0 (the group is held as zeros), a group
// with a value that is not finite has the step NaN.
//   Rounding.  x and s have 8 significant bits each, x = X 2^a, s = S 2^b, so x / s - (k + 1/2) is a whole number over 2 S 2^j:
// either zero or at least 2^-12 of the quotient (2^-16 for the 127 steps of the 8-bit rows).  The product with
// (1 + 2^-19) / s, off by 2^-22 at most, therefore rounds every quotient as the exact one would be, and a quotient that is a
// half exactly away from zero, without a division for each value.
//
// A tile is 16 rows of 64 dimensions of K and of V, 1152 contiguous bytes (nine 128-byte lines, so a range of rows is one
// bulk copy).  A byte holds dimension 2i in its low half and 2i + 1 in its high half, as u + 8 (1 .. 15), so that one mask gives the attention
// four codes as bytes.  Bytes lie where its matrix fragments want them:
//   bytes    0 ..  511   K: two rows together, 16 dimensions of the even row, the same of the odd one, and so on
//   bytes  512 .. 1023   V: four rows together, their bytes of two dimensions side by side; the eight 16-byte units of a row quad q (eight
//                        dimensions each) in the order unit ^ 2q, which spreads the four quads over the shared-memory banks
//   bytes 1024 .. 1087   K steps, two bf16 a row
//   bytes 1088 .. 1151   V steps
// A (sequence, head) slab is [ceil(N_max / 16)][hd / 64] tiles.
#pragma once

#include "bt_common.cuh"

namespace bt {
namespace kv4 {

constexpr int kTileRows = 16;
constexpr int kTileBytes = 1152;
constexpr int kPartBytes = 512;       // K codes, V codes
constexpr int kStepsAt = 1024;        // K steps; V steps 64 bytes later
constexpr uint32_t kZeroCodes = 0x88888888u;
constexpr float kRoundUpHalves = 1.0f + 1.0f / 524288.0f;   // 1 + 2^-19
constexpr float kLeastStep = 1.17549435e-38f;               // 2^-126

__host__ __device__ __forceinline__ int64_t slab_bytes(int cap, int hd)
{
    return (int64_t)((cap + kTileRows - 1) / kTileRows) * (hd / 64) * kTileBytes;
}

// where the codes of dimensions 8 j .. 8 j + 7 (four bytes) of a row lie: four bytes of K in a word, four of V a word apart
__device__ __forceinline__ int k_codes_at(int row, int j) { return (row >> 1) * 64 + (j >> 1) * 16 + (row & 1) * 8 + (j & 1) * 4; }
__device__ __forceinline__ int v_unit_at(int quad, int j) { return kPartBytes + quad * 128 + (j ^ (2 * quad)) * 16; }
__device__ __forceinline__ int v_codes_at(int row, int j) { return v_unit_at(row >> 2, j) + (row & 3); }

// four words of four bytes each, transposed: the codes of four rows to and from the bytes of a V unit
__device__ __forceinline__ uint4 transpose4x4(const uint4& r)
{
    const uint32_t a = __byte_perm(r.x, r.y, 0x5140), b = __byte_perm(r.z, r.w, 0x5140);   // bytes 0 and 1 of two rows
    const uint32_t c = __byte_perm(r.x, r.y, 0x7362), d = __byte_perm(r.z, r.w, 0x7362);   // bytes 2 and 3
    return make_uint4(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632), __byte_perm(c, d, 0x5410), __byte_perm(c, d, 0x7632));
}

// The larger magnitudes of two pairs of bf16 (their signs mean nothing), NaN where one is.
__device__ __forceinline__ uint32_t magnitude_max(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t magnitude_max8(const uint4& r) { return magnitude_max(magnitude_max(r.x, r.y), magnitude_max(r.z, r.w)); }
// the largest of both halves, as the bits of a magnitude: 0x7f80 and above where it is not finite
__device__ __forceinline__ uint32_t magnitude_of(uint32_t pair)
{
    pair &= 0x7fff7fffu;
    return max(pair & 0xffffu, pair >> 16);
}

__device__ __forceinline__ float reciprocal(float x)   // 2^-23 off at most; x normal
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Step of a group with this largest magnitude, and what its values are multiplied with to get codes.  (The product with 1 / MOST in place of a
// division: A / MOST, A a number of 8 bits, is never half-way between two of those, and 2^-16 of it or more away, so the rounding to
// bf16 is the quotient's.)
struct Step {
    uint32_t bits;   // bf16
    float inv;
    bool finite;
};
template <int MOST>
__device__ __forceinline__ Step step_of_group(uint32_t magnitude)
{
    Step st;
    st.finite = magnitude < 0x7f80u;
    const float s = __bfloat162float(__float2bfloat16_rn(__uint_as_float(magnitude << 16) * (1.0f / MOST)));
    const bool some = st.finite && s >= kLeastStep;
    st.bits = !st.finite ? 0x7fffu : some ? __float_as_uint(s) >> 16 : 0u;
    st.inv = some ? reciprocal(s) * kRoundUpHalves : 0.f;
    return st;
}

// 8 finite values -> 8 codes of four bits.  Adding 1.5 * 2^23 + 8 leaves the code in the low bits, of which two make a byte.
__device__ __forceinline__ uint32_t codes8(const uint4& r, float inv)
{
    constexpr float kWhole = 12582912.0f + 8.0f;
    float f[8];
    unpack8(r, f);
    uint32_t t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = __float_as_uint(fmaf(f[i], inv, kWhole));
#pragma unroll
    for (int i = 0; i < 8; i += 2) t[i] += t[i + 1] * 16u;   // the low byte
    return __byte_perm(__byte_perm(t[0], t[2], 0x0040), __byte_perm(t[4], t[6], 0x0040), 0x5410);
}

// Four lanes hold a group (8 values each): its step, on all four of them.
__device__ __forceinline__ Step step_of_lanes(const uint4& r)
{
    uint32_t m = magnitude_max8(r);
    m = magnitude_max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = magnitude_max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    return step_of_group<7>(magnitude_of(m));
}

// 8 codes -> 8 bf16 values: code - 8 is exact in bf16 (as 128 + code less 136), the product with the step is rounded once.
__device__ __forceinline__ uint4 values8(uint32_t codes, uint32_t step)
{
    const uint32_t s2 = __byte_perm(step, 0u, 0x1010);
    uint32_t v[4];   // dimensions i and i + 4
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = ((codes >> (4 * i)) & 0x000f000fu) | 0x43004300u;
        asm("{\n\t.reg .b32 u;\n\tsub.rn.bf16x2 u, %1, %2;\n\tmul.rn.bf16x2 %0, u, %3;\n\t}" : "=r"(v[i]) : "r"(x), "r"(0x43084308u), "r"(s2));
    }
    return make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
}

// Division of numbers below 2^31 by a launch's constant: the high word of a product with ceil(2^k / d), k = 31 + bits of d - 1.
struct Divisor {
    uint32_t mul, shift;   // mul == 0: by one
};
inline Divisor divisor_of(uint32_t d)
{
    if (d <= 1) return {0u, 0u};
    uint32_t bits = 0;
    while ((1ull << bits) < d) ++bits;
    return {(uint32_t)(((1ull << (31 + bits)) + d - 1) / d), bits - 1};
}
__device__ __forceinline__ int divide(int n, const Divisor& d) { return d.mul ? (int)(__umulhi((uint32_t)n, d.mul) >> d.shift) : n; }

}  // namespace kv4
}  // namespace bt
