// 32-bit values in products with 16-bit data.
#pragma once
#include "tile.hpp"

namespace nsl {

// A fragment as a sum of fragments of the matrix cores' type, the largest
// first. bfloat16 and float32 data are one piece, float16 data (whose range
// the sums would leave) two of bfloat16, without loss; 32-bit values that meet
// 16-bit data are N pieces of bfloat16, 8 bits each. Products leave out what
// is below the last piece's rounding.
template <class F, int N> struct Pieces { F p[N]; };
template <class T> constexpr int data_pieces() { return std::is_same<T, _Float16>::value ? 2 : 1; }
template <class T> using piece = std::conditional_t<std::is_same<T, float>::value, f8, b8>;

// All but the last piece are the value's next 8 bits as they are (two values'
// upper halves are one instruction), the last one is rounded.
template <int N> __device__ inline Pieces<b8, N> cut(f8 x) {
    Pieces<b8, N> r;
#pragma unroll
    for (int i = 0; i + 1 < N; ++i) {
        u4 u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float even = x[2 * j], odd = x[2 * j + 1];
            const unsigned e = __builtin_bit_cast(unsigned, even), o = __builtin_bit_cast(unsigned, odd);
            u[j] = __builtin_amdgcn_perm(o, e, 0x07060302u);
            x[2 * j] = even - __builtin_bit_cast(float, e & 0xffff0000u);
            x[2 * j + 1] = odd - __builtin_bit_cast(float, o & 0xffff0000u);
        }
        r.p[i] = __builtin_bit_cast(b8, u);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) r.p[N - 1][j] = static_cast<__bf16>(x[j]);
    return r;
}
__device__ inline f8 wide_of(f8 f) { return f; }
template <class F> __device__ inline f8 wide_of(F f) {
    f8 x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = static_cast<float>(f[j]);
    return x;
}
__device__ inline Pieces<f8, 1> data_of(f8 f) { return {{f}}; }
__device__ inline Pieces<b8, 1> data_of(b8 f) { return {{f}}; }
__device__ inline Pieces<b8, 2> data_of(h8 f) { return cut<2>(wide_of(f)); }
template <class T, int N> __device__ inline auto sum_of(f8 x) {
    if constexpr (sizeof(T) == 4)
        return Pieces<f8, 1>{{x}};
    else
        return cut<N>(x);
}

template <class F, int NA, int NB>
__device__ inline acc16 product(const Pieces<F, NA>& a, const Pieces<F, NB>& b, acc16 c) {
    constexpr int kLast = NA > NB ? NA : NB;
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            if (i + j < kLast) c = mma(a.p[i], b.p[j], c);
    return c;
}

__device__ inline f8 octet(const acc16& c, int s) {
    f8 x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = c[8 * s + j];
    return x;
}

}  // namespace nsl
