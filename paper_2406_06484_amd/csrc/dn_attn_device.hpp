// Device-side pieces that the attention operators share: 16-byte words of a row, row sums, 8-bit conversion, the map from a packed
// row to its sequence.
#pragma once
#include "dn_attn_host.hpp"
#include "dn_device.hpp"

namespace dn {

struct fp8 {}; // e4m3 pages

template <typename T> __device__ inline void unpack16(const uint4 &w, float (&f)[16 / sizeof(T)]) {
    const unsigned d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) f[i] = __uint_as_float(d[i]);
        else { f[2 * i] = __uint_as_float(d[i] << 16); f[2 * i + 1] = __uint_as_float(d[i] & 0xffff0000u); }
    }
}
template <typename T> __device__ inline uint4 pack16(const float (&f)[16 / sizeof(T)]) {
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
    vec v;
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i) v[i] = (T)f[i];
    return __builtin_bit_cast(uint4, v);
}

__device__ inline uint2 to_fp8x8(const float (&f)[8]) {
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[4], f[5], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[6], f[7], hi, true);
    return make_uint2((unsigned)lo, (unsigned)hi);
}
__device__ inline void from_fp8x8(const uint2 &w, float (&f)[8]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)(i ? w.y : w.x), false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)(i ? w.y : w.x), true);
        f[4 * i] = a[0]; f[4 * i + 1] = a[1]; f[4 * i + 2] = b[0]; f[4 * i + 3] = b[1];
    }
}

// x combined over the lanes of an aligned group of N, in all of them: lane swaps on the vector ALU, no LDS traffic.  Every
// step joins two halves whose members already agree, so the mirrored patterns of the DPP rows serve as well as exact swaps.
template <int CTRL> __device__ inline float dpp(float x) {
    return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, false));
}
template <int N, typename F> __device__ inline float lanes_join(float x, F f) {
    if constexpr (N >= 2) x = f(x, dpp<0xB1>(x));   // lane ^ 1
    if constexpr (N >= 4) x = f(x, dpp<0x4E>(x));   // lane ^ 2
    if constexpr (N >= 8) x = f(x, dpp<0x141>(x));  // mirror in 8
    if constexpr (N >= 16) x = f(x, dpp<0x140>(x)); // mirror in 16
    if constexpr (N >= 32) {
        const unsigned u = __float_as_uint(x);
        const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    }
    if constexpr (N >= 64) {
        const unsigned u = __float_as_uint(x);
        const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        x = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    }
    return x;
}
template <int N> __device__ inline float lanes_sum(float x) { return lanes_join<N>(x, [](float a, float b) { return a + b; }); }
template <int N> __device__ inline float lanes_max(float x) { return lanes_join<N>(x, [](float a, float b) { return fmaxf(a, b); }); }

// The sequence that packed row t lies in: the number of n in [0, N) with cu[n + 1] <= t, by 64-way probes of the whole wave (t
// is the wave's).  Returns N for a row in front of the first sequence or past the last one; always in [0, N], whatever the array holds.
__device__ inline int seq_of_row(const int32_t *cu, int N, int t) {
    const int lane = threadIdx.x & 63, first = N > 0 ? cu[0] : 0; // (fetched beside the first probes)
    int lo = 0, hi = N; // the answer lies in [lo, hi]
    while (lo < hi) {
        const int step = (hi - lo + 63) >> 6, at = lo + lane * step; // probe lane asks whether the answer is over `at`
        const bool over = at < hi && cu[at + 1] <= t;
        const int c = __builtin_popcountll(__ballot(over));
        if (c == 0) break;
        lo = min(hi, lo + (c - 1) * step + 1);
        if (c < 64) hi = min(hi, lo - 1 + step);
    }
    return __builtin_amdgcn_readfirstlane(t < first ? N : lo);
}

} // namespace dn
