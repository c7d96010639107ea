// Device-side pieces of the operators around a layer's mixer.
#pragma once
#include "dn_attn_device.hpp"
#include "dn_layer_host.hpp"

namespace dn {

// V elements of type T as they are loaded and stored: V sizeof(T) is 4, 8 or a multiple of 16 bytes.
template <typename T, int V> struct Word {
    static constexpr int N = V * (int)sizeof(T) / 4;
    unsigned w[N];
    __device__ inline void zero() {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = 0;
    }
    __device__ inline void load(const T *p) {
        if constexpr (N == 1) w[0] = *reinterpret_cast<const unsigned *>(p);
        else if constexpr (N == 2) { const uint2 x = *reinterpret_cast<const uint2 *>(p); w[0] = x.x; w[1] = x.y; }
        else {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) { const uint4 x = reinterpret_cast<const uint4 *>(p)[i]; w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w; }
        }
    }
    __device__ inline void store(T *p) const {
        if constexpr (N == 1) *reinterpret_cast<unsigned *>(p) = w[0];
        else if constexpr (N == 2) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        else {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) reinterpret_cast<uint4 *>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
    }
    // past the caches
    __device__ inline void store_once(T *p) const {
        typedef unsigned raw __attribute__((ext_vector_type(N < 4 ? N : 4)));
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            raw r;
#pragma unroll
            for (int j = 0; j < (N < 4 ? N : 4); ++j) r[j] = w[i + j];
            __builtin_nontemporal_store(r, reinterpret_cast<raw *>(p) + i / 4);
        }
    }
    __device__ inline void store(T *p, bool once) const {
        if (once) store_once(p);
        else store(p);
    }
    __device__ inline float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    }
    __device__ inline void unpack(float (&f)[V]) const {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = get(i);
    }
    __device__ inline void pack(const float (&f)[V]) {
        if constexpr (V == 1) {
            w[0] = __float_as_uint(f[0]);
            return;
        }
        typedef T vec __attribute__((ext_vector_type(V)));
        typedef unsigned raw __attribute__((ext_vector_type(N)));
        vec v;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (T)f[i];
        const raw r = __builtin_bit_cast(raw, v);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = r[i];
    }
};

} // namespace dn
