// A few neighbouring elements in one access of up to 16 bytes.
#pragma once
#include "common.h"

namespace mmt {

// V neighbouring elements as loaded
template <int BYTES> struct Bytes;
template <> struct Bytes<16> { typedef u32x4 type; };
template <> struct Bytes<8> { typedef u32x2 type; };
template <> struct Bytes<4> { typedef uint32_t type; };
template <> struct Bytes<2> { typedef uint16_t type; };

template <typename T, int V> struct Chunk {
    typedef typename Bytes<V * sizeof(T)>::type raw;
    union { raw r; T e[V]; };
    __device__ __forceinline__ void load(const T *p) { r = *reinterpret_cast<const raw *>(p); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<raw *>(p) = r; }
    __device__ __forceinline__ float get(int i) const { return Elem<T>::load(&e[i]); }
    __device__ __forceinline__ void set(const float (&v)[V]) {
        if constexpr (sizeof(T) == 4 || V == 1) {
#pragma unroll
            for (int i = 0; i < V; ++i) Elem<T>::store(&e[i], v[i]);
        } else {
            uint32_t w[V / 2];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
            __builtin_memcpy(&r, w, sizeof(r));
        }
    }
};

}  // namespace mmt
