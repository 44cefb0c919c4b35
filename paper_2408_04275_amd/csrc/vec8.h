// Eight elements at a time: 16 bytes of bf16, 32 of fp32, widened to fp32.
#pragma once
#include "common.h"

namespace mmt {

__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16_t *p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&v)[8]) {
    uint4 a;
    a.x = pack_bf16x2(v[0], v[1]); a.y = pack_bf16x2(v[2], v[3]);
    a.z = pack_bf16x2(v[4], v[5]); a.w = pack_bf16x2(v[6], v[7]);
    *reinterpret_cast<uint4 *>(p) = a;
}

// Streaming forms for tensors that a kernel passes over once and that are far larger than the caches.
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
__device__ __forceinline__ void load8_stream(const bf16_t *p, float (&v)[8]) {
    const u32x4_t a = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8_stream(const float *p, float (&v)[8]) { load8(p, v); }
__device__ __forceinline__ void store8_stream(bf16_t *p, const float (&v)[8]) {
    u32x4_t a;
    a[0] = pack_bf16x2(v[0], v[1]); a[1] = pack_bf16x2(v[2], v[3]);
    a[2] = pack_bf16x2(v[4], v[5]); a[3] = pack_bf16x2(v[6], v[7]);
    __builtin_nontemporal_store(a, reinterpret_cast<u32x4_t *>(p));
}
__device__ __forceinline__ void store8_stream(float *p, const float (&v)[8]) { store8(p, v); }

// Eight elements as loaded, not yet widened to fp32: what a kernel holds for a row it has requested ahead of time
// (four registers per chunk in bf16 instead of eight).
template <typename T> struct Raw8;
template <> struct Raw8<bf16_t> { uint4 a; };
template <> struct Raw8<float> { float4 a, b; };
__device__ __forceinline__ void load_raw8(const bf16_t *p, Raw8<bf16_t> &r) {
    // streaming form: each of these tensors is passed over once (norm backward at the 7B shape: 49.8 -> 46.4 us)
    const u32x4_t a = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p));
    r.a = make_uint4(a[0], a[1], a[2], a[3]);
}
__device__ __forceinline__ void load_raw8(const float *p, Raw8<float> &r) {
    r.a = *reinterpret_cast<const float4 *>(p); r.b = *reinterpret_cast<const float4 *>(p + 4);
}
__device__ __forceinline__ Raw8<bf16_t> load_plain8(const bf16_t *p) { return {*reinterpret_cast<const uint4 *>(p)}; }
__device__ __forceinline__ Raw8<float> load_plain8(const float *p) { return {*reinterpret_cast<const float4 *>(p), *reinterpret_cast<const float4 *>(p + 4)}; }
__device__ __forceinline__ void unpack8(const Raw8<bf16_t> &r, float (&v)[8]) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack8(const Raw8<float> &r, float (&v)[8]) {
    v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w; v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}

}  // namespace mmt
