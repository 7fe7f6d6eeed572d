// Vectors of VEC elements (a whole 128-bit access of the type, or a single element where rows are shorter than one) at any
// element of a tensor: rows of any length start anywhere, and the memory pipeline takes such accesses as they are.  Loads hand
// out raw bits, so that many can be under way before the first is widened.
#pragma once
#include "e4m3.hpp"

namespace fsk {

// STREAM: with the streaming hint; without it where neighbouring workgroups write the rest of a line (the cache then puts it
// together, with the hint every piece goes to memory by itself).
// ALIGN: the bytes that p's address is a multiple of (an alignment in the type of a deduced pointer would be lost).
template <bool STREAM, int ALIGN, typename V> __device__ __forceinline__ void put(V v, void* p) {
  typename AtAlignment<V, ALIGN>::type* const q = reinterpret_cast<typename AtAlignment<V, ALIGN>::type*>(p);
  if constexpr (STREAM) __builtin_nontemporal_store(v, q);
  else *q = v;
}

template <typename IO, typename T, int VEC> __device__ __forceinline__ void store_as(bool stream, T* p, const float (&v)[VEC]) {
  if (stream) IO::template store<true>(p, v);
  else IO::template store<false>(p, v);
}

template <typename T, int VEC> struct VecIo {
  static_assert(VEC == Elem<T>::VEC, "a whole vector, or one element");
  typedef u32x4 Raw;
  typedef typename AtAlignment<u32x4, sizeof(T)>::type Place;
  template <bool STREAM> __device__ __forceinline__ static Raw load(const T* p) {
    const Place* q = reinterpret_cast<const Place*>(p);
    return STREAM ? __builtin_nontemporal_load(q) : *q;
  }
  __device__ __forceinline__ static void widen(Raw r, float (&v)[VEC]) { unpack(r, v, (const T*)nullptr); }
  template <bool STREAM = true> __device__ __forceinline__ static void store(T* p, const float (&v)[VEC]) {
    u32x4 w;
    if constexpr (sizeof(T) == 4) w = __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
    else w = u32x4{pack2(v[0], v[1], (const T*)nullptr), pack2(v[2], v[3], (const T*)nullptr), pack2(v[4], v[5], (const T*)nullptr),
                   pack2(v[6], v[7], (const T*)nullptr)};
    put<STREAM, sizeof(T)>(w, p);
  }
};
template <typename T> struct VecIo<T, 1> {
  typedef float Raw;
  template <bool STREAM> __device__ __forceinline__ static Raw load(const T* p) { return load1(p); }
  __device__ __forceinline__ static void widen(Raw r, float (&v)[1]) { v[0] = r; }
  template <bool STREAM = true> __device__ __forceinline__ static void store(T* p, const float (&v)[1]) { put1(p, v[0]); }
  template <typename U> __device__ __forceinline__ static void put1(U* p, float v) { store1(p, v); }
  __device__ __forceinline__ static void put1(e4m3_t* p, float v) { store1_in_range(p, v); }
};
// half a vector of a 16-bit type
template <typename T> struct HalfVecIo {
  typedef u32x2 Raw;
  typedef typename AtAlignment<u32x2, 2>::type Place;
  template <bool STREAM> __device__ __forceinline__ static Raw load(const T* p) {
    const Place* q = reinterpret_cast<const Place*>(p);
    return STREAM ? __builtin_nontemporal_load(q) : *q;
  }
  __device__ __forceinline__ static void widen(Raw r, float (&v)[4]) {
    float w[8];
    unpack(u32x4{r.x, r.y, 0u, 0u}, w, (const T*)nullptr);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = w[e];
  }
  template <bool STREAM = true> __device__ __forceinline__ static void store(T* p, const float (&v)[4]) {
    put<STREAM, 2>(u32x2{pack2(v[0], v[1], (const T*)nullptr), pack2(v[2], v[3], (const T*)nullptr)}, p);
  }
};
template <> struct VecIo<f16_t, 4> : HalfVecIo<f16_t> {};
template <> struct VecIo<bf16_t, 4> : HalfVecIo<bf16_t> {};
template <> struct VecIo<e4m3_t, 8> {
  typedef u32x2 Raw;
  typedef AtAlignment<u32x2, 1>::type Place;
  template <bool STREAM> __device__ __forceinline__ static Raw load(const e4m3_t* p) {
    const Place* q = reinterpret_cast<const Place*>(p);
    return STREAM ? __builtin_nontemporal_load(q) : *q;
  }
  __device__ __forceinline__ static void widen(Raw r, float (&v)[8]) {
    unpack_e4m3(r.x, v[0], v[1], v[2], v[3]);
    unpack_e4m3(r.y, v[4], v[5], v[6], v[7]);
  }
  template <bool STREAM = true> __device__ __forceinline__ static void store(e4m3_t* p, const float (&v)[8]) {
    const u32x2 w = {pack_e4m3_in_range(v[0], v[1], v[2], v[3]), pack_e4m3_in_range(v[4], v[5], v[6], v[7])};
    put<STREAM, 1>(w, p);
  }
};
template <> struct VecIo<e4m3_t, 4> {
  typedef uint32_t Raw;
  typedef AtAlignment<uint32_t, 1>::type Place;
  template <bool STREAM> __device__ __forceinline__ static Raw load(const e4m3_t* p) {
    const Place* q = reinterpret_cast<const Place*>(p);
    return STREAM ? __builtin_nontemporal_load(q) : *q;
  }
  __device__ __forceinline__ static void widen(Raw r, float (&v)[4]) { unpack_e4m3(r, v[0], v[1], v[2], v[3]); }
  template <bool STREAM = true> __device__ __forceinline__ static void store(e4m3_t* p, const float (&v)[4]) {
    put<STREAM, 1>(pack_e4m3_in_range(v[0], v[1], v[2], v[3]), p);
  }
};

// Element `i` behind a pointer that the whole workgroup shares, at a distance of less than 2^32 bytes: a scalar base and one
// vector register instead of a 64-bit address per access.
template <typename T> __device__ __forceinline__ const T* near_element(const T* base, uint32_t i) {
  return reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + (uint32_t)(i * (uint32_t)sizeof(T)));
}
template <typename T> __device__ __forceinline__ T* near_element(T* base, uint32_t i) {
  return reinterpret_cast<T*>(reinterpret_cast<char*>(base) + (uint32_t)(i * (uint32_t)sizeof(T)));
}

// Passes over values that a thread keeps as raw bits (a workgroup's registers hold them all).  Left alone, the compiler keeps the
// widened values of one pass for the next, and works on all steps of a pass at once: several times the registers.
// again(): the bits may have changed, what was made of them is made anew.  done(): the step's results are wanted here.
template <typename R> __device__ __forceinline__ void again(R& raw) { asm volatile("" : "+v"(raw)); }
template <int N> __device__ __forceinline__ void done(float (&v)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) asm volatile("" : "+v"(v[e]));
}

}  // namespace fsk
