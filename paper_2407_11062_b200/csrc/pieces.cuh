// 8 or 16 neighbouring bf16 numbers, moved at once: 16 bytes, or 32 where everything is aligned to them.  (Or 1, 2, 4.)
//
// With 32 bytes a warp's load is whole 1 KB runs and a thread needs half as many of them; with them goes a block for every
// piece, not blocks that stay.  gated.cu, norm.cu and rotary.cu have what it brought.
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace eqat {

template <int N>
struct Piece {
  uint32_t w[N / 2];
};
template <>
struct Piece<1> {
  eqat_bf16 w;
};

// Read once: no line of the SM's cache is taken.
template <int N>
__device__ __forceinline__ Piece<N> load_piece(const eqat_bf16* p) {
  Piece<N> v;
  if constexpr (N == 16) {
    ptx::ld_global_once_256(p, v.w);
  } else if constexpr (N == 1) {
    v.w = ptx::ld_global(p);
  } else if constexpr (N == 2) {
    v.w[0] = ptx::ld_global(reinterpret_cast<const uint32_t*>(p));
  } else if constexpr (N == 4) {
    const uint2 u = ptx::ld_global(reinterpret_cast<const uint2*>(p));
    v.w[0] = u.x, v.w[1] = u.y;
  } else {
    const uint4 u = ptx::ld_global_once(reinterpret_cast<const uint4*>(p));
    v.w[0] = u.x, v.w[1] = u.y, v.w[2] = u.z, v.w[3] = u.w;
  }
  return v;
}
template <int N>
__device__ __forceinline__ void store_piece(eqat_bf16* p, const Piece<N>& v) {
  if constexpr (N == 16) ptx::st_global_256(p, v.w);
  else if constexpr (N == 1) *p = v.w;
  else if constexpr (N == 2) *reinterpret_cast<uint32_t*>(p) = v.w[0];
  else if constexpr (N == 4) *reinterpret_cast<uint2*>(p) = make_uint2(v.w[0], v.w[1]);
  else *reinterpret_cast<uint4*>(p) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
}

template <int N>
__device__ __forceinline__ void unpack(const Piece<N>& v, float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    f[2 * i] = __uint_as_float(v.w[i] << 16);
    f[2 * i + 1] = __uint_as_float(v.w[i] & 0xFFFF0000u);
  }
}
template <int N>
__device__ __forceinline__ Piece<N> pack(const float (&f)[N]) {
  Piece<N> v;
#pragma unroll
  for (int i = 0; i < N / 2; ++i) v.w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
  return v;
}

// Whether all of these (null ones do not count) start on 32 bytes.
template <typename... P>
inline bool aligned32(P... p) {
  return ((reinterpret_cast<uintptr_t>(p) | ...) & 31u) == 0;
}

}  // namespace eqat
