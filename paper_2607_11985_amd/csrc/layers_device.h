// layers_device.h -- device helpers of the layers' kernels: packs of 16 bytes,
// sums over lanes and workgroups.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace vqc {

using f16 = _Float16;
using bf16 = __bf16;

template <typename T>
constexpr int kPack = 16 / (int)sizeof(T);

// 16 bytes of a row, at any alignment of its elements: global memory takes 16-byte
// accesses at element alignment, so an odd row stride needs no path of its own.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
  T v[kPack<T>];
};

// The pack of columns [c, c + kPack) of a row of `cols`; `fill` beyond the end.
template <typename T>
__device__ __forceinline__ Pack<T> load_pack(const T* row, int64_t c, int64_t cols, T fill) {
  Pack<T> p;
  if (c + kPack<T> <= cols) {
    p = *reinterpret_cast<const Pack<T>*>(row + c);
  } else {
#pragma unroll
    for (int i = 0; i < kPack<T>; ++i) {
      p.v[i] = fill;
      if (c + i < cols) p.v[i] = row[c + i];
    }
  }
  return p;
}

// The same in two steps, for loads that are to be in flight together: load_raw has no branch
// and takes no element out (either makes the compiler wait for each load by itself: 16-bit
// scores of 4096 x 32768 took 90 us that way and take 75), taken makes the pack of it where it
// is used.  Near the end of a row the 16 bytes before it are read and then shifted.
// SHORT: rows of fewer than kPack columns, read by elements; otherwise cols >= kPack.
typedef uint32_t Raw __attribute__((ext_vector_type(4)));
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)), may_alias)) RawAt {
  Raw r;
};

// The same value, of which the compiler does not know that: it keeps nothing derived from it in
// registers beyond its use.
__device__ __forceinline__ Raw opaque(Raw r) {
  asm("" : "+v"(r));
  return r;
}

template <typename T, bool SHORT = false, typename I>
__device__ __forceinline__ Raw load_raw(const T* row, I c, I cols) {
  if constexpr (SHORT) return __builtin_bit_cast(Raw, load_pack<T>(row, c, cols, (T)0.f));
  const I last = cols - kPack<T>;
  return reinterpret_cast<const RawAt<T>*>(row + (c < last ? c : last))->r;
}

template <typename T, bool SHORT = false, typename I>
__device__ __forceinline__ Pack<T> taken(Raw r, I c, I cols, T fill) {
  constexpr int V = kPack<T>;
  const I over = c + V - cols;  // elements behind the end
  if (over > 0) {
    Pack<T> f;
#pragma unroll
    for (int i = 0; i < V; ++i) f.v[i] = fill;
    if constexpr (SHORT) {
      const Pack<T> p = __builtin_bit_cast(Pack<T>, r);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c + i < cols) f.v[i] = p.v[i];
      return f;
    }
    const uint32_t filled = __builtin_bit_cast(Raw, f)[0];
    const uint32_t bytes = (uint32_t)(over < V ? over : V) * sizeof(T);
    if (bytes & 16) r = Raw{filled, filled, filled, filled};
    if (bytes & 8) r = Raw{r[2], r[3], filled, filled};
    if (bytes & 4) r = Raw{r[1], r[2], r[3], filled};
    if constexpr (sizeof(T) == 2)
      if (bytes & 2)
        r = Raw{r[0] >> 16 | r[1] << 16, r[1] >> 16 | r[2] << 16, r[2] >> 16 | r[3] << 16,
                r[3] >> 16 | filled << 16};
  }
  return __builtin_bit_cast(Pack<T>, r);
}

template <typename T>
__device__ __forceinline__ void store_pack(T* row, int64_t c, int64_t cols, const Pack<T>& p) {
  if (c + kPack<T> <= cols) {
    *reinterpret_cast<Pack<T>*>(row + c) = p;
  } else {
#pragma unroll
    for (int i = 0; i < kPack<T>; ++i)
      if (c + i < cols) row[c + i] = p.v[i];
  }
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}

// The value of lane ^ N (N a power of two), by VALU moves alone.
template <int N>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
  if constexpr (N == 1) return dpp<0xB1>(x);        // quad_perm [1,0,3,2]
  if constexpr (N == 2) return dpp<0x4E>(x);        // quad_perm [2,3,0,1]
  if constexpr (N == 4) return dpp<0x1B>(dpp<0x141>(x));  // half-row mirror, then quad reversed
  if constexpr (N == 8) return dpp<0x128>(x);       // row rotated by 8
  if constexpr (N == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return (threadIdx.x & 16) ? r[0] : r[1];
  }
  if constexpr (N == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return (threadIdx.x & 32) ? r[0] : r[1];
  }
}

template <int N>
__device__ __forceinline__ float lane_xor(float x) {
  return __builtin_bit_cast(float, lane_xor<N>(__builtin_bit_cast(uint32_t, x)));
}

// Sum over aligned groups of G <= 64 lanes, in every lane.
template <int G>
__device__ __forceinline__ float lanes_sum(float x) {
  if constexpr (G > 1) x += lane_xor<1>(x);
  if constexpr (G > 2) x += lane_xor<2>(x);
  if constexpr (G > 4) x += lane_xor<4>(x);
  if constexpr (G > 8) x += lane_xor<8>(x);
  if constexpr (G > 16) x += lane_xor<16>(x);
  if constexpr (G > 32) x += lane_xor<32>(x);
  return x;
}

// Sums of N values over groups of G threads (16, 64, or a multiple of 64 up to the
// workgroup), in every thread.  `red` holds N floats per wave; the caller
// alternates between two such buffers, so that one barrier per sum is enough.
// Every thread of the workgroup calls it where G > 64.
template <int G, int N>
__device__ __forceinline__ void group_sums(float (&v)[N], float* red) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lanes_sum<(G < 64 ? G : 64)>(v[i]);
  if constexpr (G > 64) {
    const int wave = threadIdx.x >> 6;
    constexpr int W = G / 64;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) red[wave * N + i] = v[i];
    __syncthreads();
    const int first = wave / W * W;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = red[first * N + i];
#pragma unroll
      for (int w = 1; w < W; ++w) s += red[(first + w) * N + i];
      v[i] = s;
    }
  }
}

template <typename F>
int by_dtype(int dtype, F&& f) {
  switch (dtype) {
    case 0: return f(float{});
    case 1: return f(f16{});
    case 2: return f(bf16{});
    default: return (int)hipErrorInvalidValue;
  }
}

}  // namespace vqc
