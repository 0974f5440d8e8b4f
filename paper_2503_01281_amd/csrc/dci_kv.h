// What the attention kernels and the key/value cache's kernels share: chunks of 16 columns of a row, in any of the types a row may have.
#ifndef DCI_KV_H_
#define DCI_KV_H_

#include "dci_internal.h"

namespace dci {

constexpr int kE4M3 = 3;  // rows of the cache, beside DCI_F32 / DCI_BF16 / DCI_F16
constexpr int kChunk = 16;  // columns to a lane: 16 bytes of a cached row

inline int log2_up(int64_t x) {
  int l = 0;
  while (((int64_t)1 << l) < x) ++l;
  return l;
}
inline int kv_width(int head_dim) { return (head_dim + kChunk - 1) / kChunk * kChunk; }
constexpr int type_bytes(int type) { return type == kE4M3 ? 1 : type == DCI_F32 ? 4 : 2; }
inline bool known_type(int32_t type) { return type == DCI_F32 || type == DCI_BF16 || type == DCI_F16; }
inline bool aligned_rows(const void* base, int type) { return reinterpret_cast<uintptr_t>(base) % (unsigned)type_bytes(type) == 0; }

// The current device is the context's while this lives, whatever it was before.
struct OnDevice {
  int before = -1;
  hipError_t err;
  explicit OnDevice(int device) {
    int now = -1;
    err = hipGetDevice(&now);
    if (err == hipSuccess && now != device) {
      err = hipSetDevice(device);
      if (err == hipSuccess) before = now;
    }
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

int32_t check_kv_cache(dci_ctx* ctx, const dci_kv_cache* cache);

// Sixteen bytes anywhere: the loads and stores of rows need no alignment beyond their type's.
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef unsigned u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef unsigned u32_any __attribute__((aligned(1)));
__device__ __forceinline__ uint4 load_16(const char* p) {
  const u32x4_any v = *reinterpret_cast<const u32x4_any*>(p);
  return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void store_16(char* p, uint4 v) {
  const u32x4_any u = {v.x, v.y, v.z, v.w};
  *reinterpret_cast<u32x4_any*>(p) = u;
}
// Past the caches
__device__ __forceinline__ void store_16_past(char* p, uint4 v) {
  const u32x4_any u = {v.x, v.y, v.z, v.w};
  __builtin_nontemporal_store(u, reinterpret_cast<u32x4_any*>(p));
}

// COLS columns of a row as they lie in memory.
template <int TYPE, int COLS = kChunk>
struct Chunk {
  static constexpr int kWords = type_bytes(TYPE) * COLS / 16;  // of 16 bytes
  uint4 w[kWords];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < kWords; ++j) w[j] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int j = 0; j < kWords; ++j) w[j] = load_16(p + 16 * j);
  }
  // The first `cols` (1 .. COLS) of them from p, the others 0; wide: by 16 bytes (cols are a multiple of them), else number by number.
  __device__ __forceinline__ void load(const char* p, int cols, bool wide) {
    if (TYPE == kE4M3) {
      w[0] = *reinterpret_cast<const uint4*>(p);
    } else if (wide) {
#pragma unroll
      for (int j = 0; j < kWords; ++j)
        w[j] = j * (16 / type_bytes(TYPE)) < cols ? load_16(p + 16 * j) : make_uint4(0, 0, 0, 0);
    } else {
      unsigned u[kWords * 4];
#pragma unroll
      for (int j = 0; j < kWords * 4; ++j) u[j] = 0;
#pragma unroll
      for (int j = 0; j < COLS; ++j) {
        if (j < cols) {
          if (TYPE == DCI_F32) u[j] = reinterpret_cast<const unsigned*>(p)[j];
          else u[j / 2] |= (unsigned)reinterpret_cast<const unsigned short*>(p)[j] << (16 * (j & 1));
        }
      }
#pragma unroll
      for (int j = 0; j < kWords; ++j) w[j] = make_uint4(u[4 * j], u[4 * j + 1], u[4 * j + 2], u[4 * j + 3]);
    }
  }
  __device__ __forceinline__ unsigned word(int j) const {
    const uint4& x = w[j / 4];
    return j % 4 == 0 ? x.x : j % 4 == 1 ? x.y : j % 4 == 2 ? x.z : x.w;
  }
  // Numbers 2 j and 2 j + 1
  __device__ __forceinline__ void pair(int j, float& a, float& b) const {
    if (TYPE == DCI_F32) {
      a = __uint_as_float(word(2 * j));
      b = __uint_as_float(word(2 * j + 1));
    } else if (TYPE == DCI_BF16) {
      a = __uint_as_float(word(j) << 16);
      b = __uint_as_float(word(j) & 0xFFFF0000u);
    } else if (TYPE == DCI_F16) {
      typedef _Float16 half2 __attribute__((ext_vector_type(2)));
      const half2 h = __builtin_bit_cast(half2, word(j));
      a = (float)h.x;
      b = (float)h.y;
    } else {
      typedef float f2 __attribute__((ext_vector_type(2)));
      const f2 f = (j & 1) ? __builtin_amdgcn_cvt_pk_f32_fp8((int)word(j / 2), true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)word(j / 2), false);
      a = f.x;
      b = f.y;
    }
  }
};

// x[j] = x[j + by], 0 beyond the end (by < 16)
template <int N>
__device__ __forceinline__ void shift_down(float (&x)[N], int by) {
#pragma unroll
  for (int step = 8; step; step >>= 1) {
    const bool go = by & step;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float far = j + step < N ? x[j + step < N ? j + step : j] : 0.f;
      x[j] = go ? far : x[j];
    }
  }
}

// 16 columns from p as numbers
template <int TYPE, int COLS>
__device__ __forceinline__ void read_chunk_as(const char* p, int cols, bool wide, float (&x)[COLS]) {
  Chunk<TYPE, COLS> c;
  c.load(p, cols, wide);
#pragma unroll
  for (int j = 0; j < COLS / 2; ++j) c.pair(j, x[2 * j], x[2 * j + 1]);
}
// Whatever their type
template <int COLS>
__device__ __forceinline__ void read_chunk(int type, const char* p, int cols, bool wide, float (&x)[COLS]) {
  if (type == DCI_F32) read_chunk_as<DCI_F32>(p, cols, wide, x);
  else if (type == DCI_BF16) read_chunk_as<DCI_BF16>(p, cols, wide, x);
  else read_chunk_as<DCI_F16>(p, cols, wide, x);
}

template <int TYPE>
__device__ __forceinline__ unsigned two(float a, float b) {  // both rounded to nearest even
  if (TYPE == DCI_BF16) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 f = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(f, b2));
  }
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  const h2 h = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(unsigned, h);
}
template <int TYPE, int COLS>
__device__ __forceinline__ void write_chunk_as(char* p, int cols, bool wide, const float (&x)[COLS]) {
  constexpr int kPer = 16 / type_bytes(TYPE);
  unsigned u[COLS * type_bytes(TYPE) / 4];
#pragma unroll
  for (int j = 0; j < COLS; ++j) {
    if (TYPE == DCI_F32) u[j] = __float_as_uint(x[j]);
    else if (j % 2 == 0) u[j / 2] = two<TYPE>(x[j], x[j + 1]);
  }
  if (wide) {
#pragma unroll
    for (int j = 0; j < COLS / kPer; ++j)
      if (j * kPer < cols) store_16(p + 16 * j, make_uint4(u[4 * j], u[4 * j + 1], u[4 * j + 2], u[4 * j + 3]));
  } else {
#pragma unroll
    for (int j = 0; j < COLS; ++j) {
      if (j < cols) {
        if (TYPE == DCI_F32) reinterpret_cast<unsigned*>(p)[j] = u[j];
        else reinterpret_cast<unsigned short*>(p)[j] = (unsigned short)(u[j / 2] >> (16 * (j & 1)));
      }
    }
  }
}
template <int COLS>
__device__ __forceinline__ void write_chunk(int type, char* p, int cols, bool wide, const float (&x)[COLS]) {
  if (type == DCI_F32) write_chunk_as<DCI_F32>(p, cols, wide, x);
  else if (type == DCI_BF16) write_chunk_as<DCI_BF16>(p, cols, wide, x);
  else write_chunk_as<DCI_F16>(p, cols, wide, x);
}

// What a lane gets of its neighbours: the lane 1, 2 away, and (where the quads, the eights agree within themselves) 4, 8 away
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true));
}
// Sums of N numbers each over groups of 1 << log2 lanes (log2 <= 5), in all of the lanes
template <int N>
__device__ __forceinline__ void sum_lanes(float* x, int log2) {
#define DCI_STEP(STEP_, CTRL_)                              \
  if (log2 > STEP_) {                                       \
    _Pragma("unroll") for (int i = 0; i < N; ++i) x[i] += dpp<CTRL_>(x[i]); \
  }
  DCI_STEP(0, 0xB1)   // quad_perm 1 0 3 2
  DCI_STEP(1, 0x4E)   // quad_perm 2 3 0 1
  DCI_STEP(2, 0x141)  // the other half of eight, mirrored
  DCI_STEP(3, 0x140)  // the other half of sixteen, mirrored
#undef DCI_STEP
  if (log2 > 4) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += __shfl_xor(x[i], 16, kWave);
  }
}
// The maximum likewise
__device__ __forceinline__ float max_lanes(float x, int log2) {
  if (log2 > 0) x = fmaxf(x, dpp<0xB1>(x));
  if (log2 > 1) x = fmaxf(x, dpp<0x4E>(x));
  if (log2 > 2) x = fmaxf(x, dpp<0x141>(x));
  if (log2 > 3) x = fmaxf(x, dpp<0x140>(x));
  return x;
}

}  // namespace dci

#endif  // DCI_KV_H_
