// One AdamW step over many tensors (blr_adamw_step in blr.h).
//
// Per value, in float32:
//     m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  r = sqrt(v)
//     w = w (1 - lr wd) - m / (r / sqrt(1 - b2^t) + eps) * lr / (1 - b1^t)
// What the moments take is rounded operation by operation (no contraction): an
// 8-bit code must not hang on how the compiler fuses a sum, or two builds would
// drift apart by whole codes. Bound by memory with float32 moments: 28 bytes a
// value with float32 everywhere, 28 with bfloat16 parameters and float32 masters
// (190 M values: 771 us, 6.9 TB/s). With 8-bit moments about 10 bytes a value
// are left and the instructions bound the kernel; the quotient, a thousandth of
// w, is then approximate to two units in the last place.
//
// Layout: the tensors' records travel in the kernel's parameters (nothing is
// copied to the device, nothing is kept between calls), up to kMaxTensors a
// launch. A block takes one chunk of kChunk values of one tensor, found by a
// binary search over the records' first chunks; a warp takes 256 consecutive
// values at a time, 8 a lane, which is also the block that shares a scale of
// the 8-bit moments: its maximum is one warp reduction, in registers.
#include <math.h>

#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "blr_host.h"

namespace {

using blr::fail;

constexpr int kThreads = 256;
constexpr int kGroup = 256;   // values a warp takes at a time, one scale of the 8-bit moments
// Values a block takes. A block first finds its tensor; with 8-bit moments, where that counts, 16384 values
// spread it over eight groups a warp (285 -> 259 us of 95 M values; with float32 moments, which wait for
// memory alone, 771 -> 794). A small model (under 4 M values) keeps its blocks many.
constexpr int kChunk = 4096, kCodesChunk = 16384;
constexpr int64_t kSmallModel = (int64_t)4 << 20;
constexpr int kMaxTensors = 448;
constexpr int kFewTensors = 32;
constexpr float kE4m3Max = 448.0f;
constexpr float kE4m3Tiny = 0.001953125f;  // 2^-9, the smallest positive code

template <int CAP>
struct Table {
  blr_adamw_tensor t[CAP];
  uint32_t first[CAP];  // first chunk of each tensor
  uint32_t wide[(CAP + 31) / 32];  // whether its pointers allow wide accesses
  int count, chunk;
};
static_assert(sizeof(Table<kMaxTensors>) < 32000, "kernel parameters hold 32764 bytes");

struct Hyper {
  float b1, c1, b2, c2;  // beta1, 1 - beta1, beta2, 1 - beta2
  float root_scale;      // 1 / sqrt(1 - beta2^step)
  float eps;
  float keep;            // 1 - lr weight_decay
  float rate;            // lr / (1 - beta1^step)
  const float* grad_scale;
};

// 8 values of a tensor, as floats.
template <typename T> struct Eight;
template <> struct Eight<float> {
  static __device__ __forceinline__ void load(const float* p, float (&x)[8]) {
    asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]),
                   "=f"(x[7])
                 : "l"(p));
  }
  static __device__ __forceinline__ void store(float* p, const float (&x)[8]) {
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(x[0]), "f"(x[1]),
                 "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                 : "memory");
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ void put(float* p, float x) { *p = x; }
};
template <> struct Eight<__nv_bfloat16> {
  static __device__ __forceinline__ void load(const __nv_bfloat16* p, float (&x)[8]) {
    const uint4 r = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
  }
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
};

// e4m3 codes (two at a time) to and from floats, by the conversion instructions.
__device__ __forceinline__ float2 from_e4m3x2(uint16_t c) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c, __NV_E4M3);
  return __half22float2(__half2(h));
}
__device__ __forceinline__ uint16_t to_e4m3x2(float a, float b) {
  return (uint16_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// The codes of a lane's 8 values: 8 bytes, or single bytes of a ragged or unaligned group.
__device__ __forceinline__ uint2 load_codes(const uint8_t* p, int n, bool wide) {
  if (wide) return __ldcs(reinterpret_cast<const uint2*>(p));
  uint32_t w[2] = {0u, 0u};
  for (int i = 0; i < 8; ++i)
    if (i < n) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void decode(uint2 c, float (&x)[8]) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = from_e4m3x2((uint16_t)(w[i >> 1] >> (16 * (i & 1))));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

// Writes the codes and the scale of a warp's group. A NaN stays with its own value; ROOT: values are not
// negative, and a positive one is stored as no less than the smallest code.
template <bool ROOT>
__device__ __forceinline__ void store_codes(uint8_t* p, float* scale, int n, bool wide, const float (&x)[8]) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
  top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));  // magnitudes order as their bits
  const float inverse = top > 0.0f ? fminf(__fmul_rn(__fdiv_rn(1.0f, top), kE4m3Max), 3.402823466e38f) : 0.0f;
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint16_t c[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float y[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        y[j] = __fmul_rn(x[4 * h + 2 * i + j], inverse);
        if (ROOT) y[j] = y[j] > 0.0f ? fmaxf(y[j], kE4m3Tiny) : y[j];
      }
      c[i] = to_e4m3x2(y[0], y[1]);
    }
    w[h] = (uint32_t)c[0] | (uint32_t)c[1] << 16;
  }
  if (wide) {
    __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
  } else {
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
  if ((threadIdx.x & 31) == 0) *scale = __fmul_rn(top, 1.0f / kE4m3Max);
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, bool wide, float (&x)[8]) {
  if (wide) {
    Eight<T>::load(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? Eight<T>::one(p + i) : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, bool wide, const float (&x)[8]) {
  if (wide) {
    Eight<T>::store(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) Eight<T>::put(p + i, x[i]);
  }
}

template <typename T, int BITS, bool MASTER, int CAP>
__global__ void __launch_bounds__(kThreads, BITS == 8 ? 5 : 1)
adamw_kernel(const __grid_constant__ Table<CAP> table, const __grid_constant__ Hyper h) {
  // the last tensor whose first chunk is not after this block
  int lo = 0, hi = table.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (table.first[mid] <= blockIdx.x) lo = mid; else hi = mid - 1;
  }
  const blr_adamw_tensor& t = table.t[lo];
  const int64_t n = t.n, begin = (int64_t)(blockIdx.x - table.first[lo]) * table.chunk;
  const bool aligned = (table.wide[lo >> 5] >> (lo & 31)) & 1u;
  const float gs = h.grad_scale == nullptr ? 1.0f : __ldg(h.grad_scale);
  const bool scaled = h.grad_scale != nullptr;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kStride = (kThreads / 32) * kGroup;
  for (int64_t at = begin + warp * kGroup; at < min(n, begin + table.chunk); at += kStride) {  // by whole warps
    float w[8], g[8], m[8], v[8];
    const bool wide = aligned && at + kGroup <= n;
    const int64_t i0 = at + lane * 8, block = at / kGroup;
    const int left = wide ? 8 : (int)max((int64_t)0, min((int64_t)8, n - i0));
    if constexpr (MASTER) {
      load8<float>(t.w + i0, left, wide, w);
    } else {
      load8<T>(static_cast<const T*>(t.p) + i0, left, wide, w);
    }
    load8<T>(static_cast<const T*>(t.g) + i0, left, wide, g);
    if constexpr (BITS == 32) {
      load8<float>(static_cast<const float*>(t.m) + i0, left, wide, m);
      load8<float>(static_cast<const float*>(t.v) + i0, left, wide, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float gi = __fmul_rn(g[i], gs);
        m[i] = __fadd_rn(__fmul_rn(m[i], h.b1), __fmul_rn(gi, h.c1));
        v[i] = __fadd_rn(__fmul_rn(v[i], h.b2), __fmul_rn(__fmul_rn(gi, gi), h.c2));
        const float d = __fadd_rn(__fmul_rn(__fsqrt_rn(v[i]), h.root_scale), h.eps);
        w[i] = __fsub_rn(__fmul_rn(w[i], h.keep), __fmul_rn(__fdiv_rn(m[i], d), h.rate));
      }
      store8<float>(static_cast<float*>(t.m) + i0, left, wide, m);
      store8<float>(static_cast<float*>(t.v) + i0, left, wide, v);
    } else {
      const uint2 mc = load_codes(static_cast<const uint8_t*>(t.m) + i0, left, wide);
      const uint2 vc = load_codes(static_cast<const uint8_t*>(t.v) + i0, left, wide);
      const float ms = t.m_scale[block], vs = t.v_scale[block];
      decode(mc, m);
      decode(vc, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float gi = scaled ? __fmul_rn(g[i], gs) : g[i], r0 = __fmul_rn(v[i], vs);
        m[i] = __fadd_rn(__fmul_rn(__fmul_rn(m[i], ms), h.b1), __fmul_rn(gi, h.c1));
        v[i] = __fsqrt_rn(__fadd_rn(__fmul_rn(__fmul_rn(r0, r0), h.b2), __fmul_rn(__fmul_rn(gi, gi), h.c2)));
        w[i] = w[i] * h.keep - __fdividef(m[i], v[i] * h.root_scale + h.eps) * h.rate;
        if (!wide && i >= left) m[i] = v[i] = 0.0f;  // values past the end have no part in the scale
      }
      store_codes<false>(static_cast<uint8_t*>(t.m) + i0, t.m_scale + block, left, wide, m);
      store_codes<true>(static_cast<uint8_t*>(t.v) + i0, t.v_scale + block, left, wide, v);
    }
    if constexpr (MASTER) store8<float>(t.w + i0, left, wide, w);
    store8<T>(static_cast<T*>(t.p) + i0, left, wide, w);
  }
}

template <typename T, int BITS, bool MASTER, int CAP>
blr_status launch(const blr_adamw_tensor* tensors, int64_t& at, int64_t count, int chunk, const Hyper& h,
                  cudaStream_t stream) {
  Table<CAP> table;
  table.count = 0;
  table.chunk = chunk;
  for (uint32_t& w : table.wide) w = 0;
  int64_t chunks = 0;
  for (; at < count && table.count < CAP; ++at) {
    const blr_adamw_tensor& t = tensors[at];
    if (t.n == 0) continue;
    const int64_t more = (t.n + chunk - 1) / chunk;
    if (chunks + more > 0x7fffffff) {
      if (table.count == 0) return fail(BLR_ERR_UNSUPPORTED, "tensor %lld is too large", (long long)at);
      break;
    }
    const size_t a = sizeof(T) == 4 ? 32 : 16, am = BITS == 32 ? 32 : 8;
    if (blr::aligned(t.p, a) && blr::aligned(t.g, a) && blr::aligned(t.m, am) && blr::aligned(t.v, am) &&
        (!MASTER || blr::aligned(t.w, 32)))
      table.wide[table.count >> 5] |= 1u << (table.count & 31);
    table.t[table.count] = t;
    table.first[table.count++] = (uint32_t)chunks;
    chunks += more;
  }
  if (table.count == 0) return BLR_OK;
  adamw_kernel<T, BITS, MASTER, CAP><<<(unsigned)chunks, kThreads, 0, stream>>>(table, h);
  return blr::cuda_check(cudaGetLastError(), "blr_adamw_step");
}

template <typename T, int BITS, bool MASTER>
blr_status step_all(const blr_adamw_tensor* tensors, int64_t count, const Hyper& h, cudaStream_t stream) {
  int64_t at = 0, values = 0;
  for (int64_t i = 0; i < count; ++i) values += tensors[i].n;
  const int chunk = BITS == 8 && values >= kSmallModel ? kCodesChunk : kChunk;
  while (at < count) {
    // a small table keeps the launch of a small model short
    if (count - at <= kFewTensors)
      BLR_TRY((launch<T, BITS, MASTER, kFewTensors>(tensors, at, count, chunk, h, stream)));
    else
      BLR_TRY((launch<T, BITS, MASTER, kMaxTensors>(tensors, at, count, chunk, h, stream)));
  }
  return BLR_OK;
}

}  // namespace

blr_status blr_adamw_step(int64_t count, const blr_adamw_tensor* tensors, blr_dtype io, int bits,
                          double lr, double beta1, double beta2, double eps, double weight_decay,
                          int64_t step, const float* grad_scale, blr_stream_t stream) {
  if (count < 0) return fail(BLR_ERR_INVALID_ARG, "negative count");
  if (io != BLR_F32 && io != BLR_BF16) return fail(BLR_ERR_INVALID_ARG, "unknown io dtype %d", (int)io);
  if (bits != 32 && bits != 8) return fail(BLR_ERR_INVALID_ARG, "bits=%d is neither 32 nor 8", bits);
  if (!isfinite(lr) || !isfinite(weight_decay))
    return fail(BLR_ERR_INVALID_ARG, "lr and weight_decay must be finite");
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
    return fail(BLR_ERR_INVALID_ARG, "beta1 and beta2 must lie in [0, 1)");
  if (!(eps > 0.0) || !isfinite(eps)) return fail(BLR_ERR_INVALID_ARG, "eps must be finite and > 0");
  if (step < 1) return fail(BLR_ERR_INVALID_ARG, "step must be at least 1");
  BLR_TRY(blr::optional(grad_scale, "grad_scale", 4));
  if (count == 0) return BLR_OK;
  if (tensors == nullptr) return fail(BLR_ERR_INVALID_ARG, "tensors is NULL");
  const size_t e = io == BLR_F32 ? 4 : 2;
  bool master = false, first = true;
  for (int64_t i = 0; i < count; ++i) {
    const blr_adamw_tensor& t = tensors[i];
    if (t.n < 0) return fail(BLR_ERR_INVALID_ARG, "tensor %lld has a negative size", (long long)i);
    if (t.n == 0) continue;
    BLR_TRY(blr::need(t.p, "p", e));
    BLR_TRY(blr::need(t.g, "g", e));
    BLR_TRY(blr::need(t.m, "m", bits == 32 ? 4 : 1));
    BLR_TRY(blr::need(t.v, "v", bits == 32 ? 4 : 1));
    if (bits == 8) {
      BLR_TRY(blr::need(t.m_scale, "m_scale", 4));
      BLR_TRY(blr::need(t.v_scale, "v_scale", 4));
    }
    if (!first && master != (t.w != nullptr))
      return fail(BLR_ERR_INVALID_ARG, "master weights in some records only");
    master = t.w != nullptr;
    first = false;
    if (master) {
      if (io == BLR_F32) return fail(BLR_ERR_INVALID_ARG, "float32 parameters have no master weights");
      BLR_TRY(blr::need(t.w, "w", 4));
    }
  }
  Hyper h;
  h.b1 = (float)beta1;
  h.c1 = (float)(1.0 - beta1);
  h.b2 = (float)beta2;
  h.c2 = (float)(1.0 - beta2);
  h.root_scale = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
  h.eps = (float)eps;
  h.keep = (float)(1.0 - lr * weight_decay);
  h.rate = (float)(lr / (1.0 - pow(beta1, (double)step)));
  h.grad_scale = grad_scale;
  if (io == BLR_F32)
    return bits == 32 ? step_all<float, 32, false>(tensors, count, h, stream)
                      : step_all<float, 8, false>(tensors, count, h, stream);
  if (master)
    return bits == 32 ? step_all<__nv_bfloat16, 32, true>(tensors, count, h, stream)
                      : step_all<__nv_bfloat16, 8, true>(tensors, count, h, stream);
  return bits == 32 ? step_all<__nv_bfloat16, 32, false>(tensors, count, h, stream)
                    : step_all<__nv_bfloat16, 8, false>(tensors, count, h, stream);
}
