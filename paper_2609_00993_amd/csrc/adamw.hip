// An AdamW step over many tensors, with states in 32 bits or in blocks of 8 (include/moepd_adamw.h).
// One launch: the table lists every chunk's tensor, a workgroup takes one chunk.  What bounds
// it is memory: 28 bytes an element with 32-bit states beside bf16 weights and float32
// masters, 16.1 with 8-bit states.  201 million elements: 1088 us and 624, 5.2 TB/s both (a copy: 5.03); with nontemporal
// accesses 1180 and 652.
#include <math.h>
#include <string.h>

#include <memory>
#include <vector>

#include "common.h"
#include "moepd_adamw.h"
#include "swiglu.h"
#include "tiles.h"

namespace moepd {
namespace {

struct AdamTensor {
  uint8_t* param;
  float* master;
  const uint8_t* grad;
  uint8_t* m;
  uint8_t* v;
  uint8_t* ms;
  uint8_t* vs;
  long long n;
  long long first;  // its first chunk
  float decay;
  int32_t param_bf16, grad_bf16;
  int32_t reserved;
};

struct AdamArgs {
  const AdamTensor* tensors;
  const int32_t* tensor_of;  // each chunk's
  long long chunks;
  int runs;  // of 2048 elements to a chunk
  float b1, a1, b2, a2, eps;
  double log_b1, log_b2;
  const float* lr;
  const int32_t* step;
  const float* scale;
  uint32_t seed;
};

constexpr int kAdamRun = 256 * 8;  // elements of a workgroup's pass
constexpr int kAdamRuns = 4;       // passes of a chunk of a large table

typedef uint32_t u32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any1 __attribute__((ext_vector_type(2), aligned(1)));

__device__ __forceinline__ uint32_t adam_mix(uint32_t a) {
  a ^= a >> 16;
  a *= 0x6A09E667u;
  a ^= a >> 15;
  a *= 0xBB67AE85u;
  return a ^ (a >> 16);
}

// 8 elements from `at` on (those past n as 0), and back.
__device__ __forceinline__ void adam_load(const uint8_t* p, bool bf16, long long at, int in, float (&v)[8]) {
  if (in >= 8) {
    if (bf16) {
      const u32x4_any q = *reinterpret_cast<const u32x4_any*>(p + 2 * at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(q[i] << 16);
        v[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
      }
    } else {
      const u32x4_any4 a = *reinterpret_cast<const u32x4_any4*>(p + 4 * at);
      const u32x4_any4 b = *reinterpret_cast<const u32x4_any4*>(p + 4 * at + 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = __uint_as_float(a[i]);
        v[4 + i] = __uint_as_float(b[i]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.f;
      if (i < in) v[i] = bf16 ? bf16_to_f32(reinterpret_cast<const uint16_t*>(p)[at + i]) : reinterpret_cast<const float*>(p)[at + i];
    }
  }
}
__device__ __forceinline__ void adam_store(uint8_t* p, bool bf16, long long at, int in, const float (&v)[8]) {
  if (in >= 8) {
    if (bf16) {
      *reinterpret_cast<u32x4_any*>(p + 2 * at) =
          u32x4_any{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    } else {
      *reinterpret_cast<u32x4_any4*>(p + 4 * at) =
          u32x4_any4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
      *reinterpret_cast<u32x4_any4*>(p + 4 * at + 16) =
          u32x4_any4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < in) {
        if (bf16) reinterpret_cast<uint16_t*>(p)[at + i] = f32_to_bf16(v[i]);
        else reinterpret_cast<float*>(p)[at + i] = v[i];
      }
  }
}
__device__ __forceinline__ uint64_t adam_load_codes(const uint8_t* p, long long at, int in) {
  if (in >= 8) {
    const u32x2_any1 q = *reinterpret_cast<const u32x2_any1*>(p + at);
    return q[0] | (uint64_t)q[1] << 32;
  }
  uint64_t c = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < in) c |= (uint64_t)p[at + i] << (8 * i);
  return c;
}
__device__ __forceinline__ void adam_store_codes(uint8_t* p, long long at, int in, uint64_t c) {
  if (in >= 8) {
    *reinterpret_cast<u32x2_any1*>(p + at) = u32x2_any1{(uint32_t)c, (uint32_t)(c >> 32)};
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < in) p[at + i] = (uint8_t)(c >> (8 * i));
}

// What a block's scale byte multiplies by.
__device__ __forceinline__ float adam_scale(uint32_t S) {
  return __uint_as_float(S == 255u ? 0x7fc00000u : S == 0u ? 0x00400000u : S << 23);
}
// m from E4M3, the square root of v from five exponent and three mantissa bits.
__device__ __forceinline__ void adam_decode_m(uint64_t c, float s, float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int w = (int)(uint32_t)(c >> (32 * h));
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    v[4 * h] = lo[0] * s;
    v[4 * h + 1] = lo[1] * s;
    v[4 * h + 2] = hi[0] * s;
    v[4 * h + 3] = hi[1] * s;
  }
}
__device__ __forceinline__ void adam_decode_v(uint64_t c, float s, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = (uint32_t)(c >> (8 * i)) & 255u;
    const float f = __uint_as_float((b << 20) + (97u << 23));  // (1 + f / 8) 2^(e - 30)
    v[i] = (b < 8u ? 2.f * (f - 0x1p-30f) : f) * s;
  }
}

// The scale byte that puts a block's largest magnitude (its bits, over the four lanes that hold
// the block) into [2^above, 2^(above + 1)).
__device__ __forceinline__ uint32_t adam_block_scale(uint32_t bits, int above) {
  uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)bits, 0xB1, 0xF, 0xF, false);  // quad_perm [1,0,3,2]
  bits = o > bits ? o : bits;
  o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)bits, 0x4E, 0xF, 0xF, false);  // quad_perm [2,3,0,1]
  bits = o > bits ? o : bits;
  if (bits >= 0x7f800000u) return 255u;
  if (bits == 0u) return 0u;
  const int S = __builtin_amdgcn_frexp_expf(__uint_as_float(bits)) - 1 - above + 127;
  return (uint32_t)(S < 0 ? 0 : S > 254 ? 254 : S);
}
// A magnitude under a block's scale to a code of three mantissa bits whose smallest normal number
// is 2^LOW: the cut-off 20 mantissa bits and r 2^4 carry into the code, below 2^LOW in steps of 2^(LOW - 3).
template <int LOW>
__device__ __forceinline__ uint32_t adam_code(float q, uint32_t r) {
  const uint32_t normal = ((__float_as_uint(q) + (r << 4)) >> 20) - ((126u + LOW) << 3);
  const uint32_t low = (uint32_t)__builtin_fmaf(q, __uint_as_float((127u + 3u - LOW) << 23), (float)r * 0x1p-16f);
  return q < __uint_as_float((127u + LOW) << 23) ? low : normal;
}

// The hardware's root (1 ulp), which takes numbers below the normal ones as 0: with a small eps, or
// none, these are what an update is divided by.
__device__ __forceinline__ float adam_root(float v) {
  const bool low = v < 0x1p-126f;
  return __builtin_amdgcn_sqrtf(v * (low ? 0x1p64f : 1.f)) * (low ? 0x1p-32f : 1.f);
}

template <bool SMALL>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
  const long long chunk = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (chunk >= a.chunks) return;
  const float scale = a.scale ? *a.scale : 1.f;
  if (!(__builtin_fabsf(scale) < INFINITY)) return;
  const int number = __builtin_amdgcn_readfirstlane(a.tensor_of[chunk]);
  const AdamTensor t = a.tensors[number];
  const int steps = max(*a.step, 1);
  const float lr = *a.lr;
  // 1 - beta^t without its cancellation for small t
  const float c1 = -expm1f((float)(steps * a.log_b1)), c2 = -expm1f((float)(steps * a.log_b2));
  const float i1 = 1.f / c1, i2 = 1.f / sqrtf(c2);
  const uint32_t key0 = adam_mix(adam_mix(adam_mix(a.seed) + (uint32_t)steps) + (uint32_t)number);
  const long long base = (chunk - t.first) * a.runs * (long long)kAdamRun;
  for (int run = 0; run < a.runs; ++run) {
    const long long at = base + (long long)run * kAdamRun + 8 * threadIdx.x;
    if (base + (long long)run * kAdamRun >= t.n) return;
    const long long left = t.n - at;
    const int in = left < 0 ? 0 : left > 8 ? 8 : (int)left;
    float g[8], p[8], m[8], v[8];
    const bool own = !t.master;
    adam_load(t.grad, t.grad_bf16, at, in, g);
    adam_load(own ? t.param : (const uint8_t*)t.master, own && t.param_bf16, at, in, p);
    if constexpr (SMALL) {
      const uint64_t mc = adam_load_codes(t.m, at, in), vc = adam_load_codes(t.v, at, in);
      adam_decode_m(mc, adam_scale(in > 0 ? t.ms[at / 32] : 0u), m);
      adam_decode_v(vc, adam_scale(in > 0 ? t.vs[at / 32] : 0u), v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= v[i];
    } else {
      adam_load(t.m, false, at, in, m);
      adam_load(t.v, false, at, in, v);
    }
    {
#pragma clang fp contract(off)  // the roundings of the formulas as they stand
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        g[i] *= scale;
        m[i] = a.b1 * m[i] + a.a1 * g[i];
        v[i] = a.b2 * v[i] + a.a2 * g[i] * g[i];
      }
    }
    float root[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      root[i] = SMALL ? sqrtf(v[i]) : adam_root(v[i]);
      // the hardware's reciprocal, too, takes numbers below the normal ones as 0
      const float d = __builtin_fmaf(root[i], i2, a.eps), k = d < 0x1p-64f ? 0x1p64f : 1.f;
      const float u = m[i] * i1 * k * __builtin_amdgcn_rcpf(d * k);
      p[i] -= lr * __builtin_fmaf(t.decay, p[i], u);
    }
    if (t.master) adam_store((uint8_t*)t.master, false, at, in, p);
    adam_store(t.param, t.param_bf16, at, in, p);
    if constexpr (SMALL) {
      const uint32_t hi = (uint32_t)(at >> 32);
      const uint32_t key = hi ? adam_mix(key0 + hi) : key0;
      uint32_t mb = 0, vb = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i >= in) m[i] = root[i] = 0.f;
        const uint32_t x = __float_as_uint(m[i]) & 0x7fffffffu, y = __float_as_uint(root[i]) & 0x7fffffffu;
        mb = x > mb ? x : mb;
        vb = y > vb ? y : vb;
      }
      const uint32_t S = adam_block_scale(mb, 7), R = adam_block_scale(vb, 0);
      uint64_t mc = 0, vc = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t word = adam_mix(((uint32_t)at + i) ^ key);
        uint32_t x = adam_code<-6>(ldexpf(__builtin_fabsf(m[i]), 127 - (int)S), word >> 16);
        uint32_t y = adam_code<-29>(ldexpf(root[i], 127 - (int)R), word & 0xffffu);
        x |= m[i] < 0.f ? 128u : 0u;
        y = root[i] > 0.f && y == 0u ? 1u : y;
        mc |= (uint64_t)(S == 255u ? 0u : x) << (8 * i);
        vc |= (uint64_t)(R == 255u ? 0u : y) << (8 * i);
      }
      adam_store_codes(t.m, at, in, mc);
      adam_store_codes(t.v, at, in, vc);
      if (in > 0 && (threadIdx.x & 3) == 0) {
        t.ms[at / 32] = (uint8_t)S;
        t.vs[at / 32] = (uint8_t)R;
      }
    } else {
      adam_store(t.m, false, at, in, m);
      adam_store(t.v, false, at, in, v);
    }
  }
}

template <bool SMALL>
__global__ __launch_bounds__(256) void adamw_read_kernel(AdamTensor t, uint8_t* m_out, uint8_t* v_out, bool bf16) {
  const long long at = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * kAdamRun + 8 * threadIdx.x;
  const long long left = t.n - at;
  if (left <= 0) return;
  const int in = left > 8 ? 8 : (int)left;
  float v[8];
  if (m_out) {
    if constexpr (SMALL) adam_decode_m(adam_load_codes(t.m, at, in), adam_scale(t.ms[at / 32]), v);
    else adam_load(t.m, false, at, in, v);
    adam_store(m_out, bf16, at, in, v);
  }
  if (v_out) {
    if constexpr (SMALL) {
      adam_decode_v(adam_load_codes(t.v, at, in), adam_scale(t.vs[at / 32]), v);
    } else {
      adam_load(t.v, false, at, in, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = sqrtf(v[i]);
    }
    adam_store(v_out, bf16, at, in, v);
  }
}

bool type_ok(int32_t t) { return t == MOE_DTYPE_F32 || t == MOE_DTYPE_BF16; }
bool at_element(const void* p, int32_t t) { return (uintptr_t)p % (t == MOE_DTYPE_F32 ? 4 : 2) == 0; }

}  // namespace
}  // namespace moepd

using namespace moepd;

struct moe_adamw {
  int device = 0;
  int bits = 32;
  void* mem = nullptr;
  const AdamTensor* tensors = nullptr;
  const int32_t* tensor_of = nullptr;
  long long chunks = 0;
  int runs = 1;
  std::vector<AdamTensor> host;
};

extern "C" {

int moe_adamw_create(const moe_adamw_tensor_t* tensors, int32_t count, int32_t state_bits, moe_adamw_t** out) {
  if (out) *out = nullptr;
  if (!out || !tensors || count < 1 || count > 65536 || (state_bits != 32 && state_bits != 8)) return MOE_ERR_INVALID_ARG;
  const bool small = state_bits == 8;
  long long total = 0;
  for (int i = 0; i < count; ++i) {
    const moe_adamw_tensor_t& t = tensors[i];
    if (t.n < 0 || t.n > (1LL << 40) || !type_ok(t.param_dtype) || !type_ok(t.grad_dtype) || !isfinite(t.weight_decay))
      return MOE_ERR_INVALID_ARG;
    if (t.n == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v || (small && (!t.m_scales || !t.v_scales)) ||
        (!small && (t.m_scales || t.v_scales)))
      return MOE_ERR_INVALID_ARG;
    if (!at_element(t.param, t.param_dtype) || !at_element(t.grad, t.grad_dtype) || (uintptr_t)t.master % 4 ||
        (!small && ((uintptr_t)t.m | (uintptr_t)t.v) % 4))
      return MOE_ERR_INVALID_ARG;
    total += (t.n + kAdamRun - 1) / kAdamRun;
  }
  // Chunks of four passes where these still make 16 workgroups a CU.
  const int runs = total >= 4 * 4096 ? kAdamRuns : 1;
  try {
    std::vector<AdamTensor> host((size_t)count);
    std::vector<int32_t> of;
    long long chunks = 0;
    for (int i = 0; i < count; ++i) {
      const moe_adamw_tensor_t& t = tensors[i];
      const long long each = (long long)kAdamRun * runs, here = (t.n + each - 1) / each;
      host[i] = AdamTensor{(uint8_t*)t.param, t.master, (const uint8_t*)t.grad, (uint8_t*)t.m, (uint8_t*)t.v, t.m_scales,
                           t.v_scales, t.n, chunks, (float)t.weight_decay, t.param_dtype == MOE_DTYPE_BF16,
                           t.grad_dtype == MOE_DTYPE_BF16, 0};
      chunks += here;
      if (chunks > (1LL << 31) - (1 << 16)) return MOE_ERR_INVALID_ARG;
      of.insert(of.end(), (size_t)here, i);
    }
    std::unique_ptr<moe_adamw> h(new moe_adamw);
    h->bits = state_bits;
    h->chunks = chunks;
    h->runs = runs;
    const size_t table = sizeof(AdamTensor) * (size_t)count, list = sizeof(int32_t) * of.size();
    std::vector<uint8_t> bytes(table + list);
    memcpy(bytes.data(), host.data(), table);
    if (list) memcpy(bytes.data() + table, of.data(), list);
    h->host.swap(host);
    int st = MOE_OK;
    if (hipGetDevice(&h->device) != hipSuccess) st = MOE_ERR_HIP;
    else if (hipMalloc(&h->mem, bytes.size()) != hipSuccess) st = MOE_ERR_OOM;
    else if (hipMemcpy(h->mem, bytes.data(), bytes.size(), hipMemcpyHostToDevice) != hipSuccess) st = MOE_ERR_HIP;
    if (st != MOE_OK) {
      (void)hipGetLastError();
      if (h->mem) (void)hipFree(h->mem);
      return st;
    }
    h->tensors = static_cast<const AdamTensor*>(h->mem);
    h->tensor_of = reinterpret_cast<const int32_t*>(static_cast<uint8_t*>(h->mem) + table);
    *out = h.release();
    return MOE_OK;
  } catch (...) {
    return MOE_ERR_OOM;
  }
}

int moe_adamw_step(moe_adamw_t* h, double beta1, double beta2, double eps, const float* lr, const int32_t* step,
                   const float* grad_scale, uint32_t seed, hipStream_t stream) {
  if (!h || !stream || !lr || !step || ((uintptr_t)lr | (uintptr_t)step | (uintptr_t)grad_scale) % 4)
    return MOE_ERR_INVALID_ARG;
  if (!(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) || !(eps >= 0) || !isfinite(eps)) return MOE_ERR_INVALID_ARG;
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess) return MOE_ERR_HIP;
  if (device != h->device) return MOE_ERR_INVALID_ARG;
  if (h->chunks == 0) return MOE_OK;
  const float eps32 = eps > 0 ? fmaxf((float)eps, 0x1p-149f) : 0.f;  // above 0, as eps is: 0 / eps stays 0
  const AdamArgs a{h->tensors, h->tensor_of, h->chunks, h->runs, (float)beta1, (float)(1.0 - beta1), (float)beta2,
                   (float)(1.0 - beta2), eps32, log(beta1), log(beta2), lr, step, grad_scale, seed};
  const dim3 grid = grid_of(h->chunks, 256);
  if (h->bits == 8) adamw_kernel<true><<<grid, 256, 0, stream>>>(a);
  else adamw_kernel<false><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_adamw_read(moe_adamw_t* h, int32_t index, void* m, void* root_v, int32_t dtype, hipStream_t stream) {
  if (!h || !stream || index < 0 || (size_t)index >= h->host.size() || !type_ok(dtype) || !at_element(m, dtype) ||
      !at_element(root_v, dtype))
    return MOE_ERR_INVALID_ARG;
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess) return MOE_ERR_HIP;
  if (device != h->device) return MOE_ERR_INVALID_ARG;
  const AdamTensor& t = h->host[(size_t)index];
  if (t.n == 0 || (!m && !root_v)) return MOE_OK;
  const dim3 grid = grid_of((t.n + kAdamRun - 1) / kAdamRun, 256);
  const bool bf16 = dtype == MOE_DTYPE_BF16;
  if (h->bits == 8) adamw_read_kernel<true><<<grid, 256, 0, stream>>>(t, (uint8_t*)m, (uint8_t*)root_v, bf16);
  else adamw_read_kernel<false><<<grid, 256, 0, stream>>>(t, (uint8_t*)m, (uint8_t*)root_v, bf16);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_adamw_destroy(moe_adamw_t* h) {
  if (!h) return MOE_OK;
  // freeing waits for the device's work
  int device = -1, st = MOE_OK;
  if (hipGetDevice(&device) != hipSuccess || (device != h->device && hipSetDevice(h->device) != hipSuccess)) st = MOE_ERR_HIP;
  if (hipFree(h->mem) != hipSuccess) st = MOE_ERR_HIP;
  if (device >= 0 && device != h->device) (void)hipSetDevice(device);
  delete h;
  return st;
}

}  // extern "C"
