// 8-bit caches (Sec. 6 names KV-cache quantisation as compatible with the method): e4m3 bytes with one scale per KV head,
//   k ~ byte * k_scale[head],   v ~ byte * v_scale[head].
// kv8_scales finds the scales (largest magnitude at the top of the format, 448), kv8_write quantises rows as they enter the
// cache, with the encoding-time rotation of the keys on the way, kv8_read brings rows back.  All three are bound by memory:
// one pass, 16-byte accesses, a thread keeps the two channel ranges that the rotation pairs.  90k tokens of 8 heads of 128
// channels in bf16: scales 88 us (4.2 TB/s), write 105 (5.3 TB/s read and written); 27100 rows back to bf16: 36 us (4.6 TB/s);
// small calls are bound by the host's launch (an append of 16 tokens 10.4 us, the kernel 6.6).  Walking the write backwards,
// so that it begins with what the scales' pass left in the last-level cache, changed nothing.
#include <cstdint>

#include "kernels.hpp"

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kTop = 448.f;  // largest e4m3 value
constexpr int kPart = 16;      // channels of a piece: 16 bytes of cache

// sixteen elements as fp32
__device__ inline void load16(const __bf16* p, float (&x)[kPart]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bf16x8 v = reinterpret_cast<const bf16x8*>(p)[i];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[8 * i + e] = static_cast<float>(v[e]);
  }
}
__device__ inline void load16(const float* p, float (&x)[kPart]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const floatx4 v = reinterpret_cast<const floatx4*>(p)[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * i + e] = v[e];
  }
}
// channels i .. i+15 (lo) and their partners at + D/2 (hi), rotated by table row `row` in fp32
__device__ inline void rotate16(const float* row, int i, float (&lo)[kPart], float (&hi)[kPart]) {
  const floatx4* const cs = reinterpret_cast<const floatx4*>(row + 2 * i);
#pragma unroll
  for (int e = 0; e < kPart / 2; ++e) {
    const floatx4 t = cs[e];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const float c = t[2 * z], s = t[2 * z + 1], u = lo[2 * e + z], w = hi[2 * e + z];
      lo[2 * e + z] = fmaf(u, c, -(w * s));
      hi[2 * e + z] = fmaf(w, c, u * s);
    }
  }
}

__device__ inline int64_t thread_index() { return (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * 256 + threadIdx.x; }

__device__ inline const float* table_row(const Kv8Params& p, int tok) {
  int id = p.positions ? p.positions[tok] : p.first_id + tok;
  id = min(max(id, 0), p.n_pos - 1);
  return p.table + static_cast<int64_t>(id) * p.head_dim;
}

// What the quotients by a scale are made from.  A scale without a finite inverse (0, or so small that nothing divided by it
// is) quantises to zeros.
struct Divisor {
  float scale, inv;
};
__device__ inline Divisor divisor(float scale) {
  const float inv = 1.f / scale;
  return inv - inv == 0.f && scale - scale == 0.f ? Divisor{scale, inv} : Divisor{0.f, 0.f};
}

// x / scale to the nearest e4m3 value, ties to even; what lies beyond the format becomes its largest value, NaN stays NaN.  The
// quotient is x * inv (off by one step of fp32 or so) corrected by its exact remainder.  Without the correction values near a
// tie land on its other side: the bytes of a 90k pool differed from the same in elementary fp32 operations by 2.9e-3 (relative
// 2-norm), with it by 4e-5 to 1.4e-4 over several inputs (a rotated key, or a scale, one step of fp32 off; either side may be
// the closer one to 64 bits), for 197 us instead of 191.
__device__ inline uintx4 quantise16(const float (&x)[kPart], Divisor d) {
  uintx4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float z = x[4 * i + e] * d.inv;
      // (the sign from z: the correction turns -0 into 0)
      y[e] = z >= kTop ? kTop : z <= -kTop ? -kTop : copysignf(fmaf(fmaf(-z, d.scale, x[4 * i + e]), d.inv, z), z);
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    out[i] = static_cast<unsigned>(w);
  }
  return out;
}

// largest finite magnitude
__device__ inline void take_max(float& top, const float (&x)[kPart]) {
#pragma unroll
  for (int e = 0; e < kPart; ++e) {
    const float a = fabsf(x[e]);
    top = a < INFINITY ? fmaxf(top, a) : top;
  }
}

__global__ void kv8_zero_scales_kernel(float* k_scale, float* v_scale, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) k_scale[i] = v_scale[i] = 0.f;
}

// A workgroup takes tokens blockIdx.x, + gridDim.x, ... in groups, a thread the same (head, part) of each: its maxima stay in
// registers.  Scales are non-negative, so that their bits order like integers: one atomic maximum per workgroup and head,
// whose result does not depend on the order.  blockIdx.y: heads beyond the threads of a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void kv8_scales_kernel(Kv8Params p) {
  const int half_dim = p.head_dim / 2, parts = half_dim / kPart;  // 4 or 2
  const int heads_here = min(p.n_kv_heads - static_cast<int>(blockIdx.y) * (256 / parts), 256 / parts);
  const int per_token = heads_here * parts, tokens_here = 256 / per_token;
  const int in_tok = threadIdx.x % per_token, t0 = threadIdx.x / per_token;
  const int part = in_tok % parts, head_in = in_tok / parts, head = blockIdx.y * (256 / parts) + head_in;
  __shared__ unsigned top_sh[2][128];
  for (int i = threadIdx.x; i < 256; i += 256) top_sh[i / 128][i % 128] = 0;
  __syncthreads();
  float k_top = 0.f, v_top = 0.f;
  if (t0 < tokens_here) {
    for (int64_t tok = static_cast<int64_t>(blockIdx.x) * tokens_here + t0; tok < p.n_tokens; tok += static_cast<int64_t>(gridDim.x) * tokens_here) {
      const T* const kp = static_cast<const T*>(p.k.ptr) + tok * p.k.stride_tok + head * p.k.stride_head + part * kPart;
      const T* const vp = static_cast<const T*>(p.v.ptr) + tok * p.v.stride_tok + head * p.v.stride_head + part * kPart;
      float a[kPart], b[kPart], c[kPart], d[kPart];
      load16(kp, a);
      load16(kp + half_dim, b);
      load16(vp, c);
      load16(vp + half_dim, d);
      if (p.table) rotate16(table_row(p, static_cast<int>(tok)), part * kPart, a, b);
      take_max(k_top, a);
      take_max(k_top, b);
      take_max(v_top, c);
      take_max(v_top, d);
    }
    atomicMax(&top_sh[0][head_in], __float_as_uint(k_top));
    atomicMax(&top_sh[1][head_in], __float_as_uint(v_top));
  }
  __syncthreads();
  if (threadIdx.x < 2 * heads_here) {
    const int which = threadIdx.x / heads_here, h = threadIdx.x % heads_here;
    float* const scale = (which ? p.v_scale : p.k_scale) + blockIdx.y * (256 / parts) + h;
    atomicMax(reinterpret_cast<unsigned*>(scale), __float_as_uint(__uint_as_float(top_sh[which][h]) / kTop));
  }
}

// One thread: sixteen channels and their partners of K and of V, of one (token, head).
template <typename T>
__global__ __launch_bounds__(256) void kv8_write_kernel(Kv8Params p) {
  const int half_dim = p.head_dim / 2, parts = half_dim / kPart;
  const int64_t idx = thread_index();
  const int part = static_cast<int>(idx % parts);
  const int head = static_cast<int>((idx / parts) % p.n_kv_heads);
  const int64_t tok = idx / (static_cast<int64_t>(parts) * p.n_kv_heads);
  if (tok >= p.n_tokens) return;
  const int64_t row = p.rows ? p.rows[tok] : p.first_row + tok;
  if (row < 0 || row >= p.n_cache_rows) return;  // a token without a place
  const T* const kp = static_cast<const T*>(p.k.ptr) + tok * p.k.stride_tok + head * p.k.stride_head + part * kPart;
  const T* const vp = static_cast<const T*>(p.v.ptr) + tok * p.v.stride_tok + head * p.v.stride_head + part * kPart;
  float a[kPart], b[kPart], c[kPart], d[kPart];
  load16(kp, a);
  load16(kp + half_dim, b);
  load16(vp, c);
  load16(vp + half_dim, d);
  if (p.table) rotate16(table_row(p, static_cast<int>(tok)), part * kPart, a, b);
  const Divisor ki = divisor(p.k_scale[head]), vi = divisor(p.v_scale[head]);
  unsigned char* const ko = static_cast<unsigned char*>(const_cast<void*>(p.k8.ptr)) + row * p.k8.stride_tok + head * p.k8.stride_head + part * kPart;
  unsigned char* const vo = static_cast<unsigned char*>(const_cast<void*>(p.v8.ptr)) + row * p.v8.stride_tok + head * p.v8.stride_head + part * kPart;
  *reinterpret_cast<uintx4*>(ko) = quantise16(a, ki);
  *reinterpret_cast<uintx4*>(ko + half_dim) = quantise16(b, ki);
  *reinterpret_cast<uintx4*>(vo) = quantise16(c, vi);
  *reinterpret_cast<uintx4*>(vo + half_dim) = quantise16(d, vi);
}

// One thread: as many channels of K and of V as make sixteen bytes of the result, so that a wave's stores fill whole lines
// (16 channels to a thread, two or four stores of it 16 bytes apart: 41 us for 27100 rows, so 36.4).
template <typename T>
__global__ __launch_bounds__(256) void kv8_read_kernel(Kv8Params p) {
  constexpr int kCh = 16 / sizeof(T);
  typedef T out_t __attribute__((ext_vector_type(kCh)));
  typedef unsigned raw_t __attribute__((ext_vector_type(2)));
  const int parts = p.head_dim / kCh;
  const int64_t idx = thread_index();
  const int part = static_cast<int>(idx % parts);
  const int head = static_cast<int>((idx / parts) % p.n_kv_heads);
  const int64_t tok = idx / (static_cast<int64_t>(parts) * p.n_kv_heads);
  if (tok >= p.n_tokens) return;
  const int64_t row = p.rows ? p.rows[tok] : p.first_row + tok;
  const bool there = row >= 0 && row < p.n_cache_rows;  // (a row that is not gives zeros)
  auto stored = [&](const TensorView& from) {
    raw_t raw{0, 0};
    if (there) {
      const unsigned* const at = reinterpret_cast<const unsigned*>(static_cast<const unsigned char*>(from.ptr) + row * from.stride_tok + head * from.stride_head + part * kCh);
      if constexpr (kCh == 8) raw = *reinterpret_cast<const raw_t*>(at);
      else raw[0] = *at;
    }
    return raw;
  };
  auto bring = [&](const raw_t& raw, const TensorView& to, float scale) {
    out_t x;
#pragma unroll
    for (int i = 0; i < kCh / 4; ++i) {
      const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(raw[i]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(raw[i]), true);
      x[4 * i] = static_cast<T>(lo[0] * scale);
      x[4 * i + 1] = static_cast<T>(lo[1] * scale);
      x[4 * i + 2] = static_cast<T>(hi[0] * scale);
      x[4 * i + 3] = static_cast<T>(hi[1] * scale);
    }
    *reinterpret_cast<out_t*>(static_cast<T*>(const_cast<void*>(to.ptr)) + tok * to.stride_tok + head * to.stride_head + part * kCh) = x;
  };
  const raw_t k8 = stored(p.k8), v8 = stored(p.v8);  // (both, before the stores that they may not pass)
  // (a scale may be infinite or no number, and zero times it is none)
  const float k_scale = there ? p.k_scale[head] : 0.f, v_scale = there ? p.v_scale[head] : 0.f;
  bring(k8, p.k, k_scale);
  bring(v8, p.v, v_scale);
}

// A grid counts its threads per dimension in 32 bits.
dim3 grid_of(int64_t threads) {
  const int64_t blocks = (threads + 255) / 256, wide = int64_t{1} << 23;
  return blocks <= wide ? dim3(static_cast<unsigned>(blocks)) : dim3(static_cast<unsigned>(wide), static_cast<unsigned>((blocks + wide - 1) / wide));
}

}  // namespace

hipError_t launch_kv8_scales(const Kv8Params& p, bool bf16, bool running, hipStream_t stream) {
  if (!running) {
    kv8_zero_scales_kernel<<<grid_of(p.n_kv_heads), dim3(256), 0, stream>>>(p.k_scale, p.v_scale, p.n_kv_heads);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  if (p.n_tokens == 0) return hipSuccess;
  const int parts = p.head_dim / 2 / kPart, heads = 256 / parts;  // of a workgroup: at most 64 or 128 heads
  const int tokens = 256 / (parts * (p.n_kv_heads < heads ? p.n_kv_heads : heads));
  const int64_t wanted = (static_cast<int64_t>(p.n_tokens) + tokens - 1) / tokens;
  const dim3 grid(static_cast<unsigned>(wanted < 2048 ? wanted : 2048), static_cast<unsigned>((p.n_kv_heads + heads - 1) / heads));
  if (bf16) kv8_scales_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(p);
  else kv8_scales_kernel<float><<<grid, dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_kv8_write(const Kv8Params& p, bool bf16, hipStream_t stream) {
  if (p.n_tokens == 0) return hipSuccess;
  const dim3 grid = grid_of(static_cast<int64_t>(p.n_tokens) * p.n_kv_heads * (p.head_dim / 2 / kPart));
  if (bf16) kv8_write_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(p);
  else kv8_write_kernel<float><<<grid, dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_kv8_read(const Kv8Params& p, bool bf16, hipStream_t stream) {
  if (p.n_tokens == 0) return hipSuccess;
  const dim3 grid = grid_of(static_cast<int64_t>(p.n_tokens) * p.n_kv_heads * (p.head_dim / (bf16 ? 8 : 4)));
  if (bf16) kv8_read_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(p);
  else kv8_read_kernel<float><<<grid, dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}
