// The operators around a block of experts: its output joined with the residual stream and normed for the next block
// (moe_lrc_norm_join), and activations brought to 8-bit floating point in blocks of 128 (moe_lrc_block_quantize).
#include <cmath>

#include "internal.h"
#include "route_body.h"

namespace lrc {
namespace {

constexpr float kE4m3Max = 448.f, kSmallestScale = 0x1p-126f;

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// two floats to bf16, to the nearest, ties to even, NaN kept
__device__ inline uint32_t bf16_pair(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 p = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, p);
}
__device__ inline void unpack8(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
}
__device__ inline uint4 pack8(const float (&f)[8]) {
  return make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
}
__device__ inline void load8(const float* p, float (&f)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ inline void store8(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

template <int OFF> __device__ inline float sum_step(float v) {
  uint32_t a, b;
  lane_pair<OFF>(__float_as_uint(v), a, b);
  return __uint_as_float(a) + __uint_as_float(b);
}
__device__ inline float wave_sum_f32(float v) {
  v = sum_step<32>(v); v = sum_step<16>(v); v = sum_step<8>(v);
  v = sum_step<4>(v); v = sum_step<2>(v); return sum_step<1>(v);
}
template <int OFF> __device__ inline uint32_t max_step(uint32_t v) {
  uint32_t a, b;
  lane_pair<OFF>(v, a, b);
  return max(a, b);
}

// u g / (1 + exp(-g)) within 8 units of 2^-24, from t = exp(-|g|), which cannot overflow: t = 2^hi (1 + lo ln 2) with -|g| log2(e) =
// hi + lo in two words, so that v_exp_f32's one rounding is all that a large |g| costs; the quotient by v_rcp_f32 and one step of
// Newton's.  The library's exp and an IEEE division take the kernel from the memory's time to the vector units'.
// v_exp_f32 gives 0 below 2^-126, but u can lift the product of a smaller t back into the normal range.  FAR, for lanes that have such
// a gate (2048 x 14336 with it for all lanes 33.1 us, for those 31.6, without 31.1): below 2^-100 t is taken 2^160 times as large, of which one half goes into
// u and one into the product, so that only the result can underflow.
constexpr float kFarGate = -69.f;                          // (exp(-69) = 2^-99.5)
template <bool FAR> __device__ inline float silu_product(float g, float u) {
#pragma clang fp contract(off)                             // (hi + 160 from the product before its rounding would count lo twice)
  const float x = fmaxf(-fabsf(g), FAR ? -300.f : -200.f), hi = x * 1.44269504f;
  const float lo = fmaf(x, 1.925963e-8f, fmaf(x, 1.44269504f, -hi));           // (the second constant: what the first leaves of log2(e))
  const bool far = FAR && hi < -100.f;
  const float t0 = __builtin_amdgcn_exp2f(far ? hi + 160.f : hi), t = fmaf(t0, lo * 0.693147181f, t0), d = far ? 1.f : 1.f + t;
  float r = __builtin_amdgcn_rcpf(d);
  r = fmaf(fmaf(-d, r, 1.f), r, r);
  const float back = far && g < 0.f ? 0x1p-80f : 1.f, y = g * (g < 0.f ? t : 1.f) * r;
  return FAR ? y * (u * back) * back : y * u;
}

// Eight neighbouring values of a block of 128, which 16 neighbouring lanes of a row hold (lanes past its end: zeros): the
// block's scale and the eight codes.  The largest magnitude is taken of the bit patterns, in which an infinity or a NaN is above
// every number.  Both quotients are those of an IEEE division, from a product with the reciprocal and one correction by what it leaves:
// where a block's largest value makes ties of others, a scale or quotient that is one unit off decides them the other way, a
// whole code apart.  The correction is exact unless that remainder underflows, hence the division for the smallest scales.
__device__ inline float corrected_quotient(float a, float b, float inv) {
  const float q = a * inv;
  return fmaf(fmaf(-b, q, a), inv, q);
}
__device__ inline uint2 quantize8(const float (&v)[8], float& scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  top = max_step<1>(max_step<2>(max_step<4>(max_step<8>(top))));
  scale = top == 0 ? 1.f : fmaxf(corrected_quotient(__uint_as_float(top), kE4m3Max, 1.f / kE4m3Max), kSmallestScale);
  if (top >= 0x7f800000u) scale = __builtin_nanf("");
  const float inv = 1.f / scale;
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = corrected_quotient(v[i], scale, inv);
  if (scale < 0x1p-90f)
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = v[i] / scale;
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = __builtin_amdgcn_fmed3f(q[i], -kE4m3Max, kE4m3Max);       // (a product may round past the largest code's value)
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
  return make_uint2(uint32_t(lo), uint32_t(hi));
}

// W wavefronts a row (one: four rows to a block), V chunks of eight columns a lane.  A row stays in registers from its one
// read to its one write; sums of squares, the residual sum and the norm are fp32, and what is written is rounded once.  Rows of up to 1024
// columns take a wavefront each and need no barrier; longer ones four or eight, so that a lane holds at most 32 columns of both inputs.
// Bound: memory where there are many rows (2048 x 4096, gate per token, all four outputs: 14.1 us for 76 MB, 5.4 TB/s, the inputs partly
// from the last cache); the two chains of row sum and launch where there are few (1 x 4096: 3.4 us on the GPU, 333 x 2048 in fp32 5.0).
template <int V, int W, bool R32>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void join_kernel(const moe_lrc_join j) {
  constexpr int kLanes = 64 * W;
  __shared__ float part[2][W];
  const int tid = W == 1 ? threadIdx.x & 63 : threadIdx.x, wave = threadIdx.x >> 6;
  const size_t t = W == 1 ? size_t(blockIdx.x) * 4 + wave : blockIdx.x;
  if (t >= size_t(j.T)) return;                            // (a whole wavefront, and with W > 1 no such block)
  const int H = j.H, chunks = H / 8;
  const uint16_t* branch = reinterpret_cast<const uint16_t*>(j.branch) + t * j.branch_stride;
  float b[V][8], u[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = tid + kLanes * v;
    const bool in = c < chunks;
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (j.branch && in) raw = reinterpret_cast<const uint4*>(branch)[c];
    unpack8(raw, b[v]);
#pragma unroll
    for (int i = 0; i < 8; ++i) u[v][i] = 0.f;
    if (j.residual && in) {
      if constexpr (R32) load8(reinterpret_cast<const float*>(j.residual) + t * j.residual_stride + 8 * c, u[v]);
      else unpack8(reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(j.residual) + t * j.residual_stride)[c], u[v]);
    }
  }
  auto row_sum = [&](float s, int at) {
    s = wave_sum_f32(s);
    if constexpr (W > 1) {
      if ((tid & 63) == 0) part[at][wave] = s;
      __syncthreads();
      s = part[at][0];
#pragma unroll
      for (int w = 1; w < W; ++w) s += part[at][w];
    }
    return s;
  };
  if (j.branch) {
    float rstd = j.scale;
    if (j.post_weight) {
      float s = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(b[v][i], b[v][i], s);
      rstd *= rsqrtf(row_sum(s, 0) / float(H) + j.eps);
    }
    if (j.gate_kind == MOE_LRC_GATE_TOKEN) rstd *= reinterpret_cast<const float*>(j.gate)[t * j.gate_stride];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = tid + kLanes * v;
      if (c >= chunks) continue;
      float f[8];
      if (j.post_weight) {
        load8(j.post_weight + 8 * c, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) b[v][i] *= f[i];
      }
      if (j.gate_kind == MOE_LRC_GATE_CHANNEL || j.gate_kind == MOE_LRC_GATE_ELEMENT) {
        if (j.gate_kind == MOE_LRC_GATE_CHANNEL) load8(reinterpret_cast<const float*>(j.gate) + 8 * c, f);
        else unpack8(reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(j.gate) + t * j.gate_stride)[c], f);
#pragma unroll
        for (int i = 0; i < 8; ++i) b[v][i] *= f[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) u[v][i] = fmaf(b[v][i], rstd, u[v][i]);
    }
  }
  if (j.out_residual) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = tid + kLanes * v;
      if (c >= chunks) continue;
      if constexpr (R32) store8(reinterpret_cast<float*>(j.out_residual) + t * j.out_residual_stride + 8 * c, u[v]);
      else reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(j.out_residual) + t * j.out_residual_stride)[c] = pack8(u[v]);
    }
  }
  if (!j.out_norm && !j.codes) return;
  float s = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(u[v][i], u[v][i], s);
  const float rstd = rsqrtf(row_sum(s, 1) / float(H) + j.eps);
  const int blocks = (H + 127) / 128;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = tid + kLanes * v;
    const bool in = c < chunks;
    float f[8];
    if (in) load8(j.pre_weight + 8 * c, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) u[v][i] = in ? u[v][i] * rstd * f[i] : 0.f;
    if (j.out_norm && in) reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(j.out_norm) + t * j.out_norm_stride)[c] = pack8(u[v]);
    if (j.codes) {
      float scale;
      const uint2 q = quantize8(u[v], scale);
      if (in) reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(j.codes) + t * H)[c] = q;
      if (in && (tid & 15) == 0) j.scales[t * blocks + c / 16] = scale;
    }
  }
}

// 16 lanes a block of 128, 16 such blocks of one row to a workgroup: one 16-byte load of each half and one 8-byte store a lane, nothing shared.
// Bound: memory, near a copy's rate: SwiGLU of 2048 x 14336 31.6 us for 148 MB, 4.7 TB/s (a 2 GiB copy 4.96; 29.5 us without the correction of the
// quotients and the look for far gates, so the vector units are as good as full); 64 x 14336 3.4 us on the GPU.
template <bool SWIGLU>
__global__ __launch_bounds__(256) void quantize_kernel(const uint16_t* __restrict__ x, int64_t stride, int K, int per_row,
                                                       uint8_t* __restrict__ codes, float* __restrict__ scales) {
  const size_t t = blockIdx.x / per_row;
  const int c = (int(blockIdx.x) - int(t) * per_row) * 256 + int(threadIdx.x), chunks = K / 8;
  const bool in = c < chunks;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (in) {
    const uint16_t* row = x + t * stride;
    unpack8(reinterpret_cast<const uint4*>(row)[c], v);
    if constexpr (SWIGLU) {
      float u[8];
      unpack8(reinterpret_cast<const uint4*>(row + K)[c], u);
      float least = v[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) least = fminf(least, v[i]);
      if (least < kFarGate) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = silu_product<true>(v[i], u[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = silu_product<false>(v[i], u[i]);
      }
    }
  }
  float scale;
  const uint2 q = quantize8(v, scale);
  if (in) reinterpret_cast<uint2*>(codes + t * K)[c] = q;
  if (in && (threadIdx.x & 15) == 0) scales[t * ((K + 127) / 128) + c / 16] = scale;
}

bool misaligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) & (bytes - 1); }

template <bool R32> hipError_t launch_join(const moe_lrc_join& j, hipStream_t s) {
  const int chunks = j.H / 8;
  auto go = [&](auto kernel, int rows, int threads) {
    hipLaunchKernelGGL(kernel, dim3((j.T + rows - 1) / rows), dim3(threads), 0, s, j);
  };
  if (chunks <= 64) go(join_kernel<1, 1, R32>, 4, 256);
  else if (chunks <= 128) go(join_kernel<2, 1, R32>, 4, 256);
  else if (chunks <= 256) go(join_kernel<1, 4, R32>, 1, 256);
  else if (chunks <= 512) go(join_kernel<2, 4, R32>, 1, 256);
  else if (chunks <= 1024) go(join_kernel<4, 4, R32>, 1, 256);
  else go(join_kernel<4, 8, R32>, 1, 512);
  return hipGetLastError();
}

}  // namespace
}  // namespace lrc

using namespace lrc;

extern "C" {

int moe_lrc_norm_join(const moe_lrc_join* jp, void* stream) {
  if (!jp) return set_error(MOE_LRC_EINVAL, "norm_join: null argument");
  const moe_lrc_join& j = *jp;
  if (j.T < 0 || j.T > (1 << 22)) return set_error(MOE_LRC_EINVAL, "norm_join: T outside 0..2^22");
  if (j.H < 8 || j.H > 16384 || j.H % 8) return set_error(MOE_LRC_ESHAPE, "norm_join: H must be a multiple of 8 in 8..16384");
  if (j.residual_f32 != 0 && j.residual_f32 != 1) return set_error(MOE_LRC_EINVAL, "norm_join: residual_f32 must be 0 or 1");
  if (j.gate_kind < MOE_LRC_GATE_NONE || j.gate_kind > MOE_LRC_GATE_ELEMENT) return set_error(MOE_LRC_EINVAL, "norm_join: unknown gate_kind");
  if (!std::isfinite(j.scale) || !std::isfinite(j.eps) || j.eps < 0.f)
    return set_error(MOE_LRC_EINVAL, "norm_join: scale and eps must be finite, eps not negative");
  if (!j.codes != !j.scales) return set_error(MOE_LRC_EINVAL, "norm_join: codes and scales come together");
  if (j.T == 0) return MOE_LRC_OK;
  if (!j.branch && !j.residual) return set_error(MOE_LRC_EINVAL, "norm_join: neither branch nor residual");
  if (!j.out_residual && !j.out_norm && !j.codes) return set_error(MOE_LRC_EINVAL, "norm_join: no output");
  if ((j.out_norm || j.codes) && !j.pre_weight) return set_error(MOE_LRC_EINVAL, "norm_join: pre_weight is null");
  if ((j.gate_kind != MOE_LRC_GATE_NONE) != (j.gate != nullptr)) return set_error(MOE_LRC_EINVAL, "norm_join: gate and gate_kind do not agree");
  if (!j.branch && (j.post_weight || j.gate)) return set_error(MOE_LRC_EINVAL, "norm_join: post_weight and gate need a branch");
  for (const void* p : {j.branch, j.residual, (const void*)j.post_weight, (const void*)j.pre_weight, (const void*)j.out_residual, (const void*)j.out_norm})
    if (misaligned(p, 16)) return set_error(MOE_LRC_EINVAL, "norm_join: arrays must be 16-byte aligned");
  if (misaligned(j.gate, j.gate_kind == MOE_LRC_GATE_TOKEN ? 4 : 16) || misaligned(j.codes, 8) || misaligned(j.scales, 4))
    return set_error(MOE_LRC_EINVAL, "norm_join: gate must be 16-byte aligned (per token: 4), codes 8, scales 4");
  auto bad = [&](const void* p, int64_t stride) { return p && (stride < j.H || stride % 8); };
  if (bad(j.branch, j.branch_stride) || bad(j.residual, j.residual_stride) || bad(j.out_residual, j.out_residual_stride) ||
      bad(j.out_norm, j.out_norm_stride) || (j.gate_kind == MOE_LRC_GATE_ELEMENT && bad(j.gate, j.gate_stride)) ||
      (j.gate_kind == MOE_LRC_GATE_TOKEN && j.gate_stride < 1))
    return set_error(MOE_LRC_EINVAL, "norm_join: row strides must be multiples of 8 and at least H (gate per token: at least 1)");
  if ((j.out_residual && j.out_residual == j.residual && j.out_residual_stride != j.residual_stride) ||
      (j.out_norm && j.out_norm == j.branch && j.out_norm_stride != j.branch_stride))
    return set_error(MOE_LRC_EINVAL, "norm_join: an array updated in place keeps its stride");
  LRC_HIP(j.residual_f32 ? launch_join<true>(j, (hipStream_t)stream) : launch_join<false>(j, (hipStream_t)stream));
  return MOE_LRC_OK;
}

int moe_lrc_block_quantize(const void* x, int64_t x_stride, int T, int K, int swiglu, void* codes, float* scales, void* stream) {
  if (T < 0) return set_error(MOE_LRC_EINVAL, "block_quantize: T is negative");
  if (K < 8 || K % 8) return set_error(MOE_LRC_ESHAPE, "block_quantize: K must be a positive multiple of 8");
  if (swiglu != 0 && swiglu != 1) return set_error(MOE_LRC_EINVAL, "block_quantize: swiglu must be 0 or 1");
  if (T == 0) return MOE_LRC_OK;
  if (!x || !codes || !scales) return set_error(MOE_LRC_EINVAL, "block_quantize: null argument");
  if (misaligned(x, 16) || misaligned(codes, 8) || misaligned(scales, 4))
    return set_error(MOE_LRC_EINVAL, "block_quantize: x must be 16-byte aligned, codes 8, scales 4");
  if (x_stride % 8 || x_stride < int64_t(swiglu + 1) * K)
    return set_error(MOE_LRC_EINVAL, "block_quantize: x_stride must be a multiple of 8 and at least the row's length");
  const int per_row = (K / 8 + 255) / 256;
  if (int64_t(T) * per_row > 0xffffff) return set_error(MOE_LRC_ESHAPE, "block_quantize: more than 2^24 pieces of 2048 columns");
  const dim3 grid(T * per_row), block(256);
  if (swiglu) hipLaunchKernelGGL(quantize_kernel<true>, grid, block, 0, (hipStream_t)stream, (const uint16_t*)x, x_stride, K, per_row, (uint8_t*)codes, scales);
  else hipLaunchKernelGGL(quantize_kernel<false>, grid, block, 0, (hipStream_t)stream, (const uint16_t*)x, x_stride, K, per_row, (uint8_t*)codes, scales);
  LRC_HIP(hipGetLastError());
  return MOE_LRC_OK;
}

}  // extern "C"
