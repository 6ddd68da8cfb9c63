// Routing of many tokens by sigmoid scores (moe_lrc_set_routing).  The selection is the exact one and the weights are rounded once, from
// fp64; but the fp64 products of all tokens with all experts, bounded by the issue of products and conversions, are far from the memory's time: 48 us
// for 4096 tokens, 128 experts and H = 2048.  Almost all of them only show that an expert is not selected, and a bound shows that as well:
//   1. logits on the bf16 matrix cores, with an error that is bounded (kGamma): gate_bounds_kernel;
//   2. per token, from the interval that each key lies in: the groups that stay and the experts that can be among the top_k.  Their
//      logits in fp64, and from these the selection, its order and the weights: select_bounds_kernel.
// Whole call, all products in fp64 -> this, us, Top-8 with 4 of 8 groups: T = 4096, E = 128, H = 2048 55 -> 29, H = 512 25 -> 18; T = 16384
// 194 -> 97; E = 64, T = 4096 64 -> 27; E = 256, H = 7168, T = 4096 259 -> 87.  (From how many tokens on: kBoundTokens.)
// Where the bounds say nothing (infinities, NaN, logits beyond 2^20 or of rows so large that delta is 1/8) a token's wavefront takes all
// experts in fp64.
#include <cmath>
#include <type_traits>

#include "internal.h"
#include "route_body.h"
#include "route_bounds.h"

namespace lrc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short ushort2_v __attribute__((ext_vector_type(2)));
typedef int int4_v __attribute__((ext_vector_type(4)));
typedef float float4_v __attribute__((ext_vector_type(4)));

constexpr int kTokens = 32, kExperts = 64, kWaves = 4, kDepth = 2;

// Tile of 64 experts x 32 tokens; a wavefront takes a quarter of the hidden dimension by itself, 64 values of every row at a time, kDepth
// such pieces in its own part of LDS, fetched by direct copies (16-byte unit u of a row lies at place u ^ (row & 7)).  The blocks of
// the first experts also write the tokens' norms and pre-scale exponents.
// Bound: a wavefront's chain of copy, LDS and products, with one on each SIMD: T = 4096, E = 128, H = 2048 8.9 us (the bytes alone 3).  With pieces three deep
// 9.3, by eight wavefronts one deep 9.3.
__device__ inline void gate_bounds(const uint16_t* __restrict__ x, const uint16_t* __restrict__ wg, int T, int H, int E, float* __restrict__ logits,
                                   float* __restrict__ norms, int32_t* __restrict__ tok_exp) {
  constexpr int kRows = kExperts + kTokens, kFetch = kRows / 8, kStage = kRows * 128, kOwn = kDepth * kStage, TE = kExperts / 16, TT = kTokens / 16;
  static_assert(TE * TT * 64 * 16 <= kOwn, "the sums are joined where the pieces lay");
  __shared__ __align__(1024) uint8_t lds[kWaves * kOwn];
  __shared__ float square[kWaves][kTokens];
  __shared__ uint32_t peak[kWaves][kTokens];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = blockIdx.x * kTokens, e0 = blockIdx.y * kExperts, pieces = H / 64;
  const int ve = min(kExperts, E - e0), vt = min(kTokens, T - t0);
  const int each = (pieces + kWaves - 1) / kWaves, lo = wave * each, hi = min(pieces, lo + each);
  const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(wg + size_t(e0) * H), 0, uint32_t(ve) * H * 2, 0x00020000);
  const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(x + size_t(t0) * H), 0, uint32_t(vt) * H * 2, 0x00020000);
  const int own = wave * kOwn;
  auto lds_at = [&](int byte) { return reinterpret_cast<__attribute__((address_space(3))) void*>(reinterpret_cast<uintptr_t>(lds + byte)); };
  uint32_t from[kFetch];                     // (rows past the last one: the last one again, not written out)
#pragma unroll
  for (int q = 0; q < kFetch; ++q) {
    const int r = 8 * q + (lane >> 3);
    from[q] = uint32_t(8 * q < kExperts ? min(r, ve - 1) : min(r - kExperts, vt - 1)) * uint32_t(H) * 2 + ((lane & 7) ^ (lane >> 3)) * 16;
  }
  auto request = [&](int piece, int stage) { // (past the last one: the last one again, not used)
    const int at = min(piece, hi - 1) * 128;
#pragma unroll
    for (int q = 0; q < kFetch; ++q)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(8 * q < kExperts ? wr : xr, lds_at(own + stage * kStage + q * 1024), 16, from[q], at, 0, 0);
  };
  float4_v acc[TE][TT], part[TE][TT];
  float sq[TT];
  ushort2_v top[TT];
#pragma unroll
  for (int j = 0; j < TT; ++j) {
    sq[j] = 0.f;
    top[j] = ushort2_v{0, 0};
#pragma unroll
    for (int i = 0; i < TE; ++i) {
      acc[i][j] = float4_v{0.f, 0.f, 0.f, 0.f};
      part[i][j] = float4_v{0.f, 0.f, 0.f, 0.f};
    }
  }
  const int row = lane & 15, place = own + row * 128 + ((lane >> 4) ^ (row & 7)) * 16;
  if (lo < hi) {                             // (else an empty share)
#pragma unroll
    for (int d = 0; d < kDepth; ++d) request(lo + d, d);
    int stage = 0;
    for (int piece = lo; piece < hi; ++piece) {
      constexpr int kLeft = (kDepth - 1) * kFetch;
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0x0f70 | (kLeft & 15) | (kLeft >> 4 << 14));
      asm volatile("" ::: "memory");
      int4_v w[TE][2], t[TT][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < TE; ++i) w[i][h] = *reinterpret_cast<const int4_v*>(lds + stage * kStage + (place ^ (64 * h)) + i * 2048);
#pragma unroll
        for (int j = 0; j < TT; ++j) t[j][h] = *reinterpret_cast<const int4_v*>(lds + stage * kStage + (place ^ (64 * h)) + kExperts * 128 + j * 2048);
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0xc07f);    // lgkmcnt(0): the operands are in registers, their place takes another piece
      asm volatile("" ::: "memory");
      request(piece + kDepth, stage);
      stage = stage == kDepth - 1 ? 0 : stage + 1;
#pragma unroll
      for (int j = 0; j < TT; ++j)
#pragma unroll
        for (int i = 0; i < TE; ++i) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            part[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[i][h]), __builtin_bit_cast(bf16x8, t[j][h]), part[i][j], 0, 0, 0);
        }
      if ((piece - lo) % (kChain / 2) == kChain / 2 - 1 || piece == hi - 1)
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
          for (int i = 0; i < TE; ++i) {
            acc[i][j] += part[i][j];
            part[i][j] = float4_v{0.f, 0.f, 0.f, 0.f};
          }
      if (e0 == 0) {
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const uint32_t u = uint32_t(t[j][h][q]);
              sq[j] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, u), __builtin_bit_cast(bf16x2, u), sq[j], false);
              top[j] = __builtin_elementwise_max(top[j], __builtin_bit_cast(ushort2_v, u & 0x7fff7fffu));
            }
      }
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);      // (the copies that nothing reads have landed: their places are taken for the sums)
  }
  float4_v* red = reinterpret_cast<float4_v*>(lds + own);
#pragma unroll
  for (int i = 0; i < TE; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) red[(i * TT + j) * 64 + lane] = acc[i][j];
#pragma unroll
  for (int j = 0; j < TT; ++j) {
    sq[j] += __shfl_xor(sq[j], 16);
    sq[j] += __shfl_xor(sq[j], 32);
    uint32_t most = max(top[j].x, top[j].y);
    most = max(most, uint32_t(__shfl_xor(int(most), 16)));
    most = max(most, uint32_t(__shfl_xor(int(most), 32)));
    if (lane < 16) { square[wave][16 * j + lane] = sq[j]; peak[wave][16 * j + lane] = most; }
  }
  __syncthreads();
  for (int v = wave; v < TE * TT; v += kWaves) {
    float4_v sum = reinterpret_cast<const float4_v*>(lds)[v * 64 + lane];
#pragma unroll
    for (int o = 1; o < kWaves; ++o) sum += reinterpret_cast<const float4_v*>(lds + o * kOwn)[v * 64 + lane];
    const int e = e0 + v / TT * 16 + (lane >> 4) * 4, t = t0 + v % TT * 16 + row;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (t < T && e + r < E) logits[size_t(t) * E + e + r] = sum[r];
  }
  if (e0 == 0 && threadIdx.x < kTokens && t0 + int(threadIdx.x) < T) {
    float s = 0.f;
    uint32_t m = 0;
#pragma unroll
    for (int o = 0; o < kWaves; ++o) { s += square[o][threadIdx.x]; m = max(m, peak[o][threadIdx.x]); }
    norms[t0 + threadIdx.x] = norm_above(s);
    const int eb = int(m >> 7);
    if (tok_exp) tok_exp[t0 + threadIdx.x] = eb == 0 ? 0 : min(60, max(-60, 127 - eb));
  }
}
__global__ __launch_bounds__(64 * kWaves) void gate_bounds_kernel(const uint16_t* x, const uint16_t* wg, int T, int H, int E, float* logits, float* norms,
                                                                  int32_t* tok_exp) {
  gate_bounds(x, wg, T, H, E, logits, norms, tok_exp);
}

// The largest 2-norm of a gate row, rounded up: a workgroup a row, joined by the maximum of the bit patterns, in which an infinity or
// a NaN is above every number.
__global__ __launch_bounds__(256) void gate_norm_kernel(const uint16_t* __restrict__ wg, int H, uint32_t* __restrict__ norm) {
  __shared__ double part[4];
  const uint4* row = reinterpret_cast<const uint4*>(wg + size_t(blockIdx.x) * H);
  double sum = 0.0;
  for (int c = threadIdx.x; c < H / 8; c += 256) {
    const uint4 v = row[c];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const double lo = bf16_to_double(w[q] & 0xffffu), hi = bf16_to_double(w[q] >> 16);
      sum = fma(lo, lo, fma(hi, hi, sum));
    }
  }
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    const float n = float(sqrt(part[0] + part[1] + part[2] + part[3])) * 1.001f;
    atomicMax(norm, n == n ? __float_as_uint(n) : 0x7fc00000u);
  }
}

// A float's bits in an unsigned order that is the numbers' (0 lies below all of them), and back.
__device__ inline uint32_t ordered32(float v) {
  const uint32_t u = __float_as_uint(v);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ inline float from_ordered32(uint32_t o) { return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o); }

// One wavefront a token, USED registers that hold an expert in some lane.  T = 4096, E = 128, H = 2048, Top-8, 4 of 8 groups: 21.5 us, of which the
// interval of each key 2, the groups 4, the top_k-th lower end 1.5, the exact logits 12 and the list 1.5.  Bound: one chain of steps up to the list of
// candidates (35% of the wavefronts' time is waiting); then VALU instructions (65% of the whole time), about half of them of the
// fp64 products (three a product: bf16 to fp32, to fp64, the product) of the experts that can be selected, top_k and a few per cent more,
// and the L2s, which their rows are read from: 1.29 M requests of 128 bytes, 165 MB in 10 to 12 us, the 12 to 13 TB/s that the
// 8-bit product's kernels get of them at most.
template <int USED>
__global__ __launch_bounds__(256) void select_bounds_kernel(const uint16_t* __restrict__ x_all, const uint16_t* __restrict__ wg,
                                                            const float* __restrict__ gate_bias, const float* __restrict__ logits,
                                                            const float* __restrict__ norms, const float* __restrict__ gate_norm, int T, int H, int E, int top_k,
                                                            ScoredRule r, int32_t* __restrict__ idx, float* __restrict__ w_out) {
  __shared__ double own[4][256];
  __shared__ int32_t listed[4][256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = blockIdx.x * 4 + wave;
  if (t >= T) return;
  double* lds = own[wave];
  uint2* ends = reinterpret_cast<uint2*>(lds);
  int32_t* list = listed[wave];
  const uint16_t* x = x_all + size_t(t) * H;
  int32_t* idx_t = idx + size_t(t) * top_k;
  float* w_t = w_out + size_t(t) * top_k;
  auto in_order = [] {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  auto exact = [&](int n, auto&& put) {      // put(i, logit of the expert list[i]) for the first n, each in one lane
    auto some = [&](int i0, auto n_) {
      constexpr int N = decltype(n_)::value;
      const double l = exact_logits<N>(x, wg, H, lane, [&](int i) { return __builtin_amdgcn_readfirstlane(list[min(i0 + i, n - 1)]); });
      const int i = i0 + expert_of<N>(lane);
      if ((lane & (N == 8 ? 7 : 15)) == 0 && i < n) put(i, l + (gate_bias ? (double)gate_bias[list[i]] : 0.0));
    };
    for (int i0 = 0; i0 < n; i0 += 8) n - i0 > 4 ? some(i0, std::integral_constant<int, 8>()) : some(i0, std::integral_constant<int, 4>());
  };
  const float inf = __builtin_huge_valf();
  const float delta = kGamma * norms[t] * *gate_norm * 1.001f + 0x1p-100f;
  float a[USED], bias[USED];
  bool fine = delta < 0x1p-3f;               // (else bounds say too little; an infinity, not a number: not so)
#pragma unroll
  for (int m = 0; m < USED; ++m) {
    const int e = lane + 64 * m;
    const bool in = e < E;
    a[m] = in ? logits[size_t(t) * E + e] + (gate_bias ? gate_bias[e] : 0.f) : 0.f;
    bias[m] = in && r.select_bias ? r.select_bias[e] : 0.f;
    fine &= fabsf(a[m]) < 0x1p20f;
  }
  // The intervals of the keys.  A sigmoid's slope is s (1 - s) and changes by exp(delta) at most over delta < 1/8; the gate's bias is added in
  // fp32 here and the exponential taken of a product (2^-24 of |a| each), the score errs by a few of its own 2^-24, the key's sum by one
  // more.  A bias of -infinity bars the expert whatever its score.
  float low[USED], high[USED];
#pragma unroll
  for (int m = 0; m < USED; ++m) {
    const bool in = lane + 64 * m < E && bias[m] != -inf;
    const float score = __builtin_amdgcn_rcpf(1.f + __expf(-a[m]));
    const float err = 1.15f * score * (1.f - score) * (delta + 0x1p-22f * fabsf(a[m])) + 0x1p-20f + 0x1p-22f * fabsf(bias[m]);
    low[m] = in ? score + bias[m] - err : -inf;
    high[m] = in ? score + bias[m] + err : -inf;
  }
  unsigned long long kept = ~0ull;           // the groups that stay
  const int size = E / r.n_groups;
  if (r.top_groups < r.n_groups && __all(fine)) {
    const bool two = r.group_best == 2;
    // lane g: the two highest of group g, of the lower and of the upper ends
#pragma unroll
    for (int m = 0; m < USED; ++m)
      if (lane + 64 * m < E) ends[lane + 64 * m] = make_uint2(ordered32(low[m]), ordered32(high[m]));
    in_order();
    uint32_t lf_o = ordered32(-inf), ls_o = lf_o, hf_o = lf_o, hs_o = lf_o;
    const int begin = min(lane, r.n_groups - 1) * size;
    for (int i0 = 0; i0 < size; i0 += 8) {
      uint2 k[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) k[i] = ends[begin + min(i0 + i, size - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i0 + i >= size) break;
        ls_o = max(ls_o, min(lf_o, k[i].x));
        lf_o = max(lf_o, k[i].x);
        hs_o = max(hs_o, min(hf_o, k[i].y));
        hf_o = max(hf_o, k[i].y);
      }
    }
    in_order();
    const float lf = from_ordered32(lf_o), ls = from_ordered32(ls_o), hf = from_ordered32(hf_o), hs = from_ordered32(hs_o);
    // (the sums of two in fp32: one rounding, taken outwards; not a number where one of the two is barred)
    const float wl = two ? lf + ls - 0x1p-22f * (fabsf(lf) + fabsf(ls)) : lf, wh = two ? hf + hs + 0x1p-22f * (fabsf(hf) + fabsf(hs)) : hf;
    const float lo_g = wl == wl ? wl : -inf, hi_g = wh == wh ? wh : -inf;
    int may = 0, must = 0;                   // groups that may be worth as much or more, that are worth more
    for (int g = 0; g < r.n_groups; ++g) {
      const float ol = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lo_g), g)), oh = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(hi_g), g));
      may += g != lane && oh >= lo_g;
      must += ol > hi_g;
    }
    const bool group = lane < r.n_groups;
    const unsigned long long sure = __ballot(group && may < r.top_groups), open = __ballot(group && may >= r.top_groups && must < r.top_groups);
    const int wanted = r.top_groups - __popcll(sure);
    kept = sure;
    if (__popcll(open) <= wanted) {
      kept |= open;
    } else {                                 // the open groups by their exact worth: from the experts that can be among a group's best
      const float least = two ? ls : lf;     // (lane g: no expert below it is)
      int n = 0;
#pragma unroll
      for (int m = 0; m < USED; ++m) {
        const int e = lane + 64 * m, g = min(e / size, r.n_groups - 1);
        const float bar = __shfl(least, g);
        const bool can = e < E && (open >> g & 1) && high[m] >= bar;
        const unsigned long long who = __ballot(can);
        if (can) list[n + __popcll(who & ((1ull << lane) - 1))] = e;
        n += __popcll(who);
        if (e < E) lds[e] = -__builtin_huge_val();
      }
      in_order();
      exact(n, [&](int i, double l) {
        const int e = list[i];
        lds[e] = 1.0 / (1.0 + exp(-l)) + (r.select_bias ? (double)r.select_bias[e] : 0.0);
      });
      in_order();
      double first = -__builtin_huge_val(), second = first;
      if (open >> lane & 1)
        for (int i = 0; i < size; ++i) {
          const double k = lds[lane * size + i];
          second = fmax(second, fmin(first, k));
          first = fmax(first, k);
        }
      in_order();
      const double worth = two ? first + second : first;
      int ahead = 0;
      for (unsigned long long gs = open; gs; gs &= gs - 1) {
        const int g = __ffsll(gs) - 1;
        const double other = lane_double(worth, g);
        ahead += other > worth || (other == worth && g < lane);
      }
      kept |= __ballot((open >> lane & 1) && ahead < wanted);
    }
  }
  // The experts that can be selected: those whose key may reach the top_k-th highest lower end.  listed in the order of their indexes.
  uint32_t head[USED];                        // (0: of a group that does not stay)
#pragma unroll
  for (int m = 0; m < USED; ++m) {
    const int e = lane + 64 * m;
    head[m] = e < E && (kept >> (e / size) & 1) ? ordered32(low[m]) : 0u;
  }
  uint32_t bar = 0;
  {
    uint32_t left[USED];
#pragma unroll
    for (int m = 0; m < USED; ++m) left[m] = head[m];
    for (int found = 0; found < top_k;) {    // (a pass takes all that hold the highest: top_k passes at most)
      uint32_t most = left[0];
#pragma unroll
      for (int m = 1; m < USED; ++m) most = max(most, left[m]);
      bar = wave_max_u32(most);
      if (bar == 0) break;
#pragma unroll
      for (int m = 0; m < USED; ++m) {
        found += __popcll(__ballot(left[m] == bar));
        if (left[m] == bar) left[m] = 0;
      }
    }
  }
  int n = 0;
#pragma unroll
  for (int m = 0; m < USED; ++m) {
    const bool can = head[m] != 0 && ordered32(high[m]) >= bar;
    const unsigned long long who = __ballot(can);
    if (can) list[n + __popcll(who & ((1ull << lane) - 1))] = lane + 64 * m;
    n += __popcll(who);
  }
  const bool whole = !__all(fine) || n > 64; // no bounds, or more than one a lane: every expert exactly
  if (whole) {
    in_order();
    n = E;
#pragma unroll
    for (int m = 0; m < USED; ++m)
      if (lane + 64 * m < E) list[lane + 64 * m] = lane + 64 * m;
  }
  in_order();
  exact(n, [&](int i, double l) { lds[i] = l; });
  in_order();
  if (whole) {
    double v[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int m = 0; m < USED; ++m) v[m] = lane + 64 * m < E ? lds[lane + 64 * m] : 0.0;
    in_order();
    float all_bias[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int m = 0; m < USED; ++m) all_bias[m] = bias[m];
    select_scored(v, all_bias, lane, E, top_k, r, lds, idx_t, w_t);
    return;
  }
  // lane j: the j-th of them; its rank among the keys, its place among the selected by score (ties: the lower index first)
  const bool here = lane < n;
  const int my_e = here ? list[lane] : 0;
  const double my_s = here ? 1.0 / (1.0 + exp(-lds[lane])) : 0.0;
  const double my_k = here ? my_s + (r.select_bias ? (double)r.select_bias[my_e] : 0.0) : -__builtin_huge_val();
  int rank = 0;
  for (int i = 0; i < n && n > top_k; ++i) {
    const double other = lane_double(my_k, i);
    rank += other > my_k || (other == my_k && i < lane);
  }
  const unsigned long long chosen = __ballot(here && rank < top_k);
  int place = 0;
  double sum = 0.0;
  for (unsigned long long cs = chosen; cs; cs &= cs - 1) {
    const int i = __ffsll(cs) - 1;
    const double other = lane_double(my_s, i);
    place += other > my_s || (other == my_s && i < lane);
    sum += other;
  }
  if (chosen >> lane & 1) {
    idx_t[place] = my_e;
    w_t[place] = (float)((r.renormalize && sum != 0.0 ? my_s / sum : my_s) * (double)r.scale);
  }
}

}  // namespace

hipError_t launch_gate_norm(const moe_lrc_layer* L, hipStream_t s) {
  const hipError_t e = hipMemsetAsync(L->d_gate_norm, 0, 4, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(gate_norm_kernel, dim3(L->cfg.n_experts), dim3(256), 0, s, L->d_wg, L->cfg.hidden, reinterpret_cast<uint32_t*>(L->d_gate_norm));
  return hipGetLastError();
}

hipError_t launch_route_scored_many(const moe_lrc_layer* L, const void* x, int T, int32_t* idx, float* w, int32_t* tok_exp, hipStream_t s) {
  const moe_lrc_config& c = L->cfg;
  float* logits = reinterpret_cast<float*>(L->d_logits);       // [T][E], and the norms [T] behind them: less than the T * E doubles that are there
  float* norms = logits + size_t(T) * c.n_experts;
  hipLaunchKernelGGL(gate_bounds_kernel, dim3((T + kTokens - 1) / kTokens, (c.n_experts + kExperts - 1) / kExperts), dim3(64 * kWaves), 0, s,
                     (const uint16_t*)x, L->d_wg, T, c.hidden, c.n_experts, logits, norms, tok_exp);
  const auto select = c.n_experts <= 64 ? select_bounds_kernel<1> : c.n_experts <= 128 ? select_bounds_kernel<2> : select_bounds_kernel<4>;
  hipLaunchKernelGGL(select, dim3((T + 3) / 4), dim3(256), 0, s, (const uint16_t*)x, L->d_wg, L->has_bias ? L->d_bias : nullptr, logits, norms,
                     L->d_gate_norm, T, c.hidden, c.n_experts, c.top_k, L->rule, idx, w);
  return hipGetLastError();
}

}  // namespace lrc
