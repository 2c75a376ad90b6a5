// paged_codes.cu -- Keys and Values quantised into 8-bit pages as they are
// written (rotated on the way), and tokens of the pages read back.
//
// Mathematics: a row (token, head) x becomes e4m3 codes c = round(x / 2^e) and
// the scale 2^e with the least e >= -15 for which max |x| <= 448 x 2^e; it stands
// for c x 2^e.  The rounding is the only one: the rotation's fp32 results go into
// it.  A power of two loses nothing against a scale of any value (a code's
// relative step does not depend on its size) and makes the product exact.
#include "rope.cuh"

namespace qwm {
namespace {
using namespace ptx;

constexpr int NT = 256;
constexpr int kMaxTokens = 16;                     // tokens of a CTA

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// sign(a) x min(|a|, b) for b > 0; NaN stays NaN
__device__ __forceinline__ float clamp_nan(float a, float b) {
  float r;
  asm("min.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// One pass, as in rope.cu: the bound is HBM (a Key or Value 2 bytes in and 1 out, a
// Query 2 and 2).  D / 16 neighbouring lanes have a row, two 16-byte vectors each: the
// two of a rotated pair of vectors (halves), or neighbours; the row's maximum is
// three (two) shuffles.
template <typename T, bool INTERLEAVED, int D>
__global__ void __launch_bounds__(NT) store_kernel(const RopeArgs a, int tokens_per_cta) {
  extern __shared__ float4 table4[];               // (cos, sin) [tokens_per_cta][P]
  float2* table = reinterpret_cast<float2*>(table4);
  __shared__ int64_t places[kMaxTokens];
  constexpr int LPR = D / 16, hpar = NT / LPR;     // lanes of a row, rows side by side
  const int tid = threadIdx.x;
  const int n0 = blockIdx.x * tokens_per_cta;      // (N <= 2^30)
  const int nt = (int)min((int64_t)tokens_per_cta, a.N - n0);
  const int P = a.P, u = tid % LPR, hl = tid / LPR;
  grid_begin();
  const bool two = !INTERLEAVED && u < P / 8;      // the vectors of 8 pairs
  const int c0 = INTERLEAVED ? 16 * u : (two ? 8 * u : 2 * P + 16 * (u - P / 8));
  const int c1 = two ? c0 + P : c0 + 8;
  const bool on = a.inv_freq != nullptr;
  const bool turn0 = on && (INTERLEAVED ? c0 < 2 * P : two), turn1 = on && INTERLEAVED && c1 < 2 * P;
  const int H = a.total_heads;
  const int step_t = hpar / H, step_h = hpar % H;
  int t = hl / H, h = hl % H;
  uint4 x, y;
  int rt, rh, rs;                                  // token (-1: none), head and tensor of the row in flight
  auto fetch = [&]() {
    rt = -1;
    rs = 0;
    x = y = make_uint4(0, 0, 0, 0);
    if (t < nt) {
      int hs = h, s = 0;
      if (a.nseg > 1 && hs >= a.seg[0].heads) { hs -= a.seg[0].heads; s = 1; }
      if (a.nseg > 2 && s == 1 && hs >= a.seg[1].heads) { hs -= a.seg[1].heads; s = 2; }
      const RopeSegment& g = a.seg[s];
      const T* src = static_cast<const T*>(g.src) + wide(n0 + t, g.s_tok) + wide(hs, g.s_head);
      x = __ldcs(reinterpret_cast<const uint4*>(src + c0));
      y = __ldcs(reinterpret_cast<const uint4*>(src + c1));
      rt = t;
      rh = hs;
      rs = s;
      t += step_t;
      h += step_h;
      if (h >= H) { h -= H; ++t; }
    }
  };
  fetch();
  if (tid < nt) places[tid] = place_of(a, n0 + tid);
  if (on) {
    for (int i = tid; i < nt * P; i += NT) {
      const int tt = i / P, j = i - tt * P;
      const int axis = j < a.pairs[0] ? 0 : (j < a.pairs[0] + a.pairs[1] ? 1 : 2);
      table[i] = turn(a.pos[wide(n0 + tt, 3) + axis], a.inv_freq[j], a.sign);
    }
  }
  __syncthreads();
  for (; __any_sync(0xFFFFFFFFu, rt >= 0); fetch()) {
    const RopeSegment& g = a.seg[rs];
    float f[16];                                   // channels c0 .. c0 + 7 and c1 .. c1 + 7
    {
      const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float2 v = Elem<T>::unpack(w[k]);
        f[2 * k] = v.x;
        f[2 * k + 1] = v.y;
      }
    }
    if (rt >= 0 && g.rotate && (turn0 || turn1)) {
      const float2* cs = table + rt * P;
      if (INTERLEAVED) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (k < 4 ? !turn0 : !turn1) continue;
          const float2 c = cs[c0 / 2 + k];
          const float p = f[2 * k], q = f[2 * k + 1];
          f[2 * k] = p * c.x - q * c.y;
          f[2 * k + 1] = p * c.y + q * c.x;
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float2 c = cs[c0 + k];
          const float p = f[k], q = f[8 + k];
          f[k] = p * c.x - q * c.y;
          f[8 + k] = p * c.y + q * c.x;
        }
      }
    }
    if (rt >= 0 && g.page < 0) {
      T* dst = static_cast<T*>(g.dst) + wide(n0 + rt, g.d_tok) + wide(rh, g.d_head);
      *reinterpret_cast<uint4*>(dst + c0) = make_uint4(Elem<T>::pack(f[0], f[1]), Elem<T>::pack(f[2], f[3]),
                                                       Elem<T>::pack(f[4], f[5]), Elem<T>::pack(f[6], f[7]));
      *reinterpret_cast<uint4*>(dst + c1) = make_uint4(Elem<T>::pack(f[8], f[9]), Elem<T>::pack(f[10], f[11]),
                                                       Elem<T>::pack(f[12], f[13]), Elem<T>::pack(f[14], f[15]));
    }
    const int64_t place = rt >= 0 && g.page >= 0 ? places[rt] : -1;
    if (!__any_sync(0xFFFFFFFFu, place >= 0)) continue;
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) most = max_nan(most, fabsf(f[k]));
#pragma unroll
    for (int d = 1; d < LPR; d <<= 1) most = max_nan(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
    if (__any_sync(0xFFFFFFFFu, !(most <= kCodeMost))) {
      // beyond what codes and scales hold: +-kCodeMost, and a NaN stays one
      if (place >= 0 && !(most <= 65504.0f)) record_status(a.status, QWM_ERR_NONFINITE);
      most = 0.0f;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        f[k] = clamp_nan(f[k], kCodeMost);
        most = fmaxf(most, fabsf(f[k]));
      }
#pragma unroll
      for (int d = 1; d < LPR; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
    }
    if (place < 0) continue;
    const uint32_t e = code_exponent(most);
    const float inv = code_inverse(e);
    uint32_t c[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      c[k] = to_codes(f[4 * k] * inv, f[4 * k + 1] * inv, f[4 * k + 2] * inv, f[4 * k + 3] * inv);
    const int64_t row = place + ((int64_t)(g.page * a.kv_heads + rh) << a.page_log2);
    uint8_t* dst = static_cast<uint8_t*>(a.pages) + row * D;
    if (INTERLEAVED) {
      *reinterpret_cast<uint4*>(dst + c0) = make_uint4(c[0], c[1], c[2], c[3]);
    } else {
      *reinterpret_cast<uint2*>(dst + c0) = make_uint2(c[0], c[1]);
      *reinterpret_cast<uint2*>(dst + c1) = make_uint2(c[2], c[3]);
    }
    if (u == 0) a.scales[row] = code_scale(e);
  }
}

template <typename T, bool IL, int D>
cudaError_t go(const RopeArgs& a, cudaStream_t s) {
  // tokens of a CTA: two rows for each thread, as long as the grid still covers
  // the SMs about four times
  constexpr int hpar = NT / (D / 16);
  int64_t tpc = (2 * hpar + a.total_heads - 1) / a.total_heads;
  const int64_t most = a.N / (4 * 152);
  if (tpc > most) tpc = most;
  if (tpc > kMaxTokens) tpc = kMaxTokens;
  if (tpc < 1) tpc = 1;
  const unsigned grid = (unsigned)((a.N + tpc - 1) / tpc);
  return launch_ahead(store_kernel<T, IL, D>, dim3(grid), NT, (size_t)tpc * a.P * sizeof(float2), s, 1, a, (int)tpc);
}
template <typename T>
cudaError_t pick(const RopeArgs& a, bool il, cudaStream_t s) {
  if (a.D == 64) return il ? go<T, true, 64>(a, s) : go<T, false, 64>(a, s);
  return il ? go<T, true, 128>(a, s) : go<T, false, 128>(a, s);
}

// Read-back.  One pass, HBM-bound: of 8-bit pages 1 byte in and 2 out an element.
// 8 channels a lane, so that a warp writes whole lines.
constexpr int kFlight = 4;                         // rows in flight of a thread
template <typename T, bool CODES>
__global__ void __launch_bounds__(NT) read_kernel(const ReadArgs a, int tokens_per_cta) {
  __shared__ int64_t places[kMaxTokens];
  const int tid = threadIdx.x;
  const int n0 = blockIdx.x * tokens_per_cta;
  const int nt = (int)min((int64_t)tokens_per_cta, a.N - n0);
  grid_begin();
  if (tid < nt) places[tid] = place_of(a, n0 + tid);
  __syncthreads();
  const int U = a.D / 8, hpar = NT / U, u = tid % U;
  const int first = a.out[0] ? 0 : 1, H = a.kv_heads, each = H * (a.out[0] && a.out[1] ? 2 : 1);
  for (int r0 = tid / U; r0 < nt * each; r0 += hpar * kFlight) {
    uint4 x[kFlight];
    uint32_t sc[kFlight];
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      const int r = r0 + i * hpar, t = r / each, h = r % each;
      x[i] = make_uint4(0, 0, 0, 0);
      sc[i] = 0;
      if (r >= nt * each || places[t] < 0) continue;
      const int64_t row = places[t] + ((int64_t)(first * H + h) << a.page_log2);
      if (CODES) {
        const uint2 c = __ldcs(reinterpret_cast<const uint2*>(a.pages + row * a.D) + u);
        x[i].x = c.x;
        x[i].y = c.y;
        sc[i] = *reinterpret_cast<const uint16_t*>(a.scales + row);
      } else {
        x[i] = __ldcs(reinterpret_cast<const uint4*>(a.pages + row * a.D * 2) + u);
      }
    }
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      const int r = r0 + i * hpar, t = r / each, h = r % each;
      if (r >= nt * each) continue;
      const bool v = first + (h >= H ? 1 : 0);
      if (CODES) {
        const uint32_t s2 = sc[i] * 0x10001u;
        uint32_t w[4];
        from_codes(x[i].x, w[0], w[1]);
        from_codes(x[i].y, w[2], w[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          w[k] = mul_f16x2(w[k], s2);
          if (Elem<T>::bf16) {
            const float2 f = Elem<__half>::unpack(w[k]);
            w[k] = Elem<T>::pack(f.x, f.y);
          }
        }
        x[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      T* dst = static_cast<T*>(v ? a.out[1] : a.out[0]) + wide(n0 + t, v ? a.o_tok[1] : a.o_tok[0]) +
               wide(h >= H ? h - H : h, v ? a.o_head[1] : a.o_head[0]) + 8 * u;
      *reinterpret_cast<uint4*>(dst) = x[i];
    }
  }
}

template <typename T>
cudaError_t go_read(const ReadArgs& a, cudaStream_t s) {
  const int hpar = NT / (a.D / 8), each = a.kv_heads * (a.out[0] && a.out[1] ? 2 : 1);
  int64_t tpc = (kFlight * hpar + each - 1) / each;
  const int64_t most = a.N / (4 * 152);
  if (tpc > most) tpc = most;
  if (tpc > kMaxTokens) tpc = kMaxTokens;
  if (tpc < 1) tpc = 1;
  const unsigned grid = (unsigned)((a.N + tpc - 1) / tpc);
  return launch_ahead(a.scales ? read_kernel<T, true> : read_kernel<T, false>, dim3(grid), NT, 0, s, 1, a, (int)tpc);
}

}  // namespace

cudaError_t launch_store(const RopeArgs& a, int dtype, bool interleaved, cudaStream_t s) {
  return dtype == QWM_F16 ? pick<__half>(a, interleaved, s) : pick<__nv_bfloat16>(a, interleaved, s);
}

cudaError_t launch_read(const ReadArgs& a, int dtype, cudaStream_t s) {
  return dtype == QWM_F16 ? go_read<__half>(a, s) : go_read<__nv_bfloat16>(a, s);
}

}  // namespace qwm
