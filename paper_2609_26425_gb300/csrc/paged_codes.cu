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
__device__ __forceinline__ float max_abs_nan(float a, float b, float c) {   // of the magnitudes
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// sign(a) x min(|a|, b) for b > 0; NaN stays NaN
__device__ __forceinline__ float clamp_nan(float a, float b) {
  float r;
  asm("min.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// One pass, as in rope.cu: the bound is HBM (a Key or Value 2 bytes in and 1 out, a
// Query 2 and 2).  D / 16 neighbouring lanes have a row, two 16-byte vectors each, a
// half of the row apart (halves: the two of a rotated pair, and what passes), so that
// they read and write whole lines; the row's maximum is three (two) shuffles.  The table of
// angles lies in the order the lanes read it: [token][two pairs of four][lane].  (With
// neighbouring vectors and the table in the pairs' order, L1 was the bound: 4680 x 120
// heads 54 us against 46.)
template <typename T, bool INTERLEAVED, int D>
__global__ void __launch_bounds__(NT, 6) store_kernel(const RopeArgs a, int tokens_per_cta) {
  constexpr int LPR = D / 16, hpar = NT / LPR;     // lanes of a row, rows side by side
  extern __shared__ float4 table4[];               // (cos, sin, cos, sin) [tokens_per_cta][4][LPR]
  __shared__ int64_t places[kMaxTokens];
  const int tid = threadIdx.x;
  const int n0 = blockIdx.x * tokens_per_cta;      // (N <= 2^30)
  const int nt = (int)min((int64_t)tokens_per_cta, a.N - n0);
  const int P = a.P, u = tid % LPR, hl = tid / LPR;
  grid_begin();
  const bool two = !INTERLEAVED && u < P / 8;      // the vectors of 8 pairs
  const int c0 = INTERLEAVED || two ? 8 * u : P + 8 * u;                       // (2 P + 8 (u - P / 8))
  const int c1 = c0 + (INTERLEAVED ? D / 2 : two ? P : D / 2 - P);
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
      // interleaved, pairs 4 u + 0 .. 3 are vector u's, and those of vector u + LPR follow all of these
      const int of = INTERLEAVED ? (j / 4) % LPR : j / 8, at = INTERLEAVED ? (j / (4 * LPR)) * 4 + j % 4 : j % 8;
      reinterpret_cast<float2*>(table4)[((tt * 4 + at / 2) * LPR + of) * 2 + at % 2] =
          turn<true>(a.pos[wide(n0 + tt, 3) + axis], a.inv_freq[j], a.sign);
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
      const float4* cs = table4 + rt * 4 * LPR + u;
#pragma unroll
      for (int k = 0; k < 4; ++k) {                // two pairs
        if (INTERLEAVED && (k < 2 ? !turn0 : !turn1)) continue;
        const float4 c = cs[k * LPR];
        if (INTERLEAVED) {
          const float p0 = f[4 * k], q0 = f[4 * k + 1], p1 = f[4 * k + 2], q1 = f[4 * k + 3];
          f[4 * k] = p0 * c.x - q0 * c.y;
          f[4 * k + 1] = p0 * c.y + q0 * c.x;
          f[4 * k + 2] = p1 * c.z - q1 * c.w;
          f[4 * k + 3] = p1 * c.w + q1 * c.z;
        } else {
          const float p0 = f[2 * k], q0 = f[8 + 2 * k], p1 = f[2 * k + 1], q1 = f[8 + 2 * k + 1];
          f[2 * k] = p0 * c.x - q0 * c.y;
          f[8 + 2 * k] = p0 * c.y + q0 * c.x;
          f[2 * k + 1] = p1 * c.z - q1 * c.w;
          f[8 + 2 * k + 1] = p1 * c.w + q1 * c.z;
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
    for (int k = 0; k < 16; k += 2) most = max_abs_nan(most, f[k], f[k + 1]);
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
    *reinterpret_cast<uint2*>(dst + c0) = make_uint2(c[0], c[1]);
    *reinterpret_cast<uint2*>(dst + c1) = make_uint2(c[2], c[3]);
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
  return launch_ahead(store_kernel<T, IL, D>, dim3(grid), NT, a.P ? (size_t)tpc * D * 4 : 0, s, 1, a, (int)tpc);
}
template <typename T>
cudaError_t pick(const RopeArgs& a, bool il, cudaStream_t s) {
  if (a.D == 64) return il ? go<T, true, 64>(a, s) : go<T, false, 64>(a, s);
  return il ? go<T, true, 128>(a, s) : go<T, false, 128>(a, s);
}

// Read-back.  One pass, HBM-bound: of 8-bit pages 1 byte in and 2 out an element.  D / 16
// lanes a row, two vectors of 8 channels each, half a row apart, so that a warp writes whole
// lines; a CTA takes kFlight rows (token; Key, Value; head) for each of its threads, all of
// them on their way at once, and looks up the pages of its next rows meanwhile.
constexpr int kFlight = 4, kReadCtas = 4 * 152;
template <typename T, bool CODES, int D>
__global__ void __launch_bounds__(NT, 4) read_kernel(const ReadArgs a) {
  constexpr int LPR = D / 16, hpar = NT / LPR, RPC = hpar * kFlight;   // lanes of a row, rows side by side, rows of a turn
  static_assert(RPC <= NT, "a thread for each token of a turn (one row a token, at the most)");
  __shared__ int64_t places[2][RPC];
  const int tid = threadIdx.x, u = tid % LPR;
  const int first = a.out[0] ? 0 : 1, H = a.kv_heads, each = H * (a.out[0] && a.out[1] ? 2 : 1);
  const int64_t rows = a.N * each;
  grid_begin();
  // a turn's rows r0 .. r0 + RPC - 1 are those of tokens n0 .., from head h0 on
  struct Turn {
    int64_t n0;
    int h0, tokens;
  };
  auto look_up = [&](int64_t r0, int64_t* at) -> Turn {
    Turn w{0, 0, 0};
    if (r0 >= rows) return w;
    w.n0 = r0 / each;
    w.h0 = (int)(r0 - w.n0 * each);
    w.tokens = (int)min((int64_t)((w.h0 + RPC - 1) / each + 1), a.N - w.n0);   // <= RPC
    if (tid < w.tokens) at[tid] = place_of(a, w.n0 + tid);
    return w;
  };
  const int step_t = hpar / each, step_h = hpar % each;
  auto next = [&](int& t, int& h) {
    t += step_t;
    h += step_h;
    if (h >= each) { h -= each; ++t; }
  };
  Turn now = look_up((int64_t)blockIdx.x * RPC, places[0]);
  __syncthreads();
  for (int64_t r0 = (int64_t)blockIdx.x * RPC, k = 0; r0 < rows; r0 += (int64_t)gridDim.x * RPC, ++k) {
    const int64_t* at = places[k & 1];
    uint4 x[kFlight][2];                             // 16-bit pages: as they are; codes: in x and y
    uint32_t sc[kFlight];
    int t = (now.h0 + tid / LPR) / each, h = (now.h0 + tid / LPR) % each;
    int ts = t, hs = h;
#pragma unroll
    for (int i = 0; i < kFlight; ++i, next(t, h)) {
      x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
      sc[i] = 0;
      const int64_t place = t < now.tokens ? at[t] : -1;
      if (place < 0) continue;
      const int64_t row = place + ((int64_t)(first * H + h) << a.page_log2);
      if (CODES) {
        const uint2* src = reinterpret_cast<const uint2*>(a.pages + row * D) + u;
        const uint2 c0 = __ldcs(src), c1 = __ldcs(src + LPR);
        x[i][0].x = c0.x; x[i][0].y = c0.y;
        x[i][1].x = c1.x; x[i][1].y = c1.y;
        sc[i] = *reinterpret_cast<const uint16_t*>(a.scales + row);
      } else {
        const uint4* src = reinterpret_cast<const uint4*>(a.pages + row * D * 2) + u;
        x[i][0] = __ldcs(src);
        x[i][1] = __ldcs(src + LPR);
      }
    }
    const Turn after = look_up(r0 + (int64_t)gridDim.x * RPC, places[~k & 1]);
#pragma unroll
    for (int i = 0; i < kFlight; ++i, next(ts, hs)) {
      if (ts >= now.tokens) continue;
      if (CODES) {
        const uint32_t s2 = sc[i] * 0x10001u;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          uint32_t w[4];
          from_codes(x[i][z].x, w[0], w[1]);
          from_codes(x[i][z].y, w[2], w[3]);
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            // (in fp32 for bf16, which has values that binary16 has not where a caller wrote the scale)
            if (Elem<T>::bf16) {
              const float2 f = Elem<__half>::unpack(w[m]), g = Elem<__half>::unpack(s2);
              w[m] = Elem<T>::pack(f.x * g.x, f.y * g.x);
            } else {
              w[m] = mul_f16x2(w[m], s2);
            }
          }
          x[i][z] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      const bool v = first + (hs >= H ? 1 : 0);
      T* dst = static_cast<T*>(v ? a.out[1] : a.out[0]) + (now.n0 + ts) * (v ? a.o_tok[1] : a.o_tok[0]) +
               wide(hs >= H ? hs - H : hs, v ? a.o_head[1] : a.o_head[0]) + 8 * u;
      *reinterpret_cast<uint4*>(dst) = x[i][0];
      *reinterpret_cast<uint4*>(dst + D / 2) = x[i][1];
    }
    now = after;
    __syncthreads();
  }
}

template <typename T, int D>
cudaError_t go_read(const ReadArgs& a, cudaStream_t s) {
  constexpr int RPC = NT / (D / 16) * kFlight;
  const int64_t rows = a.N * a.kv_heads * (a.out[0] && a.out[1] ? 2 : 1), turns = (rows + RPC - 1) / RPC;
  const unsigned grid = (unsigned)(turns < kReadCtas ? turns : kReadCtas);
  return launch_ahead(a.scales ? read_kernel<T, true, D> : read_kernel<T, false, D>, dim3(grid), NT, 0, s, 1, a);
}

}  // namespace

cudaError_t launch_store(const RopeArgs& a, int dtype, bool interleaved, cudaStream_t s) {
  return dtype == QWM_F16 ? pick<__half>(a, interleaved, s) : pick<__nv_bfloat16>(a, interleaved, s);
}

cudaError_t launch_read(const ReadArgs& a, int dtype, cudaStream_t s) {
  if (dtype == QWM_F16) return a.D == 64 ? go_read<__half, 64>(a, s) : go_read<__half, 128>(a, s);
  return a.D == 64 ? go_read<__nv_bfloat16, 64>(a, s) : go_read<__nv_bfloat16, 128>(a, s);
}

}  // namespace qwm
