// rope.cu -- rotary positions over three axes, and the paged append that
// applies them on the way.
//
// Mathematics: pair i of a token's channels turns by t = pos[axis(i)] *
// inv_freq[i].  One pass over the data: every element is read once and written
// once, so the bound is HBM (4 bytes an element; the angles cost 12 bytes a
// token).  A CTA takes a few tokens: its threads fill a table of (cos t, sin t) of
// those tokens, shared by all heads of Queries and Keys, then turn 16-byte
// vectors, a row of 64 to 256 channels in neighbouring threads.
#include "rope.cuh"

namespace qwm {
namespace {
using namespace ptx;

constexpr int NT = 256;

constexpr int kMaxTokens = 16;                     // tokens of a CTA

// 32 registers for neighbouring channels, so that 8 CTAs fit an SM (34 and 36: rotation of
// 4680 x 80 heads 36.8 us, append of 4680 x 120 56.2; with 32 33.2 and 50.5).
template <typename T, bool INTERLEAVED, bool PAGED>
__global__ void __launch_bounds__(NT, INTERLEAVED ? 8 : 6) rope_kernel(const RopeArgs a, int tokens_per_cta) {
  extern __shared__ float4 table4[];               // (cos, sin) [tokens_per_cta][P]
  float2* table = reinterpret_cast<float2*>(table4);
  __shared__ int64_t places[kMaxTokens];
  const int tid = threadIdx.x;
  const int n0 = blockIdx.x * tokens_per_cta;      // (N <= 2^30)
  const int nt = (int)min((int64_t)tokens_per_cta, a.N - n0);
  const int P = a.P, nvec = a.D / 8;
  // units of a head's row: interleaved, its nvec vectors; halves, P / 8 pairs
  // of vectors (u, u + P / 8) and the vectors that pass
  const int pv = INTERLEAVED ? P / 4 : P / 8;      // rotated units
  const int U = INTERLEAVED ? nvec : nvec - pv;
  const int hpar = NT / U;                         // rows (token, head) side by side
  const int u = tid % U, hl = tid / U;
  grid_begin();
  const bool active = hl < hpar;
  const bool turned = a.inv_freq != nullptr && u < pv;
  const bool two = !INTERLEAVED && u < pv;         // two vectors a unit
  const int c0 = 8 * (INTERLEAVED || two ? u : u + pv);
  const int c1 = c0 + P;
  // This thread's rows are hl, hl + hpar, ... of the CTA's tokens x heads, one in
  // flight (the first on its way while the table is made): 1300 to 2000 threads
  // an SM keep 32 to 64 KB in flight, and more rows per thread were slower (two:
  // append of 4680 x 120 heads 51 -> 56 us, four: 63; the writes of a page's
  // heads then come further apart).
  const int H = a.total_heads;
  const int step_t = hpar / H, step_h = hpar % H;
  int t = active ? hl / H : nt, h = hl % H;
  uint4 x, y;
  int rt, rh, rs;                                  // token (-1: none), head and tensor of the row in flight
  auto fetch = [&]() {
    rt = -1;
    if (t < nt) {
      int hs = h, s = 0;
      if (a.nseg > 1 && hs >= a.seg[0].heads) { hs -= a.seg[0].heads; s = 1; }
      if (a.nseg > 2 && s == 1 && hs >= a.seg[1].heads) { hs -= a.seg[1].heads; s = 2; }
      const RopeSegment& g = a.seg[s];
      const T* src = static_cast<const T*>(g.src) + wide(n0 + t, g.s_tok) + wide(hs, g.s_head);
      x = __ldcs(reinterpret_cast<const uint4*>(src + c0));
      if (two) y = __ldcs(reinterpret_cast<const uint4*>(src + c1));
      rt = t;
      rh = hs;
      rs = s;
      t += step_t;
      h += step_h;
      if (h >= H) { h -= H; ++t; }
    }
  };
  fetch();
  if (PAGED && tid < nt) places[tid] = place_of(a, n0 + tid) * a.D;   // elements
  if (a.inv_freq) {
    for (int i = tid; i < nt * P; i += NT) {
      const int tt = i / P, j = i - tt * P;
      const int axis = j < a.pairs[0] ? 0 : (j < a.pairs[0] + a.pairs[1] ? 1 : 2);
      table[i] = turn(a.pos[wide(n0 + tt, 3) + axis], a.inv_freq[j], a.sign);
    }
  }
  __syncthreads();
  for (; rt >= 0; fetch()) {
    const RopeSegment& g = a.seg[rs];
    T* dst;
    if (!PAGED || g.page < 0) {
      dst = static_cast<T*>(g.dst) + wide(n0 + rt, g.d_tok) + wide(rh, g.d_head);
    } else {
      const int64_t at = places[rt];
      if (at < 0) continue;
      dst = static_cast<T*>(a.pages) + at + wide(g.page * a.kv_heads + rh, a.D << a.page_log2);
    }
    if (turned && g.rotate) {
      uint32_t* xw = reinterpret_cast<uint32_t*>(&x);
      uint32_t* yw = reinterpret_cast<uint32_t*>(&y);
      const float4* cs = reinterpret_cast<const float4*>(table + rt * P) + u * (INTERLEAVED ? 2 : 4);
      if (INTERLEAVED) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const float4 c = cs[w];
          const float2 v = Elem<T>::unpack(xw[2 * w]), z = Elem<T>::unpack(xw[2 * w + 1]);
          xw[2 * w] = Elem<T>::pack(v.x * c.x - v.y * c.y, v.x * c.y + v.y * c.x);
          xw[2 * w + 1] = Elem<T>::pack(z.x * c.z - z.y * c.w, z.x * c.w + z.y * c.z);
        }
      } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float4 c = cs[w];
          const float2 v = Elem<T>::unpack(xw[w]), z = Elem<T>::unpack(yw[w]);
          xw[w] = Elem<T>::pack(v.x * c.x - z.x * c.y, v.y * c.z - z.y * c.w);
          yw[w] = Elem<T>::pack(v.x * c.y + z.x * c.x, v.y * c.w + z.y * c.z);
        }
      }
    }
    *reinterpret_cast<uint4*>(dst + c0) = x;
    if (two) *reinterpret_cast<uint4*>(dst + c1) = y;
  }
}

template <typename T, bool IL>
cudaError_t go(const RopeArgs& a, cudaStream_t s) {
  // tokens of a CTA: two rows for each thread, as long as the grid still covers
  // the SMs about four times
  const int U = IL ? a.D / 8 : a.D / 8 - a.P / 8;
  const int hpar = NT / U;
  int64_t tpc = (2 * hpar + a.total_heads - 1) / a.total_heads;
  const int64_t most = a.N / (4 * 152);
  if (tpc > most) tpc = most;
  if (tpc > kMaxTokens) tpc = kMaxTokens;
  if (tpc < 1) tpc = 1;
  const unsigned grid = (unsigned)((a.N + tpc - 1) / tpc);
  const size_t smem = (size_t)tpc * a.P * sizeof(float2);
  return launch_ahead(a.pages ? rope_kernel<T, IL, true> : rope_kernel<T, IL, false>, dim3(grid), NT, smem, s, 1, a, (int)tpc);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, int dtype, bool interleaved, cudaStream_t s) {
  if (dtype == QWM_F16) return interleaved ? go<__half, true>(a, s) : go<__half, false>(a, s);
  return interleaved ? go<__nv_bfloat16, true>(a, s) : go<__nv_bfloat16, false>(a, s);
}

}  // namespace qwm
