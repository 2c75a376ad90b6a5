// rope.cu -- rotary positions over three axes, and the paged append that
// applies them on the way.
//
// Mathematics: pair i of a token's channels turns by t = pos[axis(i)] *
// inv_freq[i].  One pass over the data: every element is read once and written
// once, so the bound is HBM (4 bytes an element; the angles cost 12 bytes a
// token).  A CTA takes a few tokens: its threads fill a table of (cos t, sin t) of
// those tokens, shared by all heads of Queries and Keys, then turn 16-byte
// vectors, a row of 64 to 256 channels in neighbouring threads.
#include "paged.cuh"

namespace qwm {
namespace {
using namespace ptx;

constexpr int NT = 256;

// (cos, sin) of pos * f, exact to the fp32 rounding of the reduced angle at every
// position.  The angle is taken in turns, as a 64-bit fraction whose whole turns fall
// off the top (after Payne and Hanek, who form only the bits of a product that a
// reduction keeps): f = m 2^e with a 24-bit m, f / (2 pi) = m 2^e C with C = 1 / (2 pi) to 128
// bits, cut below 2^-64 of a turn, times the position (2^-33 of a turn at 2^31).  What
// is left beside the nearest quarter turn is at most pi / 4 in fp32, where the fast sine
// and cosine are good to 2^-21: far below the output's 2^-9 or 2^-12.  An f of 2^24 or
// more, an infinity or a NaN gives NaN.
__device__ __forceinline__ float2 turn(int pos, float f, float sign) {
  constexpr uint64_t kC1 = 0x28BE60DB9391054Aull, kC0 = 0x7F09D5F47D4D3770ull;   // floor(2^128 / (2 pi))
  constexpr float kTurn = (float)(6.283185307179586476925286766559 / 18446744073709551616.0);
  const uint32_t w = __float_as_uint(f), ex = (w >> 23) & 255u;
  const uint64_t m = (w & 0x7FFFFFu) | (ex ? 0x800000u : 0u);
  const int down = 150 - (int)max(ex, 1u);         // -e
  const uint64_t c0 = __umul64hi(m, kC0), lo = m * kC1 + c0, hi = __umul64hi(m, kC1) + (lo < c0);
  const uint64_t g = down <= 0 ? lo : (down < 64 ? (lo >> down) | (hi << (64 - down)) : (down < 128 ? hi >> (down - 64) : 0));
  const uint64_t t = (uint64_t)(int64_t)pos * g;
  const uint64_t q = (t + (1ull << 61)) >> 62;      // quarter turns
  float sn, cs;
  __sincosf((float)(int64_t)(t - (q << 62)) * kTurn, &sn, &cs);
  if (ex >= 127 + 24) cs = __uint_as_float(0x7FFFFFFFu);
  const float c = q & 1 ? sn : cs, d = q & 1 ? cs : sn;
  // a quarter turn on is (-sn, cs), and so forth
  const float sc = (q + 1) & 2 ? -c : c, ss = q & 2 ? -d : d;
  return make_float2(sc, (w >> 31) ? -(sign * ss) : sign * ss);
}

constexpr int kMaxTokens = 16;                     // tokens of a CTA

__device__ __forceinline__ int64_t wide(int a, int b) { return (int64_t)a * b; }

// Where a token's first Key goes in the pages (elements), < 0: nowhere.
struct Place {
  int64_t at;
};
__device__ __forceinline__ Place place_of(const RopeArgs& a, int64_t n) {
  int lo = 0, hi = a.B;                            // last b with q_off[b] <= n
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (a.q_off[m] <= n) lo = m; else hi = m;
  }
  const int64_t q0 = a.q_off[lo], q1 = a.q_off[lo + 1], kv = a.kv_len[lo];
  int64_t cap = (int64_t)a.table_stride << a.page_log2;
  if (cap > a.max_kv) cap = a.max_kv;
  Place r{-1};
  if (!(n >= q0 && n < q1 && q1 <= a.N && q1 - q0 <= a.max_q && kv >= 0 && kv <= cap)) {
    record_status(a.status, QWM_ERR_INVALID_ARG);
    return r;
  }
  const int64_t p = kv - q1 + n;
  if (p < 0) return r;
  const int64_t page = a.table[(int64_t)lo * a.table_stride + (p >> a.page_log2)];
  if (page < 0 || page >= a.num_pages) {
    record_status(a.status, QWM_ERR_INVALID_ARG);
    return r;
  }
  r.at = (((page * 2 * a.kv_heads) << a.page_log2) + (p & ((1 << a.page_log2) - 1))) * a.D;
  return r;
}

// 32 registers for neighbouring channels, so that 8 CTAs fit an SM (34 and 36: rotation of
// 4680 x 80 heads 36.8 us, append of 4680 x 120 56.2; with 32 33.2 and 50.5).
template <typename T, bool INTERLEAVED, bool PAGED>
__global__ void __launch_bounds__(NT, INTERLEAVED ? 8 : 6) rope_kernel(const RopeArgs a, int tokens_per_cta) {
  extern __shared__ float4 table4[];               // (cos, sin) [tokens_per_cta][P]
  float2* table = reinterpret_cast<float2*>(table4);
  __shared__ Place places[kMaxTokens];
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
  if (PAGED && tid < nt) places[tid] = place_of(a, n0 + tid);
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
      const Place pl = places[rt];
      if (pl.at < 0) continue;
      dst = static_cast<T*>(a.pages) + pl.at + wide(g.page * a.kv_heads + rh, a.D << a.page_log2);
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
  return launch_ahead(a.pages ? rope_kernel<T, IL, true> : rope_kernel<T, IL, false>, dim3(grid), NT, smem, s, a, (int)tpc);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, int dtype, bool interleaved, cudaStream_t s) {
  if (dtype == QWM_F16) return interleaved ? go<__half, true>(a, s) : go<__half, false>(a, s);
  return interleaved ? go<__nv_bfloat16, true>(a, s) : go<__nv_bfloat16, false>(a, s);
}

}  // namespace qwm
