// rope.cu -- rotary positions over three axes, and the paged append that
// applies them on the way.
//
// Mathematics: pair i of a token's channels turns by t = pos[axis(i)] *
// inv_freq[i].  One pass over the data: every element is read once and written
// once, so the bound is HBM (4 bytes an element; the angles cost 12 bytes a
// token).  A CTA takes a few tokens: its threads first fill a table of (cos t,
// sin t) of those tokens, shared by all heads of Queries and Keys, then move
// 16-byte vectors, several in flight per thread.
#include "paged.cuh"

namespace qwm {
namespace {
using namespace ptx;

constexpr int NT = 256;
constexpr int kMaxPairs = 128;

// (cos, sin) of pos * f.  The product is carried as hi + lo (exact for |pos| <
// 2^24; the rest of a larger position adds its own product), then reduced by
// whole turns with 2 pi in three fp32 parts (Cody and Waite's method), twice so
// that a quotient above 2^23 leaves nothing behind.  The reduced angle is
// within an fp32 rounding of the exact one, where the fast sine and cosine are
// good to 2^-21 absolute: far below the output's 2^-9 or 2^-12.
__device__ __forceinline__ float2 turn(int pos, float f, float sign) {
  constexpr float kInv = 0.15915494309189535f;  // 1 / (2 pi)
  // 2 pi = c1 + c2 + c3, each the fp32 rounding of what the ones before leave
  constexpr double kTwoPi = 6.283185307179586476925286766559;
  constexpr float c1 = (float)kTwoPi;
  constexpr float c2 = (float)(kTwoPi - (double)c1);
  constexpr float c3 = (float)(kTwoPi - (double)c1 - (double)c2);
  const float p = (float)pos;
  const float rest = (float)(pos - (int64_t)p);
  const float hi = p * f;
  float lo = fmaf(p, f, -hi);
  lo = fmaf(rest, f, lo);
  float r = hi;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float n = rintf(r * kInv);
    r = fmaf(-n, c1, r);
    lo = fmaf(-n, c2, lo);
    lo = fmaf(-n, c3, lo);
    const float s = r + lo;   // renormalise: r + lo is unchanged
    lo = lo - (s - r);
    r = s;
  }
  float sn, cs;
  __sincosf(r + lo, &sn, &cs);
  return make_float2(cs, sign * sn);
}

// Up to kLoads 16-byte vectors are in flight per thread.
constexpr int kLoads = 4;

template <typename T, bool INTERLEAVED, bool PAGED>
__global__ void __launch_bounds__(NT) rope_kernel(const RopeArgs a, int tokens_per_cta) {
  extern __shared__ float2 table[];  // [tokens_per_cta][P]
  const int tid = threadIdx.x;
  const int64_t n0 = (int64_t)blockIdx.x * tokens_per_cta;
  const int nt = (int)min((int64_t)tokens_per_cta, a.N - n0);
  const int P = a.P, nvec = a.D / 8;
  // units of a head's row: interleaved, its nvec vectors; halves, P / 8 pairs
  // of vectors (u, u + P / 8) and the vectors that pass
  const int pv = INTERLEAVED ? P / 4 : P / 8;      // rotated units
  const int U = INTERLEAVED ? nvec : nvec - pv;
  const int hpar = NT / U;                         // heads side by side
  const int u = tid % U, hl = tid / U;
  if (a.inv_freq) {
    for (int i = tid; i < nt * P; i += NT) {
      const int t = i / P, j = i - t * P;
      const int axis = j < a.pairs[0] ? 0 : (j < a.pairs[0] + a.pairs[1] ? 1 : 2);
      table[i] = turn(a.pos[(n0 + t) * 3 + axis], a.inv_freq[j], a.sign);
    }
    __syncthreads();
  }
  if (hl >= hpar) return;
  const bool turned = a.inv_freq != nullptr && u < pv;
  const bool two = !INTERLEAVED && u < pv;         // two vectors a unit
  const int c0 = 8 * (INTERLEAVED || two ? u : u + pv);
  const int c1 = c0 + P;
  for (int t = 0; t < nt; ++t) {
    const int64_t n = n0 + t;
    // the page and slot of the token
    int64_t block0 = -1;
    int slot = 0;
    if (PAGED) {
      int lo = 0, hi = a.B;                        // last b with q_off[b] <= n
      while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (a.q_off[m] <= n) lo = m; else hi = m;
      }
      const int64_t q0 = a.q_off[lo], q1 = a.q_off[lo + 1], kv = a.kv_len[lo];
      int64_t cap = (int64_t)a.table_stride << a.page_log2;
      if (cap > a.max_kv) cap = a.max_kv;
      const bool ok = n >= q0 && n < q1 && q1 <= a.N && q1 - q0 <= a.max_q && kv >= 0 && kv <= cap;
      if (!ok) {
        if (tid == 0) record_status(a.status, QWM_ERR_INVALID_ARG);
      } else {
        const int64_t p = kv - q1 + n;
        if (p >= 0) {
          const int64_t page = a.table[(int64_t)lo * a.table_stride + (p >> a.page_log2)];
          if (page >= 0 && page < a.num_pages) {
            block0 = page * 2 * a.kv_heads;
            slot = (int)(p & ((1 << a.page_log2) - 1));
          } else if (tid == 0) {
            record_status(a.status, QWM_ERR_INVALID_ARG);
          }
        }
      }
    }
    float2 cs[8];
    if (turned) {
      constexpr int K = INTERLEAVED ? 4 : 8;
#pragma unroll
      for (int k = 0; k < K; ++k) cs[k] = table[t * P + u * K + k];
    }
    for (int h0 = hl; h0 < a.total_heads; h0 += kLoads * hpar) {
      uint4 x[kLoads], y[kLoads];
      T* dst[kLoads];
      bool rot[kLoads];
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        int h = h0 + k * hpar;
        dst[k] = nullptr;
        rot[k] = false;
        if (h < a.total_heads) {
          int s = 0;
          if (a.nseg > 1 && h >= a.seg[0].heads) { h -= a.seg[0].heads; s = 1; }
          if (a.nseg > 2 && s == 1 && h >= a.seg[1].heads) { h -= a.seg[1].heads; s = 2; }
          const RopeSegment& g = a.seg[s];
          const T* src = static_cast<const T*>(g.src) + n * g.s_tok + h * g.s_head;
          if (!PAGED || g.page < 0) dst[k] = static_cast<T*>(g.dst) + n * g.d_tok + h * g.d_head;
          else if (block0 >= 0)
            dst[k] = static_cast<T*>(a.pages) +
                     (((block0 + (int64_t)g.page * a.kv_heads + h) << a.page_log2) + slot) * a.D;
          rot[k] = g.rotate != 0;
          if (dst[k]) {
            x[k] = *reinterpret_cast<const uint4*>(src + c0);
            if (two) y[k] = *reinterpret_cast<const uint4*>(src + c1);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        if (!dst[k]) continue;
        if (turned && rot[k]) {
          uint32_t* xw = reinterpret_cast<uint32_t*>(&x[k]);
          uint32_t* yw = reinterpret_cast<uint32_t*>(&y[k]);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            if (INTERLEAVED) {
              const float2 v = Elem<T>::unpack(xw[w]);
              xw[w] = Elem<T>::pack(v.x * cs[w].x - v.y * cs[w].y, v.x * cs[w].y + v.y * cs[w].x);
            } else {
              const float2 v = Elem<T>::unpack(xw[w]), z = Elem<T>::unpack(yw[w]);
              const float2 ca = cs[2 * w], cb = cs[2 * w + 1];
              xw[w] = Elem<T>::pack(v.x * ca.x - z.x * ca.y, v.y * cb.x - z.y * cb.y);
              yw[w] = Elem<T>::pack(v.x * ca.y + z.x * ca.x, v.y * cb.y + z.y * cb.x);
            }
          }
        }
        *reinterpret_cast<uint4*>(dst[k] + c0) = x[k];
        if (two) *reinterpret_cast<uint4*>(dst[k] + c1) = y[k];
      }
    }
  }
}

template <typename T, bool IL>
cudaError_t go(const RopeArgs& a, cudaStream_t s) {
  // one token a CTA until the grid fills the SMs several times over, then four
  const int tpc = a.N >= 4096 ? 4 : 1;
  const unsigned grid = (unsigned)((a.N + tpc - 1) / tpc);
  const size_t smem = (size_t)tpc * a.P * sizeof(float2);
  if (a.pages) rope_kernel<T, IL, true><<<grid, NT, smem, s>>>(a, tpc);
  else rope_kernel<T, IL, false><<<grid, NT, smem, s>>>(a, tpc);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, int dtype, bool interleaved, cudaStream_t s) {
  if (dtype == QWM_F16) return interleaved ? go<__half, true>(a, s) : go<__half, false>(a, s);
  return interleaved ? go<__nv_bfloat16, true>(a, s) : go<__nv_bfloat16, false>(a, s);
}

}  // namespace qwm
