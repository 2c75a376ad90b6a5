// paged_step.cu -- attention of a few rows of a sequence over its pages: single
// new tokens and short drafts (Query tokens x grouped heads <= 32 rows).
//
// Mathematics: softmax over the visible keys with a running maximum m and sum l
// per row (O and l scaled by 2^((m_old - m_new) c) when m grows), so one pass
// over K and V suffices.  The bound is HBM: K and V of the visible tokens are
// read once per cache head for all the grouped Query heads.
//
// A CTA takes one (sequence, cache head, part of the keys): a producer warp
// keeps a ring of 64-key tiles in flight by TMA, four warps take 16 keys each
// and carry their own m, l and O through the part (no barrier between them in
// the loop), then the four are merged through shared memory.  The rows are the
// M = 16 side of mma.sync: a tcgen05 tile would be 128 rows high for the 1 to 32
// used here, and its TMEM round trip is longer than the whole of a short step.
// Parts of one group are joined by the CTA that finishes last, in part order,
// so the result does not depend on which one that is.
#include "paged.cuh"

namespace qwm {
namespace {
using namespace ptx;

constexpr int TK = 64;                   // keys per tile
constexpr int kWarps = 4;                // consumer warps, 16 keys each
constexpr int NT = (kWarps + 1) * 32;
constexpr int kRing = 96 * 1024;         // bytes of tiles in flight; two CTAs per SM

template <int D>
constexpr int stages() { return kRing / (2 * TK * D * 2); }

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// Byte of 16-byte chunk `chunk` (8 channels) of key `key` in a tile [D / 64][64
// keys][128 bytes], 128-byte swizzled.
__device__ __forceinline__ uint32_t at(int key, int chunk) {
  return (uint32_t)((chunk >> 3) * (TK * 128) + key * 128 + (((chunk & 7) ^ (key & 7)) << 4));
}

template <typename T, int D, int MT>
__global__ void __launch_bounds__(NT) paged_step(const __grid_constant__ CUtensorMap map, const PagedArgs a) {
  constexpr int ST = stages<D>();
  constexpr int KS = D / 16;                       // k16 steps of Q K^T, n16 blocks of P V
  constexpr int ROWS = 16 * MT;
  constexpr uint32_t HALF = TK * D * 2;            // bytes of a K or V tile
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  __shared__ uint64_t bars[2 * ST];
  __shared__ float s_ml[kWarps][ROWS][2];
  __shared__ int s_err, s_last;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int part = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
  Seq sq;
  if (!load_seq(a, b, sq) && part == 0 && hk == 0 && tid == 0) record_status(a.status, QWM_ERR_INVALID_ARG);
  if (sq.qn == 0) return;
  const int rows = sq.qn * a.G;                    // <= ROWS
  const int p0 = sq.kv - sq.qn;
  const Tiles tl = make_tiles<TK>(p0, sq.kv - 1, sq.kv, a.block, a.window, a.sinks);
  // this part's tiles: parts of equal length, as many as the length wants
  const int per = max((tl.n + a.nsplit - 1) / a.nsplit, a.min_tiles);
  const int parts = max(1, (tl.n + per - 1) / per);
  if (part >= parts) return;
  const int t0 = part * per, t1 = min(tl.n, t0 + per);

  auto full = [&](int s) { return smem_u32(&bars[s]); };
  auto empty = [&](int s) { return smem_u32(&bars[ST + s]); };
  if (tid == 0) {
    for (int s = 0; s < ST; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), kWarps);
    }
    s_err = 0;
    fence_mbar_init();
  }
  __syncthreads();

  float o[MT][2 * KS][4];
  float m_run[MT][2], l_run[MT][2];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m_run[mt][0] = m_run[mt][1] = -INFINITY;
    l_run[mt][0] = l_run[mt][1] = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[mt][i][k] = 0.0f;
  }
  const float sl2 = a.scale * 1.4426950408889634f;

  if (warp == kWarps) {
    // ---------------------------------------------------------- producer
    // lane = box * 4 + (Keys, Values) * 2 + channel half; a box is the part of
    // a page that lies in the tile.  Boxes that no row sees are not read.
    const int box_log2 = min(a.page_log2, 6);
    const int boxes = TK >> box_log2;
    const int box = lane >> 2, kv = (lane >> 1) & 1, half = lane & 1;
    const bool mine = box < boxes && half * 64 < D;
    const int32_t* trow = a.table + (int64_t)b * a.table_stride;
    auto page_of = [&](int t, bool& want) -> int {
      const int j0 = tile_at(tl, t) * TK + (box << box_log2);
      want = mine && any_sees(tl, j0, j0 + (1 << box_log2), a.sinks);
      return want ? trow[j0 >> a.page_log2] : 0;
    };
    bool want = false;
    int page = t0 < t1 ? page_of(t0, want) : 0;
    bool ok = true;
    int t = t0;
    for (; t < t1 && !a.idle; ++t) {
      const int i = t - t0, s = i % ST;
      if (i >= ST && !(ok = __all_sync(0xFFFFFFFFu, mbar_wait(empty(s), ((i / ST) - 1) & 1, a.wait_ns)))) break;
      bool want_n = false;
      int page_n = 0;
      if (t + 1 < t1) page_n = page_of(t + 1, want_n);   // its latency runs beside the copies
      if (want && (page < 0 || page >= a.num_pages)) {   // not followed: the first page in its place
        record_status(a.status, QWM_ERR_INVALID_ARG);
        page = 0;
      }
      const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, want)) * (128u << box_log2);
      if (lane == 0) mbar_arrive_expect_tx(full(s), bytes);
      __syncwarp();
      if (want) {
        const int j0 = tile_at(tl, t) * TK + (box << box_log2);
        const uint32_t dst = smem_u32(sm) + s * 2 * HALF + kv * HALF + half * (TK * 128) + ((box << box_log2) * 128);
        tma_load_3d(dst, &map, half * 64, j0 & ((1 << a.page_log2) - 1), (page * 2 + kv) * a.Hk + hk, full(s));
      }
      __syncwarp();
      page = page_n;
      want = want_n;
    }
    if (!ok) {
      // a wait ran out: let the copies in flight land before the CTA ends
      if (lane == 0) s_err = 1;
      for (int u = max(t0, t - ST); u < t; ++u) mbar_wait(full((u - t0) % ST), ((u - t0) / ST) & 1, kDrainNs);
    }
  } else {
    // ---------------------------------------------------------- consumers
    const int g = lane >> 2, tq = lane & 3;
    uint32_t qf[MT][KS][4];
    int hi[MT][2], lo[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int rr = 0; rr < 2; ++rr) {
        const int r = mt * 16 + rr * 8 + g;
        const bool has = r < rows;
        const int tok = has ? r / a.G : 0;
        const Span sp = has ? row_span(p0 + tok, sq.kv, a.block, a.window) : Span{0, 0};
        hi[mt][rr] = sp.hi;
        lo[mt][rr] = sp.lo;
        const T* src = static_cast<const T*>(a.q) + (sq.q0 + tok) * a.q_tok + (int64_t)(hk * a.G + (has ? r % a.G : 0)) * a.q_head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          qf[mt][ks][rr] = has ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + tq * 2) : 0u;
          qf[mt][ks][2 + rr] = has ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + 8 + tq * 2) : 0u;
        }
      }
    const int mrow = lane & 7, mi = lane >> 3;
    const int kkey = warp * 16 + (mi >> 1) * 8 + mrow, kch = mi & 1;      // K: (keys 0-7 | 8-15) x (chunk, chunk + 1)
    const int vkey = warp * 16 + (mi & 1) * 8 + mrow, vch = mi >> 1;      // V: the same, keys innermost
    bool ok = true;
    for (int t = t0; t < t1; ++t) {
      const int i = t - t0, s = i % ST;
      if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(full(s), (i / ST) & 1, a.wait_ns)))) break;
      const uint32_t kb = smem_u32(sm) + s * 2 * HALF, vb = kb + HALF;
      const int j0 = tile_at(tl, t) * TK + warp * 16;                      // this warp's keys
      const bool open = all_see(tl, j0, j0 + 16, a.sinks);
      if (any_sees(tl, j0, j0 + 16, a.sinks)) {
        float sc[MT][2][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k) sc[mt][n][k] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          uint32_t bf[4];
          ldsm4(kb + at(kkey, 2 * ks + kch), bf);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            Elem<T>::mma(sc[mt][0], qf[mt][ks], bf[0], bf[1]);
            Elem<T>::mma(sc[mt][1], qf[mt][ks], bf[2], bf[3]);
          }
        }
        if (!open) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (!sees(j0 + n * 8 + tq * 2 + (k & 1), lo[mt][k >> 1], hi[mt][k >> 1], a.sinks))
                  sc[mt][n][k] = -INFINITY;
        }
        // running maximum of each row, moved only when a key of this slice is
        // above it: the four lanes of a row agree through two shuffles then
        bool grow = false;
        float top[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int rr = 0; rr < 2; ++rr) {
            top[mt][rr] = fmaxf(fmaxf(sc[mt][0][2 * rr], sc[mt][0][2 * rr + 1]), fmaxf(sc[mt][1][2 * rr], sc[mt][1][2 * rr + 1]));
            grow |= top[mt][rr] > m_run[mt][rr];
          }
        if (__any_sync(0xFFFFFFFFu, grow)) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int rr = 0; rr < 2; ++rr) {
              float v = top[mt][rr];
              v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 1));
              v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 2));
              const float mn = fmaxf(m_run[mt][rr], v);
              const float al = mn == m_run[mt][rr] ? 1.0f : ex2f((m_run[mt][rr] - mn) * sl2);
              m_run[mt][rr] = mn;
              l_run[mt][rr] *= al;
#pragma unroll
              for (int n = 0; n < 2 * KS; ++n) {
                o[mt][n][2 * rr] *= al;
                o[mt][n][2 * rr + 1] *= al;
              }
            }
        }
        uint32_t pf[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          // a row that has seen nothing yet keeps 0 as its reference: 2^-inf = 0
          const float mb0 = m_run[mt][0] == -INFINITY ? 0.0f : m_run[mt][0] * sl2;
          const float mb1 = m_run[mt][1] == -INFINITY ? 0.0f : m_run[mt][1] * sl2;
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const float x0 = ex2f(fmaf(sc[mt][n][0], sl2, -mb0)), x1 = ex2f(fmaf(sc[mt][n][1], sl2, -mb0));
            const float y0 = ex2f(fmaf(sc[mt][n][2], sl2, -mb1)), y1 = ex2f(fmaf(sc[mt][n][3], sl2, -mb1));
            l_run[mt][0] += x0 + x1;
            l_run[mt][1] += y0 + y1;
            pf[mt][2 * n] = Elem<T>::pack(x0, x1);
            pf[mt][2 * n + 1] = Elem<T>::pack(y0, y1);
          }
        }
        if (open) {
#pragma unroll
          for (int nb = 0; nb < KS; ++nb) {
            uint32_t bf[4];
            ldsm4t(vb + at(vkey, 2 * nb + vch), bf);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              Elem<T>::mma(o[mt][2 * nb], pf[mt], bf[0], bf[1]);
              Elem<T>::mma(o[mt][2 * nb + 1], pf[mt], bf[2], bf[3]);
            }
          }
        } else {
          // Keys that no row sees may hold anything (0 x inf is not 0): their
          // Values are cleared in the fragments.  Keys that some rows see and
          // others do not (drafts of several tokens): if one holds an infinity
          // or a NaN, the product is taken token by token and only that
          // token's rows keep it.
          auto keep = [&](int klo, int khi, int j) -> uint32_t {
            return (sees(j, klo, khi, a.sinks) ? 0xFFFFu : 0u) | (sees(j + 1, klo, khi, a.sinks) ? 0xFFFF0000u : 0u);
          };
          const int ja = j0 + tq * 2;
          const uint32_t ma = keep(tl.lo_min, tl.hi_max, ja), mb = keep(tl.lo_min, tl.hi_max, ja + 8);
          bool odd = false;
          if (sq.qn > 1) {
#pragma unroll
            for (int nb = 0; nb < KS; ++nb) {
              uint32_t bf[4];
              ldsm4t(vb + at(vkey, 2 * nb + vch), bf);
              odd |= nonfinite2<T>(bf[0] & ma) || nonfinite2<T>(bf[1] & mb) || nonfinite2<T>(bf[2] & ma) ||
                     nonfinite2<T>(bf[3] & mb);
            }
            odd = __any_sync(0xFFFFFFFFu, odd);
          }
          const int turns = odd ? sq.qn : 1;
          for (int tk = 0; tk < turns; ++tk) {
            uint32_t wa = ma, wb = mb;
            bool own[MT][2];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int rr = 0; rr < 2; ++rr) own[mt][rr] = !odd || (mt * 16 + rr * 8 + g) / a.G == tk;
            if (odd) {
              const Span sp = row_span(p0 + tk, sq.kv, a.block, a.window);
              wa = keep(sp.lo, sp.hi, ja);
              wb = keep(sp.lo, sp.hi, ja + 8);
            }
#pragma unroll
            for (int nb = 0; nb < KS; ++nb) {
              uint32_t bf[4];
              ldsm4t(vb + at(vkey, 2 * nb + vch), bf);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                  float acc[4];
#pragma unroll
                  for (int k = 0; k < 4; ++k) acc[k] = o[mt][2 * nb + n][k];
                  Elem<T>::mma(acc, pf[mt], bf[2 * n] & wa, bf[2 * n + 1] & wb);
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    if (own[mt][k >> 1]) o[mt][2 * nb + n][k] = acc[k];
                }
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(s));
    }
    if (!ok && lane == 0) s_err = 1;
    // the four lanes of a row hold its sum in parts
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int rr = 0; rr < 2; ++rr) {
        float l = l_run[mt][rr];
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
        if (tq == 0) {
          s_ml[warp][mt * 16 + rr * 8 + g][0] = m_run[mt][rr];
          s_ml[warp][mt * 16 + rr * 8 + g][1] = l;
        }
      }
  }
  __syncthreads();   // every tile has been read: the ring becomes the warps' O
  if (s_err) {
    if (tid == 0) record_status(a.status, QWM_ERR_TIMEOUT);
  }
  float* so = reinterpret_cast<float*>(sm);        // [warp][ROWS][D]
  if (warp < kWarps) {
    const int g = lane >> 2, tq = lane & 3;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int n = 0; n < 2 * KS; ++n)
#pragma unroll
        for (int rr = 0; rr < 2; ++rr)
          *reinterpret_cast<float2*>(so + ((warp * ROWS + mt * 16 + rr * 8 + g) * D + n * 8 + tq * 2)) =
              make_float2(o[mt][n][2 * rr], o[mt][n][2 * rr + 1]);
  }
  __syncthreads();

  // (max, sum, O) of a row's channels 4c.. over the four warps
  const int64_t group = (int64_t)b * a.Hk + hk;
  auto emit = [&](int r, int c, float m, float l, float4 v) {
    const int tok = r / a.G, h = hk * a.G + r % a.G;
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    T* dst = static_cast<T*>(a.out) + (sq.q0 + tok) * a.o_tok + (int64_t)h * a.o_head + 4 * c;
    *reinterpret_cast<uint2*>(dst) = make_uint2(Elem<T>::pack(v.x * inv, v.y * inv), Elem<T>::pack(v.z * inv, v.w * inv));
    if (a.lse && c == 0) a.lse[(int64_t)h * a.N + sq.q0 + tok] = m == -INFINITY ? -INFINITY : m * a.scale + logf(l);
  };
  const int maxrows = a.max_q * a.G;
  for (int i = tid; i < rows * (D / 4); i += NT) {
    const int r = i / (D / 4), c = i % (D / 4);
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s_ml[w][r][0]);
    const float ref = m == -INFINITY ? 0.0f : m;
    float l = 0.0f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = ex2f((s_ml[w][r][0] - ref) * sl2);
      const float4 x = *reinterpret_cast<const float4*>(so + ((w * ROWS + r) * D + 4 * c));
      l = fmaf(s_ml[w][r][1], f, l);
      v.x = fmaf(x.x, f, v.x); v.y = fmaf(x.y, f, v.y); v.z = fmaf(x.z, f, v.z); v.w = fmaf(x.w, f, v.w);
    }
    if (parts == 1) {
      emit(r, c, m, l, v);
    } else {
      const int64_t pr = (group * a.nsplit + part) * maxrows + r;
      *reinterpret_cast<float4*>(a.part_o + pr * D + 4 * c) = v;
      if (c == 0) a.part_ml[pr] = make_float2(m, l);
    }
  }
  if (parts == 1) return;
  // the part that arrives last joins all of them
  __threadfence();
  __syncthreads();
  if (tid == 0) s_last = atomicAdd(a.counter + group, 1) == parts - 1;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  for (int i = tid; i < rows * (D / 4); i += NT) {
    const int r = i / (D / 4), c = i % (D / 4);
    const int64_t pr = group * a.nsplit * maxrows + r;
    float m = -INFINITY;
    for (int p = 0; p < parts; ++p) m = fmaxf(m, __ldcg(&a.part_ml[pr + (int64_t)p * maxrows].x));
    const float ref = m == -INFINITY ? 0.0f : m;
    float l = 0.0f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const int64_t at_p = pr + (int64_t)p * maxrows;
      const float2 ml = __ldcg(&a.part_ml[at_p]);
      const float4 x = __ldcg(reinterpret_cast<const float4*>(a.part_o + at_p * D + 4 * c));
      const float f = ex2f((ml.x - ref) * sl2);
      l = fmaf(ml.y, f, l);
      v.x = fmaf(x.x, f, v.x); v.y = fmaf(x.y, f, v.y); v.z = fmaf(x.z, f, v.z); v.w = fmaf(x.w, f, v.w);
    }
    emit(r, c, m, l, v);
  }
  if (tid == 0) a.counter[group] = 0;
}

template <typename T, int D, int MT>
cudaError_t go(const PagedArgs& a, const CUtensorMap& map, cudaStream_t s) {
  constexpr int smem = kRing + 1024;
  static_assert(kWarps * 16 * MT * D * 4 <= kRing, "the ring holds the merge");
  cudaError_t e = cudaFuncSetAttribute(paged_step<T, D, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  paged_step<T, D, MT><<<dim3(a.nsplit, a.Hk, a.B), NT, smem, s>>>(map, a);
  return cudaGetLastError();
}
template <typename T, int D>
cudaError_t pick(const PagedArgs& a, const CUtensorMap& map, cudaStream_t s) {
  return a.max_q * a.G <= 16 ? go<T, D, 1>(a, map, s) : go<T, D, 2>(a, map, s);
}

}  // namespace

PagedPlan plan_step(int B, int Hk, int rows, int64_t max_visible, int nsm, bool split) {
  PagedPlan p{};
  p.step = 1;
  p.groups = B * Hk;
  p.rows = rows;
  const int64_t tiles = (max_visible + TK - 1) / TK + 2;
  // Parts of at least 8 tiles (512 keys: a part's O costs about a fiftieth of
  // its K and V), and about three waves of two CTAs per SM, so that sequences
  // of unequal length even out.
  p.min_tiles = 8;
  p.nsplit = 1;
  if (split) {
    const int64_t want = (6 * (int64_t)nsm + p.groups - 1) / p.groups;
    const int64_t most = (tiles + p.min_tiles - 1) / p.min_tiles;
    p.nsplit = (int)(want < most ? want : most);
    if (p.nsplit > 256) p.nsplit = 256;
    if (p.nsplit < 1) p.nsplit = 1;
  }
  return p;
}

cudaError_t launch_paged_step(const PagedArgs& a, const CUtensorMap& map, int D, int dtype, cudaStream_t s) {
  if (dtype == QWM_F16) return D == 64 ? pick<__half, 64>(a, map, s) : pick<__half, 128>(a, map, s);
  return D == 64 ? pick<__nv_bfloat16, 64>(a, map, s) : pick<__nv_bfloat16, 128>(a, map, s);
}

}  // namespace qwm
