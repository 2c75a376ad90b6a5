// paged_step.cu -- attention of a few rows of a sequence over its pages: single
// new tokens and short drafts (Query tokens x grouped heads <= 16 rows).
//
// Mathematics: softmax over the visible keys with a running maximum m and sum l
// per row (O and l scaled by 2^((m_old - m_new) c) when m grows), so one pass
// over K and V suffices.  The bound is HBM: K and V of the visible tokens are
// read once per cache head for all the grouped Query heads.
//
// The tiles of all (sequence, cache head) groups form one line, which the CTAs (one
// per SM) share out evenly whatever the lengths are; a CTA walks its stretch
// group by group.  Two producer warps, one of K and one of V, keep a ring of tiles
// (64 or 128 keys) in flight by TMA.  One warp for both sent them one after the
// other: 32 sequences of 100 to 30000 keys x 8 heads, window 8192, took 84.3 us and
// take 80.8 with two; one token over 517 keys x 12 heads in pages of 16, where a
// tile is many copies, 9.9 and 8.1.  Of eight more warps four take a quarter of a
// tile's keys each, the other four those of the next tile, and carry their own
// m, l and O through the group (no barrier between them in the loop); then they
// are merged through shared memory.  The rows are the M = 16 side of mma.sync: a
// tcgen05 tile would be 128 rows high for the 1 to 16 used here, and its TMEM
// round trip is longer than the whole of a short step.  P is rounded to the cache's
// type for the product, after its sum (error against 64 bits 1.0 to 1.1 times the
// fp32 form's).
// A group cut by the ends of stretches is joined by the CTA that finishes last,
// in the order of the keys, so the result does not depend on which one that is.
#include "paged.cuh"

namespace qwm {
namespace {
using namespace ptx;

constexpr int kWarps = 8;                // consumer warps
constexpr int NT = (kWarps + 2) * 32;    // and two producers, of K and of V
// What a group costs a CTA beside its tiles (Queries, merge, output: about 5 K
// cycles), in tiles' time (1.3 K cycles when all CTAs stream).
constexpr int kGroupCost = 4;

// KP 16-key groups of a warp.  A tile's chain of products, exponentials and
// products takes as long for two groups as for one, so two where the chain bounds
// (64 channels; whole groups), one where HBM does and finer slots keep it busier
// (128 channels on the line: 131071 keys 86 us with one, 91 with two; 517 keys x 12
// whole groups 8.9 and 7.6; all four with one producer warp for K and V).
template <int D, int KP_>
struct Shape {
  static constexpr int KP = KP_;
  static constexpr int TK = 64 * KP;                           // keys per tile
  static constexpr int SLOT = TK * D * 2;                      // bytes of a K or V tile
  static constexpr int NS = SLOT == 32768 ? 4 : 8;             // slots of the ring: K, V, K, V, ...
  static_assert(NS % 4 == 0, "an even number of tiles: a slot belongs to one warp group");
  static constexpr int MERGE = NS * SLOT;                      // the warps' O [warp][16][D], beside the ring so that
                                                               // the next group's tiles come in meanwhile
  static constexpr int TOTAL = MERGE + kWarps * 16 * D * 4 + 1024;
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// Byte of 16-byte chunk `chunk` (8 channels) of key `key` in a tile [D / 64][TK
// keys][128 bytes], 128-byte swizzled.
template <int TK>
__device__ __forceinline__ uint32_t at(int key, int chunk) {
  return (uint32_t)((chunk >> 3) * (TK * 128) + key * 128 + (((chunk & 7) ^ (key & 7)) << 4));
}

__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {   // a >= 0, b > 0
  return ((a | b) >> 32) ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

template <typename T, int D, int KP>
__global__ void __launch_bounds__(NT, 1) paged_step(const __grid_constant__ CUtensorMap map, const PagedArgs a) {
  using L = Shape<D, KP>;
  constexpr int NS = L::NS, TK = L::TK;
  constexpr int KS = D / 16;                       // k16 steps of Q K^T, n16 blocks of P V
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  __shared__ uint64_t bars[2 * NS];
  __shared__ float s_ml[kWarps][16][2];
  __shared__ int64_t s_scan[kWarps + 2], s_first;
  __shared__ Seq s_sq;
  __shared__ Tiles s_tl;
  __shared__ int s_last, s_seq;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // tiles of a group of sequence b (one for a group that has rows and sees
  // nothing: its output is written all the same)
  auto tiles_of = [&](int b, Seq& sq, Tiles& tl) -> int {
    // on the line CTA 0 looks at every sequence, of whole groups each CTA at its own
    if (!load_seq(a, b, sq) && (a.nsplit == 1 || blockIdx.x == 0)) record_status(a.status, QWM_ERR_INVALID_ARG);
    if (sq.qn == 0) return 0;
    tl = make_tiles<TK>(sq.kv - sq.qn, sq.kv - 1, sq.kv, a.block, a.window, a.sinks);
    return max(tl.n, 1);
  };
  auto full = [&](int s) { return smem_u32(&bars[s]); };
  auto empty = [&](int s) { return smem_u32(&bars[NS + s]); };
  if (tid == 0) {
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), kWarps / 2);
    }
    fence_mbar_init();
  }
  grid_begin();
  // The line: a group of sequence b takes n(b) + kGroupCost places, its tiles
  // last; sequence b's groups follow those of the sequences before it.  A scan
  // over the sequences gives the total and the sequence in which this CTA's
  // stretch begins: up to 32 sequences by each warp for itself, more by the CTA,
  // each thread with a run of sequences.  Without a workspace, a CTA takes the
  // group of its number.
  const bool split = a.nsplit > 1;
  Seq sq;
  Tiles tl;
  int b, n, hk;
  int64_t x0, x1, g0, share = 0;
  if (split) {
    const bool alone = a.B <= 32;
    const int who = alone ? lane : tid, run = alone ? 1 : (a.B + NT - 1) / NT;
    const int b0 = min(a.B, who * run), b1 = min(a.B, b0 + run);
    int64_t mine = 0;
    for (int i = b0; i < b1; ++i) {
      n = tiles_of(i, sq, tl);
      mine += n ? n + kGroupCost : 0;
    }
    int64_t incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t x = __shfl_up_sync(0xFFFFFFFFu, incl, d);
      if (lane >= d) incl += x;
    }
    int64_t before = incl - mine, total = __shfl_sync(0xFFFFFFFFu, incl, 31);
    if (!alone) {
      if (lane == 31) s_scan[warp] = incl;
      __syncthreads();
      total = 0;
#pragma unroll
      for (int w = 0; w < kWarps + 2; ++w) {
        if (w < warp) before += s_scan[w];
        total += s_scan[w];
      }
    }
    before *= a.Hk;
    mine *= a.Hk;
    total *= a.Hk;
    share = max(divide(total + gridDim.x - 1, gridDim.x), (int64_t)a.min_tiles);
    x0 = blockIdx.x * share;
    if (x0 >= total) return;
    x1 = min(total, x0 + share);
    const bool here = x0 >= before && x0 < before + mine;
    if (alone) {
      // lane `src` has the sequence
      const int src = __ffs(__ballot_sync(0xFFFFFFFFu, here)) - 1;
      auto from = [&](auto v) { return __shfl_sync(0xFFFFFFFFu, v, src); };
      b = src;
      sq.q0 = from(sq.q0);
      sq.qn = from(sq.qn);
      sq.kv = from(sq.kv);
      tl.lo_min = from(tl.lo_min);
      tl.lo_max = from(tl.lo_max);
      tl.hi_min = from(tl.hi_min);
      tl.hi_max = from(tl.hi_max);
      tl.n_win = from(tl.n_win);
      tl.w_start = from(tl.w_start);
      tl.n = from(tl.n);
      g0 = from(before);
      __syncthreads();                              // the barriers are set up
    } else {
      if (here) {
        int64_t at = before;
        for (int i = b0; i < b1; ++i) {
          n = tiles_of(i, sq, tl);
          const int64_t len = n ? (int64_t)(n + kGroupCost) * a.Hk : 0;
          if (x0 < at + len) {
            s_seq = i;
            s_first = at;
            s_sq = sq;
            s_tl = tl;
            break;
          }
          at += len;
        }
      }
      __syncthreads();
      b = s_seq;
      sq = s_sq;
      tl = s_tl;
      g0 = s_first;
    }
    n = max(tl.n, 1);
    hk = (int)divide(x0 - g0, n + kGroupCost);
    g0 += (int64_t)hk * (n + kGroupCost);
  } else {
    b = blockIdx.x / a.Hk;
    hk = blockIdx.x % a.Hk;
    n = tiles_of(b, sq, tl);
    if (n == 0) return;
    x0 = g0 = 0;
    x1 = n + kGroupCost;
    __syncthreads();
  }
  // The CTA's piece of the current group: tiles t0 .. t1 - 1, none if t0 >= t1.
  int t0, t1;
  auto piece = [&]() {
    const int64_t first = g0 + kGroupCost;
    t0 = (int)max((int64_t)0, x0 - first);
    t1 = (int)min((int64_t)n, x1 - first);
  };
  auto next_group = [&]() -> bool {
    g0 += n + kGroupCost;
    if (g0 >= x1) return false;
    if (++hk == a.Hk) {
      hk = 0;
      do n = tiles_of(++b, sq, tl); while (n == 0);
    }
    return true;
  };

  if (warp >= kWarps) {
    // ---------------------------------------------------------- producers of K and V
    // lane = box * 2 + channel half; a box is the part of a page (at most 64 tokens
    // of it) that lies in the tile.  Boxes that no row sees are not read.
    const int kv = warp - kWarps;
    const int box_log2 = min(a.page_log2, 6);
    const int box = lane >> 1, half = lane & 1;
    const bool mine = box < (TK >> box_log2) && half * 64 < D;
    const uint32_t dst = smem_u32(sm) + half * (TK * 128) + ((box << box_log2) * 128);
    bool ok = true;
    int i = 0;                                     // tiles sent
    do {
      piece();
      t1 = min(t1, tl.n);
      const int32_t* trow = a.table + (int64_t)b * a.table_stride;
      auto page_of = [&](int t, bool& want) -> int {
        const int j0 = tile_at(tl, t) * TK + (box << box_log2);
        want = mine && any_sees(tl, j0, j0 + (1 << box_log2), a.sinks);
        return want ? trow[j0 >> a.page_log2] : 0;
      };
      bool want = false;
      int page = t0 < t1 ? page_of(t0, want) : 0;
      for (int t = t0; t < t1 && !a.idle; ++t) {
        bool want_n = false;
        int page_n = 0;
        if (t + 1 < t1) page_n = page_of(t + 1, want_n);   // its latency runs beside the copies
        if (want && (page < 0 || page >= a.num_pages)) {   // not followed: the first page in its place
          record_status(a.status, QWM_ERR_INVALID_ARG);
          page = 0;
        }
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, want)) * (128u << box_log2);
        const int y = (tile_at(tl, t) * TK + (box << box_log2)) & ((1 << a.page_log2) - 1);
        const int s = (2 * i + kv) % NS;
        if (i >= NS / 2 && !(ok = __all_sync(0xFFFFFFFFu, mbar_wait(empty(s), (i / (NS / 2) - 1) & 1, a.wait_ns)))) break;
        if (lane == 0) mbar_arrive_expect_tx(full(s), bytes);
        __syncwarp();
        if (want) tma_load_3d(dst + s * L::SLOT, &map, half * 64, y, (page * 2 + kv) * a.Hk + hk, full(s));
        __syncwarp();
        ++i;
        page = page_n;
        want = want_n;
      }
    } while (ok && next_group());
    if (!ok && lane == 0) record_status(a.status, QWM_ERR_TIMEOUT);
    // The last copies land before this warp ends, and so before the CTA can: the
    // consumers may have given up on them.  Otherwise this is the wait the
    // consumers are in as well.
    for (int u = max(0, i - NS / 2); u < i; ++u) mbar_wait(full((2 * u + kv) % NS), (u / (NS / 2)) & 1, kDrainNs);
    return;
  }

  // ------------------------------------------------------------ consumers
  const float sl2 = a.scale * 1.4426950408889634f;
  const int g = lane >> 2, tq = lane & 3;
  const int wg = warp >> 2, key0 = (warp & 3) * 16 * KP;                // tile parity, first key of the tile
  const int mrow = lane & 7, mi = lane >> 3;
  const int kkey = key0 + (mi >> 1) * 8 + mrow, kch = mi & 1;           // K: (keys 0-7 | 8-15) x (chunk, chunk + 1)
  const int vkey = key0 + (mi & 1) * 8 + mrow, vch = mi >> 1;           // V: the same, keys innermost
  const int maxrows = a.max_q * a.G;
  float* so = reinterpret_cast<float*>(sm + L::MERGE);                  // [warp][16][D]
  bool ok = true;                                                       // no wait of this warp has run out
  int filled = 0;                                                       // slots of the pieces before
  do {
    piece();
    if (t0 >= t1) continue;
    const int rows = sq.qn * a.G;                                       // <= 16
    const int t_end = min(t1, tl.n);
    const int64_t group = (int64_t)b * a.Hk + hk, first = g0 + kGroupCost;
    const bool whole = first >= x0 && first + n <= x1;                  // the group is this CTA's alone
    const int64_t c0 = whole ? 0 : divide(first, share), c1 = whole ? 0 : divide(first + n - 1, share);   // its CTAs
    const int parts = (int)(c1 - c0) + 1;
    const int p0 = sq.kv - sq.qn;
    // the fragments of mma.sync: this lane has rows g and g + 8 (index rr)
    float o[2 * KS][4];
    float m_run[2], l_run[2];
    uint32_t qf[KS][4];
    int hi[2], lo[2];
#pragma unroll
    for (int k = 0; k < 2 * KS; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[k][e] = 0.0f;
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      m_run[rr] = -INFINITY;
      l_run[rr] = 0.0f;
      const int r = rr * 8 + g;
      const bool has = r < rows;
      const int tok = has ? r / a.G : 0;
      const Span sp = has ? row_span(p0 + tok, sq.kv, a.block, a.window) : Span{0, 0};
      hi[rr] = sp.hi;
      lo[rr] = sp.lo;
      const T* src = static_cast<const T*>(a.q) + (sq.q0 + tok) * a.q_tok + (int64_t)(hk * a.G + (has ? r % a.G : 0)) * a.q_head;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[ks][rr] = has ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + tq * 2) : 0u;
        qf[ks][2 + rr] = has ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + 8 + tq * 2) : 0u;
      }
    }
    // This warp group's tiles are those of its parity in the CTA's count of tiles,
    // so that a slot of the ring is always the same group's: a group that did not
    // wait for every use of a slot could take the phase before the one it waits
    // for as done (a parity tells only two apart).
    for (int t = t0 + (((filled >> 1) + wg) & 1); t < t_end && ok; t += 2) {
      const int i = filled + 2 * (t - t0), s = i % NS;                   // slots s and s + 1
      const int j0 = tile_at(tl, t) * TK + key0;                         // this warp's keys: j0 .. j0 + 16 KP - 1
      if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(full(s), (i / NS) & 1, a.wait_ns)))) break;
      const uint32_t kb = smem_u32(sm) + s * L::SLOT, vb = kb + L::SLOT;
      const bool open = all_see(tl, j0, j0 + 16 * KP, a.sinks), any = any_sees(tl, j0, j0 + 16 * KP, a.sinks);
      uint32_t pf[KP][4];
      if (any) {
        float sc[KP][2][4];
#pragma unroll
        for (int kp = 0; kp < KP; ++kp)
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[kp][k][e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int kp = 0; kp < KP; ++kp) {
            uint32_t bf[4];
            ldsm4(kb + at<TK>(kkey + 16 * kp, 2 * ks + kch), bf);
            Elem<T>::mma(sc[kp][0], qf[ks], bf[0], bf[1]);
            Elem<T>::mma(sc[kp][1], qf[ks], bf[2], bf[3]);
          }
        if (!open) {
#pragma unroll
          for (int kp = 0; kp < KP; ++kp)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (!sees(j0 + kp * 16 + k * 8 + tq * 2 + (e & 1), lo[e >> 1], hi[e >> 1], a.sinks)) sc[kp][k][e] = -INFINITY;
        }
        // running maximum of each row, moved only when a key of this slice is
        // above it: the four lanes of a row agree through two shuffles then
        bool grow = false;
        float top[2];
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) {
          top[rr] = -INFINITY;
#pragma unroll
          for (int kp = 0; kp < KP; ++kp)
            top[rr] = fmaxf(top[rr], fmaxf(fmaxf(sc[kp][0][2 * rr], sc[kp][0][2 * rr + 1]),
                                           fmaxf(sc[kp][1][2 * rr], sc[kp][1][2 * rr + 1])));
          grow |= top[rr] > m_run[rr];
        }
        if (__any_sync(0xFFFFFFFFu, grow)) {
#pragma unroll
          for (int rr = 0; rr < 2; ++rr) {
            float v = top[rr];
            v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 1));
            v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 2));
            const float mn = fmaxf(m_run[rr], v);
            const float al = mn == m_run[rr] ? 1.0f : ex2f((m_run[rr] - mn) * sl2);
            m_run[rr] = mn;
            l_run[rr] *= al;
#pragma unroll
            for (int k = 0; k < 2 * KS; ++k) {
              o[k][2 * rr] *= al;
              o[k][2 * rr + 1] *= al;
            }
          }
        }
        // a row that has seen nothing yet keeps 0 as its reference: 2^-inf = 0
        const float mb0 = m_run[0] == -INFINITY ? 0.0f : m_run[0] * sl2;
        const float mb1 = m_run[1] == -INFINITY ? 0.0f : m_run[1] * sl2;
#pragma unroll
        for (int kp = 0; kp < KP; ++kp)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float v0 = ex2f(fmaf(sc[kp][k][0], sl2, -mb0)), v1 = ex2f(fmaf(sc[kp][k][1], sl2, -mb0));
            const float w0 = ex2f(fmaf(sc[kp][k][2], sl2, -mb1)), w1 = ex2f(fmaf(sc[kp][k][3], sl2, -mb1));
            l_run[0] += v0 + v1;
            l_run[1] += w0 + w1;
            pf[kp][2 * k] = Elem<T>::pack(v0, v1);
            pf[kp][2 * k + 1] = Elem<T>::pack(w0, w1);
          }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(s));
      if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(full(s + 1), (i / NS) & 1, a.wait_ns)))) break;
      if (open) {
#pragma unroll
        for (int kp = 0; kp < KP; ++kp)
#pragma unroll
          for (int nb = 0; nb < KS; ++nb) {
            uint32_t bf[4];
            ldsm4t(vb + at<TK>(vkey + 16 * kp, 2 * nb + vch), bf);
            Elem<T>::mma(o[2 * nb], pf[kp], bf[0], bf[1]);
            Elem<T>::mma(o[2 * nb + 1], pf[kp], bf[2], bf[3]);
          }
      } else if (any) {
        // Keys that no row sees may hold anything (0 x inf is not 0): their
        // Values are cleared in the fragments.  Keys that some rows see and
        // others do not (drafts of several tokens): if one holds an infinity
        // or a NaN, the product is taken token by token and only that
        // token's rows keep it.
        auto keep = [&](int klo, int khi, int j) -> uint32_t {
          return (sees(j, klo, khi, a.sinks) ? 0xFFFFu : 0u) | (sees(j + 1, klo, khi, a.sinks) ? 0xFFFF0000u : 0u);
        };
#pragma unroll
        for (int kp = 0; kp < KP; ++kp) {
          const int ja = j0 + kp * 16 + tq * 2;
          const uint32_t ma = keep(tl.lo_min, tl.hi_max, ja), mb = keep(tl.lo_min, tl.hi_max, ja + 8);
          bool odd = false;
          if (sq.qn > 1) {
#pragma unroll
            for (int nb = 0; nb < KS; ++nb) {
              uint32_t bf[4];
              ldsm4t(vb + at<TK>(vkey + 16 * kp, 2 * nb + vch), bf);
              odd |= nonfinite2<T>(bf[0] & ma) || nonfinite2<T>(bf[1] & mb) || nonfinite2<T>(bf[2] & ma) ||
                     nonfinite2<T>(bf[3] & mb);
            }
            odd = __any_sync(0xFFFFFFFFu, odd);
          }
          const int turns = odd ? sq.qn : 1;
          for (int tk = 0; tk < turns; ++tk) {
            uint32_t wa = ma, wb = mb;
            bool own[2];
#pragma unroll
            for (int rr = 0; rr < 2; ++rr) own[rr] = !odd || (rr * 8 + g) / a.G == tk;
            if (odd) {
              const Span sp = row_span(p0 + tk, sq.kv, a.block, a.window);
              wa = keep(sp.lo, sp.hi, ja);
              wb = keep(sp.lo, sp.hi, ja + 8);
            }
#pragma unroll
            for (int nb = 0; nb < KS; ++nb) {
              uint32_t bf[4];
              ldsm4t(vb + at<TK>(vkey + 16 * kp, 2 * nb + vch), bf);
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                float acc[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = o[2 * nb + k][e];
                Elem<T>::mma(acc, pf[kp], bf[2 * k] & wa, bf[2 * k + 1] & wb);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (own[e >> 1]) o[2 * nb + k][e] = acc[e];
              }
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(s + 1));
    }
    filled += 2 * max(0, t_end - t0);
    if (!ok && lane == 0) record_status(a.status, QWM_ERR_TIMEOUT);

    // -------------------------------------------------------- the warps' (max, sum, O) of the piece
    named_bar_sync(1, kWarps * 32);                  // the last piece's have been read
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      const int r = rr * 8 + g;
      float l = l_run[rr];                           // the four lanes of a row hold its sum in parts
      l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
      l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
      if (r >= rows) continue;
      if (tq == 0) {
        s_ml[warp][r][0] = m_run[rr];
        s_ml[warp][r][1] = l;
      }
#pragma unroll
      for (int k = 0; k < 2 * KS; ++k)
        *reinterpret_cast<float2*>(so + ((warp * 16 + r) * D + k * 8 + tq * 2)) = make_float2(o[k][2 * rr], o[k][2 * rr + 1]);
    }
    named_bar_sync(1, kWarps * 32);
    auto emit = [&](int r, int c, float m, float l, float4 v) {
      const int tok = r / a.G, h = hk * a.G + r % a.G;
      const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
      T* dst = static_cast<T*>(a.out) + (sq.q0 + tok) * a.o_tok + (int64_t)h * a.o_head + 4 * c;
      *reinterpret_cast<uint2*>(dst) = make_uint2(Elem<T>::pack(v.x * inv, v.y * inv), Elem<T>::pack(v.z * inv, v.w * inv));
      if (a.lse && c == 0) a.lse[(int64_t)h * a.N + sq.q0 + tok] = m * a.scale + logf(l);   // -inf + log 0; NaN with a NaN l
    };
    // (m, l, O) of row r's channels 4c .. over the first `count` entries of s_ml and so
    auto merge = [&](int count, int r, int c, float& m, float& l, float4& v) {
      m = -INFINITY;
      for (int w = 0; w < count; ++w) m = fmaxf(m, s_ml[w][r][0]);
      const float ref = m == -INFINITY ? 0.0f : m;
      l = 0.0f;
      v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int w = 0; w < count; ++w) {
        const float f = ex2f((s_ml[w][r][0] - ref) * sl2);
        const float4 x = *reinterpret_cast<const float4*>(so + ((w * 16 + r) * D + 4 * c));
        l = fmaf(s_ml[w][r][1], f, l);
        v.x = fmaf(x.x, f, v.x); v.y = fmaf(x.y, f, v.y); v.z = fmaf(x.z, f, v.z); v.w = fmaf(x.w, f, v.w);
      }
    };
    for (int idx = tid; idx < rows * (D / 4); idx += kWarps * 32) {
      const int r = idx / (D / 4), c = idx % (D / 4);
      float m, l;
      float4 v;
      merge(kWarps, r, c, m, l, v);
      if (parts == 1) {
        emit(r, c, m, l, v);
      } else {
        // a CTA's places: 0 for a group that began before its stretch, 1 for one that begins in it
        const int64_t pr = (2 * (int64_t)blockIdx.x + (first >= x0 ? 1 : 0)) * maxrows + r;
        *reinterpret_cast<float4*>(a.part_o + pr * D + 4 * c) = v;
        if (c == 0) a.part_ml[pr] = make_float2(m, l);
      }
    }
    if (parts == 1) continue;
    // -------------------------------------------------------- the CTA that arrives last joins all parts
    __threadfence();
    named_bar_sync(1, kWarps * 32);
    if (tid == 0) s_last = atomicAdd(a.counter + group, 1) == parts - 1;
    named_bar_sync(1, kWarps * 32);
    if (!s_last) continue;
    __threadfence();
    // part p's rows: the first CTA's second place, the others' first
    auto place = [&](int p) { return (2 * (c0 + p) + (p == 0 ? 1 : 0)) * maxrows; };
    // A warp takes whole rows (where there are fewer rows than warps and more
    // parts than a warp has in flight, the warps share a row's parts out), a lane
    // four channels.
    constexpr int LPR = D / 4, RPW = 32 / LPR;        // lanes per row, rows per warp at a time
    constexpr int PU = 20;                            // parts in flight
    const int rr = (rows + RPW - 1) / RPW;
    const int slices = rr > 4 || parts <= PU ? 1 : (rr > 2 ? 2 : (rr > 1 ? 4 : 8)), sl = warp % slices;
    const int q0 = parts * sl / slices, q1 = parts * (sl + 1) / slices;
    for (int rb = (warp / slices) * RPW; rb < rows; rb += (kWarps / slices) * RPW) {
      const int r = rb + lane / LPR, c = lane % LPR;
      float m = -INFINITY, l = 0.0f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r >= rows) continue;
      for (int p = q0; p < q1; p += PU) {
        float2 ml[PU];
        float4 x[PU];
#pragma unroll
        for (int u = 0; u < PU; ++u) {
          const int64_t at_p = place(min(p + u, q1 - 1)) + r;
          ml[u] = __ldcg(&a.part_ml[at_p]);
          x[u] = __ldcg(reinterpret_cast<const float4*>(a.part_o + at_p * D + 4 * c));
        }
        float mn = m;
#pragma unroll
        for (int u = 0; u < PU; ++u) mn = fmaxf(mn, ml[u].x);
        const float ref = mn == -INFINITY ? 0.0f : mn;
        const float al = ex2f((m - ref) * sl2);
        m = mn;
        l *= al;
        v.x *= al; v.y *= al; v.z *= al; v.w *= al;
#pragma unroll
        for (int u = 0; u < PU; ++u) {
          if (p + u >= q1) break;
          const float f = ex2f((ml[u].x - ref) * sl2);
          l = fmaf(ml[u].y, f, l);
          v.x = fmaf(x[u].x, f, v.x); v.y = fmaf(x[u].y, f, v.y); v.z = fmaf(x[u].z, f, v.z); v.w = fmaf(x[u].w, f, v.w);
        }
      }
      if (slices == 1) {
        emit(r, c, m, l, v);
      } else {
        *reinterpret_cast<float4*>(so + ((sl * 16 + r) * D + 4 * c)) = v;
        if (c == 0) {
          s_ml[sl][r][0] = m;
          s_ml[sl][r][1] = l;
        }
      }
    }
    if (slices > 1) {
      named_bar_sync(1, kWarps * 32);
      for (int idx = tid; idx < rows * (D / 4); idx += kWarps * 32) {
        const int r = idx / (D / 4), c = idx % (D / 4);
        float m, l;
        float4 v;
        merge(slices, r, c, m, l, v);
        emit(r, c, m, l, v);
      }
    }
    if (tid == 0) a.counter[group] = 0;
  } while (next_group());
}

template <typename T, int D, int KP>
cudaError_t go(const PagedArgs& a, const CUtensorMap& map, cudaStream_t s) {
  constexpr int smem = Shape<D, KP>::TOTAL;
  static bool done[64];
  cudaError_t e = allow_smem(paged_step<T, D, KP>, smem, done);
  if (e != cudaSuccess) return e;
  return launch_ahead(paged_step<T, D, KP>, dim3((unsigned)(a.nsplit > 1 ? a.nsplit : a.B * a.Hk)), NT, smem, s, map, a);
}
template <typename T>
cudaError_t pick(const PagedArgs& a, const CUtensorMap& map, int D, cudaStream_t s) {
  if (D == 64) return go<T, 64, 2>(a, map, s);
  return a.nsplit > 1 ? go<T, 128, 1>(a, map, s) : go<T, 128, 2>(a, map, s);
}

}  // namespace

PagedPlan plan_step(int B, int Hk, int D, int rows, int64_t max_visible, int nsm, bool split) {
  PagedPlan p{};
  p.step = 1;
  p.groups = B * Hk;
  p.rows = rows;
  // the shortest stretch, in places (3 and 6 were no better from 300 to 4000 keys)
  p.min_tiles = 4;
  p.nsplit = 1;
  const int64_t tiles = (max_visible + 63) / 64 + 1;                  // of 64 keys, of a group at most
  // Whole groups, a CTA each, take their waves x (a CTA's start and end and its
  // tiles), the line an even share of all places after its start, parts and join.
  // In us, fitted to 1 to 8 sequences of 64 to 2000 keys; a tile's time is its own
  // chain's, or its share of HBM when many CTAs stream.  Long groups are shared:
  // they seldom have one length.  More groups than counters fill the SMs uncut.
  // 12 groups of 1000 keys of 128 channels take 8.8 us whole and 9.2 shared, of
  // 2000 keys 13.3 and 10.2; 48 of 1500 keys 11.2 and 13.0, of 2000 13.5 and 12.7;
  // 8 groups of 1000 keys of 64 channels 6.7 and 8.4.  Near the change the two are
  // close, and 96 groups of 2000 keys swing: 17 to 20 us either way.
  const double chain = D == 128 ? 0.29 : 0.24, hbm = D == 128 ? 0.71 : 0.4;
  const double stream = p.groups < nsm ? hbm * p.groups / nsm : hbm;
  const double each = stream > chain ? stream : chain;
  const double whole = (double)((p.groups + nsm - 1) / nsm) * ((D == 128 ? 4.0 : 2.8) + tiles * each);
  const double shared = (D == 128 ? 8.2 : 7.6) + (D == 128 ? 0.44 : 0.33) * (double)(tiles + kGroupCost) * p.groups / nsm;
  if (split && (tiles > 40 || whole > shared) && p.groups <= QWM_PAGED_COUNTER_BYTES / 4) {
    // a CTA per SM, or as many as have min_tiles places each
    const int64_t places = ((max_visible + (D == 128 ? 63 : 127)) / (D == 128 ? 64 : 128) + 1 + kGroupCost) * p.groups;
    const int64_t want = (places + p.min_tiles - 1) / p.min_tiles;
    p.nsplit = (int)(want < nsm ? want : nsm);
  }
  return p;
}

cudaError_t launch_paged_step(const PagedArgs& a, const CUtensorMap& map, int D, int dtype, cudaStream_t s) {
  if (dtype == QWM_F16) return pick<__half>(a, map, D, s);
  return pick<__nv_bfloat16>(a, map, D, s);
}

}  // namespace qwm
