// paged.cuh -- shared definitions of the paged storage's kernels: arguments,
// what a row sees, element types.
#pragma once

#include "qwm_internal.cuh"
#include "ptx_sm103.cuh"

namespace qwm {

// ------------------------------------------------------------ rope and append
struct RopeSegment {            // a tensor [N][heads][D] and where its rows go
  const void* src;
  void* dst;
  int32_t s_tok, s_head;        // strides in elements
  int32_t d_tok, d_head;
  int32_t heads;
  int32_t rotate;               // 0: copied
  int32_t page;                 // -1: to dst; 0 / 1: to the Keys / Values of the token's page
};
struct RopeArgs {
  RopeSegment seg[3];
  int32_t nseg, total_heads;
  int32_t D, pairs[3], P;
  float sign;                   // -1: the gradient
  int64_t N;
  const float* inv_freq;        // [P]; null: nothing is rotated
  const int32_t* pos;           // [N][3]
  // paged destinations
  const int32_t *q_off, *kv_len, *table;
  int32_t B, table_stride, page_log2, kv_heads, max_q, max_kv;
  int64_t num_pages;
  void* pages;
  __half* scales;               // of the rows of 8-bit pages; null: 16-bit pages
  int32_t* status;
};
cudaError_t launch_rope(const RopeArgs& a, int dtype, bool interleaved, cudaStream_t s);
cudaError_t launch_store(const RopeArgs& a, int dtype, bool interleaved, cudaStream_t s);

// ------------------------------------------------------------ read-back
struct ReadArgs {
  const uint8_t* pages;
  const __half* scales;         // null: 16-bit pages
  void* out[2];                 // Keys, Values (null: not wanted)
  int32_t o_tok[2], o_head[2];  // strides in elements
  int32_t D;
  int64_t N;
  const int32_t *q_off, *kv_len, *table;
  int32_t B, table_stride, page_log2, kv_heads, max_q, max_kv;
  int64_t num_pages;
  int32_t* status;
};
cudaError_t launch_read(const ReadArgs& a, int dtype, cudaStream_t s);

// ------------------------------------------------------------ attention
struct PagedArgs {
  const void* q;
  void* out;
  int64_t q_tok, q_head, o_tok, o_head;  // strides in elements
  float* lse;                            // [Hq][N] or null
  int64_t N;
  const int32_t *q_off, *kv_len, *table;
  int32_t B, table_stride, max_q, max_kv;
  int32_t Hk, G;                         // cache heads, Query heads per cache head
  int32_t page_log2;
  int64_t num_pages;
  const void* pages;
  const __half* scales;                  // of the rows of 8-bit pages; null: 16-bit pages
  int32_t block, window, sinks;
  float scale;
  int32_t* status;
  uint64_t wait_ns;
  int32_t idle;                          // nonzero: the producers load nothing (test hook)
  // split along the keys.  chunk: at most nsplit parts of a group, of at least
  // min_tiles tiles; step: nsplit CTAs share the line of all tiles, at least
  // min_tiles places each.  nsplit 1: no split
  int32_t nsplit, min_tiles;
  int32_t wide, blocks;                  // step: tiles of 256 keys; blocks of 8 rows of a head (1: one, of all)
  int32_t whole, rtiles;                 // chunk: >= 0: groups in one line, of which so many first ones are not cut;
                                         // row tiles of a sequence and head
  float* part_o;                         // chunk [group][nsplit][D / 4][row][4]; step [CTA][2][row][D]
  float2* part_ml;                       // running (max, sum): chunk [group][nsplit][row], the maximum as the
                                         // power that P is taken against; step [CTA][2][row]
  int32_t* counter;                      // step: [group], zero between calls
};

// Launch shape of an attention call: which kernel, and its split.
struct PagedPlan {
  int32_t step;      // 1: paged_step.cu, 0: paged_chunk.cu
  int32_t groups;    // (sequence, head, row tile) triples of the grid
  int32_t rows;      // rows of a group
  int32_t nsplit, min_tiles;
  int32_t whole;     // chunk: groups not cut (-1: none, or all if nsplit is 1)
  int32_t wide;      // step: tiles of 256 keys (8-bit pages of 64 channels)
  int32_t blocks;    // step: blocks of 8 rows that a cache head's rows are taken in (1: all together)
};
PagedPlan plan_step(int B, int Hk, int D, int rows, int64_t max_visible, int nsm, bool split, bool codes);
PagedPlan plan_chunk(int B, int Hk, int D, int64_t rows, int64_t max_visible, int nsm, bool split, bool codes);
cudaError_t launch_paged_step(const PagedArgs& a, const CUtensorMap& map, int D, int dtype, cudaStream_t s);
// (half_map: of 8-bit pages of 128 channels, boxes of 64 of them)
cudaError_t launch_paged_chunk(const PagedArgs& a, const CUtensorMap& map, const CUtensorMap& half_map, int D, int dtype,
                               cudaStream_t s);
// Limit of the waits that let copies and MMAs in flight finish after another
// wait has run out, before a CTA gives up its shared memory and TMEM.
constexpr uint64_t kDrainNs = 1000000000ull;
// cudaFuncSetAttribute once per device for a kernel with dynamic shared memory
// (`done`: the caller's static).
template <class K>
inline cudaError_t allow_smem(K kernel, int bytes, bool (&done)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < 64 && done[dev]) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
  return e;
}
// A launch that may be set up while the kernel before it on the stream still
// runs (programmatic dependent launch).  Every thread of the kernel calls
// grid_begin() before its first access to global memory: it waits for that
// kernel's end, then lets the next one be set up.  Back to back this hides the
// launch and the start of a CTA, 1 to 2 us of a short step's 5 to 12.
// `cluster`: CTAs of a cluster, along x.
template <class... P, class... A>
inline cudaError_t launch_ahead(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, int cluster,
                                A&&... args) {
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}
// Rows (Query tokens x Query heads per cache head) up to which a sequence goes
// to the step kernel.  With 16 rows of 128 channels it takes 67 us against the
// chunk kernel's 77 (one sequence of 131071 tokens, 4 cache heads), 20 against 16
// (4000 tokens); a step kernel with a second tile of 16 rows lost on nearly every
// length (24 rows: 88 against 79 us and 27 against 16).
constexpr int kStepRows = 16;
// (Over codes step_blocks() says how many blocks of rows the step kernel takes, 0: none.)
int step_blocks(int B, int Hk, int D, int64_t rows, int64_t max_visible, int nsm, bool codes);

// Pages as rows of D channels, [num_pages * 2 * heads][page_tokens][D]: boxes of
// 64 channels x min(page_tokens, 64) tokens, 128-byte swizzle.
bool make_page_map(CUtensorMap* m, const void* pages, int64_t blocks, int page_tokens, int D, int dtype);
// The same of 8-bit pages: boxes of `width` (64 or 128) codes x min(page_tokens, 64) tokens,
// swizzled by that many bytes.
bool make_code_map(CUtensorMap* m, const void* pages, int64_t blocks, int page_tokens, int D, int width);

// ------------------------------------------------------------ device helpers
#ifdef __CUDACC__

// See launch_ahead.
__device__ __forceinline__ void grid_begin() {
  asm volatile("griddepcontrol.wait;\n\tgriddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ void record_status(int32_t* status, int code) {
  if (status) atomicCAS(status, 0, code);
}

// The row of a token's first Key in the pages, as ((page * 2) * heads) * page_tokens + slot,
// < 0: nowhere.  Row n of the call belongs to the last sequence that begins at or before it.
template <class A>
__device__ __forceinline__ int64_t place_of(const A& a, int64_t n) {
  int lo = 0, hi = a.B;                            // last b with q_off[b] <= n
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (a.q_off[m] <= n) lo = m; else hi = m;
  }
  const int64_t q0 = a.q_off[lo], q1 = a.q_off[lo + 1], kv = a.kv_len[lo];
  int64_t cap = (int64_t)a.table_stride << a.page_log2;
  if (cap > a.max_kv) cap = a.max_kv;
  if (!(n >= q0 && n < q1 && q1 <= a.N && q1 - q0 <= a.max_q && kv >= 0 && kv <= cap)) {
    record_status(a.status, QWM_ERR_INVALID_ARG);
    return -1;
  }
  const int64_t p = kv - q1 + n;
  if (p < 0) return -1;
  const int64_t page = a.table[(int64_t)lo * a.table_stride + (p >> a.page_log2)];
  if (page < 0 || page >= a.num_pages) {
    record_status(a.status, QWM_ERR_INVALID_ARG);
    return -1;
  }
  return ((page * 2 * a.kv_heads) << a.page_log2) + (p & ((1 << a.page_log2) - 1));
}

// Sequence b of the batch: its rows [q0, q0 + qn) and length kv, held to the
// ranges that the tensors and the page table have.  False: something was out, or the
// first sequence does not start at row 0 or the last one not end at N, so that rows are
// left out (their sequences are as good as ever).
struct Seq {
  int64_t q0;
  int32_t qn, kv;
};
template <class A>
__device__ __forceinline__ bool load_seq(const A& a, int b, Seq& s) {
  const int64_t q0 = a.q_off[b], q1 = a.q_off[b + 1];
  const int64_t kv = a.kv_len[b];
  int64_t cap = (int64_t)a.table_stride << a.page_log2;
  if (cap > a.max_kv) cap = a.max_kv;
  const bool ok = q0 >= 0 && q1 >= q0 && q1 <= a.N && q1 - q0 <= a.max_q && kv >= 0 && kv <= cap;
  s.q0 = ok ? q0 : 0;
  s.qn = ok ? (int32_t)(q1 - q0) : 0;
  s.kv = ok ? (int32_t)kv : 0;
  const int64_t left = (b == 0 ? q0 : 0) | (b == a.B - 1 ? a.N - q1 : 0);   // rows left out
  return ok && left == 0;
}

// The tokens a Query at token p sees: [0, min(sinks, hi)) and [lo, hi).
struct Span {
  int32_t lo, hi;
};
__device__ __forceinline__ Span row_span(int p, int kv, int block, int window) {
  Span r{0, 0};
  if (p < 0) return r;
  const int64_t e = ((int64_t)(p / block) + 1) * block;
  r.hi = (int)(e < kv ? e : kv);
  const int64_t lo = window > 0 ? e - window : 0;
  r.lo = lo < 0 ? 0 : (lo > r.hi ? r.hi : (int)lo);
  return r;
}

// What the rows of tokens p0 <= p <= p1 of a sequence see together, as a list
// of tiles of TK keys: the window's from its second tile on, its first tile (cut
// by the rows' windows), then tiles that hold first tokens before it (few keys).
// The first tile taken gives the running maxima their start, so it is one that
// the rows see whole where there is such a tile.  lo and hi of a row grow with its token, so the first and the last row bound
// all.
struct Tiles {
  int32_t lo_min, lo_max, hi_min, hi_max;  // over the rows; a row with p < 0 has hi = 0
  int32_t n_win, w_start, n;
};
template <int TK>
__device__ __forceinline__ Tiles make_tiles(int p0, int p1, int kv, int block, int window, int sinks) {
  Tiles t;
  const Span a = row_span(p0 < 0 ? 0 : p0, kv, block, window), b = row_span(p1, kv, block, window);
  t.lo_min = a.lo;
  t.hi_min = p0 < 0 ? 0 : a.hi;
  t.lo_max = b.lo;
  t.hi_max = b.hi;
  const int s_end = min(min(sinks, t.lo_min), t.hi_max);
  const int n_first = (s_end + TK - 1) / TK;
  t.w_start = max(t.lo_min / TK, n_first);
  t.n_win = max(0, (t.hi_max + TK - 1) / TK - t.w_start);
  t.n = t.hi_max == 0 ? 0 : t.n_win + n_first;
  return t;
}
__device__ __forceinline__ int tile_at(const Tiles& t, int i) {
  return i < t.n_win ? t.w_start + (i + 1 < t.n_win ? i + 1 : 0) : i - t.n_win;
}
__device__ __forceinline__ bool sees(int j, int lo, int hi, int sinks) { return j < hi && (j >= lo || j < sinks); }
// Whether some row of the tiles sees a token of [j0, j1).
__device__ __forceinline__ bool any_sees(const Tiles& t, int j0, int j1, int sinks) {
  return j0 < t.hi_max && (j1 > t.lo_min || j0 < sinks);
}
// Whether every row sees every token of [j0, j1).
__device__ __forceinline__ bool all_see(const Tiles& t, int j0, int j1, int sinks) {
  return j1 <= t.hi_min && (j0 >= t.lo_max || j1 <= sinks);
}

__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The two element types.
template <typename T>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
  static constexpr bool bf16 = true;
  static constexpr uint32_t kExp = 0x7F80u;  // exponent field: all ones in infinities and NaN
  // How far (as a power of two) P may grow before it is taken against a new maximum,
  // and the power below 1 that the largest P of a new maximum has.  P, l and O are
  // floating-point multiples of the same power, so only the types' ranges bound the
  // two.  Together they are 0: P never passes 1, and O holds every Value that an
  // ordinary sum holds (with P from 1 to 2^40 Values of 2^100 became infinite).  The
  // price is at the other end, where Values below 2^-86 leave fp32's normal range.
  // Less room costs time: 2^14 takes 66.2 us where 2^40 takes 63.3 (880 Queries x 12
  // heads over 17600 keys), 2^6 86.9.
  static constexpr int kTau = 40, kBias = 40;
  __device__ static __forceinline__ uint32_t pack(float a, float b) { return ptx::pack_bf16(a, b); }
  __device__ static __forceinline__ float2 unpack(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  }
  __device__ static __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <>
struct Elem<__half> {
  static constexpr bool bf16 = false;
  static constexpr uint32_t kExp = 0x7C00u;
  static constexpr int kTau = 14, kBias = 0;  // P at most 65504; O has fp32's range above that
  __device__ static __forceinline__ uint32_t pack(float a, float b) { return ptx::pack_f16(a, b); }
  __device__ static __forceinline__ float2 unpack(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  }
  __device__ static __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
// ------------------------------------------------------------ 8-bit storage
// A row (token, head) of 8-bit pages stands for code x scale: e4m3 codes and a binary16
// power of two 2^e, -15 <= e <= 8, so that every product is a binary16 (and a bf16) number:
// codes are multiples of 2^-9 and binary16 of 2^-24, and 240 x 2^8 is the largest e4m3
// multiple of a power of two below 65504.
constexpr float kCodeMost = 61440.0f;

// The scale's biased exponent for a row whose largest magnitude is `most` <= kCodeMost: the
// least e >= -15 with most <= 448 x 2^e (448 = 1.75 x 2^8: a mantissa above 0.75 carries).
__device__ __forceinline__ uint32_t code_exponent(float most) {
  const int e = (int)((__float_as_uint(most) + 0x1FFFFFu) >> 23) - 8;
  return (uint32_t)max(e, 127 - 15);
}
// 2^e (and 2^-e) of a biased exponent 112 <= e <= 135
__device__ __forceinline__ __half code_scale(uint32_t e) { return __float2half_rn(__uint_as_float(e << 23)); }
__device__ __forceinline__ float code_inverse(uint32_t e) { return __uint_as_float((254u - e) << 23); }

// Four values (already divided by their scale) as codes, the first in the low byte.
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
  uint32_t w;
  asm("{\n\t.reg .b16 l, h;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\t"
      "mov.b32 %0, {l, h};\n\t}"
      : "=r"(w)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return w;
}
// Four codes as two pairs of binary16 numbers (exact; a NaN code gives NaN).
__device__ __forceinline__ void from_codes(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\t"
      "mov.b32 {l, h}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, l;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// The type that products over the pages are taken in.
template <typename T, bool C8>
struct OperandOf {
  using type = T;
};
template <typename T>
struct OperandOf<T, true> {
  using type = __half;
};
template <typename T, bool C8>
using Operand = typename OperandOf<T, C8>::type;

// bf16 Queries as binary16: a row is taken times the power of two that brings its largest
// finite magnitude to [2^14, 2^15) (2^127 at the most), and its logits' scale by the inverse.
// Exact but for elements 2^-29 and less of the largest, which round to a multiple of 2^-39 of
// it (rows below 2^-113: of 2^-152).
// The largest magnitude's bits of eight elements, infinities and NaN left out.
__device__ __forceinline__ uint32_t finite_max(uint4 v) {
  const uint32_t w[4] = {v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu, v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu};
  const uint32_t both = ptx::vmax_u16x2(ptx::vmax_u16x2(w[0], w[1]), ptx::vmax_u16x2(w[2], w[3]));
  uint32_t top = max(both & 0xFFFFu, both >> 16);
  if (top >= 0x7F80u) {
    top = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t lo = w[k] & 0x7FFFu, hi = w[k] >> 16;
      top = max(top, max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u));
    }
  }
  return top;
}
__device__ __forceinline__ int row_power(uint32_t top) { return min(14 + 127 - (int)(top >> 7), 127); }   // -113 .. 127
// x 2^up in two steps, each a normal number
__device__ __forceinline__ float times_pow2(float x, int up) {
  const int h = up >> 1;
  return x * __uint_as_float((uint32_t)(127 + h) << 23) * __uint_as_float((uint32_t)(127 + up - h) << 23);
}
__device__ __forceinline__ uint32_t scaled_f16(uint32_t w, int up) {
  const float2 f = Elem<__nv_bfloat16>::unpack(w);
  const float s = __uint_as_float((uint32_t)(127 + up) << 23);
  return Elem<__half>::pack(f.x * s, f.y * s);
}
__device__ __forceinline__ uint4 scaled_f16(uint4 v, int up) {
  return make_uint4(scaled_f16(v.x, up), scaled_f16(v.y, up), scaled_f16(v.z, up), scaled_f16(v.w, up));
}
// The scale of a row's logits, normal and finite (0 x inf and inf x 0 are not 0)
__device__ __forceinline__ float row_scale(float sl2, int up) {
  return fminf(fmaxf(times_pow2(sl2, -up), 1.2e-38f), 1.0e38f);
}

// Whether a word of two elements holds an infinity or a NaN.
template <typename T>
__device__ __forceinline__ bool nonfinite2(uint32_t w) {
  const uint32_t lo = w & Elem<T>::kExp, hi = (w >> 16) & Elem<T>::kExp;
  return lo == Elem<T>::kExp || hi == Elem<T>::kExp;
}

#endif  // __CUDACC__

}  // namespace qwm
