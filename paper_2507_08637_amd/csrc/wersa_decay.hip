// Causal linear attention with a decay for each head: per (sequence, head)
//   S_t = lambda S_{t-1} + k_t v_t^T  (dk x dv),   o_t = scale q_t^T S_t,   lambda = exp(log_decay[h])
//
// Whole sequences go in chunks of 64 rows.  With D_ts = lambda^(t-s) for s <= t, else 0, and S the state before the chunk
//   O  = (scale (Q K^T) o D) V + scale diag(lambda^(t+1)) Q S,     S' = lambda^64 S + (K o lambda^(63-s))^T V
// A workgroup walks the chunks of one segment of a sequence with S in registers.  Where (sequence, head) pairs alone do not
// fill the device, sequences are split into segments: one launch forms what every segment adds to the state, one
// adds these up to the states that the segments begin with, and the walk starts everywhere at once.
//
// The derivative is three more walks.  With G_t = dL/dS_t, G_t = lambda G_{t+1} + scale q_t do_t^T:
//   dq_t = scale S_t do_t     the walk with (do, v, k) in the place of (q, k, v)
//   dk_t = G_t v_t            the walk from the last row to the first, with (v, do, q)
//   dv_t = G_t^T k_t          the same with (k, q, do)
// The walk back multiplies with lambda after a row where the walk forward does before it: `shift` below.
#include "wersa_internal.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace wersa {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 64;

// lambda^e for e >= 0.  The clamp keeps 0 * log_decay apart from 0 * inf: a decay of zero (log_decay = -inf) leaves lambda^0 = 1.
__device__ __forceinline__ float log2_decay(const float *log_decay, int h) { return (log_decay[h] < -1e4f ? -1e4f : log_decay[h]) * 1.44269504f; }
__device__ __forceinline__ float decay_pow(float l2, int e) { return exp2f(l2 * (float)e); }

struct Strides {
  int64_t b, h, n;
};

// The rows of one sequence, and of one segment of it.  Packed sequences lie in rows offsets[b] .. offsets[b + 1] of one tensor.  Segment s of
// sequence b has slot floor(begin / seg) + b + s: the slots of a sequence lie behind those of the one before it whatever the lengths are, so that the grid
// is known without them; some slots stay empty.  Offsets are clamped into the tensor: no value of theirs leads out of it.
struct Sequences {
  const int32_t *offsets;   // null: B sequences of n rows each
  int B, n, seg, segs;      // segs: segments of a sequence that is not packed
  __host__ __device__ int slots() const { return offsets ? n / seg + B : B * segs; }
  __device__ __forceinline__ int begin(int b) const { return offsets ? min(max(offsets[b], 0), n) : 0; }
  __device__ __forceinline__ int rows(int b) const { return offsets ? max(min(offsets[b + 1], n) - begin(b), 0) : n; }
  __device__ __forceinline__ int first_slot(int b) const { return offsets ? begin(b) / seg + b : b * segs; }
  __device__ __forceinline__ int segments(int b) const { return offsets ? max(1, (rows(b) + seg - 1) / seg) : segs; }
};
struct Segment {
  int b, s, rows;           // rows == -1: nothing here
  int64_t row0;
};
__device__ __forceinline__ Segment segment_of(const Sequences &q, int slot) {
  Segment r;
  if (!q.offsets) {
    r.b = slot / q.segs;
    r.s = slot % q.segs;
  } else {
    int lo = 0, hi = q.B - 1;   // the last sequence that does not begin behind this slot
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (q.first_slot(mid) <= slot) lo = mid; else hi = mid - 1;
    }
    r.b = lo;
    r.s = slot - q.first_slot(lo);
  }
  const int have = q.rows(r.b);
  r.row0 = (int64_t)q.begin(r.b) + (int64_t)r.s * q.seg;
  r.rows = r.s < 0 || r.s >= q.segments(r.b) ? -1 : min(q.seg, have - r.s * q.seg);
  return r;
}

struct Walk {
  const void *q, *k, *v;
  void *o;
  Strides sq, sk, sv, so;
  const float *log_decay;
  const float *init;        // states that the walk begins with: by slot (by_slot) or by sequence; null: zeros
  float *fin;               // states that it ends with, by sequence (or local sums by slot: STATES)
  const int32_t *cache;     // rows of init and fin (by sequence) that the sequences have, null: sequence b has row b
  int cache_rows;
  Sequences seq;
  int H, kw, vw;            // widths of k and v
  int64_t si, sj;           // strides of a state's rows (k) and columns (v)
  float intra, inter, gain; // factors of the chunk's products, of the state's part and of what goes into the state
  bool by_slot, reverse;
  bool heads_first;         // the grid's order
};

// Heads that lie side by side in memory go side by side through the grid.
__device__ __forceinline__ int slot_of(const Walk &a) { return a.heads_first ? blockIdx.y : blockIdx.x; }
__device__ __forceinline__ int head_of(const Walk &a) { return a.heads_first ? blockIdx.x : blockIdx.y; }

__device__ __forceinline__ int cache_row(const Walk &a, int b) {   // -1: none
  const int r = a.cache ? a.cache[b] : b;
  return r < 0 || r >= a.cache_rows ? -1 : r;
}

// The rows of a segment in one tensor, chunk by chunk in the walk's order, as buffers that end at the last row: loads of rows that are not there, or
// of columns past the width, return zeros, stores to them do nothing, by the bounds check of the buffer instructions.
constexpr int64_t kMostRowStride = 1 << 24;   // elements: 63 rows of 4 bytes stay below 2^32
typedef __amdgpu_buffer_rsrc_t Buffer;
struct Rows {
  const char *low;    // of the segment's rows, the first in memory
  uint32_t step;      // bytes from row to row
  int width;          // bytes of a row
  int rows;
  bool reverse;
  struct Chunk {
    Buffer b;
    uint32_t missing; // the walk back: bytes by which a partial chunk's rows lie lower
  };
  __device__ __forceinline__ Chunk chunk(int r0) const {
    const int have = max(0, min(kChunk, rows - r0));
    const uint64_t p = (uint64_t)low + (uint64_t)(uint32_t)(reverse ? rows - r0 - have : r0) * step;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)p), hi = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32));
    const uint32_t bytes = __builtin_amdgcn_readfirstlane(have ? (uint32_t)(have - 1) * step + width : 0);
    return Chunk{__builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)hi << 32 | lo), 0, (int)bytes, 0x00020000),
                 reverse ? (uint32_t)(kChunk - have) * step : 0};
  }
  // Of a byte of a row of a chunk; `rows` further on in the chunk.
  __device__ __forceinline__ uint32_t offset(int row, int byte) const { return (uint32_t)(reverse ? kChunk - 1 - row : row) * step + byte; }
  __device__ __forceinline__ uint32_t further(int rows) const { return (uint32_t)(reverse ? -rows : rows) * step; }
};
// Bytes past the width are none of the buffer's: joined in by `or` at the access.
__device__ __forceinline__ uint32_t outside(int byte, int width) { return byte < width ? 0u : 0xffffffc0u; }
// Aux 2: non-temporal, by the caches, which keep what comes after.
template <bool NT> __device__ __forceinline__ u32x4 load_piece(const Rows::Chunk &c, uint32_t at) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(c.b, (int)at, 0, NT ? 2 : 0));
}
__device__ __forceinline__ void store_piece(const Rows::Chunk &c, uint32_t at, u32x4 v) { __builtin_amdgcn_raw_buffer_store_b128(v, c.b, (int)at, 0, 2); }
// Rows of `seg` for head h of a tensor.
__device__ __forceinline__ Rows rows_of(const void *p, const Strides &s, const Segment &seg, const Walk &a, int h, int cols, int element) {
  const int64_t at = (a.seq.offsets ? 0 : seg.b * s.b) + h * s.h + seg.row0 * s.n;
  return Rows{(const char *)p + at * element, (uint32_t)(s.n * element), cols * element, seg.rows, a.reverse};
}
// The same value, of which the compiler knows nothing: what follows from it is formed where it is used, not kept in registers around a loop.
__device__ __forceinline__ uint32_t opaque(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}
// A thread's pieces of a tile of D values a row of E per piece, PIECES of them: THREADS threads take whole rows one behind the other from `row0` on.  FULL: no columns past the
// width.
template <int D, int E, int PIECES, int THREADS, bool FULL> struct TilePieces {
  uint32_t at, out;
  __device__ __forceinline__ TilePieces(const Rows &r, int row0, int t) : at(r.offset(row0 + t / (D / E), t % (D / E) * 16)), out(outside(t % (D / E) * 16, r.width)) {}
  template <bool NT> __device__ __forceinline__ void load(const Rows &r, int r0, u32x4 (&p)[PIECES]) const {
    const Rows::Chunk c = r.chunk(r0);
    uint32_t x = opaque(at) - c.missing;
#pragma unroll
    for (int i = 0; i < PIECES; ++i, x += r.further(THREADS * E / D)) p[i] = load_piece<NT>(c, FULL ? x : x | out);
  }
  __device__ __forceinline__ void store(const Rows &r, int r0, const u32x4 (&p)[PIECES]) const {
    const Rows::Chunk c = r.chunk(r0);
    uint32_t x = opaque(at) - c.missing;
#pragma unroll
    for (int i = 0; i < PIECES; ++i, x += r.further(THREADS * E / D)) store_piece(c, FULL ? x : x | out, p[i]);
  }
};

// ---- float32 matrix instructions -----------------------------------------------------------------
// v_mfma_f32_16x16x4_f32 (c = lane % 16, g = lane / 16): A row c, k = g;  B column c, k = g;  C/D: acc[i] is row 4 g + i, column c.
// Four of them take k = 4 g + i of a 16-wide slice: four consecutive values per lane.
__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// A wave's part of a chunk's work and of the state.  Rows 16 t .. of the chunk: the weights of a later tile have more rows to them, so that which wave has which goes by the
// workgroup (all first waves of a compute unit's workgroups share a SIMD).  Of the state RT row tiles from row0 on and CW column tiles from col0 on: at width 32 a wave has one
// row tile and half of the columns; with eight waves two of them share rows and rows of the state, and each has half of the columns, of the outputs too.
template <int DK, int DV, int WAVES = 4> struct Part {
  static constexpr int HALVES = WAVES / 4, RT = DK < 64 ? 1 : DK / 64, CT = DV / 16, CW = DK < 64 ? CT / 2 : CT / HALVES;
  int t, half, row0, col0;
  __device__ __forceinline__ Part(int wave)
      : t((wave + blockIdx.x + blockIdx.y) & 3), half(wave >> 2), row0(DK < 64 ? 16 * (wave & 1) : DK / 4 * (wave & 3)),
        col0(DK < 64 ? DV / 2 * (wave >> 1) : DV / HALVES * half) {}
};
// Products of a wave's 16 own rows (four consecutive values of a row in a lane) with rows 16 jt .. of the chunk in LDS.
template <int D> __device__ __forceinline__ f32x4 products_f32(const float *rows, int jt, const f32x4 (&own)[D / 16], int g, int c) {
  f32x4 p = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < D / 16; ++j) {
    const f32x4 s = *(const f32x4 *)(rows + (16 * jt + c) * (D + 4) + 16 * j + 4 * g);
#pragma unroll
    for (int i = 0; i < 4; ++i) p = mfma_f32(s[i], own[j][i], p);
  }
  return p;
}
// The own 16 rows of a tensor in that layout.
template <int D> __device__ __forceinline__ void load_own_f32(const Rows &r, int r0, uint32_t at, int g, f32x4 (&own)[D / 16]) {
  const Rows::Chunk c = r.chunk(r0);
#pragma unroll
  for (int j = 0; j < D / 16; ++j) own[j] = __builtin_bit_cast(f32x4, load_piece<false>(c, (at + 64 * j - c.missing) | outside(64 * j + 16 * g, r.width)));
}
template <int D, int THREADS, int PIECES> __device__ __forceinline__ void put_tile_f32(float *rows, int tid, const u32x4 (&p)[PIECES]) {
#pragma unroll
  for (int i = 0; i < PIECES; ++i) *(u32x4 *)(rows + (tid / (D / 4) + 4 * THREADS / D * i) * (D + 4) + tid % (D / 4) * 4) = p[i];
}
template <typename P, int RT, int CW, typename F>
__device__ __forceinline__ void each_of_state(const Walk &a, f32x4 (&S)[RT][CW], const P &part, int g, int lane_c, F f) {
  const int c = (int)opaque((uint32_t)lane_c);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int ct = 0; ct < CW; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = part.row0 + 16 * rt + 4 * g + i, col = part.col0 + 16 * ct + c;
        S[rt][ct][i] = f(S[rt][ct][i], r < a.kw && col < a.vw, r * a.si + col * a.sj);
      }
}
// Of the weights of own rows 16 t + c against rows 16 jt + 4 g + i of the chunk: lambda to the distance; the rest of the row is masked.
struct WeightsF32 {
  float on[4], before[4], apart[3], reach;
  int t, ahead;
  __device__ __forceinline__ WeightsF32(const Walk &a, float l2, int t, int g, int c) : t(t), ahead(c - 4 * g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      on[i] = ahead >= i ? a.intra * decay_pow(l2, ahead - i) : 0.f;
      before[i] = a.intra * decay_pow(l2, 16 + ahead - i);
    }
#pragma unroll
    for (int jt = 0; jt < 3; ++jt) apart[jt] = decay_pow(l2, 16 * max(t - jt - 1, 0));
    reach = a.inter * decay_pow(l2, 16 * t + c + (a.reverse ? 0 : 1));
  }
  __device__ __forceinline__ f32x4 operator()(f32x4 p, int jt) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = jt < t ? p[i] * before[i] * (jt == 0 ? apart[0] : jt == 1 ? apart[1] : apart[2]) : ahead >= i ? p[i] * on[i] : 0.f;
    return p;
  }
};
// Columns 16 ct + c of rows 16 jt + 4 g + i of the chunk in LDS, rows of D values.
template <int D, int TILES> __device__ __forceinline__ void columns_f32(const float *rows, int jt, int g, int c, float (&v)[TILES][4]) {
#pragma unroll
  for (int ct = 0; ct < TILES; ++ct)
#pragma unroll
    for (int i = 0; i < 4; ++i) v[ct][i] = rows[(16 * jt + 4 * g + i) * (D + 4) + 16 * ct + c];
}
// S <- keep S + (K o weight)^T V over the chunk's rows.
template <int DK, int DV, typename P, int RT, int CW>
__device__ __forceinline__ void update_state_f32(const P &part, f32x4 (&S)[RT][CW], float keep, const float *Ks, const float *Vs, const float *weight, int g, int c) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int ct = 0; ct < CW; ++ct) S[rt][ct] *= keep;
#pragma unroll
  for (int jt = 0; jt < 4; ++jt) {
    const f32x4 wt = *(const f32x4 *)(weight + 16 * jt + 4 * g);
    float V[CW][4];
    columns_f32<DV>(Vs + part.col0, jt, g, c, V);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float kt = Ks[(16 * jt + 4 * g + i) * (DK + 4) + part.row0 + 16 * rt + c] * wt[i];
#pragma unroll
        for (int ct = 0; ct < CW; ++ct) S[rt][ct] = mfma_f32(kt, V[ct][i], S[rt][ct]);
      }
  }
}

// The output of a wave's 16 own rows: what the state gives (`inter`, a tile of columns at a time) and the weighted rows of the chunk, `weight` their weights for rows 16 jt ..
// A weight that is masked is a zero, and in a product of matrices a zero times what is not a number or not finite is not a number: rows that come later would reach back.  So results that
// are not finite are formed again, with such values left out; where none of a row's own reach is among them, that is the result.
// D / HALVES columns of the output, from `col` on.
template <int D, int HALVES, typename Inter, typename Weight>
__device__ __forceinline__ void weighted_rows_f32(const float *rows, const Rows &out, int r0, uint32_t at, int col, int t, int g, int c, Inter inter, Weight weight) {
  constexpr int TILES = D / 16 / HALVES;
  float probe = 0.f;
  const Rows::Chunk oc = out.chunk(r0);
  auto store = [&](int ct, f32x4 x) {
    store_piece(oc, (at + 4 * col + 64 * ct - oc.missing) | outside(4 * col + 64 * ct + 16 * g, out.width), __builtin_bit_cast(u32x4, x));
  };
  {
    f32x4 O[TILES];
#pragma unroll
    for (int ct = 0; ct < TILES; ++ct) O[ct] = inter(ct);
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      if (jt > t) break;
      float V[TILES][4];
      columns_f32<D>(rows + col, jt, g, c, V);
      const f32x4 P = weight(jt);
#pragma unroll
      for (int ct = 0; ct < TILES; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) O[ct] = mfma_f32(V[ct][i], P[i], O[ct]);
    }
#pragma unroll
    for (int ct = 0; ct < TILES; ++ct) {
#pragma unroll
      for (int i = 0; i < 4; ++i) probe = fmaf(O[ct][i], 0.f, probe);   // not a number if one is not finite
      store(ct, O[ct]);
    }
  }
  if (!__any(!(probe == 0.f))) return;
#pragma unroll 1
  for (int ct = 0; ct < TILES; ++ct) {
    f32x4 all = inter(ct), finite = all, met = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int jt = 0; jt <= t; ++jt) {
      const f32x4 P = weight(jt);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = rows[(16 * jt + 4 * g + i) * (D + 4) + col + 16 * ct + c];
        const bool fine = fabsf(v) < __builtin_inff();
        all = mfma_f32(v, P[i], all);
        finite = mfma_f32(fine ? v : 0.f, P[i], finite);
        met = mfma_f32(fine ? 0.f : 1.f, 16 * jt + 4 * g + i <= 16 * t + c ? 1.f : 0.f, met);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) all[i] = met[i] > 0.f ? all[i] : finite[i];
    store(ct, all);
  }
}

// Weights are formed as their transpose (the chunk's rows down the registers, own rows on the lanes), which is the layout that the product with V takes them in.
// Eight waves at width 128, where LDS holds one workgroup to a compute unit: two to a SIMD, which form their rows' weights twice.
// Up to width 32 near memory (128 slices of 4000 rows: 64 us, 4.1 TB/s), above by the matrix units: 32 slices of 8192 rows, width 64, 86 us, 3.1 TB/s; 16 slices, width 128, 136 us, 2.0 TB/s,
// about 92 of the 157 TFLOP/s that float32 matrix instructions have at their nominal clock.
constexpr int f32_waves(int dk, int dv) { return dk > 64 || dv > 64 ? 8 : 4; }
template <int DK, int DV, bool STATES>
__global__ __launch_bounds__(64 * f32_waves(DK, DV)) void walk_f32_kernel(Walk a) {
  constexpr int WAVES = f32_waves(DK, DV), THREADS = 64 * WAVES, LK = DK + 4, LV = DV + 4, PK = kChunk * DK / 4 / THREADS, PV = kChunk * DV / 4 / THREADS;   // pieces of a thread
  typedef Part<DK, DV, WAVES> P4;
  extern __shared__ __align__(16) float lds[];
  float *Ks = lds, *Vs = Ks + kChunk * LK, *weight = Vs + kChunk * LV, *St = weight + kChunk;
  const int slot = slot_of(a), h = head_of(a);
  const Segment seg = segment_of(a.seq, slot);
  if (seg.rows < 0) return;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  const bool last = a.reverse ? seg.s == 0 : seg.s == a.seq.segments(seg.b) - 1;
  if (STATES && last) return;   // nothing begins with what the last one adds
  const P4 part(wave);
  const int col = DV / P4::HALVES * part.half;   // of the outputs
  const Rows qr = rows_of(a.q, a.sq, seg, a, h, a.kw, 4), kr = rows_of(a.k, a.sk, seg, a, h, a.kw, 4), vr = rows_of(a.v, a.sv, seg, a, h, a.vw, 4),
             orow = rows_of(a.o, a.so, seg, a, h, a.vw, 4);
  const float l2 = log2_decay(a.log_decay, h);
  const int64_t state_size = (int64_t)a.kw * a.vw;

  f32x4 S[P4::RT][P4::CW];   // S[rt][ct][i] is row row0 + 16 rt + 4 g + i, column col0 + 16 ct + c
  const int own = cache_row(a, seg.b);
  const int64_t from = a.by_slot ? (int64_t)slot : own;
  const float *init = STATES || !a.init || from < 0 ? nullptr : a.init + (from * a.H + h) * state_size;
  each_of_state(a, S, part, g, c, [&](float, bool there, int64_t at) { return init && there ? init[at] : 0.f; });
  const WeightsF32 weights(a, l2, part.t, g, c);

  u32x4 rk[PK], rv[PV];
  f32x4 rq[DK / 16];
  const TilePieces<DK, 4, PK, THREADS, false> kp(kr, 0, tid);
  const TilePieces<DV, 4, PV, THREADS, false> vp(vr, 0, tid);
  const uint32_t qat = qr.offset(16 * part.t + c, 16 * g), oat = orow.offset(16 * part.t + c, 16 * g);
  auto request = [&](int r0) {
    kp.template load<false>(kr, r0, rk);
    vp.template load<false>(vr, r0, rv);
    if (!STATES) load_own_f32<DK>(qr, r0, qat, g, rq);
  };

  request(0);
  for (int r0 = 0; r0 < seg.rows; r0 += kChunk) {
    const int rows = min(kChunk, seg.rows - r0);
    // what was requested, and the state, into LDS
    put_tile_f32<DK, THREADS>(Ks, tid, rk);
    put_tile_f32<DV, THREADS>(Vs, tid, rv);
    if (tid < kChunk) weight[tid] = a.gain * decay_pow(l2, max(rows - 1 - tid, 0) + (a.reverse ? 1 : 0));
    f32x4 Q[DK / 16];
    if (!STATES) {
#pragma unroll
      for (int j = 0; j < DK / 16; ++j) Q[j] = rq[j];
#pragma unroll
      for (int rt = 0; rt < P4::RT; ++rt)
#pragma unroll
        for (int ct = 0; ct < P4::CW; ++ct) *(f32x4 *)(St + (part.col0 + 16 * ct + c) * LK + part.row0 + 16 * rt + 4 * g) = S[rt][ct];
    }
    __syncthreads();
    request(r0 + kChunk);
    if (!STATES)
      weighted_rows_f32<DV, P4::HALVES>(Vs, orow, r0, oat, col, part.t, g, c,
                                        [&](int ct) { return products_f32<DK>(St + col * LK, ct, Q, g, c) * weights.reach; },
                                        [&](int jt) { return weights(products_f32<DK>(Ks, jt, Q, g, c), jt); });
    update_state_f32<DK, DV>(part, S, decay_pow(l2, rows), Ks, Vs, weight, g, c);
    __syncthreads();
  }

  float *fin = nullptr;
  if (STATES) fin = a.fin + ((int64_t)slot * a.H + h) * state_size;
  else if (last && a.fin && own >= 0) fin = a.fin + ((int64_t)own * a.H + h) * state_size;
  if (fin) each_of_state(a, S, part, g, c, [&](float x, bool there, int64_t at) { if (there) fin[at] = x; return x; });
}

// The two walks back of the derivative as one, k and v of `a` being q and dout: own rows of keys and values, G^T k and the weighted rows of dout give dv, G v and the
// weighted rows of q give dk.  Reads four tensors and writes two, where two walks read three and write one each, and forms G once.
struct Back {
  const void *k, *v;
  void *dk, *dv;
  Strides sk, sv, sdk, sdv;
};
template <int DK, int DV>
__global__ __launch_bounds__(64 * f32_waves(DK, DV)) void back_f32_kernel(Walk a, Back b) {
  constexpr int WAVES = f32_waves(DK, DV), THREADS = 64 * WAVES, LK = DK + 4, LV = DV + 4, PK = kChunk * DK / 4 / THREADS, PV = kChunk * DV / 4 / THREADS;
  typedef Part<DK, DV, WAVES> P4;
  constexpr int KT = DK / 16, CT = P4::CT;
  extern __shared__ __align__(16) float lds[];
  float *Qs = lds, *Ds = Qs + kChunk * LK, *weight = Ds + kChunk * LV, *Gt = weight + kChunk;
  const int slot = slot_of(a), h = head_of(a);
  const Segment seg = segment_of(a.seq, slot);
  if (seg.rows < 0) return;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  const P4 part(wave);
  const int vcol = DV / P4::HALVES * part.half, kcol = DK / P4::HALVES * part.half;   // of dv and of dk
  const Rows qr = rows_of(a.k, a.sk, seg, a, h, a.kw, 4), dr = rows_of(a.v, a.sv, seg, a, h, a.vw, 4), kr = rows_of(b.k, b.sk, seg, a, h, a.kw, 4),
             vr = rows_of(b.v, b.sv, seg, a, h, a.vw, 4), dkr = rows_of(b.dk, b.sdk, seg, a, h, a.kw, 4), dvr = rows_of(b.dv, b.sdv, seg, a, h, a.vw, 4);
  const float l2 = log2_decay(a.log_decay, h);
  const int64_t state_size = (int64_t)a.kw * a.vw;

  f32x4 G[P4::RT][P4::CW];
  const int64_t from = a.by_slot ? (int64_t)slot : seg.b;
  const float *init = a.init ? a.init + (from * a.H + h) * state_size : nullptr;
  each_of_state(a, G, part, g, c, [&](float, bool there, int64_t at) { return init && there ? init[at] : 0.f; });
  const WeightsF32 weights(a, l2, part.t, g, c);

  u32x4 rq[PK], rd[PV];
  f32x4 K[KT], V[CT];
  const TilePieces<DK, 4, PK, THREADS, false> qp(qr, 0, tid);
  const TilePieces<DV, 4, PV, THREADS, false> dp(dr, 0, tid);
  // Places of own rows are formed where they are used: of four strides, they take registers that width 128 has not (229 us kept, 219 so, 16 slices of 8192 rows).
  auto at_of = [&](const Rows &r) { return r.offset(16 * part.t + (int)opaque((uint32_t)c), 16 * g); };
  auto request = [&](int r0) {
    qp.template load<false>(qr, r0, rq);
    dp.template load<false>(dr, r0, rd);
  };
  auto request_own = [&](int r0) {
    load_own_f32<DK>(kr, r0, at_of(kr), g, K);
    load_own_f32<DV>(vr, r0, at_of(vr), g, V);
  };
  request(0);
  request_own(0);
  for (int r0 = 0; r0 < seg.rows; r0 += kChunk) {
    const int rows = min(kChunk, seg.rows - r0);
    put_tile_f32<DK, THREADS>(Qs, tid, rq);
    put_tile_f32<DV, THREADS>(Ds, tid, rd);
    if (tid < kChunk) weight[tid] = a.gain * decay_pow(l2, max(rows - 1 - tid, 0) + 1);
#pragma unroll
    for (int rt = 0; rt < P4::RT; ++rt)
#pragma unroll
      for (int ct = 0; ct < P4::CW; ++ct) *(f32x4 *)(Gt + (part.col0 + 16 * ct + c) * LK + part.row0 + 16 * rt + 4 * g) = G[rt][ct];
    __syncthreads();
    request(r0 + kChunk);
    weighted_rows_f32<DV, P4::HALVES>(Ds, dvr, r0, at_of(dvr), vcol, part.t, g, c, [&](int ct) { return products_f32<DK>(Gt + vcol * LK, ct, K, g, c) * weights.reach; },
                                      [&](int jt) { return weights(products_f32<DK>(Qs, jt, K, g, c), jt); });
    weighted_rows_f32<DK, P4::HALVES>(Qs, dkr, r0, at_of(dkr), kcol, part.t, g, c, [&](int kt) {   // G v: rows of G down the lanes, its columns four values apart in Gt
      f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < CT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = mfma_f32(Gt[(16 * j + 4 * g + i) * LK + kcol + 16 * kt + c], V[j][i], acc);
      return acc * weights.reach;
    }, [&](int jt) { return weights(products_f32<DV>(Ds, jt, V, g, c), jt); });
    request_own(r0 + kChunk);
    update_state_f32<DK, DV>(part, G, decay_pow(l2, rows), Qs, Ds, weight, g, c);
    __syncthreads();
  }
  if (a.fin && seg.s == 0) {
    float *fin = a.fin + ((int64_t)seg.b * a.H + h) * state_size;
    each_of_state(a, G, part, g, c, [&](float x, bool there, int64_t at) { if (there) fin[at] = x; return x; });
  }
}

// ---- bf16 matrix instructions --------------------------------------------------------------------
// v_mfma_f32_16x16x32_bf16 (c = lane % 16, g = lane / 16): A row c, k = 8 g + q;  B column c, k = 8 g + q;  C/D: acc[i] is row 4 g + i, column c.
// The order of k is free as long as both operands have the same: in products over the chunk's rows, slot q of lane group g is row 4 g + q (q < 4) or
// 16 + 4 g + q - 4 of 32.  That is what two tiles of P leave in a lane's registers, and what two transposing reads bring.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma_bf16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// ds_read_b64_tr_b16: within each group of 16 lanes, lane i passes the address of four consecutive 16-bit values, taken as row i / 4,
// columns 4 (i % 4) .. + 3 of a 4 x 16 block, and receives column i of that block.
__device__ __forceinline__ bf16x8 read_transposed(uint32_t lo, uint32_t hi) {
  typedef __attribute__((address_space(3))) s16x4 *lds_s16x4_ptr;
  const bf16x4 a = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)lo));
  const bf16x4 b = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)hi));
  return bf16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}
// Rows of D values in LDS, their 16-byte pieces permuted by the row so that no read or write meets another in a bank (64 banks of 4 bytes): 16-byte accesses by one
// column of 16 rows, and transposing reads of 32 bytes of 8 rows: rows 4 g + .. of two lane groups, or with NATURAL rows 8 g + ...  Against rows 32 bytes longer
// than the data, at width 128: half of the cycles of LDS were conflicts.  The permutation goes by the row's last four bits and is an exclusive or, so that a lane needs
// one address for all tiles of a kind: other rows are a constant further on, other columns one `or` away.
template <int D, bool NATURAL> __device__ __forceinline__ uint32_t lds_at(int row, int col) {   // in bytes
  int f;
  if (D == 128) f = NATURAL ? (row & 3) << 1 | (row & 8) | (row >> 2 & 1) : (row & 7) << 1 | (row >> 3 & 1);
  else if (D == 32) f = NATURAL ? row >> 2 & 3 : (row >> 1 & 2) | (row >> 3 & 1);
  else f = NATURAL ? (row & 2) | (row & 8) >> 1 | (row >> 2 & 1) : (row & 6) | (row >> 3 & 1);
  return 2 * (row * D + ((col >> 3 ^ f) << 3 | (col & 7)));
}
template <typename V> __device__ __forceinline__ V lds_read(uint32_t at) { return *(__attribute__((address_space(3))) const V *)at; }
template <typename V> __device__ __forceinline__ void lds_write(uint32_t at, V v) { *(__attribute__((address_space(3))) V *)at = v; }
// What a lane reads: the operand with a row of LDS per lane (rows 16 t + c, columns 32 j + 8 g ..), and the transposed one (below).  `lds`: where LDS begins (a multiple of
// 256); `rows`, a tile's place from there, is a constant, and so part of the instruction.
template <int D, bool NATURAL> struct RowOperand {
  uint32_t at;
  __device__ __forceinline__ RowOperand(uint32_t lds, int g, int c) : at(opaque(lds + lds_at<D, NATURAL>(c, 8 * g))) {}
  __device__ __forceinline__ bf16x8 operator()(uint32_t rows, int t, int j) const { return lds_read<bf16x8>((at ^ 64 * j) + (rows + 32 * t * D)); }
};
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
}
// x w as the sum of three bf16 values, 24 bits of it: keys times their weight enter the state like float32.  (The packed values are hidden from the compiler, which
// would round every element a second time to take it apart.)
__device__ __forceinline__ void three_terms(bf16x8 x, f32x4 w0, f32x4 w1, bf16x8 (&t)[3]) {
  const u32x4 p = __builtin_bit_cast(u32x4, x);
  u32x4 q[3];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo = __uint_as_float(p[i] << 16) * (i < 2 ? w0[2 * i] : w1[2 * i - 4]), hi = __uint_as_float(p[i] & 0xffff0000u) * (i < 2 ? w0[2 * i + 1] : w1[2 * i - 3]);
#pragma unroll
    for (int u = 0; u < 3; ++u) {
      uint32_t r = pack2(lo, hi);
      if (u < 2) {
        asm("" : "+v"(r));
        lo -= __uint_as_float(r << 16);
        hi -= __uint_as_float(r & 0xffff0000u);
      }
      q[u][i] = r;
    }
  }
#pragma unroll
  for (int u = 0; u < 3; ++u) t[u] = __builtin_bit_cast(bf16x8, q[u]);
}

// The decays of a wave's part of a chunk's weights: 16 own rows on the lanes, 16 other rows down the registers.  lambda^(c - 4 g - i) on the diagonal tile,
// lambda^(16 + c - 4 g - i) times a power of lambda^16, the same for the whole wave, on those before it.
struct Weights {
  float on[4], before[4], apart[3], reach;
  int w, ahead;   // ahead: c - 4 g
  __device__ __forceinline__ Weights(const Walk &a, float l2, int w, int g, int c) : w(w), ahead(c - 4 * g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      on[i] = ahead >= i ? a.intra * decay_pow(l2, ahead - i) : 0.f;
      before[i] = a.intra * decay_pow(l2, 16 + ahead - i);
    }
#pragma unroll
    for (int jt = 0; jt < 3; ++jt) apart[jt] = decay_pow(l2, 16 * max(w - jt - 1, 0));
    reach = a.inter * decay_pow(l2, 16 * w + c + (a.reverse ? 0 : 1));
  }
  // Products of the own rows `b` with the chunk's rows in LDS, weighted: operands of the products with the other tensor's rows.
  template <int D> __device__ __forceinline__ void products(uint32_t lds, uint32_t rows, const bf16x8 (&b)[D / 32], int g, int c, bf16x8 (&P)[2]) const {
    const RowOperand<D, false> operand(lds, g, c);
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      f32x4 p = f32x4{0.f, 0.f, 0.f, 0.f};
      if (jt <= w) {
#pragma unroll
        for (int j = 0; j < D / 32; ++j) p = mfma_bf16(operand(rows, jt, j), b[j], p);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = jt < w ? p[i] * before[i] * apart[jt < 3 ? jt : 0] : ahead >= i ? p[i] * on[i] : 0.f;
      }
      const bf16x4 r = __builtin_convertvector(p, bf16x4);
#pragma unroll
      for (int i = 0; i < 4; ++i) P[jt >> 1][4 * (jt & 1) + i] = r[i];
    }
  }
};
// A tile's 16 columns of 32 rows of LDS from `row` (a multiple of 32) on, down the slots of k: rows 4 g + q and 16 + 4 g + q - 4 (see above), or 8 g + q with NATURAL.
template <int D, bool NATURAL> struct ColumnOperand {
  uint32_t at;
  __device__ __forceinline__ ColumnOperand(uint32_t lds, int g, int c) : at(opaque(lds + lds_at<D, NATURAL>((NATURAL ? 8 : 4) * g + (c >> 2), 4 * (c & 3)))) {}
  __device__ __forceinline__ bf16x8 operator()(uint32_t rows, int row, int ct) const {
    const uint32_t lo = (at ^ 32 * ct) + (rows + 2 * row * D);
    return read_transposed(lo, NATURAL ? (at ^ (32 * ct + 16)) + (rows + 2 * (row + 4) * D) : (at ^ 32 * ct) + (rows + 2 * (row + 16) * D));
  }
};
// Two tiles of an output, whose 16 columns each lie four to a lane, as eight columns in a row per lane: from column 16 (g % 2) + 8 (g / 2) of the 32 on.
__device__ __forceinline__ u32x4 pack_pair(f32x4 x, f32x4 y) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 a = __builtin_bit_cast(u32x2, __builtin_convertvector(x, bf16x4)), b = __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
  const auto r0 = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), r1 = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  return u32x4{r0[0], r1[0], r0[1], r1[1]};
}
// A thread's pieces of a tile into LDS (rows 2048 / D apart, a multiple of 16), and a wave's rows of a state, as columns and rounded to bf16.
template <int D, int PIECES> __device__ __forceinline__ void put_tile(uint32_t at, const u32x4 (&p)[PIECES]) {
#pragma unroll
  for (int i = 0; i < PIECES; ++i) lds_write(at + 4096 * i, p[i]);
}
template <int DK, int DV, bool NATURAL>
__device__ __forceinline__ void put_state(uint32_t lds, uint32_t St, const Part<DK, DV> &part, const f32x4 (&S)[Part<DK, DV>::RT][Part<DK, DV>::CW], int g, int c) {
  const uint32_t at = opaque(lds + 2 * part.col0 * DK + lds_at<DK, NATURAL>(c, part.row0 + 4 * g));
#pragma unroll
  for (int rt = 0; rt < Part<DK, DV>::RT; ++rt)
#pragma unroll
    for (int ct = 0; ct < Part<DK, DV>::CW; ++ct) lds_write((at ^ 32 * rt) + (St + 32 * ct * DK), __builtin_convertvector(S[rt][ct], bf16x4));
}
// What a wave has written to LDS for itself is read after this: LDS takes a wave's accesses in their order, and the compiler keeps it.
__device__ __forceinline__ void own_lds() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// A wave's 16 rows of a tensor on their way between memory, where whole lines of them are read and written, and the operands' layout: through 32 D bytes of LDS of its own.
template <int D, bool FULL> struct OwnRows {
  static constexpr int J = D / 32;
  TilePieces<D, 8, J, 64, FULL> pieces;
  uint32_t put;
  __device__ __forceinline__ OwnRows(const Rows &r, uint32_t stage, int w, int lane) : pieces(r, 16 * w, lane), put(stage + lds_at<D, false>(lane / (D / 8), lane % (D / 8) * 8)) {}
  // (rows 512 / D further on: the permutation by the row is another constant)
  __device__ __forceinline__ static uint32_t piece(uint32_t at, int i) { return (at ^ 16 * (D == 128 ? (i & 1) * 8 + (i >> 1) : i)) + 1024 * i; }
  __device__ __forceinline__ void operands(const u32x4 (&raw)[J], uint32_t stage, int g, int c, bf16x8 (&b)[J]) const {
    const uint32_t at = opaque(put);
#pragma unroll
    for (int i = 0; i < J; ++i) lds_write(piece(at, i), raw[i]);
    own_lds();
    const RowOperand<D, false> operand(stage, g, c);
#pragma unroll
    for (int j = 0; j < J; ++j) b[j] = operand(0, 0, j);
    own_lds();
  }
  __device__ __forceinline__ void out(const Rows &r, int r0) const {   // what pair_at's places hold
    own_lds();
    const uint32_t at = opaque(put);
    u32x4 raw[J];
#pragma unroll
    for (int i = 0; i < J; ++i) raw[i] = lds_read<u32x4>(piece(at, i));
    pieces.store(r, r0, raw);
    own_lds();
  }
};
// Where a lane's eight columns of a pair of tiles (the first one, the others an exclusive or of 64 bytes apart) lie in the wave's own LDS.
template <int D> __device__ __forceinline__ uint32_t pair_at(uint32_t stage, int g, int c) { return opaque(stage + lds_at<D, false>(c, 16 * (g & 1) + 8 * (g >> 1))); }
__device__ __forceinline__ void put_weights(uint32_t stage, int lane, const Walk &a, float l2, int behind) {   // behind: rows after the chunk's first one
  lds_write(stage + 4 * lane, a.gain * decay_pow(l2, max(behind - lane, 0) + (a.reverse ? 1 : 0)));
  own_lds();
}
// The output of a wave's 16 own rows into its own LDS: tile by tile what the state gives (`inter`) and the weights P times the chunk's rows.
// A weight that is masked is a zero, and in a product of matrices a zero times what is not a number or not finite is not a number: rows that come later would reach back.  So results that
// are not finite are formed again, with such values left out; where none of a row's own reach is among them, that is the result.
template <int D, typename Inter>
__device__ __forceinline__ void weighted_rows(uint32_t lds, uint32_t rows, uint32_t pair, const bf16x8 (&P)[2], int t, int g, int c, Inter inter) {
  const ColumnOperand<D, false> columns(lds, g, c);
  float probe = 0.f;
  auto tiles = [&](auto halves) {   // of the chunk's rows: the first 32 rows have no weights for the others
    f32x4 O[2];
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) {
      f32x4 acc = inter(ct);
#pragma unroll
      for (int jj = 0; jj < decltype(halves)::value; ++jj) acc = mfma_bf16(columns(rows, 32 * jj, ct), P[jj], acc);
#pragma unroll
      for (int i = 0; i < 4; ++i) probe = fmaf(acc[i], 0.f, probe);   // not a number if one is not finite
      O[ct & 1] = acc;
      if (ct & 1) lds_write(pair ^ 32 * (ct - 1), pack_pair(O[0], O[1]));
    }
  };
  if (t < 2) tiles(std::integral_constant<int, 1>{});
  else tiles(std::integral_constant<int, 2>{});
  if (!__any(!(probe == 0.f))) return;
  bf16x8 reach[2];   // one for the rows that a row has weights for
#pragma unroll
  for (int jj = 0; jj < 2; ++jj)
#pragma unroll
    for (int q = 0; q < 8; ++q) reach[jj][q] = 32 * jj + 4 * g + (q < 4 ? q : 12 + q) <= 16 * t + c ? (__bf16)1.f : (__bf16)0.f;
#pragma unroll 1
  for (int ct0 = 0; ct0 < D / 16; ct0 += 2) {
    f32x4 O[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      f32x4 all = inter(ct0 + e), finite = all, met = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        const bf16x8 v = columns(rows, 32 * jj, ct0 + e);
        u32x4 clean = __builtin_bit_cast(u32x4, v), ones;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool lo = (clean[i] & 0x7f80u) == 0x7f80u, hi = (clean[i] & 0x7f800000u) == 0x7f800000u;
          ones[i] = (lo ? 0x3f80u : 0u) | (hi ? 0x3f800000u : 0u);
          clean[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
        }
        all = mfma_bf16(v, P[jj], all);
        finite = mfma_bf16(__builtin_bit_cast(bf16x8, clean), P[jj], finite);
        met = mfma_bf16(__builtin_bit_cast(bf16x8, ones), reach[jj], met);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) O[e][i] = met[i] > 0.f ? all[i] : finite[i];
    }
    lds_write(pair ^ 32 * ct0, pack_pair(O[0], O[1]));
  }
}
// S <- keep S + (K o weight)^T V over the chunk's rows in LDS.  weight: the wave's own table of the chunk's rows.  SUM: keep is 1.
template <int DK, int DV, bool SUM>
__device__ __forceinline__ void update_state(const Part<DK, DV> &part, f32x4 (&S)[Part<DK, DV>::RT][Part<DK, DV>::CW], float keep, uint32_t lds, uint32_t Ks, uint32_t Vs,
                                             uint32_t weight, int g, int c) {
  constexpr int RT = Part<DK, DV>::RT, CW = Part<DK, DV>::CW;
  ColumnOperand<DK, false> keys(lds, g, c);
  keys.at ^= 2 * part.row0;
  ColumnOperand<DV, false> values(lds, g, c);
  if (DK < 64) values.at ^= 2 * part.col0;
  bf16x8 K[RT][2][3];
#pragma unroll
  for (int jj = 0; jj < 2; ++jj) {
    const f32x4 w0 = lds_read<f32x4>(weight + 128 * jj + 16 * g), w1 = lds_read<f32x4>(weight + 128 * jj + 64 + 16 * g);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) three_terms(keys(Ks, 32 * jj, rt), w0, w1, K[rt][jj]);
  }
#pragma unroll
  for (int ct = 0; ct < CW; ++ct) {
    const bf16x8 V[2] = {values(Vs, 0, ct), values(Vs, 32, ct)};
    if (!SUM) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) S[rt][ct] *= keep;
    }
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int u = 2; u >= 0; --u)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) S[rt][ct] = mfma_bf16(K[rt][jj][u], V[jj], S[rt][ct]);
  }
}

// As walk_f32_kernel, for bf16 tensors.  P and the state as an operand of the output are rounded to bf16, like the output (each 2^-9 of a result in the root mean square; P in two terms would
// take the error of a result from 0.0023 to 0.0020 of it, for 4 %); what goes into the state is not.  Bound by memory: width 128, 32 slices of 65536 rows, 446 to 459 us on two cards, 4.7 TB/s
// (without the update of the state 416 where it took 462; loads and stores alone 380 to 400); width 64, 8 slices of 131072, 89 to 96 us, 5.6 TB/s; forming states alone 211 to 214 us, 5.0 TB/s (199 without the
// products), and 53 to 60 us, 4.5 to 5.1 TB/s.
template <int DK, int DV, bool FULL, bool STATES, bool NT>
__global__ __launch_bounds__(256, DK + DV <= 64 ? 4 : DK + DV <= 128 ? 3 : 2) void walk_bf16_kernel(Walk a) {
  constexpr int PK = kChunk * DK / 8 / 256, PV = kChunk * DV / 8 / 256;   // pieces of a thread
  typedef Part<DK, DV> P4;
  constexpr int QJ = DK / 32, STAGE = STATES ? 256 : 32 * (DK > DV ? DK : DV);   // bytes of LDS that a wave has for itself
  // The walk that forms states only waits for memory alone: it has tiles twice, in LDS and under way.
  constexpr int SETS = STATES ? 2 : 1, SET = 2 * kChunk * (DK + DV);
  extern __shared__ __align__(16) unsigned char lds_bytes[];
  // in LDS: K, V, the columns of the state as rows, the waves' own parts
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds_bytes;
  constexpr uint32_t Ks = 0, Vs = 2 * kChunk * DK, St = SETS * SET;
  const int slot = slot_of(a), h = head_of(a);
  const Segment seg = segment_of(a.seq, slot);
  if (seg.rows < 0) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  const P4 part(w);
  const int t = part.t;
  const uint32_t stage = lds + SETS * SET + (STATES ? 0 : 2 * DV * DK) + STAGE * w;
  const bool last = a.reverse ? seg.s == 0 : seg.s == a.seq.segments(seg.b) - 1;
  if (STATES && last) return;
  const Rows qr = rows_of(a.q, a.sq, seg, a, h, a.kw, 2), kr = rows_of(a.k, a.sk, seg, a, h, a.kw, 2), vr = rows_of(a.v, a.sv, seg, a, h, a.vw, 2),
             orow = rows_of(a.o, a.so, seg, a, h, a.vw, 2);
  const float l2 = log2_decay(a.log_decay, h);
  const int64_t state_size = (int64_t)a.kw * a.vw;

  f32x4 S[P4::RT][P4::CW];   // S[rt][ct][i] is row row0 + 16 rt + 4 g + i, column col0 + 16 ct + c
  const int own = cache_row(a, seg.b);
  const int64_t from = a.by_slot ? (int64_t)slot : own;
  const float *init = STATES || !a.init || from < 0 ? nullptr : a.init + (from * a.H + h) * state_size;
  each_of_state(a, S, part, g, c, [&](float, bool there, int64_t at) { return init && there ? init[at] : 0.f; });
  const Weights weights(a, l2, t, g, c);

  u32x4 rk[SETS][PK], rv[SETS][PV], rq[QJ];
  const TilePieces<DK, 8, PK, 256, FULL> kp(kr, 0, tid);
  const TilePieces<DV, 8, PV, 256, FULL> vp(vr, 0, tid);
  const OwnRows<DK, FULL> qo(qr, stage, t, lane);
  const OwnRows<DV, FULL> oo(orow, stage, t, lane);
  const uint32_t kput = lds + Ks + lds_at<DK, false>(tid / (DK / 8), tid % (DK / 8) * 8), vput = lds + Vs + lds_at<DV, false>(tid / (DV / 8), tid % (DV / 8) * 8);
  auto request = [&](int r0, int set) {
    kp.template load<NT>(kr, r0, rk[set]);
    vp.template load<NT>(vr, r0, rv[set]);
  };

#pragma unroll
  for (int set = 0; set < SETS; ++set) request(set * kChunk, set);
  if (!STATES) qo.pieces.template load<NT>(qr, 0, rq);
  for (int r1 = 0; r1 < seg.rows; r1 += SETS * kChunk) {
#pragma unroll
    for (int set = 0; set < SETS; ++set) {
      const int r0 = r1 + set * kChunk, rows = min(kChunk, seg.rows - r0);
      if (set && rows <= 0) break;
      put_tile<DK, PK>(kput + set * SET, rk[set]);
      put_tile<DV, PV>(vput + set * SET, rv[set]);
      bf16x8 Q[QJ];
      if (!STATES) {
        put_state<DK, DV, false>(lds, St, part, S, g, c);
        qo.operands(rq, stage, g, c, Q);
      }
      __syncthreads();
      request(r0 + SETS * kChunk, set);
      if (!STATES) {
        bf16x8 P[2];
        weights.products<DK>(lds, Ks, Q, g, c, P);
        const RowOperand<DK, false> state(lds, g, c);
        weighted_rows<DV>(lds, Vs, pair_at<DV>(stage, g, c), P, t, g, c, [&](int ct) {
          f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < QJ; ++j) acc = mfma_bf16(state(St, ct, j), Q[j], acc);
          return acc * weights.reach;
        });
        oo.out(orow, r0);
        qo.pieces.template load<NT>(qr, r0 + kChunk, rq);
      }
      // the walk that forms states only weights rows by the segment's end, and has no sum to scale
      put_weights(stage, lane, a, l2, STATES ? seg.rows - 1 - r0 : rows - 1);
      update_state<DK, DV, STATES>(part, S, decay_pow(l2, rows), lds, Ks + set * SET, Vs + set * SET, stage, g, c);
      if (SETS == 1) __syncthreads();   // (with two sets every wave is past this one's reads at the next set's barrier)
    }
  }

  float *fin = nullptr;
  if (STATES) fin = a.fin + ((int64_t)slot * a.H + h) * state_size;
  else if (last && a.fin && own >= 0) fin = a.fin + ((int64_t)own * a.H + h) * state_size;
  if (fin) each_of_state(a, S, part, g, c, [&](float x, bool there, int64_t at) { if (there) fin[at] = x; return x; });
}

// As back_f32_kernel, for bf16 tensors.  Width 128, 32 slices of 65536 rows: 654 to 670 us on two cards, 4.8 to 4.9 TB/s (630 without the update of the state where it took 672); two walks took 2 x 502.
template <int DK, int DV, bool FULL, bool NT>
__global__ __launch_bounds__(256, DK + DV <= 64 ? 4 : 2) void back_bf16_kernel(Walk a, Back b) {
  constexpr int PK = kChunk * DK / 8 / 256, PV = kChunk * DV / 8 / 256;
  typedef Part<DK, DV> P4;
  constexpr int KJ = DK / 32, VJ = DV / 32, STAGE = 32 * (DK > DV ? DK : DV);
  extern __shared__ __align__(16) unsigned char lds_bytes[];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds_bytes;
  constexpr uint32_t Qs = 0, Ds = 2 * kChunk * DK, Gt = Ds + 2 * kChunk * DV;
  const int slot = slot_of(a), h = head_of(a);
  const Segment seg = segment_of(a.seq, slot);
  if (seg.rows < 0) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  const P4 part(w);
  const int t = part.t;
  const uint32_t stage = lds + Gt + 2 * DV * DK + STAGE * w;
  const Rows qr = rows_of(a.k, a.sk, seg, a, h, a.kw, 2), dr = rows_of(a.v, a.sv, seg, a, h, a.vw, 2), kr = rows_of(b.k, b.sk, seg, a, h, a.kw, 2),
             vr = rows_of(b.v, b.sv, seg, a, h, a.vw, 2), dkr = rows_of(b.dk, b.sdk, seg, a, h, a.kw, 2), dvr = rows_of(b.dv, b.sdv, seg, a, h, a.vw, 2);
  const float l2 = log2_decay(a.log_decay, h);
  const int64_t state_size = (int64_t)a.kw * a.vw;

  f32x4 G[P4::RT][P4::CW];
  const int64_t from = a.by_slot ? (int64_t)slot : seg.b;
  const float *init = a.init ? a.init + (from * a.H + h) * state_size : nullptr;
  each_of_state(a, G, part, g, c, [&](float, bool there, int64_t at) { return init && there ? init[at] : 0.f; });
  const Weights weights(a, l2, t, g, c);

  u32x4 rq[PK], rd[PV], rk[KJ], rv[VJ];
  const TilePieces<DK, 8, PK, 256, FULL> qp(qr, 0, tid);
  const TilePieces<DV, 8, PV, 256, FULL> dp(dr, 0, tid);
  const OwnRows<DK, FULL> ko(kr, stage, t, lane), dko(dkr, stage, t, lane);
  const OwnRows<DV, FULL> vo(vr, stage, t, lane), dvo(dvr, stage, t, lane);
  const uint32_t qput = lds + Qs + lds_at<DK, false>(tid / (DK / 8), tid % (DK / 8) * 8), dput = lds + Ds + lds_at<DV, false>(tid / (DV / 8), tid % (DV / 8) * 8);
  auto request = [&](int r0) {
    qp.template load<NT>(qr, r0, rq);
    dp.template load<NT>(dr, r0, rd);
  };
  auto request_own = [&](int r0) {
    ko.pieces.template load<NT>(kr, r0, rk);
    vo.pieces.template load<NT>(vr, r0, rv);
  };

  request(0);
  request_own(0);
  for (int r0 = 0; r0 < seg.rows; r0 += kChunk) {
    const int rows = min(kChunk, seg.rows - r0);
    put_tile<DK, PK>(qput, rq);
    put_tile<DV, PV>(dput, rd);
    put_state<DK, DV, true>(lds, Gt, part, G, g, c);
    bf16x8 K[KJ], V[VJ];
    ko.operands(rk, stage, g, c, K);
    vo.operands(rv, stage, g, c, V);
    __syncthreads();
    request(r0 + kChunk);
    bf16x8 P[2];
    weights.products<DK>(lds, Qs, K, g, c, P);
    {
      const RowOperand<DK, true> state(lds, g, c);
      weighted_rows<DV>(lds, Ds, pair_at<DV>(stage, g, c), P, t, g, c, [&](int ct) {
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < KJ; ++j) acc = mfma_bf16(state(Gt, ct, j), K[j], acc);
        return acc * weights.reach;
      });
      dvo.out(dvr, r0);
    }
    weights.products<DV>(lds, Ds, V, g, c, P);
    {
      const ColumnOperand<DK, true> state(lds, g, c);
      weighted_rows<DK>(lds, Qs, pair_at<DK>(stage, g, c), P, t, g, c, [&](int kt) {
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < VJ; ++j) acc = mfma_bf16(state(Gt, 32 * j, kt), V[j], acc);
        return acc * weights.reach;
      });
      dko.out(dkr, r0);
    }
    request_own(r0 + kChunk);
    put_weights(stage, lane, a, l2, rows - 1);
    update_state<DK, DV, false>(part, G, decay_pow(l2, rows), lds, Qs, Ds, stage, g, c);
    __syncthreads();
  }
  if (a.fin && seg.s == 0) {
    float *fin = a.fin + ((int64_t)seg.b * a.H + h) * state_size;
    each_of_state(a, G, part, g, c, [&](float x, bool there, int64_t at) { if (there) fin[at] = x; return x; });
  }
}

// Packed sequences lie one behind the other: rows of none are those before the first one and those behind the last one. Zeros to them, for nothing else writes them, in
// up to three tensors. With a launch of their own (sequences of one segment) or beside the scan's workgroups, which costs no time of its own where there are no such rows.
struct Outside {
  void *to[3];              // the first one null: not wanted
  Strides stride[3];
  int width[3];
  int element;
};
__device__ __forceinline__ void clear_outside(const Sequences &q, const Outside &a, int h, int group, int groups) {
  typedef u32x4 u32x4_any __attribute__((aligned(2)));
  const int first = q.begin(0), last = max(first, q.begin(q.B)), rows = first + q.n - last;
#pragma unroll
  for (int u = 0; u < 3; ++u) {
    if (!a.to[u]) break;
    const int per_row = a.width[u] * a.element / 16, at_once = (int)blockDim.x / per_row, mine = (int)threadIdx.x / per_row;   // pieces of 16 bytes; whole rows at a time
    char *to = (char *)a.to[u] + h * a.stride[u].h * a.element + (int)threadIdx.x % per_row * 16;
    if (mine < at_once)
      for (int64_t i = (int64_t)group * at_once + mine; i < rows; i += (int64_t)groups * at_once)
        *(u32x4_any *)(to + (i < first ? i : i + (last - first)) * a.stride[u].n * a.element) = u32x4{0, 0, 0, 0};
  }
}
__global__ __launch_bounds__(256) void clear_kernel(Sequences seq, Outside a) { clear_outside(seq, a, blockIdx.y, blockIdx.x, gridDim.x); }

// What the segments of a sequence add to the state, in place, to the states that they begin with: E values of a state per thread, over all
// segments in their order (from the last one with `reverse`).  Few states are bound by the way to memory and back of each round of requests: rounds have many,
// and a thread has one value, so that there are threads; many states (packed prompts) by the launch of their workgroups: four values then.  24 packed prompts, 16 heads
// of 128 x 128: 77 us with one value; 8 slices of 64 x 64, 96 segments: 31 us with four values and rounds of eight.
template <int E, int ROUND>
__global__ __launch_bounds__(256) void scan_kernel(Walk a, float *local, Outside outside) {
  typedef float V __attribute__((ext_vector_type(E)));
  const int h = blockIdx.y, b = blockIdx.z;
  if (b == a.seq.B) {
    clear_outside(a.seq, outside, h, blockIdx.x, gridDim.x);
    return;
  }
  const int64_t state_size = (int64_t)a.kw * a.vw, e = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * E;
  if (e >= state_size) return;
  const int segs = a.seq.segments(b), have = a.seq.rows(b), own = cache_row(a, b);
  const float l2 = log2_decay(a.log_decay, h);
  V run = V(0.f);
  if (a.init && own >= 0) run = *(const V *)(a.init + ((int64_t)own * a.H + h) * state_size + e);
  const int64_t step = a.H * state_size;
  float *p = local + ((int64_t)a.seq.first_slot(b) * a.H + h) * state_size + e;
  const float full = decay_pow(l2, a.seq.seg), tail = decay_pow(l2, have - (segs - 1) * a.seq.seg);
  for (int s0 = 0; s0 < segs; s0 += ROUND) {
    V x[ROUND];
#pragma unroll
    for (int u = 0; u < ROUND; ++u) {
      const int s = a.reverse ? segs - 1 - s0 - u : s0 + u;
      x[u] = s0 + u < segs - 1 ? *(const V *)(p + s * step) : V(0.f);   // the last one has added nothing
    }
#pragma unroll
    for (int u = 0; u < ROUND; ++u) {
      const int s = a.reverse ? segs - 1 - s0 - u : s0 + u;
      if (s0 + u < segs) *(V *)(p + s * step) = run;
      run = run * (s == segs - 1 ? tail : full) + x[u];
    }
  }
}

// ---- one token -------------------------------------------------------------------------------------
// S <- lambda S + k v^T, o = scale q^T S.  Bound by the state's way through memory.  A workgroup has W columns of a state, W / 4 threads to a
// row (16 bytes each), all rows of a thread requested before the first is used.  NT: states that will not be in the last-level cache when their next token comes pass by it
// (256 users, 16 heads of 128 x 128, 268 MB of states, three layers in turn: 111 us, 101 with NT; one layer over and over, which the cache holds most of: 84, 102 with NT).
constexpr int64_t kCachedStates = 128 << 20;   // half of the last-level cache
struct Step {
  const void *q, *k, *v;
  void *o;
  Strides sq, sk, sv, so;
  const float *log_decay;
  float *state;
  const int32_t *cache;
  int cache_rows, H, kw, vw;
  float scale;
};
template <typename T, int W, bool NT>
__global__ __launch_bounds__(256) void step_kernel(Step a) {
  constexpr int TPR = W / 4, ROWS = 256 / TPR, PASS = (128 + ROWS - 1) / ROWS;
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, col = blockIdx.x * W + tid % TPR * 4, r0 = tid / TPR;
  __shared__ float key[128], query[128];
  __shared__ f32x4 part[4][TPR];
  const int own0 = a.cache ? a.cache[b] : b, own = own0 < 0 || own0 >= a.cache_rows ? -1 : own0;
  const T *q = (const T *)a.q + b * a.sq.b + h * a.sq.h, *k = (const T *)a.k + b * a.sk.b + h * a.sk.h, *v = (const T *)a.v + b * a.sv.b + h * a.sv.h;
  T *o = (T *)a.o + b * a.so.b + h * a.so.h;
  const bool there = own >= 0 && col < a.vw;
  const float mine = tid % 128 < a.kw ? ld((tid < 128 ? k : q) + tid % 128) : 0.f;
  f32x4 vv = f32x4{0.f, 0.f, 0.f, 0.f}, sum = vv, x[PASS];
  float *s = a.state + ((int64_t)own * a.H + h) * a.kw * a.vw + col;
  if (there) {
#pragma unroll
    for (int i = 0; i < 4; ++i) vv[i] = ld(v + col + i);
#pragma unroll
    for (int u = 0; u < PASS; ++u)
      if (r0 + u * ROWS < a.kw) {
        const f32x4 *p = (const f32x4 *)(s + (r0 + u * ROWS) * a.vw);
        x[u] = NT ? __builtin_nontemporal_load(p) : *p;
      }
  }
  (tid < 128 ? key : query)[tid % 128] = mine;
  const float lambda = decay_pow(log2_decay(a.log_decay, h), 1);
  __syncthreads();
  if (there) {
#pragma unroll
    for (int u = 0; u < PASS; ++u)
      if (r0 + u * ROWS < a.kw) {
        const float kk = key[r0 + u * ROWS], qq = query[r0 + u * ROWS];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[u][i] = x[u][i] * lambda + kk * vv[i];
          sum[i] += qq * x[u][i];
        }
        f32x4 *p = (f32x4 *)(s + (r0 + u * ROWS) * a.vw);
        if (NT) __builtin_nontemporal_store(x[u], p);
        else *p = x[u];
      }
  }
  // over the rows: lanes of a wave, then the four waves
#pragma unroll
  for (int d = TPR; d < 64; d *= 2)
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], d);
  if ((tid & 63) < TPR) part[tid >> 6][tid & 63] = sum;
  __syncthreads();
  if (tid < TPR && col < a.vw) {
#pragma unroll
    for (int i = 0; i < 4; ++i) st(o + col + i, a.scale * ((part[0][tid][i] + part[1][tid][i]) + (part[2][tid][i] + part[3][tid][i])));
  }
}

// ---- host ------------------------------------------------------------------------------------------
// Rows of a segment, by what a forward pass takes.  The device holds `held` workgroups of a walk at a time; with all of them a chunk takes `full` us of each, a workgroup alone needs
// `alone`.  More than one segment to a sequence costs the launch that forms states (about 0.45 of a walk without the last segments), the scan's traffic and two launches.
// us of a recorded forward pass with this rule, in parentheses with as many segments as the device holds: 48 x 8 slices of 501 rows, width 64, 28 (54); 16 x 16 of 300 16 (35); 8 x 8 of 500
// 20 (22); 16 x 16 of 1000, width 128, 77 (104); 8 of 2000, width 64, 18 in segments of two chunks, 65 in one; 64 of 2048, width 128, 84, 128 in one; 32 of 65536, walk alone:
// 519 in 512 segments, 615 in 768.
struct Pace {
  int held;
  float full, alone;
};
Pace pace(const wersa_decay_desc &c) {
  const int width = c.dk > c.dv ? c.dk : c.dv;
  if (c.dtype == WERSA_BF16) return width <= 32 ? Pace{1024, 3.7f, 1.7f} : width <= 64 ? Pace{768, 5.0f, 2.1f} : Pace{512, 7.8f, 4.2f};
  return width <= 32 ? Pace{768, 6.2f, 2.5f} : width <= 64 ? Pace{512, 10.2f, 5.0f} : Pace{256, 17.f, 17.f};
}
int segment_rows(const wersa_decay_desc &c) {
  const Pace p = pace(c);
  if (c.packed) {
    // Lengths are not known here.  Seven eighths as many whole segments as the device holds: every sequence has a partial one on top.  Geometric mean of nine batches of 8 to 60 prompts, widths 32 to
    // 128, with six draws of long-tailed lengths each: 125 us, 138 with five eighths, 129 with six, 135 with eight, 139 with nine, 132 with twelve.  Two chunks at least.
    const int64_t want = (int64_t)p.held * 7 / 8 / c.H;
    if (want <= 1) return INT32_MAX / 2;
    const int64_t rows = ((c.n + want - 1) / want + kChunk - 1) / kChunk * kChunk;
    return (int)(rows < 2 * kChunk ? 2 * kChunk : rows);
  }
  const int64_t slices = (int64_t)c.H * c.B, chunks = ((int64_t)c.n + kChunk - 1) / kChunk;
  auto walk = [&](int64_t each, int64_t segments) {   // us of `segments` workgroups per slice over `each` chunks
    const double load = (double)slices * segments / p.held;
    return each * (load <= 1 ? std::max<double>(p.alone, p.full * load) : p.full * std::ceil(load));
  };
  int64_t best = chunks + 1;   // more than there are: one segment
  double least = walk(chunks, 1);
  auto consider = [&](int64_t each) {
    const int64_t k = each < 1 ? 1 : (chunks + each - 1) / each;
    if (k < 2) return;
    const double us = walk(each, k) * (1 + 0.45 * (k - 1) / k) + 12 + (double)slices * k * c.dk * c.dv * 8 / 5e6;
    if (us < least) least = us, best = each;
  };
  for (const int64_t each : {1, 2, 3, 4, 6, 8}) consider(each);
  for (int64_t rounds = 1; rounds <= 3; ++rounds) {
    const int64_t k = p.held * rounds / slices;
    if (k >= 2) consider((chunks + k - 1) / k);
  }
  return (int)(best * kChunk);
}
Sequences sequences(const wersa_decay_desc &c, const int32_t *offsets) {
  Sequences s;
  s.offsets = offsets;
  s.B = c.B;
  s.n = c.n;
  s.seg = segment_rows(c);
  s.segs = c.n > 0 ? (c.n + s.seg - 1) / s.seg : 1;
  return s;
}
// How walks go through memory, where a head's rows are whole lines of 128 bytes (others share lines with their neighbours, and take up to twice as long either way).
bool whole_lines(const wersa_decay_desc &c) {
  const int e = c.dtype == WERSA_F32 ? 4 : 2;
  return c.dk * e % 128 == 0 && c.dv * e % 128 == 0;
}
// Heads that lie side by side in a row go side by side through the grid: 24 packed prompts, 16 heads, 65536 rows, width 128 in bf16: walk 336 us, 304 so; float32, width 32, 128 slices of
// 4000 rows: 68, 65.  With heads apart in memory the walks would take longer so (loads and stores alone: 380, 448).
bool heads_first(const wersa_decay_desc &c, const Sequences &s) { return c.stride_v[1] < c.stride_v[2] && whole_lines(c) && s.slots() <= 65535; }   // (blockIdx.y)
// Walks in bf16 read by the caches what these would not keep to the next kernel: 8 slices of 131072 rows, width 64 (134 MB a tensor), walk 112 us, 100 so; 1024 of 500 rows (65 MB) would take
// 66 for 61.  The walk that forms states never does: the next one finds part of what it read (the same 8 slices: 117 us for 112).
constexpr int64_t kLastLevelCache = 256 << 20;
bool passes_caches(const wersa_decay_desc &c) {
  return whole_lines(c) && ((int64_t)c.packed * c.n + (1 - c.packed) * (int64_t)c.B * c.n) * c.H * (2 * c.dk + c.dv) * 2 > kLastLevelCache;
}
int64_t state_slots_of(const wersa_decay_desc &c) {   // 0: every sequence is one segment
  const int seg = segment_rows(c);
  if (c.n <= seg) return 0;
  return c.packed ? (int64_t)c.n / seg + c.B : (int64_t)c.B * ((c.n + seg - 1) / seg);
}
size_t states_bytes(const wersa_decay_desc &c) { return (size_t)state_slots_of(c) * c.H * c.dk * c.dv * sizeof(float); }

bool strides_ok(const int64_t *s, const wersa_decay_desc &c, int width) {
  if (s[0] < 0 || s[1] < 0 || s[2] < 0) return false;
  if (!c.packed && c.B > 1 && s[0] == 0) return false;
  if (c.H > 1 && s[1] == 0) return false;
  return c.n <= 1 || s[2] >= width;
}
// What is written: heads and sequences must not lie on each other, as those that are only read may. Sorted by stride, a dimension begins anew behind what the ones before it take.
bool apart(const int64_t *s, const wersa_decay_desc &c, int width) {
  struct { int64_t stride, count; } dim[3] = {{s[0], c.packed ? 1 : c.B}, {s[1], c.H}, {s[2], c.n}};
  std::sort(dim, dim + 3, [](auto &x, auto &y) { return x.stride < y.stride; });
  __int128 taken = width;
  for (const auto &d : dim)
    if (d.count > 1) {
      if (d.stride < taken) return false;
      taken += (__int128)d.stride * (d.count - 1);
    }
  return true;
}
// A gradient's strides: those of its tensor where the descriptor has none.
const int64_t *strides_of_gradient(const int64_t *own, const int64_t *tensor) { return own[0] == 0 && own[1] == 0 && own[2] == 0 ? tensor : own; }
wersa_status written(const int64_t *s, const wersa_decay_desc &c, int width) {
  if (s[0] < 0 || s[1] < 0 || s[2] < 0 || !apart(s, c, width)) return WERSA_ERR_INVALID_ARG;
  return c.n > 1 && s[2] > kMostRowStride ? WERSA_ERR_UNSUPPORTED : WERSA_OK;
}
wersa_status validate(const wersa_decay_desc *c) {
  if (!c) return WERSA_ERR_INVALID_ARG;
  if (c->B < 1 || c->H < 1 || c->n < 0 || c->dk < 1 || c->dv < 1) return WERSA_ERR_INVALID_ARG;
  if (c->dtype != WERSA_F32 && c->dtype != WERSA_BF16) return WERSA_ERR_INVALID_ARG;
  if ((c->packed != 0 && c->packed != 1) || (c->clear != 0 && c->clear != 1)) return WERSA_ERR_INVALID_ARG;
  if (!(c->scale - c->scale == 0.f)) return WERSA_ERR_INVALID_ARG;   // not finite
  if (!strides_ok(c->stride_q, *c, c->dk) || !strides_ok(c->stride_k, *c, c->dk) || !strides_ok(c->stride_v, *c, c->dv) ||
      !strides_ok(c->stride_o, *c, c->dv))
    return WERSA_ERR_INVALID_ARG;
  if (c->dk % 16 != 0 || c->dv % 16 != 0 || c->dk > 128 || c->dv > 128) return WERSA_ERR_UNSUPPORTED;
  for (const int64_t *s : {c->stride_q, c->stride_k, c->stride_v, c->stride_o})
    if (c->n > 1 && s[2] > kMostRowStride) return WERSA_ERR_UNSUPPORTED;
  if (c->H > 65535 || c->B > 65535 || c->n > (1 << 30)) return WERSA_ERR_UNSUPPORTED;
  return WERSA_OK;
}
bool misaligned(const void *p, size_t a) { return ((uintptr_t)p % a) != 0; }
// A lone row's stride may be anything (0, one element, past 32 bits). Rows that are not there are told from it by their distance from it: they get the width.
Strides strides(const int64_t *s, const wersa_decay_desc &c, int width) { return Strides{s[0], s[1], c.n > 1 ? s[2] : width}; }
template <typename K, typename... Args> bool launch(const char *name, K kern, int threads, size_t smem, const Walk &a, hipStream_t st, Args... more) {
  if (smem > 65536 &&
      hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != hipSuccess)
    return false;
  WERSA_STAGE(name, st, kern<<<a.heads_first ? dim3(a.H, a.seq.slots()) : dim3(a.seq.slots(), a.H), threads, smem, st>>>(a, more...));
  return true;
}
constexpr size_t f32_lds(int dk, int dv, bool state) { return sizeof(float) * (kChunk * (dk + 4 + dv + 4 + 1) + (state ? dv * (dk + 4) : 0)); }
template <int DK, int DV, bool STATES> bool launch_walk_as(const wersa_decay_desc &c, const Walk &a, hipStream_t st) {
  const char *name = STATES ? "wersa_decay_states" : "wersa_decay_walk";
  if (c.dtype == WERSA_F32) return launch(name, &walk_f32_kernel<DK, DV, STATES>, 64 * f32_waves(DK, DV), f32_lds(DK, DV, !STATES), a, st);
  constexpr size_t sets = STATES ? 2 : 1, smem = 2 * (sets * kChunk * (DK + DV) + (STATES ? 0 : DV * DK)) + 4 * (STATES ? 256 : 32 * (DK > DV ? DK : DV));
  if (a.kw != DK || a.vw != DV) return launch(name, &walk_bf16_kernel<DK, DV, false, STATES, false>, 256, smem, a, st);
  return !STATES && DK > 32 && passes_caches(c) ? launch(name, &walk_bf16_kernel<DK, DV, true, STATES, !STATES && (DK > 32)>, 256, smem, a, st)
                                                : launch(name, &walk_bf16_kernel<DK, DV, true, STATES, false>, 256, smem, a, st);
}
template <bool STATES> bool launch_walk(const wersa_decay_desc &c, const Walk &a, hipStream_t st) {
  if (a.kw <= 32 && a.vw <= 32) return launch_walk_as<32, 32, STATES>(c, a, st);
  if (a.kw <= 64) return a.vw <= 64 ? launch_walk_as<64, 64, STATES>(c, a, st) : launch_walk_as<64, 128, STATES>(c, a, st);
  return a.vw <= 64 ? launch_walk_as<128, 64, STATES>(c, a, st) : launch_walk_as<128, 128, STATES>(c, a, st);
}
template <int DK, int DV> bool launch_back_as(const wersa_decay_desc &c, const Walk &a, const Back &b, hipStream_t st) {
  if (c.dtype == WERSA_F32) return launch("wersa_decay_back", &back_f32_kernel<DK, DV>, 64 * f32_waves(DK, DV), f32_lds(DK, DV, true), a, st, b);
  constexpr size_t smem = 2 * (kChunk * (DK + DV) + DV * DK) + 4 * 32 * (DK > DV ? DK : DV);
  if (a.kw != DK || a.vw != DV) return launch("wersa_decay_back", &back_bf16_kernel<DK, DV, false, false>, 256, smem, a, st, b);
  return DK > 32 && passes_caches(c) ? launch("wersa_decay_back", &back_bf16_kernel<DK, DV, true, (DK > 32)>, 256, smem, a, st, b)
                                     : launch("wersa_decay_back", &back_bf16_kernel<DK, DV, true, false>, 256, smem, a, st, b);
}
bool launch_back(const wersa_decay_desc &c, const Walk &a, const Back &b, hipStream_t st) {
  if (a.kw <= 32 && a.vw <= 32) return launch_back_as<32, 32>(c, a, b, st);
  if (a.kw <= 64) return a.vw <= 64 ? launch_back_as<64, 64>(c, a, b, st) : launch_back_as<64, 128>(c, a, b, st);
  return a.vw <= 64 ? launch_back_as<128, 64>(c, a, b, st) : launch_back_as<128, 128>(c, a, b, st);
}
// Returns whether rows of no sequence are cleared.
bool launch_scan(const Walk &a, float *local, const Outside &outside, hipStream_t st) {
  const int size = a.kw * a.vw;
  const bool clear = outside.to[0] && a.seq.B < 65535;   // (blockIdx.z)
  const int depth = a.seq.B + clear;
  if ((int64_t)size * a.H * a.seq.B >= 1 << 21)   // eight waves of four values to a SIMD
    WERSA_STAGE("wersa_decay_scan", st, (scan_kernel<4, 8><<<dim3((size / 4 + 255) / 256, a.H, depth), 256, 0, st>>>(a, local, outside)));
  else
    WERSA_STAGE("wersa_decay_scan", st, (scan_kernel<1, 32><<<dim3((size + 63) / 64, a.H, depth), 64, 0, st>>>(a, local, outside)));
  return clear;
}
void launch_clear(const wersa_decay_desc &c, const Sequences &seq, const Outside &outside, hipStream_t st) {
  const int64_t across = std::min<int64_t>(((int64_t)c.n * std::max(c.dk, c.dv) * outside.element / 16 + 255) / 256, std::max(1, 2048 / c.H));
  WERSA_STAGE("wersa_decay_clear", st, (clear_kernel<<<dim3((unsigned)across, c.H), 256, 0, st>>>(seq, outside)));
}

}  // namespace
}  // namespace wersa

using namespace wersa;

extern "C" {

size_t wersa_decay_workspace_bytes(const wersa_decay_desc *desc, int for_backward) {
  (void)for_backward;
  return validate(desc) == WERSA_OK ? states_bytes(*desc) + 256 : 0;
}

size_t wersa_decay_saved_bytes(const wersa_decay_desc *desc) { return validate(desc) == WERSA_OK ? states_bytes(*desc) + 256 : 0; }

wersa_status wersa_decay_forward(const wersa_decay_desc *desc, const void *q, const void *k, const void *v, const float *log_decay,
                                 const int32_t *offsets, const float *initial_state, float *final_state, const int32_t *slots,
                                 int32_t state_slots, void *out, void *saved, void *workspace, size_t workspace_bytes, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  const wersa_decay_desc &c = *desc;
  if (c.n > 0 && (!q || !k || !v || !out)) return WERSA_ERR_INVALID_ARG;
  if (!log_decay || (c.packed != 0) != (offsets != nullptr)) return WERSA_ERR_INVALID_ARG;
  if ((initial_state || final_state) && state_slots < (slots ? 1 : c.B)) return WERSA_ERR_INVALID_ARG;
  if (misaligned(initial_state, 16) || misaligned(final_state, 16)) return WERSA_ERR_INVALID_ARG;
  if (const wersa_status ws = written(c.stride_o, c, c.dv)) return ws;
  const bool split = state_slots_of(c) > 0;
  if (split && !saved && (!workspace || workspace_bytes < states_bytes(c) || misaligned(workspace, 256))) return WERSA_ERR_WORKSPACE;
  if (misaligned(saved, 256)) return WERSA_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)hip_stream;
  Walk a{};
  a.q = q, a.k = k, a.v = v, a.o = out;
  a.sq = strides(c.stride_q, c, c.dk), a.sk = strides(c.stride_k, c, c.dk), a.sv = strides(c.stride_v, c, c.dv), a.so = strides(c.stride_o, c, c.dv);
  a.log_decay = log_decay;
  a.init = initial_state, a.cache = slots, a.cache_rows = state_slots;
  a.seq = sequences(c, offsets);
  a.heads_first = heads_first(c, a.seq);
  a.H = c.H, a.kw = c.dk, a.vw = c.dv, a.si = c.dv, a.sj = 1;
  a.intra = a.inter = c.scale, a.gain = 1.f;
  Outside outside{{}, {}, {}, c.dtype == WERSA_F32 ? 4 : 2};
  bool clear = c.packed && c.clear && c.n > 0;
  if (clear) outside.to[0] = out, outside.stride[0] = a.so, outside.width[0] = c.dv;
  if (split) {
    float *local = (float *)(saved ? saved : workspace);
    a.fin = local;
    if (!launch_walk<true>(c, a, st)) return WERSA_ERR_LAUNCH;
    if (launch_scan(a, local, outside, st)) clear = false;
    a.init = local, a.by_slot = true;
  }
  if (clear) launch_clear(c, a.seq, outside, st);
  a.fin = final_state;
  if (!launch_walk<false>(c, a, st)) return WERSA_ERR_LAUNCH;
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

wersa_status wersa_decay_backward(const wersa_decay_desc *desc, const void *q, const void *k, const void *v, const float *log_decay,
                                  const int32_t *offsets, const float *initial_state, const void *dout, const float *dfinal_state,
                                  const void *saved, void *dq, void *dk, void *dv, float *dinitial_state, void *workspace,
                                  size_t workspace_bytes, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  const wersa_decay_desc &c = *desc;
  if (c.n > 0 && (!q || !k || !v || !dout || !dq || !dk || !dv)) return WERSA_ERR_INVALID_ARG;
  if (!log_decay || (c.packed != 0) != (offsets != nullptr)) return WERSA_ERR_INVALID_ARG;
  if (misaligned(initial_state, 16) || misaligned(dfinal_state, 16) || misaligned(dinitial_state, 16)) return WERSA_ERR_INVALID_ARG;
  const int64_t *gq = strides_of_gradient(c.stride_dq, c.stride_q), *gk = strides_of_gradient(c.stride_dk, c.stride_k), *gv = strides_of_gradient(c.stride_dv, c.stride_v);
  for (const wersa_status ws : {written(gq, c, c.dk), written(gk, c, c.dk), written(gv, c, c.dv)})
    if (ws != WERSA_OK) return ws;
  const bool split = state_slots_of(c) > 0;
  if (split && !saved) return WERSA_ERR_INVALID_ARG;
  if (misaligned(saved, 256) || (split && (!workspace || workspace_bytes < states_bytes(c) || misaligned(workspace, 256))))
    return WERSA_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)hip_stream;
  Walk a{};
  a.log_decay = log_decay;
  a.cache_rows = c.B;
  a.seq = sequences(c, offsets);
  a.heads_first = heads_first(c, a.seq);
  a.H = c.H;
  const Strides sq = strides(c.stride_q, c, c.dk), sk = strides(c.stride_k, c, c.dk), sv = strides(c.stride_v, c, c.dv), so = strides(c.stride_o, c, c.dv);
  const Strides sdq = strides(gq, c, c.dk), sdk = strides(gk, c, c.dk), sdv = strides(gv, c, c.dv);
  // dq: states transposed
  Walk f = a;
  f.q = dout, f.k = v, f.v = k, f.o = dq;
  f.sq = so, f.sk = sv, f.sv = sk, f.so = sdq;
  f.kw = c.dv, f.vw = c.dk, f.si = 1, f.sj = c.dv;
  f.intra = f.inter = c.scale, f.gain = 1.f;
  f.init = split ? (const float *)saved : initial_state;
  f.by_slot = split;
  if (!launch_walk<false>(c, f, st)) return WERSA_ERR_LAUNCH;
  // dv, and the gradient of the state
  a.reverse = true;
  a.intra = c.scale, a.inter = 1.f, a.gain = c.scale;
  a.init = dfinal_state;
  Walk r = a;
  r.q = k, r.k = q, r.v = dout, r.o = dv;
  r.sq = sk, r.sk = sq, r.sv = so, r.so = sdv;
  r.kw = c.dk, r.vw = c.dv, r.si = c.dv, r.sj = 1;
  Outside outside{{}, {}, {}, c.dtype == WERSA_F32 ? 4 : 2};
  bool clear = c.packed && c.n > 0;
  if (clear) outside = Outside{{dq, dk, dv}, {sdq, sdk, sdv}, {c.dk, c.dk, c.dv}, outside.element};
  if (split) {
    r.fin = (float *)workspace;
    if (!launch_walk<true>(c, r, st)) return WERSA_ERR_LAUNCH;
    if (launch_scan(r, (float *)workspace, outside, st)) clear = false;
    r.init = (const float *)workspace;
    r.by_slot = true;
  }
  if (clear) launch_clear(c, a.seq, outside, st);
  r.fin = dinitial_state;
  if (!launch_back(c, r, Back{k, v, dk, dv, sk, sv, sdk, sdv}, st)) return WERSA_ERR_LAUNCH;
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

wersa_status wersa_decay_step(const wersa_decay_desc *desc, const void *q, const void *k, const void *v, const float *log_decay,
                              float *state, const int32_t *slots, int32_t state_slots, void *out, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  const wersa_decay_desc &c = *desc;
  if (c.n != 1 || c.packed || !q || !k || !v || !log_decay || !state || !out) return WERSA_ERR_INVALID_ARG;
  if (state_slots < (slots ? 1 : c.B) || misaligned(state, 16)) return WERSA_ERR_INVALID_ARG;
  if (const wersa_status ws = written(c.stride_o, c, c.dv)) return ws;
  hipStream_t st = (hipStream_t)hip_stream;
  const Step a{q, k, v, out, strides(c.stride_q, c, c.dk), strides(c.stride_k, c, c.dk), strides(c.stride_v, c, c.dv), strides(c.stride_o, c, c.dv), log_decay,
               state, slots, state_slots, c.H, c.dk, c.dv, c.scale};
  auto launch = [&](auto w, auto nt) {
    constexpr int W = decltype(w)::value;
    constexpr bool NT = decltype(nt)::value;
    const dim3 grid((c.dv + W - 1) / W, c.H, c.B);
    if (c.dtype == WERSA_F32) WERSA_STAGE("wersa_decay_step", st, (step_kernel<float, W, NT><<<grid, 256, 0, st>>>(a)));
    else WERSA_STAGE("wersa_decay_step", st, (step_kernel<bf16_t, W, NT><<<grid, 256, 0, st>>>(a)));
  };
  // Whole rows to a workgroup, however few states there are: 16 columns to one instead take 3.0 us for 8 states of 64 x 64 (3.2 with whole rows), 5.4 for 64 of 128 x 128 (4.5), 13.3
  // for 256 (8.3).
  const int64_t bytes = (int64_t)c.B * c.H * c.dk * c.dv * 4;
  auto by_width = [&](auto nt) { c.dv <= 64 ? launch(std::integral_constant<int, 64>{}, nt) : launch(std::integral_constant<int, 128>{}, nt); };
  if (bytes < kCachedStates) by_width(std::false_type{});
  else by_width(std::true_type{});
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

}  // extern "C"
