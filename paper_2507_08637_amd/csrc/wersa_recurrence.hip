// Gated linear recurrence, channel by channel:
//   a_t = sigmoid(gate_t),   h_t = a_t h_{t-1} + (1 - a_t) x_t,   out_t = h_t
// over whole or packed sequences, its derivative, and one token at a time on a cache of states.  With G_t = dL/dh_t = dout_t + a_{t+1} G_{t+1}:
//   dx_t = (1 - a_t) G_t,   dgate_t = G_t (h_{t-1} - x_t) a_t (1 - a_t),   dh_{-1} = a_0 G_0
// Bound by memory: three tensors forwards, five backwards (h is formed again from x and gate, which costs no more bytes than reading it, and keeps its 32 bits).
//
// A span of rows acts on the state before it as h -> A h + H, and spans join as (A', H') after (A, H) = (A A', A' H + H').  A workgroup has a tile of kRows rows and
// 32 lanes' channels; a thread has R neighbouring rows of V channels in registers, from which it forms its (A, H) at once and, when its state is known, its outputs: the
// tensors are read once.  States pass from tile to tile through the workspace: each tile leaves its (A, H) there as soon as it has them, the last one of a group of tiles
// the state behind it, and a tile adds up the state before its group and the (A, H) of the group's tiles before it.  The order is fixed, and so are the bits.
// A tile waits for earlier tiles only, and tiles are handed out in their order by a counter, so that those have begun before it does: every wait ends.
#include "wersa_rows.h"

namespace wersa {
namespace {

constexpr int kThreads = 512, kLanes = 32, kSpans = kThreads / kLanes;   // spans of R rows that a tile has
constexpr int kR = 8, kRows = kSpans * kR;
constexpr int kGroup = 32;                // tiles of a group
constexpr int kWaves = kThreads / 64;
constexpr uint32_t kNone = 0xffffffffu;   // what the workspace holds where nothing has been left; no number has these bits (NaNs are stored with others)
constexpr int kPolls = 1 << 23;           // of a wait, some seconds: only a workspace that is written by others meanwhile comes to this

// V channels of a row: raw bits as they came.
template <typename T, int V> struct Raw { uint32_t u[V * sizeof(T) / 4]; };

struct Job {
  const void *x, *gate, *dout;
  const int32_t *offsets, *slots;
  const float *initial, *dfinal;
  float *final, *dinitial;            // either may be null
  void *out, *dx, *dgate;
  float *saved;                       // [batch entry][tile][C]: the state before each tile; null: not wanted
  uint32_t *counter;                  // the workspace: tiles handed out,
  uint64_t *spans;                    // [chain][tile][channels of a slab]: (A, H),
  uint32_t *states;                   // [chain][group][channels of a slab]: the state behind a group
  int64_t sx[2], sg[2], so[2], sdx[2], sdg[2];
  int B, n, C, tiles, slabs, chains, state_slots, clear;
};

template <typename T> __device__ __forceinline__ void gate_parts(float g, float &a, float &rest) {
  // e^-|g| with one rounding of the exponent for bfloat16 (|g| 2^-24 of it), for float32 with the exponent's low part
  constexpr float kLog2e = 1.44269504f, kLog2eLow = 1.92596299e-8f, kLn2 = 0.69314718f;
  const float m = fabsf(g), t = m * kLog2e;
  float e = __builtin_amdgcn_exp2f(-t);
  if (sizeof(T) == 4 && m < 200.f) e -= e * (kLn2 * (fmaf(m, kLog2e, -t) + m * kLog2eLow));
  const float s = __builtin_amdgcn_rcpf(1.f + e), small = e * s;
  a = g >= 0.f ? s : small;
  rest = g >= 0.f ? small : s;
}
// The smaller of a and 1 - a with the sign of the gate: both of them from one register, each with all its digits.
__device__ __forceinline__ void parts_of(float s, float &a, float &rest) {
  const float small = fabsf(s), big = 1.f - small;
  const bool keeps = !(__float_as_uint(s) >> 31);
  a = keeps ? big : small;
  rest = keeps ? small : big;
}
__device__ __forceinline__ float packed_parts(float g, float a, float rest) { return g >= 0.f ? rest : -a; }

template <typename T, int V> __device__ __forceinline__ float channel(const Raw<T, V> &p, int i) {
  if (sizeof(T) == 4) return __uint_as_float(p.u[i]);
  return __uint_as_float(i & 1 ? p.u[i / 2] & 0xffff0000u : p.u[i / 2] << 16);
}
template <typename T, int V> struct __attribute__((packed, aligned(2))) AnyRaw { Raw<T, V> raw; };
template <typename T, int V> __device__ __forceinline__ Raw<T, V> load_channels(const T *p, int valid) {
  if (valid >= V) return reinterpret_cast<const AnyRaw<T, V> *>(p)->raw;
  Raw<T, V> r;
#pragma unroll
  for (int i = 0; i < (int)(V * sizeof(T) / 4); ++i) r.u[i] = 0;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < valid) r.u[i * (int)sizeof(T) / 4] |= sizeof(T) == 4 ? __float_as_uint(ld(p + i)) : (__float_as_uint(ld(p + i)) >> 16) << 16 * (i & 1);
  return r;
}
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, b16x2)); }
template <typename T, int V> __device__ __forceinline__ void store_channels(T *p, int valid, const float (&v)[V]) {
  if (valid >= V) {
    AnyRaw<T, V> r;
#pragma unroll
    for (int i = 0; i < (int)(V * sizeof(T) / 4); ++i) r.raw.u[i] = sizeof(T) == 4 ? __float_as_uint(v[i]) : two_bf16(v[2 * i], v[2 * i + 1 < V ? 2 * i + 1 : 0]);
    *reinterpret_cast<AnyRaw<T, V> *>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < valid) st(p + i, v[i]);
  }
}

// A span's (A, H).  A below 0: the state before the span does not reach its end (a sequence begins within), whatever it is.
struct Span { float A, H; };
__device__ __forceinline__ float after(const Span &s, float h) { return s.A < 0.f ? s.H : fmaf(s.A, h, s.H); }
__device__ __forceinline__ Span join(const Span &first, const Span &second) {
  if (second.A < 0.f) return second;
  return Span{first.A < 0.f ? -1.f : first.A * second.A, fmaf(second.A, first.H, second.H)};
}

__device__ __forceinline__ uint32_t plain_bits(float v) { return v != v ? 0x7fc00000u : __float_as_uint(v); }
__device__ __forceinline__ void leave(uint64_t *to, const Span &s) {
  __hip_atomic_store(to, (uint64_t)plain_bits(s.H) << 32 | plain_bits(s.A), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void leave(uint32_t *to, float h) { __hip_atomic_store(to, plain_bits(h), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ Span await(const uint64_t *from) {
  for (int i = 0; i < kPolls; ++i) {
    const uint64_t v = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if ((uint32_t)v != kNone) return Span{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
    __builtin_amdgcn_s_sleep(1);
  }
  return Span{-1.f, __uint_as_float(0x7fc00000u)};
}
__device__ __forceinline__ float await(const uint32_t *from) {
  for (int i = 0; i < kPolls; ++i) {
    const uint32_t v = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (v != kNone) return __uint_as_float(v);
    __builtin_amdgcn_s_sleep(1);
  }
  return __uint_as_float(0x7fc00000u);
}

// The state before tile `at` of a chain (channels CH: those of threads below CH), which has left its (A, H): `begin` for the first one, whose (A, H) has it
// in it (the first tile alone reads the initial states, before it leaves anything, so that the final ones may be written over them).
template <int CH>
__device__ __forceinline__ float state_before(const Job &a, int chain, int at, float begin, Span (*joined)[CH]) {
  if (at == 0) return begin;
  const int group = at / kGroup, from = group * kGroup, count = at - from, each = (count + kWaves - 1) / kWaves;
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, i0 = min(wave * each, count), i1 = min(i0 + each, count);
  const uint64_t *spans = a.spans + ((int64_t)chain * a.tiles + from) * CH;
#pragma unroll
  for (int c = lane; c < CH; c += 64) {
    Span s{1.f, 0.f};
    for (int i = i0; i < i1; ++i) s = join(s, await(spans + (int64_t)i * CH + c));
    joined[wave][c] = s;
  }
  float h = 0.f;
  if (threadIdx.x < CH && group > 0) h = await(a.states + ((int64_t)chain * ((a.tiles + kGroup - 1) / kGroup) + group - 1) * CH + threadIdx.x);
  __syncthreads();
  if (threadIdx.x < CH) {
#pragma unroll
    for (int w = 0; w < kWaves; ++w) h = after(joined[w][threadIdx.x], h);
  }
  return h;
}
// What tile `at` leaves to those behind it: (A, H) as soon as it has them; behind the last tile of a group the state, when the one before is known.
template <int CH> __device__ __forceinline__ void leave_span(const Job &a, int chain, int at, const Span &s) {
  if (at % kGroup != kGroup - 1 && at + 1 < a.tiles) leave(a.spans + ((int64_t)chain * a.tiles + at) * CH + threadIdx.x, s);
}
template <int CH> __device__ __forceinline__ void leave_state(const Job &a, int chain, int at, float h) {
  if (at % kGroup == kGroup - 1 && at + 1 < a.tiles) leave(a.states + ((int64_t)chain * ((a.tiles + kGroup - 1) / kGroup) + at / kGroup) * CH + threadIdx.x, h);
}

// Packed sequences: what a row is.
constexpr int kFirst = 1 << 16, kLast = 1 << 17, kOutside = 1 << 18;   // beside the sequence's number
__device__ __forceinline__ int offset_of(const Job &a, int b) { return min(max(a.offsets[b], 0), a.n); }
__device__ __forceinline__ int row_kind(const Job &a, int t) {
  int lo = 0, hi = a.B;     // the last sequence that begins at or before row t
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (offset_of(a, mid) <= t) lo = mid;
    else hi = mid;
  }
  const int begin = offset_of(a, lo), end = offset_of(a, lo + 1);
  if (t < begin || t >= end) return kOutside;
  return lo | (t == begin ? kFirst : 0) | (t == end - 1 ? kLast : 0);
}
__device__ __forceinline__ int64_t slot_of(const Job &a, int b) {   // below 0: none
  if (!a.slots) return b;
  const int s = a.slots[b];
  return s >= 0 && s < a.state_slots ? s : -1;
}

// Which tile of which chain a workgroup has.
__device__ __forceinline__ bool next_tile(const Job &a, int &chain, int &at) {
  __shared__ uint32_t ticket;
  if (a.tiles == 1) {
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    chain = (int)id;
    at = 0;
    return id < a.chains;
  }
  if (threadIdx.x == 0) ticket = atomicAdd(a.counter, 1u) + 1;   // (the counter begins at kNone)
  __syncthreads();
  at = ticket / a.chains;
  chain = ticket % a.chains;
  return at < a.tiles;
}

template <typename T, int V, bool PACKED>
__global__ __launch_bounds__(kThreads, 4) void recurrence_kernel(Job a) {
  constexpr int CH = kLanes * V;
  __shared__ Span part[kSpans][CH], joined[kWaves][CH];
  __shared__ float before[CH];
  __shared__ int kinds[PACKED ? kRows : 1];
  int chain, tile;
  if (!next_tile(a, chain, tile)) return;
  const int batch = chain / a.slabs, c0 = (chain % a.slabs) * CH, lane = threadIdx.x % kLanes, span = threadIdx.x / kLanes;
  const int c = c0 + lane * V, valid = a.C - c, row0 = tile * kRows + span * kR, rows = min(max(a.n - row0, 0), kR);
  const T *x = (const T *)a.x + batch * a.sx[0] + c, *gate = (const T *)a.gate + batch * a.sg[0] + c;
  Raw<T, V> rx[kR], rg[kR];
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    const int64_t t = min(row0 + r, a.n - 1);
    rx[r] = load_channels<T, V>(x + t * a.sx[1], valid);
    rg[r] = load_channels<T, V>(gate + t * a.sg[1], valid);
  }
  if (PACKED) {
    for (int r = threadIdx.x; r < kRows; r += kThreads) kinds[r] = tile * kRows + r < a.n ? row_kind(a, tile * kRows + r) : kOutside;
    __syncthreads();
  }
  float da[kR][V], db[kR][V];
  Span s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) s[i] = Span{1.f, 0.f};
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    const int kind = PACKED ? kinds[span * kR + r] : 0;
    const bool live = PACKED ? !(kind & kOutside) : r < rows;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float keep, rest;
      gate_parts<T>(channel(rg[r], i), keep, rest);
      da[r][i] = live ? keep : 1.f;
      db[r][i] = live ? rest * channel(rx[r], i) : 0.f;
    }
    if (PACKED && (kind & kFirst) && live) {   // what the state before adds, if there is one; the row itself cuts off what came before
      const int64_t slot = a.initial ? slot_of(a, kind & 0xffff) : -1;
      if (slot >= 0) {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i < valid) db[r][i] = fmaf(da[r][i], a.initial[slot * a.C + c + i], db[r][i]);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] = Span{-1.f, db[r][i]};
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        s[i].H = fmaf(da[r][i], s[i].H, db[r][i]);
        if (!PACKED) s[i].A *= da[r][i];
        else s[i].A = s[i].A < 0.f ? s[i].A : s[i].A * da[r][i];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) part[span][lane * V + i] = s[i];
  __syncthreads();
  float begin = 0.f;
  const int mine = c0 + threadIdx.x;
  Span all{1.f, 0.f};
  if (threadIdx.x < CH) {
#pragma unroll
    for (int q = 0; q < kSpans; ++q) {
      const Span p = part[q][threadIdx.x];
      part[q][threadIdx.x] = all;
      all = join(all, p);
    }
    if (!PACKED && tile == 0 && a.initial && mine < a.C) {
      const int64_t slot = slot_of(a, batch);
      if (slot >= 0) begin = a.initial[slot * a.C + mine];
    }
    if (tile == 0) all = Span{-1.f, after(all, begin)};
    leave_span<CH>(a, chain, tile, all);
  }
  const float h0 = state_before<CH>(a, chain, tile, begin, joined);
  if (threadIdx.x < CH) {
    before[threadIdx.x] = h0;
    leave_state<CH>(a, chain, tile, after(all, h0));
    if (a.saved && mine < a.C) a.saved[((int64_t)batch * a.tiles + tile) * a.C + mine] = h0;
  }
  __syncthreads();
  float h[V];
#pragma unroll
  for (int i = 0; i < V; ++i) h[i] = after(part[span][lane * V + i], before[lane * V + i]);
  T *out = (T *)a.out + batch * a.so[0] + c;
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    const int kind = PACKED ? kinds[span * kR + r] : 0;
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = PACKED && (kind & kFirst) ? db[r][i] : fmaf(da[r][i], h[i], db[r][i]);
    if (r < rows) {
      if (!PACKED || !(kind & kOutside)) store_channels<T, V>(out + (row0 + r) * a.so[1], valid, h);
      else if (a.clear) {
        float zeros[V];
#pragma unroll
        for (int i = 0; i < V; ++i) zeros[i] = 0.f;
        store_channels<T, V>(out + (row0 + r) * a.so[1], valid, zeros);
      }
    }
    if (PACKED && (kind & kLast) && a.final) {
      const int64_t slot = slot_of(a, kind & 0xffff);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (slot >= 0 && i < valid) a.final[slot * a.C + c + i] = h[i];
    }
  }
  if (!PACKED && a.final && rows > 0 && row0 + rows == a.n) {   // (rows past the end leave h as it is)
    const int64_t slot = slot_of(a, batch);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (slot >= 0 && i < valid) a.final[slot * a.C + c + i] = h[i];
  }
  if (PACKED && a.final) {   // sequences without rows, the tiles' share of them each
    const int each = (a.B + a.tiles - 1) / a.tiles, end = min((tile + 1) * each, a.B);
    for (int b = tile * each + threadIdx.x / CH; b < end; b += kThreads / CH) {
      const int channel_of = c0 + threadIdx.x % CH;
      const int64_t slot = slot_of(a, b);
      if (offset_of(a, b) >= offset_of(a, b + 1) && slot >= 0 && channel_of < a.C)
        a.final[slot * a.C + channel_of] = a.initial ? a.initial[slot * a.C + channel_of] : 0.f;
    }
  }
}

// Tiles from the last one to the first.  States are by sequence.
template <typename T, int V, bool PACKED>
__global__ __launch_bounds__(kThreads, 4) void recurrence_back_kernel(Job a) {
  constexpr int CH = kLanes * V;
  __shared__ Span part[kSpans][CH], back[kSpans][CH], joined[kWaves][CH];
  __shared__ float before[CH];
  __shared__ int kinds[PACKED ? kRows : 1];
  int chain, at;
  if (!next_tile(a, chain, at)) return;
  const int tile = a.tiles - 1 - at;
  const int batch = chain / a.slabs, c0 = (chain % a.slabs) * CH, lane = threadIdx.x % kLanes, span = threadIdx.x / kLanes;
  const int c = c0 + lane * V, valid = a.C - c, row0 = tile * kRows + span * kR, rows = min(max(a.n - row0, 0), kR);
  const T *x = (const T *)a.x + batch * a.sx[0] + c, *gate = (const T *)a.gate + batch * a.sg[0] + c, *dout = (const T *)a.dout + batch * a.so[0] + c;
  Raw<T, V> rx[kR], rg[kR], rd[kR];
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    const int64_t t = min(row0 + r, a.n - 1);
    rg[r] = load_channels<T, V>(gate + t * a.sg[1], valid);
    rx[r] = load_channels<T, V>(x + t * a.sx[1], valid);
    rd[r] = load_channels<T, V>(dout + t * a.so[1], valid);
  }
  if (PACKED) {
    for (int r = threadIdx.x; r < kRows; r += kThreads) kinds[r] = tile * kRows + r < a.n ? row_kind(a, tile * kRows + r) : kOutside;
    __syncthreads();
  }
  float both[kR][V];    // a and 1 - a of each row (rows that are not there: a = 1)
  Span s[V], b[V];
#pragma unroll
  for (int i = 0; i < V; ++i) s[i] = b[i] = Span{1.f, 0.f};
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    const int kind = PACKED ? kinds[span * kR + r] : 0;
    const bool live = PACKED ? !(kind & kOutside) : r < rows;
    const bool first = PACKED && live && (kind & kFirst);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float g = channel(rg[r], i);
      float keep, rest;
      gate_parts<T>(g, keep, rest);
      both[r][i] = live ? packed_parts(g, keep, rest) : 0.f;
      float add = live ? rest * channel(rx[r], i) : 0.f;
      if (!live) keep = 1.f;
      if (first) {
        if (a.initial && i < valid) add = fmaf(keep, a.initial[(int64_t)(kind & 0xffff) * a.C + c + i], add);
        s[i] = Span{-1.f, add};
      } else {
        s[i].H = fmaf(keep, s[i].H, add);
        if (!PACKED) s[i].A *= keep;
        else s[i].A = s[i].A < 0.f ? s[i].A : s[i].A * keep;
      }
    }
  }
#pragma unroll
  for (int r = kR - 1; r >= 0; --r) {
    const int kind = PACKED ? kinds[span * kR + r] : 0;
    const bool live = PACKED ? !(kind & kOutside) : r < rows;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float keep, rest, d = live ? channel(rd[r], i) : 0.f;
      parts_of(both[r][i], keep, rest);
      if (PACKED && (kind & kLast) && live && a.dfinal && i < valid) d += a.dfinal[(int64_t)(kind & 0xffff) * a.C + c + i];
      b[i].H = keep * (d + b[i].H);
      if (PACKED && live && (kind & kFirst)) b[i].H = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    b[i].A = s[i].A;
    part[span][lane * V + i] = s[i];
    back[span][lane * V + i] = b[i];
  }
  __syncthreads();
  float begin = 0.f;
  const int mine = c0 + threadIdx.x;
  Span all{1.f, 0.f};
  if (threadIdx.x < CH) {
#pragma unroll
    for (int q = kSpans - 1; q >= 0; --q) {
      const Span p = back[q][threadIdx.x];
      back[q][threadIdx.x] = all;
      all = join(all, p);
    }
    if (!PACKED && at == 0 && a.dfinal && mine < a.C) begin = a.dfinal[(int64_t)batch * a.C + mine];
    if (at == 0) all = Span{-1.f, after(all, begin)};
    leave_span<CH>(a, chain, at, all);
    float h = mine < a.C ? a.saved[((int64_t)batch * a.tiles + tile) * a.C + mine] : 0.f;
#pragma unroll
    for (int q = 0; q < kSpans; ++q) {    // the state before each span
      const Span p = part[q][threadIdx.x];
      part[q][threadIdx.x].H = h;
      h = after(p, h);
    }
  }
  const float g0 = state_before<CH>(a, chain, at, begin, joined);
  if (threadIdx.x < CH) {
    before[threadIdx.x] = g0;
    leave_state<CH>(a, chain, at, after(all, g0));
  }
  __syncthreads();
  float h[V], carry[V], earlier[kR][V];    // earlier: the state before each row
#pragma unroll
  for (int i = 0; i < V; ++i) {
    h[i] = part[span][lane * V + i].H;
    carry[i] = after(back[span][lane * V + i], before[lane * V + i]);
  }
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    const int kind = PACKED ? kinds[span * kR + r] : 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float keep, rest;
      parts_of(both[r][i], keep, rest);
      if (PACKED && (kind & kFirst)) h[i] = a.initial && i < valid ? a.initial[(int64_t)(kind & 0xffff) * a.C + c + i] : 0.f;
      earlier[r][i] = h[i];
      h[i] = (PACKED ? !(kind & kOutside) : r < rows) ? fmaf(keep, h[i], rest * channel(rx[r], i)) : h[i];
    }
  }
  T *dx = (T *)a.dx + batch * a.sdx[0] + c, *dgate = (T *)a.dgate + batch * a.sdg[0] + c;
#pragma unroll
  for (int r = kR - 1; r >= 0; --r) {
    const int kind = PACKED ? kinds[span * kR + r] : 0;
    const bool live = PACKED ? !(kind & kOutside) : r < rows;
    float gx[V], gg[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float keep, rest, d = live ? channel(rd[r], i) : 0.f;
      parts_of(both[r][i], keep, rest);
      if (PACKED && (kind & kLast) && live && a.dfinal && i < valid) d += a.dfinal[(int64_t)(kind & 0xffff) * a.C + c + i];
      const float G = d + carry[i];
      gx[i] = live ? rest * G : 0.f;
      carry[i] = live ? keep * G : carry[i];
      gg[i] = live ? gx[i] * keep * (earlier[r][i] - channel(rx[r], i)) : 0.f;
    }
    if (r < rows) {
      store_channels<T, V>(dx + (row0 + r) * a.sdx[1], valid, gx);
      store_channels<T, V>(dgate + (row0 + r) * a.sdg[1], valid, gg);
    }
    if (PACKED && live && (kind & kFirst)) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (a.dinitial && i < valid) a.dinitial[(int64_t)(kind & 0xffff) * a.C + c + i] = carry[i];
        carry[i] = 0.f;
      }
    }
  }
  if (!PACKED && a.dinitial && row0 == 0) {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < valid) a.dinitial[(int64_t)batch * a.C + c + i] = carry[i];
  }
  if (PACKED && a.dinitial) {
    const int each = (a.B + a.tiles - 1) / a.tiles, end = min((tile + 1) * each, a.B);
    for (int q = tile * each + threadIdx.x / CH; q < end; q += kThreads / CH) {
      const int channel_of = c0 + threadIdx.x % CH;
      if (offset_of(a, q) >= offset_of(a, q + 1) && channel_of < a.C)
        a.dinitial[(int64_t)q * a.C + channel_of] = a.dfinal ? a.dfinal[(int64_t)q * a.C + channel_of] : 0.f;
    }
  }
}

// The workspace before a launch that waits in it.
__global__ __launch_bounds__(256) void recurrence_ready_kernel(u32x4 *p, int64_t count) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) p[i] = u32x4{kNone, kNone, kNone, kNone};
}

// No rows at all: states go on as they are.
__global__ __launch_bounds__(256) void recurrence_states_kernel(Job a, const float *from, float *to) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)a.B * a.C; i += (int64_t)gridDim.x * 256) {
    const int64_t slot = slot_of(a, (int)(i / a.C));
    if (slot >= 0) to[slot * a.C + i % a.C] = from ? from[slot * a.C + i % a.C] : 0.f;
  }
}

// One token: four channels to a thread, blockIdx.y the sequence.
template <typename T>
__global__ __launch_bounds__(256) void recurrence_step_kernel(Job a) {
  constexpr int V = 4;
  const int c = (blockIdx.x * 256 + threadIdx.x) * V, valid = a.C - c;
  if (valid <= 0) return;
  const int64_t slot = slot_of(a, blockIdx.y);
  const Raw<T, V> rx = load_channels<T, V>((const T *)a.x + blockIdx.y * a.sx[0] + c, valid), rg = load_channels<T, V>((const T *)a.gate + blockIdx.y * a.sg[0] + c, valid);
  float h[V];
  Raw<float, V> state;
  if (slot >= 0) state = load_channels<float, V>(a.final + slot * a.C + c, valid);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float keep, rest;
    gate_parts<float>(channel(rg, i), keep, rest);
    h[i] = slot >= 0 ? fmaf(keep, channel(state, i), rest * channel(rx, i)) : 0.f;
  }
  if (slot >= 0) store_channels<float, V>(a.final + slot * a.C + c, valid, h);
  store_channels<T, V>((T *)a.out + blockIdx.y * a.so[0] + c, valid, h);
}

// Rows and batch entries of what is written do not share memory.
bool apart(const int64_t *s, int N, int n, int C) {
  if (n > 1 && s[1] < C) return false;
  if (N <= 1) return true;
  const int64_t rows = n > 1 ? (int64_t)(n - 1) * s[1] + C : C;
  return s[0] >= rows || (s[0] >= C && n > 1 && s[1] >= (int64_t)(N - 1) * s[0] + C);
}

wersa_status validate(const wersa_recurrence_desc *c) {
  if (!c) return WERSA_ERR_INVALID_ARG;
  if (c->B < 1 || c->n < 0 || c->C < 1) return WERSA_ERR_INVALID_ARG;
  if (c->dtype != WERSA_F32 && c->dtype != WERSA_BF16) return WERSA_ERR_INVALID_ARG;
  if ((c->packed != 0 && c->packed != 1) || (c->clear != 0 && c->clear != 1)) return WERSA_ERR_INVALID_ARG;
  const int64_t most = (int64_t)1 << 40;
  for (const int64_t *s : {c->stride_x, c->stride_gate})
    for (int i = 0; i < 2; ++i)
      if (s[i] < 0 || s[i] > most) return WERSA_ERR_INVALID_ARG;
  if (c->B > 65535 || c->n > 1 << 30 || c->C > 1 << 20) return WERSA_ERR_UNSUPPORTED;
  const int64_t tiles = (c->n + kRows - 1) / kRows, chains = (int64_t)(c->packed ? 1 : c->B) * ((c->C + kLanes * 2 - 1) / (kLanes * 2));
  if (tiles * chains >= (int64_t)1 << 31) return WERSA_ERR_UNSUPPORTED;
  return WERSA_OK;
}
bool written_apart(const wersa_recurrence_desc &c, std::initializer_list<const int64_t *> strides) {
  for (const int64_t *s : strides)
    if (s[0] < 0 || s[1] < 0 || s[0] > (int64_t)1 << 40 || s[1] > (int64_t)1 << 40 || !apart(s, c.packed ? 1 : c.B, c.n, c.C)) return false;
  return true;
}

// Channels of a lane: 8 bytes of a row, 4 where that is the whole row.
int lane_channels(const wersa_recurrence_desc &c) { return c.dtype == WERSA_BF16 && c.C > kLanes * 2 ? 4 : 2; }

struct Layout {
  size_t spans, states, total;   // byte offsets in the workspace; the counter comes first
  int tiles, slabs, chains;
};
Layout layout_of(const wersa_recurrence_desc &c) {
  Layout l;
  const int ch = lane_channels(c) * kLanes;
  l.tiles = (c.n + kRows - 1) / kRows;
  l.slabs = (c.C + ch - 1) / ch;
  l.chains = l.slabs * (c.packed ? 1 : c.B);
  l.spans = 256;
  l.states = l.spans + (size_t)l.chains * l.tiles * ch * 8;
  l.total = l.states + ((size_t)l.chains * ((l.tiles + kGroup - 1) / kGroup) * ch * 4 + 255) / 256 * 256;
  if (l.tiles <= 1) l.total = 256;
  return l;
}

template <typename F> void by_type(const wersa_recurrence_desc &c, F f) {
  auto packed = [&](auto *type, auto v) {
    if (c.packed) f(type, v, std::true_type{});
    else f(type, v, std::false_type{});
  };
  if (c.dtype == WERSA_F32) packed((float *)nullptr, std::integral_constant<int, 2>{});
  else if (lane_channels(c) == 4) packed((bf16_t *)nullptr, std::integral_constant<int, 4>{});
  else packed((bf16_t *)nullptr, std::integral_constant<int, 2>{});
}

Job job_of(const wersa_recurrence_desc &c, const Layout &l, void *workspace) {
  Job a{};
  a.B = c.B, a.n = c.n, a.C = c.C, a.clear = c.clear, a.state_slots = c.B;
  a.tiles = l.tiles, a.slabs = l.slabs, a.chains = l.chains;
  for (int i = 0; i < 2; ++i) a.sx[i] = c.stride_x[i], a.sg[i] = c.stride_gate[i], a.so[i] = c.stride_o[i], a.sdx[i] = c.stride_dx[i], a.sdg[i] = c.stride_dgate[i];
  char *ws = (char *)workspace;
  a.counter = (uint32_t *)ws;
  if (ws) a.spans = (uint64_t *)(ws + l.spans), a.states = (uint32_t *)(ws + l.states);
  return a;
}

void make_ready(const Layout &l, void *workspace, hipStream_t st) {
  if (l.tiles <= 1) return;
  const int64_t count = (int64_t)(l.total / 16);
  WERSA_STAGE("wersa_recurrence_ready", st, (recurrence_ready_kernel<<<(unsigned)std::min<int64_t>((count + 255) / 256, 1024), 256, 0, st>>>((u32x4 *)workspace, count)));
}

wersa_status pass_states(const Job &a, const float *from, float *to, hipStream_t st) {
  if (to) WERSA_STAGE("wersa_recurrence_states", st,
                      (recurrence_states_kernel<<<(unsigned)std::min<int64_t>(((int64_t)a.B * a.C + 255) / 256, 1024), 256, 0, st>>>(a, from, to)));
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

}  // namespace
}  // namespace wersa

using namespace wersa;

extern "C" {

size_t wersa_recurrence_workspace_bytes(const wersa_recurrence_desc *desc) { return validate(desc) == WERSA_OK ? layout_of(*desc).total : 0; }

size_t wersa_recurrence_saved_bytes(const wersa_recurrence_desc *desc) {
  if (validate(desc) != WERSA_OK) return 0;
  const Layout l = layout_of(*desc);
  return std::max<size_t>(256, ((size_t)(desc->packed ? 1 : desc->B) * l.tiles * desc->C * 4 + 255) / 256 * 256);
}

wersa_status wersa_recurrence_forward(const wersa_recurrence_desc *desc, const void *x, const void *gate, const int32_t *offsets, const float *initial_state,
                                      float *final_state, const int32_t *slots, int32_t state_slots, void *out, void *saved, void *workspace,
                                      size_t workspace_bytes, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  if (!written_apart(*desc, {desc->stride_o}) || (desc->packed != 0) != (offsets != nullptr) || (slots && state_slots < 0)) return WERSA_ERR_INVALID_ARG;
  if (desc->n > 0 && (!x || !gate || !out)) return WERSA_ERR_INVALID_ARG;
  const Layout l = layout_of(*desc);
  if (l.tiles > 1 && (!workspace || workspace_bytes < l.total || misaligned(workspace, 256))) return WERSA_ERR_WORKSPACE;
  if (misaligned(saved, 256)) return WERSA_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)hip_stream;
  Job a = job_of(*desc, l, workspace);
  a.x = x, a.gate = gate, a.offsets = offsets, a.initial = initial_state, a.final = final_state, a.slots = slots, a.out = out, a.saved = (float *)saved;
  if (slots) a.state_slots = state_slots;
  if (desc->n == 0) return pass_states(a, initial_state, final_state, st);
  make_ready(l, workspace, st);
  by_type(*desc, [&](auto *type, auto v, auto packed) {
    typedef typename std::remove_pointer<decltype(type)>::type T;
    WERSA_STAGE("wersa_recurrence", st, (recurrence_kernel<T, decltype(v)::value, decltype(packed)::value><<<grid_of((int64_t)l.chains * l.tiles), kThreads, 0, st>>>(a)));
  });
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

wersa_status wersa_recurrence_backward(const wersa_recurrence_desc *desc, const void *x, const void *gate, const int32_t *offsets, const float *initial_state,
                                       const void *dout, const float *dfinal_state, const void *saved, void *dx, void *dgate, float *dinitial_state,
                                       void *workspace, size_t workspace_bytes, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  if (!written_apart(*desc, {desc->stride_dx, desc->stride_dgate}) || desc->stride_o[0] < 0 || desc->stride_o[1] < 0 || (desc->packed != 0) != (offsets != nullptr))
    return WERSA_ERR_INVALID_ARG;
  if (desc->n > 0 && (!x || !gate || !dout || !saved || !dx || !dgate)) return WERSA_ERR_INVALID_ARG;
  const Layout l = layout_of(*desc);
  if (l.tiles > 1 && (!workspace || workspace_bytes < l.total || misaligned(workspace, 256))) return WERSA_ERR_WORKSPACE;
  if (misaligned(saved, 256)) return WERSA_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)hip_stream;
  Job a = job_of(*desc, l, workspace);
  a.x = x, a.gate = gate, a.offsets = offsets, a.initial = initial_state, a.dout = dout, a.dfinal = dfinal_state, a.saved = (float *)const_cast<void *>(saved);
  a.dx = dx, a.dgate = dgate, a.dinitial = dinitial_state;
  if (desc->n == 0) return pass_states(a, dfinal_state, dinitial_state, st);
  make_ready(l, workspace, st);
  by_type(*desc, [&](auto *type, auto v, auto packed) {
    typedef typename std::remove_pointer<decltype(type)>::type T;
    WERSA_STAGE("wersa_recurrence_back", st, (recurrence_back_kernel<T, decltype(v)::value, decltype(packed)::value><<<grid_of((int64_t)l.chains * l.tiles), kThreads, 0, st>>>(a)));
  });
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

wersa_status wersa_recurrence_step(const wersa_recurrence_desc *desc, const void *x, const void *gate, float *state, const int32_t *slots, int32_t state_slots,
                                   void *out, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  if (desc->n != 1 || desc->packed || !written_apart(*desc, {desc->stride_o}) || !x || !gate || !state || !out || (slots && state_slots < 0)) return WERSA_ERR_INVALID_ARG;
  hipStream_t st = (hipStream_t)hip_stream;
  Job a = job_of(*desc, layout_of(*desc), nullptr);
  a.x = x, a.gate = gate, a.final = state, a.slots = slots, a.out = out;
  if (slots) a.state_slots = state_slots;
  const dim3 grid((desc->C + 1023) / 1024, desc->B);
  if (desc->dtype == WERSA_F32) WERSA_STAGE("wersa_recurrence_step", st, (recurrence_step_kernel<float><<<grid, 256, 0, st>>>(a)));
  else WERSA_STAGE("wersa_recurrence_step", st, (recurrence_step_kernel<bf16_t><<<grid, 256, 0, st>>>(a)));
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

}  // extern "C"
