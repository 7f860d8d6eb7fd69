// Rows of an embedding for tokens, and the gradient of its weights by sorted tokens:
//   out[i] = scale weight[token_i],   dweight[v] = scale (sum of dout[i] over the places i that hold token v)
// A token outside 0 .. vocabulary - 1 has no row: zeros, and no part in the gradient.
//
// The gradient.  Places are sorted by token, stably (radix sort, up to nine bits a pass), and the sorted list is cut into pieces of equal length, however unequal the tokens'
// counts: each piece adds up its rows of dout in order, a token that lies within a piece goes straight to dweight, what a piece has of a token that goes on
// beyond it goes to the workspace and is added up afterwards in the order of the pieces.  dout is read once, dweight written once, no float atomics.
#include "wersa_rows.h"

namespace wersa {
namespace {

constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kRowsAhead = 2;         // rows of out that a thread has in flight
constexpr size_t kCached = (size_t)256 << 20;   // bytes that the last-level cache holds: a larger dout, read once, is read past it
constexpr int kClearRows = 16;        // rows that a workgroup of the clearing step looks at

struct SortPlan {
  int64_t tile;       // places of a workgroup, a multiple of kSortThreads
  int tiles, passes, bits;   // bits of a pass's digit
};
// A workgroup for each compute unit, whose counts each of them adds up by itself.  400000 tokens, two passes: 52 us with 64 workgroups, 36 with 256.
SortPlan sort_plan(int64_t tokens, int vocabulary) {
  SortPlan p;
  int bits = 1;
  while ((int64_t)1 << bits < vocabulary) ++bits;
  p.passes = (bits + kDigitBits - 1) / kDigitBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  const int64_t each = (tokens + 255) / 256;
  p.tile = std::min<int64_t>((each + kSortThreads - 1) / kSortThreads * kSortThreads, 1 << 19);
  p.tile = std::max<int64_t>(p.tile, kSortThreads);
  p.tiles = (int)((tokens + p.tile - 1) / p.tile);
  return p;
}

// A thread has four neighbouring columns, or two times four, so that rows of either type are read and written in whole lines.
template <typename T> struct Quad { uint32_t u[sizeof(T)]; };
template <typename T> struct __attribute__((packed, aligned(2))) AnyQuad { Quad<T> q; };
typedef uint32_t words2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> __device__ __forceinline__ float value(const Quad<T> &q, int i) {
  if (sizeof(T) == 4) return __uint_as_float(q.u[i]);
  return __uint_as_float(i & 1 ? q.u[i / 2] & 0xffff0000u : q.u[i / 2] << 16);
}
template <bool PAST, typename T> __device__ __forceinline__ Quad<T> load_quad(const T *row, int col, int cols) {
  Quad<T> q = {};
  if (col + 4 <= cols) {
    if constexpr (sizeof(T) == 4) {
      const words4 *p = reinterpret_cast<const words4 *>(row + col);
      const words4 v = PAST ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
      for (int i = 0; i < 4; ++i) q.u[i] = v[i];
    } else {
      const words2 *p = reinterpret_cast<const words2 *>(row + col);
      const words2 v = PAST ? __builtin_nontemporal_load(p) : *p;
      q.u[0] = v[0], q.u[1] = v[1];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + i < cols) q.u[i * (int)sizeof(T) / 4] |= sizeof(T) == 4 ? __float_as_uint(ld(row + col + i)) : (__float_as_uint(ld(row + col + i)) >> 16) << 16 * (i & 1);
  }
  return q;
}
template <typename T> __device__ __forceinline__ void store_quad(T *row, int col, int cols, const float (&v)[4], float scale) {
  if (col + 4 <= cols) {
    if constexpr (sizeof(T) == 4) {
      words4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i] * scale);
      *reinterpret_cast<words4 *>(row + col) = w;
    } else {
      words2 w;
#pragma unroll
      for (int i = 0; i < 2; ++i) w[i] = (uint32_t)f32_to_bf16(v[2 * i] * scale) | (uint32_t)f32_to_bf16(v[2 * i + 1] * scale) << 16;
      *reinterpret_cast<words2 *>(row + col) = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + i < cols) st(row + col + i, v[i] * scale);
  }
}
template <typename T> constexpr int kQuads = sizeof(T) == 4 ? 1 : 2;   // of a thread: 16 bytes of a row of out

// Threads of a row: one for each 16 bytes of out, as a power of two, 8 at least and a workgroup at most.
int lanes_of(const wersa_embedding_desc &c) {
  const int64_t pieces = ((int64_t)c.cols * (c.dtype == WERSA_F32 ? 4 : 2) + 15) / 16;
  int lanes = 8;
  while (lanes < 256 && lanes < pieces) lanes *= 2;
  return lanes;
}
// Sorted places of a piece: as many as leave two workgroups to a compute unit (longer pieces have fewer parts to join), between 8 and 128.
// 31999 places of 512 columns in float32: sums 21 us and joins 10; with four workgroups to a unit 22 and 12; with one, before long runs were shared out, 27 and 13.5 for 20 and 20.
int piece_of(const wersa_embedding_desc &c) {
  const int lanes = lanes_of(c), e = c.dtype == WERSA_F32 ? 4 : 8;
  const int64_t slabs = (c.cols + lanes * e - 1) / (lanes * e), each = c.tokens * lanes * slabs / (256 * 512);
  int piece = 8;
  while (piece < 128 && piece * 2 <= each) piece *= 2;
  return piece;
}

struct Workspace {
  size_t count, counts, keys[2], places[2], partial, total;   // byte offsets
};
Workspace workspace_of(const wersa_embedding_desc &c) {
  const SortPlan p = sort_plan(c.tokens, c.vocabulary);
  Workspace w;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) / 256 * 256;
    return was;
  };
  w.count = take(4);
  w.counts = take((size_t)p.tiles * kDigits * 4);
  for (int i = 0; i < 2; ++i) w.keys[i] = take((size_t)c.tokens * 4), w.places[i] = take((size_t)c.tokens * 4);
  w.partial = take((size_t)((c.tokens + piece_of(c) - 1) / piece_of(c)) * 2 * c.cols * 4);
  w.total = at;
  return w;
}

// Where a pass reads: the tokens themselves, or what the pass before it left.
struct Source {
  const void *tokens;
  int token_bytes, vocabulary;
  const uint32_t *keys, *places;    // null: the tokens
};
__device__ __forceinline__ bool read_source(const Source &s, int64_t i, uint32_t &key, uint32_t &place) {
  if (s.keys) {
    key = s.keys[i];
    place = s.places[i];
    return true;
  }
  const int64_t t = s.token_bytes == 8 ? ((const int64_t *)s.tokens)[i] : (int64_t)((const int32_t *)s.tokens)[i];
  key = (uint32_t)t;
  place = (uint32_t)i;
  return t >= 0 && t < s.vocabulary;
}

// counts[tile][digit]
__global__ __launch_bounds__(kSortThreads) void embedding_count_kernel(Source s, const uint32_t *count, int64_t tokens, int64_t tile, int shift, int digits, uint32_t *counts) {
  __shared__ uint32_t hist[kDigits];
  for (int d = threadIdx.x; d < digits; d += kSortThreads) hist[d] = 0;
  __syncthreads();
  const int64_t n = s.keys ? (int64_t)*count : tokens, begin = blockIdx.x * tile, end = min(begin + tile, n);
  for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads) {
    uint32_t key, place;
    if (read_source(s, i, key, place)) atomicAdd(&hist[(key >> shift) & (digits - 1)], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads) counts[(int64_t)blockIdx.x * digits + d] = hist[d];
}

// Places go to where their digit begins, behind those of earlier tiles, of earlier waves and of earlier lanes: a stable order.  A wave takes 64 neighbours at a
// time; the lanes of one digit find each other by one ballot per bit.
__global__ __launch_bounds__(kSortThreads) void embedding_scatter_kernel(Source s, uint32_t *count, int64_t tokens, int64_t tile, int shift, int bits, const uint32_t *counts,
                                                                         uint32_t *keys, uint32_t *places) {
  __shared__ uint32_t start[kSortWaves][kDigits];
  __shared__ uint32_t waves_sum[kSortWaves], counted[2][kSortThreads];
  const int digits = 1 << bits, wave = threadIdx.x / 64, lane = threadIdx.x & 63;
  for (int i = threadIdx.x; i < kSortWaves * kDigits; i += kSortThreads) (&start[0][0])[i] = 0;
  const int64_t n = s.keys ? (int64_t)*count : tokens;
  const int64_t share = tile / kSortWaves, begin = blockIdx.x * tile + wave * share, end = min(begin + share, n);
  __syncthreads();
  for (int64_t i = begin + lane; i < end; i += 64) {
    uint32_t key, place;
    if (read_source(s, i, key, place)) atomicAdd(&start[wave][(key >> shift) & (digits - 1)], 1u);
  }
  // of each digit: all places, and those of earlier tiles, the tiles shared out among as many threads as there are for a digit
  uint32_t all = 0, before = 0;
  {
    const int digit = threadIdx.x & (digits - 1), shares = kSortThreads >> bits;
#pragma unroll 8
    for (int t = threadIdx.x >> bits; t < (int)gridDim.x; t += shares) {
      const uint32_t c = counts[(int64_t)t * digits + digit];
      all += c;
      before += t < (int)blockIdx.x ? c : 0;
    }
    counted[0][threadIdx.x] = all;
    counted[1][threadIdx.x] = before;
    __syncthreads();
    all = before = 0;
    if ((int)threadIdx.x < digits)
      for (int i = threadIdx.x; i < kSortThreads; i += digits) all += counted[0][i], before += counted[1][i];
  }
  uint32_t upto = all;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t v = __shfl_up(upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 63) waves_sum[wave] = upto;
  __syncthreads();
  uint32_t lower = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    lower += w < wave ? waves_sum[w] : 0;
    sum += waves_sum[w];
  }
  if (!s.keys && blockIdx.x == 0 && threadIdx.x == 0) *count = sum;   // places that hold a row's token
  if ((int)threadIdx.x < digits) {
    uint32_t at = lower + upto - all + before;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = start[w][threadIdx.x];
      start[w][threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int64_t i0 = begin; i0 < end; i0 += 64) {   // (the same for a wave's lanes)
    uint32_t key = 0, place = 0;
    const bool have = i0 + lane < end && read_source(s, i0 + lane, key, place);
    const uint32_t digit = (key >> shift) & (digits - 1);
    uint64_t same = __ballot(have);
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = __ballot((digit >> b) & 1);
      same &= (digit >> b) & 1 ? set : ~set;
    }
    if (have) {
      const int first = __ffsll((unsigned long long)same) - 1;
      const uint32_t rank = __popcll(same & (((uint64_t)1 << lane) - 1));
      uint32_t at = 0;
      if (lane == first) at = atomicAdd(&start[wave][digit], (uint32_t)__popcll(same));
      at = __shfl(at, first) + rank;
      keys[at] = key;
      places[at] = place;
    }
  }
}

// First place in the sorted list whose token is not below `key`.
__device__ __forceinline__ int64_t lower_bound(const uint32_t *keys, int64_t n, uint32_t key) {
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (keys[mid] < key) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

struct SumJob {
  const uint32_t *count, *keys, *places;
  const void *dout;
  void *dweight;
  float *partial;            // [piece][2][cols]: of a token that began before the piece, of one that goes on behind it
  int64_t stride_out, stride_weight;
  int cols, vocabulary, piece;
  float scale;
};

// Rows of dweight whose token is nowhere: zeros, kClearRows rows to a workgroup.  They need the sorted list only, and lie in the launch of the sums: sorting, sums and zeros
// with the lookup 458 us for 467 with a launch of their own (131072 places, 65536 rows of 2048 columns), 74 for 81 (31999, 50021 of 512).
template <typename W> __device__ __forceinline__ void clear_rows(const SumJob &a, int64_t row0) {
  __shared__ bool there[kClearRows];
  const int64_t n = a.count ? (int64_t)*a.count : 0;
  if (threadIdx.x < kClearRows) {
    const int64_t row = row0 + threadIdx.x;
    bool found = row >= a.vocabulary;
    if (!found && n > 0) {
      const int64_t at = lower_bound(a.keys, n, (uint32_t)row);
      found = at < n && a.keys[at] == (uint32_t)row;
    }
    there[threadIdx.x] = found;
  }
  __syncthreads();
  constexpr int E = 16 / sizeof(W);
  float zeros[E];
#pragma unroll
  for (int i = 0; i < E; ++i) zeros[i] = 0.f;
  for (int r = 0; r < kClearRows; ++r)
    if (!there[r])
      for (int col = threadIdx.x * E; col < a.cols; col += 256 * E) store_piece<W, E>((W *)a.dweight + (row0 + r) * a.stride_weight, col, a.cols, zeros);
}

// LANES threads to a piece; blockIdx.z: further columns, the last one the rows that are cleared.  PAST: dout is more than the last-level cache holds.  Bound by memory: 131072 places of 2048 columns in bf16,
// sums alone, 171 to 177 us, 744 MB at 4.3 TB/s; with 16 rows ahead 251, with 4 178; dout through the caches 209.
template <typename T, typename W, int LANES, bool PAST>
__global__ __launch_bounds__(256) void embedding_sum_kernel(SumJob a) {
  constexpr int Q = kQuads<T>, AHEAD = 8;
  const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (blockIdx.z == gridDim.z - 1) {
    if (block * kClearRows < a.vocabulary) clear_rows<W>(a, block * kClearRows);
    return;
  }
  if (!a.count) return;
  const int64_t n = *a.count, piece = block * (256 / LANES) + threadIdx.x / LANES, begin = piece * a.piece, end = min(begin + a.piece, n);
  const int col = (blockIdx.z * LANES * Q + threadIdx.x % LANES) * 4;
  if (begin >= end || col >= a.cols) return;
  float acc[Q][4] = {};
  uint32_t key = a.keys[begin];
  bool head = begin > 0 && a.keys[begin - 1] == key;
  const bool on = end < n && a.keys[end] == a.keys[end - 1];
  float *partial = a.partial + piece * 2 * a.cols;
  const auto put = [&](bool tail) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int at = col + q * LANES * 4;
      if (head) store_quad<float>(partial, at, a.cols, acc[q], 1.f);
      else if (tail) store_quad<float>(partial + a.cols, at, a.cols, acc[q], 1.f);
      else store_quad<W>((W *)a.dweight + (int64_t)key * a.stride_weight, at, a.cols, acc[q], a.scale);
    }
  };
  for (int64_t i0 = begin; i0 < end; i0 += AHEAD) {
    uint32_t k[AHEAD];
    Quad<T> row[AHEAD][Q];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int64_t at = min(i0 + i, end - 1);
      k[i] = a.keys[at];
      const T *from = (const T *)a.dout + (int64_t)a.places[at] * a.stride_out;
#pragma unroll
      for (int q = 0; q < Q; ++q) row[i][q] = load_quad<PAST, T>(from, col + q * LANES * 4, a.cols);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (i0 + i < end) {
        if (k[i] != key) {
          put(false);
          head = false;
          key = k[i];
#pragma unroll
          for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[q][j] = 0.f;
        }
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[q][j] += value(row[i][q], j);
      }
    }
  }
  put(on);
}

// Tokens that go on over boundaries of pieces, each at its first such boundary: the parts in the order of the pieces.  A workgroup looks at kJoinWaves boundaries and 256
// columns: a wave joins the token of its own one where that has up to kAlone parts, and all of them share out what has more.
// Bound by the longest run of parts: 31999 places 6.6 to 6.8 us.
constexpr int kJoinWaves = 8, kAlone = 32;
struct Parts { int64_t p; int count; uint32_t key; };
__device__ __forceinline__ void add_parts(const SumJob &a, const Parts &of, int from, int to, int col, float (&acc)[4]) {
  constexpr int AHEAD = 16;
  for (int i0 = from; i0 < to; i0 += AHEAD) {
    Quad<float> row[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int part = min(i0 + i, to - 1);
      row[i] = load_quad<false, float>(a.partial + (part == 0 ? (of.p - 1) * 2 + 1 : (of.p - 1 + part) * 2) * a.cols, col, a.cols);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (i0 + i < to) {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += value(row[i], j);
      }
    }
  }
}
template <typename W>
__global__ __launch_bounds__(kJoinWaves * 64) void embedding_join_kernel(SumJob a) {
  __shared__ Parts long_ones[kJoinWaves];
  __shared__ int many[kJoinWaves];
  __shared__ float sums[kJoinWaves][4][64];
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, col = (blockIdx.z * 64 + lane) * 4;
  const int64_t n = *a.count, p = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kJoinWaves + wave + 1, at = p * a.piece;
  Parts mine{p, 0, 0};
  if (at < n) {
    mine.key = a.keys[at];
    if (a.keys[at - 1] == mine.key && (at <= a.piece || a.keys[at - a.piece - 1] != mine.key)) {
      mine.count = 1;   // the tail of piece p - 1 and the heads of p, p + 1 ... as far as the token goes
      for (bool more = true; more;) {
        const int64_t next = at + (int64_t)(mine.count - 1 + lane) * a.piece;
        const uint64_t same = __ballot(next < n && a.keys[next < n ? next : at] == mine.key);
        more = same == ~0ull;
        mine.count += more ? 64 : __ffsll((unsigned long long)~same) - 1;
      }
    }
  }
  if (lane == 0) long_ones[wave] = mine, many[wave] = mine.count > kAlone;
  if (mine.count > 0 && mine.count <= kAlone) {
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    add_parts(a, mine, 0, mine.count, col, acc);
    store_quad<W>((W *)a.dweight + (int64_t)mine.key * a.stride_weight, col, a.cols, acc, a.scale);
  }
  __syncthreads();
  for (int w = 0; w < kJoinWaves; ++w) {
    if (!many[w]) continue;   // (the same for every thread)
    const Parts of = long_ones[w];
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    add_parts(a, of, (int)((int64_t)of.count * wave / kJoinWaves), (int)((int64_t)of.count * (wave + 1) / kJoinWaves), col, acc);
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[j] = 0.f;
#pragma unroll
        for (int v = 0; v < kJoinWaves; ++v) acc[j] += sums[v][j][lane];
      }
      store_quad<W>((W *)a.dweight + (int64_t)of.key * a.stride_weight, col, a.cols, acc, a.scale);
    }
    __syncthreads();
  }
}

// LANES threads to a row of out, kRowsAhead rows to a thread.  Bound by memory: 131072 places of 2048 columns, bf16 from float32, 199 to 219 us: 512 MiB are written, and 663 MB
// read past the L2 caches, each of which has a copy of the rows that come often (the distinct rows have 213 MB).
template <typename T, typename W, int LANES>
__global__ __launch_bounds__(256) void embedding_kernel(Source s, const void *weight, void *out, int64_t tokens, int64_t stride_weight, int64_t stride_out, int cols, float scale) {
  constexpr int Q = kQuads<T>, GROUPS = 256 / LANES;
  const int64_t row0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (GROUPS * kRowsAhead) + threadIdx.x / LANES;
  uint32_t key[kRowsAhead], place;
  bool have[kRowsAhead];
#pragma unroll
  for (int r = 0; r < kRowsAhead; ++r) have[r] = row0 + r * GROUPS < tokens && read_source(s, row0 + r * GROUPS, key[r], place);
  for (int col = threadIdx.x % LANES * 4; col < cols; col += LANES * Q * 4) {
    Quad<W> q[kRowsAhead][Q];
#pragma unroll
    for (int r = 0; r < kRowsAhead; ++r)
#pragma unroll
      for (int i = 0; i < Q; ++i)
        q[r][i] = load_quad<false, W>((const W *)weight + (have[r] ? (int64_t)key[r] : 0) * stride_weight, col + i * LANES * 4, have[r] ? cols : 0);
#pragma unroll
    for (int r = 0; r < kRowsAhead; ++r)
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = have[r] ? value(q[r][i], j) : 0.f;
        if (row0 + r * GROUPS < tokens) store_quad<T>((T *)out + (row0 + r * GROUPS) * stride_out, col + i * LANES * 4, cols, v, have[r] ? scale : 1.f);
      }
  }
}

wersa_status validate(const wersa_embedding_desc *c) {
  if (!c) return WERSA_ERR_INVALID_ARG;
  if (c->tokens < 0 || c->vocabulary < 1 || c->cols < 1) return WERSA_ERR_INVALID_ARG;
  for (const int32_t t : {c->dtype, c->weight_dtype})
    if (t != WERSA_F32 && t != WERSA_BF16) return WERSA_ERR_INVALID_ARG;
  if (c->token_bytes != 4 && c->token_bytes != 8) return WERSA_ERR_INVALID_ARG;
  if ((c->tokens > 1 && c->stride_out < c->cols) || (c->vocabulary > 1 && c->stride_weight < c->cols)) return WERSA_ERR_INVALID_ARG;
  if (c->tokens >= (int64_t)1 << 31 || c->cols > 1 << 20) return WERSA_ERR_UNSUPPORTED;
  return WERSA_OK;
}

// Types of out and of the weights, and the threads of a row.
template <typename F> void by_types(const wersa_embedding_desc &c, F f) {
  auto lanes = [&](auto *t, auto *w) {
    switch (lanes_of(c)) {
      case 8: return f(t, w, std::integral_constant<int, 8>{});
      case 16: return f(t, w, std::integral_constant<int, 16>{});
      case 32: return f(t, w, std::integral_constant<int, 32>{});
      case 64: return f(t, w, std::integral_constant<int, 64>{});
      case 128: return f(t, w, std::integral_constant<int, 128>{});
      default: return f(t, w, std::integral_constant<int, 256>{});
    }
  };
  float *f32 = nullptr;
  bf16_t *b16 = nullptr;
  if (c.dtype == WERSA_F32) c.weight_dtype == WERSA_F32 ? lanes(f32, f32) : lanes(f32, b16);
  else c.weight_dtype == WERSA_F32 ? lanes(b16, f32) : lanes(b16, b16);
}

}  // namespace
}  // namespace wersa

using namespace wersa;

extern "C" {

wersa_status wersa_embedding_forward(const wersa_embedding_desc *desc, const void *tokens, const void *weight, void *out, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  if (desc->tokens == 0) return WERSA_OK;
  if (!tokens || !weight || !out) return WERSA_ERR_INVALID_ARG;
  hipStream_t st = (hipStream_t)hip_stream;
  const Source s{tokens, desc->token_bytes, desc->vocabulary, nullptr, nullptr};
  by_types(*desc, [&](auto *t, auto *w, auto lanes) {
    typedef typename std::remove_pointer<decltype(t)>::type T;
    typedef typename std::remove_pointer<decltype(w)>::type W;
    constexpr int L = decltype(lanes)::value;
    WERSA_STAGE("wersa_embedding", st, (embedding_kernel<T, W, L><<<grid_of((desc->tokens + 256 / L * kRowsAhead - 1) / (256 / L * kRowsAhead)), 256, 0, st>>>(
        s, weight, out, desc->tokens, desc->stride_weight, desc->stride_out, desc->cols, desc->scale)));
  });
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

size_t wersa_embedding_workspace_bytes(const wersa_embedding_desc *desc) { return validate(desc) == WERSA_OK ? workspace_of(*desc).total : 0; }

wersa_status wersa_embedding_backward(const wersa_embedding_desc *desc, const void *tokens, const void *dout, void *dweight, void *workspace,
                                      size_t workspace_bytes, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  if (!dweight || (desc->tokens > 0 && (!tokens || !dout))) return WERSA_ERR_INVALID_ARG;
  if (desc->tokens > 0 && (!workspace || workspace_bytes < wersa_embedding_workspace_bytes(desc) || misaligned(workspace, 256))) return WERSA_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)hip_stream;
  char *ws = (char *)workspace;
  const SortPlan p = sort_plan(desc->tokens, desc->vocabulary);
  const Workspace at = workspace_of(*desc);
  uint32_t *count = desc->tokens ? (uint32_t *)(ws + at.count) : nullptr, *counts = (uint32_t *)(ws + at.counts);
  Source s{tokens, desc->token_bytes, desc->vocabulary, nullptr, nullptr};
  for (int pass = 0; pass < p.passes && desc->tokens > 0; ++pass) {
    uint32_t *keys = (uint32_t *)(ws + at.keys[pass & 1]), *places = (uint32_t *)(ws + at.places[pass & 1]);
    WERSA_STAGE("wersa_embedding_count", st, (embedding_count_kernel<<<p.tiles, kSortThreads, 0, st>>>(s, count, desc->tokens, p.tile, pass * p.bits, 1 << p.bits, counts)));
    WERSA_STAGE("wersa_embedding_scatter", st, (embedding_scatter_kernel<<<p.tiles, kSortThreads, 0, st>>>(s, count, desc->tokens, p.tile, pass * p.bits, p.bits, counts, keys, places)));
    s.keys = keys, s.places = places;
  }
  const SumJob a{count, s.keys, s.places, dout, dweight, (float *)(ws + at.partial), desc->stride_out, desc->stride_weight, desc->cols, desc->vocabulary, piece_of(*desc), desc->scale};
  by_types(*desc, [&](auto *t, auto *w, auto lanes) {
    typedef typename std::remove_pointer<decltype(t)>::type T;
    typedef typename std::remove_pointer<decltype(w)>::type W;
    constexpr int L = decltype(lanes)::value, E = 4 * kQuads<T>;
    const int64_t pieces = (desc->tokens + a.piece - 1) / a.piece, clears = ((int64_t)desc->vocabulary + kClearRows - 1) / kClearRows;
    dim3 grid = grid_of(std::max((pieces + 256 / L - 1) / (256 / L), clears));
    grid.z = (desc->cols + L * E - 1) / (L * E) + 1;
    const auto sum = (size_t)desc->tokens * desc->cols * sizeof(T) > kCached ? embedding_sum_kernel<T, W, L, true> : embedding_sum_kernel<T, W, L, false>;
    WERSA_STAGE("wersa_embedding_sum", st, (sum<<<grid, 256, 0, st>>>(a)));
    if (pieces > 1) {
      dim3 joins = grid_of((pieces - 1 + kJoinWaves - 1) / kJoinWaves);
      joins.z = (desc->cols + 255) / 256;
      WERSA_STAGE("wersa_embedding_join", st, (embedding_join_kernel<W><<<joins, kJoinWaves * 64, 0, st>>>(a)));
    }
  });
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

}  // extern "C"
