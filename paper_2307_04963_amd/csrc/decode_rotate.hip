// Heads turned by their positions, alone or on the way into the paged cache, and the
// cache's reordering behind a choice of beams.
//
// Rotation of the pair (a, b) by t = position * frequency: a cos t - b sin t,
// b cos t + a sin t.  t in float32 loses 0.06 at position 10^6, so it is float64 until
// it is reduced to an eighth of a turn around the nearest quarter; sine and cosine of
// that are Taylor polynomials in float32 (remainders below 2^-28 at pi / 4).
//
// Bound by HBM: every value is read and written once (measured: 251 MB of float32 39 us, 6.4 TB/s; prompts of 6000
// rows into the cache, 157 MB, 26 us; one token of 32 heads 2.0 us, a launch; units of 8 or 4 bytes 4 to 5.5 TB/s,
// odd ones 1.7 in bf16).  A workgroup takes a tile of rows;
// their cosines and sines are made once into LDS for all of a row's heads, then a lane
// takes 16 bytes (of each half, or of neighbours), at any alignment.
#include "decode_dev.hpp"

namespace dycl {
namespace k {

namespace {

constexpr int kThreads = 256, kMaxRows = 64, kTableSize = 2048;

// (cos, sin) of position * frequency
__device__ __forceinline__ float2 turn(int32_t position, double frequency) {
  double t = static_cast<double>(position) * frequency * 0.15915494309189533577;   // in turns
  t -= rint(t);
  const double quarter = rint(t * 4.0);
  const float x = static_cast<float>((t - quarter * 0.25) * 6.283185307179586477);
  const float x2 = x * x;
  float s = __builtin_fmaf(x2, 1.f / 362880.f, -1.f / 5040.f);
  s = __builtin_fmaf(x2, s, 1.f / 120.f);
  s = __builtin_fmaf(x2, s, -1.f / 6.f);
  s = __builtin_fmaf(x2 * x, s, x);
  float c = __builtin_fmaf(x2, -1.f / 3628800.f, 1.f / 40320.f);
  c = __builtin_fmaf(x2, c, -1.f / 720.f);
  c = __builtin_fmaf(x2, c, 1.f / 24.f);
  c = __builtin_fmaf(x2, c, -0.5f);
  c = __builtin_fmaf(x2, c, 1.f);
  const int n = static_cast<int>(quarter) & 3;
  const float cc = n & 1 ? s : c, ss = n & 1 ? c : s;
  return make_float2(n == 1 || n == 2 ? -cc : cc, n >= 2 ? -ss : ss);
}

// x / d for x * d < 2^32, m = ceil(2^32 / d) (d > 1; 0 stands for d = 1, 1 for quotients that are all 0)
struct Divide {
  uint32_t m;
  explicit Divide(int d, bool below = false) : m(below ? 1 : d > 1 ? static_cast<uint32_t>(((uint64_t(1) << 32) + d - 1) / d) : 0) {}
  __device__ int operator()(int x) const { return m ? static_cast<int>(__umulhi(static_cast<uint32_t>(x), m)) : x; }
};

struct Units {
  int rows;                      // of a tile
  int turned, copied, plain;     // units of a head's turned and other values, of a head of v
  int of_q, of_row;              // units of q's heads, of a whole row
  Divide row, head, v_head, pair;
};

// cosines and sines of a tile's rows
__device__ __forceinline__ void make_table(const RotateArgs& p, const Units& u, int64_t r0, int rows, float2* table) {
  for (int i = threadIdx.x; i < rows * p.pairs; i += kThreads) {
    const int r = u.pair(i);
    float2 cs = turn(p.positions[r0 + r], p.frequencies[i - r * p.pairs]);
    cs.x *= p.magnitude;
    cs.y *= p.magnitude * p.sign;
    table[i] = cs;
  }
}

template <bool F32>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs p, Units u) {
  __shared__ float2 table[kTableSize];
  __shared__ int64_t pages[kMaxRows];          // page of the row's token, -1: none
  __shared__ int32_t places[kMaxRows];
  const int t = threadIdx.x, per_head = u.turned + u.copied;
  constexpr size_t size = F32 ? 4 : 2;
  constexpr int W = kWide<F32>;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * u.rows; r0 < p.n; r0 += static_cast<int64_t>(gridDim.x) * u.rows) {
    const int rows = static_cast<int>(min(p.n - r0, static_cast<int64_t>(u.rows)));
    for (int r = t; r < rows; r += kThreads) {
      const int32_t at = p.positions[r0 + r];
      places[r] = at;
      pages[r] = p.k ? page_of(p.cache, p.sequence ? p.sequence[r0 + r] : r0 + r, at) : -1;
    }
    make_table(p, u, r0, rows, table);
    __syncthreads();
    for (int i = t; i < rows * u.of_row; i += kThreads) {
      const int r = u.row(i);
      int w = i - r * u.of_row;
      const char* from;
      char* to;
      bool to_cache = true, turned;
      int first, count, head;
      if (w < u.of_q) {
        head = u.head(w);
        w -= head * per_head;
        from = static_cast<const char*>(p.q) + (static_cast<size_t>(r0 + r) * p.ldq + static_cast<size_t>(head) * p.dim) * size;
        to = static_cast<char*>(p.q_out) + (static_cast<size_t>(r0 + r) * p.ldo + static_cast<size_t>(head) * p.dim) * size;
        to_cache = false;
        turned = w < u.turned;
      } else {
        if (pages[r] < 0) continue;
        w -= u.of_q;
        const bool is_v = w >= p.cache.heads * per_head;
        if (is_v) {
          w -= p.cache.heads * per_head;
          head = u.v_head(w);
          w -= head * u.plain;
        } else {
          head = u.head(w);
          w -= head * per_head;
        }
        from = static_cast<const char*>(is_v ? p.v : p.k) +
               (static_cast<size_t>(r0 + r) * (is_v ? p.ldv : p.ldk) + static_cast<size_t>(head) * p.dim) * size;
        const int64_t slot = places[r] & ((1 << p.cache.page_shift) - 1);
        to = reinterpret_cast<char*>((is_v ? p.cache.values : p.cache.keys) + token_at(p.cache, pages[r], head, slot));
        turned = !is_v && w < u.turned;
        if (is_v) w += u.turned;               // (counted as copied from the head's first value)
        first = is_v ? 0 : 2 * p.pairs;
        first += W * (w - u.turned);
      }
      if (!to_cache) first = 2 * p.pairs + W * (w - u.turned);
      float a[W], b[W];
      if (!turned) {
        count = min(W, p.dim - first);
        read_values<F32, W>(from + first * size, count, a);
        if (to_cache)
          write_values<false, W>(to + first * 2, count, a);
        else {
          if (p.padding && places[r] < 0)
#pragma unroll
            for (int j = 0; j < W; ++j) a[j] = 0.f;
          write_values<F32, W>(to + first * size, count, a);
        }
        continue;
      }
      const bool none = !to_cache && p.padding && places[r] < 0;
      const float2* cs = table + r * p.pairs;
      if (p.interleaved) {
        first = W * w;
        count = min(W, 2 * p.pairs - first);
        read_values<F32, W>(from + first * size, count, a);
#pragma unroll
        for (int j = 0; j < W / 2; ++j) {
          const float2 c = cs[min(W / 2 * w + j, p.pairs - 1)];
          b[2 * j] = none ? 0.f : a[2 * j] * c.x - a[2 * j + 1] * c.y;
          b[2 * j + 1] = none ? 0.f : a[2 * j + 1] * c.x + a[2 * j] * c.y;
        }
        if (to_cache)
          write_values<false, W>(to + first * 2, count, b);
        else
          write_values<F32, W>(to + first * size, count, b);
      } else {
        first = W * w;
        count = min(W, p.pairs - first);
        read_values<F32, W>(from + first * size, count, a);
        read_values<F32, W>(from + (p.pairs + first) * size, count, b);
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float2 c = cs[min(first + j, p.pairs - 1)];
          const float y = a[j] * c.x - b[j] * c.y;
          b[j] = none ? 0.f : b[j] * c.x + a[j] * c.y;
          a[j] = none ? 0.f : y;
        }
        if (to_cache) {
          write_values<false, W>(to + first * 2, count, a);
          write_values<false, W>(to + (p.pairs + first) * 2, count, b);
        } else {
          write_values<F32, W>(to + first * size, count, a);
          write_values<F32, W>(to + (p.pairs + first) * size, count, b);
        }
      }
    }
    __syncthreads();             // (the next tile's table)
  }
}

// The same where every unit is whole (the pairs, the values past them and a head are multiples of W values): no
// branches between units, so a lane requests several before the table is made.  A unit is W values
// (INTERLEAVED) or two times W: of both halves, or neighbours among the values that are copied (the last ones
// twice where they are odd).  CACHE: keys and values too.
template <bool F32, int W, bool INTERLEAVED, bool CACHE>
__global__ __launch_bounds__(kThreads) void rotate_wide_kernel(RotateArgs p, Units u) {
  __shared__ float2 table[kTableSize];
  __shared__ int64_t pages[kMaxRows];
  __shared__ int32_t places[kMaxRows];
  constexpr int PARTS = INTERLEAVED ? 1 : 2, WORDS = F32 ? W : W / 2, AHEAD = (WORDS == 4 ? 4 : 8) / PARTS;
  constexpr int64_t size = F32 ? 4 : 2;
  typedef uint32_t words __attribute__((ext_vector_type(WORDS), aligned(2)));
  const int t = threadIdx.x, per_head = u.turned + u.copied, of_k = p.cache.heads * per_head;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * u.rows; r0 < p.n; r0 += static_cast<int64_t>(gridDim.x) * u.rows) {
    const int rows = static_cast<int>(min(p.n - r0, static_cast<int64_t>(u.rows))), total = rows * u.of_row;
    for (int i0 = 0; i0 < total; i0 += AHEAD * kThreads) {
      int row[AHEAD], head[AHEAD], unit[AHEAD], kind[AHEAD], at[AHEAD][PARTS];     // kind 0: q, 1: k, 2: v
      words raw[AHEAD][PARTS];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int i = min(i0 + j * kThreads + t, total - 1);     // (past the end the last one again: no branch here either)
        const int r = u.row(i);
        int w = i - r * u.of_row, k = 0;
        if (CACHE && w >= u.of_q) {
          w -= u.of_q;
          k = w >= of_k ? 2 : 1;
          if (k == 2) w -= of_k;
        }
        const int h = CACHE && k == 2 ? u.v_head(w) : u.head(w);
        w -= h * (CACHE && k == 2 ? u.plain : per_head);
        const bool turned = w < u.turned && !(CACHE && k == 2);
        const int past = CACHE && k == 2 ? w : w - u.turned, begin = CACHE && k == 2 ? 0 : 2 * p.pairs;
        at[j][0] = turned ? w * W : begin + past * W * PARTS;
        if constexpr (PARTS == 2) at[j][1] = turned ? w * W + p.pairs : min(at[j][0] + W, p.dim - W);
        row[j] = r, head[j] = h, unit[j] = turned ? w : -1, kind[j] = k;
        const char* from = static_cast<const char*>(!CACHE || k == 0 ? p.q : k == 1 ? p.k : p.v);
        from += ((r0 + r) * (!CACHE || k == 0 ? p.ldq : k == 1 ? p.ldk : p.ldv) + static_cast<int64_t>(h) * p.dim) * size;
#pragma unroll
        for (int q = 0; q < PARTS; ++q) raw[j][q] = *reinterpret_cast<const words*>(from + at[j][q] * size);
      }
      if (i0 == 0) {
        for (int r = t; r < rows; r += kThreads) {
          const int32_t place = p.positions[r0 + r];
          places[r] = place;
          if (CACHE) pages[r] = page_of(p.cache, p.sequence ? p.sequence[r0 + r] : r0 + r, place);
        }
        make_table(p, u, r0, rows, table);
        lds_barrier();                   // (the requests go on)
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        if (i0 + j * kThreads + t >= total) continue;
        float f[PARTS][W];
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
#pragma unroll
          for (int x = 0; x < WORDS; ++x) {
            const uint32_t e = raw[j][q][x];
            if constexpr (F32) {
              f[q][x] = __uint_as_float(e);
            } else {
              f[q][2 * x] = __uint_as_float(e << 16);
              f[q][2 * x + 1] = __uint_as_float(e & 0xffff0000u);
            }
          }
        }
        const bool turned = unit[j] >= 0;
        const float2* cs = table + row[j] * p.pairs + (turned ? unit[j] : 0) * (INTERLEAVED ? W / 2 : W);
        if (turned) {
          if constexpr (INTERLEAVED) {
#pragma unroll
            for (int x = 0; x < W; x += 2) {
              const float2 c = cs[x / 2];
              const float y = f[0][x] * c.x - f[0][x + 1] * c.y;
              f[0][x + 1] = f[0][x + 1] * c.x + f[0][x] * c.y;
              f[0][x] = y;
            }
          } else {
#pragma unroll
            for (int x = 0; x < W; ++x) {
              const float2 c = cs[x];
              const float y = f[0][x] * c.x - f[1][x] * c.y;
              f[1][x] = f[1][x] * c.x + f[0][x] * c.y;
              f[0][x] = y;
            }
          }
        }
        const int r = row[j];
        if (!CACHE || kind[j] == 0) {
          char* to = static_cast<char*>(p.q_out) + ((r0 + r) * p.ldo + static_cast<int64_t>(head[j]) * p.dim) * size;
          const bool none = CACHE && p.padding && places[r] < 0;
#pragma unroll
          for (int q = 0; q < PARTS; ++q) {
            if (none)
#pragma unroll
              for (int x = 0; x < W; ++x) f[q][x] = 0.f;
            put_values<F32, W>(to + at[j][q] * size, f[q]);
          }
        } else if (pages[r] >= 0) {
          uint16_t* to = (kind[j] == 2 ? p.cache.values : p.cache.keys) +
                         token_at(p.cache, pages[r], head[j], places[r] & ((1 << p.cache.page_shift) - 1));
#pragma unroll
          for (int q = 0; q < PARTS; ++q) put_values<false, W>(to + at[j][q], f[q]);
        }
      }
    }
    __syncthreads();             // (the next tile's table)
  }
}

// A row's table and length, and the begun page's tokens: one workgroup per row and head.
__global__ __launch_bounds__(kThreads) void fork_kernel(ForkArgs p) {
  const int heads = p.cache.keys ? p.cache.heads : 1;
  for (int64_t i = blockIdx.x; i < p.n * heads; i += gridDim.x) {
    const int64_t row = i / heads;
    const int head = static_cast<int>(i - row * heads);
    const int64_t parent = p.parents[row];
    const bool live = parent >= 0 && parent < p.cache.sequences;
    int64_t length = live ? p.lengths[parent] : 0;
    length = max(int64_t(0), min(length, static_cast<int64_t>(p.cache.max_pages) << p.cache.page_shift));
    const int64_t begun = length >> p.cache.page_shift;
    const int used = static_cast<int>(length & ((1 << p.cache.page_shift) - 1));
    if (head == 0 && p.new_tables) {
      if (threadIdx.x == 0) p.new_lengths[row] = static_cast<int32_t>(length);
      for (int j = threadIdx.x; j < p.cache.max_pages; j += kThreads)
        p.new_tables[row * p.ldn + j] = !live ? -1 : j == begun ? p.fresh[row] : p.cache.tables[parent * p.cache.ldt + j];
    }
    if (!p.cache.keys || !used) continue;
    const int64_t from = page_of(p.cache, parent, length), to = p.fresh[row];
    if (from < 0 || to < 0 || to >= p.cache.pages || to == from) continue;
    const int64_t a = token_at(p.cache, from, head, 0), b = token_at(p.cache, to, head, 0);
    const int vectors = used * (p.cache.dim / 8);
    for (int j = threadIdx.x; j < 2 * vectors; j += kThreads) {
      uint16_t* t = j < vectors ? p.cache.keys : p.cache.values;
      const int64_t at = 8 * static_cast<int64_t>(j < vectors ? j : j - vectors);
      *reinterpret_cast<uint4*>(t + b + at) = *reinterpret_cast<const uint4*>(t + a + at);
    }
  }
}

constexpr int64_t kMaxGrid = 1 << 16;

}  // namespace

namespace {

template <bool F32, int W>
void launch_wide(const RotateArgs& a, const Units& u, dim3 grid, hipStream_t stream) {
  if (a.k && a.interleaved)
    hipLaunchKernelGGL((rotate_wide_kernel<F32, W, true, true>), grid, dim3(kThreads), 0, stream, a, u);
  else if (a.k)
    hipLaunchKernelGGL((rotate_wide_kernel<F32, W, false, true>), grid, dim3(kThreads), 0, stream, a, u);
  else if (a.interleaved)
    hipLaunchKernelGGL((rotate_wide_kernel<F32, W, true, false>), grid, dim3(kThreads), 0, stream, a, u);
  else
    hipLaunchKernelGGL((rotate_wide_kernel<F32, W, false, false>), grid, dim3(kThreads), 0, stream, a, u);
}

}  // namespace

void decode_rotate(const RotateArgs& a, hipStream_t stream) {
  // Values of a unit: 16, 8 or 4 bytes, the most that the sizes are multiples of.  (An odd number of pairs in halves, or an odd dim or rest: the
  // kernel that looks at every unit's length, at a third of the rate: 32768 rows of 16 heads of 72 in bf16, 9 pairs 98 us, 18 33.)
  const int rest = a.dim - 2 * a.pairs, most = a.f32 ? kWide<true> : kWide<false>;
  int wide = most;
  while (wide > 1 && ((a.interleaved ? 2 * a.pairs : a.pairs) % wide || rest % wide || a.dim % wide)) wide /= 2;
  const bool whole = wide > 1;
  if (!whole) wide = most;
  // (a whole unit of halves is two vectors)
  const int vectors = whole && !a.interleaved ? 2 : 1;
  auto units = [&](int values, int of) { return (values + wide * of - 1) / (wide * of); };
  const int turned = units(a.interleaved ? 2 * a.pairs : a.pairs, 1), copied = units(rest, vectors);
  const int plain = units(a.dim, vectors), q_heads = a.q ? a.q_heads : 0, heads = a.k ? a.cache.heads : 0;
  const int of_q = q_heads * (turned + copied), of_row = of_q + heads * (turned + copied + plain);
  // Rows of a tile, fewer where they would not fill the CUs: about two units per lane, and with a cache ten, for each tile waits for its
  // rows' pages.  Measured over rows of 64 to 16384 values, 300 to 32768 of them, both types: 512 units are within 7 % of the best of
  // 128 to 2048; 128 take up to twice as long where rows are narrow (32768 of 16 heads of 72: 67 us, 33), 2048 17 % more
  // (8000 of 32 of 128: 31, 27).  With a cache, eight layouts, 300 to 20000 rows: 2560 within 10 % of the best of 256 to 5120; 256 up to
  // half as much again (20000 of 16 + 2 heads of 128: 64, 41), 5120 17 % more (6000 of 32 + 8 of 128: 37, 32).  Tiles
  // at least: 4096 instead of 1024 take up to twice as long (8000 rows of 64: 9 us, 4), 256 from 22 % less to 6 % more; with a cache 256
  // instead of 512 up to 30 % more and 1024 up to half as much again (2000 rows of 16 + 2 heads of 128: 9.9, 7.6, 9.3 us; of 4 + 1 of 64: 4.5, 4.9, 7.3).
  int64_t rows = (whole ? (a.k ? 2560 : 512) * (most / wide) : 1024) / of_row;
  if (a.pairs) rows = std::min<int64_t>(rows, kTableSize / a.pairs);
  rows = std::max<int64_t>(1, std::min<int64_t>({rows, kMaxRows, a.n / (a.k ? 512 : 1024)}));
  // (a row may have 98304 units, q's, k's and v's 65536 values in pairs: the square passes 2^32, but then the tile is one row)
  const Units u{static_cast<int>(rows), turned, copied, plain, of_q, of_row, Divide(of_row, rows == 1), Divide(turned + copied), Divide(plain),
                Divide(std::max(1, a.pairs))};
  const dim3 grid(static_cast<unsigned>(std::min((a.n + rows - 1) / rows, kMaxGrid)));
  if (a.f32 && wide == 4 && whole)
    launch_wide<true, 4>(a, u, grid, stream);
  else if (a.f32 && whole)
    launch_wide<true, 2>(a, u, grid, stream);
  else if (whole && wide == 8)
    launch_wide<false, 8>(a, u, grid, stream);
  else if (whole && wide == 4)
    launch_wide<false, 4>(a, u, grid, stream);
  else if (whole)
    launch_wide<false, 2>(a, u, grid, stream);
  else if (a.f32)
    hipLaunchKernelGGL(rotate_kernel<true>, grid, dim3(kThreads), 0, stream, a, u);
  else
    hipLaunchKernelGGL(rotate_kernel<false>, grid, dim3(kThreads), 0, stream, a, u);
  launched("rotation");
}

void decode_fork(const ForkArgs& a, hipStream_t stream) {
  const int64_t blocks = a.n * (a.cache.keys ? a.cache.heads : 1);
  hipLaunchKernelGGL(fork_kernel, dim3(static_cast<unsigned>(std::min(blocks, kMaxGrid))), dim3(kThreads), 0, stream, a);
  launched("reordering of the cache");
}

}  // namespace k
}  // namespace dycl
