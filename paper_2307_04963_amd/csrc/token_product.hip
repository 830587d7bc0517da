// The bf16 products of the token operators on the matrix cores:
//   y[r, o] = epilogue(sum_k x[row(r), k] w[o, k])
// over one layer's rows, or over every expert's rows of a partition, whose
// sizes only the device knows.
//
// v_mfma_f32_16x16x32_bf16 takes 16 weight rows as A and 16 tokens as B, so a
// lane ends up with four results of one token.  Weights are packed once so that
// a wave's A operand is 1 KB in lane order (a contiguous load, from memory or
// into LDS, and a conflict-free read), and so that the four results of a
// strip's blocks adjoin: row r of block b is output 8 (r / 4) + 4 b + r % 4 of
// the strip, which leaves a lane eight consecutive outputs to store.  A gated
// strip alternates blocks of the two products, and a lane holds both factors.
#include <type_traits>

#include "token_dev.hpp"

namespace dycl {
namespace k {

namespace {

constexpr int kFrag = 512;                    // elements of one 16 x 32 operand block

// A launch holds less than 2^32 threads: of workgroups of up to 512, fewer than this.
constexpr int64_t kLaunchBlocks = (int64_t(1) << 23) - 1;

// ---- weights -----------------------------------------------------------------

// A workgroup takes 128 inputs of one strip: rows come in runs of 256 bytes, and
// the blocks leave from LDS as they lie in the packed layout.  (A lane's own 16 bytes
// of each row, in the blocks' order, took three times as long.)
template <int P>                              // products: 2 with a gate
__global__ __launch_bounds__(256) void token_pack_kernel(const uint16_t* w, const uint16_t* gate, int n, int k, int strips, int steps,
                                                         int64_t block0, uint16_t* packed) {
  constexpr int CH = 16, PITCH = CH + 1;      // 16-byte chunks of a row's 128 inputs
  __shared__ uint4 rows[P][kStrip][PITCH];
  const int parts = (steps + 3) / 4;          // (steps of 32 inputs)
  const int64_t block = block0 + blockIdx.x;
  const int64_t q = block / parts;
  const int part = static_cast<int>(block - q * parts);
  const int64_t e = q / strips;
  const int strip = static_cast<int>(q - e * strips);
#pragma unroll
  for (int i = threadIdx.x; i < P * kStrip * CH; i += 256) {
    const int ch = i % CH, r = i / CH % kStrip, which = i / (CH * kStrip);
    const int o = strip * kStrip + r, c = part * 128 + ch * 8;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (o < n && c < k) {
      const uint16_t* src = (which ? gate : w) + (e * n + o) * k + c;
      if (c + 8 <= k) {
        v = load16(src);
      } else {
        uint32_t t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = c + j < k ? src[j] : 0;
        v = make_uint4(t[0] | t[1] << 16, t[2] | t[3] << 16, t[4] | t[5] << 16, t[6] | t[7] << 16);
      }
    }
    rows[which][r][ch] = v;
  }
  __syncthreads();
  const int left = steps - part * 4 < 4 ? steps - part * 4 : 4;
  uint4* out = reinterpret_cast<uint4*>(packed) + ((e * strips + strip) * steps + part * 4) * (2 * P * 64);
#pragma unroll
  for (int i = threadIdx.x; i < 4 * 2 * P * 64; i += 256) {
    const int lane = i % 64, b = i / 64 % (2 * P), step = i / (128 * P);
    if (step >= left) continue;
    const int row = lane & 15, half = P == 2 ? b >> 1 : b, which = P == 2 ? b & 1 : 0;
    out[i] = rows[which][8 * (row >> 2) + 4 * half + (row & 3)][step * 4 + (lane >> 4)];
  }
}

// Rows that no 16-byte load could start at, or whose end a K step would pass, copied to
// rows of a whole number of steps: 1237 x 1003 in 3.7 to 4.4 us, mostly the launch.
__global__ __launch_bounds__(256) void token_align_kernel(const uint16_t* x, int64_t ldx, int64_t n, int d, uint16_t* out,
                                                          int64_t ldo) {
  const int64_t per = ldo / 8;
  for (int64_t q = blockIdx.x * 256L + threadIdx.x; q < n * per; q += gridDim.x * 256L) {
    const int64_t row = q / per;
    const int c = static_cast<int>(q - row * per) * 8;
    const uint16_t* src = x + row * ldx + c;
    uint4 v;
    if (c + 8 <= d) {
      v = load16(src);
    } else {
      uint32_t e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = c + j < d ? src[j] : 0;
      v = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    }
    reinterpret_cast<uint4*>(out + row * ldo)[c / 8] = v;
  }
}

// ---- tiles ---------------------------------------------------------------------

// Rows [row0, row0 + rows) of the product, all of one layer.
struct Tile {
  int expert;
  int64_t row0;
  int rows;
};

// The tile that `found`'s first lane holds: expert e0 + lane with rows [lo, hi) and
// `incl` tiles up to its last, t of which (counted alike) is the one.
__device__ __forceinline__ void take_tile(int lo, int hi, int incl, int e0, int t, uint64_t found, int bm, Tile& out) {
  const int from = __ffsll(static_cast<unsigned long long>(found)) - 1;
  const int first = __builtin_amdgcn_readlane(lo, from), end = __builtin_amdgcn_readlane(hi, from);
  const int last = first + (t - __builtin_amdgcn_readlane(incl, from) + (end - first + bm - 1) / bm) * bm;
  out.expert = e0 + from;
  out.row0 = last;
  out.rows = end - last < bm ? end - last : bm;
}

// Row tile `t` of `bm` rows: expert after expert.  False past the last one.
// Every wave finds it for itself.
__device__ __forceinline__ bool find_tile(const ProductArgs& p, int bm, int64_t t, Tile& out) {
  if (!p.offsets) {
    out.expert = 0;
    out.row0 = t * bm;
    const int64_t left = p.rows - out.row0;
    out.rows = static_cast<int>(left < bm ? left : bm);
    return left > 0;
  }
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int e0 = 0; e0 < p.experts; e0 += 64) {
    const int e = e0 + lane;
    const int lo = e < p.experts ? p.offsets[e] : 0, hi = e < p.experts ? p.offsets[e + 1] : 0;
    const int incl = scan_lanes((hi - lo + bm - 1) / bm);
    const uint64_t found = __ballot(t < before + incl);
    if (found) {
      take_tile(lo, hi, incl, e0, static_cast<int>(t - before), found, bm, out);
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// The tile of this workgroup: row tile and column tile.  Workgroups are dealt
// round-robin over the 8 XCDs, so each XCD takes a contiguous range of the
// tiles, in which runs of kGroup row tiles go over the columns together: 32
// workgroups that are resident at a time share 8 row tiles and 4 column tiles
// in their XCD's L2.
constexpr int kGroup = 8;

__device__ __forceinline__ bool tile_of(const ProductArgs& p, int bm, int col_tiles, Tile& out, int& col) {
  int64_t row_tiles = (p.rows + bm - 1) / bm;
  int lo = 0, hi = 0, incl = 0;                     // up to 64 experts: one scan for both uses
  const int lane = threadIdx.x & 63;
  if (p.offsets) {
    row_tiles = 0;
    for (int e0 = 0; e0 < p.experts; e0 += 64) {
      const int e = e0 + lane;
      lo = e < p.experts ? p.offsets[e] : 0;
      hi = e < p.experts ? p.offsets[e + 1] : 0;
      incl = scan_lanes((hi - lo + bm - 1) / bm);
      row_tiles += __builtin_amdgcn_readlane(incl, 63);
    }
  }
  const int64_t all = row_tiles * col_tiles, each = all >> 3;
  const int64_t wg = blockIdx.x;
  if (wg >= all) return false;
  const int64_t t = wg < each * 8 ? (wg & 7) * each + (wg >> 3) : wg;
  const int64_t group = t / (kGroup * col_tiles);
  const int in = static_cast<int>(t - group * (kGroup * col_tiles));
  const int64_t left = row_tiles - group * kGroup;
  const int height = left < kGroup ? static_cast<int>(left) : kGroup;
  col = in / height;
  const int64_t row_tile = group * kGroup + (in - col * height);
  if (!p.offsets || p.experts > 64) return find_tile(p, bm, row_tile, out);
  take_tile(lo, hi, incl, 0, static_cast<int>(row_tile), __ballot(row_tile < incl), bm, out);
  return true;
}

__device__ __forceinline__ int64_t source_row(const ProductArgs& p, int64_t row) {
  return p.order ? p.order[row] / p.order_k : row;
}

// ---- epilogues -------------------------------------------------------------------

// values [o, o + 8) of an expert's bias vector (0 past the end or without one)
__device__ __forceinline__ void bias8(const ProductArgs& p, const float* bias, int expert, int o, float (&r)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = bias && o + j < p.N ? bias[static_cast<int64_t>(expert) * p.N + o + j] : 0.f;
}

// Outputs o to o + 7 of one row: bias, activation or gate, residual.  a and b are
// the strip's blocks, ga and gb the gate's.  (Without fused multiply-adds, which one
// kernel's instance might get and another's not: a row's bits are the same in all.)
template <bool GATED, int ACT>
__device__ __forceinline__ void finish8(const ProductArgs& p, int64_t row, int o, const f32x4& a, const f32x4& b, const f32x4& ga, const f32x4& gb,
                                        const float (&bias)[8], const float (&gate_bias)[8], float (&v)[8]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = (j < 4 ? a[j & 3] : b[j & 3]) + bias[j];
    if (GATED)
      v[j] *= token_act((j < 4 ? ga[j & 3] : gb[j & 3]) + gate_bias[j], ACT);
    else
      v[j] = token_act(v[j], ACT);
  }
  if (o + 8 > p.N) {
    // the padding's zero weights make NaN of an infinite input: what is stored there is 0
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (o + j >= p.N) v[j] = 0.f;
  }
  if (p.residual) {
    const uint16_t* r = p.residual + row * p.ldr + o;
    if (o + 8 <= p.N) {
      const uint4 q = load16(r);
      const uint32_t e[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] += __uint_as_float(e[j] << 16);
        v[2 * j + 1] += __uint_as_float(e[j] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (o + j < p.N) v[j] += bf2f(r[j]);
    }
  }
}

__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

__device__ __forceinline__ void store8(const ProductArgs& p, int64_t row, int o, const float (&v)[8]) {
  if (o >= p.N_store) return;
  const bool whole = o + 8 <= p.N_store;
  if (p.y_f32) {
    float* y = static_cast<float*>(p.y) + row * p.ldy + o;
    if (whole) {
      store16(y, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
      store16(y + 4, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (o + j < p.N_store) y[j] = v[j];
    }
    return;
  }
  uint16_t* y = static_cast<uint16_t*>(p.y) + row * p.ldy + o;
  if (whole) {
    store16(y, pack8(v));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (o + j < p.N_store) y[j] = f2bf(v[j]);
  }
}

// f with the activation as a constant: in every element's way, its branches took
// longer than the sums of a short contraction
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == TACT_NONE) f(std::integral_constant<int, TACT_NONE>{});
  else if (act == TACT_RELU) f(std::integral_constant<int, TACT_RELU>{});
  else if (act == TACT_GELU) f(std::integral_constant<int, TACT_GELU>{});
  else f(std::integral_constant<int, TACT_SILU>{});
}

// The sums of a wave's TB x RB blocks, from row `row0` of the tile and strip
// `strip`, to y.  (Rows of bf16 passed through LDS and stored in runs of the tile's
// width took as long as the lanes' own 16-byte pieces.)
template <int TB, int RB, bool GATED>
__device__ __forceinline__ void tile_epilogue(const ProductArgs& p, const Tile& tile, int row0, int strip, const f32x4 (&acc)[TB][RB]) {
  constexpr int NB = GATED ? 4 : 2;
  const int lane = threadIdx.x & 63;
  // strip after strip of a row, so that a wave's two pieces of a line leave together
  // (8192 rows of 8 of 64 experts, when their results were 16 bits wide: 919 us in 256 x
  // 256 tiles and 277 MB written by the second product; row after row of a strip 940 and 348)
  auto finish = [&](auto act) __attribute__((always_inline)) {
    constexpr int C = RB / NB;
    const int o0 = strip * kStrip + 8 * (lane >> 4);
    float b8[C][8], g8[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      bias8(p, p.bias, tile.expert, o0 + c * kStrip, b8[c]);
      bias8(p, GATED ? p.gate_bias : nullptr, tile.expert, o0 + c * kStrip, g8[c]);
    }
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      const int row = row0 + b * 16 + (lane & 15);
      if (row >= tile.rows) continue;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int o = o0 + c * kStrip, at = c * NB;
        if (o >= p.N_store) continue;
        float v[8];
        if (GATED)
          finish8<true, act>(p, tile.row0 + row, o, acc[b][at], acc[b][at + 2 < RB ? at + 2 : 0], acc[b][at + 1], acc[b][at + 3 < RB ? at + 3 : 0], b8[c], g8[c], v);
        else
          finish8<false, act>(p, tile.row0 + row, o, acc[b][at], acc[b][at + 1], acc[b][at], acc[b][at], b8[c], g8[c], v);
        store8(p, tile.row0 + row, o, v);
      }
    }
  };
  with_act(p.act, finish);
}

// ---- many rows: tiles through LDS --------------------------------------------------

// BM tokens x BN weight rows (gated: BN / 2 outputs), K steps of 32 through a ring
// of S stages of LDS filled by direct loads.  A token row of a stage is 64 bytes
// whose four 16-byte chunks are stored at chunk ^ -(row / 4) % 4, so the lanes that
// a read serves at a time lie in different bank groups; rows past the tile's end
// repeat its last one, inputs past K read zeros.
//
// The waves form two groups, one wave of each on every SIMD, half a step apart:
// while one group's matrix instructions run, the other reads its next operands
// from LDS and requests a later step's loads; a barrier swaps them.  In halves of
// steps counted from the start, group 0 reads step h in half 2 h and multiplies in
// 2 h + 1, group 1 one half later.  So stage h % S has been read by all after half
// 2 h + 1 and takes the loads of step h + S from half 2 h + 2 on (in the group's read
// of step h + 1), and what a wave requested for step h + 1 has to be there before
// half 2 h + 2: it waits for that at the end of its read of step h.  With the waves
// in step, all reading and then all multiplying, 8192 x 4096 x 8192 took 4 % longer;
// with four waves of 128 x 128 each, 14 %; with 32 x 32 x 16 instructions 9 %.
__device__ __align__(16) const uint16_t g_zeros[8] = {0, 0, 0, 0, 0, 0, 0, 0};

template <int N>
__device__ __forceinline__ void wait_all_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int BM, int BN, int WM, int WN, int S, bool GATED>
__device__ __forceinline__ void tile_product(const ProductArgs& p, const Tile& tile, int col, int strips, int steps, char* smem) {
  constexpr int NT = 64 * WM * WN;
  constexpr int NB = GATED ? 4 : 2;                 // blocks per strip
  constexpr int WTM = BM / WM, WTN = BN / WN;
  constexpr int TB = WTM / 16, RB = WTN / 16;
  constexpr int A_BYTES = BM * 64, B_BYTES = BN * 64, STAGE = A_BYTES + B_BYTES;
  constexpr int JA = BM * 4 / NT, JB = BN * 4 / NT, J = JA + JB;
  constexpr int TS = BN / 16 / NB;                  // strips per tile
  static_assert(WM * WN == 8, "two groups of four waves");
  static_assert(BM * 4 % NT == 0 && BN * 4 % NT == 0 && JA > 0 && JB > 0 && RB % NB == 0 && WTM % 16 == 0, "tile shape");
  static_assert(S >= 3 && J * (S - 2) < 64, "stages");
  const int strip0 = col * TS;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;

  // this thread's rows of x, as byte offsets, and the K chunk that it loads of each
  const uint16_t* const a_base = p.order ? p.x : p.x + tile.row0 * p.ldx;
  int64_t a_off[JA];
  int a_k[JA];
#pragma unroll
  for (int j = 0; j < JA; ++j) {
    const int r = (j * NT + tid) >> 2;
    const int chunk = ((tid & 3) ^ -(r >> 2)) & 3;
    const int64_t row = r < tile.rows ? r : tile.rows - 1;
    a_k[j] = chunk * 8;
    a_off[j] = ((p.order ? p.order[tile.row0 + row] / p.order_k : row) * p.ldx + chunk * 8) * 2;
  }
  const uint16_t* const b_base = p.w + (static_cast<int64_t>(tile.expert) * strips + strip0) * steps * (NB * kFrag);
  uint32_t b_off[JB];
#pragma unroll
  for (int j = 0; j < JB; ++j) {
    const int q = (j * NT + tid) >> 6;              // block of the stage
    int s = q / NB;
    s = strip0 + s < strips ? s : strips - 1 - strip0;
    b_off[j] = (static_cast<uint32_t>(s) * steps * NB + q % NB) * (kFrag * 2) + lane * 16;
  }
  // (steps below `near` have all their inputs, at offsets of 32 bits from one base)
  const int near = p.far ? 0 : p.K / 32;
  auto load = [&](int h, char* stage) __attribute__((always_inline)) {
    if (h < near) {
#pragma unroll
      for (int j = 0; j < JA; ++j) load_lds16(a_base + h * 32, static_cast<uint32_t>(a_off[j]), stage + (j * NT + wave * 64) * 16);
    } else {
#pragma unroll
      for (int j = 0; j < JA; ++j) {
        const char* src = reinterpret_cast<const char*>(a_base + h * 32) + a_off[j];
        if (h * 32 + a_k[j] >= p.K) src = reinterpret_cast<const char*>(g_zeros);
        load_lds16(src, stage + (j * NT + wave * 64) * 16);
      }
    }
    const char* const b_step = reinterpret_cast<const char*>(b_base) + static_cast<int64_t>(h) * (NB * kFrag * 2);
#pragma unroll
    for (int j = 0; j < JB; ++j) load_lds16(b_step, b_off[j], stage + A_BYTES + (j * NT + wave * 64) * 16);
  };
  const int xr = wm * WTM + (lane & 15);
  const int x_at = xr * 64 + (((lane >> 4) ^ -(xr >> 2)) & 3) * 16, w_at = A_BYTES + wn * (RB * 1024) + lane * 16;

  f32x4 acc[TB][RB];
#pragma unroll
  for (int b = 0; b < TB; ++b)
#pragma unroll
    for (int c = 0; c < RB; ++c) acc[b][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 x[TB], w[RB];

  auto read = [&](const char* stage) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < RB; ++c) w[c] = *reinterpret_cast<const bf16x8*>(stage + w_at + c * 1024);
#pragma unroll
    for (int b = 0; b < TB; ++b) x[b] = *reinterpret_cast<const bf16x8*>(stage + x_at + b * 1024);
  };
  auto multiply = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int b = 0; b < TB; ++b)
#pragma unroll
      for (int c = 0; c < RB; ++c) acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[c], x[b], acc[b][c], 0, 0, 0);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
  };

  const int nh = steps;
#pragma unroll
  for (int h = 0; h < S - 1; ++h)
    if (h < nh) load(h, smem + h * STAGE);
  if (nh >= S - 1)
    wait_vm_barrier<J * (S - 2)>();
  else
    wait_vm_barrier<0>();
  if (wave >= 4) lds_barrier();                     // group 1 is half a step behind

  // step h reads stage h % S (`cur`) and loads step h + S - 1 into the stage before it
  char* cur = smem;
  char* prev = smem + (S - 1) * STAGE;
  int h = 0;
  for (; h + S - 1 < nh; ++h) {
    read(cur);
    load(h + S - 1, prev);
    wait_all_barrier<J * (S - 2)>();
    multiply();
    lds_barrier();
    prev = cur;
    cur = cur == smem + (S - 1) * STAGE ? smem : cur + STAGE;
  }
  for (; h < nh; ++h) {
    read(cur);
    wait_all_barrier<0>();
    multiply();
    lds_barrier();
    cur = cur == smem + (S - 1) * STAGE ? smem : cur + STAGE;
  }
  if (wave < 4) lds_barrier();
  tile_epilogue<TB, RB, GATED>(p, tile, wm * WTM, strip0 + wn * (RB / NB), acc);
}

// 256 x 256 tiles, one workgroup per CU; an expert's last tile, where it has 128
// rows or fewer, takes half the time.  128 x 256 tiles on three stages leave room for two
// workgroups, one's epilogue beside the other's products: better for short K.
//
// Measured: gated 8192 x 4096 x 4096 395 us = 1.39 PF, matrix cores 72% busy at the
// clock that the power limit leaves (1.8 to 1.95 GHz); a library's product of that size
// reaches 1.5 PF.  8192 rows of 8 of 64 experts: 2048 -> 2 x 1024 in 549 us (1.0 PF; 2.3
// GB pass the L2s for 0.8 GB of rows and weights), 1024 -> 2048 in 402 us (0.68 PF; 0.94 GB
// read, 0.54 GB of float32 results written).
template <int BM, bool GATED>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(BM == 256 ? 2 : 4)))
void token_tile_kernel(ProductArgs p, int strips, int steps, int col_tiles) {
  constexpr int S = BM == 256 ? 4 : 3;
  __shared__ __align__(16) char smem[S * (BM + 256) * 64];
  Tile tile;
  int col;
  if (!tile_of(p, BM, col_tiles, tile, col)) return;
  if (BM == 128 || tile.rows > 128)
    tile_product<BM, 256, 2, 4, S, GATED>(p, tile, col, strips, steps, smem);
  else
    tile_product<128, 256, 2, 4, S, GATED>(p, tile, col, strips, steps, smem);
}

// ---- fewer rows: small tiles, a deep ring -------------------------------------------

// BM tokens x BN weight rows, KT times 64 inputs per stage of a ring of S.  Every wave
// loads, W pieces of 1 KB at a time: eight token rows of 128 bytes, whose eight 16-byte
// chunks are stored at chunk ^ (row / 2) % 8, or a block of weights.  The first WM x WN
// waves multiply, each its part of the tile over all steps in order, the order of the
// large tiles: a row's sums are the same bits whichever kernel takes it.  One barrier
// per stage: behind it, the stage read a turn ago takes the loads of the stage S - 1 ahead.
// Where RB is less than a strip's blocks, its sums meet in LDS.
//
// Few rows are bound by the weights' way from memory: 5 x 4096 x 4096, 34 MB in 7.3 us; one
// row through eight experts 2048 -> 2 x 1024 -> 2048, 101 MB in 11.8 + 7.9 us = 5.1 TB/s; 333
// rows crowded on about half of 32 experts, 1024 -> 2048 -> 1024, 155 MB in 17.6 + 17.4 us =
// 4.4 TB/s.  More rows are bound by the stages' turns (one barrier and a first read of LDS
// each) while a CU holds one or two tiles: 1237 x 1008 x 777 10.9 us on 140 CUs.
template <int BM, int BN, int WM, int WN, int W, int KT, int S, bool GATED>
__global__ __launch_bounds__(64 * W) void token_ring_kernel(ProductArgs p, int strips, int steps, int col_tiles) {
  constexpr int NB = GATED ? 4 : 2;                 // blocks per strip and step
  constexpr int AU = BM / 8, BU = BN / 8;           // pieces per 64 inputs
  constexpr int JA = KT * AU / W, JB = KT * BU / W, J = JA + JB;
  constexpr int CA = AU > W ? AU / W : 1, CB = BU > W ? BU / W : 1;   // of them different ones of a wave
  constexpr int A_BYTES = BM * 128, PART = A_BYTES + BN * 128, STAGE = KT * PART;
  constexpr int TB = BM / 16 / WM, RB = BN / 16 / WN;                 // blocks of a wave
  constexpr int TS = BN / 16 / NB;                  // strips per tile
  static_assert(KT * AU % W == 0 && KT * BU % W == 0 && (W % AU == 0 || AU % W == 0) && (W % BU == 0 || BU % W == 0), "a wave's pieces repeat");
  static_assert(W % 2 == 0 && AU % 2 == 0, "a wave loads one chunk of its rows");
  static_assert(WM * WN <= W && TB * WM * 16 == BM && RB * WN * 16 == BN && (RB % NB == 0 || NB % RB == 0), "tile shape");
  constexpr int PARTS = RB < NB ? NB / RB : 1;      // waves that share a strip
  static_assert(S >= 2 && J * (S - 2) < 64 && S * STAGE <= 160 * 1024, "stages");
  __shared__ __align__(16) char smem[S * STAGE];

  Tile tile;
  int col;
  if (!tile_of(p, BM, col_tiles, tile, col)) return;
  const int strip0 = col * TS;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // this lane's rows of x, as byte offsets, and the K chunk that it loads of each; this wave's blocks of weights
  const uint16_t* const a_base = p.order ? p.x : p.x + tile.row0 * p.ldx;
  // (row / 2 % 8 is the same for all of a wave's pieces: they lie whole times 16 rows apart)
  const int a_k = ((lane ^ (((wave & 1) << 2) + (lane >> 4))) & 7) * 8;
  int64_t a_off[CA];
#pragma unroll
  for (int j = 0; j < CA; ++j) {
    const int r = (j * W + wave) % AU * 8 + (lane >> 3);
    const int64_t row = r < tile.rows ? r : tile.rows - 1;
    a_off[j] = ((p.order ? p.order[tile.row0 + row] / p.order_k : row) * p.ldx + a_k) * 2;
  }
  const uint16_t* const b_base = p.w + (static_cast<int64_t>(tile.expert) * strips + strip0) * steps * (NB * kFrag);
  uint32_t b_off[CB];
#pragma unroll
  for (int j = 0; j < CB; ++j) {
    const int c = (j * W + wave) % BU;
    const int s = strip0 + c / (2 * NB) < strips ? c / (2 * NB) : strips - 1 - strip0;
    b_off[j] = (static_cast<uint32_t>(s) * steps * NB + c % (2 * NB)) * (kFrag * 2) + lane * 16;
  }
  const int all = steps / 2, near = p.far ? 0 : p.K / 64;   // times 64 inputs: in all, and with all of them at offsets of 32 bits
  // (those past the last one repeat it: every stage is as many loads)
  auto load = [&](int i, char* stage) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < JA; ++j) {
      const int u = j * W + wave, q = u / AU, h0 = i * KT + q, h = h0 < all ? h0 : all - 1;
      char* const to = stage + q * PART + u % AU * 1024;
      if (h < near) {
        load_lds16(a_base + h * 64, static_cast<uint32_t>(a_off[j % CA]), to);
      } else {
        const char* src = reinterpret_cast<const char*>(a_base + h * 64) + a_off[j % CA];
        if (h * 64 + a_k >= p.K) src = reinterpret_cast<const char*>(g_zeros);
        load_lds16(src, to);
      }
    }
#pragma unroll
    for (int j = 0; j < JB; ++j) {
      const int u = j * W + wave, q = u / BU, h0 = i * KT + q, h = h0 < all ? h0 : all - 1;
      const char* const b_step = reinterpret_cast<const char*>(b_base) + static_cast<int64_t>(h) * (2 * NB * kFrag * 2);
      load_lds16(b_step, b_off[j % CB], stage + q * PART + A_BYTES + u % BU * 1024);
    }
  };

  const int wm = wave / WN, wn = wave % WN;
  const int xr = wm * (TB * 16) + (lane & 15);
  f32x4 acc[TB][RB];
#pragma unroll
  for (int b = 0; b < TB; ++b)
#pragma unroll
    for (int c = 0; c < RB; ++c) acc[b][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const char* part) __attribute__((always_inline)) {
    bf16x8 x[2][TB], w[2][RB];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int c = 0; c < RB; ++c) {
        const int blk = wn * RB + c;                // block of the tile: strip blk / NB
        w[s][c] = *reinterpret_cast<const bf16x8*>(part + A_BYTES + ((blk / NB * 2 + s) * NB + blk % NB) * 1024 + lane * 16);
      }
#pragma unroll
      for (int b = 0; b < TB; ++b)
        x[s][b] = *reinterpret_cast<const bf16x8*>(part + (xr + b * 16) * 128 + (((s * 4 + (lane >> 4)) ^ (xr >> 1)) & 7) * 16);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int b = 0; b < TB; ++b)
#pragma unroll
        for (int c = 0; c < RB; ++c) acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[s][c], x[s][b], acc[b][c], 0, 0, 0);
  };

  const int turns = (all + KT - 1) / KT;
#pragma unroll
  for (int i = 0; i < S - 1; ++i)
    if (i < turns) load(i, smem + i * STAGE);
  char* cur = smem;
  char* prev = smem + (S - 1) * STAGE;
  for (int i = 0; i < turns; ++i) {
    if (i + S - 1 <= turns)
      wait_all_barrier<J * (S - 2)>();
    else
      wait_all_barrier<0>();
    if (i + S - 1 < turns) load(i + S - 1, prev);
    if (wave < WM * WN) {
      const int left = all - i * KT;
      if (left >= KT) {
#pragma unroll
        for (int q = 0; q < KT; ++q) multiply(cur + q * PART);
      } else {
        for (int q = 0; q < left; ++q) multiply(cur + q * PART);
      }
    }
    prev = cur;
    cur = cur == smem + (S - 1) * STAGE ? smem : cur + STAGE;
  }
  if constexpr (PARTS == 1) {
    if (wave < WM * WN) tile_epilogue<TB, RB, GATED>(p, tile, wm * (TB * 16), strip0 + wn * (RB / NB), acc);
  } else {
    // a strip's sums meet in its first wave
    f32x4* const sums = reinterpret_cast<f32x4*>(smem);
    const int part = wn % PARTS;
    lds_barrier();
    if (wave < WM * WN && part > 0) {
#pragma unroll
      for (int b = 0; b < TB; ++b)
#pragma unroll
        for (int c = 0; c < RB; ++c) sums[((wave * TB + b) * RB + c) * 64 + lane] = acc[b][c];
    }
    lds_barrier();
    if (wave >= WM * WN || part > 0) return;
    f32x4 strip[TB][NB];
#pragma unroll
    for (int b = 0; b < TB; ++b)
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        if (c < RB)
          strip[b][c] = acc[b][c];
        else
          strip[b][c] = sums[(((wave + c / RB) * TB + b) * RB + c % RB) * 64 + lane];
      }
    tile_epilogue<TB, NB, GATED>(p, tile, wm * (TB * 16), strip0 + wn / PARTS, strip);
  }
}

// ---- the experts' results, weighted and summed ----------------------------------------

// Eight outputs per lane, float32 until the one rounding of the sum: held in fewer bits,
// the results' own roundings come to more than the sum's.  A row's slots and weights
// come first, then up to eight experts' results are requested together: taken one by
// one, each waited for its slot and then for its values.  Bound by HBM: 8192 rows of 2048,
// 8 experts each, 606 MB in 124 us = 4.9 TB/s.
__global__ __launch_bounds__(256) void token_combine_kernel(CombineArgs p) {
  const int per = (p.d + 7) / 8;
  const int64_t all = p.n * per;
  for (int64_t q = blockIdx.x * 256L + threadIdx.x; q < all; q += gridDim.x * 256L) {
    const int64_t row = q / per;
    const int o = static_cast<int>(q - row * per) * 8;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    const bool whole = o + 8 <= p.d;
    if (p.residual) {
      const uint16_t* r = p.residual + row * p.ldr + o;
      if (whole) {
        const uint4 f = load16(r);
        const uint32_t e[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[2 * j] = __uint_as_float(e[j] << 16);
          v[2 * j + 1] = __uint_as_float(e[j] & 0xffff0000u);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (o + j < p.d) v[j] = bf2f(r[j]);
      }
    }
    for (int j0 = 0; j0 < p.k; j0 += 8) {
      int slot[8];
      float w[8];
      float4 f[8][2];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = j0 + j < p.k;
        slot[j] = in ? p.slots[row * p.k + j0 + j] : -1;
        w[j] = in ? p.weights[row * p.k + j0 + j] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (slot[j] >= 0) {
          const float4* part = reinterpret_cast<const float4*>(p.part + slot[j] * p.ldp + o);
          f[j][0] = part[0];
          f[j][1] = part[1];
        }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (slot[j] >= 0) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            v[4 * q] = fmaf(w[j], f[j][q].x, v[4 * q]);
            v[4 * q + 1] = fmaf(w[j], f[j][q].y, v[4 * q + 1]);
            v[4 * q + 2] = fmaf(w[j], f[j][q].z, v[4 * q + 2]);
            v[4 * q + 3] = fmaf(w[j], f[j][q].w, v[4 * q + 3]);
          }
        }
    }
    uint16_t* out = p.out + row * p.ldo + o;
    if (whole) {
      store16(out, pack8(v));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (o + j < p.d) out[j] = f2bf(v[j]);
    }
  }
}

// an upper bound of the row tiles of `bm` rows
int64_t row_tiles(const ProductArgs& a, int bm) {
  const int64_t whole = (a.rows + bm - 1) / bm;
  if (!a.offsets) return whole;
  const int64_t ragged = a.experts < a.rows ? a.experts : a.rows;
  return whole + ragged;
}

template <int BM, bool GATED>
void tiles(const ProductArgs& a, hipStream_t s) {
  const int strips = strips_of(a.N), steps = steps_of(a.K), per = 256 / (GATED ? 64 : 32);
  const int cols = (strips + per - 1) / per;
  token_tile_kernel<BM, GATED><<<static_cast<unsigned>(row_tiles(a, BM) * cols), 512, 0, s>>>(a, strips, steps, cols);
}

template <int BM, int BN, int WM, int WN, int W, int KT, int S, bool GATED>
void ring(const ProductArgs& a, hipStream_t s) {
  const int strips = strips_of(a.N), steps = steps_of(a.K), per = BN / (GATED ? 64 : 32);
  const int cols = (strips + per - 1) / per;
  token_ring_kernel<BM, BN, WM, WN, W, KT, S, GATED><<<static_cast<unsigned>(row_tiles(a, BM) * cols), 64 * W, 0, s>>>(a, strips, steps, cols);
}

// Which kernel: the one whose estimate is least.  A round of tiles (256 CUs, per_cu
// workgroups each) takes `round` microseconds and `full` per 64 inputs, `alone` where
// each CU has one; fitted to 457 plain and 443 gated products of 1 to 8192 rows, 512
// to 20000 outputs and 256 to 8192 inputs, their weights from memory: the choice is 0.2% and
// 0.3% slower there than each product's best.  Leaving a shape out costs 0.4 to 3% on
// average.  Beside some, us of a product of their own and of another shape.
// (rows x inputs x outputs; gated: two products.)
struct Shape {
  int bm, bn, per_cu;
  float alone, full, round;
};
constexpr Shape kPlain[] = {
    {256, 256, 1, 1.20f, 1.548f, 10.0f},
    {128, 256, 2, 1.00f, 2.045f, 5.5f},
    {64, 128, 2, 0.441f, 0.716f, 3.5f},
    {64, 128, 1, 0.415f, 0.391f, 3.4f},    // 300 x 4096 x 4096: 29.5 (64 x 128, two per CU: 31.6)
    {64, 64, 1, 0.266f, 0.259f, 3.2f},     // 256 x 4096 x 4096: 20.8 (32 x 64: 30.5)
    {32, 64, 1, 0.178f, 0.180f, 3.1f},     // 100 x 4096 x 4096: 15.5 (32 x 32: 19.5)
    {32, 32, 1, 0.114f, 0.127f, 3.2f},     // 48 x 4096 x 4096: 11.9 (32 x 64: 16.0)
    {16, 32, 1, 0.079f, 0.099f, 3.3f},     // 1 x 4096 x 4096: 10.1
    {16, 32, 4, 0.160f, 0.266f, 2.9f},     // 4 x 1024 x 20000: 10.0 (one per CU: 14.4)
};
constexpr Shape kGated[] = {
    {256, 256, 1, 1.22f, 1.547f, 8.3f},
    {128, 256, 2, 1.05f, 1.936f, 4.7f},
    {64, 128, 2, 0.423f, 0.727f, 3.7f},
    {64, 128, 1, 0.415f, 0.417f, 3.5f},    // 512 x 2048 x 2048: 16.8 (two per CU: 17.6)
    {64, 64, 1, 0.273f, 0.290f, 3.6f},     // 256 x 2048 x 2048: 12.9 (32 x 64: 18.7)
    {32, 64, 1, 0.190f, 0.206f, 3.4f},     // 64 x 4096 x 4096: 19.4 (64 x 64: 23.8)
    {16, 64, 1, 0.165f, 0.177f, 3.2f},     // 1 x 4096 x 4096: 16.3 (32 x 64: 16.7)
    {16, 64, 2, 0.215f, 0.300f, 3.1f},     // 16 rows of 8 of 64 experts, 2048 -> 2 x 1024 -> 2048: 130 a call (one per CU: 138)
    {16, 64, 5, 0.360f, 0.541f, 3.0f},     // 9 rows of 5 of 128 experts, 784 -> 2 x 960 -> 784: 38 a call (two per CU: 45)
};

// Estimated time of a shape for a layer's rows (with a partition: of the average
// expert, whose last tile is half full; of 256 rows, one up to half full takes half
// the time).  For the two products of 20 expert layers (1 to 8192 rows, 8 to 128 experts,
// 1 to 8 of them a row, skewed or not) the choice is 0.8% slower than each product's best on
// the average, at worst 10% (2048 rows of 8 of 128 experts: 128 rows each, where 256 x 256
// tiles beat 128 x 256).  Steps taken as 7 or 14% longer for experts' weights, as one size
// of them would have it, make that 1.0%.
inline float estimate(const Shape& t, const ProductArgs& a, bool gated) {
  const float steps = static_cast<float>(steps_of(a.K) / 2);
  const float cols = ceilf(strips_of(a.N) * (gated ? 64.f : 32.f) / t.bn);
  float rows = ceilf(static_cast<float>(a.rows) / t.bm);
  if (a.offsets) {
    const float mean = static_cast<float>(a.rows) / a.experts;
    const float each = mean / t.bm + (t.bm == 256 ? 0.4f : 0.5f);
    rows = (mean < 1.f ? a.rows : a.experts) * (each > 1.f ? each : 1.f);
  }
  const float tiles = rows * cols, slots = 256.f * t.per_cu;
  const float whole = floorf(tiles / slots), rest = tiles - whole * slots;
  float us = whole * (t.round + steps * t.full);
  if (rest > 0.f) us += t.round + steps * (rest <= 256.f ? t.alone : t.full);
  return us;
}

// -1 where no shape's tiles are as few as a launch holds
template <size_t C>
int best_of(const Shape (&shapes)[C], const ProductArgs& a, bool gated) {
  int best = -1;
  float least = 0.f;
  for (int i = 0; i < static_cast<int>(C); ++i) {
    const int64_t cols = (strips_of(a.N) * int64_t(gated ? 64 : 32) + shapes[i].bn - 1) / shapes[i].bn;
    if (row_tiles(a, shapes[i].bm) * cols >= kLaunchBlocks) continue;
    const float t = estimate(shapes[i], a, gated);
    if (best < 0 || t < least) {
      best = i;
      least = t;
    }
  }
  return best;
}

void plain(const ProductArgs& a, int shape, hipStream_t s) {
  switch (shape) {
    case 0: return tiles<256, false>(a, s);
    case 1: return tiles<128, false>(a, s);
    case 2: return ring<64, 128, 2, 4, 8, 1, 3, false>(a, s);
    case 3: return ring<64, 128, 2, 4, 8, 2, 3, false>(a, s);
    case 4: return ring<64, 64, 4, 2, 8, 2, 3, false>(a, s);
    case 5: return ring<32, 64, 2, 2, 8, 4, 3, false>(a, s);
    case 6: return ring<32, 32, 2, 2, 8, 4, 4, false>(a, s);
    case 7: return ring<16, 32, 1, 2, 8, 8, 3, false>(a, s);
    default: return ring<16, 32, 1, 2, 4, 2, 3, false>(a, s);
  }
}

void gated(const ProductArgs& a, int shape, hipStream_t s) {
  switch (shape) {
    case 0: return tiles<256, true>(a, s);
    case 1: return tiles<128, true>(a, s);
    case 2: return ring<64, 128, 2, 2, 8, 1, 3, true>(a, s);
    case 3: return ring<64, 128, 4, 2, 8, 2, 3, true>(a, s);
    case 4: return ring<64, 64, 4, 1, 8, 2, 3, true>(a, s);
    case 5: return ring<32, 64, 2, 2, 8, 4, 3, true>(a, s);
    case 6: return ring<16, 64, 1, 4, 8, 4, 3, true>(a, s);
    case 7: return ring<16, 64, 1, 4, 4, 2, 3, true>(a, s);
    default: return ring<16, 64, 1, 2, 2, 1, 3, true>(a, s);
  }
}

}  // namespace

void token_pack(const uint16_t* w, const uint16_t* gate, int experts, int n, int k, uint16_t* packed, hipStream_t s) {
  const int strips = strips_of(n), steps = steps_of(k);
  const int64_t blocks = static_cast<int64_t>(experts) * strips * ((steps + 3) / 4);
  for (int64_t b = 0; b < blocks; b += kLaunchBlocks) {
    const unsigned here = static_cast<unsigned>(blocks - b < kLaunchBlocks ? blocks - b : kLaunchBlocks);
    if (gate)
      token_pack_kernel<2><<<here, 256, 0, s>>>(w, gate, n, k, strips, steps, b, packed);
    else
      token_pack_kernel<1><<<here, 256, 0, s>>>(w, gate, n, k, strips, steps, b, packed);
    launched("packing");
  }
}

void token_align_rows(const uint16_t* x, int64_t ldx, int64_t n, int d, uint16_t* out, int64_t ldo, hipStream_t s) {
  const int64_t blocks = (n * (ldo / 8) + 255) / 256;
  token_align_kernel<<<static_cast<unsigned>(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(x, ldx, n, d, out, ldo);
  launched("aligned rows");
}

int token_product_shape(const ProductArgs& a) { return a.gated ? best_of(kGated, a, true) : best_of(kPlain, a, false); }

void token_product_tile(int shape, bool gated, int tile[3]) {
  const Shape& t = gated ? kGated[shape] : kPlain[shape];
  tile[0] = t.bm;
  tile[1] = gated ? t.bn / 2 : t.bn;
  tile[2] = t.per_cu;
}

void token_product(const ProductArgs& args, int shape, hipStream_t s) {
  ProductArgs a = args;
  // rows of x that a tile reads, times their pitch: offsets of 32 bits?
  a.far = (a.order ? a.x_rows : 256) * a.ldx * 2 >= int64_t(1) << 32;
  a.gated ? gated(a, shape, s) : plain(a, shape, s);
  launched("product");
}

void token_combine(const CombineArgs& a, hipStream_t s) {
  const int64_t blocks = (a.n * ((a.d + 7) / 8) + 255) / 256;
  token_combine_kernel<<<static_cast<unsigned>(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(a);
  launched("weighted sum");
}

}  // namespace k
}  // namespace dycl
