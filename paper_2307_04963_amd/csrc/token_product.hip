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
#include "token_dev.hpp"

namespace dycl {
namespace k {

namespace {

constexpr int kFrag = 512;                    // elements of one 16 x 32 operand block

// ---- weights -----------------------------------------------------------------

__global__ __launch_bounds__(256) void token_pack_kernel(const uint16_t* w, const uint16_t* gate, int n, int k, int strips,
                                                         int steps, uint16_t* packed, int64_t vectors) {
  const int nb = gate ? 4 : 2;
  for (int64_t q = blockIdx.x * 256L + threadIdx.x; q < vectors; q += gridDim.x * 256L) {
    const int lane = q & 63;
    int64_t r = q >> 6;
    const int b = static_cast<int>(r % nb);
    r /= nb;
    const int step = static_cast<int>(r % steps);
    r /= steps;
    const int strip = static_cast<int>(r % strips);
    const int64_t e = r / strips;
    const int row = lane & 15, half = gate ? b >> 1 : b;
    const int o = strip * kStrip + 8 * (row >> 2) + 4 * half + (row & 3);
    const int k0 = step * 32 + 8 * (lane >> 4);
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0;
    if (o < n) {
      const uint16_t* src = (gate && (b & 1) ? gate : w) + (e * n + o) * k;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k0 + j < k) v[j] = src[k0 + j];
    }
    reinterpret_cast<uint4*>(packed)[q] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
  }
}

__global__ __launch_bounds__(256) void token_align_kernel(const uint16_t* x, int64_t ldx, int64_t n, int d, uint16_t* out,
                                                          int64_t ldo) {
  const int64_t per = ldo / 8;
  for (int64_t q = blockIdx.x * 256L + threadIdx.x; q < n * per; q += gridDim.x * 256L) {
    const int64_t row = q / per;
    const int c = static_cast<int>(q - row * per) * 8;
    const uint16_t* src = x + row * ldx + c;
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < d ? src[j] : 0;
    reinterpret_cast<uint4*>(out + row * ldo)[c / 8] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
  }
}

// ---- tiles ---------------------------------------------------------------------

// the same value in every lane, in a scalar register
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Rows [row0, row0 + rows) of the product, all of one layer.
struct Tile {
  int expert;
  int64_t row0;
  int rows;
};

// Row tile `t` of `bm` rows: expert after expert.  False past the last one.
// Every wave finds it for itself.  `total` receives the number of tiles if
// `count_all`.
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
    const int tiles = (hi - lo + bm - 1) / bm;
    int incl = tiles;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(incl, o);
      if (lane >= o) incl += u;
    }
    const uint64_t found = __ballot(t < before + incl);
    if (found) {
      const int from = __ffsll(static_cast<unsigned long long>(found)) - 1;
      const int in = static_cast<int>(t - before) - uniform(__shfl(incl, from) - __shfl(tiles, from));
      const int first = uniform(__shfl(lo, from)) + in * bm, end = uniform(__shfl(hi, from));
      out.expert = e0 + from;
      out.row0 = first;
      out.rows = end - first < bm ? end - first : bm;
      return true;
    }
    before += uniform(__shfl(incl, 63));
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
  if (p.offsets) {
    row_tiles = 0;
    const int lane = threadIdx.x & 63;
    for (int e0 = 0; e0 < p.experts; e0 += 64) {
      const int e = e0 + lane;
      const int rows = e < p.experts ? p.offsets[e + 1] - p.offsets[e] : 0;
      int tiles = (rows + bm - 1) / bm;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) tiles += __shfl_xor(tiles, o);
      row_tiles += uniform(tiles);
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
  return find_tile(p, bm, group * kGroup + (in - col * height), out);
}

__device__ __forceinline__ int64_t source_row(const ProductArgs& p, int64_t row) {
  return p.order ? p.order[row] / p.order_k : row;
}

// Eight consecutive outputs of one row from `o`: bias, activation or gate,
// residual, store.  a: the strip's first block, b: its second; ga, gb: the gate's.
template <bool GATED>
__device__ __forceinline__ void finish8(const ProductArgs& p, int expert, int64_t row, int o, f32x4 a, f32x4 b, f32x4 ga, f32x4 gb) {
  if (o >= p.N_store) return;
  float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  const float g[8] = {ga[0], ga[1], ga[2], ga[3], gb[0], gb[1], gb[2], gb[3]};
  const float* bias = p.bias ? p.bias + static_cast<int64_t>(expert) * p.N : nullptr;
  const float* gbias = GATED && p.gate_bias ? p.gate_bias + static_cast<int64_t>(expert) * p.N : nullptr;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (bias && o + j < p.N) v[j] += bias[o + j];
    if (GATED) {
      float u = g[j];
      if (gbias && o + j < p.N) u += gbias[o + j];
      v[j] *= token_act(u, p.act);
    } else {
      v[j] = token_act(v[j], p.act);
    }
  }
  if (o + 8 > p.N) {
    // the padding's zero weights make NaN of an infinite input: what is stored there is 0
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (o + j >= p.N) v[j] = 0.f;
  }
  const bool whole = o + 8 <= p.N_store;
  if (p.residual) {
    const uint16_t* r = p.residual + row * p.ldr + o;
    if (whole && reinterpret_cast<uintptr_t>(r) % 16 == 0) {
      const uint4 q = *reinterpret_cast<const uint4*>(r);
      const uint32_t e[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] += __uint_as_float(e[j] << 16);
        v[2 * j + 1] += __uint_as_float(e[j] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (o + j < p.N_store) v[j] += bf2f(r[j]);
    }
  }
  if (p.y_f32) {
    float* y = static_cast<float*>(p.y) + row * p.ldy + o;
    if (whole && reinterpret_cast<uintptr_t>(y) % 16 == 0) {
      reinterpret_cast<float4*>(y)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(y)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (o + j < p.N_store) y[j] = v[j];
    }
  } else {
    uint16_t* y = static_cast<uint16_t*>(p.y) + row * p.ldy + o;
    if (whole && reinterpret_cast<uintptr_t>(y) % 16 == 0) {
      *reinterpret_cast<uint4*>(y) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (o + j < p.N_store) y[j] = f2bf(v[j]);
    }
  }
}

// ---- few rows per layer: the weights go from memory to the registers --------------

// A workgroup takes one strip of 32 outputs for up to 16 TB rows of one layer;
// its waves take the K steps in turn and add their sums through LDS.
template <int TB, bool GATED, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void token_skinny_kernel(ProductArgs p, int strips, int steps) {
  constexpr int NB = GATED ? 4 : 2, ACC = TB * NB;
  constexpr int U = TB == 1 ? 4 : 2;           // steps whose operands are in flight together
  __shared__ f32x4 sums[WAVES][ACC][64];
  Tile tile;
  const int64_t t = blockIdx.x / strips;
  const int strip = static_cast<int>(blockIdx.x - t * strips);
  if (!find_tile(p, 16 * TB, t, tile)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  const uint16_t* xr[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    const int r = b * 16 + (lane & 15);
    xr[b] = p.x + source_row(p, tile.row0 + (r < tile.rows ? r : tile.rows - 1)) * p.ldx + 8 * (lane >> 4);
  }
  const bf16x8* w = reinterpret_cast<const bf16x8*>(p.w) +
                    (static_cast<int64_t>(tile.expert) * strips + strip) * steps * (NB * 64) + lane;
  f32x4 acc[TB][NB];
#pragma unroll
  for (int b = 0; b < TB; ++b)
#pragma unroll
    for (int c = 0; c < NB; ++c) acc[b][c] = f32x4{0.f, 0.f, 0.f, 0.f};

  // wave i takes steps [i, i + 1) * steps / WAVES
  const int s0 = wave * steps / WAVES, s1 = (wave + 1) * steps / WAVES;
  const int k_lane = 8 * (lane >> 4);
  for (int s = s0; s < s1; s += U) {
    bf16x8 wf[U][NB], xf[U][TB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int su = s + u < s1 ? s + u : s1 - 1;
#pragma unroll
      for (int c = 0; c < NB; ++c) wf[u][c] = w[(static_cast<int64_t>(su) * NB + c) * 64];
      const bool in = s + u < s1 && su * 32 + k_lane < p.K;
#pragma unroll
      for (int b = 0; b < TB; ++b) {
        uint4 q = make_uint4(0, 0, 0, 0);
        if (in) q = *reinterpret_cast<const uint4*>(xr[b] + su * 32);
        xf[u][b] = __builtin_bit_cast(bf16x8, q);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int b = 0; b < TB; ++b)
#pragma unroll
        for (int c = 0; c < NB; ++c)
          acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[u][c], xf[u][b], acc[b][c], 0, 0, 0);
  }
#pragma unroll
  for (int b = 0; b < TB; ++b)
#pragma unroll
    for (int c = 0; c < NB; ++c) sums[wave][b * NB + c][lane] = acc[b][c];
  __syncthreads();
  for (int b = wave; b < TB; b += WAVES) {
    f32x4 r[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) r[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
      for (int i = 0; i < WAVES; ++i) r[c] += sums[i][b * NB + c][lane];
    const int row = b * 16 + (lane & 15);
    const int o = strip * kStrip + 8 * (lane >> 4);
    if (row < tile.rows) {
      if (GATED)
        finish8<true>(p, tile.expert, tile.row0 + row, o, r[0], r[2], r[1], r[3]);
      else
        finish8<false>(p, tile.expert, tile.row0 + row, o, r[0], r[1], r[0], r[1]);
    }
  }
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
// 2 h + 1, group 1 one half later.  So stage h % S is read by all after half 2 h + 1
// and takes the loads of step h + S from half 2 h + 2 on (in the group's read of
// step h + 1), and what a wave requested for step h + 1 has to be there before half
// 2 h + 2: it waits for that at the end of its read of step h.
__device__ __align__(16) const uint16_t g_zeros[8] = {0, 0, 0, 0, 0, 0, 0, 0};

template <int N>
__device__ __forceinline__ void wait_all_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int BM, int BN, int WM, int WN, int S, bool GATED>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(2)))
void token_tile_kernel(ProductArgs p, int strips, int steps, int col_tiles) {
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
  __shared__ __align__(16) char smem[S * STAGE];

  Tile tile;
  int col;
  if (!tile_of(p, BM, col_tiles, tile, col)) return;
  const int strip0 = col * TS;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;

  // this thread's rows of x and the K chunk that it loads of each
  const uint16_t* a_src[JA];
  int a_k[JA];
#pragma unroll
  for (int j = 0; j < JA; ++j) {
    const int r = (j * NT + tid) >> 2;
    const int chunk = ((tid & 3) ^ -(r >> 2)) & 3;
    a_k[j] = chunk * 8;
    a_src[j] = p.x + source_row(p, tile.row0 + (r < tile.rows ? r : tile.rows - 1)) * p.ldx + chunk * 8;
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
  auto load = [&](int h, char* stage) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < JA; ++j) {
      const uint16_t* src = a_src[j] + h * 32;
      if (h * 32 + a_k[j] >= p.K) src = g_zeros;
      load_lds16(src, stage + (j * NT + wave * 64) * 16);
    }
#pragma unroll
    for (int j = 0; j < JB; ++j)
      load_lds16(b_base, b_off[j] + static_cast<uint32_t>(h) * (NB * kFrag * 2), stage + A_BYTES + (j * NT + wave * 64) * 16);
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

#pragma unroll
  for (int b = 0; b < TB; ++b) {
    const int row = wm * WTM + b * 16 + (lane & 15);
    if (row >= tile.rows) continue;
#pragma unroll
    for (int c = 0; c < RB; c += NB) {
      const int strip = strip0 + (wn * RB + c) / NB;
      const int o = strip * kStrip + 8 * (lane >> 4);
      if (GATED)
        finish8<true>(p, tile.expert, tile.row0 + row, o, acc[b][c], acc[b][c + 2], acc[b][c + 1], acc[b][c + 3]);
      else
        finish8<false>(p, tile.expert, tile.row0 + row, o, acc[b][c], acc[b][c + 1], acc[b][c], acc[b][c + 1]);
    }
  }
}

// ---- the experts' results, weighted and summed ----------------------------------------

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
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (o + j < p.d) v[j] = bf2f(r[j]);
    }
    for (int j = 0; j < p.k; ++j) {
      const int slot = p.slots[row * p.k + j];
      if (slot < 0) continue;
      const float w = p.weights[row * p.k + j];
      const uint4 f = *reinterpret_cast<const uint4*>(p.part + slot * p.ldp + o);
      const uint32_t e[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = fmaf(w, __uint_as_float(e[i] << 16), v[2 * i]);
        v[2 * i + 1] = fmaf(w, __uint_as_float(e[i] & 0xffff0000u), v[2 * i + 1]);
      }
    }
    uint16_t* out = p.out + row * p.ldo + o;
    if (whole && reinterpret_cast<uintptr_t>(out) % 16 == 0) {
      *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
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

template <int TB, bool GATED>
void skinny(const ProductArgs& a, hipStream_t s) {
  const int strips = strips_of(a.N), steps = steps_of(a.K);
  token_skinny_kernel<TB, GATED, 4><<<static_cast<unsigned>(row_tiles(a, 16 * TB) * strips), 256, 0, s>>>(a, strips, steps);
}

template <int BM, int BN, int WM, int WN, int S, bool GATED>
void tiles(const ProductArgs& a, hipStream_t s) {
  const int strips = strips_of(a.N), steps = steps_of(a.K), per = BN / (GATED ? 64 : 32);
  const int cols = (strips + per - 1) / per;
  token_tile_kernel<BM, BN, WM, WN, S, GATED>
      <<<static_cast<unsigned>(row_tiles(a, BM) * cols), 64 * WM * WN, 0, s>>>(a, strips, steps, cols);
}

template <bool GATED>
void product(const ProductArgs& a, hipStream_t s) {
  const int64_t per = a.offsets ? a.rows / a.experts : a.rows;     // rows of a layer, on average
  if (per <= 16) return skinny<1, GATED>(a, s);
  if (per <= 32) return skinny<2, GATED>(a, s);
#ifndef SX
#define SX 4
#endif
  if (per <= 512) return tiles<128, 256, 2, 4, SX, GATED>(a, s);
  tiles<256, 256, 2, 4, SX, GATED>(a, s);
}

}  // namespace

void token_pack(const uint16_t* w, const uint16_t* gate, int experts, int n, int k, uint16_t* packed, hipStream_t s) {
  const int64_t vectors = static_cast<int64_t>(packed_elements(experts, n, k, gate != nullptr) / 8);
  const int64_t blocks = (vectors + 255) / 256;
  token_pack_kernel<<<static_cast<unsigned>(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(w, gate, n, k, strips_of(n), steps_of(k), packed, vectors);
}

void token_align_rows(const uint16_t* x, int64_t ldx, int64_t n, int d, uint16_t* out, int64_t ldo, hipStream_t s) {
  const int64_t blocks = (n * (ldo / 8) + 255) / 256;
  token_align_kernel<<<static_cast<unsigned>(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(x, ldx, n, d, out, ldo);
}

void token_product(const ProductArgs& a, hipStream_t s) { a.gated ? product<true>(a, s) : product<false>(a, s); }

void token_combine(const CombineArgs& a, hipStream_t s) {
  const int64_t blocks = (a.n * ((a.d + 7) / 8) + 255) / 256;
  token_combine_kernel<<<static_cast<unsigned>(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(a);
}

}  // namespace k
}  // namespace dycl
