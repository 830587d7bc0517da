// The norm after a block, its gate, the residual sum and the norm before the
// next block in one pass:
//   z = post(y) * act(gate) * channel_scale * row_gate;  h = a x + z;  u = pre(h)
// Bound by HBM: x, y and the gate are read once, h and u written once.  T
// lanes hold a row in registers, so both norms' statistics (float32; the
// layer norm's variance from the centred values) come from one read.  A
// workgroup walks over rows with the weights in registers up to 8192 values (read
// for every row they would double the loads), and requests the next row before
// it reduces the present one.  Rows at any alignment are read 16 bytes per lane;
// element by element, 1999 rows of 1003 took twice as long.  Beyond 16384 values
// the row ahead does not fit the registers and goes through scratch, from 8193 on
// where 8 does not divide the row: about half the rate.
//
// Measured: 16384 x 4096 in bf16, both norms, 537 MB in 102 us = 5.3 TB/s, about the
// rate of a plain copy (5.2 to 5.5); 1999 x 1003, x in float32, with a gate, row gates
// and biases 10 to 12 us, where the bytes would take 5 (three dependent trips to memory
// before a row ends: the weights, a row's gate and then its values, and the gate's
// behind the first norm); 1 x 2048 2.8 us, a launch.
#include "token_dev.hpp"

namespace dycl {
namespace k {

namespace {

// 8 elements of a row, as loaded
template <bool F32>
struct Raw {
  uint4 v[F32 ? 2 : 1];
};

// 8 consecutive elements from `i0` (rows may start at any element); TAIL: a row's
// last ones are fewer
template <bool F32, bool TAIL>
__device__ __forceinline__ Raw<F32> load8(const void* row, int i0, int d) {
  Raw<F32> r;
#pragma unroll
  for (int q = 0; q < (F32 ? 2 : 1); ++q) r.v[q] = make_uint4(0, 0, 0, 0);
  if (TAIL ? i0 + 8 <= d : i0 < d) {
    const char* p = static_cast<const char*>(row) + static_cast<size_t>(i0) * (F32 ? 4 : 2);
#pragma unroll
    for (int q = 0; q < (F32 ? 2 : 1); ++q) r.v[q] = load16(p + 16 * q);
  } else if (TAIL && i0 < d) {
    uint32_t e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      e[j] = 0;
      if (i0 + j < d) e[j] = F32 ? static_cast<const uint32_t*>(row)[i0 + j] : static_cast<const uint16_t*>(row)[i0 + j];
    }
    if constexpr (F32) {
      r.v[0] = make_uint4(e[0], e[1], e[2], e[3]);
      r.v[1] = make_uint4(e[4], e[5], e[6], e[7]);
    } else {
      r.v[0] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    }
  }
  return r;
}

template <bool F32>
__device__ __forceinline__ void unpack8(const Raw<F32>& r, float* f) {
  if constexpr (F32) {
    const uint32_t e[8] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w, r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w};
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(e[j]);
  } else {
    const uint32_t e[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f[2 * j] = __uint_as_float(e[j] << 16);
      f[2 * j + 1] = __uint_as_float(e[j] & 0xffff0000u);
    }
  }
}

template <bool TAIL>
__device__ __forceinline__ void store8(void* row, bool f32, int i0, int d, const float* f) {
  if (TAIL ? i0 + 8 <= d : i0 < d) {
    if (f32) {
      float* p = static_cast<float*>(row) + i0;
      store16(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
      store16(p + 4, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
    } else {
      store16(static_cast<uint16_t*>(row) + i0, make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])));
    }
  } else if (TAIL && i0 < d) {
#pragma unroll
    for (int j = 0; j < 7; ++j) {
      if (i0 + j >= d) continue;
      if (f32)
        static_cast<float*>(row)[i0 + j] = f[j];
      else
        static_cast<uint16_t*>(row)[i0 + j] = f2bf(f[j]);
    }
  }
}

// the sum over the T lanes of a row; `slot` is this reduction's own LDS
template <int T>
__device__ __forceinline__ float row_sum(float v, float* slot) {
  v = wave_sum(v);
  if constexpr (T > 64) {
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) v += slot[w];
  }
  return v;
}

template <int T, int NV, bool TAIL, bool XF, bool YF, bool BIAS>
__global__ __launch_bounds__(T < 256 ? 256 : T) void token_norm_kernel(NormArgs p) {
  constexpr int ROWS = T < 256 ? 256 / T : 1;
  // a reduction's slot is written again two rows later at the earliest, with
  // a barrier of the row between
  __shared__ float slots[2][4][T > 64 ? T / 64 : 1];
  const int t = threadIdx.x % T;
  const int64_t step = static_cast<int64_t>(gridDim.x) * ROWS;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / T;
  const int d = p.d;
  auto at = [&](int i) { return (i * T + t) * 8; };
  auto in = [&](int i, int j) { return TAIL ? at(i) + j < d : at(i) < d; };

  // post's weight and bias with the channel's scale, pre's weight and bias: kept, or
  // (of the widest rows, which leave no room) read again for every row
  constexpr bool KEEP = T < 512;
  constexpr int NW = KEEP ? NV : 1;
  float pw[NW][8], pb[NW][8], qw[NW][8], qb[NW][8];
  auto weights = [&](const float* w, int i, float otherwise, float (&out)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = otherwise;
    if (w) unpack8<true>(load8<true, TAIL>(w, at(i), d), out);
  };
  auto post_weights = [&](int i) __attribute__((always_inline)) {
    const int k = KEEP ? i : 0;
    float scale[8];
    weights(p.channel_scale, i, 1.f, scale);
    weights(p.post_w, i, 1.f, pw[k]);
    if (BIAS) weights(p.post_b, i, 0.f, pb[k]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      pw[k][j] *= scale[j];
      if (BIAS) pb[k][j] *= scale[j];
    }
  };
  auto pre_weights = [&](int i) __attribute__((always_inline)) {
    const int k = KEEP ? i : 0;
    weights(p.pre_w, i, 1.f, qw[k]);
    if (BIAS) weights(p.pre_b, i, 0.f, qb[k]);
  };
  if constexpr (KEEP) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      post_weights(i);
      pre_weights(i);
    }
  }

  const float inv_d = 1.0f / static_cast<float>(d);
  Raw<XF> xr[NV];
  Raw<YF> yr[NV];
  float rg = 1.f;
  auto request = [&](int64_t row) {
    rg = p.row_gate ? p.row_gate[row] : 1.f;
    const char* xp = static_cast<const char*>(p.x) + row * p.ldx * (XF ? 4 : 2);
    const char* yp = static_cast<const char*>(p.y) + row * p.ldy * (YF ? 4 : 2);
#pragma unroll
    for (int i = 0; i < NV; ++i) xr[i] = load8<XF, TAIL>(xp, at(i), d);
    if (p.y && rg != 0.f) {
#pragma unroll
      for (int i = 0; i < NV; ++i) yr[i] = load8<YF, TAIL>(yp, at(i), d);
    }
  };

  if (first >= p.n) return;
  request(first);
  int parity = 0;
  // (T > 64: a row per workgroup, so every lane takes the same turns)
  for (int64_t row = first; row < p.n; row += step, parity ^= 1) {
    float h[NV][8], z[NV][8];
    const float gate_of_row = rg;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      unpack8<XF>(xr[i], h[i]);
      unpack8<YF>(yr[i], z[i]);
    }
    if (row + step < p.n) request(row + step);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] *= p.residual_scale;

    // (a skipped row takes its turn in the reductions, of zeros)
    if (p.y) {
      if (gate_of_row == 0.f) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) z[i][j] = 0.f;
      }
      float mean = 0.f, inv = 1.f;
      if (p.post == 2) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) s += z[i][j];
        mean = row_sum<T>(s, slots[parity][0]) * inv_d;
      }
      if (p.post != 0) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float c = in(i, j) ? z[i][j] - mean : 0.f;
            s = fmaf(c, c, s);
          }
        inv = rsqrtf(row_sum<T>(s, slots[parity][1]) * inv_d + p.eps);
      }
      if (gate_of_row != 0.f) {
        const char* gp = static_cast<const char*>(p.gate) + row * p.ldg * (YF ? 4 : 2);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int k = KEEP ? i : 0;
          if (!KEEP) post_weights(i);
          float g[8];
          if (p.gate) unpack8<YF>(load8<YF, TAIL>(gp, at(i), d), g);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float v = (z[i][j] - mean) * inv;
            v = BIAS ? fmaf(v, pw[k][j], pb[k][j]) : v * pw[k][j];
            if (p.gate) v *= p.gate_act == 0 ? g[j] : (p.gate_act == 1 ? 1.f : g[j]) * sigmoid_fast(g[j]);
            h[i][j] = fmaf(v, gate_of_row, h[i][j]);
          }
        }
      }
    }
    if (p.h) {
      char* hp = static_cast<char*>(p.h) + row * p.ldh * (XF ? 4 : 2);
#pragma unroll
      for (int i = 0; i < NV; ++i) store8<TAIL>(hp, XF, at(i), d, h[i]);
    }
    if (p.u) {
      float mean = 0.f, inv = 1.f;
      if (p.pre == 2) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) s += in(i, j) ? h[i][j] : 0.f;
        mean = row_sum<T>(s, slots[parity][2]) * inv_d;
      }
      if (p.pre != 0) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float c = in(i, j) ? h[i][j] - mean : 0.f;
            s = fmaf(c, c, s);
          }
        inv = rsqrtf(row_sum<T>(s, slots[parity][3]) * inv_d + p.eps);
      }
      char* up = static_cast<char*>(p.u) + row * p.ldu * (p.u_f32 ? 4 : 2);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int k = KEEP ? i : 0;
        if (!KEEP) pre_weights(i);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float c = (h[i][j] - mean) * inv;
          v[j] = BIAS ? fmaf(c, qw[k][j], qb[k][j]) : c * qw[k][j];
        }
        store8<TAIL>(up, p.u_f32, at(i), d, v);
      }
    }
  }
}

template <int T, int NV, bool TAIL, bool XF, bool YF>
void launch(const NormArgs& a, hipStream_t s) {
  constexpr int NT = T < 256 ? 256 : T, ROWS = T < 256 ? 256 / T : 1;
  const int64_t blocks = (a.n + ROWS - 1) / ROWS;
  const int most = 256 * (T >= 512 ? 2 : 6);
  const dim3 grid(static_cast<unsigned>(blocks < most ? blocks : most));
  if (a.post_b || a.pre_b)
    token_norm_kernel<T, NV, TAIL, XF, YF, true><<<grid, NT, 0, s>>>(a);
  else
    token_norm_kernel<T, NV, TAIL, XF, YF, false><<<grid, NT, 0, s>>>(a);
  launched("norm");
}

template <int T, int NV, bool TAIL>
void by_type(const NormArgs& a, hipStream_t s) {
  if (a.x_f32)
    a.y_f32 ? launch<T, NV, TAIL, true, true>(a, s) : launch<T, NV, TAIL, true, false>(a, s);
  else
    a.y_f32 ? launch<T, NV, TAIL, false, true>(a, s) : launch<T, NV, TAIL, false, false>(a, s);
}

// Lanes per row and pieces of 8 values per lane, both norms over 2^26 values in bf16
// (us, beside another form that holds the row): 512 as <64, 1> 100 (<64, 2> 122); 1024 as
// <64, 2> 103 (<256, 1> 119); 2048 as <256, 1> 101 (<64, 4> 100, but 32 rows 3.3 against 5.0);
// 4096 as <256, 2> 102 (<512, 1> 115); 8192 as <256, 4> 99 (<512, 2> 102); 12288 as <1024, 2> 111
// (<512, 4> 123); 16384 as <1024, 2> 108 (<512, 4> 120); 16001 180 (189); 32768 171, 20001 314.
template <bool TAIL>
void by_size(const NormArgs& a, hipStream_t s) {
  if (a.d <= 512) return by_type<64, 1, TAIL>(a, s);
  if (a.d <= 1024) return by_type<64, 2, TAIL>(a, s);
  if (a.d <= 2048) return by_type<256, 1, TAIL>(a, s);
  if (a.d <= 4096) return by_type<256, 2, TAIL>(a, s);
  if (a.d <= 8192) return by_type<256, 4, TAIL>(a, s);
  if (a.d <= 16384) return by_type<1024, 2, TAIL>(a, s);
  by_type<1024, 4, TAIL>(a, s);
}

}  // namespace

void token_norm(const NormArgs& a, hipStream_t s) { a.d % 8 ? by_size<true>(a, s) : by_size<false>(a, s); }

}  // namespace k
}  // namespace dycl
