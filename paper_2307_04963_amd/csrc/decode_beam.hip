// The choice of the next tokens: the k largest of scores[w] + log softmax(logits[w])[t]
// over a sequence's beams w and words t, the lowest w * words + t among equals.
//
// log softmax only shifts a beam's logits, so a beam's best candidates are those of its
// logits.  A workgroup takes a segment of a row into registers: sum of exponentials
// around its maximum, and its k largest.  From the lanes' maxima comes a bound that k values reach
// and few others; those that reach it go to LDS and are ranked by counting the larger ones.  Where more reach it than LDS
// holds (a row of equal values) the k are taken one after the other.  A second kernel sums a beam's segments, in order, and
// takes the k largest of the segments' lists the same way.
//
// Bound by HBM in float32 (a logit is read once); about 12 vector instructions per logit, the exponential at a quarter of their
// rate, which is 25 us for 67 million.  Measured: 512 rows of 131072 logits in float32 44 us
// (6.0 TB/s; 54 behind a reordering whose writes are still on their way), in bf16 38 us (3.5 TB/s), where neither the bytes (25 us)
// nor the instructions are the bound: a workgroup's requests, its sums and its list follow one another;
// the second kernel 4 us for one sequence, 6 for 64 of 1024 candidates, 13 for 16 of 12800.
#include "decode_dev.hpp"

namespace dycl {
namespace k {

namespace {

constexpr int kThreads = 256, kWaves = 4, kRoom = 512;
constexpr float kClosed = -__builtin_inff(), kLog2e = 1.44269504088896340736f, kLargest = 3.402823466e38f, kFar = 1e6f;

// a value and an index as one number: larger values first, then lower indices; 0 is none
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);       // (-0 becomes 0: they are equal)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) {
  return v == kClosed ? 0 : static_cast<uint64_t>(ordered(v)) << 32 | (0xffffffffu - index);
}
__device__ __forceinline__ uint32_t index_of(uint64_t key) { return 0xffffffffu - static_cast<uint32_t>(key); }

// a bound that at least k of the wave's 64 values reach, within 2^-7 below the k-th largest; -inf where fewer are open
__device__ __forceinline__ float bound_of(float v, int k) {
  const uint32_t o = ordered(v) >> 16;
  uint32_t t = 0;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t with = t | 1u << bit;
    if (__popcll(__ballot(o >= with)) >= k) t = with;
  }
  return t <= (ordered(kClosed) >> 16) ? kClosed : value_of(t << 16);
}

struct Chosen {                        // in LDS
  uint64_t keys[kRoom];
  uint64_t best[kWaves];
  float bounds[2][kWaves];
  int count;
};

// A bound that k of the workgroup's values reach if v is each lane's largest; -inf where fewer lanes are
// open: the larger of two such, the least of the waves' ceil(k / 4)-th largest (close where the waves are alike) and the
// largest of their k-th (where one has most of them).  All threads call it; what was written to LDS before is visible
// after it.
__device__ __forceinline__ float bound_of_all(Chosen& s, float v, int k) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float share = bound_of(v, (k + kWaves - 1) / kWaves), alone = bound_of(v, k);
  if (lane == 0) s.bounds[0][wave] = share, s.bounds[1][wave] = alone;
  __syncthreads();
  return fmaxf(fminf(fminf(s.bounds[0][0], s.bounds[0][1]), fminf(s.bounds[0][2], s.bounds[0][3])),
               fmaxf(fmaxf(s.bounds[1][0], s.bounds[1][1]), fmaxf(s.bounds[1][2], s.bounds[1][3])));
}

// The k largest of the candidates in `s`: rank r's key to put(r, key), r below the number of them and k.
template <class PUT>
__device__ __forceinline__ void rank_all(const Chosen& s, int k, PUT&& put) {
  const int n = s.count;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t key = s.keys[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += s.keys[j] > key;
    if (rank < k) put(rank, key);
  }
}

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) {
    const uint64_t o = static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(v), w));
    v = o > v ? o : v;
  }
  return v;
}

struct Segments {
  int count, size;                     // of a row; words of one
  float2* state;                       // [row][segment]: maximum, sum of exponentials around it
  uint64_t* lists;                     // [row][segment][k] keys, largest first, 0 past the last
};

// the wave's largest, in all lanes
__device__ __forceinline__ float wave_top(float v) {
  v = fmaxf(v, rotate16<8>(v));
  v = fmaxf(v, rotate16<4>(v));
  v = fmaxf(v, rotate16<2>(v));
  v = fmaxf(v, rotate16<1>(v));
  return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}

// V: groups of 8 values per lane
template <bool F32, int V>
__global__ __launch_bounds__(kThreads) void segment_kernel(BeamArgs p, Segments g, uint32_t base) {
  __shared__ Chosen s;
  __shared__ float2 waves[kWaves];
  // W consecutive values per lane and request (16 bytes), `kThreads * W` further on the next
  constexpr int kSize = kThreads * 8 * V, W = F32 ? 4 : 8, kBytes = F32 ? 4 : 2;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t item = base + blockIdx.x;
  const uint32_t row = item / g.count;
  const int start = static_cast<int>(item - row * g.count) * kSize, first = start + W * threadIdx.x;
  auto index = [&](int i) { return first + i / W * (kThreads * W) + i % W; };
  const char* from = static_cast<const char*>(p.logits) + (static_cast<int64_t>(row) * p.ldl + first) * kBytes;
  float v[8 * V];
  if (start + kSize <= p.words) {                      // (all requests at once, no tests between them)
    uint4 raw[8 * V / W];
#pragma unroll
    for (int i = 0; i < 8 * V / W; ++i) raw[i] = load16(from + i * kThreads * 16);
#pragma unroll
    for (int i = 0; i < 8 * V / W; ++i) {
      const uint32_t e[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (F32) {
          v[4 * i + j] = __uint_as_float(e[j]);
        } else {
          v[8 * i + 2 * j] = __uint_as_float(e[j] << 16);
          v[8 * i + 2 * j + 1] = __uint_as_float(e[j] & 0xffff0000u);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) {
      v[i] = kClosed;
      const char* at = from + (i / W * (kThreads * W) + i % W) * kBytes;
      if (index(i) < p.words) v[i] = F32 ? *reinterpret_cast<const float*>(at) : bf2f(*reinterpret_cast<const uint16_t*>(at));
    }
  }
  if (threadIdx.x == 0) s.count = 0;
  // beams without candidates of their own: the second kernel skips them too
  const float score = p.scores[row];
  if ((p.ended && p.ended[row]) || !(score > kClosed)) return;     // (the same for the whole workgroup)
  float tops[2 * V], top, m, sum = 0.f;                // of four values, of all the lane's, of the wave's
  auto maxima = [&] {
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) tops[i] = fmaxf(fmaxf(v[4 * i], v[4 * i + 1]), fmaxf(v[4 * i + 2], v[4 * i + 3]));
    top = tops[0];
#pragma unroll
    for (int i = 1; i < 2 * V; ++i) top = fmaxf(top, tops[i]);
    m = wave_top(top);
  };
  maxima();
  // Ordinary values: 2^(v log2 e - a) by one multiplication and addition, a the rounded m log2 e, and what that
  // rounding took, less than 2^-3 up to kFar, put right at the end.  (From 10^9 on it passes the exponential's range.)
  const float a = m == kClosed ? 0.f : m * kLog2e;
#pragma unroll
  for (int i = 0; i < 8 * V; ++i) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(v[i], kLog2e, -a));
  if (m != kClosed) sum *= __builtin_amdgcn_exp2f(-__builtin_fmaf(m, kLog2e, -a));
  if (__any(!(sum < kLargest)) || (m != kClosed && !(fabsf(m) < kFar))) {
    // NaN among them, which is closed, +infinity, which is the largest finite value, or values far from 0
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) v[i] = fminf(fmaxf(v[i], kClosed), kLargest);
    maxima();
    const float around = m == kClosed ? 0.f : m;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) sum += __builtin_amdgcn_exp2f((v[i] - around) * kLog2e);
  }
  sum = wave_sum(sum);
  if (lane == 0) waves[wave] = make_float2(m, sum);
  const float bound = bound_of_all(s, top, p.k);
  if (threadIdx.x == 0) {
    const float all = fmaxf(fmaxf(waves[0].x, waves[1].x), fmaxf(waves[2].x, waves[3].x)), base2 = all == kClosed ? 0.f : all;
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += __builtin_amdgcn_exp2f((waves[w].x - base2) * kLog2e) * waves[w].y;
    g.state[item] = make_float2(all, total);
  }
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) {
    if (!__any(tops[i] >= bound)) continue;            // (few: most are one comparison for four values of 64 lanes)
#pragma unroll
    for (int j = 4 * i; j < 4 * i + 4; ++j)
      if (v[j] >= bound && v[j] > kClosed) {
        const int at = atomicAdd(&s.count, 1);
        if (at < kRoom) s.keys[at] = key_of(v[j], index(j));
      }
  }
  __syncthreads();
  uint64_t* list = g.lists + static_cast<int64_t>(item) * p.k;
  if (s.count <= kRoom) {
    rank_all(s, p.k, [&](int rank, uint64_t key) { list[rank] = key; });
    for (int i = s.count + threadIdx.x; i < p.k; i += kThreads) list[i] = 0;
    return;
  }
  uint64_t before = ~uint64_t(0);
  for (int round = 0; round < p.k; ++round) {
    uint64_t best = 0;
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) {
      const uint64_t key = key_of(v[i], index(i));
      best = key < before && key > best ? key : best;
    }
    best = wave_max(best);
    if (lane == 0) s.best[wave] = best;
    __syncthreads();
    best = max(max(s.best[0], s.best[1]), max(s.best[2], s.best[3]));
    if (threadIdx.x == 0) list[round] = best;
    before = best;
    __syncthreads();
  }
}

// One sequence: its beams' sums, then the k largest of all lists.  FLAT: a thread keeps up to kFlat of the lists' entries,
// requested at once.  Else the k lists with the largest first entries are chosen (any other's first entry has k
// larger ones), and their entries, k * k at most, kept.
constexpr int kFlat = 8, kKept = kBeamMaxK * kBeamMaxK / kThreads;
template <bool FLAT>
__global__ __launch_bounds__(kThreads) void choose_kernel(BeamArgs p, Segments g) {
  __shared__ Chosen s;
  __shared__ float2 shift[kBeamMaxBeams];      // a beam's largest logit, and the value of that one; -inf: none of its logits
  __shared__ float kept[kBeamMaxBeams];        // an ended beam's score, -inf: it has not ended
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t b = blockIdx.x;
  const int lists = p.beams * g.count, entries = lists * p.k;
  const uint64_t* all = g.lists + b * entries;
  uint64_t own[FLAT ? kFlat : kKept];
  if constexpr (FLAT) {
    // The lists' first entries first, so that every wave has some of them.  (Of a beam without candidates the entries are
    // whatever the workspace held; they are not used.)
#pragma unroll
    for (int j = 0; j < kFlat; ++j) {
      const int i = threadIdx.x + j * kThreads;
      own[j] = 0;
      if (j * kThreads < entries && i < entries) own[j] = all[i % lists * p.k + i / lists];
    }
  }
  if (threadIdx.x == 0) s.count = 0;
  // 16 lanes per beam
  const int part = threadIdx.x & 15;
  for (int w = threadIdx.x >> 4; w < p.beams; w += kThreads / 16) {
    const int64_t row = b * p.beams + w;
    const float given = p.scores[row], score = fminf(given, kLargest);
    const bool open = given > kClosed, over = p.ended && p.ended[row], reads = open && !over;
    const float2* state = g.state + row * g.count;
    float2 one[2];                             // (its first ones, requested at once)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      one[j] = make_float2(kClosed, 0.f);
      if (part + 16 * j < g.count) one[j] = state[part + 16 * j];
      if (!reads) one[j] = make_float2(kClosed, 0.f);
    }
    float m = fmaxf(one[0].x, one[1].x);
    for (int i = part + 32; i < g.count && reads; i += 16) m = fmaxf(m, state[i].x);
    m = fmaxf(m, rotate16<8>(m));
    m = fmaxf(m, rotate16<4>(m));
    m = fmaxf(m, rotate16<2>(m));
    m = fmaxf(m, rotate16<1>(m));
    float total = 0.f;
    if (m > kClosed) {
      total = __builtin_amdgcn_exp2f((one[0].x - m) * kLog2e) * one[0].y + __builtin_amdgcn_exp2f((one[1].x - m) * kLog2e) * one[1].y;
      for (int i = part + 32; i < g.count; i += 16) total += __builtin_amdgcn_exp2f((state[i].x - m) * kLog2e) * state[i].y;
    }
    total = sum16(total);
    if (part == 0) {
      shift[w] = make_float2(m, score - logf(total));
      kept[w] = open && over ? score : kClosed;
    }
  }
  __syncthreads();
  // (a sum past the least finite value is closed, as -infinity is)
  auto valued = [&](uint64_t key, int w) -> uint64_t {
    if (!key || shift[w].x == kClosed) return 0;
    return key_of((value_of(static_cast<uint32_t>(key >> 32)) - shift[w].x) + shift[w].y, w * p.words + index_of(key));
  };
  const uint64_t ended = threadIdx.x < p.beams && kept[threadIdx.x] > kClosed ? key_of(kept[threadIdx.x], threadIdx.x * p.words + p.end) : 0;
  auto value_at = [](uint64_t key) { return key ? value_of(static_cast<uint32_t>(key >> 32)) : kClosed; };
  // keys that reach the bound, into LDS; visible after it
  auto take = [&](uint64_t key, float bound) {
    if (!key || value_at(key) < bound) return;
    const int at = atomicAdd(&s.count, 1);
    if (at < kRoom) s.keys[at] = key;
  };
  // the largest of the workgroup's best(before), those of each thread below `before`
  auto next = [&](uint64_t best) {
    best = wave_max(best);
    if (lane == 0) s.best[wave] = best;
    __syncthreads();
    best = max(max(s.best[0], s.best[1]), max(s.best[2], s.best[3]));
    __syncthreads();
    return best;
  };
  if constexpr (FLAT) {
#pragma unroll
    for (int j = 0; j < kFlat; ++j) {
      const int i = threadIdx.x + j * kThreads;
      if (j * kThreads < entries && i < entries) own[j] = valued(own[j], i % lists / g.count);
    }
  } else {
    __shared__ int chosen[kBeamMaxK];
    auto key_at = [&](int list, int i) {         // (a list of a closed beam is not read)
      const int w = list / g.count;
      return shift[w].x == kClosed ? uint64_t(0) : valued(all[static_cast<int64_t>(list) * p.k + i], w);
    };
    auto list_of = [&](uint64_t key) {
      const int w = static_cast<int>(index_of(key) / p.words);
      return w * g.count + static_cast<int>(index_of(key) - w * p.words) / g.size;
    };
    if (threadIdx.x < p.k) chosen[threadIdx.x] = -1;
    uint64_t head = 0;
    for (int i = threadIdx.x; i < lists; i += kThreads) head = max(head, key_at(i, 0));
    const float bound = bound_of_all(s, value_at(head), p.k);
    for (int i = threadIdx.x; i < lists; i += kThreads) take(key_at(i, 0), bound);
    __syncthreads();
    if (s.count <= kRoom) {
      rank_all(s, p.k, [&](int rank, uint64_t key) { chosen[rank] = list_of(key); });
    } else {
      uint64_t before = ~uint64_t(0);
      for (int round = 0; round < p.k; ++round) {
        uint64_t best = 0;
        for (int i = threadIdx.x; i < lists; i += kThreads) {
          const uint64_t key = key_at(i, 0);
          best = key < before && key > best ? key : best;
        }
        before = next(best);
        if (threadIdx.x == 0 && before) chosen[round] = list_of(before);
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) s.count = 0;
#pragma unroll
    for (int j = 0; j < kKept; ++j) {
      const int i = threadIdx.x + j * kThreads;
      own[j] = 0;
      if (j * kThreads < p.k * p.k && i < p.k * p.k) {
        const int list = chosen[i % p.k];        // (first entries first, as above)
        if (list >= 0) own[j] = key_at(list, i / p.k);
      }
    }
  }
  uint64_t head = ended;
#pragma unroll
  for (uint64_t key : own) head = max(head, key);
  const float bound = bound_of_all(s, value_at(head), p.k);
#pragma unroll
  for (uint64_t key : own) take(key, bound);
  take(ended, bound);
  __syncthreads();
  auto put = [&](int rank, uint64_t key) {
    const int64_t at = b * p.k + rank;
    if (!key) {
      p.parents[at] = p.tokens[at] = -1;
      p.new_scores[at] = kClosed;
      p.new_ended[at] = 0;
      return;
    }
    const uint32_t index = index_of(key);
    const int w = static_cast<int>(index / p.words), word = static_cast<int>(index - w * p.words);
    p.parents[at] = static_cast<int32_t>(b * p.beams + w);
    p.tokens[at] = word;
    p.new_scores[at] = value_of(static_cast<uint32_t>(key >> 32));
    p.new_ended[at] = word == p.end || kept[w] > kClosed;
  };
  if (s.count <= kRoom) {
    rank_all(s, p.k, put);
    for (int i = s.count + threadIdx.x; i < p.k; i += kThreads) put(i, 0);
    return;
  }
  uint64_t before = ~uint64_t(0);
  for (int round = 0; round < p.k; ++round) {
    uint64_t best = ended < before ? ended : 0;
#pragma unroll
    for (uint64_t key : own) best = key < before && key > best ? key : best;
    before = next(best);
    if (threadIdx.x == 0) put(round, before);
  }
}

// Values of a segment follow from the words alone, so a row's sum does too.
int groups_of(int words) { return words <= 65536 ? 2 : 4; }
int segments_of(int words) { return (words + kThreads * 8 * groups_of(words) - 1) / (kThreads * 8 * groups_of(words)); }

// workgroups of a launch (a grid counts fewer than 2^32 threads)
constexpr uint32_t kMaxGrid = 1u << 23;

template <bool F32, int V>
void segments(const BeamArgs& a, const Segments& g, uint32_t items, hipStream_t stream) {
  for (uint32_t base = 0; base < items; base += kMaxGrid) {
    hipLaunchKernelGGL((segment_kernel<F32, V>), dim3(std::min(items - base, kMaxGrid)), dim3(kThreads), 0, stream, a, g, base);
    launched("choice of tokens, segments");
  }
}

}  // namespace

size_t decode_beam_workspace(int64_t sequences, int beams, int words, int k) {
  return static_cast<size_t>(sequences) * beams * segments_of(words) * (8 + static_cast<size_t>(k) * 8);
}

void decode_beam(const BeamArgs& a, hipStream_t stream) {
  Segments g;
  g.count = segments_of(a.words);
  g.size = kThreads * 8 * groups_of(a.words);
  const uint32_t items = static_cast<uint32_t>(a.sequences * a.beams * g.count);     // (below 2^24 rows of at most 128)
  g.lists = static_cast<uint64_t*>(a.workspace);
  g.state = reinterpret_cast<float2*>(g.lists + static_cast<int64_t>(items) * a.k);
  const bool four = groups_of(a.words) == 4;
  if (a.f32 && four)
    segments<true, 4>(a, g, items, stream);
  else if (a.f32)
    segments<true, 2>(a, g, items, stream);
  else if (four)
    segments<false, 4>(a, g, items, stream);
  else
    segments<false, 2>(a, g, items, stream);
  const dim3 grid(static_cast<unsigned>(a.sequences)), threads(kThreads);
  if (static_cast<int64_t>(a.beams) * g.count * a.k <= kFlat * kThreads)
    hipLaunchKernelGGL(choose_kernel<true>, grid, threads, 0, stream, a, g);
  else
    hipLaunchKernelGGL(choose_kernel<false>, grid, threads, 0, stream, a, g);
  launched("choice of tokens");
}

}  // namespace k
}  // namespace dycl
