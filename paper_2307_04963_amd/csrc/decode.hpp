// Host-side launchers of the decoding operators' kernels (include/dycl_decode.h).
// They do not check arguments: the C entry points validate every one before any
// launch, and each launcher is called with at least one row.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace dycl {
namespace k {

// A layer's paged cache and the tables that lead to it.
struct PagedArgs {
  uint16_t *keys, *values;       // [pages][heads][page][dim]
  int64_t pages;
  int page_shift;                // log2 of the tokens of a page
  int heads, dim;
  const int32_t* tables;         // [sequences][max_pages], pitch ldt
  int64_t ldt, sequences;
  int max_pages;
};

struct RotateArgs {
  const void *q, *k, *v;         // rows of q_heads, heads, heads heads; null: none (k and v together)
  void* q_out;
  int64_t ldq, ldk, ldv, ldo;
  int f32;
  const int32_t *positions, *sequence;   // sequence null: row r is sequence r
  const double* frequencies;     // [pairs], null where pairs is 0
  int pairs, interleaved;
  float magnitude, sign;         // sign -1: the adjoint
  int64_t n;
  int q_heads, dim;
  int padding;                   // 1: rows of negative position are padding
  PagedArgs cache;               // where k and v go
};
constexpr int kRotateMaxPairs = 2048, kRotateMaxWidth = 65536;
void decode_rotate(const RotateArgs& a, hipStream_t stream);

struct AttendArgs {
  const uint16_t* q;
  int64_t ldq, n;
  int q_heads;
  float scale;
  PagedArgs cache;
  const int32_t *lengths, *sequence;
  int64_t max_length, window;    // window 0: none
  const uint8_t* mask;
  int64_t ldm;
  uint16_t* out;
  int64_t ldo;
  void* workspace;
};
constexpr int kAttendMaxDim = 256;
size_t decode_attend_workspace(int64_t n, int q_heads, int heads, int dim, int64_t max_length, int64_t window);
// false: more parts than a launch counts (nothing is launched)
bool decode_attend(const AttendArgs& a, hipStream_t stream);

struct BeamArgs {
  const void* logits;
  int f32;
  int64_t ldl;
  const float* scores;
  const uint8_t* ended;
  int end;
  int64_t sequences;
  int beams, words, k;
  int32_t *parents, *tokens;
  float* new_scores;
  uint8_t* new_ended;
  void* workspace;
};
constexpr int kBeamMaxK = 64, kBeamMaxBeams = 64, kBeamMaxWords = 1 << 20;
size_t decode_beam_workspace(int64_t sequences, int beams, int words, int k);
void decode_beam(const BeamArgs& a, hipStream_t stream);

struct ForkArgs {
  PagedArgs cache;               // keys null: only tables and lengths; sequences: the rows
  const int32_t *lengths, *parents, *fresh;
  int64_t n;
  int32_t* new_tables;           // null: not written
  int64_t ldn;
  int32_t* new_lengths;
};
void decode_fork(const ForkArgs& a, hipStream_t stream);

}  // namespace k
}  // namespace dycl
