// C entry points of the decoding operators (include/dycl_decode.h): argument
// checks and launches.  Nothing thrown crosses them.
#include "../../include/dycl_decode.h"

#include "abi_checks.hpp"
#include "decode.hpp"

namespace {

using dycl::guarded;
using namespace dycl::checks;
using namespace dycl::k;

// log2 of a page's tokens; -1 where it is not allowed
int shift_of(int page) {
  for (int s = 3; s <= 10; ++s)
    if (page == 1 << s) return s;
  return -1;
}

void need_rotation(const char* op, const double* frequencies, int pairs, int layout, float magnitude, int dim) {
  need(pairs >= 0 && pairs <= dim / 2 && pairs <= kRotateMaxPairs, op, "pairs outside [0, min(dim / 2, 2048)]");
  need(pairs == 0 || frequencies, op, "null frequencies");
  need(at(frequencies, 8), op, "frequencies not aligned to 8 bytes");
  need(layout == DYCL_ROTATE_HALF || layout == DYCL_ROTATE_INTERLEAVED, op, "unknown layout of the pairs");
  need(magnitude - magnitude == 0.f, op, "magnitude not finite");
}

void need_sizes(const char* op, int heads, int page, int dim, int max_pages, int64_t pages, int64_t sequences) {
  need(heads >= 1 && heads <= kRotateMaxWidth, op, "heads outside [1, 65536]");
  need(dim >= 8 && dim <= kAttendMaxDim && dim % 8 == 0, op, "dim not a multiple of 8 in [8, 256]");
  need(shift_of(page) >= 0, op, "page not a power of two in [8, 1024]");
  need(max_pages >= 1 && int64_t(max_pages) * page < kMaxRows, op, "max_pages * page outside [1, 2^31)");
  need(pages >= 1 && pages < kMaxRows, op, "pages outside [1, 2^31)");
  need(sequences >= 0 && sequences < kMaxRows, op, "sequences outside [0, 2^31)");
}

PagedArgs paged(const uint16_t* keys, const uint16_t* values, int64_t pages, int heads, int page, int dim,
                const int32_t* tables, int64_t ldt, int64_t sequences, int max_pages) {
  PagedArgs c;
  c.keys = const_cast<uint16_t*>(keys);
  c.values = const_cast<uint16_t*>(values);
  c.pages = pages;
  c.page_shift = shift_of(page);
  c.heads = heads;
  c.dim = dim;
  c.tables = tables;
  c.ldt = ldt;
  c.sequences = sequences;
  c.max_pages = max_pages;
  return c;
}

// a window that reaches as far as any row is none
int64_t window_of(int64_t window, int64_t max_length) { return window >= max_length ? 0 : window; }

const char* const kUnaligned = "a pointer not aligned to its element (keys, values, workspace: 16 bytes)";

}  // namespace

extern "C" {

int dycl_op_rotate(const void* x, int type, int64_t ldx, const int32_t* positions, const double* frequencies, int pairs,
                   int layout, float magnitude, int adjoint, int64_t n, int heads, int dim, void* y, int64_t ldy,
                   void* hip_stream) {
  return guarded([&] {
    const char* op = "dycl_op_rotate";
    need(n >= 0 && n < kMaxRows, op, "n outside [0, 2^31)");
    need(heads >= 1 && dim >= 2 && int64_t(heads) * dim <= kRotateMaxWidth, op, "heads below 1, dim below 2 or heads * dim above 65536");
    need(type_ok(type), op, "unknown element type");
    need(pairs >= 1, op, "no pairs");
    need_rotation(op, frequencies, pairs, layout, magnitude, dim);
    if (n == 0) return static_cast<int>(DYCL_OK);
    need(x && y && positions, op, "null x, y or positions");
    need(pitch_ok(ldx, int64_t(heads) * dim) && pitch_ok(ldy, int64_t(heads) * dim), op, "a row pitch below the row");
    need(at(x, size_of(type)) && at(y, size_of(type)) && at(positions, 4), op, kUnaligned);
    need(x != y || ldx == ldy, op, "y is x with another pitch");
    RotateArgs a{};
    a.q = x;
    a.ldq = ldx;
    a.q_out = y;
    a.ldo = ldy;
    a.f32 = type == DYCL_F32;
    a.positions = positions;
    a.frequencies = frequencies;
    a.pairs = pairs;
    a.interleaved = layout == DYCL_ROTATE_INTERLEAVED;
    a.magnitude = magnitude;
    a.sign = adjoint ? -1.f : 1.f;
    a.n = n;
    a.q_heads = heads;
    a.dim = dim;
    decode_rotate(a, static_cast<hipStream_t>(hip_stream));
    return static_cast<int>(DYCL_OK);
  });
}

int dycl_op_append(const void* k, int64_t ldk, const void* v, int64_t ldv, const void* q, int64_t ldq, void* q_out,
                   int64_t ldo, int type, const int32_t* positions, const int32_t* sequence, const double* frequencies,
                   int pairs, int layout, float magnitude, int64_t n, int q_heads, int heads, int dim,
                   const int32_t* tables, int64_t ldt, int64_t sequences, int max_pages, uint16_t* keys,
                   uint16_t* values, int64_t pages, int page, void* hip_stream) {
  return guarded([&] {
    const char* op = "dycl_op_append";
    need(n >= 0 && n < kMaxRows, op, "n outside [0, 2^31)");
    need_sizes(op, heads, page, dim, max_pages, pages, sequences);
    need(int64_t(heads) * dim <= kRotateMaxWidth, op, "heads * dim above 65536");
    need(type_ok(type), op, "unknown element type");
    need_rotation(op, frequencies, pairs, layout, magnitude, dim);
    need((q == nullptr) == (q_out == nullptr), op, "q and q_out are given together");
    need(!q || (q_heads >= 1 && int64_t(q_heads) * dim <= kRotateMaxWidth), op, "q_heads below 1 or q_heads * dim above 65536");
    need(sequence || n == sequences, op, "without `sequence` there are as many rows as sequences");
    if (n == 0) return static_cast<int>(DYCL_OK);
    need(k && v && positions && (tables || sequences == 0) && keys && values, op, "null k, v, positions, tables, keys or values");
    const int64_t width = int64_t(heads) * dim, q_width = int64_t(q_heads) * dim;
    need(pitch_ok(ldk, width) && pitch_ok(ldv, width) && (!q || (pitch_ok(ldq, q_width) && pitch_ok(ldo, q_width))) &&
             pitch_ok(ldt, max_pages),
         op, "a row pitch below the row");
    need(at(k, size_of(type)) && at(v, size_of(type)) && at(q, size_of(type)) && at(q_out, size_of(type)) &&
             at(positions, 4) && at(sequence, 4) && at(tables, 4) && at(keys, 16) && at(values, 16),
         op, kUnaligned);
    need(keys != values, op, "keys and values are the same");
    need(!q || q != q_out || ldq == ldo, op, "q_out is q with another pitch");
    RotateArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_out = q_out;
    a.ldq = ldq;
    a.ldk = ldk;
    a.ldv = ldv;
    a.ldo = ldo;
    a.f32 = type == DYCL_F32;
    a.positions = positions;
    a.sequence = sequence;
    a.frequencies = frequencies;
    a.pairs = pairs;
    a.interleaved = layout == DYCL_ROTATE_INTERLEAVED;
    a.magnitude = magnitude;
    a.sign = 1.f;
    a.n = n;
    a.q_heads = q_heads;
    a.dim = dim;
    a.padding = 1;
    a.cache = paged(keys, values, pages, heads, page, dim, tables, ldt, sequences, max_pages);
    decode_rotate(a, static_cast<hipStream_t>(hip_stream));
    return static_cast<int>(DYCL_OK);
  });
}

size_t dycl_op_attend_workspace(int64_t n, int q_heads, int heads, int dim, int64_t max_length, int64_t window) {
  if (n < 1 || n >= kMaxRows || heads < 1 || q_heads < heads || q_heads % heads || n * q_heads >= kMaxRows || dim < 8 ||
      dim > kAttendMaxDim || max_length < 0 || max_length >= kMaxRows - 4096 || window < 0)
    return 0;
  return decode_attend_workspace(n, q_heads, heads, dim, max_length, window_of(window, max_length));
}

int dycl_op_attend(const uint16_t* q, int64_t ldq, int64_t n, int q_heads, int heads, int dim, float scale,
                   const uint16_t* keys, const uint16_t* values, int64_t pages, int page, const int32_t* tables,
                   int64_t ldt, int64_t sequences, int max_pages, const int32_t* lengths, const int32_t* sequence,
                   int64_t max_length, int64_t window, const uint8_t* mask, int64_t ldm, uint16_t* out, int64_t ldo,
                   void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&] {
    const char* op = "dycl_op_attend";
    need(n >= 0 && n < kMaxRows, op, "n outside [0, 2^31)");
    need_sizes(op, heads, page, dim, max_pages, pages, sequences);
    need(q_heads >= heads && q_heads % heads == 0, op, "q_heads not a multiple of heads");
    need(n * q_heads < kMaxRows, op, "n * q_heads outside [0, 2^31)");
    need(max_length >= 0 && max_length <= int64_t(max_pages) * page && max_length < kMaxRows - 4096, op,
         "max_length outside [0, max_pages * page] or above 2^31 - 4097");
    need(window >= 0, op, "negative window");
    need(scale > -1e38f && scale < 1e38f, op, "scale not finite, or above 1e38");
    need(sequence || n == sequences, op, "without `sequence` there are as many rows as sequences");
    if (n == 0) return static_cast<int>(DYCL_OK);
    need(q && keys && values && (tables || sequences == 0) && lengths && out, op, "null q, keys, values, tables, lengths or out");
    const int64_t width = int64_t(q_heads) * dim;
    need(pitch_ok(ldq, width) && pitch_ok(ldo, width) && pitch_ok(ldt, max_pages) && (!mask || pitch_ok(ldm, max_length)), op,
         "a row pitch below the row");
    need(at(q, 2) && at(out, 2) && at(keys, 16) && at(values, 16) && at(tables, 4) && at(lengths, 4) && at(sequence, 4) &&
             at(workspace, 16),
         op, kUnaligned);
    need(out != q, op, "out is q");
    window = window_of(window, max_length);
    const size_t bytes = decode_attend_workspace(n, q_heads, heads, dim, max_length, window);
    need(bytes == 0 || (workspace && workspace_bytes >= bytes), op, "workspace too small");
    AttendArgs a{};
    a.q = q;
    a.ldq = ldq;
    a.n = n;
    a.q_heads = q_heads;
    a.scale = scale;
    a.cache = paged(keys, values, pages, heads, page, dim, tables, ldt, sequences, max_pages);
    a.lengths = lengths;
    a.sequence = sequence;
    a.max_length = max_length;
    a.window = window;
    a.mask = mask;
    a.ldm = ldm;
    a.out = out;
    a.ldo = ldo;
    a.workspace = workspace;
    need(decode_attend(a, static_cast<hipStream_t>(hip_stream)), op, "more parts than a launch counts");
    return static_cast<int>(DYCL_OK);
  });
}

size_t dycl_op_beam_workspace(int64_t sequences, int beams, int words, int k) {
  if (sequences < 1 || beams < 1 || beams > kBeamMaxBeams || words < 1 || words > kBeamMaxWords || k < 1 || k > kBeamMaxK ||
      sequences >= kMaxRows || sequences * beams >= int64_t(1) << 24)
    return 0;
  return decode_beam_workspace(sequences, beams, words, k);
}

int dycl_op_beam(const void* logits, int type, int64_t ldl, const float* scores, const uint8_t* ended, int end,
                 int64_t sequences, int beams, int words, int k, int32_t* parents, int32_t* tokens, float* new_scores,
                 uint8_t* new_ended, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&] {
    const char* op = "dycl_op_beam";
    need(beams >= 1 && beams <= kBeamMaxBeams, op, "beams outside [1, 64]");
    need(k >= 1 && k <= kBeamMaxK, op, "k outside [1, 64]");
    need(words >= 1 && words <= kBeamMaxWords, op, "words outside [1, 2^20]");
    need(sequences >= 0 && sequences < kMaxRows && sequences * beams < int64_t(1) << 24, op, "sequences * beams outside [0, 2^24)");
    need(type_ok(type), op, "unknown element type");
    need(!ended || (end >= 0 && end < words), op, "ended beams without an end token in [0, words)");
    if (sequences == 0) return static_cast<int>(DYCL_OK);
    need(logits && scores && parents && tokens && new_scores && new_ended, op, "a null tensor");
    need(pitch_ok(ldl, words), op, "a row pitch below words");
    need(at(logits, size_of(type)) && at(scores, 4) && at(parents, 4) && at(tokens, 4) && at(new_scores, 4) && at(workspace, 16), op,
         kUnaligned);
    need(new_scores != scores && (!ended || new_ended != ended), op, "new scores or flags are the old ones");
    need(workspace && workspace_bytes >= decode_beam_workspace(sequences, beams, words, k), op, "workspace too small");
    BeamArgs a{};
    a.logits = logits;
    a.f32 = type == DYCL_F32;
    a.ldl = ldl;
    a.scores = scores;
    a.ended = ended;
    a.end = end;
    a.sequences = sequences;
    a.beams = beams;
    a.words = words;
    a.k = k;
    a.parents = parents;
    a.tokens = tokens;
    a.new_scores = new_scores;
    a.new_ended = new_ended;
    a.workspace = workspace;
    decode_beam(a, static_cast<hipStream_t>(hip_stream));
    return static_cast<int>(DYCL_OK);
  });
}

int dycl_op_fork(const int32_t* tables, int64_t ldt, const int32_t* lengths, int64_t rows, int max_pages,
                 const int32_t* parents, const int32_t* fresh, int64_t n, int32_t* new_tables, int64_t ldn,
                 int32_t* new_lengths, uint16_t* keys, uint16_t* values, int64_t pages, int heads, int page, int dim,
                 void* hip_stream) {
  return guarded([&] {
    const char* op = "dycl_op_fork";
    need(n >= 0 && n < kMaxRows, op, "n outside [0, 2^31)");
    need((keys == nullptr) == (values == nullptr), op, "keys and values are given together");
    need((new_tables == nullptr) == (new_lengths == nullptr), op, "new tables and lengths are given together");
    need_sizes(op, keys ? heads : 1, page, keys ? dim : 8, max_pages, keys ? pages : 1, rows);
    need(at(keys, 16) && at(values, 16), op, kUnaligned);
    need(!keys || keys != values, op, "keys are the values");
    if (n == 0) return static_cast<int>(DYCL_OK);
    need(keys || new_tables, op, "neither a cache nor new tables");
    need(((tables && lengths) || rows == 0) && parents && fresh, op, "null tables, lengths, parents or fresh");
    need(pitch_ok(ldt, max_pages) && (!new_tables || pitch_ok(ldn, max_pages)), op, "a row pitch below the row");
    need(at(tables, 4) && at(lengths, 4) && at(parents, 4) && at(fresh, 4) && at(new_tables, 4) && at(new_lengths, 4), op,
         kUnaligned);
    need(new_tables != tables && new_lengths != lengths, op, "new tables or lengths are the old ones");
    ForkArgs a{};
    a.cache = paged(keys, values, pages, keys ? heads : 1, page, keys ? dim : 8, tables, ldt, rows, max_pages);
    a.lengths = lengths;
    a.parents = parents;
    a.fresh = fresh;
    a.n = n;
    a.new_tables = new_tables;
    a.ldn = ldn;
    a.new_lengths = new_lengths;
    decode_fork(a, static_cast<hipStream_t>(hip_stream));
    return static_cast<int>(DYCL_OK);
  });
}

}  // extern "C"
