// Parameters and launcher of the rotary row kernels (implemented in rope.hip).
// Only host/rope.cpp calls it, after validating everything.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fck {

// One tensor's rows: `rows` tokens of `heads` heads of d values.
struct RopeRows {
  const void* in;         // row r at in + src * in_stride, src = r or gpos[r]
  void* out;              // row r at out + r * out_stride (strides in elements)
  int64_t in_stride, out_stride;
  const int32_t* gather;  // packed rows (gpos), or null: row r itself
  const int32_t* gpos;    // the tokens' positions in the packed sequence
  const int32_t* first;   // per 64 rows: the segment of the first of them
  int32_t end;            // seg[4 * i + end]: rows up to segment i's last (0 local, 1 received)
  int32_t rows, heads;
  int32_t rotate;         // 0: copied (or rounded) only
  int32_t per_block;      // rows per workgroup, a power of two up to kRopeRows
  int32_t blocks;
  int32_t step_t, step_q;  // 256 units further: rows, and units of a row
};

constexpr int kRopeRows = 32;
constexpr int kRopeSets = 5;
// units of two 16-byte pieces of a row
constexpr int rope_units(int d, bool in_f32) { return d / (in_f32 ? 8 : 16); }

struct RopeParams {
  RopeRows set[kRopeSets];
  int32_t n_sets;
  int32_t pairs;            // rotated pairs of a head
  int32_t packed_pos;       // positions counted in the packed sequence, not the document
  float amplitude;
  float sign;               // 1: rotated forwards, -1: back
  const int32_t* seg;       // 4 int32 per segment: local end, received end, document start, 0
  uint64_t turn[64];        // per pair: turns per position, 64-bit fixed point
};

enum { kRopeHalves = 0, kRopeNeighbours = 1, kRopeHalvesOdd = 2 };

hipError_t launch_rope(const RopeParams& p, int d, int layout, bool in_f32, bool out_f32,
                       hipStream_t s);

}  // namespace fck
