// Layouts of the microscaled 4-bit matrices, shared by their quantizer, importer, exporters and products.
//
// Linear form.  Rows in tiles of 128, K in blocks of 256; one record per (row tile, K block), K blocks of a tile contiguous:
//   | codes 16384 | scale atoms |      17408 B (MXFP4, two atoms) or 18432 B (NVFP4, four)
//   codes: row r, byte b of its 128 at (r/8)*1024 + (b/16)*128 + (r%8)*16 + b%16: un-swizzled K-major core matrices, those of 8 rows adjacent
//          along K, so that any run of 8-row groups is contiguous and serves as A or as B operand of tcgen05.mma
//   scale atom a: what one tcgen05.cp moves, four scales of each of the tile's rows: row r, scale s at (r%32)*16 + (r/32)*4 + s.
//          MXFP4: 128 K an atom, NVFP4: 64 K
// K is padded to 256 with codes and scales of zero; rows behind R are not written (they only reach outputs that are not stored).
//
// Experts' form (MXFP4).  Every expert's rows in tiles of 128, K in steps of 128; one record per (expert, row tile, step), steps of a
// tile contiguous:  | codes 8192 | scale atom |      8704 B
//   codes: row r, byte b of its 64 at (r/8)*512 + (b/16)*128 + (r%8)*16 + b%16; the atom has four scales of 32 K
// Rows are padded to 128 and K to 128 with zeros: a padded row of a gate is a zero of what follows.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../../include/sdq_mx4.h"

namespace sdq {
namespace mx4 {

constexpr int ROWS = 128;                  // rows of a tile
constexpr int KREC = 256;                  // K of a record (linear form)
constexpr int KSTEP = 128;                 // K of a step (experts' form)
constexpr uint32_t ATOM = 512;
constexpr uint32_t CODES = 16384;          // code bytes of a record
constexpr uint32_t ECODES = 8192, ERECORD = ECODES + ATOM;   // of an expert's tile and step

__host__ __device__ constexpr uint32_t atoms(int fmt) { return fmt == SDQ_FMT_NVFP4 ? 4u : 2u; }
__host__ __device__ constexpr uint32_t record(int fmt) { return CODES + atoms(fmt) * ATOM; }
__host__ __device__ inline uint32_t atom_off(uint32_t row, uint32_t s) { return (row & 31) * 16 + (row >> 5) * 4 + s; }

struct Dims {
  int64_t tiles, kblocks;                  // row tiles (of one expert), records or steps along K
  size_t factors, total;                   // offset of the row factors
};
inline Dims dims(int64_t E, int64_t R, int64_t K, int fmt) {
  Dims d;
  auto al = [](size_t x) { return (x + 255) & ~(size_t)255; };
  d.tiles = (R + ROWS - 1) / ROWS;
  if (E == 0) {
    d.kblocks = (K + KREC - 1) / KREC;
    d.factors = al((size_t)d.tiles * d.kblocks * record(fmt));
    d.total = d.factors + (fmt == SDQ_FMT_NVFP4 ? al((size_t)d.tiles * ROWS * 4) : 0);
  } else {
    d.kblocks = (K + KSTEP - 1) / KSTEP;
    d.factors = d.total = al((size_t)E * d.tiles * d.kblocks * ERECORD);
  }
  return d;
}
// sizes whose buffers stay far from what 63 bits and the grids can count
inline bool size_ok(int64_t E, int64_t R, int64_t K) {
  return E >= 0 && E <= (1 << 16) && R >= 1 && K >= 1 && R <= ((int64_t)1 << 36) && K <= ((int64_t)1 << 30) &&
         (E ? E : 1) * ((R + 127) / 128) <= ((int64_t)1 << 40) / ((K + 127) / 128);
}
inline size_t dtype_bytes(int32_t dtype) { return dtype == SDQ_FP32 ? 4 : 2; }
inline bool dtype_ok(int32_t dtype) { return dtype >= SDQ_BF16 && dtype <= SDQ_FP32; }
inline bool fmt_ok(int32_t fmt) { return fmt == SDQ_FMT_MXFP4 || fmt == SDQ_FMT_NVFP4; }
// whether a descriptor is one that these calls have filled in
inline bool desc_ok(const sdq_mx4_t* q) {
  if (!q || !q->dev || !fmt_ok(q->fmt) || !size_ok(q->E, q->R, q->K) || (q->E && q->fmt != SDQ_FMT_MXFP4)) return false;
  const Dims d = dims(q->E, q->R, q->K, q->fmt);
  return q->bytes >= d.total && q->factors == d.factors && ((uintptr_t)q->dev & 255) == 0;
}

}  // namespace mx4
}  // namespace sdq
