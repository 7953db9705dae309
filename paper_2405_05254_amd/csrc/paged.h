// The cache in pages of 64 rows: where a value lies inside a page, and the launchers of what writes and reads it. The order
// is the matrix cores': whatever a wavefront loads with 16 bytes a lane, 1 KiB in a row, is a ready operand of a
// 16x16x32 product, 32 dimensions of 16 rows in the K plane, 32 rows of 16 dimensions in the V plane.
#pragma once
#include "yoco_common.h"

namespace yoco {

constexpr int kPageRows = 64;
constexpr int kCodeGroup = 64;           // dimensions that share a 4-bit scale and minimum

__host__ __device__ inline size_t page_bytes(int d, int dtype) { return dtype == YOCO_INT4 ? (size_t)36 * d : (size_t)128 * d; }

// bf16: element of row r, dimension e
__host__ __device__ inline int k16_at(int r, int e, int d) { return ((r / 16 * (d / 32) + e / 32) * 64 + e / 8 % 4 * 16 + r % 16) * 8 + e % 8; }
__host__ __device__ inline int v16_at(int r, int e) { return ((e / 16 * 2 + r / 32) * 64 + r % 16 / 4 * 16 + e % 16) * 8 + r / 16 % 2 * 4 + r % 4; }
// 4 bits: the byte; dimension e is its nibble e % 2 (K), e / 16 % 2 (V). Bytes hold values of one row only.
__host__ __device__ inline int k4_byte(int r, int e, int d) {
  const int i = r / 16 * (d / 32) + e / 32;
  return (i / 4 * 64 + e / 8 % 4 * 16 + r % 16) * 16 + i % 4 * 4 + e % 8 / 2;
}
__host__ __device__ inline int v4_byte(int r, int e) { return (e / 32 * 64 + r % 16 / 4 * 16 + e % 16) * 16 + r / 16 * 4 + r % 4; }
// ... and the scale of its group; the minimum follows (two bf16)
__host__ __device__ inline int param4_byte(int r, int e, int d) { return 32 * d + (r * (d / kCodeGroup) + e / kCodeGroup) * 4; }

// A number's bits, hidden from the optimiser: built to assume that no float is a NaN, it would drop a test for one.
__device__ __forceinline__ unsigned opaque_bits(float x) {
  unsigned u = __float_as_uint(x);
  asm("" : "+v"(u));
  return u;
}
__device__ __forceinline__ bool not_finite(float x) { return (opaque_bits(x) & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool is_nan(float x) { return (opaque_bits(x) & 0x7fffffffu) > 0x7f800000u; }

// New rows, behind the checks: row t of sequence b is row b * T + t of k, v and q (strides in elements).
struct AppendView {
  yoco_paged_cache c;
  const int32_t* table;
  int B, cols;
  const int64_t* pos;
  const int64_t* rows;                   // or null: T of each sequence
  int64_t T;
  const void *k, *v, *q;                 // q: or null
  void* q_out;
  int64_t k_stride, v_stride, q_stride;
  int Hq;                                // 0 without q
  const uint64_t* turns;
  int rot, neighbours;                   // rot: 0 without a rotation
};
hipError_t launch_paged_append(const AppendView& a, int src_dtype, hipStream_t s);
hipError_t launch_paged_read(const yoco_paged_cache& c, const int32_t* table, int B, int cols, const int64_t* pos, int64_t T, void* k, void* v, int dst_dtype,
                             hipStream_t s);

struct PagedAttnView {
  yoco_paged_cache c;
  const int32_t* table;
  int B, cols;
  const void* q;
  void* o;
  const int64_t* lens;
  int T, Hq;
  float scale;
};
size_t paged_attn_workspace(const PagedAttnView& a);
hipError_t launch_paged_attn(const PagedAttnView& a, void* workspace, unsigned long long tag, hipStream_t s);

// Beam search (beam.hip).
struct SelectView {
  const void* logits;
  int64_t stride;
  const float* scores;
  const uint8_t* done;                   // or null
  int eos, B, W, V;
  int32_t *parent, *token;
  float* scores_out;
  uint8_t* done_out;
};
size_t beam_select_workspace(int B, int W, int V);
hipError_t launch_beam_select(const SelectView& a, int dtype, void* workspace, hipStream_t s);
hipError_t launch_beam_reorder_pages(const yoco_paged_cache& c, int32_t* table, const int32_t* home, int B, int W, int cols, const int32_t* parent, const int64_t* lens,
                                     hipStream_t s);
constexpr int kReorderMost = 32;         // buffers of one launch
struct ReorderRows {
  void* mem[kReorderMost];
  int64_t pieces[kReorderMost];          // 16-byte pieces of a row
};
hipError_t launch_beam_reorder_rows(const ReorderRows& r, int n, int B, int W, const int32_t* parent, hipStream_t s);

}  // namespace yoco
