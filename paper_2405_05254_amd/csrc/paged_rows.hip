// Rows into pages and back: the rotation to their positions, the 4-bit coding, and the order inside a page.
//
// A row of a head is d / 8 threads with 8 dimensions each, and the threads of a workgroup are 2048 / d such rows. The angle of
// a pair at a position is a whole number of 2^-64 turns times the position, wrapped: exact wherever the position is. Cosine and
// sine of its upper 32 bits are formed once for a row and workgroup, because all heads share them.
#include "lanes.h"
#include "paged.h"

namespace yoco {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct LaneMin {
  static __device__ __forceinline__ float of(float a, float b) { return fminf(a, b); }
};

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x4 a = *(const f32x4*)(p + 4 * i);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 * i + j] = a[j];
  }
}
__device__ __forceinline__ void load8(const bf16_t* p, float (&x)[8]) {
  const u32x4 a = *(const u32x4*)p;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = __uint_as_float(a[j] << 16);
    x[2 * j + 1] = __uint_as_float(a[j] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) *(f32x4*)(p + 4 * i) = (f32x4){x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&x)[8]) {
  u32x4 a;
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] = (unsigned)f32_to_bf16(x[2 * j]) | ((unsigned)f32_to_bf16(x[2 * j + 1]) << 16);
  *(u32x4*)p = a;
}

// Cosine and sine of pair p at a position: the upper 32 bits of the phase are a signed part of a turn.
__device__ __forceinline__ float2 turn_of(uint64_t turns, int64_t pos) {
  const int32_t part = (int32_t)(((uint64_t)pos * turns) >> 32);
  const float a = (float)part * (float)(6.283185307179586 / 4294967296.0);
  float s, c;
  sincosf(a, &s, &c);
  return make_float2(c, s);
}

// Products and sums rounded apart, as the formulas print them.
__device__ __forceinline__ float turned(float x, float y, float c, float s) {        // x c + y s
#pragma clang fp contract(off)
  const float a = x * c, b = y * s;
  return a + b;
}

// Dimensions e0 .. e0 + 7 of a row, rotated; src points at the row's head.
template <typename S>
__device__ __forceinline__ void rotated(const S* src, int e0, int rot, int neighbours, const float2* cs, float (&x)[8]) {
  load8(src + e0, x);
  if (e0 >= rot) return;                                                            // rot is a multiple of 16
  if (neighbours) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 t = cs[e0 / 2 + j];
      const float a = x[2 * j], b = x[2 * j + 1];
      x[2 * j] = turned(a, b, t.x, -t.y);
      x[2 * j + 1] = turned(b, a, t.x, t.y);
    }
    return;
  }
  const int half = rot / 2, p0 = e0 < half ? e0 : e0 - half;
  float y[8];
  load8(src + (e0 < half ? e0 + half : p0), y);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 t = cs[p0 + j];
    x[j] = turned(x[j], y[j], t.x, e0 < half ? -t.y : t.y);
  }
}

// The codes of 8 of a group's 64 dimensions, its 8 threads side by side: 4 bits each, lowest dimension first. `param`: bf16 scale and minimum.
// A group that holds what is not finite, or whose range is not, stands for NaN.
__device__ __forceinline__ unsigned code8(const float (&x)[8], unsigned& param) {
#pragma clang fp contract(off)
  float lo = x[0], hi = x[0];
  unsigned bad = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    lo = fminf(lo, x[j]);
    hi = fmaxf(hi, x[j]);
    bad |= not_finite(x[j]);
  }
  float b = (float)bad;
  lo = over8<LaneMin>(lo);
  hi = over8<LaneMax>(hi);
  b = over8<LaneMax>(b);
  const float range = hi - lo;
  const unsigned base = f32_to_bf16(lo);
  unsigned scale = f32_to_bf16(range * (float)(1.0 / 15.0));
  if (scale < 0x0080u) scale = 0;                                                   // below the normal numbers: all of one value
  if (b > 0.f || not_finite(range) || (scale & 0x7f80u) == 0x7f80u || (base & 0x7f80u) == 0x7f80u) {
    param = 0x7fc00000u;                                                            // scale 0, minimum NaN
    return 0;
  }
  param = scale | (base << 16);
  const float s = __uint_as_float(scale << 16), base_f = __uint_as_float(base << 16), inv = scale ? 1.f / s : 0.f;
  unsigned codes = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float y = (x[j] - base_f) * inv;
    codes |= (unsigned)(int)fminf(fmaxf(rintf(y), 0.f), 15.f) << (4 * j);
  }
  return codes;
}

// One new row a workgroup, and 2048 / d of its heads: queries, then keys, then values.
template <typename S, int D, bool CODED>
__global__ void __launch_bounds__(256) append_kernel(AppendView a) {
  __shared__ float2 cs[64];
  constexpr int kThreads = D / 8, kHeads = 256 / kThreads;
  const int64_t row = blockIdx.x;
  const int b = (int)(row / a.T);
  const int64_t t = row - (int64_t)b * a.T, pos = a.pos[b] + t;
  if ((int)threadIdx.x < a.rot / 2) cs[threadIdx.x] = turn_of(a.turns[threadIdx.x], pos);
  __syncthreads();
  const int item = blockIdx.y * kHeads + threadIdx.x / kThreads, e0 = threadIdx.x % kThreads * 8;
  if (item >= a.Hq + 2 * a.c.Hkv) return;
  float x[8];
  if (item < a.Hq) {
    rotated((const S*)a.q + row * a.q_stride + (int64_t)item * D, e0, a.rot, a.neighbours, cs, x);
    store8((S*)a.q_out + (row * a.Hq + item) * D + e0, x);
    return;
  }
  if (a.rows && t >= a.rows[b]) return;
  if (pos < 0 || pos >= (int64_t)a.cols * kPageRows) return;
  const int page = a.table[(int64_t)b * a.cols + pos / kPageRows];
  if (page < 0 || page >= a.c.n_pages) return;
  const int g = item - a.Hq, r = (int)(pos % kPageRows);
  const bool is_v = g >= a.c.Hkv;
  const int head = is_v ? g - a.c.Hkv : g;
  if (is_v) load8((const S*)a.v + row * a.v_stride + (int64_t)head * D + e0, x);
  else rotated((const S*)a.k + row * a.k_stride + (int64_t)head * D, e0, a.rot, a.neighbours, cs, x);
  char* const at = (char*)(is_v ? a.c.v : a.c.k) + ((int64_t)page * a.c.Hkv + head) * page_bytes(D, CODED ? YOCO_INT4 : YOCO_BF16);
  if (!CODED) {
    if (!is_v) {
      store8((bf16_t*)at + k16_at(r, e0, D), x);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) ((bf16_t*)at)[v16_at(r, e0 + j)] = f32_to_bf16(x[j]);
    }
    return;
  }
  unsigned param;
  const unsigned codes = code8(x, param);
  if (!is_v) {
    *(unsigned*)(at + k4_byte(r, e0, D)) = codes;
  } else {
    const unsigned other = __shfl_xor(codes, 2);                                    // 16 dimensions further on, or back
    if (e0 / 16 % 2 == 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) at[v4_byte(r, e0 + j)] = (char)(((codes >> (4 * j)) & 15u) | (((other >> (4 * j)) & 15u) << 4));
    }
  }
  if (e0 % kCodeGroup == 0) *(unsigned*)(at + param4_byte(r, e0, D)) = param;
}

// The value that a code stands for.
__device__ __forceinline__ float decoded(unsigned code, unsigned param) {
  return fmaf((float)code, __uint_as_float(param << 16), __uint_as_float(param & 0xffff0000u));
}

// 8 dimensions of a row and head a thread; z: K or V.
template <typename S>
__global__ void __launch_bounds__(256) read_kernel(yoco_paged_cache c, const int32_t* __restrict__ table, int B, int cols, const int64_t* __restrict__ pos0, int64_t T,
                                                   S* __restrict__ k, S* __restrict__ v) {
  const int threads = c.d / 8;
  const int64_t unit = (int64_t)blockIdx.x * (256 / threads) + threadIdx.x / threads;            // row and head
  if (unit >= (int64_t)B * T * c.Hkv) return;
  const int64_t row = unit / c.Hkv;
  const int head = (int)(unit - row * c.Hkv), b = (int)(row / T), e0 = threadIdx.x % threads * 8;
  const int64_t pos = pos0[b] + (row - (int64_t)b * T);
  const bool is_v = blockIdx.y;
  float x[8] = {};
  const int page = pos >= 0 && pos < (int64_t)cols * kPageRows ? table[(int64_t)b * cols + pos / kPageRows] : -1;
  if (page >= 0 && page < c.n_pages) {
    const int r = (int)(pos % kPageRows);
    const char* const at = (const char*)(is_v ? c.v : c.k) + ((int64_t)page * c.Hkv + head) * page_bytes(c.d, c.dtype);
    if (c.dtype == YOCO_INT4) {
      const unsigned param = *(const unsigned*)(at + param4_byte(r, e0, c.d));
      if (!is_v) {
        const unsigned codes = *(const unsigned*)(at + k4_byte(r, e0, c.d));
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = decoded((codes >> (4 * j)) & 15u, param);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = decoded(((unsigned)(unsigned char)at[v4_byte(r, e0 + j)] >> (e0 / 16 % 2 * 4)) & 15u, param);
      }
    } else if (!is_v) {
      load8((const bf16_t*)at + k16_at(r, e0, c.d), x);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = bf16_to_f32(((const bf16_t*)at)[v16_at(r, e0 + j)]);
    }
  }
  store8((is_v ? v : k) + unit * c.d + e0, x);
}

}  // namespace

hipError_t launch_paged_append(const AppendView& a, int src_dtype, hipStream_t s) {
  const int heads = 2048 / a.c.d;
  const dim3 grid((unsigned)(a.B * a.T), (unsigned)((a.Hq + 2 * a.c.Hkv + heads - 1) / heads)), block(256);
  auto go = [&](auto* kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
  const bool coded = a.c.dtype == YOCO_INT4;
  if (src_dtype == YOCO_F32) {
    if (a.c.d == 128) coded ? go(&append_kernel<float, 128, true>) : go(&append_kernel<float, 128, false>);
    else coded ? go(&append_kernel<float, 64, true>) : go(&append_kernel<float, 64, false>);
  } else {
    if (a.c.d == 128) coded ? go(&append_kernel<bf16_t, 128, true>) : go(&append_kernel<bf16_t, 128, false>);
    else coded ? go(&append_kernel<bf16_t, 64, true>) : go(&append_kernel<bf16_t, 64, false>);
  }
  return hipGetLastError();
}

hipError_t launch_paged_read(const yoco_paged_cache& c, const int32_t* table, int B, int cols, const int64_t* pos, int64_t T, void* k, void* v, int dst_dtype,
                             hipStream_t s) {
  const int64_t units = (int64_t)B * T * c.Hkv, each = 2048 / c.d;
  const dim3 grid((unsigned)((units + each - 1) / each), 2), block(256);
  if (dst_dtype == YOCO_F32) hipLaunchKernelGGL(read_kernel<float>, grid, block, 0, s, c, table, B, cols, pos, T, (float*)k, (float*)v);
  else hipLaunchKernelGGL(read_kernel<bf16_t>, grid, block, 0, s, c, table, B, cols, pos, T, (bf16_t*)k, (bf16_t*)v);
  return hipGetLastError();
}

}  // namespace yoco
