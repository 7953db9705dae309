// Attention over a cache in pages: o = softmax(scale q.k) v for the last T rows of every sequence, causal, d 64 or 128.
#include "lanes.h"
#include "paged.h"

namespace yoco {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// One query row and head a workgroup; its wavefronts take turns at the pages, a lane a row for the scores and d / 64 dimensions for the sums.
template <int D, bool CODED>
__global__ void __launch_bounds__(256) attn_kernel(PagedAttnView a) {
  constexpr int kOwn = D / 64;
  __shared__ float qs[D], ps[4][64], os[4][D], ms[4], ls[4];
  const int h = blockIdx.x % a.Hq, i = blockIdx.x / a.Hq, b = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t row = ((int64_t)b * a.T + i) * a.Hq + h, most = (int64_t)a.cols * kPageRows;
  const int64_t len = a.lens[b] < 0 ? 0 : a.lens[b] > most ? most : a.lens[b], seen = len - a.T + 1 + i;
  if ((int)threadIdx.x < D) qs[threadIdx.x] = bf16_to_f32(((const bf16_t*)a.q)[row * D + threadIdx.x]) * (a.scale * kLog2e);
  __syncthreads();
  const int head = h / (a.Hq / a.c.Hkv);
  float m = -INFINITY, l = 0.f, o[kOwn] = {};
  for (int64_t p = wave; p * kPageRows < seen; p += 4) {
    const int page = a.table[(int64_t)b * a.cols + p];
    if (page < 0 || page >= a.c.n_pages) continue;
    const int64_t at = ((int64_t)page * a.c.Hkv + head) * page_bytes(D, CODED ? YOCO_INT4 : YOCO_BF16);
    const char *kp = (const char*)a.c.k + at, *vp = (const char*)a.c.v + at;
    float s = 0.f;
    for (int e = 0; e < D; ++e) {
      float x;
      if (CODED) {
        const unsigned param = *(const unsigned*)(kp + param4_byte(lane, e, D));
        const unsigned code = ((unsigned)(unsigned char)kp[k4_byte(lane, e, D)] >> (e % 2 * 4)) & 15u;
        x = fmaf((float)code, __uint_as_float(param << 16), __uint_as_float(param & 0xffff0000u));
      } else {
        x = bf16_to_f32(((const bf16_t*)kp)[k16_at(lane, e, D)]);
      }
      s = fmaf(x, qs[e], s);
    }
    if (p * kPageRows + lane >= seen) s = -INFINITY;
    const float m_new = fmaxf(m, over64<LaneMax>(s)), base = m_new == -INFINITY ? 0.f : m_new;
    const float w = __builtin_amdgcn_exp2f(s - base), f = __builtin_amdgcn_exp2f(m - base);
    m = m_new;
    l = l * f + over64<LaneSum>(w);
    ps[wave][lane] = w;
    const int rows = seen - p * kPageRows < kPageRows ? (int)(seen - p * kPageRows) : kPageRows;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int e = lane + 64 * j;
      float sum = o[j] * f;
      for (int r = 0; r < rows; ++r) {
        float x;
        if (CODED) {
          const unsigned param = *(const unsigned*)(vp + param4_byte(r, e, D));
          const unsigned code = ((unsigned)(unsigned char)vp[v4_byte(r, e)] >> (e / 16 % 2 * 4)) & 15u;
          x = fmaf((float)code, __uint_as_float(param << 16), __uint_as_float(param & 0xffff0000u));
        } else {
          x = bf16_to_f32(((const bf16_t*)vp)[v16_at(r, e)]);
        }
        sum = fmaf(ps[wave][r], x, sum);
      }
      o[j] = sum;
    }
  }
#pragma unroll
  for (int j = 0; j < kOwn; ++j) os[wave][lane + 64 * j] = o[j];
  if (lane == 0) {
    ms[wave] = m;
    ls[wave] = l;
  }
  __syncthreads();
  if ((int)threadIdx.x < D) {
    const float M = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3])), base = M == -INFINITY ? 0.f : M;
    float sum = 0.f, total = 0.f;
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(ms[w] - base);
      total = fmaf(f, ls[w], total);
      sum = fmaf(f, os[w][threadIdx.x], sum);
    }
    ((bf16_t*)a.o)[row * D + threadIdx.x] = f32_to_bf16(opaque_bits(total) ? sum / total : 0.f);
  }
}

}  // namespace

size_t paged_attn_workspace(const PagedAttnView&) { return 0; }

hipError_t launch_paged_attn(const PagedAttnView& a, void*, unsigned long long, hipStream_t s) {
  const dim3 grid((unsigned)(a.T * a.Hq), (unsigned)a.B), block(256);
  auto go = [&](auto* kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
  if (a.c.d == 128) a.c.dtype == YOCO_INT4 ? go(&attn_kernel<128, true>) : go(&attn_kernel<128, false>);
  else a.c.dtype == YOCO_INT4 ? go(&attn_kernel<64, true>) : go(&attn_kernel<64, false>);
  return hipGetLastError();
}

}  // namespace yoco
