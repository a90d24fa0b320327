// Rotary positions of a packed batch's queries and keys, and the write of keys and values into
// the paged bf16 cache (spec_rope_kv).
//
//   a = 2 pi * frac(position * turns[i] / 2^64)
//   y1 = f (x1 cos a - x2 sin a),  y2 = f (x2 cos a + x1 sin a)
// for the pairs (x1, x2) = (x[i], x[i + rot/2]) or (x[2i], x[2i + 1]). A turn is 2^64, so the
// product of position and frequency loses whole turns by overflowing, without a rounding: the
// angle is as good at position 2^31 as at 0. Sines are in fp32, results rounded once to bf16.
#include <cuda_bf16.h>

#include "chunk.cuh"
#include "kv_fp8.cuh"

namespace specv {
namespace {

constexpr int kRopeThreads = 256;

struct RopeParams {
  spec_rope_args_t a;
  int rows_per_block, heads;  // heads: Hq + 2 Hkv
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
  float factor;
};

__device__ __forceinline__ float2 unpack2(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Rotates the pairs (x0[e], x1[e]) of two vectors of 8 elements by 8 angles.
__device__ __forceinline__ void rotate_halves(uint4& x0, uint4& x1, const float* c, const float* s) {
  uint32_t* a = reinterpret_cast<uint32_t*>(&x0);
  uint32_t* b = reinterpret_cast<uint32_t*>(&x1);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 p = unpack2(a[e]), q = unpack2(b[e]);
    a[e] = pack2(p.x * c[2 * e] - q.x * s[2 * e], p.y * c[2 * e + 1] - q.y * s[2 * e + 1]);
    b[e] = pack2(q.x * c[2 * e] + p.x * s[2 * e], q.y * c[2 * e + 1] + p.y * s[2 * e + 1]);
  }
}
// Rotates the adjacent pairs of a vector of 8 elements by 4 angles.
__device__ __forceinline__ void rotate_pairs(uint4& x, const float* c, const float* s) {
  uint32_t* a = reinterpret_cast<uint32_t*>(&x);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 p = unpack2(a[e]);
    a[e] = pack2(p.x * c[e] - p.y * s[e], p.y * c[e] + p.x * s[e]);
  }
}

// A block takes rows_per_block rows: their sines first, in shared memory, then items of two
// 16-byte vectors (the two halves' vectors of 8 pairs, or 16 adjacent elements). What bounds it is
// memory: 32,744 rows of 32 + 2 x 8 heads of 128 take 125 to 132 us (805 MB, 6.1 to 6.4 TB/s, where a copy
// reaches 6.8), against 154 with a row a block and one item in flight; 1,024 rows 6.1 us, of which their
// 25 MB are 4. Few rows get a block each, so that all SMs load.
constexpr int kRopeRows = 8;
template <int D>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeParams p) {
  extern __shared__ __align__(16) float table[];  // [rows][2][rot / 2]: cosines, sines
  const spec_rope_args_t& a = p.a;
  __shared__ int pos_of[kRopeRows], slot_of[kRopeRows];
  constexpr int kItems = D / 16;
  const int half = a.rot_dim / 2;
  pdl_wait_prior();
  const int row0 = blockIdx.x * p.rows_per_block, nrows = min(p.rows_per_block, a.rows - row0);
  if (threadIdx.x < nrows) {
    const int slot = a.slots != nullptr ? a.slots[row0 + threadIdx.x] : -1;
    const int pos = a.positions[row0 + threadIdx.x];
    const bool past = slot >= 0 && slot / a.page_size >= a.num_pages;
    pos_of[threadIdx.x] = pos;
    slot_of[threadIdx.x] = past ? -1 : slot;
    if (past && pos >= 0 && a.status != nullptr) set_status(a.status, SPEC_FLAG_BAD_PAGE);
  }
  for (int i = threadIdx.x; i < nrows * half; i += kRopeThreads) {
    const int r = i / half, f = i - r * half;
    const int pos = a.positions[row0 + r];
    const uint64_t turn = static_cast<uint64_t>(static_cast<int64_t>(pos)) * a.turns[f];
    float c, s;
    sincospif(static_cast<float>(static_cast<int64_t>(turn)) * 1.0842021724855044e-19f, &s, &c);  // 2^-63
    table[(2 * r) * half + f] = c * p.factor;
    table[(2 * r + 1) * half + f] = s * p.factor;
  }
  __syncthreads();
  // Thread: item `it` of heads (head, row) hr, hr + step, ..; two are in flight together.
  const int it = threadIdx.x % kItems, step = kRopeThreads / kItems;
  const bool turned_item = it * 16 < a.rot_dim;
  int head = threadIdx.x / kItems, r = 0;
  auto settle = [&]() {
    while (head >= p.heads) {
      head -= p.heads;
      ++r;
    }
  };
  settle();
  while (r < nrows) {
    uint4 x0[2], x1[2];
    __nv_bfloat16 *out[2], *cached[2];
    int d0[2], d1[2], row_of[2];
    bool turned[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      out[k] = cached[k] = nullptr;
      if (r < nrows) {
        const int64_t row = row0 + r;
        const bool is_q = head < a.num_q_heads, is_v = head >= a.num_q_heads + a.num_kv_heads;
        const int h = is_q ? head : (is_v ? head - a.num_q_heads - a.num_kv_heads : head - a.num_q_heads);
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(is_q ? a.q : (is_v ? a.v : a.k));
        if (src != nullptr && pos_of[r] >= 0) {
          // where the two vectors are within the head
          turned[k] = !is_v && turned_item;
          const bool apart = turned[k] && !a.interleaved;
          d0[k] = apart ? it * 8 : it * 16;
          d1[k] = apart ? half + it * 8 : it * 16 + 8;
          row_of[k] = r;
          src += row * (is_q ? p.q_stride : (is_v ? p.v_stride : p.k_stride)) + static_cast<int64_t>(h) * D;
          const int slot = slot_of[r];
          if (!is_q && slot >= 0) {
            const int page = slot / a.page_size;
            cached[k] = static_cast<__nv_bfloat16*>(is_v ? a.v_cache : a.k_cache) +
                        ((static_cast<int64_t>(page) * a.num_kv_heads + h) * a.page_size + slot % a.page_size) * D;
          }
          if (is_q) out[k] = static_cast<__nv_bfloat16*>(a.q_out);
          else if (!is_v) out[k] = static_cast<__nv_bfloat16*>(a.k_out);
          if (out[k]) out[k] += row * (is_q ? p.q_out_stride : p.k_out_stride) + static_cast<int64_t>(h) * D;
          if (out[k] || cached[k]) {
            x0[k] = *reinterpret_cast<const uint4*>(src + d0[k]);
            x1[k] = *reinterpret_cast<const uint4*>(src + d1[k]);
          }
        }
      }
      head += step;
      settle();
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (!out[k] && !cached[k]) continue;
      if (turned[k]) {
        const float* c = table + 2 * row_of[k] * half + 8 * it;
        if (a.interleaved) {
          rotate_pairs(x0[k], c, c + half);
          rotate_pairs(x1[k], c + 4, c + half + 4);
        } else {
          rotate_halves(x0[k], x1[k], c, c + half);
        }
      }
      if (out[k]) {
        *reinterpret_cast<uint4*>(out[k] + d0[k]) = x0[k];
        *reinterpret_cast<uint4*>(out[k] + d1[k]) = x1[k];
      }
      if (cached[k]) {
        *reinterpret_cast<uint4*>(cached[k] + d0[k]) = x0[k];
        *reinterpret_cast<uint4*>(cached[k] + d1[k]) = x1[k];
      }
    }
  }
}

}  // namespace

cudaError_t launch_rope(const spec_rope_args_t& a, int sms, cudaStream_t stream) {
  RopeParams p;
  p.a = a;
  p.heads = a.num_q_heads + 2 * a.num_kv_heads;
  const int64_t dq = static_cast<int64_t>(a.num_q_heads) * a.head_dim, dk = static_cast<int64_t>(a.num_kv_heads) * a.head_dim;
  p.q_stride = a.q_row_stride ? a.q_row_stride : dq;
  p.k_stride = a.k_row_stride ? a.k_row_stride : dk;
  p.v_stride = a.v_row_stride ? a.v_row_stride : dk;
  p.q_out_stride = a.q_out_row_stride ? a.q_out_row_stride : dq;
  p.k_out_stride = a.k_out_row_stride ? a.k_out_row_stride : dk;
  p.factor = a.factor == 0.f ? 1.f : a.factor;
  // several rows a block once there are blocks for all SMs, so that threads have few idle turns
  p.rows_per_block = a.rows >= kRopeRows * 8 * sms ? kRopeRows : 1;
  const size_t smem = static_cast<size_t>(p.rows_per_block) * a.rot_dim * sizeof(float);
  const dim3 grid((a.rows + p.rows_per_block - 1) / p.rows_per_block);
  return launch_overlapped(a.head_dim == 128 ? rope_kernel<128> : rope_kernel<64>, grid, kRopeThreads, smem, stream, p);
}

}  // namespace specv
