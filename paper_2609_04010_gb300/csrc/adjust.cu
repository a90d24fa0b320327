// Penalties for repeated tokens, biases and grammar masks on logits rows
// (spec_adjust_logits).
//
// A block takes 2,048 tokens of the vocabulary of one sequence, for some of its rows. It counts
// the history's tokens of its range in shared memory once (integer atomics, so the counts do
// not depend on their order) and lists the tokens that are counted or biased. It then copies
// its logits under their mask bits, eight a thread (eight that the mask hides together are
// written without being read), and last rewrites the listed tokens, shared out over all
// threads: a few in a hundred logits, but so spread that handled in the copy they would hold
// up most warps (353 us at 64 x 16 x 128,256). The logits are read and written once; memory
// bounds it: 64 x 16 x 128,256 bf16 logits take 91 us, 5.9 TB/s (0.87 of the measured copy
// rate), 8 x 8 of them 12.8 us, a third of it the launch and a third the history. Fetching the
// first rows meanwhile into L2 gained nothing (13.3 us; 95.7 with all rows).
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "kv_fp8.cuh"

namespace specv {
namespace {

constexpr int kThreads = 256;
constexpr int kSlice = kAdjustSlice;
static_assert(kSlice == kThreads * 8, "eight tokens a thread");
constexpr uint32_t kPrompt = 0x80000000u, kBlock = 0x40000000u, kBias = 0x20000000u;  // beside a count
constexpr uint32_t kCount = 0x1fffffffu;

template <typename T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Eight logits of a thread, as the 16-byte words they are loaded and stored in.
template <typename T>
struct Eight {
  static constexpr int kWords = static_cast<int>(sizeof(T)) / 2;
  union {
    uint4 w[kWords];
    T x[8];
  };
  __device__ Eight() {}
};

struct Seq {
  float rep, freq, pres;
  const float* bias;  // the sequence's bias values
};

// The formula for one logit; c = its count word, bi = its place in the bias list.
__device__ __forceinline__ float adjust_one(float x, int v, uint32_t c, uint32_t bi, const Seq& q,
                                            const int* btok, int nblk) {
  int cnt = static_cast<int>(c & kCount);
  if (c & kBlock)
    for (int i = 0; i < nblk; ++i) cnt += btok[i] == v;
  if (cnt > 0 || (c & kPrompt)) x = x > 0.f ? __fdiv_rn(x, q.rep) : __fmul_rn(x, q.rep);
  if (cnt > 0) {
    x = __fsub_rn(x, __fmul_rn(q.freq, static_cast<float>(cnt)));
    x = __fsub_rn(x, q.pres);
  }
  if (c & kBias) x = __fadd_rn(x, __ldg(q.bias + bi));
  return x;
}

// VEC: rows are 16-byte aligned and a thread's eight tokens are consecutive; otherwise they
// are 32 apart, so that a warp's loads of one element each are.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 6) adjust_kernel(spec_adjust_args_t a, int rows) {
  __shared__ __align__(16) uint32_t count[kSlice];  // output count and flags
  __shared__ uint32_t place[kSlice];                // first place in the bias list
  __shared__ uint16_t list[kSlice];                 // the tokens with a count or a bias
  __shared__ int nlist;
  __shared__ int btok[64];
  const int tid = threadIdx.x, b = blockIdx.x;  // low token ids, which text uses most, start first
  const int v0 = blockIdx.y * kSlice, nv = min(kSlice, a.vocab - v0);
  const int G = a.gamma;
  const int row0 = blockIdx.z * rows, row1 = min(G, row0 + rows);  // this block's rows
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    reinterpret_cast<uint4*>(count)[tid + i * kThreads] = make_uint4(0, 0, 0, 0);
  }
  if (a.bias_tokens)
    for (int i = tid; i < kSlice; i += kThreads) place[i] = 0xffffffffu;
  if (tid == 0) nlist = 0;
  pdl_wait_prior();
  Seq q;
  q.rep = a.repetition ? a.repetition[b] : 1.f;
  q.freq = a.frequency ? a.frequency[b] : 0.f;
  q.pres = a.presence ? a.presence[b] : 0.f;
  q.bias = a.bias_values + static_cast<int64_t>(b) * a.max_bias;
  const bool penal = q.rep != 1.f || q.freq != 0.f || q.pres != 0.f;
  if (tid < 64) btok[tid] = a.block_tokens && tid < G ? a.block_tokens[static_cast<int64_t>(b) * G + tid] : -1;
  __syncthreads();
  const auto index = [&](int token) { return static_cast<uint32_t>(token) - static_cast<uint32_t>(v0); };
  if (penal && a.history) {
    const int hl = min(max(a.history_len[b], 0), a.max_history);
    const int pl = a.prompt_len ? min(max(a.prompt_len[b], 0), hl) : 0;
    const int32_t* h = a.history + static_cast<int64_t>(b) * a.max_history;
    auto add = [&](int token, int i) {
      const uint32_t u = index(token);
      if (u >= static_cast<uint32_t>(nv)) return;
      if (i < pl) atomicOr(&count[u], kPrompt);
      else atomicAdd(&count[u], 1u);
    };
    int i0 = 0;  // tokens taken four at a time, two loads in flight
    if ((reinterpret_cast<uintptr_t>(h) & 15u) == 0) {
      for (; i0 + 8 * kThreads <= hl; i0 += 8 * kThreads) {
        int4 t[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) t[e] = __ldg(reinterpret_cast<const int4*>(h + i0) + tid + e * kThreads);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int at = i0 + (tid + e * kThreads) * 4;
          add(t[e].x, at);
          add(t[e].y, at + 1);
          add(t[e].z, at + 2);
          add(t[e].w, at + 3);
        }
      }
    }
    for (; i0 < hl; i0 += 8 * kThreads) {
      int t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = i0 + tid + e * kThreads;
        t[e] = at < hl ? __ldg(h + at) : -1;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) add(t[e], i0 + tid + e * kThreads);
    }
  }
  if (penal && tid < G) {
    const uint32_t u = index(btok[tid]);
    if (u < static_cast<uint32_t>(nv)) atomicOr(&count[u], kBlock);
  }
  if (a.bias_tokens) {
    const int32_t* t = a.bias_tokens + static_cast<int64_t>(b) * a.max_bias;
    for (int i = tid; i < a.max_bias; i += kThreads) {
      const uint32_t u = index(__ldg(t + i));
      if (u >= static_cast<uint32_t>(nv)) continue;
      atomicMin(&place[u], static_cast<uint32_t>(i));
      atomicOr(&count[u], kBias);
    }
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (count[tid + e * kThreads]) list[atomicAdd(&nlist, 1)] = static_cast<uint16_t>(tid + e * kThreads);
  const int nmask = (a.vocab - 1) / 32 + 1;
  const T* in = static_cast<const T*>(a.logits) + static_cast<int64_t>(b) * G * a.vocab + v0;
  T* out = static_cast<T*>(a.out) + static_cast<int64_t>(b) * G * a.vocab + v0;
  const uint32_t* mask = a.allowed ? a.allowed + static_cast<int64_t>(b) * G * nmask : nullptr;
  // ---- the copy: this thread's tokens are u0 + e * (VEC ? 1 : 32) of the range ----
  const int u0 = VEC ? tid * 8 : (tid >> 5) * 256 + (tid & 31);
  const int word0 = (v0 + (VEC ? u0 : (tid >> 5) * 256)) >> 5;
  constexpr int U = VEC ? 4 / Eight<T>::kWords : 2;  // rows in flight
  for (int j0 = row0; j0 < (u0 < nv ? row1 : 0); j0 += U) {
    uint32_t keep[U];  // the mask's eight bits for each row
#pragma unroll
    for (int r = 0; r < U; ++r) {
      keep[r] = j0 + r < row1 ? 0xffu : 0u;
      if (mask && j0 + r < row1) {
        const uint32_t* w = mask + static_cast<int64_t>(j0 + r) * nmask + word0;
        if (VEC) {
          keep[r] = __ldg(reinterpret_cast<const uint8_t*>(w) + ((u0 >> 3) & 3));
        } else {
          keep[r] = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (u0 + e * 32 < nv) keep[r] |= (__ldg(w + e) >> (tid & 31) & 1u) << e;
        }
      }
    }
    Eight<T> x[U];
#pragma unroll
    for (int r = 0; r < U; ++r) {
      if (!keep[r]) continue;
      const T* src = in + static_cast<int64_t>(j0 + r) * a.vocab + u0;
      if (VEC) {
#pragma unroll
        for (int w = 0; w < Eight<T>::kWords; ++w) x[r].w[w] = __ldcs(reinterpret_cast<const uint4*>(src) + w);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (u0 + e * 32 < nv) x[r].x[e] = src[e * 32];
      }
    }
#pragma unroll
    for (int r = 0; r < U; ++r) {
      if (j0 + r >= row1) break;
      if (keep[r] != 0xffu) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(keep[r] >> e & 1)) x[r].x[e] = from_f32<T>(-INFINITY);
      }
      T* dst = out + static_cast<int64_t>(j0 + r) * a.vocab + u0;
      if (VEC) {
#pragma unroll
        for (int w = 0; w < Eight<T>::kWords; ++w) reinterpret_cast<uint4*>(dst)[w] = x[r].w[w];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (u0 + e * 32 < nv) dst[e * 32] = x[r].x[e];
      }
    }
  }
  // ---- the listed tokens (out already holds their logits, so it may be the input) ----
  __syncthreads();
  const int n = nlist;
  constexpr int W = 2;  // in flight
  const int items = n * (row1 - row0);
  for (int it0 = tid; it0 < items; it0 += W * kThreads) {
    int64_t at[W];
    int row[W], u[W];
    float x[W];
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const int it = it0 + e * kThreads;
      at[e] = -1;
      if (it >= items) continue;
      row[e] = row0 + it / n;
      u[e] = list[it % n];
      const int v = v0 + u[e];
      if (mask && !(__ldg(mask + static_cast<int64_t>(row[e]) * nmask + (v >> 5)) >> (v & 31) & 1u)) continue;
      at[e] = static_cast<int64_t>(row[e]) * a.vocab + u[e];
      x[e] = to_f32<T>(out[at[e]]);
    }
#pragma unroll
    for (int e = 0; e < W; ++e) {
      if (at[e] < 0) continue;
      const int nblk = a.block_shift ? row[e] : row[e] + 1;
      out[at[e]] = from_f32<T>(adjust_one(x[e], v0 + u[e], count[u[e]], place[u[e]], q, btok, nblk));
    }
  }
}

template <typename T>
cudaError_t launch_typed(const spec_adjust_args_t& a, bool vec, int sms, cudaStream_t stream) {
  // rows are shared out among blocks (each counts the history again) until there are about two
  // rounds of them
  const int64_t blocks = static_cast<int64_t>(a.batch) * ((a.vocab - 1) / kSlice + 1);
  const int64_t splits = std::min<int64_t>(a.gamma, std::max<int64_t>(1, 12 * sms / blocks));
  const int rows = static_cast<int>((a.gamma + splits - 1) / splits);
  const dim3 grid(a.batch, (a.vocab - 1) / kSlice + 1, (a.gamma - 1) / rows + 1);
  return launch_overlapped(vec ? adjust_kernel<T, true> : adjust_kernel<T, false>, grid, kThreads, 0, stream, a, rows);
}

}  // namespace

cudaError_t launch_adjust(const spec_adjust_args_t& a, int sms, cudaStream_t stream) {
  const size_t esz = a.logits_dtype == SPEC_BF16 ? 2 : 4;
  // whole groups of eight in aligned rows
  const bool vec = a.vocab % 8 == 0 &&
                   ((reinterpret_cast<uintptr_t>(a.logits) | reinterpret_cast<uintptr_t>(a.out)) & 15u) == 0;
  (void)cudaGetLastError();
  return esz == 2 ? launch_typed<__nv_bfloat16>(a, vec, sms, stream) : launch_typed<float>(a, vec, sms, stream);
}

}  // namespace specv
