// Penalties for repeated tokens, biases and grammar masks on logits rows
// (spec_adjust_logits).
//
// A block takes a slice of the vocabulary of one sequence, for all of its rows. It counts
// the history's tokens of the slice in shared memory once (integer atomics, so the counts
// do not depend on their order) and then streams the rows: almost every group of eight
// logits has no counted and no biased token, which one bit per group says, and is copied
// under its eight mask bits; the few others take the formula with the counts. A group that
// the mask hides whole is written without being read. The logits are read and written once.
#include <cuda_bf16.h>

#include <cmath>

#include "kv_fp8.cuh"

namespace specv {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxSlice = 4096;  // tokens of a block: 32 KB of counts and bias places
constexpr uint32_t kPrompt = 0x80000000u;

struct AdjustParams {
  spec_adjust_args_t a;
  int slice, nmask;
};

__device__ __forceinline__ float load_logit(const float* p) { return *p; }
__device__ __forceinline__ float load_logit(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_logit(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_logit(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

struct Seq {
  float rep, freq, pres;
  const float* bias;  // the sequence's bias values
};

// The formula for one logit; c = count word, bi = place in the bias list (or none).
__device__ __forceinline__ float adjust_one(float x, int v, uint32_t c, uint32_t bi, const Seq& q,
                                            const int* btok, int nblk) {
  int cnt = static_cast<int>(c & ~kPrompt);
  for (int i = 0; i < nblk; ++i) cnt += btok[i] == v;
  if (cnt > 0 || (c & kPrompt)) x = x > 0.f ? __fdiv_rn(x, q.rep) : __fmul_rn(x, q.rep);
  if (cnt > 0) {
    x = __fsub_rn(x, __fmul_rn(q.freq, static_cast<float>(cnt)));
    x = __fsub_rn(x, q.pres);
  }
  if (bi != 0xffffffffu) x = __fadd_rn(x, __ldg(q.bias + bi));
  return x;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) adjust_kernel(AdjustParams p) {
  extern __shared__ __align__(16) uint32_t smem[];
  const spec_adjust_args_t& a = p.a;
  const int S = p.slice;
  uint32_t* count = smem;              // [S]: output count, bit 31 = in the prompt
  uint32_t* place = count + S;         // [S]: first place in the bias list
  uint32_t* dirty = place + S;         // [S / 256]: one bit per eight tokens
  __shared__ int btok[64];
  const int tid = threadIdx.x, b = blockIdx.y;
  const int v0 = blockIdx.x * S, nv = min(S, a.vocab - v0);
  const int G = a.gamma;
  Seq q;
  q.rep = a.repetition ? a.repetition[b] : 1.f;
  q.freq = a.frequency ? a.frequency[b] : 0.f;
  q.pres = a.presence ? a.presence[b] : 0.f;
  q.bias = a.bias_values + static_cast<int64_t>(b) * a.max_bias;
  const bool penal = q.rep != 1.f || q.freq != 0.f || q.pres != 0.f;
  for (int i = tid; i < S; i += kThreads) {
    count[i] = 0;
    place[i] = 0xffffffffu;
  }
  for (int i = tid; i < S / 256; i += kThreads) dirty[i] = 0;
  if (tid < 64) btok[tid] = a.block_tokens && tid < G ? a.block_tokens[b * G + tid] : -1;
  __syncthreads();
  auto mark = [&](int u) { atomicOr(&dirty[u >> 8], 1u << ((u >> 3) & 31)); };
  if (penal && a.history) {
    const int hl = min(max(a.history_len[b], 0), a.max_history);
    const int pl = a.prompt_len ? min(max(a.prompt_len[b], 0), hl) : 0;
    const int32_t* h = a.history + static_cast<int64_t>(b) * a.max_history;
    for (int i = tid; i < hl; i += kThreads) {
      const uint32_t u = static_cast<uint32_t>(__ldg(h + i)) - static_cast<uint32_t>(v0);
      if (u >= static_cast<uint32_t>(nv)) continue;
      if (i < pl) atomicOr(&count[u], kPrompt); else atomicAdd(&count[u], 1u);
      mark(u);
    }
  }
  if (penal && tid < G) {
    const uint32_t u = static_cast<uint32_t>(btok[tid]) - static_cast<uint32_t>(v0);
    if (u < static_cast<uint32_t>(nv)) mark(u);
  }
  if (a.bias_tokens) {
    const int32_t* t = a.bias_tokens + static_cast<int64_t>(b) * a.max_bias;
    for (int i = tid; i < a.max_bias; i += kThreads) {
      const uint32_t u = static_cast<uint32_t>(__ldg(t + i)) - static_cast<uint32_t>(v0);
      if (u >= static_cast<uint32_t>(nv)) continue;
      atomicMin(&place[u], static_cast<uint32_t>(i));
      mark(u);
    }
  }
  __syncthreads();
  const T* in = static_cast<const T*>(a.logits);
  T* out = static_cast<T*>(a.out);
  const int groups = (nv + 7) / 8;
  for (int64_t it = tid; it < static_cast<int64_t>(groups) * G; it += kThreads) {
    const int j = static_cast<int>(it / groups), g = static_cast<int>(it % groups);
    const int64_t row = static_cast<int64_t>(b) * G + j;
    const uint32_t* mask = a.allowed ? a.allowed + row * p.nmask : nullptr;
    const bool slow = dirty[g >> 5] >> (g & 31) & 1;
    const int nblk = penal ? (a.block_shift ? j : j + 1) : 0;
    for (int e = 0; e < 8; ++e) {
      const int u = g * 8 + e;
      if (u >= nv) break;
      const int v = v0 + u;
      const int64_t at = row * a.vocab + v;
      if (mask && !(__ldg(mask + (v >> 5)) >> (v & 31) & 1)) {
        store_logit(out + at, -INFINITY);
        continue;
      }
      float x = load_logit(in + at);
      if (slow) x = adjust_one(x, v, count[u], place[u], q, btok, nblk);
      store_logit(out + at, x);
    }
  }
}

}  // namespace

cudaError_t launch_adjust(const spec_adjust_args_t& a, cudaStream_t stream) {
  AdjustParams p;
  p.a = a;
  p.slice = kMaxSlice;
  p.nmask = (a.vocab - 1) / 32 + 1;
  const dim3 grid((a.vocab - 1) / p.slice + 1, a.batch);
  const size_t smem = (2 * p.slice + p.slice / 256) * sizeof(uint32_t);
  (void)cudaGetLastError();
  if (a.logits_dtype == SPEC_BF16) adjust_kernel<__nv_bfloat16><<<grid, kThreads, smem, stream>>>(p);
  else adjust_kernel<float><<<grid, kThreads, smem, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace specv
