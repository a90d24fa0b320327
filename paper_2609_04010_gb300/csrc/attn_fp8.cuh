// Internal helpers of the attention kernels over the 8-bit cache: launch parameters, and
// the merge of split-KV partials (each keeps an unnormalised fp32 output, its base-2
// maximum m and its sum l).
#pragma once

#include "attn_common.cuh"
#include "kv_fp8.cuh"

namespace specv {

// AttnParams with k_cache = the 8-bit cache (v_cache unused) and its scales.
struct AttnFp8Params : AttnParams {
  const float* kv_scale;  // [num_pages][Hkv][2]
  int4* splits;           // [P.splits][2]: units to merge (tensor-core kernels)
  int split_by_unit;      // a place for each unit in it, else for each block
  int blocks;             // of the tensor-core kernels' grid
};

inline AttnFp8Params make_attn_fp8_params(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws) {
  AttnFp8Params p{};
  p.batch = a.batch;
  p.gamma = a.gamma;
  p.hq = a.num_q_heads;
  p.hkv = a.num_kv_heads;
  p.hunits = a.num_kv_heads;
  p.group = a.num_q_heads / a.num_kv_heads;
  p.rows = P.rows;
  p.row_tiles = P.row_tiles;
  p.page_size = a.page_size;
  p.max_pages = a.max_pages_per_seq;
  p.num_pages = a.num_pages;
  p.nsplit = P.nsplit;
  p.tiles_per_split = P.tiles_per_split;
  p.slot_rows = P.slot_rows;
  p.max_keys = a.max_pages_per_seq * a.page_size;
  const float scale = a.softmax_scale != 0.f ? a.softmax_scale : 1.f / sqrtf(static_cast<float>(a.head_dim));
  p.scale_log2 = scale * kLog2e;
  p.q = a.q;
  p.k_cache = a.kv_cache;
  p.kv_scale = a.kv_scale;
  p.page_table = a.page_table;
  p.kv_len = a.kv_len;
  p.out = a.out;
  p.lse = a.lse;
  p.status = reinterpret_cast<uint32_t*>(ws);
  p.tickets = reinterpret_cast<uint32_t*>(ws + P.tickets);
  p.splits = reinterpret_cast<int4*>(ws + P.split_notes);
  p.split_by_unit = P.splits < P.grid;
  p.blocks = P.grid;
  p.partial_o = reinterpret_cast<float*>(ws + P.partial_o);
  p.partial_ml = reinterpret_cast<float2*>(ws + P.partial_ml);
  p.tree_mask = a.tree_mask;
  return p;
}

#ifdef __CUDACC__
// 1 / l for a row's output: 0 for a bad sequence (l = -1) or a row that saw no key (l = 0);
// NaN stays NaN.
__device__ __forceinline__ float fp8_inv(float l) { return l <= 0.f ? 0.f : 1.f / l; }

// lse of a row from its base-2 maximum and sum.
__device__ __forceinline__ float fp8_lse(float m, float l) {
  return l <= 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

__device__ __forceinline__ void write_fp8_lse(const AttnParams& p, int b, int g, int row, float m, float l) {
  if (!p.lse) return;
  const int j = row / p.group, h = g * p.group + row % p.group;
  p.lse[(static_cast<int64_t>(b) * p.gamma + j) * p.hq + h] = fp8_lse(m, l);
}

// Merges and writes 8 columns (from 8 * c8) of row `row` of KV head g, whose n parts are row
// `hr` of the slots slot_of(0 .. n - 1). A slot's outputs are [row][D], or with BY_COLUMNS
// [D / 4][row][4]. The loads of up to three slots are in flight together (few units have
// more; trees of 31 for 8 requests: 44.0 us, two or four 44.3).
template <int D, bool BY_COLUMNS, typename SlotOf>
__device__ __forceinline__ void merge_fp8_item(const AttnParams& p, int b, int g, int row, SlotOf slot_of, int n,
                                               int hr, int c8) {
  constexpr int SB = 3;
  float M = -INFINITY, L = 0.f, acc[8];
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  for (int s0 = 0; s0 < n; s0 += SB) {
    float2 ml[SB];
    float4 lo[SB], hi[SB];
#pragma unroll
    for (int i = 0; i < SB; ++i) {
      ml[i] = make_float2(-INFINITY, 0.f);
      lo[i] = hi[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (s0 + i < n) {
        const int64_t first = static_cast<int64_t>(slot_of(s0 + i)) * p.slot_rows;
        const float4* src = reinterpret_cast<const float4*>(p.partial_o) + first * (D / 4) +
                            (BY_COLUMNS ? 2 * c8 * p.slot_rows + hr : hr * (D / 4) + 2 * c8);
        ml[i] = __ldcg(&p.partial_ml[first + hr]);
        lo[i] = __ldcg(src);
        hi[i] = __ldcg(src + (BY_COLUMNS ? p.slot_rows : 1));
      }
    }
#pragma unroll
    for (int i = 0; i < SB; ++i) {
      if (ml[i].y < 0.f) bad = true;
      if (ml[i].y == 0.f) continue;  // saw no key
      const float m = fmaxf(M, ml[i].x);
      const float old = M == -INFINITY ? 0.f : ex2(M - m), w = m == -INFINITY ? 1.f : ex2(ml[i].x - m);
      L = L * old + ml[i].y * w;
      const float x[8] = {lo[i].x, lo[i].y, lo[i].z, lo[i].w, hi[i].x, hi[i].y, hi[i].z, hi[i].w};
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = acc[e] * old + x[e] * w;
      M = m;
    }
  }
  if (bad) L = -1.f;
  const float inv = fp8_inv(L);
  if (inv == 0.f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  }
  write_out_row<D>(p, b, g, row, c8 * 8, acc, inv);
  if (c8 == 0) write_fp8_lse(p, b, g, row, M, L);
}
#endif

}  // namespace specv
