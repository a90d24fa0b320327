// Attention of the block queries over the 8-bit KV cache on CUDA cores
// (spec_verify_attention_fp8, SPEC_ATTN_CUDA_CORES).
//
// Work unit: (sequence, KV head, row tile of 16 query rows, KV split). A tile of 64 keys is
// gathered through the page table, decoded and scaled to fp32 in shared memory; scores,
// softmax (base 2, running maximum and sum) and outputs are fp32. The last split of a unit
// to finish (atomic ticket, no waiting) merges the splits. It is the path for what the
// tensor-core kernel does not take, and a second implementation to compare it with.
#include <cuda_bf16.h>

#include <cmath>

#include "attn_fp8.cuh"

namespace specv {
namespace {

constexpr int RT = kSimtRowTile;
constexpr int TK = kSimtKeyTile;
constexpr int NT = kSimtThreads;

template <int D>
struct Smem {
  static constexpr int kStride = D + 4;  // floats per staged row (bank spread)
  float q[RT][D];
  float k[TK][kStride];
  float v[TK][kStride];
  float s[RT][TK];
  float alpha[RT], m[RT], l[RT];
  unsigned long long tmask[RT];
  int bad, last;
};

template <int D>
__global__ void __launch_bounds__(NT) attn_fp8_simt_kernel(AttnFp8Params p) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(smem_raw);
  const int split = blockIdx.x, g = blockIdx.y;
  const int b = blockIdx.z / p.row_tiles, rt = blockIdx.z % p.row_tiles;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row0 = rt * RT, nrows = min(RT, p.rows - row0);
  const int kv_len = p.kv_len[b];
  const bool len_ok = kv_len >= p.gamma && kv_len <= p.max_keys;
  const int64_t begin = static_cast<int64_t>(split) * p.tiles_per_split * TK;
  const int key_begin = static_cast<int>(min(begin, static_cast<int64_t>(p.max_keys)));
  const int key_end = len_ok ? static_cast<int>(min(static_cast<int64_t>(kv_len), begin + static_cast<int64_t>(p.tiles_per_split) * TK)) : 0;
  const int32_t* table = p.page_table + static_cast<int64_t>(b) * p.max_pages;
  if (tid == 0) sm.bad = len_ok ? 0 : 2;
  __syncthreads();
  if (key_end > key_begin) {
    const int pg1 = (key_end - 1) / p.page_size;
    for (int pg = key_begin / p.page_size + tid; pg <= pg1; pg += NT) {
      const int id = table[pg];
      if (id < 0 || id >= p.num_pages) sm.bad = 1;
    }
  }
  const __nv_bfloat16* qg = static_cast<const __nv_bfloat16*>(p.q);
  for (int i = tid; i < RT * D; i += NT) {
    const int r = i / D, d = i % D;
    float x = 0.f;
    if (r < nrows) {
      const int row = row0 + r, j = row / p.group, h = g * p.group + row % p.group;
      x = __bfloat162float(qg[((static_cast<int64_t>(b) * p.gamma + j) * p.hq + h) * D + d]) * p.scale_log2;
    }
    sm.q[r][d] = x;
  }
  if (tid < RT) {
    sm.m[tid] = -INFINITY;
    sm.l[tid] = 0.f;
    const int j = min(row0 + tid, p.rows - 1) / p.group;
    sm.tmask[tid] = p.tree_mask ? p.tree_mask[static_cast<int64_t>(b) * p.gamma + j] : 0ull;
  }
  __syncthreads();
  const bool bad = sm.bad != 0;
  const int ctx = kv_len - p.gamma;

  // P V: a thread owns 8 consecutive dims of rows rg, rg + RG, ...
  constexpr int DQ = D / 8, RG = NT / DQ, RPT = RT / RG;
  const int dq = tid % DQ, rg = tid / DQ;
  float o[RPT][8];
#pragma unroll
  for (int i = 0; i < RPT; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) o[i][e] = 0.f;

  const uint8_t* cache = static_cast<const uint8_t*>(p.k_cache);
  const int kk = tid % TK, hr = tid / TK;  // Q K^T: key kk, rows hr, hr + 2, ...
  for (int t0 = key_begin; !bad && t0 < key_end; t0 += TK) {
    constexpr int kPieces = D / 16;
    for (int c = tid; c < 2 * TK * kPieces; c += NT) {
      const int kind = c / (TK * kPieces), key = (c / kPieces) % TK, piece = c % kPieces;
      uint4 raw = make_uint4(0, 0, 0, 0);
      float sc = 0.f;
      if (t0 + key < kv_len) {
        const int64_t ph = static_cast<int64_t>(table[(t0 + key) / p.page_size]) * p.hkv + g;
        raw = __ldg(reinterpret_cast<const uint4*>(
            cache + ((ph * 2 + kind) * p.page_size + (t0 + key) % p.page_size) * D + piece * 16));
        sc = p.kv_scale[ph * 2 + kind];
        if (kind) sc = clamp_scale(sc);
      }
      float* dst = (kind ? sm.v[key] : sm.k[key]) + piece * 16;
      const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 a = from_e4m3x2(w[e] & 0xffffu), c2 = from_e4m3x2(w[e] >> 16);
        *reinterpret_cast<float4*>(dst + 4 * e) = make_float4(a.x * sc, a.y * sc, c2.x * sc, c2.y * sc);
      }
    }
    __syncthreads();
    {
      float acc[RT / 2];
#pragma unroll
      for (int i = 0; i < RT / 2; ++i) acc[i] = 0.f;
#pragma unroll 4
      for (int d = 0; d < D; d += 4) {
        const float4 kf = *reinterpret_cast<const float4*>(&sm.k[kk][d]);
#pragma unroll
        for (int i = 0; i < RT / 2; ++i) {
          const float4 q = *reinterpret_cast<const float4*>(&sm.q[hr + 2 * i][d]);
          acc[i] += q.x * kf.x + q.y * kf.y + q.z * kf.z + q.w * kf.w;
        }
      }
      const int rel = t0 + kk - ctx;  // block position of the key (negative: the prefix)
#pragma unroll
      for (int i = 0; i < RT / 2; ++i) {
        const int r = hr + 2 * i, j = (row0 + r) / p.group;
        const bool vis = r < nrows && (p.tree_mask ? (rel < 0 || (rel < p.gamma && ((sm.tmask[r] >> rel) & 1ull)))
                                                   : rel <= j);
        sm.s[r][kk] = vis ? acc[i] : -INFINITY;
      }
    }
    __syncthreads();
    for (int r = warp; r < RT; r += NT / 32) {
      const float a0 = sm.s[r][lane], a1 = sm.s[r][lane + 32];
      float mx = fmaxf(a0, a1);
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
      const float m_old = sm.m[r], m_new = fmaxf(m_old, mx);
      const float sub = m_new == -INFINITY ? 0.f : m_new;
      const float p0 = ex2(a0 - sub), p1 = ex2(a1 - sub);
      const float alpha = m_old == -INFINITY ? 0.f : ex2(m_old - sub);
      float sum = p0 + p1;
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
      __syncwarp();
      sm.s[r][lane] = p0;
      sm.s[r][lane + 32] = p1;
      if (lane == 0) {
        sm.alpha[r] = alpha;
        sm.m[r] = m_new;
        sm.l[r] = sm.l[r] * alpha + sum;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const float a = sm.alpha[rg + i * RG];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[i][e] *= a;
    }
    for (int k = 0; k < TK; ++k) {
      const float4 v0 = *reinterpret_cast<const float4*>(&sm.v[k][dq * 8]);
      const float4 v1 = *reinterpret_cast<const float4*>(&sm.v[k][dq * 8 + 4]);
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        const float w = sm.s[rg + i * RG][k];
        if (w == 0.f) continue;  // a hidden key adds nothing, whatever its value
        o[i][0] += w * v0.x; o[i][1] += w * v0.y; o[i][2] += w * v0.z; o[i][3] += w * v0.w;
        o[i][4] += w * v1.x; o[i][5] += w * v1.y; o[i][6] += w * v1.z; o[i][7] += w * v1.w;
      }
    }
    __syncthreads();
  }

  const int64_t unit = (static_cast<int64_t>(b) * p.hkv + g) * p.row_tiles + rt;
  if (tid == 0 && bad) set_status(p.status, sm.bad == 2 ? SPEC_FLAG_BAD_KV_LEN : SPEC_FLAG_BAD_PAGE);
  if (p.nsplit == 1) {
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int r = rg + i * RG;
      if (r < nrows) write_out_row<D>(p, b, g, row0 + r, dq * 8, o[i], bad ? 0.f : fp8_inv(sm.l[r]));
    }
    if (tid < nrows) write_fp8_lse(p, b, g, row0 + tid, sm.m[tid], bad ? -1.f : sm.l[tid]);
    return;
  }
  const int64_t slot = unit * p.nsplit + split;
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    float4* dst = reinterpret_cast<float4*>(p.partial_o + (slot * p.slot_rows + rg + i * RG) * D + dq * 8);
    dst[0] = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
    dst[1] = make_float4(o[i][4], o[i][5], o[i][6], o[i][7]);
  }
  if (tid < RT) p.partial_ml[slot * p.slot_rows + tid] = make_float2(sm.m[tid], bad ? -1.f : sm.l[tid]);
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    sm.last = atomicAdd(&p.tickets[unit], 1u) == static_cast<uint32_t>(p.nsplit - 1);
    if (sm.last) p.tickets[unit] = 0;
  }
  __syncthreads();
  if (!sm.last) return;
  __threadfence();
  for (int i = tid; i < nrows * (D / 8); i += NT)
    merge_fp8_item<D, false>(p, b, g, row0 + i / (D / 8), [&](int s) { return unit * p.nsplit + s; }, p.nsplit, i / (D / 8),
                             i % (D / 8));
}

template <int D>
cudaError_t launch_simt_d(const AttnFp8Params& p, const dim3& grid, cudaStream_t stream) {
  const size_t smem = sizeof(Smem<D>);
  const cudaError_t e = cudaFuncSetAttribute(
      attn_fp8_simt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  attn_fp8_simt_kernel<D><<<grid, NT, smem, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attn_fp8_simt(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws,
                                 cudaStream_t stream) {
  const AttnFp8Params p = make_attn_fp8_params(a, P, ws);
  const dim3 grid(P.nsplit, a.num_kv_heads, a.batch * P.row_tiles);
  return a.head_dim == 128 ? launch_simt_d<128>(p, grid, stream) : launch_simt_d<64>(p, grid, stream);
}

}  // namespace specv
