// Attention of ragged chunks over the paged caches: what a call prepares and finishes, and the
// CUDA-core kernel (spec_chunk_attention, SPEC_ATTN_CUDA_CORES).
//
//   o = sum_k 2^(s_k - m) v_k / sum_k 2^(s_k - m),  s_k = scale log2(e) q.k, over low <= k < high
//
// The CUDA-core kernel takes 16 query rows of one KV head and tiles of 64 keys, gathered through
// the page table into shared memory in fp32; scores, running maximum and sum, and outputs are
// fp32. It serves what the tensor-core kernel does not take and is a second implementation to
// compare it with; long prompts, which take the tensor cores 468 us, take it 51 ms.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "chunk.cuh"
#include "kv_fp8.cuh"

namespace specv {
namespace {

constexpr int RT = kSimtRowTile;
constexpr int NT = kSimtThreads;

template <int D, int TK>
struct Smem {
  static constexpr int kStride = D + 4;  // floats per staged row (bank spread)
  float q[RT][D];
  float k[TK][kStride];
  float v[TK][kStride];
  float s[RT][TK];
  float alpha[RT], m[RT], l[RT];
  int low[RT], high[RT];  // keys that a row sees
  int bad;
};

// Lengths of the batch, once per call: which rows a sequence has and whether they can be served;
// for the tensor cores also the work list, equal numbers of virtual steps per block. One block,
// because all of it depends on sums over the batch. What bounds it is latency: a chain of loads, two
// scans and searches, 2 to 5 us that a short call sees in full. Of 14.7 us for one token behind 512 keys
// the block of 1,024 threads took .5 more than the one of 128 that small calls get.
constexpr int kSetupThreads = 1024;
constexpr int kSetupFew = 128;    // threads for at most as many sequences and units
constexpr int kSetupKept = 1024;  // sequences and units that are kept in shared memory too

// Blocks of RT query rows (token, head of the group) of a sequence with n new tokens, for one KV head.
__device__ __forceinline__ int simt_units(const ChunkParams& p, int n) { return (n * p.group + RT - 1) / RT; }

// The exclusive prefix sum of v in thread order over a block of THREADS threads, and the total.
template <int THREADS>
__device__ __forceinline__ long long scan_block(long long v, long long* sh, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sh[warp] = x;
  __syncthreads();
  long long w = lane < THREADS / 32 ? sh[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  const long long before = warp ? __shfl_sync(0xffffffffu, w, warp - 1) : 0;
  *total = __shfl_sync(0xffffffffu, w, 31);
  __syncthreads();
  return before + x - v;
}

// Query rows as fp16 for the products with the 8-bit cache, each scaled by the power of two that takes
// its largest finite magnitude into [2^14, 2^15): bf16 values down to 2^-31 of that are exact, smaller
// ones to 2^-39 of it.
template <int D>
__device__ __forceinline__ void halve_queries(const ChunkParams& p, int64_t warp, int64_t warps) {
  constexpr int kLanes = D / 8, kEach = 32 / kLanes;  // lanes of a row, rows of a warp
  const int lane = threadIdx.x & 31, sub = lane / kLanes, piece = lane % kLanes;
  const int64_t heads = static_cast<int64_t>(p.rows) * p.hq;
  for (int64_t r0 = warp * kEach; r0 < heads; r0 += warps * kEach) {
    const int64_t r = r0 + sub;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < heads)
      v = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + r / p.hq * p.q_stride + r % p.hq * D) + piece);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t lo = w[e] & 0x7fffu, hi = w[e] >> 16 & 0x7fffu;
      top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
    }
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    // top = f * 2^(e - 127): times 2^(141 - e); both factors stay normal numbers
    const int up = top == 0 ? 0 : min(126, max(-113, 141 - static_cast<int>(top >> 7)));
    const float f = __uint_as_float(static_cast<uint32_t>(up + 127) << 23);
    uint32_t h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __half2 x = __floats2half2_rn(__uint_as_float(w[e] << 16) * f, __uint_as_float(w[e] & 0xffff0000u) * f);
      h[e] = *reinterpret_cast<const uint32_t*>(&x);
    }
    if (r < heads) {
      reinterpret_cast<uint4*>(p.q_half)[r * kLanes + piece] = make_uint4(h[0], h[1], h[2], h[3]);
      if (piece == 0) p.q_scale[r] = __uint_as_float(static_cast<uint32_t>(127 - up) << 23);
    }
  }
}

// D: 0, or the head dimension where query rows are to be made fp16, by all blocks but the first.
template <int D, int THREADS>
__global__ void __launch_bounds__(THREADS) chunk_setup_kernel(ChunkParams p) {
  if constexpr (D > 0) {
    if (blockIdx.x > 0) {
      pdl_wait_prior();
      halve_queries<D>(p, (blockIdx.x - 1) * (THREADS / 32) + (threadIdx.x >> 5), static_cast<int64_t>(gridDim.x - 1) * (THREADS / 32));
      return;
    }
  }
  __shared__ long long sh[32];
  __shared__ ChunkSeq seq_kept[kSetupKept + 1];
  __shared__ long long cum_kept[kSetupKept + 1];
  pdl_wait_prior();
  const int tid = threadIdx.x;
  long long carry = 0;
  for (int b0 = 0; b0 < p.batch; b0 += THREADS) {
    const int b = b0 + tid;
    ChunkSeq s = {0, 0, 0, 0};
    bool bad = false;
    if (b < p.batch) {
      const int r0 = p.row_start[b], r1 = p.row_start[b + 1];
      bad = !chunk_rows_ok(p, r0, r1);
      s.row0 = r0;
      s.n = bad ? 0 : r1 - r0;
      if (s.n > 0) {
        s.kv_len = p.kv_len[b];
        if (s.kv_len < s.n || s.kv_len > p.max_keys) {
          s.n = 0;
          bad = true;
        }
      }
    }
    const int units = p.blocks ? chunk_units(p, s.n) : simt_units(p, s.n);
    long long all;
    const long long before = carry + scan_block<THREADS>(units, sh, &all);
    carry += all;
    if (b < p.batch) {
      // (rows that sequences share, out of order, could make more units than there is room for)
      if (before + units > p.max_units && units > 0) {
        s.n = 0;
        bad = true;
      }
      s.first_unit = static_cast<int>(min(before, static_cast<long long>(p.max_units)));
      p.seqs[b] = s;
      p.seq_bad[b] = bad ? 1 : 0;
      if (bad) set_status(p.status, SPEC_FLAG_BAD_KV_LEN);
      if (b < kSetupKept) seq_kept[b] = s;
    }
  }
  const int nunits = static_cast<int>(min(carry, static_cast<long long>(p.max_units)));
  if (tid == 0) p.seqs[p.batch] = {0, 0, 0, nunits};
  if (!p.blocks) return;
  if (tid == 0) {
    if (p.batch <= kSetupKept) seq_kept[p.batch] = {0, 0, 0, nunits};
    p.redo[0] = make_int4(0, 0, 0, 0);
    p.cum[0] = 0;
    cum_kept[0] = 0;
  }
  __syncthreads();
  const ChunkSeq* seqs = p.batch <= kSetupKept ? seq_kept : p.seqs;
  auto first = [&](int b) { return seqs[b].first_unit; };
  const long long* cum = nunits <= kSetupKept ? cum_kept : p.cum;
  carry = 0;
  for (int u0 = 0; u0 < nunits; u0 += THREADS) {
    const int u = u0 + tid;
    int steps = 0;
    if (u < nunits) {
      int lo = 0, hi = p.batch;  // the largest b with first(b) <= u
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first(mid) <= u) lo = mid; else hi = mid;
      }
      const ChunkSeq s = seqs[lo];
      if (u - s.first_unit < chunk_units(p, s.n)) steps = chunk_unit(p, s, u - s.first_unit).length();
    }
    long long all;
    const long long before = carry + scan_block<THREADS>(steps, sh, &all);
    carry += all;
    if (u < nunits) {
      p.cum[u + 1] = before + steps;
      if (u < kSetupKept) cum_kept[u + 1] = before + steps;
    }
  }
  __syncthreads();
  const long long total = carry * p.hkv;
  const int active = static_cast<int>(min(total / kChunkTwinCost, static_cast<long long>(p.blocks)));
  if (tid == 0) {
    p.work->total = total;
    p.work->active = active;
  }
  for (int c = tid; c < p.blocks; c += THREADS) {
    if (c >= active) {
      p.work->starts[c] = {0, 0, 0, 0, 0, 0, 0, 0};
      continue;
    }
    const long long t = c * total / active;
    int lo = 0, hi = p.batch;  // the largest b whose steps begin at or before t
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cum[first(mid)] * p.hkv <= t) lo = mid; else hi = mid;
    }
    const int b = lo, f = first(b), end = first(b + 1);
    const long long base = cum[f], each = cum[end] - base;
    const int g = static_cast<int>((t - base * p.hkv) / each);
    const long long rem = t - base * p.hkv - g * each;
    lo = f;
    hi = end;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cum[mid] - base <= rem) lo = mid; else hi = mid;
    }
    const ChunkSeq s = seqs[b];
    p.work->starts[c] = {b,      g,   lo - f,   static_cast<int>(rem - (cum[lo] - base)),
                         s.row0, s.n, s.kv_len, static_cast<int>((c + 1) * total / active - t)};
  }
}

// Rows [row0, row0 + nrows) of sequence b and KV head g (row = token * group + head of the group).
template <int D, bool FP8, int TK>
__device__ void simt_rows(const ChunkParams& p, Smem<D, TK>& sm, int b, const ChunkSeq& seq, int g, int row0, int nrows) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctx = seq.kv_len - seq.n;
  const int at0 = ctx + row0 / p.group, at1 = ctx + (row0 + nrows - 1) / p.group;
  const int begin = chunk_low(p, at0), end = chunk_high(p, at1, seq.kv_len);
  const int32_t* table = p.page_table + static_cast<int64_t>(b) * p.max_pages;
  __syncthreads();  // the rows before are done with the shared memory
  if (tid == 0) sm.bad = 0;
  __syncthreads();
  for (int pg = begin / p.page_size + tid; pg <= (end - 1) / p.page_size; pg += NT) {
    const int id = table[pg];
    if (id < 0 || id >= p.num_pages) sm.bad = 1;
  }
  const __nv_bfloat16* qg = static_cast<const __nv_bfloat16*>(p.q);
  for (int i = tid; i < RT * D; i += NT) {
    const int r = i / D, d = i % D, row = row0 + r;
    float x = 0.f;
    if (r < nrows)
      x = __bfloat162float(qg[(seq.row0 + row / p.group) * p.q_stride + static_cast<int64_t>(g * p.group + row % p.group) * D + d]);
    sm.q[r][d] = x;
  }
  if (tid < RT) {
    const int at = ctx + (row0 + tid) / p.group;
    sm.low[tid] = chunk_low(p, at);
    sm.high[tid] = tid < nrows ? chunk_high(p, at, seq.kv_len) : 0;
    sm.m[tid] = -INFINITY;
    sm.l[tid] = 0.f;
  }
  __syncthreads();
  if (sm.bad) {  // the whole sequence is cleared at the end
    if (tid == 0) {
      p.seq_bad[b] = 1;
      set_status(p.status, SPEC_FLAG_BAD_PAGE);
    }
    return;
  }

  // P V: a thread owns 8 consecutive dims of rows rg, rg + RG, ...
  constexpr int DQ = D / 8, RG = NT / DQ, RPT = RT / RG;
  const int dq = tid % DQ, rg = tid / DQ;
  float o[RPT][8];
#pragma unroll
  for (int i = 0; i < RPT; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) o[i][e] = 0.f;

  constexpr int RS = NT / TK;              // Q K^T: key kk, rows hr, hr + RS, ...
  const int kk = tid % TK, hr = tid / TK;
  for (int t0 = begin / TK * TK; t0 < end; t0 += TK) {
    constexpr int kPieces = D / 8;  // 8 elements
    for (int c = tid; c < 2 * TK * kPieces; c += NT) {
      const int kind = c / (TK * kPieces), key = (c / kPieces) % TK, piece = c % kPieces, pos = t0 + key;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.f;
      if (pos >= begin && pos < end) {
        const int64_t ph = static_cast<int64_t>(table[pos / p.page_size]) * p.hkv + g;
        if constexpr (FP8) {
          const uint2 raw = __ldg(reinterpret_cast<const uint2*>(
              static_cast<const uint8_t*>(p.k_cache) + ((ph * 2 + kind) * p.page_size + pos % p.page_size) * D + piece * 8));
          float sc = p.kv_scale[ph * 2 + kind];
          if (kind) sc = clamp_scale(sc);
          const uint32_t w[2] = {raw.x, raw.y};
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float2 a = from_e4m3x2(w[e] & 0xffffu), c2 = from_e4m3x2(w[e] >> 16);
            x[4 * e] = a.x * sc; x[4 * e + 1] = a.y * sc; x[4 * e + 2] = c2.x * sc; x[4 * e + 3] = c2.y * sc;
          }
        } else {
          const uint4 raw = __ldg(reinterpret_cast<const uint4*>(
              static_cast<const __nv_bfloat16*>(kind ? p.v_cache : p.k_cache) + (ph * p.page_size + pos % p.page_size) * D + piece * 8));
          const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
          }
        }
      }
      float* dst = (kind ? sm.v[key] : sm.k[key]) + piece * 8;
      *reinterpret_cast<float4*>(dst) = make_float4(x[0], x[1], x[2], x[3]);
      *reinterpret_cast<float4*>(dst + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
    __syncthreads();
    {
      float acc[RT / RS];
#pragma unroll
      for (int i = 0; i < RT / RS; ++i) acc[i] = 0.f;
#pragma unroll 4
      for (int d = 0; d < D; d += 4) {
        const float4 kf = *reinterpret_cast<const float4*>(&sm.k[kk][d]);
#pragma unroll
        for (int i = 0; i < RT / RS; ++i) {
          const float4 q = *reinterpret_cast<const float4*>(&sm.q[hr + RS * i][d]);
          acc[i] += q.x * kf.x + q.y * kf.y + q.z * kf.z + q.w * kf.w;
        }
      }
#pragma unroll
      for (int i = 0; i < RT / RS; ++i) {
        const int r = hr + RS * i;
        const bool vis = t0 + kk >= sm.low[r] && t0 + kk < sm.high[r];
        sm.s[r][kk] = vis ? acc[i] * p.scale_log2 : -INFINITY;
      }
    }
    __syncthreads();
    for (int r = warp; r < RT; r += NT / 32) {
      const float a0 = lane < TK ? sm.s[r][lane] : -INFINITY, a1 = lane + 32 < TK ? sm.s[r][lane + 32] : -INFINITY;
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
      // weights of keys that the row does not see are marked: what it sees adds 0 * value where a weight underflows
      const int from = sm.low[r] - t0, to = sm.high[r] - t0;
      __syncwarp();
      if (lane < TK) sm.s[r][lane] = lane >= from && lane < to ? p0 : -1.f;
      if (lane + 32 < TK) sm.s[r][lane + 32] = lane + 32 >= from && lane + 32 < to ? p1 : -1.f;
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
        if (w < 0.f) continue;  // a hidden key adds nothing, whatever its value
        o[i][0] += w * v0.x; o[i][1] += w * v0.y; o[i][2] += w * v0.z; o[i][3] += w * v0.w;
        o[i][4] += w * v1.x; o[i][5] += w * v1.y; o[i][6] += w * v1.z; o[i][7] += w * v1.w;
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = rg + i * RG, row = row0 + r;
    if (r >= nrows) continue;
    const float inv = 1.f / sm.l[r];  // every row sees a key: a sum of 0 (scores of -inf) is NaN
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 pr = __floats2bfloat162_rn(o[i][2 * e] * inv, o[i][2 * e + 1] * inv);
      w[e] = *reinterpret_cast<const uint32_t*>(&pr);
    }
    const int64_t head = static_cast<int64_t>(seq.row0 + row / p.group) * p.hq + g * p.group + row % p.group;
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + head * D + dq * 8) = make_uint4(w[0], w[1], w[2], w[3]);
    if (dq == 0 && p.lse) p.lse[head] = (sm.m[r] + log2f(sm.l[r])) * 0.6931471805599453f;
  }
}

// A block owns 16 query rows of a sequence and KV head, found by its place in the prefix sums of the
// set-up (row_start itself need not rise where sequences are left out).
template <int D, bool FP8>
__global__ void __launch_bounds__(NT) chunk_simt_kernel(ChunkParams p) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Smem<D, kSimtKeyTile>& sm = *reinterpret_cast<Smem<D, kSimtKeyTile>*>(smem_raw);
  pdl_wait_prior();
  const int unit = blockIdx.x;
  if (unit >= p.seqs[p.batch].first_unit) return;
  int lo = 0, hi = p.batch;  // the largest b with first_unit <= unit
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.seqs[mid].first_unit <= unit) lo = mid; else hi = mid;
  }
  const ChunkSeq seq = p.seqs[lo];
  const int row0 = (unit - seq.first_unit) * RT, nrows = min(RT, seq.n * p.group - row0);
  if (nrows > 0) simt_rows<D, FP8>(p, sm, lo, seq, blockIdx.y, row0, nrows);
}

// The end of a call: joins the parts of units that blocks split, computes again the units in
// which a hidden value was not finite (on CUDA cores, 16 keys at a time so that the shared memory
// of a block is small), and clears the rows of sequences that could not be served. A block splits
// two units at most, so the parts, twice 128 KB of fp32 per block, are a few us of L2 traffic, spread
// over eight blocks for each joined unit.
constexpr int kFinishThreads = NT;
constexpr int kFinishParts = 8;  // blocks per joined unit
constexpr int kRedoKeys = 16;

// The block of the work list that owns virtual step t.
__device__ __forceinline__ int owner_of(long long t, long long total, int blocks) {
  return static_cast<int>(((t + 1) * blocks - 1) / total);
}

// A unit that ends in block c's first stop, having begun in an earlier block. One that is computed again
// is not joined: other blocks write its rows meanwhile.
template <int D>
__device__ __forceinline__ void join_unit(const ChunkParams& p, int c, int part, int redo) {
  ChunkWalk w;
  if (!w.begin(p, c) || w.starts_unit() || p.seq_bad[w.b] != 0) return;
  const ChunkUnit u = w.unit(p);
  if (!w.ends_unit(u)) return;
  if (redo > 0) {
    bool again = false;
    for (int i = threadIdx.x; i < redo; i += kFinishThreads) {
      const int4 e = __ldcg(&p.redo[1 + i]);
      again |= e.x == w.b && e.y == w.g && e.z == w.rt;
    }
    if (__syncthreads_or(again)) return;
  }
  const long long total = p.work->total;
  const int active = p.work->active;
  // the unit's first step, from this block's first virtual one
  const long long at = c * total / active - p.work->starts[c].off + u.start();
  const int first = owner_of(at, total, active), subs = u.twin ? 2 : 1, n = (c - first + 1) * subs;
  const int tile_rows = p.tile_tokens * p.group;
  constexpr int C8 = D / 8;
  const int rows = u.twin ? kChunkTileRows : 2 * kChunkTileRows;
  // a warp takes 8 rows x 32 columns, a thread 8 columns of a row
  const int lane = threadIdx.x & 31;
  for (int x = part * (kFinishThreads / 32) + (threadIdx.x >> 5); x < rows / 8 * (C8 / 4); x += kFinishParts * (kFinishThreads / 32)) {
    const int r = x / (C8 / 4) * 8 + (lane & 7), c8 = x % (C8 / 4) * 4 + (lane >> 3), tr = r & (kChunkTileRows - 1);
    const int token = (r >= kChunkTileRows ? p.tile_tokens : 0) + tr / p.group;
    if (tr >= tile_rows || token >= u.tokens) continue;
    float M = -INFINITY, L = 0.f, acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    constexpr int SB = 3;  // parts whose loads are in flight together
    for (int s0 = 0; s0 < n; s0 += SB) {
      float2 ml[SB];
      float4 lo[SB], hi[SB];
#pragma unroll
      for (int k = 0; k < SB; ++k) {
        ml[k] = make_float2(-INFINITY, 0.f);
        if (s0 + k < n) {
          const int cta = first + (s0 + k) / subs, sub = (s0 + k) % subs;
          const int64_t slot = 2 * static_cast<int64_t>(cta) + (cta == first ? 1 : 0);
          const int row = sub * kChunkTileRows + r;
          ml[k] = __ldcg(&p.partial_ml[slot * (2 * kChunkTileRows) + row]);
          const float4* src = reinterpret_cast<const float4*>(p.partial_o) + (slot * (D / 4) + 2 * c8) * (2 * kChunkTileRows) + row;
          lo[k] = __ldcg(src);
          hi[k] = __ldcg(src + 2 * kChunkTileRows);
        }
      }
#pragma unroll
      for (int k = 0; k < SB; ++k) {
        // saw no key (one whose scores are all NaN has no maximum either, but a sum)
        if (s0 + k >= n || (ml[k].x == -INFINITY && ml[k].y == 0.f)) continue;
        const float m = fmaxf(M, ml[k].x);
        const float old = M == -INFINITY ? 0.f : ex2(M - m), x = ex2(ml[k].x - m);
        const float v[8] = {lo[k].x, lo[k].y, lo[k].z, lo[k].w, hi[k].x, hi[k].y, hi[k].z, hi[k].w};
        L = L * old + ml[k].y * x;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = acc[e] * old + v[e] * x;
        M = m;
      }
    }
    const float inv = 1.f / L;
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 pr = __floats2bfloat162_rn(acc[2 * e] * inv, acc[2 * e + 1] * inv);
      o[e] = *reinterpret_cast<const uint32_t*>(&pr);
    }
    const int64_t head = static_cast<int64_t>(w.row0 + u.token0 + token) * p.hq + w.g * p.group + tr % p.group;
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + head * D + c8 * 8) = make_uint4(o[0], o[1], o[2], o[3]);
    if (c8 == 0 && p.lse) p.lse[head] = (M + log2f(L)) * 0.6931471805599453f;
  }
}

template <int D, bool FP8>
__global__ void __launch_bounds__(kFinishThreads) chunk_finish_kernel(ChunkParams p) {
  __shared__ Smem<D, kRedoKeys> sm;
  pdl_wait_prior();
  if (p.blocks) {
    const int redo = min(__ldcg(&p.redo[0].x), p.redo_cap);
    if (blockIdx.x > 0 && static_cast<int>(blockIdx.x) < p.blocks) join_unit<D>(p, blockIdx.x, blockIdx.y, redo);
    if (redo > 0) {
      const int tiles = (2 * p.tile_tokens * p.group + RT - 1) / RT;
      for (int64_t i = static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x; i < static_cast<int64_t>(redo) * tiles;
           i += static_cast<int64_t>(gridDim.x) * gridDim.y) {
        const int4 e = __ldcg(&p.redo[1 + i / tiles]);
        const ChunkSeq seq = p.seqs[e.x];
        const ChunkUnit u = chunk_unit(p, seq, e.z);
        const int row = static_cast<int>(i % tiles) * RT, nrows = min(RT, u.tokens * p.group - row);
        if (nrows > 0 && p.seq_bad[e.x] == 0) simt_rows<D, FP8>(p, sm, e.x, seq, e.y, u.token0 * p.group + row, nrows);
      }
    }
  }
  for (int b = blockIdx.y * gridDim.x + blockIdx.x; b < p.batch; b += gridDim.x * gridDim.y) {
    if (p.seq_bad[b] == 0) continue;
    const int r0 = p.row_start[b], r1 = p.row_start[b + 1];
    if (!chunk_rows_ok(p, r0, r1)) continue;  // there are none to clear
    const int64_t heads = static_cast<int64_t>(r1 - r0) * p.hq;
    uint4* out = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + static_cast<int64_t>(r0) * p.hq * D);
    for (int64_t i = threadIdx.x; i < heads * (D / 8); i += kFinishThreads) out[i] = make_uint4(0, 0, 0, 0);
    if (p.lse)
      for (int64_t i = threadIdx.x; i < heads; i += kFinishThreads) p.lse[static_cast<int64_t>(r0) * p.hq + i] = -INFINITY;
  }
}

template <int D, bool FP8>
cudaError_t launch_simt_d(const ChunkParams& p, cudaStream_t stream) {
  const size_t smem = sizeof(Smem<D, kSimtKeyTile>);
  const cudaError_t e = cudaFuncSetAttribute(chunk_simt_kernel<D, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  return launch_overlapped(chunk_simt_kernel<D, FP8>, dim3(p.max_units, p.hkv), NT, smem, stream, p);
}

template <int D, bool FP8>
cudaError_t launch_finish_d(const ChunkParams& p, cudaStream_t stream) {
  const dim3 grid = p.blocks ? dim3(p.blocks, kFinishParts) : dim3(p.batch < 256 ? p.batch : 256);
  return launch_overlapped(chunk_finish_kernel<D, FP8>, grid, kFinishThreads, 0, stream, p);
}

template <int THREADS>
cudaError_t launch_setup(const spec_chunk_attn_args_t& a, const ChunkPlan& P, const ChunkParams& p, cudaStream_t stream) {
  if (!p.blocks || !P.fp8) return launch_overlapped(chunk_setup_kernel<0, THREADS>, dim3(1), THREADS, 0, stream, p);
  const int64_t heads = static_cast<int64_t>(a.rows) * a.num_q_heads;
  const int each = THREADS / (a.head_dim / 8), most = 2 * P.grid * (kSetupThreads / THREADS);  // as many fit the SMs
  const int extra = static_cast<int>(heads / each < most ? (heads + each - 1) / each : most);
  return launch_overlapped(a.head_dim == 128 ? chunk_setup_kernel<128, THREADS> : chunk_setup_kernel<64, THREADS>,
                           dim3(1 + extra), THREADS, 0, stream, p);
}

ChunkParams make_chunk_params(const spec_chunk_attn_args_t& a, const ChunkPlan& P, char* ws) {
  ChunkParams p{};
  p.batch = a.batch;
  p.rows = a.rows;
  p.hq = a.num_q_heads;
  p.hkv = a.num_kv_heads;
  p.group = a.num_q_heads / a.num_kv_heads;
  p.page_size = a.page_size;
  p.max_pages = a.max_pages_per_seq;
  p.num_pages = a.num_pages;
  p.max_keys = a.max_pages_per_seq * a.page_size;
  p.causal = a.causal;
  p.window = a.window;
  const float scale = a.softmax_scale != 0.f ? a.softmax_scale : 1.f / sqrtf(static_cast<float>(a.head_dim));
  p.scale_log2 = scale * kLog2e;
  p.q_stride = a.q_row_stride ? a.q_row_stride : static_cast<int64_t>(a.num_q_heads) * a.head_dim;
  p.q = a.q;
  p.k_cache = P.fp8 ? a.kv_cache : a.k_cache;
  p.v_cache = a.v_cache;
  p.kv_scale = a.kv_scale;
  p.page_table = a.page_table;
  p.row_start = a.row_start;
  p.kv_len = a.kv_len;
  p.out = a.out;
  p.lse = a.lse;
  p.status = reinterpret_cast<uint32_t*>(ws);
  p.seqs = reinterpret_cast<ChunkSeq*>(ws + P.seqs);
  p.seq_bad = reinterpret_cast<int32_t*>(ws + P.bad);
  p.max_units = P.max_units;
  if (P.path == SPEC_ATTN_TENSOR_CORES) {
    p.tile_tokens = P.tile_tokens;
    p.blocks = P.grid;
    p.cum = reinterpret_cast<long long*>(ws + P.cum);
    p.work = reinterpret_cast<ChunkWork*>(ws + P.work);
    p.redo = reinterpret_cast<int4*>(ws + P.redo);
    p.redo_cap = P.redo_cap;
    p.partial_o = reinterpret_cast<float*>(ws + P.partial_o);
    p.partial_ml = reinterpret_cast<float2*>(ws + P.partial_ml);
    p.q_half = ws + P.q_half;
    p.q_scale = reinterpret_cast<float*>(ws + P.q_scale);
  }
  return p;
}

}  // namespace

cudaError_t launch_chunk(const spec_chunk_attn_args_t& a, const ChunkPlan& P, char* ws, cudaStream_t stream,
                         bool starve) {
  ChunkParams p = make_chunk_params(a, P, ws);
  p.starve = starve ? 1 : 0;
  const bool wide = a.head_dim == 128;
  cudaError_t e = a.batch <= kSetupFew && (!p.blocks || p.max_units <= kSetupFew) ? launch_setup<kSetupFew>(a, P, p, stream)
                                                                                : launch_setup<kSetupThreads>(a, P, p, stream);
  if (e != cudaSuccess) return e;
  if (p.blocks) e = launch_chunk_tc(a, p, stream);
  else if (P.fp8) e = wide ? launch_simt_d<128, true>(p, stream) : launch_simt_d<64, true>(p, stream);
  else e = wide ? launch_simt_d<128, false>(p, stream) : launch_simt_d<64, false>(p, stream);
  if (e != cudaSuccess) return e;
  if (P.fp8) return wide ? launch_finish_d<128, true>(p, stream) : launch_finish_d<64, true>(p, stream);
  return wide ? launch_finish_d<128, false>(p, stream) : launch_finish_d<64, false>(p, stream);
}

}  // namespace specv
