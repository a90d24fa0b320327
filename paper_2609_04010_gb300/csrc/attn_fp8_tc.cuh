// What the two tensor-core kernels of the attention over the 8-bit cache share: PTX wrappers
// for 8-bit products, the staging of keys and values, the work list, and the end of a block.
#pragma once

#include <cuda.h>  // CUtensorMap

#include "attn_fp8.cuh"
#include "tc_ptx.cuh"

namespace specv {
namespace fp8tc {

using namespace tcx;

constexpr int TK = kFp8KeyTile;  // keys per tile
constexpr int NH = 2;            // sub-units of a block
constexpr int kFlagRing = 16;    // segments' flags: more than the stages that producers run ahead

// A stage holds a tile of 128 keys: K and V of HP KV heads as [8-key group][head, K or V]
// [8 keys][D bytes], each atom of 8 rows swizzled by the width of a row.
template <int D, int HP>
struct Stage {
  static constexpr uint32_t ATOM = 8 * D;
  static constexpr uint32_t SG = 2 * HP * ATOM;  // an 8-key group
  static constexpr uint32_t BYTES = (TK / 8) * SG;
};

__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// One page of HP KV heads, keys and values (encode_fp8_map's box).
__device__ __forceinline__ void tma_load_page8(uint32_t dst, const CUtensorMap* map, int kind_head, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(0), "r"(kind_head), "r"(0), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Matrix descriptor of a tile whose rows are W bytes (128, 64 or 32) with the W-byte swizzle.
template <int W>
__device__ __forceinline__ uint64_t desc_rows(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>((lbo >> 4) & 0x3FFFu) << 16) |
         (static_cast<uint64_t>((sbo >> 4) & 0x3FFFu) << 32) | (1ull << 46) |
         (static_cast<uint64_t>(W == 128 ? 2 : W == 64 ? 4 : 6) << 61);
}
// Instruction descriptor, kind::f8f6f4: fp32 accumulator, A and B e4m3 or e5m2.
__host__ __device__ constexpr uint32_t idesc_f8(int M, int N, bool a_mn, bool b_mn, bool a_e5m2 = false,
                                                bool b_e5m2 = false) {
  return (1u << 4) | ((a_e5m2 ? 1u : 0u) << 7) | ((b_e5m2 ? 1u : 0u) << 10) | ((a_mn ? 1u : 0u) << 15) |
         ((b_mn ? 1u : 0u) << 16) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void bar_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// The two e4m3 terms of four values, each packed in order from the low byte.
__device__ __forceinline__ void split_e4m3x4(float a, float b, float c, float d, uint32_t& hi, uint32_t& lo) {
  uint32_t x, y;
  asm("{\n .reg .b16 p, q;\n .reg .b32 h, g;\n"
      " cvt.rn.satfinite.e4m3x2.f32 p, %4, %3;\n cvt.rn.satfinite.e4m3x2.f32 q, %6, %5;\n mov.b32 %0, {p, q};\n"
      " cvt.rn.f16x2.f32 %1, %4, %3;\n cvt.rn.f16x2.f32 %2, %6, %5;\n"
      " cvt.rn.f16x2.e4m3x2 h, p;\n cvt.rn.f16x2.e4m3x2 g, q;\n"
      " sub.f16x2 %1, %1, h;\n sub.f16x2 %2, %2, g;\n}"
      : "=&r"(hi), "=&r"(x), "=&r"(y)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  asm("{\n .reg .b16 r, s;\n cvt.rn.satfinite.e4m3x2.f16x2 r, %1;\n cvt.rn.satfinite.e4m3x2.f16x2 s, %2;\n"
      " mov.b32 %0, {r, s};\n}"
      : "=r"(lo)
      : "r"(x), "r"(y));
}

// The three e5m2 terms of four weights in [0, 2^15] (2^16 where scores are so large that their steps
// are 16, taken as 65504), each packed in order from the low byte. A
// weight is rounded to fp16, whose upper byte is an e5m2 number: that byte, the upper byte of
// what is left of it, and what is left then, rounded, are the terms: 3 + 3 + 3 bits, off by at most
// 2^-9 + 2^-11 of the weight. UP: the third terms times 32, so that their smallest step is 2^-21 of 1
// instead of 2^-16 (they stay below 2^16).
template <bool UP>
__device__ __forceinline__ void split_weights(const float* p, uint32_t& w1, uint32_t& w2, uint32_t& w3) {
  uint32_t x, y, r, s;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %2, %1;" : "=r"(x) : "f"(p[0]), "f"(p[1]));
  asm("cvt.rn.satfinite.f16x2.f32 %0, %2, %1;" : "=r"(y) : "f"(p[2]), "f"(p[3]));
  w1 = __byte_perm(x, y, 0x7531);
  asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(x & 0xff00ff00u));
  asm("sub.f16x2 %0, %1, %2;" : "=r"(s) : "r"(y), "r"(y & 0xff00ff00u));
  w2 = __byte_perm(r, s, 0x7531);
  asm("sub.f16x2 %0, %1, %2;" : "=r"(x) : "r"(r), "r"(r & 0xff00ff00u));
  asm("sub.f16x2 %0, %1, %2;" : "=r"(y) : "r"(s), "r"(s & 0xff00ff00u));
  if constexpr (UP) asm("mul.f16x2 %0, %0, %2;\n mul.f16x2 %1, %1, %2;" : "+r"(x), "+r"(y) : "r"(0x50005000u));
  asm("{\n .reg .b16 p, q;\n cvt.rn.satfinite.e5m2x2.f16x2 p, %1;\n cvt.rn.satfinite.e5m2x2.f16x2 q, %2;\n"
      " mov.b32 %0, {p, q};\n}"
      : "=r"(w3)
      : "r"(x), "r"(y));
}

// The slow part of a wait: polls until the phase completes, or gives up (mbar_wait).
static __device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t* status) {
  return mbar_wait(bar, parity, abort_flag, status);
}

#ifdef __CUDACC__
// ---------------------------------------------------------------------------------
// The work list: the tiles of all units, cut into equal ranges, one per block
// ---------------------------------------------------------------------------------
// First tiles are kept of each EACH-th sequence, 1 or 2: that of a sequence in between follows from
// the lengths that find() reads anyway, and half the entries leave shared memory for a stage.
template <int EACH>
__host__ __device__ constexpr int list_entries(int batch) { return (batch + EACH - 1) / EACH + 1; }

template <int EACH>
struct WorkList {
  int64_t t0, t1, total;  // this block's range, and the list's length
  const int* pb;          // [list_entries<EACH>(batch)]: first tiles, and the total
  int ovh, ctas, cta;
};

__device__ __forceinline__ int sequence_tiles(int kv_len, const AttnParams& p) {
  return (unit_tiles<TK>(kv_len, p) + p.unit_overhead) * p.hunits * p.row_tiles;
}
// First tiles of the sequences (one warp).
template <int EACH>
__device__ __forceinline__ void prefix_tiles(const AttnParams& p, int* pb) {
  const int lane = threadIdx.x & 31;
  int carry = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    const int b = b0 + lane;
    int v = b < p.batch ? sequence_tiles(p.kv_len[b], p) : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += y;
    }
    if (b < p.batch && ((b + 1) % EACH == 0 || b + 1 == p.batch)) pb[b / EACH + 1] = carry + v;
    carry += __shfl_sync(0xffffffffu, v, 31);
  }
  if (lane == 0) pb[0] = 0;
}

// Equal ranges on every SM (a multiple of the units, so that equal units have no boundary
// inside a range, measured slower before units were joined over all SMs: 135.8 against 123.2 us
// with 128 ragged units, 232 against 226 with 64 equal ones).
template <int EACH>
__device__ __forceinline__ WorkList<EACH> work_list(const AttnParams& p, const int* pb) {
  WorkList<EACH> w;
  w.pb = pb;
  w.ovh = p.unit_overhead;
  w.total = pb[list_entries<EACH>(p.batch) - 1];
  w.ctas = static_cast<int>(w.total < gridDim.x ? w.total : gridDim.x);
  w.cta = blockIdx.x;
  w.t0 = w.cta < w.ctas ? static_cast<int64_t>(w.cta) * w.total / w.ctas : 0;
  w.t1 = w.cta < w.ctas ? static_cast<int64_t>(w.cta + 1) * w.total / w.ctas : 0;
  return w;
}

// locate() in 32 bits (a list has at most INT32_MAX tiles).
template <int EACH>
__device__ __forceinline__ Seg find(int64_t at, const WorkList<EACH>& w, const AttnParams& p) {
  const int v = static_cast<int>(at), v1 = static_cast<int>(w.t1);
  int lo = 0, hi = list_entries<EACH>(p.batch) - 1;  // largest entry with pb[lo] <= v
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (w.pb[mid] <= v) lo = mid; else hi = mid;
  }
  int rem = v - w.pb[lo];  // tiles from the sequence's first
  Seg s;
  s.b = EACH * lo;
  s.kv_len = p.kv_len[s.b];
  if constexpr (EACH == 2) {
    const int next_len = s.b + 1 < p.batch ? p.kv_len[s.b + 1] : 0, tiles = sequence_tiles(s.kv_len, p);
    if (rem >= tiles) {
      rem -= tiles;
      ++s.b;
      s.kv_len = next_len;
    }
  }
  s.len_ok = s.kv_len >= p.gamma && s.kv_len <= p.max_keys;
  s.unit_tiles = unit_tiles<TK>(s.kv_len, p);
  const uint32_t vlen = s.unit_tiles + w.ovh, ub = static_cast<uint32_t>(rem) / vlen;
  const int real = v - static_cast<int>(rem - ub * vlen) + w.ovh;  // the unit's first real tile
  s.g = p.row_tiles == 1 ? ub : ub / p.row_tiles;
  s.rt = p.row_tiles == 1 ? 0 : ub - s.g * p.row_tiles;
  s.u = static_cast<int64_t>(s.b) * p.hunits * p.row_tiles + ub;
  s.unit_start = real;
  const int next = min(real + s.unit_tiles, v1), from = max(v, real);
  s.vnext = next;
  s.ntile = max(next - from, 0);
  s.tile0 = s.ntile > 0 ? from - real : 0;
  return s;
}

// Where block `cta` keeps its part of a split unit: the part that starts the unit is its last
// segment, one that goes on with a unit its first.
__device__ __forceinline__ int part_slot(int cta, bool starts) { return 2 * cta + (starts ? 1 : 0); }

// What merge_fp8_kernel is to join: units split between blocks, noted by the block with their
// last tiles. With at most as many units as blocks each unit has a place; otherwise each
// block, because only its first segment can end a split unit, and clear_split cleans it first.
__device__ __forceinline__ void clear_split(const AttnFp8Params& p) {
  if (!p.split_by_unit) p.splits[2 * blockIdx.x + 1] = make_int4(0, 0, 0, 0);
}
template <int EACH>
__device__ __forceinline__ void note_split(const AttnFp8Params& p, const Seg& s, const WorkList<EACH>& w, int tile_rows) {
  const bool split = s.tile0 > 0;
  if (s.tile0 + s.ntile != s.unit_tiles || (!split && !p.split_by_unit)) return;
  const int first = split ? owner_of(s.unit_start, w.total, w.ctas) : 0, row0 = s.rt * tile_rows;
  int4* e = p.splits + 2 * (p.split_by_unit ? s.u : blockIdx.x);
  e[0] = make_int4(s.b, s.g, row0, min(tile_rows, p.rows - row0));
  e[1] = make_int4(first, split ? w.cta - first + 1 : 0, 0, 0);
}

// Joins the parts of split units: grid (chunks of a unit's outputs, places of units). A warp
// takes 8 rows x 32 columns, a thread 8 columns of a row. Small blocks start sooner: trees of 31
// for 8 requests take 44.0 us, 44.5 with 256 threads a block. (The last block
// to finish a unit merging it alone took 12 to 15 us at the end of a call where this takes 4 to
// 6: 128 rows in 5 parts are 330 KB, an L2 round trip of one SM at a time.)
constexpr int kMergeThreads = 128;
template <int D, int HP, bool BY_COLUMNS>
__global__ void __launch_bounds__(kMergeThreads) merge_fp8_kernel(AttnFp8Params p) {
  pdl_wait_prior();
  const int4 a = __ldcg(p.splits + 2 * blockIdx.y), b = __ldcg(p.splits + 2 * blockIdx.y + 1);
  // (after a timeout a place may hold anything)
  if (b.y <= 0 || b.x < 0 || b.y > p.blocks - b.x || a.x < 0 || a.x >= p.batch || a.y < 0 || a.y >= p.hunits ||
      a.z < 0 || a.w < 0 || a.w > p.slot_rows / HP || a.w > p.rows - a.z)
    return;
  const int warp = blockIdx.x * (kMergeThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int hr = warp / (D / 32) * 8 + (lane & 7), c8 = warp % (D / 32) * 4 + (lane >> 3);
  if (hr < HP * a.w)
    merge_fp8_item<D, BY_COLUMNS>(p, a.x, a.y * HP + hr / a.w, a.z + hr % a.w,
                                  [&](int i) { return part_slot(b.x + i, i == 0); }, b.y, hr, c8);
}

template <int D, int HP, bool BY_COLUMNS>
cudaError_t launch_merge(const AttnFp8Params& p, const AttnFp8Plan& P, cudaStream_t stream) {
  const int warps = (P.slot_rows + 7) / 8 * (D / 32);
  const dim3 grid((warps + kMergeThreads / 32 - 1) / (kMergeThreads / 32), P.splits);
  return launch_overlapped(merge_fp8_kernel<D, HP, BY_COLUMNS>, grid, kMergeThreads, 0, stream, p);
}

// ---------------------------------------------------------------------------------
// Staging
// ---------------------------------------------------------------------------------
// A producer warp: the half of each tile's pages, one TMA box each, and their scales as
// scl[stage][page of the tile][head] = (sk * softmax scale * log2(e), log2(sv), 1 / sv, -).
// Two of them, because one keeps the copy engine waiting.
template <int D, int HP, int NST, int EACH>
__device__ __forceinline__ void produce(const AttnFp8Params& p, const CUtensorMap& tmap, const WorkList<EACH>& w, int half,
                                        uint32_t stages, uint32_t full, uint32_t empty, uint32_t flag_ready,
                                        float4* scl, volatile int* seg_flag, volatile int* abort_flag) {
  const int lane = threadIdx.x & 31;
  uint32_t it = 0, seg_no = 0;
  bool ok = true;
  const int psh = __ffs(p.page_size) - 1;  // log2
  const int npg = TK >> psh;               // pages of a tile
  const uint32_t box_bytes = static_cast<uint32_t>(p.page_size) * D * 2 * HP;
  for (Seg s = find(w.t0, w, p); s.ntile > 0 && ok && !p.starve; ++seg_no) {
    const bool bad_len = !s.len_ok;
    bool flag = bad_len;
    // Pages are taken 32 at a time, a lane each; the next 32 ids and scales are loaded
    // while these are in use, the ids of the 32 after them too.
    const int pages = bad_len ? 0 : (s.kv_len + p.page_size - 1) >> psh;
    const int first = s.tile0 * npg;
    const int32_t* table = p.page_table + static_cast<int64_t>(s.b) * p.max_pages;
    auto load_id = [&](int base) { return base + lane < pages ? __ldg(table + base + lane) : 0; };
    auto load_scale = [&](int id, float2* sc) {
      const bool in = id >= 0 && id < p.num_pages;
      const float2* src = reinterpret_cast<const float2*>(p.kv_scale) +
                          static_cast<int64_t>(in ? id : 0) * p.hkv + s.g * HP;
#pragma unroll
      for (int h = 0; h < HP; ++h) sc[h] = __ldg(src + h);
    };
    int base = first, id = load_id(first), id1 = load_id(first + 32), id2 = load_id(first + 64);
    float2 sc[HP], sc1[HP];
    load_scale(id, sc);
    load_scale(id1, sc1);
    for (int k = 0; k < s.ntile && ok; ++k, ++it) {
      const uint32_t st = it % NST;
      const int pg0 = first + k * npg;
      if (pg0 >= base + 32) {
        base += 32;
        id = id1;
        id1 = id2;
#pragma unroll
        for (int h = 0; h < HP; ++h) sc[h] = sc1[h];
        load_scale(id1, sc1);
        id2 = load_id(base + 64);
      }
      if (it >= NST) ok = mbar_wait(empty + 8u * st, ((it / NST) - 1) & 1, abort_flag, p.status);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      // lanes [pg0 - base, + npg) hold this tile's pages; this warp copies the half
      // [q0, q1) of them
      const int q0 = half * (npg >> 1), q1 = min(q0 + (npg >> 1), pages - pg0);
      const uint32_t dst = stages + st * Stage<D, HP>::BYTES;
      if (lane == 0 && q1 > q0) mbar_expect_tx(full + 8u * st, static_cast<uint32_t>(q1 - q0) * box_bytes);
      for (int q = q0; q < q1; ++q) {
        const int raw = __shfl_sync(0xffffffffu, id, pg0 - base + q);
        const bool in_range = raw >= 0 && raw < p.num_pages;
        flag |= !in_range;
        if (lane == 0)
          tma_load_page8(dst + static_cast<uint32_t>(q) * box_bytes, &tmap,
                         2 * ((in_range ? raw : 0) * p.hkv + s.g * HP), full + 8u * st);
      }
      const int q = base + lane - pg0;
      if (q >= q0 && q < q0 + (npg >> 1)) {
#pragma unroll
        for (int h = 0; h < HP; ++h) {
          const float sv = clamp_scale(sc[h].y);
          scl[(st * 8 + q) * HP + h] = q < q1 ? make_float4(sc[h].x * p.scale_log2, __log2f(sv), __frcp_rn(sv), 0.f)
                                              : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(full + 8u * st);
      __syncwarp();
    }
    if (ok && lane == 0) {
      seg_flag[half * kFlagRing + seg_no % kFlagRing] = flag ? 1 : 0;
      mbar_arrive(flag_ready + 8u * (seg_no % kFlagRing));
    }
    if (!has_more(s, w.t1, w.ovh)) break;
    s = find(s.vnext, w, p);
  }
  if (!ok) {  // copies still in flight (bounded)
    for (uint32_t x = it > static_cast<uint32_t>(NST) ? it - NST : 0; x < it; ++x) {
      const long long c0 = clock64();
      while (!mbar_try(full + 8u * (x % NST), (x / NST) & 1) && clock64() - c0 < kWaitCycles) {
      }
    }
  }
}

// V of keys that no row sees must be finite, because their weight of 0 is multiplied: keys
// past the end are cleared, and a NaN in a block key's value is cleared and noted in
// nanv[sub-unit][D] (a bit per block key), for the outputs of the rows that see it.
template <int D, int HP>
__device__ __forceinline__ void fix_values(const AttnParams& p, const Seg& sg, int k, unsigned char* base,
                                           unsigned long long* nanv, volatile int* nan_flag) {
  const int key0 = (sg.tile0 + k) * TK;
  const int ctx = sg.kv_len - p.gamma;
  if (!sg.len_ok || key0 + TK <= ctx) return;
  const int nvalid = min(TK, sg.kv_len - key0);
  constexpr int kPieces = D / 16;
  const int lane = threadIdx.x & 31;
  const int from = max(0, ctx - key0);
  for (int i = lane; i < (TK - from) * kPieces * HP; i += 32) {
    const int piece = i % kPieces, h = (i / kPieces) % HP, key = from + i / (kPieces * HP);
    const int ph = D == 128 ? piece ^ (key & 7) : piece ^ ((key >> 1) & 3);
    uint4* at = reinterpret_cast<uint4*>(base + (key >> 3) * Stage<D, HP>::SG + (2 * h + 1) * Stage<D, HP>::ATOM + (key & 7) * D + ph * 16);
    if (key >= nvalid) {
      *at = make_uint4(0, 0, 0, 0);
      continue;
    }
    uint4 v = *at;
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t any = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) any |= __vcmpeq4(w[e] & 0x7f7f7f7fu, 0x7f7f7f7fu);
    if (any) {
      const unsigned long long bit = 1ull << (key0 + key - ctx);
      for (int e = 0; e < 16; ++e) {
        const uint32_t sh = (e & 3) * 8;
        if ((w[e >> 2] >> sh & 0x7fu) == 0x7fu) {
          atomicOr(nanv + h * D + piece * 16 + e, bit);
          if (HP == 1) atomicOr(nanv + D + piece * 16 + e, bit);
          w[e >> 2] &= ~(0xffu << sh);
        }
      }
      nan_flag[h] = 1;
      if (HP == 1) nan_flag[1] = 1;
      *at = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  fence_async_smem();
  __syncwarp();
}
#endif

// The tensor map of the cache: a box is one page of `heads` adjacent KV heads.
bool encode_fp8_map(CUtensorMap* map, const spec_attn_fp8_args_t& a, int heads);

}  // namespace fp8tc
}  // namespace specv
