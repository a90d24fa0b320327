// Attention of the block queries over the 8-bit KV cache on tcgen05 tensor cores
// (spec_verify_attention_fp8, SPEC_ATTN_TENSOR_CORES).
//
// Both products run in e4m3 straight from the cache's bytes, which land in shared memory by
// TMA in the layout that the MMAs read; nothing is decoded on the way. They are transposed,
// with the 128 keys (or the D dims) of a tile on the MMA's M side, so that the query rows are
// its N side and a group of few rows pays for few:
//   S^T[key][row]  = K8[key][:] . Q8[row][:]          (M = 128 keys, N = rows, K = D)
//   O^T[dim][row] += sum_key V8[key][dim] P8[key][row] (M = D, N = 2 * rows, K = 128 keys)
// What is exact in the cache must not be lost on the other side, so the bf16 queries and the
// fp32 weights enter as sums of two e4m3 terms (x1 = e4m3(x), x2 = e4m3(x - x1)): for a
// query that is exact to 2^-18 of its group's largest element, for a weight to 2^-8 of
// itself. Both terms of Q accumulate into the same S; those of P are the first and the
// second half of N and are added when a unit ends.
//
// With sk, sv the scales of a key's page, m_r the row's reference and the weights
//   P = 2^(s + log2(sv) - m_r),  s = sk * S^T * softmax_scale * log2(e),
// O^T accumulates the weighted values with their scales, and sum P / sv is the softmax sum.
// m_r is chosen so that 4 <= the row's largest P <= 256 and rises only when P would pass 256
// (e4m3 ends at 448), which after a unit's first tile is rare. The second term of P is kept
// times 16, which puts its smallest step at 2^-13.
//
// A block serves NH = 2 (or 1) sub-units of at most 64 query rows: two adjacent KV heads
// (HP = 2, one box brings K and V of both: 8 KB with 16-token pages and D = 128), or two
// row halves of one KV head. Warp roles (persistent, one block per SM):
//   warp 0       producer: page ids and scales 32 pages ahead, one TMA box per page
//   warp 1       issues S^T = K Q^T into a ring of four S buffers in TMEM
//   warp 3       issues O^T += V^T P^T; clears V of keys past the sequence's end
//   warps 4..    softmax: lane quadrant = 32 keys, NG warps per quadrant share the rows;
//                they also convert Q and write the outputs
// The tiles of all units form one list that is cut into equal ranges, one per block; a unit
// split between blocks is merged from fp32 partials by the last block to finish it (atomic
// ticket, no waiting). Every mbarrier wait is bounded; after a timeout the softmax warps run
// their loops to the end without waiting, so that none is missed at a named barrier.
#include <cuda.h>  // CUtensorMap

#include "attn_fp8.cuh"
#include "tc_ptx.cuh"

namespace specv {
namespace {

using namespace tcx;

constexpr int TK = kFp8KeyTile;  // keys per tile

// NR: query rows of a sub-unit (N of the first product), 16, 32 or 64.
template <int D, int HP, int NH, int NR>
struct Cfg {
  static_assert(HP <= NH, "two heads are two sub-units");
  static constexpr int NC = NR == 64 ? 16 : 8;             // rows per softmax warp
  static constexpr int NG = NR / NC;                       // softmax warps per lane quadrant
  static constexpr uint32_t ATOM = 8 * D;                  // 8 rows of D bytes, swizzled
  static constexpr uint32_t SG = 2 * HP * ATOM;            // 8-key group: K, V of each head
  static constexpr uint32_t STAGE = (TK / 8) * SG;
  static constexpr int NST = (HP == 2 ? 2 : 4) * (128 / D);  // 128 KB in stages
  static constexpr int PB = NH == 1 ? 2 : 1;               // P buffers per sub-unit
  static constexpr int SB = 4;                             // S buffers
  static constexpr uint32_t Q_TERM = NR * D;               // one term of one sub-unit's Q
  static constexpr uint32_t P_BUF = TK * 128;              // [key][128 B]: first terms, second terms
  static constexpr uint32_t OFF_STAGE = 0;
  static constexpr uint32_t OFF_P = OFF_STAGE + NST * STAGE;
  static constexpr uint32_t OFF_Q = OFF_P + NH * PB * P_BUF;
  static constexpr uint32_t OFF_SCL = OFF_Q + NH * 2 * Q_TERM;     // float4 [NST][8 pages][HP]
  static constexpr uint32_t OFF_NAN = OFF_SCL + NST * 8 * HP * 16;  // uint64 [HP][D]: NaN block values
  // of the current and the next segment: the block keys each row sees, the rows that see
  // each block key, the rows' references
  static constexpr uint32_t OFF_VIS = OFF_NAN + HP * D * 8;           // uint64 [2][NH][NR]
  static constexpr uint32_t OFF_SEEN = OFF_VIS + 2 * NH * NR * 8;     // uint32 [2][NH][NG][64]
  static constexpr uint32_t OFF_M = OFF_SEEN + 2 * NH * NG * 64 * 4;  // float [2][NH][NR]
  static constexpr uint32_t OFF_X = OFF_M + 2 * NH * NR * 4;          // float [NH][4][NR]: cross-quadrant
  static constexpr uint32_t OFF_ROW = OFF_X + NH * 4 * NR * 4;        // int64 [NH][NR]: rows' outputs
  static constexpr uint32_t OFF_INV = OFF_ROW + NH * NR * 8;          // float [NH][NR]: their factors
  static constexpr uint32_t OFF_BAR = OFF_INV + NH * NR * 4;
  // full[NST], empty[NST], s_full[SB], s_free[SB], p_full[NH*PB], pv_done[NH*PB], seg_ready,
  // drain[2], flag_ready[8]
  static constexpr int NBAR = 2 * NST + 2 * SB + 2 * NH * PB + 1 + 2 + 8;
  static constexpr uint32_t OFF_MISC = OFF_BAR + NBAR * 8;  // tmem base, abort, pending, NaN flag
  static constexpr uint32_t OFF_FLAG = OFF_MISC + 16;       // int [8]: bad flags of segments
  static constexpr uint32_t OFF_PEND = OFF_FLAG + 32;       // int [2][8]
  static constexpr uint32_t OFF_QMAX = OFF_PEND + 64;       // uint32 [NH][16]
  static constexpr uint32_t OFF_PB = OFF_QMAX + NH * 64;    // int [batch + 1]
  static constexpr uint32_t S_COL = 0;
  static constexpr uint32_t O_COL = SB * NR;
  static constexpr uint32_t TMEM_COLS = (SB + 2 * NH) * NR <= 128 ? 128 : ((SB + 2 * NH) * NR <= 256 ? 256 : 512);
  static_assert((SB + 2 * NH) * NR <= 512, "TMEM holds 512 columns");
  static constexpr int THREADS = 128 + 128 * NG;
  static size_t smem_bytes(int batch) { return OFF_PB + 4u * (batch + 1) + 1024; }
};

// ---------------------------------------------------------------------------------
// PTX wrappers
// ---------------------------------------------------------------------------------
// One page of HP KV heads, keys and values (encode_fp8_map's box).
__device__ __forceinline__ void tma_load_page8(uint32_t dst, const CUtensorMap* map, int kind_head, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(0), "r"(kind_head), "r"(0), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void mma_e4m3(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Matrix descriptor of a tile whose rows are W bytes (128 or 64) with the W-byte swizzle.
template <int W>
__device__ __forceinline__ uint64_t desc_rows(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>((lbo >> 4) & 0x3FFFu) << 16) |
         (static_cast<uint64_t>((sbo >> 4) & 0x3FFFu) << 32) | (1ull << 46) |
         (static_cast<uint64_t>(W == 128 ? 2 : 4) << 61);
}
// Instruction descriptor, kind::f8f6f4: fp32 accumulator, e4m3 A and B.
__host__ __device__ constexpr uint32_t idesc_e4m3(int M, int N, bool a_mn, bool b_mn) {
  return (1u << 4) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
         (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
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
template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t* r) {
  if constexpr (N == 16) tmem_ld16(taddr, r);
  else tmem_ld8(taddr, r);
}
// Named barrier of the four softmax warps that share a set of rows; or-reduces `v`.
__device__ __forceinline__ bool group_any(int id, bool v) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, %2, 128, p;\n selp.u32 %0, 1, 0, q;\n}"
      : "=r"(r)
      : "r"(v ? 1u : 0u), "r"(id)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void bar_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// Sum over the warp's lanes of each of N columns: lane i ends with column i * N / 32.
template <int N>
__device__ __forceinline__ float sum_columns(float* v, int lane) {
  int n = N;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    if (n > 1) {
      const bool upper = (lane & o) != 0;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        if (i < n / 2) {
          const float send = upper ? v[i] : v[i + n / 2], keep = upper ? v[i + n / 2] : v[i];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
      }
      n >>= 1;
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
  }
  return v[0];
}
// The warp's largest x (NaN ignored).
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// The two terms of a pair of values, each term packed with a's in the low byte; UP: the
// second term times 16.
template <bool UP>
__device__ __forceinline__ void split_e4m3x2(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = to_e4m3x2(a, b);
  uint32_t x;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(x) : "f"(b), "f"(a));
  const uint32_t h = e4m3x2_to_f16x2(hi);
  uint32_t d;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(h));
  if (UP) asm("mul.f16x2 %0, %1, %2;" : "=r"(d) : "r"(d), "r"(0x4c004c00u));
  uint16_t l;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(l) : "r"(d));
  lo = l;
}

constexpr float kNoKey = -1e30f;  // a row's reference before it has seen a key

// ---------------------------------------------------------------------------------
// The kernel
// ---------------------------------------------------------------------------------
template <int D, int HP, int NH, int NR>
__global__ void __launch_bounds__(Cfg<D, HP, NH, NR>::THREADS, 1)
    attn_fp8_tc_kernel(const __grid_constant__ CUtensorMap tmap, AttnFp8Params p) {
  using C = Cfg<D, HP, NH, NR>;
  constexpr int NC = C::NC, NG = C::NG, NST = C::NST, PB = C::PB, SB = C::SB;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (NST + s); };
  auto s_full = [&](int s) { return bar0 + 8u * (2 * NST + s); };
  auto s_free = [&](int s) { return bar0 + 8u * (2 * NST + SB + s); };
  auto p_full = [&](int h, int b) { return bar0 + 8u * (2 * NST + 2 * SB + h * PB + b); };
  auto pv_done = [&](int h, int b) { return bar0 + 8u * (2 * NST + 2 * SB + NH * PB + h * PB + b); };
  const uint32_t seg_ready = bar0 + 8u * (2 * NST + 2 * SB + 2 * NH * PB);
  auto drain_bar = [&](int i) { return seg_ready + 8 + 8u * i; };
  auto flag_bar = [&](int i) { return seg_ready + 24 + 8u * i; };
  float4* scl = reinterpret_cast<float4*>(smem + C::OFF_SCL);
  unsigned long long* nanv = reinterpret_cast<unsigned long long*>(smem + C::OFF_NAN);
  float* xch = reinterpret_cast<float*>(smem + C::OFF_X);
  uint32_t* misc = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 1);
  volatile int* pend_count = reinterpret_cast<volatile int*>(misc + 2);
  volatile int* nan_flag = reinterpret_cast<volatile int*>(misc + 3);
  volatile int* seg_flag = reinterpret_cast<volatile int*>(smem + C::OFF_FLAG);
  int* pend = reinterpret_cast<int*>(smem + C::OFF_PEND);
  uint32_t* qmax = reinterpret_cast<uint32_t*>(smem + C::OFF_QMAX);
  int* pb = reinterpret_cast<int*>(smem + C::OFF_PB);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // rows of each sub-unit: one head's, or a half of a row tile's
  const int tile_rows = HP == 2 ? NR : NH * NR;
  // softmax warps whose rows are all padding take no part
  const int max_rows = min(p.rows, NR);
  const int ngroup = (max_rows + NC - 1) / NC;
  const int nsoft = 4 * ngroup;

  if (threadIdx.x == 0) {
    for (int s = 0; s < NST; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int s = 0; s < SB; ++s) {
      mbar_init(s_full(s), 1);
      mbar_init(s_free(s), nsoft);
    }
    for (int h = 0; h < NH; ++h)
      for (int b = 0; b < PB; ++b) {
        mbar_init(p_full(h, b), nsoft);
        mbar_init(pv_done(h, b), 1);
      }
    mbar_init(seg_ready, nsoft);
    mbar_init(drain_bar(0), 1);
    mbar_init(drain_bar(1), 1);
    for (int i = 0; i < 8; ++i) mbar_init(flag_bar(i), 1);
    *abort_flag = 0;
    *pend_count = 0;
    *nan_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = threadIdx.x; i < HP * D; i += C::THREADS) nanv[i] = 0ull;
  if (warp == 1) tmem_alloc(smem_u32(misc), C::TMEM_COLS);
  if (warp == 0) {
    const int per_b = p.hunits * p.row_tiles;
    int carry = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      const int b = b0 + lane;
      int v = b < p.batch ? (unit_tiles<TK>(p.kv_len[b], p) + p.unit_overhead) * per_b : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += y;
      }
      if (b < p.batch) pb[b + 1] = carry + v;
      carry += __shfl_sync(0xffffffffu, v, 31);
    }
    if (lane == 0) pb[0] = 0;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];

  // equal ranges of the tile list; with no more units than blocks a multiple of the units
  const int64_t total = pb[p.batch];
  int ctas = static_cast<int>(total < gridDim.x ? total : gridDim.x);
  {
    const int64_t units = static_cast<int64_t>(p.batch) * p.hunits * p.row_tiles;
    if (units <= static_cast<int64_t>(gridDim.x)) {
      const int aligned = static_cast<int>(units) * (static_cast<int>(gridDim.x) / static_cast<int>(units));
      if (aligned < ctas) ctas = aligned;
    }
  }
  const int cta = blockIdx.x;
  const int64_t t0 = cta < ctas ? static_cast<int64_t>(cta) * total / ctas : 0;
  const int64_t t1 = cta < ctas ? static_cast<int64_t>(cta + 1) * total / ctas : 0;
  const int OVH = p.unit_overhead;

  if (warp == 0) {
    // ============================ producer ============================
    uint32_t it = 0, seg_no = 0;
    bool ok = true;
    const int psh = __ffs(p.page_size) - 1;  // log2
    const int npg = TK >> psh;               // pages of a tile
    const uint32_t box_bytes = static_cast<uint32_t>(p.page_size) * D * 2 * HP;
    for (Seg s = locate<TK>(t0, t1, p, pb, OVH); s.ntile > 0 && ok && !p.starve; ++seg_no) {
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
      int id = load_id(first), id1 = load_id(first + 32), base = first;
      float2 sc[HP], sc1[HP];
      load_scale(id, sc);
      load_scale(id1, sc1);
      int id2 = load_id(first + 64);
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
        if (it >= NST) ok = mbar_wait(empty(st), ((it / NST) - 1) & 1, abort_flag, p.status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        // lanes [pg0 - base, + npg) hold this tile's pages
        const int q = base + lane - pg0;
        const bool mine = q >= 0 && q < npg;
        const bool valid = mine && pg0 + q < pages;
        const bool in_range = id >= 0 && id < p.num_pages;
        flag |= __any_sync(0xffffffffu, valid && !in_range);
        if (mine) {
#pragma unroll
          for (int h = 0; h < HP; ++h) {
            const float sv = clamp_scale(sc[h].y);
            scl[(st * 8 + q) * HP + h] = valid ? make_float4(sc[h].x * p.scale_log2, log2f(sv), 1.f / sv, 0.f)
                                               : make_float4(0.f, 0.f, 0.f, 0.f);
          }
        }
        const uint32_t nvalid = __popc(__ballot_sync(0xffffffffu, valid));
        __syncwarp();
        if (lane == 0) {
          if (nvalid) mbar_arrive_tx(full(st), nvalid * box_bytes);
          else mbar_arrive(full(st));
        }
        __syncwarp();
        if (valid)
          tma_load_page8(sbase + C::OFF_STAGE + st * C::STAGE + static_cast<uint32_t>(q) * box_bytes, &tmap,
                         2 * ((in_range ? id : 0) * p.hkv + s.g * HP), full(st));
        __syncwarp();
      }
      if (ok && lane == 0) {
        seg_flag[seg_no & 7] = flag ? 1 : 0;
        mbar_arrive(flag_bar(seg_no & 7));
      }
      if (!has_more(s, t1, OVH)) break;
      s = locate<TK>(s.vnext, t1, p, pb, OVH);
    }
    if (!ok) {  // copies still in flight (bounded)
      for (uint32_t x = it > static_cast<uint32_t>(NST) ? it - NST : 0; x < it; ++x) {
        const long long c0 = clock64();
        while (!mbar_try(full(x % NST), (x / NST) & 1) && clock64() - c0 < kWaitCycles) {
        }
      }
    }
  } else if (warp == 1) {
    // ============================ S^T = K Q^T ============================
    constexpr uint32_t kIdesc = idesc_e4m3(128, NR, false, false);
    uint32_t it = 0, seg_no = 0;
    bool ok = true, issued = false;
    for (Seg s = locate<TK>(t0, t1, p, pb, OVH); s.ntile > 0 && ok; ++seg_no) {
      ok = mbar_wait(seg_ready, seg_no & 1, abort_flag, p.status);
      for (int k = 0; k < s.ntile && ok; ++k, ++it) {
        const uint32_t st = it % NST;
        ok = mbar_wait(full(st), (it / NST) & 1, abort_flag, p.status);
        for (int h = 0; h < NH && ok; ++h) {
          const uint32_t y = it * NH + h, sb = y % SB;
          if (y >= SB) ok = mbar_wait(s_free(sb), ((y / SB) - 1) & 1, abort_flag, p.status);
          if (!ok) break;
          tc_fence_after();
          if (lane == 0) {
            const uint32_t kb = sbase + C::OFF_STAGE + st * C::STAGE + (HP == 2 ? h : 0) * 2 * C::ATOM;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int kk = 0; kk < D / 32; ++kk)
                mma_e4m3(tmem + C::S_COL + sb * NR, desc_rows<D>(kb + kk * 32u, 16, C::SG),
                         desc_rows<D>(sbase + C::OFF_Q + (h * 2 + t) * C::Q_TERM + kk * 32u, 16, C::ATOM), kIdesc,
                         t > 0 || kk > 0);
            mma_commit(s_full(sb));
            issued = true;
          }
          __syncwarp();
        }
      }
      if (!has_more(s, t1, OVH)) break;
      s = locate<TK>(s.vnext, t1, p, pb, OVH);
    }
    if (!ok && __any_sync(0xffffffffu, issued)) {
      if (lane == 0) mma_commit(drain_bar(0));
      __syncwarp();
      const long long c0 = clock64();
      while (!mbar_try(drain_bar(0), 0) && clock64() - c0 < kWaitCycles) {
      }
    }
  } else if (warp == 3) {
    // ============================ O^T += V^T P^T ============================
    constexpr uint32_t kIdesc = idesc_e4m3(128, 2 * NR, true, true);
    uint32_t it = 0;
    bool ok = true, issued = false;
    // V of keys that no row sees must be finite, because their weight of 0 is multiplied:
    // keys past the end are cleared, and a NaN in a block key's value is cleared and noted,
    // for the outputs of the rows that see it.
    auto fix_values = [&](uint32_t st, const Seg& sg, int k) {
      const int key0 = (sg.tile0 + k) * TK;
      const int ctx = sg.kv_len - p.gamma;
      if (!sg.len_ok || key0 + TK <= ctx) return;
      const int nvalid = min(TK, sg.kv_len - key0);
      constexpr int kPieces = D / 16;
      unsigned char* base = smem + C::OFF_STAGE + st * C::STAGE;
      const int from = max(0, ctx - key0);
      for (int i = lane; i < (TK - from) * kPieces * HP; i += 32) {
        const int piece = i % kPieces, h = (i / kPieces) % HP, key = from + i / (kPieces * HP);
        const int ph = D == 128 ? piece ^ (key & 7) : piece ^ ((key >> 1) & 3);
        uint4* at = reinterpret_cast<uint4*>(base + (key >> 3) * C::SG + (2 * h + 1) * C::ATOM + (key & 7) * D + ph * 16);
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
              w[e >> 2] &= ~(0xffu << sh);
            }
          }
          *nan_flag = 1;
          *at = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      fence_async_smem();
      __syncwarp();
    };
    for (Seg s = locate<TK>(t0, t1, p, pb, OVH); s.ntile > 0 && ok;) {
      for (int k = 0; k < s.ntile && ok; ++k, ++it) {
        const uint32_t st = it % NST;
        ok = mbar_wait(full(st), (it / NST) & 1, abort_flag, p.status);
        if (!ok) break;
        // a unit's first tile waits for its weights first: they follow the outputs of the unit
        // before, whose NaN notes are then read
        if (k > 0) fix_values(st, s, k);
        const int buf = static_cast<int>(it % PB);
        for (int h = 0; h < NH && ok; ++h) {
          ok = mbar_wait(p_full(h, buf), (it / PB) & 1, abort_flag, p.status);
          if (!ok) break;
          if (k == 0 && h == 0) fix_values(st, s, k);
          tc_fence_after();
          if (lane == 0) {
            const uint32_t vb = sbase + C::OFF_STAGE + st * C::STAGE + ((HP == 2 ? h : 0) * 2 + 1) * C::ATOM;
            const uint32_t pa = sbase + C::OFF_P + (h * PB + buf) * C::P_BUF;
#pragma unroll
            for (int kk = 0; kk < TK / 32; ++kk)
              mma_e4m3(tmem + C::O_COL + h * 2 * NR, desc_rows<D>(vb + kk * 4u * C::SG, 0, C::SG),
                       desc_rows<128>(pa + kk * 4096u, 0, 1024), kIdesc, k > 0 || kk > 0);
            mma_commit(pv_done(h, buf));
            if (h == NH - 1) mma_commit(empty(st));
            issued = true;
          }
          __syncwarp();
        }
      }
      if (!has_more(s, t1, OVH)) break;
      s = locate<TK>(s.vnext, t1, p, pb, OVH);
    }
    if (!ok && __any_sync(0xffffffffu, issued)) {
      if (lane == 0) mma_commit(drain_bar(1));
      __syncwarp();
      const long long c0 = clock64();
      while (!mbar_try(drain_bar(1), 0) && clock64() - c0 < kWaitCycles) {
      }
    }
  } else if (warp >= 4 && (warp - 4) / 4 < ngroup) {
    // ============================ softmax ============================
    const int q4 = (warp - 4) & 3, ch = (warp - 4) >> 2;  // 32 keys; rows [ch * NC, + NC)
    const int gbar = 2 + ch;                              // named barrier of this row group
    const int nthr = nsoft * 32, stid = threadIdx.x - 128;  // threads of all groups
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(q4 * 32) << 16);
    const int psh = __ffs(p.page_size) - 1;
    const int pg = (q4 * 32 + lane) >> psh;  // this lane's page of a tile
    uint32_t it = 0, seg_no = 0;
    bool dead = false;  // after a timeout: run on without waiting
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (dead) return;
      const bool ok = mbar_wait(bar, parity, abort_flag, p.status);
      dead = !__all_sync(0xffffffffu, ok);
    };
    // per-segment state, by the segment's parity
    auto vis_of = [&](uint32_t par) { return reinterpret_cast<unsigned long long*>(smem + C::OFF_VIS) + par * NH * NR; };
    auto seen_of = [&](uint32_t par) { return reinterpret_cast<uint32_t*>(smem + C::OFF_SEEN) + par * NH * NG * 64; };
    auto mref_of = [&](uint32_t par) { return reinterpret_cast<float*>(smem + C::OFF_M) + par * NH * NR; };
    // rows of sub-unit h: the unit row of its row r, and how many are real
    auto unit_row = [&](const Seg& sg, int h, int r) { return sg.rt * tile_rows + (HP == 2 ? 0 : h * NR) + r; };
    auto real_rows = [&](const Seg& sg, int h) { return min(NR, p.rows - unit_row(sg, h, 0)); };

    // Brings a segment's Q into shared memory as two e4m3 terms, scaled by the power of two
    // that takes the sub-unit's largest finite magnitude into (224, 448], and sets its
    // row state. Returns the scales in qf.
    auto start_segment = [&](const Seg& sg, uint32_t par, float* qf) {
      constexpr int kPieces = D / 16;  // 16 elements per piece: 32 B in, 16 B per term
      constexpr int kTotal = NR * kPieces;
      constexpr int kLoops = NR == 64 ? (kTotal + 383) / 384 : 1;  // rows 33.. and 17.. have 384 threads
      uint4 x[NH][kLoops][2];
#pragma unroll
      for (int h = 0; h < NH; ++h) {
#pragma unroll
        for (int i = 0; i < kLoops; ++i) {
          const int item = i * nthr + stid, r = item / kPieces, piece = item % kPieces;
          x[h][i][0] = x[h][i][1] = make_uint4(0, 0, 0, 0);
          if (r < real_rows(sg, h)) {
            const int ur = unit_row(sg, h, r), j = ur / p.group;
            const int head = (sg.g * HP + (HP == 2 ? h : 0)) * p.group + ur - j * p.group;
            const uint4* src = reinterpret_cast<const uint4*>(
                static_cast<const __nv_bfloat16*>(p.q) +
                ((static_cast<int64_t>(sg.b) * p.gamma + j) * p.hq + head) * D + piece * 16);
            x[h][i][0] = __ldg(src);
            x[h][i][1] = __ldg(src + 1);
          }
        }
      }
      // meanwhile the rows' visible block keys, and the rows that see each block key
      const unsigned long long all = p.gamma >= 64 ? ~0ull : (1ull << p.gamma) - 1;
      unsigned long long* vis = vis_of(par);
      for (int i = stid; i < NH * NR; i += nthr) {
        const int h = i / NR, r = i % NR;
        const int j = min(unit_row(sg, h, r), p.rows - 1) / p.group;
        vis[i] = all & (p.tree_mask ? __ldg(p.tree_mask + static_cast<int64_t>(sg.b) * p.gamma + j) : (2ull << j) - 1);
        mref_of(par)[i] = kNoKey;
      }
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        uint32_t mx = 0;
#pragma unroll
        for (int i = 0; i < kLoops; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t w[4] = {x[h][i][e].x, x[h][i][e].y, x[h][i][e].z, x[h][i][e].w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint32_t a = w[c] & 0x7fffu, b = (w[c] >> 16) & 0x7fffu;
              mx = max(mx, max(a < 0x7f80u ? a : 0u, b < 0x7f80u ? b : 0u));
            }
          }
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (lane == 0) qmax[h * 16 + warp - 4] = mx;
      }
      bar_sync(1, nthr);
      for (int i = warp - 4; i < NH * ngroup * 64; i += nsoft) {  // lane = row of the group
        const int key = i & 63, hg = i >> 6, h = hg / ngroup, g = hg - h * ngroup;
        const bool v = lane < NC && (vis[h * NR + g * NC + (lane & (NC - 1))] >> key & 1);
        const uint32_t m = __ballot_sync(0xffffffffu, v);
        if (lane == 0) seen_of(par)[(h * NG + g) * 64 + key] = m;
      }
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        uint32_t mx = 0;
        for (int w = 0; w < nsoft; ++w) mx = max(mx, qmax[h * 16 + w]);
        const int e = mx == 0 ? 0 : min(118, max(-100, static_cast<int>(mx >> 7) - 135 + ((mx & 0x7fu) > 0x60u ? 1 : 0)));
        qf[h] = __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
        const float inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
        for (int i = 0; i < kLoops; ++i) {
          const int item = i * nthr + stid, r = item / kPieces, piece = item % kPieces;
          if (r >= NR) continue;
          uint32_t t1w[4], t2w[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint4 u = x[h][i][c >> 1];
            const uint32_t w[2] = {(c & 1) ? u.z : u.x, (c & 1) ? u.w : u.y};
            uint32_t a[2], b[2];
#pragma unroll
            for (int d = 0; d < 2; ++d) {
              float lo = __uint_as_float(w[d] << 16) * inv, hi = __uint_as_float(w[d] & 0xffff0000u) * inv;
              lo = fabsf(lo) < INFINITY ? lo : __int_as_float(0x7fc00000);  // an infinite query is NaN
              hi = fabsf(hi) < INFINITY ? hi : __int_as_float(0x7fc00000);
              split_e4m3x2<false>(lo, hi, a[d], b[d]);
            }
            t1w[c] = a[0] | a[1] << 16;
            t2w[c] = b[0] | b[1] << 16;
          }
          const int ph = D == 128 ? piece ^ (r & 7) : piece ^ ((r >> 1) & 3);
          unsigned char* dst = smem + C::OFF_Q + h * 2 * C::Q_TERM + r * D + ph * 16;
          *reinterpret_cast<uint4*>(dst) = make_uint4(t1w[0], t1w[1], t1w[2], t1w[3]);
          *reinterpret_cast<uint4*>(dst + C::Q_TERM) = make_uint4(t2w[0], t2w[1], t2w[2], t2w[3]);
        }
      }
      fence_async_smem();
      bar_sync(1, nthr);  // the row state is set
      if (lane == 0) mbar_arrive(seg_ready);
    };

    Seg s = locate<TK>(t0, t1, p, pb, OVH);
    float qf[NH];
    if (s.ntile > 0) start_segment(s, 0, qf);
    while (s.ntile > 0) {
      const uint32_t par = seg_no & 1;
      const int ctx = s.kv_len - p.gamma;
      float* mref = mref_of(par);
      float l[NH][NC];
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int c = 0; c < NC; ++c) l[h][c] = 0.f;

      for (int k = 0; k < s.ntile; ++k) {
        const uint32_t x = it + k, st = x % NST;
        const int key0 = (s.tile0 + k) * TK;
        const bool masked = key0 + TK > ctx;
        const int rel = key0 + q4 * 32 + lane - ctx;  // block position (negative: the prefix)
        const int buf = static_cast<int>(x % PB);
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          const uint32_t y = x * NH + h, sb = y % SB;
          wait(s_full(sb), (y / SB) & 1);
          tc_fence_after();
          uint32_t raw[NC];
          const uint32_t s_tmem = lane_base + C::S_COL + sb * NR + ch * NC;
          tmem_ld<NC>(s_tmem, raw);
          if (h == 0) wait(full(st), (x / NST) & 1);  // orders the producer's scales before this
          const float4 sc = scl[(st * 8 + pg) * HP + (HP == 2 ? h : 0)];
          const float ks = sc.x * qf[h];
          // e = log2 of the key's weight and value scale for each row, over the row's
          // reference; hidden keys have none
          const float* mr = mref + h * NR + ch * NC;
          uint32_t seen = ~0u;
          if (masked && rel >= 0) seen = rel < 64 ? seen_of(par)[(h * NG + ch) * 64 + rel] : 0u;
          float e[NC];
          for (bool raised = false;; raised = true) {
            tmem_wait_ld();
            float top = -INFINITY;
#pragma unroll
            for (int c = 0; c < NC; ++c) e[c] = fmaf(__uint_as_float(raw[c]), ks, sc.y) - mr[c];
            if (masked) {
#pragma unroll
              for (int c = 0; c < NC; ++c) e[c] = (seen >> c & 1) ? e[c] : -INFINITY;
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) top = fmaxf(top, e[c]);
            if (raised || !group_any(gbar, top > 8.f)) break;
            // Some weight would pass 2^8: raise the references, so that each row's largest
            // weight so far becomes 2^2 where it was more.
            float* xc = xch + h * 4 * NR;
            float mx = -INFINITY;
            tmem_ld<NC>(s_tmem, raw);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              const float v = fmaf(__uint_as_float(raw[c]), ks, sc.y);
              const float m = warp_max((seen >> c & 1) ? v : -INFINITY);
              if (lane % NC == c) mx = m;
            }
            if (lane < NC) xc[q4 * NR + ch * NC + lane] = mx;
            bar_sync(gbar, 128);
            const int c0 = ch * NC + lane % NC;
            const float old = mref[h * NR + c0];
            mx = fmaxf(fmaxf(xc[c0], xc[NR + c0]), fmaxf(xc[2 * NR + c0], xc[3 * NR + c0])) - 2.f;
            const float now = fmaxf(old, mx);
            const float alpha = ex2(old - now);
            bar_sync(gbar, 128);
            if (q4 == 0 && lane < NC) mref[h * NR + c0] = now;
            if (k > 0) {  // O holds every earlier tile before it is scaled
              wait(pv_done(h, (x - 1) % PB), ((x - 1) / PB) & 1);
              tc_fence_after();
#pragma unroll 1
              for (int c8 = 0; c8 < 2 * NC; c8 += 8) {
                const int t = c8 / NC, c1 = c8 % NC;
                const uint32_t col = lane_base + C::O_COL + (h * 2 + t) * NR + ch * NC + c1;
                tmem_ld8(col, raw);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 8; ++c)
                  raw[c] = __float_as_uint(__uint_as_float(raw[c]) * __shfl_sync(0xffffffffu, alpha, c1 + c));
                tmem_st8(col, raw);
              }
              tmem_wait_st();
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) l[h][c] *= __shfl_sync(0xffffffffu, alpha, c);
            tmem_ld<NC>(s_tmem, raw);
            bar_sync(gbar, 128);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(s_free(sb));
          uint32_t w1[NC / 4], w2[NC / 4];
#pragma unroll
          for (int c = 0; c < NC; c += 4) {
            float pr[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              pr[i] = ex2(e[c + i]);
              l[h][c + i] = fmaf(pr[i], sc.z, l[h][c + i]);
            }
            uint32_t a0, a1, b0, b1;
            split_e4m3x2<true>(pr[0], pr[1], a0, b0);
            split_e4m3x2<true>(pr[2], pr[3], a1, b1);
            w1[c / 4] = a0 | a1 << 16;
            w2[c / 4] = b0 | b1 << 16;
          }
          if (k >= PB) wait(pv_done(h, buf), ((x / PB) - 1) & 1);  // the buffer's last products are done
          unsigned char* prow = smem + C::OFF_P + (h * PB + buf) * C::P_BUF + (q4 * 32 + lane) * 128;
          const int sw = lane & 7;
          if constexpr (NC == 16) {
            const int a = ch, b = NR / 16 + ch;
            *reinterpret_cast<uint4*>(prow + ((a ^ sw) << 4)) = make_uint4(w1[0], w1[1], w1[2], w1[3]);
            *reinterpret_cast<uint4*>(prow + ((b ^ sw) << 4)) = make_uint4(w2[0], w2[1], w2[2], w2[3]);
          } else {  // eight bytes of a 16-byte chunk
            const int a = ch >> 1, b = NR / 16 + (ch >> 1);
            *reinterpret_cast<uint2*>(prow + ((a ^ sw) << 4) + (ch & 1) * 8) = make_uint2(w1[0], w1[1]);
            *reinterpret_cast<uint2*>(prow + ((b ^ sw) << 4) + (ch & 1) * 8) = make_uint2(w2[0], w2[1]);
          }
          fence_async_smem();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full(h, buf));
        }
      }
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        const float sum = sum_columns<NC>(l[h], lane);
        if (lane % (32 / NC) == 0) xch[(h * 4 + q4) * NR + ch * NC + lane / (32 / NC)] = sum;
      }
      // The next segment's Q takes the place of this one's: every S of this segment has been
      // read. Its first scores are computed while this segment's outputs are written.
      const Seg c = s;
      const uint32_t xl = it + c.ntile - 1;
      it += c.ntile;
      float qn[NH];
#pragma unroll
      for (int h = 0; h < NH; ++h) qn[h] = 0.f;
      if (has_more(c, t1, OVH)) {
        s = locate<TK>(c.vnext, t1, p, pb, OVH);
        start_segment(s, par ^ 1, qn);
      } else {
        s.ntile = 0;
      }
      // ---- the unit's (or the part's) sums and outputs ----
      wait(flag_bar(seg_no & 7), (seg_no >> 3) & 1);
      const bool bad = seg_flag[seg_no & 7] != 0;
      const bool whole = c.tile0 == 0 && c.ntile == c.unit_tiles;
      const int64_t slot = c.u + cta;
      if (bad && stid == 0) set_status(p.status, c.len_ok ? SPEC_FLAG_BAD_PAGE : SPEC_FLAG_BAD_KV_LEN);
      bar_sync(1, nthr);
      // a thread per row: its sum, factor and place
      int64_t* row_at = reinterpret_cast<int64_t*>(smem + C::OFF_ROW);
      float* row_inv = reinterpret_cast<float*>(smem + C::OFF_INV);
      for (int i = stid; i < NH * NR; i += nthr) {
        const int h = i / NR, r = i % NR;
        if (r >= real_rows(c, h)) continue;
        const float* xs = xch + h * 4 * NR + r;
        const float L = bad ? -1.f : xs[0] + xs[NR] + xs[2 * NR] + xs[3 * NR];
        const float m = mref[i];
        if (whole) {
          const int ur = unit_row(c, h, r), j = ur / p.group;
          const int head = (c.g * HP + (HP == 2 ? h : 0)) * p.group + ur - j * p.group;
          const int64_t at = (static_cast<int64_t>(c.b) * p.gamma + j) * p.hq + head;
          row_at[i] = at * D;
          row_inv[i] = fp8_inv(L);
          if (p.lse) p.lse[at] = fp8_lse(m, L);
        } else {
          const int64_t at = slot * p.slot_rows + (HP == 2 ? h * p.rows + r : h * NR + r);
          row_at[i] = at * D;
          row_inv[i] = L <= 0.f ? 0.f : 1.f;
          p.partial_ml[at] = make_float2(m, L);
        }
      }
      bar_sync(1, nthr);
      const int d = q4 * 32 + lane;  // this lane's dim
#pragma unroll 1
      for (int h = 0; h < NH; ++h) {
        wait(pv_done(h, xl % PB), (xl / PB) & 1);
        tc_fence_after();
        const bool has_nan = *nan_flag != 0;  // noted before the products just waited for
        const int nreal = min(NC, real_rows(c, h) - ch * NC);  // of this warp's rows
#pragma unroll 1
        for (int c8 = 0; c8 < nreal; c8 += 8) {
          uint32_t a[8], b[8];
          const uint32_t col = lane_base + C::O_COL + h * 2 * NR + ch * NC + c8;
          tmem_ld8(col, a);
          tmem_ld8(col + NR, b);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (c8 + i >= nreal || d >= D) continue;
            const int r = h * NR + ch * NC + c8 + i;
            const float inv = row_inv[r];
            float o = fmaf(__uint_as_float(b[i]), 0.0625f, __uint_as_float(a[i])) * inv;
            if (inv == 0.f) o = 0.f;
            if (has_nan && inv != 0.f && (nanv[(HP == 2 ? h : 0) * D + d] & vis_of(par)[r])) o = __int_as_float(0x7fc00000);
            if (whole) static_cast<__nv_bfloat16*>(p.out)[row_at[r] + d] = __float2bfloat16_rn(o);
            else p.partial_o[row_at[r] + d] = o;
          }
        }
      }
      if (!whole && stid == 0) {
        const int c_first = owner_of(c.unit_start, total, ctas);
        const int c_last = owner_of(c.unit_start + c.unit_tiles - 1, total, ctas);
        int* e = pend + 8 * (*pend_count);
        const int row_base = c.rt * tile_rows;
        e[0] = c.b; e[1] = c.g; e[2] = row_base; e[3] = min(tile_rows, p.rows - row_base);
        e[4] = static_cast<int>(c.u + c_first); e[5] = c_last - c_first + 1;
        e[6] = static_cast<int>(c.u); e[7] = 0;
        *pend_count = *pend_count + 1;
      }
      tc_fence_before();
      bar_sync(1, nthr);  // xch, the row state and nanv are read; the next segment may set them
      for (int i = stid; i < HP * D; i += nthr) nanv[i] = 0ull;
      if (stid == 0) *nan_flag = 0;
#pragma unroll
      for (int h = 0; h < NH; ++h) qf[h] = qn[h];
      ++seg_no;
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
  // split units: one ticket each, after a fence; the block that completes a unit merges it
  if (*abort_flag) return;
  const int np = *pend_count;
  if (np == 0) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 0; i < np; ++i) {
      int* e = pend + 8 * i;
      const uint32_t prev = atomicAdd(&p.tickets[e[6]], 1u);
      e[7] = prev == static_cast<uint32_t>(e[5] - 1);
      if (e[7]) p.tickets[e[6]] = 0;
    }
  }
  __syncthreads();
  for (int i = 0; i < np; ++i) {
    const int* e = pend + 8 * i;
    if (!e[7]) continue;
    __threadfence();
    for (int h = 0; h < HP; ++h)
      merge_fp8_unit<D>(p, e[0], e[1] * HP + h, e[2], e[3], e[4], e[5], threadIdx.x, C::THREADS, h * p.rows);
  }
}

// The cache as a 4-D tensor of bytes whose box is one page of HP adjacent KV heads: D
// bytes of a row; 8 rows; K and V of the heads (stride page * D); page / 8 groups of 8 rows.
// It lands as [8-key group][head, K or V][8 keys][D bytes]: the 8-key groups of one kind
// and head sit at a uniform stride through a tile, whatever the page size.
bool encode_fp8_map(CUtensorMap* map, const spec_attn_fp8_args_t& a, int heads_per_box) {
  EncodeTiledFn enc = encoder();
  if (!enc) return false;
  const cuuint64_t D = static_cast<cuuint64_t>(a.head_dim), P = static_cast<cuuint64_t>(a.page_size);
  const cuuint64_t dims[4] = {D, 8, 2 * static_cast<cuuint64_t>(a.num_pages) * a.num_kv_heads, P / 8};
  const cuuint64_t strides[3] = {D, P * D, 8 * D};
  const cuuint32_t box[4] = {static_cast<cuuint32_t>(D), 8, static_cast<cuuint32_t>(2 * heads_per_box),
                             static_cast<cuuint32_t>(P / 8)};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(a.kv_cache), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int HP, int NH, int NR>
cudaError_t launch_typed(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws, cudaStream_t stream,
                         bool starve) {
  using C = Cfg<D, HP, NH, NR>;
  CUtensorMap map;
  if (!encode_fp8_map(&map, a, HP)) return cudaErrorInvalidValue;
  AttnFp8Params p = make_attn_fp8_params(a, P, ws);
  p.hunits = a.num_kv_heads / HP;
  p.starve = starve ? 1 : 0;
  // Starting a unit inside a block's range costs about this many tiles of time; charged
  // only where blocks hold several starts.
  p.unit_overhead = static_cast<int64_t>(a.batch) * p.hunits * P.row_tiles > P.grid ? 2 : 0;
  const size_t smem = C::smem_bytes(a.batch);
  auto kernel = attn_fp8_tc_kernel<D, HP, NH, NR>;
  const cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  kernel<<<P.grid, C::THREADS, smem, stream>>>(map, p);
  return cudaGetLastError();
}

template <int D>
cudaError_t launch_d(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws, cudaStream_t stream,
                     bool starve) {
  if (P.heads == 2) {
    if (P.rows <= 16) return launch_typed<D, 2, 2, 16>(a, P, ws, stream, starve);
    if (P.rows <= 32) return launch_typed<D, 2, 2, 32>(a, P, ws, stream, starve);
    return launch_typed<D, 2, 2, 64>(a, P, ws, stream, starve);
  }
  if (P.rows <= 16) return launch_typed<D, 1, 1, 16>(a, P, ws, stream, starve);
  if (P.rows <= 32) return launch_typed<D, 1, 1, 32>(a, P, ws, stream, starve);
  if (P.rows <= 64) return launch_typed<D, 1, 1, 64>(a, P, ws, stream, starve);
  return launch_typed<D, 1, 2, 64>(a, P, ws, stream, starve);
}

template <int D>
size_t smem_of(int heads, int rows, int batch) {
  if (heads == 2)
    return rows <= 16 ? Cfg<D, 2, 2, 16>::smem_bytes(batch)
                      : (rows <= 32 ? Cfg<D, 2, 2, 32>::smem_bytes(batch) : Cfg<D, 2, 2, 64>::smem_bytes(batch));
  return rows <= 16   ? Cfg<D, 1, 1, 16>::smem_bytes(batch)
         : rows <= 32 ? Cfg<D, 1, 1, 32>::smem_bytes(batch)
         : rows <= 64 ? Cfg<D, 1, 1, 64>::smem_bytes(batch)
                      : Cfg<D, 1, 2, 64>::smem_bytes(batch);
}

}  // namespace

bool attn_fp8_tc_fits(const spec_attn_fp8_args_t& a, int heads, int rows) {
  const size_t smem = a.head_dim == 128 ? smem_of<128>(heads, rows, a.batch) : smem_of<64>(heads, rows, a.batch);
  const int64_t tiles = (static_cast<int64_t>(a.max_pages_per_seq) * a.page_size + TK - 1) / TK + 2;
  const int64_t units = static_cast<int64_t>(a.batch) * (a.num_kv_heads / heads) * ((rows + 127) / 128);
  return smem <= kTcMaxSmem && tiles * units <= INT32_MAX &&
         2 * static_cast<int64_t>(a.num_pages) * a.num_kv_heads <= INT32_MAX;
}

cudaError_t launch_attn_fp8_tc(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws, cudaStream_t stream,
                               bool starve) {
  return a.head_dim == 128 ? launch_d<128>(a, P, ws, stream, starve) : launch_d<64>(a, P, ws, stream, starve);
}

}  // namespace specv
