// Attention of the block queries over the 8-bit KV cache on tcgen05 tensor cores, with the
// keys on the MMA's M side (spec_verify_attention_fp8, SPEC_ATTN_TENSOR_CORES, KV groups of few
// rows).
//
// Both products run in 8 bits straight from the cache's bytes, which land in shared memory by
// TMA in the layout that the MMAs read; nothing is decoded on the way. They are transposed,
// with the 128 keys (or the D dims) of a tile on the MMA's M side, so that the query rows are
// its N side and a group of few rows pays for few:
//   S^T[key][row]  = K8[key][:] . Q8[row][:]          (M = 128 keys, N = rows, K = D)
//   O^T[dim][row] += sum_key V8[key][dim] P8[key][row] (M = D, N = 3 * rows, K = 128 keys)
// What is exact in the cache must not be lost on the other side. A bf16 query enters as the sum
// of two e4m3 terms (x1 = e4m3(x), x2 = e4m3(x - x1)), exact to 2^-18 of its row's largest
// element. A weight enters as the sum of three e5m2 terms (split_weights), which is bf16's
// precision, and for every weight that counts: where one key has most of a row's weight, the
// rest of the output is the sum of thousands of weights below 2^-15 of the largest. Two e4m3
// terms, whose smallest step was 2^-13 beside a largest of 2^2, lost all of them (32,768 keys, one
// with nine tenths of the weight: off by 0.63 of the output's norm, now 0.0018). Both terms of Q
// accumulate into the same S; those of P are thirds of N and are added when a unit ends.
//
// With sk, sv the scales of a key's page, m_r the row's reference and the weights
//   P = 2^(s + log2(sv) - m_r),  s = sk * S^T * softmax_scale * log2(e),
// O^T accumulates the weighted values with their scales, and sum P / sv is the softmax sum.
// m_r is chosen so that 2^9 <= the row's largest P <= 2^15 and rises only when P would pass 2^15
// (e5m2 ends at 1.75 * 2^15), which after a unit's first tile is rare. The third term of P is kept
// times 32, which puts its smallest step at 2^-21, 2^-30 of the row's largest P.
//
// A block serves two sub-units of at most 32 query rows: two adjacent KV heads (HP = 2, one
// box brings K and V of both: 8 KB with 16-token pages and D = 128), or two halves of one KV
// head's rows (HP = 1). Shared memory beyond Q and P is stages; P's rows are as narrow as its
// weights allow (64 or 128 bytes a key), which with 16 rows a sub-unit leaves room for a third
// stage of two heads (batch 32 decoding: 103 us with two). Keys and values in stages of their own, freed
// earlier but copied in boxes of half the size, took 99. Warp roles (persistent, one block per
// SM):
//   warps 16,19  producers: page ids and scales 32 pages ahead, one TMA box per page, each
//                the half of a tile's pages
//   warp 17      issues S^T = K Q^T into two S buffers per sub-unit in TMEM
//   warp 18      issues O^T += V^T P^T; clears V of keys past the sequence's end
//   warps 0..15  softmax, eight per sub-unit: lane quadrant = 32 keys, two warps per quadrant
//                share the rows. The sub-units' warps run free of each other, so that the
//                waits of one are filled by the other's arithmetic. They also convert Q and
//                write the outputs.
// The tiles of all units form one list that is cut into equal ranges, one per block; the fp32
// parts of a unit split between blocks are joined by a second launch. Every mbarrier wait is
// bounded; after a timeout the softmax warps run their loops to the end without waiting, so
// that none is missed at a named barrier.
//
// Memory bounds it up to 16 rows: batch 32, one token a sequence, contexts 256 to 16,384, 32 / 8
// heads of 128: 92 us, 5.92 TB/s (0.87 of the measured copy rate). With 32 rows the chain of
// waits from a tile's scores to its outputs does (batch 64 / block 8: 90 us, floor 46; 87 with two
// terms a weight). With one or an odd number of KV heads, or heads of 64, a tile brings half or a
// quarter of the bytes for the same chain (32 sequences as above, 8 / 1 heads: 28 us, floor 10;
// 32 / 8 heads of 64: 61, floor 40).
#include "attn_fp8_tc.cuh"

namespace specv {
namespace {

using namespace fp8tc;

constexpr int kSoftWarps = 8 * NH;
constexpr int kThreads = 32 * (kSoftWarps + 4);

// NR: query rows of a sub-unit (N of the first product), 16 or 32.
template <int D, int HP, int NR>
struct Cfg {
  static constexpr int NC = NR / 2;                        // rows per softmax warp
  static constexpr uint32_t ATOM = Stage<D, HP>::ATOM, SG = Stage<D, HP>::SG, STAGE = Stage<D, HP>::BYTES;
  static constexpr int SB = 2;                             // S buffers per sub-unit
  static constexpr uint32_t Q_TERM = NR * D;               // one term of one sub-unit's Q
  static constexpr uint32_t PW = 4 * NR;                   // a key's weights: first, second, third terms, unused
  static constexpr uint32_t P_BUF = TK * PW;               // [key][PW], swizzled by its width
  // where a stage fits for it, the work list's first tiles are those of every second sequence
  static constexpr int EACH = NR == 16 && HP * D >= 128 ? 2 : 1;
  static constexpr int NST = ((EACH == 2 ? 216 : 208) * 1024 - NH * (P_BUF + 2 * Q_TERM)) / STAGE;  // D = 128, HP = 2: 3 or 2
  static constexpr uint32_t OFF_STAGE = 0;
  static constexpr uint32_t OFF_P = OFF_STAGE + NST * STAGE;
  static constexpr uint32_t OFF_Q = OFF_P + NH * P_BUF;
  static constexpr uint32_t OFF_SCL = OFF_Q + NH * 2 * Q_TERM;      // float4 [NST][8 pages][HP]
  static constexpr uint32_t OFF_NAN = OFF_SCL + NST * 8 * HP * 16;  // uint64 [NH][D]: NaN block values
  // of the current and the next segment: the block keys each row sees, the rows that see
  // each block key (a bit each), the rows' references
  static constexpr uint32_t OFF_VIS = OFF_NAN + NH * D * 8;          // uint64 [2][NH][NR]
  static constexpr uint32_t OFF_SEEN = OFF_VIS + 2 * NH * NR * 8;    // uint32 [2][NH][64]
  static constexpr uint32_t OFF_M = OFF_SEEN + 2 * NH * 64 * 4;      // float [2][NH][NR]
  static constexpr uint32_t OFF_QS = OFF_M + 2 * NH * NR * 4;        // float [2][NH][NR]: rows' Q scales
  static constexpr uint32_t OFF_X = OFF_QS + 2 * NH * NR * 4;        // float [NH][4][NR]: cross-quadrant
  static constexpr uint32_t OFF_ROW = OFF_X + NH * 4 * NR * 4;       // int64 [NH][NR]: rows' outputs
  static constexpr uint32_t OFF_BAR = OFF_ROW + NH * NR * 8;
  // full[NST], empty[NST], s_full[NH][SB], s_free[NH][SB], p_full[NH], pv_done[NH],
  // seg_ready[NH], drain[2], flag_ready[kFlagRing]
  static constexpr int NBAR = 2 * NST + 2 * NH * SB + 3 * NH + 2 + kFlagRing;
  static constexpr uint32_t OFF_MISC = OFF_BAR + NBAR * 8;  // tmem base, abort, NaN flags
  static constexpr uint32_t OFF_FLAG = OFF_MISC + 16;               // int [2][kFlagRing]: segments' bad flags
  static constexpr uint32_t OFF_PB = OFF_FLAG + 8 * kFlagRing;       // int [list_entries<EACH>(batch)]
  static constexpr uint32_t S_COL = 0;                      // [NH][SB][NR]
  static constexpr uint32_t O_COL = NH * SB * NR;           // [NH][first, second, third terms][NR]
  static constexpr uint32_t TMEM_COLS = NR == 16 ? 256 : 512;
  static_assert(NH * (SB + 3) * NR <= TMEM_COLS, "a power of two of columns");
  static constexpr size_t smem_bytes(int batch) { return OFF_PB + 4u * list_entries<EACH>(batch) + 1024; }
};

// ---------------------------------------------------------------------------------
// PTX wrappers
// ---------------------------------------------------------------------------------
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
constexpr float kNoKey = -1e30f;  // a row's reference before it has seen a key

// ---------------------------------------------------------------------------------
// The kernel
// ---------------------------------------------------------------------------------
template <int D, int HP, int NR>
__global__ void __launch_bounds__(kThreads, 1)
    attn_fp8_keys_kernel(const __grid_constant__ CUtensorMap tmap, AttnFp8Params p) {
  using C = Cfg<D, HP, NR>;
  constexpr int NC = C::NC, NST = C::NST, SB = C::SB;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (NST + s); };
  auto s_full = [&](int h, int b) { return bar0 + 8u * (2 * NST + h * SB + b); };
  auto s_free = [&](int h, int b) { return bar0 + 8u * (2 * NST + NH * SB + h * SB + b); };
  auto p_full = [&](int h) { return bar0 + 8u * (2 * NST + 2 * NH * SB + h); };
  auto pv_done = [&](int h) { return bar0 + 8u * (2 * NST + 2 * NH * SB + NH + h); };
  auto seg_ready = [&](int h) { return bar0 + 8u * (2 * NST + 2 * NH * SB + 2 * NH + h); };
  auto drain_bar = [&](int i) { return bar0 + 8u * (2 * NST + 2 * NH * SB + 3 * NH + i); };
  auto flag_bar = [&](int i) { return bar0 + 8u * (2 * NST + 2 * NH * SB + 3 * NH + 2 + i); };
  float4* scl = reinterpret_cast<float4*>(smem + C::OFF_SCL);
  unsigned long long* nanv = reinterpret_cast<unsigned long long*>(smem + C::OFF_NAN);
  uint32_t* misc = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 1);
  volatile int* nan_flag = reinterpret_cast<volatile int*>(misc + 2);  // [NH]
  volatile int* seg_flag = reinterpret_cast<volatile int*>(smem + C::OFF_FLAG);  // [producer][kFlagRing]
  int* pb = reinterpret_cast<int*>(smem + C::OFF_PB);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // a unit's row tile: one sub-unit's rows for each of two heads, or two sub-units' rows
  const int sub_rows = p.rows_per_cta;
  const int tile_rows = HP == 2 ? sub_rows : NH * sub_rows;
  // softmax warps whose rows are all padding take no part
  const int nsoft = sub_rows > NC ? 8 : 4;  // per sub-unit

  if (warp == 0) {
    for (int i = lane; i < C::NBAR; i += 32) {
      constexpr int b_sfree = 2 * NST + NH * SB, b_pfull = b_sfree + NH * SB, b_pv = b_pfull + NH, b_seg = b_pv + NH;
      constexpr int b_drain = b_seg + NH, b_flag = b_drain + 2;
      const int n = i < NST || i >= b_flag ? 2                                                       // full, flag_ready
                    : (i >= b_sfree && i < b_pv) || (i >= b_seg && i < b_drain) ? nsoft : 1;  // s_free, p_full, seg_ready
      mbar_init(bar0 + 8u * i, n);
    }
    if (lane < NH) nan_flag[lane] = 0;
    if (lane < 2 * kFlagRing) seg_flag[lane] = 0;
    if (lane == 0) *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = threadIdx.x; i < NH * D; i += kThreads) nanv[i] = 0ull;
  if (warp == kSoftWarps + 1) tmem_alloc(smem_u32(misc), C::TMEM_COLS);
  if (threadIdx.x == 32 * kSoftWarps)
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap)) : "memory");
  pdl_wait_prior();
  if (warp == kSoftWarps) prefix_tiles<C::EACH>(p, pb);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  const WorkList<C::EACH> w = work_list<C::EACH>(p, pb);
  if (threadIdx.x == 0) clear_split(p);

  if (warp == kSoftWarps || warp == kSoftWarps + 3) {
    // ============================ producers ============================
    produce<D, HP, NST, C::EACH>(p, tmap, w, warp == kSoftWarps ? 0 : 1, sbase + C::OFF_STAGE, full(0), empty(0), flag_bar(0), scl,
                        seg_flag, abort_flag);
  } else if (warp == kSoftWarps + 1) {
    // ============================ S^T = K Q^T ============================
    constexpr uint32_t kIdesc = idesc_f8(128, NR, false, false);
    uint32_t it = 0, seg_no = 0;
    bool ok = true, issued = false;
    for (Seg s = find(w.t0, w, p); s.ntile > 0 && ok; ++seg_no) {
      for (int k = 0; k < s.ntile && ok; ++k, ++it) {
        const uint32_t st = it % NST, sb = it % SB;
        ok = mbar_wait(full(st), (it / NST) & 1, abort_flag, p.status);
        for (int h = 0; h < NH && ok; ++h) {
          if (k == 0) ok = mbar_wait(seg_ready(h), seg_no & 1, abort_flag, p.status);
          if (ok && it >= SB) ok = mbar_wait(s_free(h, sb), ((it / SB) - 1) & 1, abort_flag, p.status);
          if (!ok) break;
          tc_fence_after();
          if (lane == 0) {
            const uint32_t kb = sbase + C::OFF_STAGE + st * C::STAGE + (HP == 2 ? h : 0) * 2 * C::ATOM;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int kk = 0; kk < D / 32; ++kk)
                mma_f8(tmem + C::S_COL + (h * SB + sb) * NR, desc_rows<D>(kb + kk * 32u, 16, C::SG),
                         desc_rows<D>(sbase + C::OFF_Q + (h * 2 + t) * C::Q_TERM + kk * 32u, 16, C::ATOM), kIdesc,
                         t > 0 || kk > 0);
            mma_commit(s_full(h, sb));
            issued = true;
          }
          __syncwarp();
        }
      }
      if (!has_more(s, w.t1, w.ovh)) break;
      s = find(s.vnext, w, p);
    }
    if (!ok && __any_sync(0xffffffffu, issued)) {
      if (lane == 0) mma_commit(drain_bar(0));
      __syncwarp();
      const long long c0 = clock64();
      while (!mbar_try(drain_bar(0), 0) && clock64() - c0 < kWaitCycles) {
      }
    }
  } else if (warp == kSoftWarps + 2) {
    // ============================ O^T += V^T P^T ============================
    constexpr uint32_t kIdesc = idesc_f8(128, 3 * NR, true, true, false, true);
    uint32_t it = 0;
    bool ok = true, issued = false;
    for (Seg s = find(w.t0, w, p); s.ntile > 0 && ok;) {
      for (int k = 0; k < s.ntile && ok; ++k, ++it) {
        const uint32_t st = it % NST;
        ok = mbar_wait(full(st), (it / NST) & 1, abort_flag, p.status);
        if (!ok) break;
        // a unit's first tile waits for its weights first: they follow the outputs of the unit
        // before, whose NaN notes are then read
        if (k == 0)
          for (int h = 0; h < NH && ok; ++h) ok = mbar_wait(p_full(h), it & 1, abort_flag, p.status);
        if (!ok) break;
        fix_values<D, HP>(p, s, k, smem + C::OFF_STAGE + st * C::STAGE, nanv, nan_flag);
        for (int h = 0; h < NH && ok; ++h) {
          ok = mbar_wait(p_full(h), it & 1, abort_flag, p.status);
          if (!ok) break;
          tc_fence_after();
          if (lane == 0) {
            const uint32_t vb = sbase + C::OFF_STAGE + st * C::STAGE + ((HP == 2 ? h : 0) * 2 + 1) * C::ATOM;
            const uint32_t pa = sbase + C::OFF_P + h * C::P_BUF;
#pragma unroll
            for (int kk = 0; kk < TK / 32; ++kk)
              mma_f8(tmem + C::O_COL + h * 3 * NR, desc_rows<D>(vb + kk * 4u * C::SG, 0, C::SG),
                       desc_rows<C::PW>(pa + kk * 32u * C::PW, 0, 8 * C::PW), kIdesc, k > 0 || kk > 0);
            mma_commit(pv_done(h));
            if (h == NH - 1) mma_commit(empty(st));
            issued = true;
          }
          __syncwarp();
        }
      }
      if (!has_more(s, w.t1, w.ovh)) break;
      s = find(s.vnext, w, p);
    }
    if (!ok && __any_sync(0xffffffffu, issued)) {
      if (lane == 0) mma_commit(drain_bar(1));
      __syncwarp();
      const long long c0 = clock64();
      while (!mbar_try(drain_bar(1), 0) && clock64() - c0 < kWaitCycles) {
      }
    }
  } else if ((warp & 7) < nsoft) {
    // ============================ softmax ============================
    // sub-unit h; lane quadrant q4 = 32 keys; rows [ch * NC, + NC)
    const int h = warp >> 3, ch = (warp >> 2) & 1, q4 = warp & 3;
    const int sbar = 1 + h, gbar = 3 + 2 * h + ch;  // named barriers of the sub-unit and of the row group
    const int nthr = nsoft * 32, stid = threadIdx.x & 255;  // threads of the sub-unit
    const int swarp = warp & 7, kvh = HP == 2 ? h : 0;
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(q4 * 32) << 16);
    const uint32_t o_col = lane_base + C::O_COL + h * 3 * NR + ch * NC;
    const int pg = (q4 * 32 + lane) / p.page_size;  // this lane's page of a tile
    float* xch = reinterpret_cast<float*>(smem + C::OFF_X) + h * 4 * NR;  // [4][NR]
    unsigned char* const pbuf = smem + C::OFF_P + h * C::P_BUF + (q4 * 32 + lane) * C::PW;
    uint32_t it = 0, seg_no = 0;
    // After a timeout the warp runs its loops to the end without waiting (nothing else
    // depends on `dead`), so that it passes every named barrier.
    bool dead = false;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (!dead && !mbar_try(bar, parity)) dead = !wait_slow(bar, parity, abort_flag, p.status);
      __syncwarp();
    };
    // per-segment state, by the segment's parity
    auto vis_of = [&](uint32_t par) {
      return reinterpret_cast<unsigned long long*>(smem + C::OFF_VIS) + (par * NH + h) * NR;
    };
    auto seen_of = [&](uint32_t par) { return reinterpret_cast<uint32_t*>(smem + C::OFF_SEEN) + (par * NH + h) * 64; };
    auto mref_of = [&](uint32_t par) { return reinterpret_cast<float*>(smem + C::OFF_M) + (par * NH + h) * NR; };
    auto qs_of = [&](uint32_t par) { return reinterpret_cast<float*>(smem + C::OFF_QS) + (par * NH + h) * NR; };
    // the unit row of row r, and how many are real
    auto unit_row = [&](const Seg& sg, int r) { return sg.rt * tile_rows + (HP == 2 ? 0 : h * sub_rows) + r; };
    auto real_rows = [&](const Seg& sg) { return min(sub_rows, p.rows - unit_row(sg, 0)); };

    // Brings a segment's Q into shared memory as two e4m3 terms, each row scaled by the power of
    // two that takes its largest finite magnitude into (224, 448], and sets its row state.
    auto start_segment = [&](const Seg& sg, uint32_t par) {
      constexpr int kPieces = D / 16;  // 16 elements per piece: 32 B in, 16 B per term
      constexpr int kLoops = NR * kPieces > 256 ? NR * kPieces / 256 : 1;  // NR > 16 has 256 threads
      const int nreal = real_rows(sg);
      uint4 x[kLoops][2];
#pragma unroll
      for (int i = 0; i < kLoops; ++i) {
        const int item = i * nthr + stid, r = item / kPieces, piece = item % kPieces;
        x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
        if (r < nreal) {
          const int ur = unit_row(sg, r), j = ur / p.group;
          const int head = (sg.g * HP + kvh) * p.group + ur - j * p.group;
          const uint4* src = reinterpret_cast<const uint4*>(
              static_cast<const __nv_bfloat16*>(p.q) +
              ((static_cast<int64_t>(sg.b) * p.gamma + j) * p.hq + head) * D + piece * 16);
          x[i][0] = __ldg(src);
          x[i][1] = __ldg(src + 1);
        }
      }
      // meanwhile the rows' visible block keys, and the rows that see each block key
      const unsigned long long all = p.gamma >= 64 ? ~0ull : (1ull << p.gamma) - 1;
      unsigned long long* vis = vis_of(par);
      for (int r = stid; r < NR; r += nthr) {
        const int j = min(unit_row(sg, r), p.rows - 1) / p.group;
        vis[r] = all & (p.tree_mask ? __ldg(p.tree_mask + static_cast<int64_t>(sg.b) * p.gamma + j) : (2ull << j) - 1);
        mref_of(par)[r] = kNoKey;
      }
      bar_sync(sbar, nthr);
      for (int i = swarp; i < 64; i += nsoft) {  // lane = row
        const uint32_t m = __ballot_sync(0xffffffffu, lane < NR && (vis[lane % NR] >> i & 1));
        if (lane == 0) seen_of(par)[i] = m;
      }
#pragma unroll
      for (int i = 0; i < kLoops; ++i) {
        const int item = i * nthr + stid, r = item / kPieces, piece = item % kPieces;
        uint32_t mx = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t w[4] = {x[i][e].x, x[i][e].y, x[i][e].z, x[i][e].w};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t a = w[c] & 0x7fffu, b = (w[c] >> 16) & 0x7fffu;
            mx = max(mx, max(a < 0x7f80u ? a : 0u, b < 0x7f80u ? b : 0u));
          }
        }
#pragma unroll
        for (int o = 1; o < kPieces; o <<= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        if (r >= NR) continue;
        const int ex = mx == 0 ? 0 : min(118, max(-100, static_cast<int>(mx >> 7) - 135 + ((mx & 0x7fu) > 0x60u ? 1 : 0)));
        const float inv = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
        if (piece == 0) qs_of(par)[r] = __uint_as_float(static_cast<uint32_t>(ex + 127) << 23);
        uint32_t t1w[4], t2w[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint4 u = x[i][c >> 1];
          const uint32_t w[2] = {(c & 1) ? u.z : u.x, (c & 1) ? u.w : u.y};
          float v[4];
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            v[d] = __uint_as_float((d & 1) ? w[d >> 1] & 0xffff0000u : w[d >> 1] << 16) * inv;
            if (!(fabsf(v[d]) < INFINITY)) v[d] = __int_as_float(0x7fc00000);  // an infinite query is NaN
          }
          split_e4m3x4(v[0], v[1], v[2], v[3], t1w[c], t2w[c]);
        }
        const int ph = D == 128 ? piece ^ (r & 7) : piece ^ ((r >> 1) & 3);
        unsigned char* dst = smem + C::OFF_Q + h * 2 * C::Q_TERM + r * D + ph * 16;
        *reinterpret_cast<uint4*>(dst) = make_uint4(t1w[0], t1w[1], t1w[2], t1w[3]);
        *reinterpret_cast<uint4*>(dst + C::Q_TERM) = make_uint4(t2w[0], t2w[1], t2w[2], t2w[3]);
      }
      fence_async_smem();
      bar_sync(sbar, nthr);  // the row state is set
      if (lane == 0) mbar_arrive(seg_ready(h));
    };

    Seg s = find(w.t0, w, p);
    if (s.ntile > 0) start_segment(s, 0);
    while (s.ntile > 0) {
      const uint32_t par = seg_no & 1;
      const int ctx = s.kv_len - p.gamma;
      float* const mr = mref_of(par) + ch * NC;
      const float* const qs = qs_of(par) + ch * NC;
      float l[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) l[c] = 0.f;

      for (int k = 0; k < s.ntile; ++k) {
        const uint32_t x = it + k, st = x % NST, sb = x % SB;
        const int key0 = (s.tile0 + k) * TK;
        const bool masked = key0 + TK > ctx;
        const int rel = key0 + q4 * 32 + lane - ctx;  // block position (negative: the prefix)
        wait(s_full(h, sb), (x / SB) & 1);
        tc_fence_after();
        uint32_t raw[NC];
        const uint32_t s_tmem = lane_base + C::S_COL + (h * SB + sb) * NR + ch * NC;
        tmem_ld<NC>(s_tmem, raw);
        wait(full(st), (x / NST) & 1);  // orders the producer's scales before this
        const float4 sc = scl[(st * 8 + pg) * HP + kvh];
        uint32_t seen = ~0u;
        if (masked && rel >= 0) seen = rel < 64 ? seen_of(par)[rel] >> (ch * NC) : 0u;
        // e = log2 of the key's weight and value scale for each row, over the row's
        // reference; hidden keys have none
        float e[NC];
        auto exponents = [&](const uint32_t* r) {
#pragma unroll
          for (int c = 0; c < NC; ++c) e[c] = fmaf(__uint_as_float(r[c]), sc.x * qs[c], sc.y) - mr[c];
          if (masked) {
#pragma unroll
            for (int c = 0; c < NC; ++c) e[c] = (seen >> c & 1) ? e[c] : -INFINITY;
          }
        };
        tmem_wait_ld();
        exponents(raw);
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < NC; ++c) top = fmaxf(top, e[c]);
        if (group_any(gbar, top > 15.f)) {
          // Some weight would pass 2^15: raise the references, so that each row's largest
          // weight so far becomes 2^9 where it was more.
          float mx = -INFINITY;
#pragma unroll 1
          for (int c8 = 0; c8 < NC; c8 += 8) {
            uint32_t t8[8];
            tmem_ld8(s_tmem + c8, t8);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const float m = warp_max((seen >> (c8 + c) & 1) ? fmaf(__uint_as_float(t8[c]), sc.x * qs[c8 + c], sc.y) : -INFINITY);
              if (lane % NC == c8 + c) mx = m;
            }
          }
          float* const xc = xch + ch * NC + lane % NC;
          if (lane < NC) xc[q4 * NR] = mx;
          bar_sync(gbar, 128);
          const float old = mr[lane % NC];
          const float now = fmaxf(old, fmaxf(fmaxf(xc[0], xc[NR]), fmaxf(xc[2 * NR], xc[3 * NR])) - 9.f);
          const float alpha = ex2(old - now);
          bar_sync(gbar, 128);
          if (q4 == 0 && lane < NC) mr[lane] = now;
          if (k > 0) {  // O holds every earlier tile before it is scaled
            wait(pv_done(h), (x - 1) & 1);
            tc_fence_after();
#pragma unroll 1
            for (int c8 = 0; c8 < 3 * NC; c8 += 8) {
              uint32_t t8[8];
              const uint32_t col = o_col + (c8 / NC) * NR + c8 % NC;
              tmem_ld8(col, t8);
              tmem_wait_ld();
#pragma unroll
              for (int c = 0; c < 8; ++c)
                t8[c] = __float_as_uint(__uint_as_float(t8[c]) * __shfl_sync(0xffffffffu, alpha, c8 % NC + c));
              tmem_st8(col, t8);
            }
            tmem_wait_st();
          }
#pragma unroll
          for (int c = 0; c < NC; ++c) l[c] *= __shfl_sync(0xffffffffu, alpha, c);
          bar_sync(gbar, 128);
          uint32_t again[NC];
          tmem_ld<NC>(s_tmem, again);
          tmem_wait_ld();
          exponents(again);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(s_free(h, sb));
        if (k > 0) wait(pv_done(h), (x - 1) & 1);  // the last products have read P
        // weights, their sums, and their three terms into shared memory
        {
          uint32_t w1[NC / 4], w2[NC / 4], w3[NC / 4];
#pragma unroll
          for (int c = 0; c < NC; c += 4) {
            float pr[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              pr[i] = ex2(e[c + i]);
              l[c + i] = fmaf(pr[i], sc.z, l[c + i]);
            }
            split_weights<true>(pr, w1[c / 4], w2[c / 4], w3[c / 4]);
          }
          if constexpr (NR == 32) {  // this warp's rows are one 16-byte chunk of each term
            const int sw = lane & 7;
            *reinterpret_cast<uint4*>(pbuf + ((ch ^ sw) << 4)) = make_uint4(w1[0], w1[1], w1[2], w1[3]);
            *reinterpret_cast<uint4*>(pbuf + (((ch + 2) ^ sw) << 4)) = make_uint4(w2[0], w2[1], w2[2], w2[3]);
            *reinterpret_cast<uint4*>(pbuf + (((ch + 4) ^ sw) << 4)) = make_uint4(w3[0], w3[1], w3[2], w3[3]);
          } else {  // half a chunk
            const int sw = lane >> 1 & 3;
            *reinterpret_cast<uint2*>(pbuf + (sw << 4) + ch * 8) = make_uint2(w1[0], w1[1]);
            *reinterpret_cast<uint2*>(pbuf + ((1 ^ sw) << 4) + ch * 8) = make_uint2(w2[0], w2[1]);
            *reinterpret_cast<uint2*>(pbuf + ((2 ^ sw) << 4) + ch * 8) = make_uint2(w3[0], w3[1]);
          }
        }
        fence_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(h));
      }
      {
        const float sum = sum_columns<NC>(l, lane);
        if (lane % (32 / NC) == 0) xch[q4 * NR + ch * NC + lane / (32 / NC)] = sum;
      }
      // The next segment's Q takes the place of this one's: every S of this segment has been
      // read. Its first scores are computed while this segment's outputs are written.
      const Seg c = s;
      const uint32_t xl = it + c.ntile - 1;
      it += c.ntile;
      if (has_more(c, w.t1, w.ovh)) {
        s = find(c.vnext, w, p);
        start_segment(s, par ^ 1);
      } else {
        s.ntile = 0;
      }
      // ---- the unit's (or the part's) sums and outputs ----
      wait(flag_bar(seg_no % kFlagRing), (seg_no / kFlagRing) & 1);
      const bool bad = (seg_flag[seg_no % kFlagRing] | seg_flag[kFlagRing + seg_no % kFlagRing]) != 0;
      const bool whole = c.tile0 == 0 && c.ntile == c.unit_tiles;
      const int64_t slot = part_slot(w.cta, c.tile0 == 0);
      if (bad && stid == 0) set_status(p.status, c.len_ok ? SPEC_FLAG_BAD_PAGE : SPEC_FLAG_BAD_KV_LEN);
      const int nrows = real_rows(c);
      bar_sync(sbar, nthr);
      // a thread per row: its sum, factor (in place of the first part of the sum) and place
      int64_t* row_at = reinterpret_cast<int64_t*>(smem + C::OFF_ROW) + h * NR;
      float* row_inv = xch;
      for (int r = stid; r < nrows; r += nthr) {
        const float L = bad ? -1.f : xch[r] + xch[NR + r] + xch[2 * NR + r] + xch[3 * NR + r];
        const float m = mref_of(par)[r];
        if (whole) {
          const int ur = unit_row(c, r), j = ur / p.group;
          const int head = (c.g * HP + kvh) * p.group + ur - j * p.group;
          const int64_t at = (static_cast<int64_t>(c.b) * p.gamma + j) * p.hq + head;
          row_at[r] = at * D;
          row_inv[r] = fp8_inv(L);
          if (p.lse) p.lse[at] = fp8_lse(m, L);
        } else {
          const int64_t at = slot * p.slot_rows + h * sub_rows + r;
          row_at[r] = at * D;
          row_inv[r] = L <= 0.f ? 0.f : 1.f;
          p.partial_ml[at] = make_float2(m, L);
        }
      }
      bar_sync(sbar, nthr);
      wait(pv_done(h), xl & 1);
      tc_fence_after();
      const bool has_nan = nan_flag[h] != 0;  // noted before the products just waited for
      const int d = q4 * 32 + lane;           // this lane's dim
      const int nreal = min(NC, nrows - ch * NC);  // of this warp's rows
#pragma unroll 1
      for (int c8 = 0; c8 < nreal; c8 += 8) {
        uint32_t a[8], b[8], t[8];
        tmem_ld8(o_col + c8, a);
        tmem_ld8(o_col + NR + c8, b);
        tmem_ld8(o_col + 2 * NR + c8, t);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (c8 + i >= nreal || d >= D) continue;
          const int r = ch * NC + c8 + i;
          const float inv = row_inv[r];
          float o = (fmaf(__uint_as_float(t[i]), 0.03125f, __uint_as_float(b[i])) + __uint_as_float(a[i])) * inv;
          if (inv == 0.f) o = 0.f;
          if (has_nan && inv != 0.f && (nanv[h * D + d] & vis_of(par)[r])) o = __int_as_float(0x7fc00000);
          if (whole) static_cast<__nv_bfloat16*>(p.out)[row_at[r] + d] = __float2bfloat16_rn(o);
          else p.partial_o[row_at[r] + d] = o;
        }
      }
      if (h == 0 && stid == 0) note_split(p, c, w, tile_rows);
      tc_fence_before();
      bar_sync(sbar, nthr);  // xch, the row state and nanv are read; the next segment may set them
      for (int i = stid; i < D; i += nthr) nanv[h * D + i] = 0ull;
      if (stid == 0) nan_flag[h] = 0;
      ++seg_no;
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == kSoftWarps + 1) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

template <int D, int HP, int NR>
cudaError_t launch_typed(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws, cudaStream_t stream,
                         bool starve) {
  using C = Cfg<D, HP, NR>;
  CUtensorMap map;
  if (!encode_fp8_map(&map, a, HP)) return cudaErrorInvalidValue;
  AttnFp8Params p = make_attn_fp8_params(a, P, ws);
  p.hunits = a.num_kv_heads / HP;
  p.rows_per_cta = P.sub_rows;
  p.starve = starve ? 1 : 0;
  // Starting a unit inside a block's range costs about this many tiles of time (its Q, the
  // pipeline's refill, its outputs). Charging it keeps blocks of many short units and of few
  // long ones equal (batch 64 / block 8, 3: 91.0 us, 4: 89.8, 5: 91.8).
  p.unit_overhead = 4;
  // the limit is one for all host threads, so every call sets the same
  constexpr size_t kMost = C::smem_bytes(kFp8TcBatch);
  static_assert(kMost <= kTcMaxSmem, "a block's shared memory");
  auto kernel = attn_fp8_keys_kernel<D, HP, NR>;
  const cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMost));
  if (e != cudaSuccess) return e;
  const cudaError_t k = launch_overlapped(kernel, dim3(P.grid), kThreads, C::smem_bytes(a.batch), stream, map, p);
  return k == cudaSuccess ? launch_merge<D, HP, false>(p, P, stream) : k;
}

template <int D, int HP>
cudaError_t launch_d(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws, cudaStream_t stream,
                     bool starve) {
  if (P.sub_rows <= 16) return launch_typed<D, HP, 16>(a, P, ws, stream, starve);
  return launch_typed<D, HP, 32>(a, P, ws, stream, starve);
}

}  // namespace

namespace fp8tc {

// The cache as a 4-D tensor of bytes whose box is one page of `heads` adjacent KV heads: D
// bytes of a row; 8 rows; K and V of the heads (stride page * D); page / 8 groups of 8 rows.
// It lands as [8-key group][head, K or V][8 keys][D bytes]: the 8-key groups of one kind
// and head sit at a uniform stride through a tile, whatever the page size.
bool encode_fp8_map(CUtensorMap* map, const spec_attn_fp8_args_t& a, int heads) {
  tcx::EncodeTiledFn enc = tcx::encoder();
  if (!enc) return false;
  const cuuint64_t D = static_cast<cuuint64_t>(a.head_dim), P = static_cast<cuuint64_t>(a.page_size);
  const cuuint64_t dims[4] = {D, 8, 2 * static_cast<cuuint64_t>(a.num_pages) * a.num_kv_heads, P / 8};
  const cuuint64_t strides[3] = {D, P * D, 8 * D};
  const cuuint32_t box[4] = {static_cast<cuuint32_t>(D), 8, static_cast<cuuint32_t>(2 * heads),
                             static_cast<cuuint32_t>(P / 8)};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(a.kv_cache), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace fp8tc

cudaError_t launch_attn_fp8_keys(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws, cudaStream_t stream,
                               bool starve) {
  if (P.heads == 2)
    return a.head_dim == 128 ? launch_d<128, 2>(a, P, ws, stream, starve) : launch_d<64, 2>(a, P, ws, stream, starve);
  return a.head_dim == 128 ? launch_d<128, 1>(a, P, ws, stream, starve) : launch_d<64, 1>(a, P, ws, stream, starve);
}

}  // namespace specv
