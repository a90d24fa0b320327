// Attention of the block queries over the 8-bit KV cache on tcgen05 tensor cores, with the
// query rows on the MMA's M side (spec_verify_attention_fp8, SPEC_ATTN_TENSOR_CORES, KV groups
// of many rows).
//
//   S[row][key] = Q8[row][:] . K8[key][:]          (M = 128 rows, N = 128 keys, K = D)
//   O[row][dim] += sum_key P8[row][key] V8[key][dim] (M = 128 rows, N = D, K = 128 keys)
// The arithmetic is attn_fp8_keys.cu's: e4m3 operands straight from the cache, queries as sums
// of two e4m3 terms, weights as sums of three e5m2 terms, weights P = 2^(s + log2(sv) - m) against
// a reference m per row, sum P / sv. Here two threads share a row, each with half of a tile's
// keys: maximum, sum and reference are their own registers, the page constants are the same for
// all lanes, and only the two warps of 32 rows wait for each other (one thread a row, when weights
// had two terms: 162 us against 115 at batch 64 / block 16, because eight warps cannot hide each
// other's waits). With few rows the M side would be padding and attn_fp8_keys.cu is faster.
//
// A block serves two sub-units of at most 128 query rows: two adjacent KV heads (HP = 2) or
// two halves of one KV head's rows. The terms of P live in TMEM over the columns of S that
// they came from (32 keys of S are 32 columns, of P 8 + 8 + 8), so that shared memory holds Q and
// K/V stages only; S is computed again once the products have read P. While one sub-unit is
// at its softmax, the tensor core works for the other. m is set so that a row's largest P is
// 2^11.5 to 2^12.5 and raised when a P would pass 2^15 (the terms add up in one accumulator, so
// the third one's smallest step is 2^-16: a P is off by 2^-28 of the row's largest at most). The
// third product costs 0.2 us a tile (batch 4, 32,768 keys: 165 us against 153 with two e4m3 terms, which
// lost the weights below 2^-14 of the largest: 0.77 of an output where attn_fp8_keys.cu lost
// 0.63). m is a whole number, so that log2(sv) - m is exact with power-of-two scales. Hidden scores
// are set to -inf in TMEM, before the two passes over a tile (the maximum, the weights), which then
// know no masks.
// Warp roles (persistent, one block per SM):
//   warps 0..15   softmax, eight per sub-unit: a lane quadrant is 32 rows, two warps a quadrant
//   warps 16, 18  producers (as in attn_fp8_keys.cu)
//   warp 17       issues S = Q K^T and O += P V; clears V of keys past the sequence's end
// Work list, split units, bounded waits: as in attn_fp8_keys.cu.
//
// What bounds it is the chain S, softmax, P V of a sub-unit: 2.6 us a tile of 128 keys, of which
// its softmax is about 1.3 (the conversions and ex2 take 0.5 of it) and the products 0.7; two
// sub-units, all that TMEM has room for with D = 128, do not cover each other fully. Batch 4, block
// 32, 64 / 8 heads, 32,768 keys take 166 us: 828 TFLOP/s of Q K^T and P V, two and a half times that
// on the tensor cores. With two terms a weight (155 us) half tiles with scores in two buffers (231),
// four threads a row (158) and weights taken before the maximum is known (276) were all slower.
// Batch 64, block 16, 32 / 8 heads, contexts 512 to 4,096: 115 us, 2.8 TB/s.
#include "attn_fp8_tc.cuh"

namespace specv {
namespace {

using namespace fp8tc;

constexpr int kSoftWarps = 8 * NH;
constexpr int kThreads = 32 * (kSoftWarps + 3);
constexpr int MR = 128;  // rows of a sub-unit's MMA tile
constexpr int HK = TK / 2;  // keys of a tile that a thread weighs

template <int D, int HP>
struct Cfg {
  static constexpr uint32_t ATOM = Stage<D, HP>::ATOM, SG = Stage<D, HP>::SG, STAGE = Stage<D, HP>::BYTES;
  static constexpr uint32_t Q_TERM = MR * D;                                // one term of one sub-unit's Q
  static constexpr int NST = (208 * 1024 - NH * 2 * Q_TERM) / STAGE;  // D = 128: 2 (HP = 2) or 4
  static constexpr uint32_t OFF_STAGE = 0;
  static constexpr uint32_t OFF_Q = OFF_STAGE + NST * STAGE;
  static constexpr uint32_t OFF_SCL = OFF_Q + NH * 2 * Q_TERM;      // float4 [NST][8 pages][HP]
  static constexpr uint32_t OFF_NAN = OFF_SCL + NST * 8 * HP * 16;  // uint64 [NH][D]: NaN block values
  static constexpr uint32_t OFF_QS = OFF_NAN + NH * D * 8;          // float [2][NH][MR]: rows' Q scales
  static constexpr uint32_t OFF_XCH = OFF_QS + 2 * NH * MR * 4;    // float [NH][2][MR]: between a row's threads
  static constexpr uint32_t OFF_BAR = OFF_XCH + NH * 2 * MR * 4;
  // full[NST], empty[NST], s_full[NH], p_full[NH], pv_done[NH], seg_ready[NH], drain,
  // flag_ready[kFlagRing]
  static constexpr int NBAR = 2 * NST + 4 * NH + 1 + kFlagRing;
  static constexpr uint32_t OFF_MISC = OFF_BAR + NBAR * 8;        // tmem base, abort, -, -, NaN flags
  static constexpr uint32_t OFF_FLAG = OFF_MISC + 32;             // int [2][kFlagRing]: segments' bad flags
  static constexpr uint32_t OFF_PB = OFF_FLAG + 8 * kFlagRing;               // int [list_entries<1>(batch)]
  static constexpr uint32_t S_COL = 0;                            // [NH][128]; P over it
  static constexpr uint32_t O_COL = NH * TK;                      // [NH][D]
  static constexpr uint32_t TMEM_COLS = 512;
  static_assert(O_COL + NH * D <= TMEM_COLS, "TMEM holds 512 columns");
  static constexpr size_t smem_bytes(int batch) { return OFF_PB + 4u * list_entries<1>(batch) + 1024; }
};

// The same with A in tensor memory (M rows on the lanes, four bytes of K per column).
__device__ __forceinline__ void mma_f8_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Whether any thread of a pair of warps has `any` (named barrier).
__device__ __forceinline__ bool pair_any(int bar, bool any) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, %2, 64, p;\n selp.u32 %0, 1, 0, q;\n}"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(any)), "r"(bar)
      : "memory");
  return r != 0;
}

// a of e = a * S + b for a page's keys; a is not 0, so that a * -inf stays -inf.
__device__ __forceinline__ float slope(float ks, float qf) {
  const float a = ks * qf;
  return a == 0.f ? 1.17549435e-38f : a;
}

// The weights of half a tile for rows whose reference is past kFar, in place of the kernel's own
// loop: that takes the reference off a product that is not rounded, while the largest exponent
// was rounded, by up to 0.25 there and by thousands far past it. Here the exponents are rounded like
// the largest before the reference is taken off, so that none passes it. Returns l plus their sum.
// (Done for all references it takes 171 us at batch 4 and 32,768 keys; as it is, 166.)
constexpr float kFar = 4194304.f;  // 2^22
template <int HP>
__device__ __forceinline__ float far_weights(uint32_t s_col, int first, const float4* sc, int psh, float qf, float m,
                                             float l) {
#pragma unroll 1
  for (int c0 = first; c0 < first + HK; c0 += 32) {
    uint32_t w[24];
#pragma unroll
    for (int c8 = 0; c8 < 32; c8 += 8) {  // few registers: this is the rare case
      uint32_t r[8];
      tmem_ld8(s_col + c0 + c8, r);
      const float4 q = sc[((c0 + c8) >> psh) * HP];
      const float a = slope(q.x, qf);
      tmem_wait_ld();
#pragma unroll
      for (int c = 0; c < 8; c += 4) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = ex2(fmaf(__uint_as_float(r[c + i]), a, q.y) - m);
          l = fmaf(p[i], q.z, l);
        }
        split_weights<false>(p, w[(c8 + c) / 4], w[8 + (c8 + c) / 4], w[16 + (c8 + c) / 4]);
      }
    }
    tmem_st16(s_col + c0, w);
    tmem_st8(s_col + c0 + 16, w + 16);
  }
  return l;
}

template <int D, int HP>
__global__ void __launch_bounds__(kThreads, 1)
    attn_fp8_rows_kernel(const __grid_constant__ CUtensorMap tmap, AttnFp8Params p) {
  using C = Cfg<D, HP>;
  constexpr int NST = C::NST;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (NST + s); };
  auto s_full = [&](int h) { return bar0 + 8u * (2 * NST + h); };
  auto p_full = [&](int h) { return bar0 + 8u * (2 * NST + NH + h); };
  auto pv_done = [&](int h) { return bar0 + 8u * (2 * NST + 2 * NH + h); };
  auto seg_ready = [&](int h) { return bar0 + 8u * (2 * NST + 3 * NH + h); };
  const uint32_t drain_bar = bar0 + 8u * (2 * NST + 4 * NH);
  auto flag_bar = [&](int i) { return bar0 + 8u * (2 * NST + 4 * NH + 1 + i); };
  float4* scl = reinterpret_cast<float4*>(smem + C::OFF_SCL);
  unsigned long long* nanv = reinterpret_cast<unsigned long long*>(smem + C::OFF_NAN);
  uint32_t* misc = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 1);
  volatile int* nan_flag = reinterpret_cast<volatile int*>(misc + 4);            // [NH]
  volatile int* seg_flag = reinterpret_cast<volatile int*>(smem + C::OFF_FLAG);  // [producer][kFlagRing]
  int* pb = reinterpret_cast<int*>(smem + C::OFF_PB);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub_rows = p.rows_per_cta;
  const int tile_rows = HP == 2 ? sub_rows : NH * sub_rows;
  // warps with rows: the sub-unit's first row is on lane 0, or, for the second of two short
  // ones, on lane 64, so that all four SM sub-partitions work
  const int nact = (sub_rows + 31) / 32;

  if (warp == 0) {
    for (int i = lane; i < C::NBAR; i += 32) {
      constexpr int b_sfull = 2 * NST, b_pfull = b_sfull + NH, b_pv = b_pfull + NH, b_seg = b_pv + NH;
      constexpr int b_drain = b_seg + NH, b_flag = b_drain + 1;
      const int n = i < NST || i >= b_flag ? 2  // full, flag_ready
                    : (i >= b_pfull && i < b_pv) || (i >= b_seg && i < b_drain) ? 2 * nact : 1;  // p_full, seg_ready
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
  if (warp == kSoftWarps) prefix_tiles<1>(p, pb);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  const WorkList<1> w = work_list<1>(p, pb);
  if (threadIdx.x == 0) clear_split(p);

  if (warp == kSoftWarps || warp == kSoftWarps + 2) {
    // ============================ producers ============================
    produce<D, HP, NST, 1>(p, tmap, w, warp == kSoftWarps ? 0 : 1, sbase + C::OFF_STAGE, full(0), empty(0), flag_bar(0), scl,
                        seg_flag, abort_flag);
  } else if (warp == kSoftWarps + 1) {
    // ============================ products ============================
    // One thread's products run in the order of their issue: the next tile's S follows at once
    // on the O += P V that reads its columns.
    constexpr uint32_t kIdescS = idesc_f8(MR, TK, false, false), kIdescO = idesc_f8(MR, D, false, true, true);
    uint32_t it = 0, seg_no = 0;
    bool ok = true, issued = false;
    auto stage_full = [&](uint32_t x) { return mbar_wait(full(x % NST), (x / NST) & 1, abort_flag, p.status); };
    auto scores = [&](int h, uint32_t st) {
      if (lane == 0) {
        const uint32_t kb = sbase + C::OFF_STAGE + st * C::STAGE + (HP == 2 ? h : 0) * 2 * C::ATOM;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int kk = 0; kk < D / 32; ++kk)
            mma_f8(tmem + C::S_COL + h * TK,
                     desc_rows<D>(sbase + C::OFF_Q + (h * 2 + t) * C::Q_TERM + kk * 32u, 16, C::ATOM),
                     desc_rows<D>(kb + kk * 32u, 16, C::SG), kIdescS, t > 0 || kk > 0);
        mma_commit(s_full(h));
        issued = true;
      }
      __syncwarp();
    };
    for (Seg s = find(w.t0, w, p); s.ntile > 0 && ok; ++seg_no) {
      ok = stage_full(it);
      for (int h = 0; h < NH && ok; ++h) {
        ok = mbar_wait(seg_ready(h), seg_no & 1, abort_flag, p.status);
        if (!ok) break;
        tc_fence_after();
        scores(h, it % NST);
      }
      for (int k = 0; k < s.ntile && ok; ++k, ++it) {
        const uint32_t st = it % NST;
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
#pragma unroll
            for (int kk = 0; kk < TK / 32; ++kk)
#pragma unroll
              for (int t = 0; t < 3; ++t)
                mma_f8_ta(tmem + C::O_COL + h * D, tmem + C::S_COL + h * TK + kk * 32u + t * 8u,
                            desc_rows<D>(vb + kk * 4u * C::SG, 0, C::SG), kIdescO, k > 0 || kk > 0 || t > 0);
            mma_commit(pv_done(h));
            if (h == NH - 1) mma_commit(empty(st));
            issued = true;
          }
          __syncwarp();
          if (k + 1 < s.ntile) {
            if (h == 0) ok = stage_full(it + 1);
            if (ok) scores(h, (it + 1) % NST);
          }
        }
      }
      if (!has_more(s, w.t1, w.ovh)) break;
      s = find(s.vnext, w, p);
    }
    if (!ok && __any_sync(0xffffffffu, issued)) {
      if (lane == 0) mma_commit(drain_bar);
      __syncwarp();
      const long long c0 = clock64();
      while (!mbar_try(drain_bar, 0) && clock64() - c0 < kWaitCycles) {
      }
    }
  } else {
    // ============================ softmax ============================
    const int h = warp >> 3, ch = warp >> 2 & 1, q4 = warp & 3, kvh = HP == 2 ? h : 0;
    const int q0 = h == 1 && sub_rows <= 64 ? 2 : 0;  // first lane quadrant of the sub-unit
    if (q4 >= q0 && q4 < q0 + nact) {
      // pbar: the two warps of 32 rows; row: this thread's row of the sub-unit
      const int sbar = 1 + h, pbar = 1 + NH + h * 4 + q4, nthr = nact * 64, row = (q4 - q0) * 32 + lane;
      const int stid = ch * nact * 32 + row;
      float* const xch = reinterpret_cast<float*>(smem + C::OFF_XCH) + h * 2 * MR;
      const uint32_t lane_base = tmem + (static_cast<uint32_t>(q4 * 32) << 16);
      const uint32_t s_col = lane_base + C::S_COL + h * TK, o_col = lane_base + C::O_COL + h * D + ch * (D / 2);
      const int psh = __ffs(p.page_size) - 1;
      uint32_t it = 0, seg_no = 0;
      // After a timeout the warp runs its loops to the end without waiting (nothing else
      // depends on `dead`), so that it passes every named barrier.
      bool dead = false;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        if (!dead && !mbar_try(bar, parity)) dead = !wait_slow(bar, parity, abort_flag, p.status);
        __syncwarp();
      };
      auto unit_row = [&](const Seg& sg, int r) { return sg.rt * tile_rows + (HP == 2 ? 0 : h * sub_rows) + r; };
      auto real_rows = [&](const Seg& sg) { return min(sub_rows, p.rows - unit_row(sg, 0)); };
      float* const qscale = reinterpret_cast<float*>(smem + C::OFF_QS) + h * MR;  // [2][NH][MR]

      // Brings the pair's rows of a segment's Q into shared memory as two e4m3 terms, each row
      // scaled by the power of two that takes its largest finite magnitude into (224, 448].
      auto start_segment = [&](const Seg& sg, uint32_t par) {
        constexpr int kPieces = D / 16;  // 16 elements per piece: 32 B in, 16 B per term
        const int nreal = real_rows(sg);
        uint4 x[kPieces / 2][2];
#pragma unroll
        for (int i = 0; i < kPieces / 2; ++i) {
          const int item = i * 64 + ch * 32 + lane, r = (q4 - q0) * 32 + item / kPieces, piece = item % kPieces;
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
#pragma unroll
        for (int i = 0; i < kPieces / 2; ++i) {
          const int item = i * 64 + ch * 32 + lane, r = (q4 - q0) * 32 + item / kPieces, piece = item % kPieces;
          uint32_t v[8] = {x[i][0].x, x[i][0].y, x[i][0].z, x[i][0].w, x[i][1].x, x[i][1].y, x[i][1].z, x[i][1].w};
          uint32_t mx = 0;
#pragma unroll
          for (int c = 0; c < 8; ++c) mx = __vmaxu2(mx, v[c] & 0x7fff7fffu);
          mx = max(mx & 0xffffu, mx >> 16);
          if (__any_sync(0xffffffffu, mx >= 0x7f80u)) {  // an infinite query is NaN; the scale ignores both
            mx = 0;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const uint32_t lo = v[c] & 0x7fffu, hi = v[c] >> 16 & 0x7fffu;
              mx = max(mx, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
              v[c] |= (lo < 0x7f80u ? 0u : 0x7fu) | (hi < 0x7f80u ? 0u : 0x7f0000u);
            }
          }
#pragma unroll
          for (int o = 1; o < kPieces; o <<= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
          const int ex = mx == 0 ? 0 : min(118, max(-100, static_cast<int>(mx >> 7) - 135 + ((mx & 0x7fu) > 0x60u ? 1 : 0)));
          const float inv = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
          if (piece == 0) qscale[par * NH * MR + r] = __uint_as_float(static_cast<uint32_t>(ex + 127) << 23);
          uint32_t t1w[4], t2w[4];
#pragma unroll
          for (int c = 0; c < 4; ++c)
            split_e4m3x4(__uint_as_float(v[2 * c] << 16) * inv, __uint_as_float(v[2 * c] & 0xffff0000u) * inv,
                                __uint_as_float(v[2 * c + 1] << 16) * inv,
                                __uint_as_float(v[2 * c + 1] & 0xffff0000u) * inv, t1w[c], t2w[c]);
          const int lr = q0 * 32 + r;  // row of the MMA tile
          const int ph = D == 128 ? piece ^ (lr & 7) : piece ^ ((lr >> 1) & 3);
          unsigned char* dst = smem + C::OFF_Q + h * 2 * C::Q_TERM + lr * D + ph * 16;
          *reinterpret_cast<uint4*>(dst) = make_uint4(t1w[0], t1w[1], t1w[2], t1w[3]);
          *reinterpret_cast<uint4*>(dst + C::Q_TERM) = make_uint4(t2w[0], t2w[1], t2w[2], t2w[3]);
        }
        fence_async_smem();
        bar_sync(pbar, 64);  // the rows' scales are set
        if (lane == 0) mbar_arrive(seg_ready(h));
      };

      Seg s = find(w.t0, w, p);
      if (s.ntile > 0) start_segment(s, 0);
      while (s.ntile > 0) {
        const uint32_t par = seg_no & 1;
        const int ctx = s.kv_len - p.gamma;
        const int ur = unit_row(s, row);
        const bool real = row < real_rows(s);
        const int j = min(ur, p.rows - 1) / p.group;
        // the block keys this row sees, a bit each
        const unsigned long long all = p.gamma >= 64 ? ~0ull : (1ull << p.gamma) - 1;
        const unsigned long long vis =
            all & (p.tree_mask ? __ldg(p.tree_mask + static_cast<int64_t>(s.b) * p.gamma + j) : (2ull << j) - 1);
        const float qf = qscale[par * NH * MR + row];
        float m = -INFINITY, l = 0.f;  // reference (-inf: no key seen yet) and sum

        for (int k = 0; k < s.ntile; ++k) {
          const uint32_t x = it + k, st = x % NST;
          const int rel0 = (s.tile0 + k) * TK - ctx;  // block position of the tile's first key
          const bool masked = rel0 + TK > 0;
          // visibility of the 32 keys from key c0 of a masked tile
          auto seen_of = [&](int c0) -> uint32_t {
            const int r = rel0 + c0;
            if (r <= -32) return ~0u;
            if (r < 0) return static_cast<uint32_t>(vis << -r) | ((1u << -r) - 1u);
            return r < 64 ? static_cast<uint32_t>(vis >> r) : 0u;
          };
          const float4* const sc = scl + st * 8 * HP + kvh;  // page g of the tile: sc[g * HP]
          wait(s_full(h), x & 1);
          tc_fence_after();
          wait(full(st), (x / NST) & 1);  // orders the producer's scales before this
          if (masked) {  // hidden keys' scores become -inf in place
#pragma unroll 1
            for (int c0 = ch * HK; c0 < ch * HK + HK; c0 += 32) {
              const uint32_t seen = seen_of(c0);
              uint32_t r[32];
              tmem_ld32(s_col + c0, r);
              tmem_wait_ld();
#pragma unroll
              for (int c = 0; c < 32; ++c) r[c] = (seen >> c & 1) ? r[c] : 0xff800000u;
              tmem_st32(s_col + c0, r);
            }
            tmem_wait_st();
          }
          // ---- the largest weighted exponent of this thread's half of the row ----
          float top = -INFINITY;
#pragma unroll
          for (int c0 = ch * HK; c0 < ch * HK + HK; c0 += 32) {
            uint32_t r[32];
            tmem_ld32(s_col + c0, r);
            tmem_wait_ld();
#pragma unroll
            for (int g = 0; g < 32; g += 16) {
              const float4 q = sc[((c0 + g) >> psh) * HP];
              float t = __uint_as_float(r[g]);
#pragma unroll
              for (int c = 1; c < 16; ++c) t = fmaxf(t, __uint_as_float(r[g + c]));
              top = fmaxf(top, fmaf(t, slope(q.x, qf), q.y));
            }
          }
          // ---- raise the reference where a weight would pass 2^15 (and at references past kFar) ----
          bool weighed = false;
          if (pair_any(pbar, top > m + 15.f || (fabsf(m) > kFar && top > -INFINITY))) {
            xch[ch * MR + row] = top;
            bar_sync(pbar, 64);
            top = fmaxf(xch[row], xch[MR + row]);
            const float now = top > m + 15.f || m == -INFINITY ? fmaxf(m, rintf(top) - 12.f) : m;
            const float alpha = m == -INFINITY ? 0.f : ex2(m - now);
            if (k > 0) {  // O holds every earlier tile before it is scaled
              wait(pv_done(h), (x - 1) & 1);
              tc_fence_after();
#pragma unroll 1
              for (int c0 = 0; c0 < D / 2; c0 += 32) {
                uint32_t raw[32];
                tmem_ld32(o_col + c0, raw);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 32; ++c) raw[c] = __float_as_uint(__uint_as_float(raw[c]) * alpha);
                tmem_st32(o_col + c0, raw);
              }
              tmem_wait_st();
              l *= alpha;
            }
            m = now;
            bar_sync(pbar, 64);  // xch is read
            if (__any_sync(0xffffffffu, fabsf(m) > kFar && m != -INFINITY)) {
              l = far_weights<HP>(s_col, ch * HK, sc, psh, qf, m == -INFINITY ? 0.f : m, l);
              weighed = true;
            }
          }
          // ---- weights, their sum, and their three terms over the columns of S ----
          const float msub = m == -INFINITY ? 0.f : m;
          if (!weighed)  // by far_weights
#pragma unroll 1
          for (int c0 = ch * HK; c0 < ch * HK + HK; c0 += 32) {
            uint32_t r[32], w[24];
            tmem_ld32(s_col + c0, r);
            float2 ab[2];  // of 16 keys each
            float inv_sv[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              const float4 q = sc[((c0 + 16 * g) >> psh) * HP];
              ab[g] = make_float2(slope(q.x, qf), q.y - msub);
              inv_sv[g] = q.z;
            }
            tmem_wait_ld();
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              float sum = 0.f;
#pragma unroll
              for (int c = 16 * g; c < 16 * g + 16; c += 4) {
                float pr[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) pr[i] = ex2(fmaf(__uint_as_float(r[c + i]), ab[g].x, ab[g].y));
                sum += (pr[0] + pr[1]) + (pr[2] + pr[3]);
                split_weights<false>(pr, w[c / 4], w[8 + c / 4], w[16 + c / 4]);
              }
              l = fmaf(sum, inv_sv[g], l);
            }
            tmem_st16(s_col + c0, w);
            tmem_st8(s_col + c0 + 16, w + 16);
          }
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full(h));
        }
        xch[ch * MR + row] = l;
        // The next segment's Q takes the place of this one's: every S of this segment has
        // been read. Its first scores wait for this segment's last products only.
        const Seg c = s;
        const uint32_t xl = it + c.ntile - 1;
        it += c.ntile;
        if (has_more(c, w.t1, w.ovh)) {
          s = find(c.vnext, w, p);
          start_segment(s, par ^ 1);
        } else {
          s.ntile = 0;
        }
        // ---- the unit's (or the part's) output row ----
        wait(flag_bar(seg_no % kFlagRing), (seg_no / kFlagRing) & 1);
        const bool bad = (seg_flag[seg_no % kFlagRing] | seg_flag[kFlagRing + seg_no % kFlagRing]) != 0;
        const bool whole = c.tile0 == 0 && c.ntile == c.unit_tiles;
        if (bad && stid == 0) set_status(p.status, c.len_ok ? SPEC_FLAG_BAD_PAGE : SPEC_FLAG_BAD_KV_LEN);
        bar_sync(pbar, 64);
        const float L = bad ? -1.f : xch[row] + xch[MR + row];
        const float inv = whole ? fp8_inv(L) : (L <= 0.f ? 0.f : 1.f);
        const int head = (c.g * HP + kvh) * p.group + ur - j * p.group;
        const int64_t out_at = (static_cast<int64_t>(c.b) * p.gamma + j) * p.hq + head;
        const int64_t slot = part_slot(w.cta, c.tile0 == 0), part_at = slot * p.slot_rows + h * sub_rows + row;
        if (real && ch == 0) {
          if (!whole) p.partial_ml[part_at] = make_float2(m, L);
          else if (p.lse) p.lse[out_at] = fp8_lse(m, L);
        }
        wait(pv_done(h), xl & 1);
        tc_fence_after();
        const bool has_nan = nan_flag[h] != 0;  // noted before the products just waited for
#pragma unroll 1
        for (int c0 = 0; c0 < D / 2; c0 += 32) {
          uint32_t raw[32];
          float o[32];
          const int d0 = ch * (D / 2) + c0;
          tmem_ld32(o_col + c0, raw);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = inv == 0.f ? 0.f : __uint_as_float(raw[i]) * inv;
          if (has_nan && inv != 0.f) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (nanv[h * D + d0 + i] & vis) o[i] = __int_as_float(0x7fc00000);
          }
          if (!real) continue;
          if (whole) {
            uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + out_at * D + d0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t v[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 pr = __floats2bfloat162_rn(o[8 * i + 2 * e], o[8 * i + 2 * e + 1]);
                v[e] = *reinterpret_cast<const uint32_t*>(&pr);
              }
              dst[i] = make_uint4(v[0], v[1], v[2], v[3]);
            }
          } else {
            float4* dst = reinterpret_cast<float4*>(p.partial_o) + slot * p.slot_rows * (D / 4) +
                          static_cast<int64_t>(d0 / 4) * p.slot_rows + h * sub_rows + row;
#pragma unroll
            for (int i = 0; i < 8; ++i) dst[i * p.slot_rows] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
          }
        }
        if (h == 0 && stid == 0) note_split(p, c, w, tile_rows);
        tc_fence_before();
        // The notes are read by all; the next segment may set them. Every warp passes this barrier,
        // because after a timeout nothing orders what they read of nan_flag.
        bar_sync(sbar, nthr);
        if (has_nan) {
          for (int i = stid; i < D; i += nthr) nanv[h * D + i] = 0ull;
          if (stid == 0) nan_flag[h] = 0;
        }
        ++seg_no;
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == kSoftWarps + 1) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

template <int D, int HP>
cudaError_t launch_typed(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws, cudaStream_t stream,
                         bool starve) {
  using C = Cfg<D, HP>;
  CUtensorMap map;
  if (!encode_fp8_map(&map, a, HP)) return cudaErrorInvalidValue;
  AttnFp8Params p = make_attn_fp8_params(a, P, ws);
  p.hunits = a.num_kv_heads / HP;
  p.rows_per_cta = P.sub_rows;
  p.starve = starve ? 1 : 0;
  // tiles of time that starting a unit costs (batch 64 / block 20, 3: 129.5 us, 4: 127.0, 5: 128.3)
  p.unit_overhead = 4;
  // the limit is one for all host threads, so every call sets the same
  constexpr size_t kMost = C::smem_bytes(kFp8TcBatch);
  static_assert(kMost <= kTcMaxSmem, "a block's shared memory");
  auto kernel = attn_fp8_rows_kernel<D, HP>;
  const cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMost));
  if (e != cudaSuccess) return e;
  const cudaError_t k = launch_overlapped(kernel, dim3(P.grid), kThreads, C::smem_bytes(a.batch), stream, map, p);
  return k == cudaSuccess ? launch_merge<D, HP, true>(p, P, stream) : k;
}

}  // namespace

cudaError_t launch_attn_fp8_rows(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws, cudaStream_t stream,
                                 bool starve) {
  if (P.heads == 2)
    return a.head_dim == 128 ? launch_typed<128, 2>(a, P, ws, stream, starve) : launch_typed<64, 2>(a, P, ws, stream, starve);
  return a.head_dim == 128 ? launch_typed<128, 1>(a, P, ws, stream, starve) : launch_typed<64, 1>(a, P, ws, stream, starve);
}

}  // namespace specv
