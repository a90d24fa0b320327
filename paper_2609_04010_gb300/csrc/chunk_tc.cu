// Attention of ragged chunks over the paged bf16 cache on tcgen05 tensor cores
// (spec_chunk_attention, SPEC_ATTN_TENSOR_CORES).
//
//   S[row][key] = Q[row][:] . K[key][:]              (M = 128 rows, N = 128 keys, K = D)
//   O[row][dim] += sum_key P[row][key] V[key][dim]   (M = 128 rows, N = D, K = 128 keys)
// with P = 2^(c S - m), c = softmax scale * log2(e), a reference m per row that is raised only
// when a weight would pass 2^8, and the output O / sum P. A block holds a unit: two M tiles of the
// query rows (token, head of the group) of consecutive tokens and one KV head. Each tile of 128
// keys is read once for both; while one M tile is at its softmax the tensor core works for the
// other. A unit with no more rows than one M tile holds them twice and gives every second tile of
// keys to each, so that single tokens keep two tiles in flight too.
//
// Warps:
//   0..3, 4..7  softmax of M tile 0 and 1, a thread per row: 128 scores from TMEM, maximum,
//               weights as bf16 over the first half of the scores' columns, from which the second
//               product reads them; at a unit's end the outputs
//   8, 9        producers of K (and Q) and of V: a TMA box per page, into two rings of tiles
//   10          products: S of the next tile follows at once on the O += P V that read its columns
//   11          passes V on, and makes that of keys that some row does not see finite first (their weight 0 is multiplied):
//               keys that no row sees are cleared; where one that some rows see is not finite, the
//               unit is noted and computed again on CUDA cores after all
// The list of units is cut into equal ranges of steps, one per block (chunk.cuh); parts of split
// units are joined by the finishing launch. Every wait is bounded: one that runs out sets
// SPEC_FLAG_TIMEOUT, and the block drains its copies and products, frees TMEM and returns.
#include <cuda.h>  // CUtensorMap
#include <cuda_bf16.h>

#include "chunk.cuh"
#include "kv_fp8.cuh"
#include "tc_ptx.cuh"

namespace specv {
namespace {

using namespace tcx;

constexpr int TK = kChunkKeyTile;
constexpr int MR = kChunkTileRows;
constexpr int kSoftWarps = 8;
constexpr int kThreads = 32 * (kSoftWarps + 4);
// registers of a softmax and of another thread: 256 * 216 + 128 * 72 = 384 * 168, the launch's
constexpr int kSoftRegs = 216, kOtherRegs = 72;
// Past this the product of a score and the scale loses whole steps of the exponent.
constexpr float kFar = 4194304.f;  // 2^22

template <int D>
struct Cfg {
  static constexpr int DH = D / 64;                 // 128-byte column halves of a row
  static constexpr uint32_t GROUP = DH * 1024;      // 8 keys of a tile: [half][8 keys][128 B]
  static constexpr uint32_t TILE = (TK / 8) * GROUP;
  static constexpr uint32_t QHALF = MR * 128;
  static constexpr uint32_t QTILE = DH * QHALF;
  static constexpr int KST = D == 128 ? 3 : 5, VST = D == 128 ? 2 : 5;
  static constexpr uint32_t OFF_Q = 0;              // [2][DH][128 rows][128 B]
  static constexpr uint32_t OFF_K = OFF_Q + 2 * QTILE;
  static constexpr uint32_t OFF_V = OFF_K + KST * TILE;
  static constexpr uint32_t OFF_ML = OFF_V + VST * TILE;  // float2 [128]: the second half's (m, l)
  static constexpr uint32_t OFF_BAR = OFF_ML + MR * 8;
  // k_full[KST], k_empty[KST], v_full[VST], v_empty[VST], v_ready[VST], s_full[2], p_full[2],
  // o_full[2], q_full, q_free, drain, joined
  static constexpr int NBAR = 2 * KST + 3 * VST + 10;
  static constexpr uint32_t OFF_MISC = OFF_BAR + NBAR * 8;  // tmem base, abort
  static constexpr uint32_t BYTES = OFF_MISC + 16;
  static constexpr size_t SMEM = BYTES + 1024;
  static_assert(SMEM <= kTcMaxSmem, "a block's shared memory");
  static constexpr uint32_t S_COL = 0, O_COL = 2 * TK, TMEM_COLS = 512;
};

__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap* map, int page_head, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(0), "r"(0), "r"(0), "r"(page_head), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_q(uint32_t dst, const CUtensorMap* map, int half, int head, int row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(half), "r"(head), "r"(row), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void bar_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// (a, b) = (a, b) * s + n, two fp32 lanes at once
__device__ __forceinline__ void fma2(float& a, float& b, float s, float n) {
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %2};\n mov.b64 z, {%3, %3};\n"
      " fma.rn.f32x2 x, x, y, z;\n mov.b64 {%0, %1}, x;\n}"
      : "+f"(a), "+f"(b)
      : "f"(s), "f"(n));
}
__device__ __forceinline__ void add2(float& a, float& b, float c, float d) {
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "+f"(a), "+f"(b)
      : "f"(c), "f"(d));
}
__device__ __forceinline__ void mul2(float& a, float& b, float s) {
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %2};\n mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "+f"(a), "+f"(b)
      : "f"(s));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

__device__ __forceinline__ void fewer_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    chunk_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ CUtensorMap map_q, const __grid_constant__ ChunkParams p) {
  using C = Cfg<D>;
  constexpr int KST = C::KST, VST = C::VST, DH = C::DH;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto k_full = [&](uint32_t s) { return bar0 + 8u * s; };
  auto k_empty = [&](uint32_t s) { return bar0 + 8u * (KST + s); };
  auto v_full = [&](uint32_t s) { return bar0 + 8u * (2 * KST + s); };
  auto v_empty = [&](uint32_t s) { return bar0 + 8u * (2 * KST + VST + s); };
  auto v_ready = [&](uint32_t s) { return bar0 + 8u * (2 * KST + 2 * VST + s); };
  constexpr uint32_t B0 = 2 * KST + 3 * VST;
  auto s_full = [&](int h) { return bar0 + 8u * (B0 + h); };
  auto p_full = [&](int h) { return bar0 + 8u * (B0 + 2 + h); };
  auto o_full = [&](int h) { return bar0 + 8u * (B0 + 4 + h); };
  const uint32_t q_full = bar0 + 8u * (B0 + 6), q_free = bar0 + 8u * (B0 + 7), drain = bar0 + 8u * (B0 + 8);
  const uint32_t joined = bar0 + 8u * (B0 + 9);  // twins: the second Q tile's place is free again
  uint32_t* misc = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NBAR; ++i) {
      // p_full: the four warps of an M tile; joined: the eight of both
      const int n = i == static_cast<int>(B0) + 2 || i == static_cast<int>(B0) + 3 ? 4 : i == static_cast<int>(B0) + 9 ? 8 : 1;
      mbar_init(bar0 + 8u * i, n);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kSoftWarps + 2) tmem_alloc(smem_u32(misc), C::TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  pdl_wait_prior();

  bool dead = false;  // a wait ran out: go on without waiting where others count on this warp
  auto wait = [&](uint32_t bar, uint32_t parity) {  // a whole warp
    if (dead) return;
    bool ok = mbar_try(bar, parity);
    if (!ok) ok = mbar_wait(bar, parity, abort_flag, p.status);
    dead = !__all_sync(0xffffffffu, ok);
  };
  ChunkWalk w;

  if (warp == kSoftWarps || warp == kSoftWarps + 1) {
    // ============================ producers ============================
    fewer_registers();
    const bool is_k = warp == kSoftWarps;
    const uint32_t nst = is_k ? KST : VST, ring = sbase + (is_k ? C::OFF_K : C::OFF_V);
    const CUtensorMap* map = is_k ? &map_k : &map_v;
    const int psh = __ffs(p.page_size) - 1, npg = TK >> psh;
    const uint32_t box = static_cast<uint32_t>(p.page_size) * D * 2;
    const uint32_t qbytes = static_cast<uint32_t>(p.tile_tokens * p.group) * 128u;
    uint32_t it = 0, seg = 0, joins = 0;
    bool was_joined = false;
    auto full = [&](uint32_t s) { return is_k ? k_full(s) : v_full(s); };
    auto empty = [&](uint32_t s) { return is_k ? k_empty(s) : v_empty(s); };
    for (bool more = !p.starve && w.begin(p, blockIdx.x); more && !dead; ++seg) {
      const int32_t* table = p.page_table + static_cast<int64_t>(w.b) * p.max_pages;
      const int pages = (w.u.high - 1 >> psh) + 1;  // of the sequence, as far as the unit sees it
      // page ids, 32 at a time, the next 32 in flight
      int base = (w.u.tile0 + w.u.step_tiles(w.s0, 0)) * npg;
      auto load_id = [&](int at) { return at + lane < pages ? __ldg(table + at + lane) : 0; };
      int id = load_id(base), id_next = load_id(base + 32);
      bool bad = false, first = true;
      const int per = w.u.twin ? 2 : 1;
      for (int x = 0; x < w.ns * per && !dead; ++x) {
        const int i = w.s0 + x / per, h = x % per;
        if (!w.u.has(i, h)) continue;
        const int tile = w.u.tile0 + w.u.step_tiles(i, h), key0 = tile * TK, pg0 = tile * npg;
        while (pg0 >= base + 32) {
          base += 32;
          id = id_next;
          id_next = load_id(base + 32);
        }
        const uint32_t st = it % nst;
        if (it >= nst) wait(empty(st), (it / nst - 1) & 1);
        if (dead) break;
        // pages with a key that the unit sees
        const int q0 = max(key0, w.u.low) - key0 >> psh, q1 = (min(key0 + TK, w.u.high) - 1 - key0 >> psh) + 1;
        if (lane == 0) mbar_arrive_tx(full(st), static_cast<uint32_t>(q1 - q0) * box);
        for (int q = q0; q < q1; ++q) {
          const int raw = __shfl_sync(0xffffffffu, id, pg0 - base + q);
          const bool in_range = raw >= 0 && raw < p.num_pages;
          bad |= !in_range;
          if (lane == 0)
            tma_load_page(ring + st * C::TILE + static_cast<uint32_t>(q) * box, map, (in_range ? raw : 0) * p.hkv + w.g, full(st));
        }
        __syncwarp();
        ++it;
        if (is_k && first) {
          // Q follows the first tile of keys, once the segment before is done with its own
          if (seg > 0) wait(q_free, (seg - 1) & 1);
          if (was_joined) wait(joined, joins++ & 1);
          if (dead) break;
          if (lane == 0) {
            const int tiles = w.u.twin ? 1 : 2;
            mbar_arrive_tx(q_full, static_cast<uint32_t>(tiles * DH) * qbytes);
            for (int m = 0; m < tiles; ++m)
              for (int half = 0; half < DH; ++half)
                tma_load_q(sbase + C::OFF_Q + m * C::QTILE + half * C::QHALF, &map_q, half, w.g * p.group,
                           w.seq.row0 + w.u.token0 + m * p.tile_tokens, q_full);
          }
          __syncwarp();
        }
        first = false;
      }
      if (bad && lane == 0) {  // the sequence is cleared at the end
        p.seq_bad[w.b] = 1;
        set_status(p.status, SPEC_FLAG_BAD_PAGE);
      }
      was_joined = w.u.twin && w.whole();
      more = w.next(p);
    }
    if (dead) {  // copies still in flight (bounded)
      for (uint32_t x = it > nst ? it - nst : 0; x < it; ++x) {
        const long long c0 = clock64();
        while (!mbar_try(full(x % nst), (x / nst) & 1) && clock64() - c0 < kWaitCycles) {
        }
      }
      if (is_k && seg > 0) {
        const long long c0 = clock64();
        while (!mbar_try(q_full, (seg - 1) & 1) && clock64() - c0 < kWaitCycles) {
        }
      }
    }
  } else if (warp == kSoftWarps + 2) {
    // ============================ products ============================
    fewer_registers();
    constexpr uint32_t kIdescS = idesc_bf16(MR, TK, false), kIdescO = idesc_bf16(MR, D, true);
    uint32_t kc = 0, vc = 0, seg = 0;  // tiles of K and V taken so far
    uint32_t pc[2] = {0, 0};           // tiles weighed by each M tile
    bool issued = false;
    auto scores = [&](int h, int tile_of_q, uint32_t st) {
      if (lane == 0) {
        const uint32_t kb = sbase + C::OFF_K + st * C::TILE, qa = sbase + C::OFF_Q + tile_of_q * C::QTILE;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          mma_bf16(tmem + C::S_COL + h * TK, desc_sw128(qa + (kk / 4) * C::QHALF + (kk % 4) * 32u, 16, 1024),
                   desc_sw128(kb + (kk / 4) * 1024u + (kk % 4) * 32u, 16, C::GROUP), kIdescS, kk > 0);
        mma_commit(s_full(h));
        issued = true;
      }
      __syncwarp();
    };
    auto release = [&](uint32_t bar) {
      if (lane == 0) mma_commit(bar);
      __syncwarp();
    };
    for (bool more = w.begin(p, blockIdx.x); more && !dead; ++seg) {
      const bool twin = w.u.twin;
      // S of step i for M tile h; the K tile is shared by both unless twin
      auto next_scores = [&](int i, int h) {
        const uint32_t st = kc % KST;
        wait(k_full(st), (kc / KST) & 1);
        if (dead) return;
        tc_fence_after();
        scores(h, twin ? 0 : h, st);
        if (twin || h == 1) {
          release(k_empty(st));
          ++kc;
        }
      };
      wait(q_full, seg & 1);
      for (int h = 0; h < 2 && !dead; ++h)
        if (w.u.has(w.s0, h)) next_scores(w.s0, h);
      const int end = w.s0 + w.ns;
      for (int i = w.s0; i < end && !dead; ++i) {
        for (int h = 0; h < 2 && !dead; ++h) {
          if (!w.u.has(i, h)) continue;
          const uint32_t st = vc % VST;
          if (twin || h == 0) {
            wait(v_full(st), (vc / VST) & 1);
            wait(v_ready(st), (vc / VST) & 1);
          }
          wait(p_full(h), pc[h] & 1);
          ++pc[h];
          if (dead) break;
          tc_fence_after();
          if (lane == 0) {
            const uint32_t vb = sbase + C::OFF_V + st * C::TILE;
#pragma unroll
            for (int kk = 0; kk < TK / 16; ++kk)
              mma_bf16_ta(tmem + C::O_COL + h * D, tmem + C::S_COL + h * TK + kk * 8u,
                          desc_sw128(vb + kk * 2u * C::GROUP, 1024, C::GROUP), kIdescO, i > w.s0 || kk > 0);
            issued = true;
          }
          __syncwarp();
          const bool goes_on = i + 1 < end && w.u.has(i + 1, h);
          if (!goes_on) release(o_full(h));
          if (twin || h == 1) {
            release(v_empty(st));
            ++vc;
          }
          if (goes_on) next_scores(i + 1, h);
        }
        // the last scores of the segment are issued: Q is free once they are done
        if (i == end - 2 || (i == end - 1 && w.ns == 1)) release(q_free);
      }
      more = w.next(p);
    }
    if (dead && __any_sync(0xffffffffu, issued)) {
      if (lane == 0) mma_commit(drain);
      __syncwarp();
      const long long c0 = clock64();
      while (!mbar_try(drain, 0) && clock64() - c0 < kWaitCycles) {
      }
    }
  } else if (warp == kSoftWarps + 3) {
    // ============================ finite values ============================
    fewer_registers();
    uint32_t vc = 0;
    for (bool more = w.begin(p, blockIdx.x); more && !dead;) {
      const int per = w.u.twin ? 2 : 1;
      bool odd = false;
      for (int x = 0; x < w.ns * per && !dead; ++x) {
        const int i = w.s0 + x / per, h = x % per;
        if (!w.u.has(i, h)) continue;
        const int key0 = (w.u.tile0 + w.u.step_tiles(i, h)) * TK;
        const uint32_t st = vc % VST;
        wait(v_full(st), (vc / VST) & 1);
        if (dead) break;
        ++vc;
        if (key0 >= w.u.full_low && key0 + TK <= w.u.full_high) {
          if (lane == 0) mbar_arrive(v_ready(st));
          continue;
        }
        unsigned char* tile = smem + C::OFF_V + st * C::TILE;
        constexpr int kPieces = D / 8;  // 16-byte pieces of a key's values
        for (int c = lane; c < TK * kPieces; c += 32) {
          const int key = c / kPieces, piece = c % kPieces, pos = key0 + key;
          if (pos >= w.u.full_low && pos < w.u.full_high) continue;
          uint4* at = reinterpret_cast<uint4*>(tile + (key >> 3) * C::GROUP + (piece >> 3) * 1024 + (key & 7) * 128 + (piece & 7) * 16);
          if (pos < w.u.low || pos >= w.u.high) {
            *at = make_uint4(0, 0, 0, 0);
          } else {
            const uint4 v = *at;
            const uint32_t e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) odd |= __vcmpeq2(e[k] & 0x7f807f80u, 0x7f807f80u) != 0;
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(v_ready(st));
      }
      if (__any_sync(0xffffffffu, odd) && lane == 0) {
        const int n = atomicAdd(&p.redo[0].x, 1);
        if (n < p.redo_cap) p.redo[1 + n] = make_int4(w.b, w.g, w.rt, 0);
      }
      more = w.next(p);
    }
  } else {
    // ============================ softmax ============================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    const int h = warp >> 2, row = (warp & 3) * 32 + lane;  // row of the M tile
    const int tok = row / p.group, head = row - tok * p.group;
    const bool in_tile = row < p.tile_tokens * p.group;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_col = tmem + lanes + C::S_COL + h * TK, o_col = tmem + lanes + C::O_COL + h * D;
    float2* const other = reinterpret_cast<float2*>(smem + C::OFF_ML);
    const float c = p.scale_log2;
    uint32_t sc = 0, oc = 0;
    auto settle = [&](uint32_t bar, uint32_t parity) {
      wait(bar, parity);
      tc_fence_after();
    };
    for (bool more = w.begin(p, blockIdx.x); more;) {
      const int token = (w.u.twin ? 0 : h * p.tile_tokens) + tok;
      const bool real = in_tile && token < w.u.tokens;
      const bool any = __any_sync(0xffffffffu, real);
      // (rows of no token see what the last one sees, nothing stale)
      const int at = w.seq.kv_len - w.seq.n + w.u.token0 + min(token, w.u.tokens - 1);
      const int low = chunk_low(p, at), high = chunk_high(p, at, w.seq.kv_len);
      float m = -INFINITY, l = 0.f;  // the reference, a score; the sum
      bool none = true;              // this M tile has had no tile of keys
      for (int i = w.s0; i < w.s0 + w.ns; ++i) {
        if (!w.u.has(i, h)) continue;
        const int key0 = (w.u.tile0 + w.u.step_tiles(i, h)) * TK;
        settle(s_full(h), sc & 1);
        ++sc;
        if (any) {
          uint32_t raw[TK];
          float* s = reinterpret_cast<float*>(raw);
#pragma unroll
          for (int c0 = 0; c0 < TK; c0 += 32) tmem_ld32(s_col + c0, raw + c0);
          tmem_wait_ld();
          if (key0 < w.u.full_low || key0 + TK > w.u.full_high) {
            const int from = low - key0, to = high - key0;  // the columns this row sees
#pragma unroll
            for (int g = 0; g < TK; g += 32) {
              const uint32_t above = to - g >= 32 ? ~0u : to - g <= 0 ? 0u : (1u << (to - g)) - 1u;
              const uint32_t below = from - g >= 32 ? ~0u : from - g <= 0 ? 0u : (1u << (from - g)) - 1u;
              const uint32_t seen = above & ~below;
#pragma unroll
              for (int k = 0; k < 32; ++k) s[g + k] = (seen >> k & 1) ? s[g + k] : -INFINITY;
            }
          }
          float t0 = s[0], t1 = s[1], t2 = s[2], t3 = s[3];
#pragma unroll
          for (int k = 4; k < TK - 4; k += 8) {
            t0 = max3(t0, s[k], s[k + 1]);
            t1 = max3(t1, s[k + 2], s[k + 3]);
            t2 = max3(t2, s[k + 4], s[k + 5]);
            t3 = max3(t3, s[k + 6], s[k + 7]);
          }
          t0 = max3(t0, s[TK - 4], s[TK - 3]);
          t1 = max3(t1, s[TK - 2], s[TK - 1]);
          const float top = max3(fmaxf(t0, t1), t2, t3);
          // raise the reference where a weight would pass 2^8 (and at first)
          const bool raise = top > m && (m == -INFINITY || (top - m) * c > 8.f);
          if (__any_sync(0xffffffffu, raise)) {
            const float now = raise ? top : m;
            const float alpha = m == -INFINITY ? 0.f : ex2((m - now) * c);
            if (!none && __any_sync(0xffffffffu, raise && m != -INFINITY)) {
              // (the scores are done, so the products before them, which O holds, are too)
#pragma unroll 1
              for (int c0 = 0; c0 < D; c0 += 16) {
                uint32_t o[16];
                tmem_ld16(o_col + c0, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 16; k += 2) mul2(reinterpret_cast<float*>(o)[k], reinterpret_cast<float*>(o)[k + 1], alpha);
                tmem_st16(o_col + c0, o);
              }
            }
            l *= alpha;
            m = now;
          }
          // weights; m c is rounded up, so that no exponent passes what the reference allows
          const float neg = m == -INFINITY ? 0.f : -__fmul_ru(m, c);
          const bool far = fabsf(neg) > kFar;
          if (__any_sync(0xffffffffu, far)) {
#pragma unroll
            for (int k = 0; k < TK; ++k) s[k] = far ? (s[k] - m) * c : fmaf(s[k], c, neg);
          } else {
#pragma unroll
            for (int k = 0; k < TK; k += 2) fma2(s[k], s[k + 1], c, neg);
          }
          float a0 = 0.f, a1 = 0.f, a2 = 0.f, a3 = 0.f;
#pragma unroll
          for (int g = 0; g < TK; g += 32) {
            uint32_t pk[16];
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              const float x = ex2(s[g + k]), y = ex2(s[g + k + 1]);
              if (k & 2) add2(a2, a3, x, y); else add2(a0, a1, x, y);
              pk[k / 2] = pack_bf16(x, y);
            }
            tmem_st16(s_col + g / 2, pk);
          }
          l += (a0 + a1) + (a2 + a3);
          tmem_wait_st();
        }
        none = false;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(h));
      }
      // ---- the unit's outputs ----
      const bool had = !none;
      if (had) {
        settle(o_full(h), oc & 1);
        ++oc;
      }
      const float mc = m == -INFINITY ? -INFINITY : fabsf(m * c) > kFar ? m * c : __fmul_ru(m, c);
      const int64_t out_row = (static_cast<int64_t>(w.seq.row0) + w.u.token0 + token) * p.hq + w.g * p.group + head;
      __nv_bfloat16* const out = static_cast<__nv_bfloat16*>(p.out) + out_row * D;
      if (w.whole() && w.u.twin) {
        // the two M tiles hold the same rows: the second hands its part over in shared memory
        // (the second Q tile's, unused here), 32 columns at a time
        float* const place = reinterpret_cast<float*>(smem + C::OFF_Q + C::QTILE);
        if (h == 1) other[row] = make_float2(had ? mc : -INFINITY, had ? l : 0.f);
        float w0 = 1.f, w1 = 0.f;
        float2 ml = make_float2(-INFINITY, 0.f);
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 32) {
          float* const buf = place + (C::QTILE >= 32768 ? (c0 & 32) * MR : 0);
          uint32_t o[32];
          if (had) {
            tmem_ld32(o_col + c0, o);
            tmem_wait_ld();
          }
          if (h == 1 && had && any) {
#pragma unroll
            for (int k = 0; k < 32; ++k) buf[k * MR + row] = __uint_as_float(o[k]);
          }
          bar_sync(1, 256);
          if (h == 0 && any) {
            if (c0 == 0) {
              ml = other[row];
              const float top = fmaxf(mc, ml.x);
              w0 = mc == -INFINITY ? 0.f : ex2(mc - top);
              w1 = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
              const float total = l * w0 + ml.y * w1;
              if (real && p.lse) p.lse[out_row] = (top + log2f(total)) * 0.6931471805599453f;
              const float inv = 1.f / total;
              w0 *= inv;
              w1 *= inv;
            }
            uint32_t pk[16];
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              float x = __uint_as_float(o[k]) * w0, y = __uint_as_float(o[k + 1]) * w0;
              if (ml.x != -INFINITY) {
                x = fmaf(buf[k * MR + row], w1, x);
                y = fmaf(buf[(k + 1) * MR + row], w1, y);
              }
              pk[k / 2] = pack_bf16(x, y);
            }
            if (real) {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                reinterpret_cast<uint4*>(out + c0)[k] = make_uint4(pk[4 * k], pk[4 * k + 1], pk[4 * k + 2], pk[4 * k + 3]);
            }
          }
          if (C::QTILE < 32768) bar_sync(1, 256);  // one buffer only
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(joined);
      } else if (w.whole()) {
        const float inv = 1.f / l;  // every row sees a key: a sum of 0 (scores of -inf) is NaN
        if (any) {
#pragma unroll 1
          for (int c0 = 0; c0 < D; c0 += 32) {
            uint32_t o[32], pk[16];
            tmem_ld32(o_col + c0, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 32; k += 2) pk[k / 2] = pack_bf16(__uint_as_float(o[k]) * inv, __uint_as_float(o[k + 1]) * inv);
            if (real) {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                reinterpret_cast<uint4*>(out + c0)[k] = make_uint4(pk[4 * k], pk[4 * k + 1], pk[4 * k + 2], pk[4 * k + 3]);
            }
          }
          if (real && p.lse) p.lse[out_row] = (mc + log2f(l)) * 0.6931471805599453f;
        }
      } else if (any) {
        // a part: its place is the block's second where it starts the unit, else its first
        const int64_t slot = static_cast<int64_t>(2 * blockIdx.x + (w.starts_unit() ? 1 : 0)) * (2 * MR) + h * MR + row;
        if (had) {
#pragma unroll 1
          for (int c0 = 0; c0 < D; c0 += 32) {
            uint32_t o[32];
            tmem_ld32(o_col + c0, o);
            tmem_wait_ld();
            if (real) {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                reinterpret_cast<uint4*>(p.partial_o + slot * D + c0)[k] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
            }
          }
        }
        if (real) p.partial_ml[slot] = make_float2(had ? mc : -INFINITY, had ? l : 0.f);
      }
      tc_fence_before();
      __syncwarp();
      more = w.next(p);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kSoftWarps + 2) tmem_dealloc(tmem, C::TMEM_COLS);
}

// K or V viewed as a 5-D tensor whose box is one page of one KV head, landing as [8 keys][128-byte
// column half][8 keys][128 B] with the 128-byte swizzle, so that the 8-key groups of a tile sit at
// one stride whatever the page size.
bool encode_cache(CUtensorMap* map, const void* base, const spec_chunk_attn_args_t& a) {
  EncodeTiledFn enc = encoder();
  if (!enc) return false;
  const cuuint64_t D = a.head_dim, groups = a.page_size / 8;
  const cuuint64_t dims[5] = {64, 8, D / 64, groups, static_cast<cuuint64_t>(a.num_pages) * a.num_kv_heads};
  const cuuint64_t strides[4] = {D * 2, 128, 8 * D * 2, a.page_size * D * 2};
  const cuuint32_t box[5] = {64, 8, static_cast<cuuint32_t>(D / 64), static_cast<cuuint32_t>(groups), 1};
  const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Q viewed as (64 columns; column halves; heads; rows), the box one column half of an M tile: the
// group's heads of tile_tokens rows. Rows past the last read zeros.
bool encode_q(CUtensorMap* map, const spec_chunk_attn_args_t& a, const ChunkParams& p) {
  EncodeTiledFn enc = encoder();
  if (!enc) return false;
  const cuuint64_t D = a.head_dim;
  const cuuint64_t dims[4] = {64, D / 64, static_cast<cuuint64_t>(a.num_q_heads), static_cast<cuuint64_t>(a.rows)};
  const cuuint64_t strides[3] = {128, D * 2, static_cast<cuuint64_t>(p.q_stride) * 2};
  const cuuint32_t box[4] = {64, 1, static_cast<cuuint32_t>(p.group), static_cast<cuuint32_t>(p.tile_tokens)};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(a.q), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t launch_d(const spec_chunk_attn_args_t& a, const ChunkParams& p, cudaStream_t stream) {
  CUtensorMap mk, mv, mq;
  if (!encode_cache(&mk, a.k_cache, a) || !encode_cache(&mv, a.v_cache, a) || !encode_q(&mq, a, p)) return cudaErrorInvalidValue;
  const cudaError_t e = cudaFuncSetAttribute(chunk_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             static_cast<int>(Cfg<D>::SMEM));
  if (e != cudaSuccess) return e;
  return launch_overlapped(chunk_tc_kernel<D>, dim3(p.blocks), kThreads, Cfg<D>::SMEM, stream, mk, mv, mq, p);
}

}  // namespace

cudaError_t launch_chunk_tc(const spec_chunk_attn_args_t& a, const ChunkParams& p, cudaStream_t stream) {
  return a.head_dim == 128 ? launch_d<128>(a, p, stream) : launch_d<64>(a, p, stream);
}

}  // namespace specv
