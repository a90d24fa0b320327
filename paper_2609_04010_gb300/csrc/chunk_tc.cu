// Attention of ragged chunks over the paged caches on tcgen05 tensor cores
// (spec_chunk_attention, SPEC_ATTN_TENSOR_CORES).
//
//   S[row][key] = Q[row][:] . K[key][:]              (M = 128 rows, N = 128 keys, K = D)
//   O[row][dim] += sum_key P[row][key] V[key][dim]   (M = 128 rows, N = D, K = 128 keys)
// with P = 2^(c S - m), c = softmax scale * log2(e), a reference m per row that is raised only
// when a weight would pass 2^8, and the output O / sum P. A block holds a unit: two M tiles of the
// query rows (token, head of the group) of consecutive tokens and one KV head. Each tile of 128
// keys is read once for both (weights are bf16, off by 2^-8 of themselves, because values are and a
// product's operands have one type; l is the fp32 sum of the weights before that, so that nothing drifts);
// while one M tile is at its softmax the tensor core works for the
// other. A unit with no more rows than one M tile holds them twice and gives every second tile of
// keys to each ("twin"), so that single tokens keep two tiles in flight too.
//
// The 8-bit cache's values are made fp16 on the way, exactly; queries are fp16 times a power of two
// per row (made beside the set-up). Its scales stay out of the products: with the key's scale sk and
// the value's sv, P = 2^(c sq sk S + log2(sv) - m) and the sum is of P / sv. P is fp16, at most 2^15.
//
// Warps:
//   0..7, 8..15 softmax of M tile 0 and 1, two threads per row, each with half of a tile's keys: 64
//               scores from TMEM, maximum, weights in 16 bits over the first half of their columns, from
//               which the second product reads them; at a unit's end half of the row's outputs
//   16, 17      producers of K (and Q) and of V: a TMA box per page, into two rings of tiles
//   18          products: S of the next tile follows at once on the O += P V that read its columns, and
//               the M tiles take turns
//   19          passes V on, and makes that of keys that some row does not see finite first (their
//               weight 0 is multiplied): keys that no row sees are cleared; where one that some rows
//               see is not finite, the unit is noted and computed again on CUDA cores after all
//   (8-bit cache: 16 brings tiles and Q, 17 and 19 convert, and do to V what 19 does)
// The list of units is cut into equal ranges of steps, one per block (chunk.cuh); parts of split
// units are joined by the finishing launch. Every wait is bounded: one that runs out sets
// SPEC_FLAG_TIMEOUT, and the block drains its copies and products, frees TMEM and returns.
//
// What bounds it. Long chunks (4,096 tokens behind 28,672, 32 / 8 heads): 1,317 us by itself, 1,565 TFLOP/s of
// Q K^T and P V (1,893 measured peak), 1,452 in a row under the power cap (1,420 of 1,717); without the
// softmax's work the same code takes 1,150 by itself, the products' own time and the turns between them.
// Whole prompts (4 x 4,093): 468 us, 1,173 TFLOP/s: a unit of 64 tokens has 17 steps on average, and its
// outputs and first weights, about 4 steps of time, are not hidden. Single tokens (32 requests to 16,384
// tokens): 195 us, 5.6 TB/s, 0.83 of the copy rate: a step's five tiles in flight. 8-bit, two chunks of 2,048
// tokens: 527 us, 1,167 TFLOP/s:
// two warps make 32,768 values fp16 a step, 2,570 of its 3,860 cycles, in shared memory that the products
// read most of the time.
// What was measured on the way (long chunk by itself): one softmax thread per row 1,697 us (eight warps cannot
// hide each other's waits); two product warps in turns 1,446; products issued by "lane == 0" instead of
// an elected lane 1,404; registers spilled throughout a role's loop 1,800 to 2,900, because next to 226 KB of
// shared memory there is hardly any L1; outputs written after the next unit's first weights 1,626. What
// the compiler still spills, 16 bytes a thread (8-bit cache: 48), a block's warps load 82 times (16,400) in
// the 200 steps of a chunk of 2,048 tokens behind 14,336: at a unit's ends (five times a softmax warp's tile).

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
constexpr int kSoftWarps = 16;
constexpr int kThreads = 32 * (kSoftWarps + 4);
constexpr int HK = TK / 2;  // keys of a tile that a thread weighs
// registers of a softmax and of another thread: 512 * 104 + 128 * 64 = 640 * 96, the launch's; the
// 8-bit cache's producer and converters need as many as the softmax
template <bool FP8>
constexpr int kSoftRegs = FP8 ? 96 : 104;
template <bool FP8>
constexpr int kOtherRegs = FP8 ? 96 : 64;
// Past this the product of a score and the scale loses whole steps of the exponent.
constexpr float kFar = 4194304.f;  // 2^22

// A stop whose outputs are being written, while the walk is at the next one.
struct Ended {
  int row;   // of its first token
  int what;  // its tokens, and what follows
  int g;
};
constexpr int kTwin = 1 << 16, kWhole = 1 << 17, kStarts = 1 << 18;

// Notes of a tile of the 8-bit cache for its converters.
struct RawTile {
  int low, high, full_low, full_high;  // of its unit
  int key0, b, g, rt;
  uint32_t stop;
  int more;  // another tile follows
};
constexpr int kConverters = kChunkConverters;

template <int D, bool FP8>
struct Cfg {
  static constexpr int DH = D / 64;                 // 128-byte column halves of a row
  static constexpr uint32_t GROUP = DH * 1024;      // 8 keys of a tile: [half][8 keys][128 B]
  static constexpr uint32_t TILE = (TK / 8) * GROUP;
  static constexpr uint32_t QHALF = MR * 128;
  static constexpr uint32_t QTILE = DH * QHALF;
  static constexpr int KST = FP8 ? (D == 128 ? 2 : 4) : (D == 128 ? 2 : 5);
  static constexpr int VST = FP8 ? KST : (D == 128 ? 3 : 5);
  static constexpr uint32_t RAW = FP8 ? TK * D : 0;  // a tile of the 8-bit cache as it is: [key][D bytes]
  static constexpr uint32_t OFF_Q = 0;              // [2][DH][128 rows][128 B]
  static constexpr uint32_t OFF_K = OFF_Q + 2 * QTILE;
  static constexpr uint32_t OFF_V = OFF_K + KST * TILE;
  static constexpr uint32_t OFF_RAW = OFF_V + VST * TILE;  // [K, V]
  // float [2][128]: between a row's two threads; or float2 [128]: a twin's (m, l)
  static constexpr uint32_t OFF_XCH = OFF_RAW + 2 * RAW;
  static constexpr uint32_t OFF_WALK = OFF_XCH + 2 * MR * 4;  // ChunkWalk [kSoftWarps, then the 8-bit producer's]
  static constexpr uint32_t OFF_LAST = OFF_WALK + (kSoftWarps + (FP8 ? 1 : 0)) * sizeof(ChunkWalk);  // Ended [kSoftWarps]
  // The scales of a tile's pages, float4 [PT tiles][8 pages]. They are written when tile t is brought; by
  // then K of tile t - 1 is converted, so S of tile e = t - 1 - KST is done, and with it the weights of
  // its M tile's tile before it. Tile e's weights may be in work, in a twin e - 1's of the other M tile,
  // and where a twin of one tile follows e - 2's (the join holds its successor): e - 2..t are in use.
  static constexpr int PT = KST + 4;
  static constexpr uint32_t OFF_PAGES = (OFF_LAST + kSoftWarps * sizeof(Ended) + 15) / 16 * 16;
  static constexpr uint32_t OFF_RAWS = OFF_PAGES + (FP8 ? PT * 8 * 16 : 0);  // RawTile [4 tiles]
  static constexpr uint32_t OFF_BAR = (OFF_RAWS + (FP8 ? 4 * sizeof(RawTile) : 0) + 7) / 8 * 8;
  // k_full[KST], k_empty[KST], v_full[VST], v_empty[VST], v_ready[VST], s_full[2], p_full[2],
  // o_full[2], q_full, q_free, drain, joined[2], raw_full[2], raw_empty[2]
  static constexpr int NBAR = 2 * KST + 3 * VST + 15;
  static constexpr uint32_t OFF_MISC = OFF_BAR + NBAR * 8;  // tmem base, abort
  static constexpr uint32_t BYTES = OFF_MISC + 16;
  static constexpr size_t SMEM = BYTES;
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
__device__ __forceinline__ void tma_load_raw(uint32_t dst, const CUtensorMap* map, int page_head_kind, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(0), "r"(page_head_kind), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_q(uint32_t dst, const CUtensorMap* map, int half, int head, int row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(half), "r"(head), "r"(row), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// Whether any thread of the two warps of 32 rows has `any` (named barrier).
__device__ __forceinline__ bool pair_any(int bar, bool any) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, %2, 64, p;\n selp.u32 %0, 1, 0, q;\n}"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(any)), "r"(bar)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void bar_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// Four lanes' 4 x 4 pieces of 16 bytes turned round: afterwards c[j] is piece (lane & 3) of the j-th
// lane of the four, so that they store 64 bytes of a row together.
__device__ __forceinline__ void turn_quad(uint4* c, int lane) {
  const bool odd = lane & 1, high = lane & 2;
  auto swap = [](uint4& a, uint4& b, bool first, int mask) {
    uint32_t* x = reinterpret_cast<uint32_t*>(&a);
    uint32_t* y = reinterpret_cast<uint32_t*>(&b);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t got = __shfl_xor_sync(0xffffffffu, first ? x[e] : y[e], mask);
      if (first) x[e] = got; else y[e] = got;
    }
  };
  swap(c[0], c[1], odd, 1);
  swap(c[2], c[3], odd, 1);
  swap(c[0], c[2], high, 2);
  swap(c[1], c[3], high, 2);
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
// (a, b) += (x, y) * s
__device__ __forceinline__ void addmul2(float& a, float& b, float x, float y, float s) {
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n mov.b64 z, {%4, %4};\n"
      " fma.rn.f32x2 x, y, z, x;\n mov.b64 {%0, %1}, x;\n}"
      : "+f"(a), "+f"(b)
      : "f"(x), "f"(y), "f"(s));
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Products whose descriptors (desc_sw128) are a low word, which an offset in 16-byte units is added
// to, and a constant high word: the issuing thread keeps few registers.
__host__ __device__ constexpr uint32_t desc_high(uint32_t sbo) { return ((sbo >> 4) & 0x3FFFu) | (1u << 14) | (2u << 29); }
__device__ __forceinline__ uint32_t desc_low(uint32_t saddr, uint32_t lbo) { return ((saddr & 0x3FFFFu) >> 4) | ((lbo >> 4) << 16); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_low, uint32_t a_high, uint32_t b_low, uint32_t b_high,
                                       uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.b32 p, %6, 0;\n mov.b64 a, {%1, %2};\n mov.b64 b, {%3, %4};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n}" ::"r"(d),
      "r"(a_low), "r"(a_high), "r"(b_low), "r"(b_high), "r"(idesc), "r"(static_cast<uint32_t>(accumulate))
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_low, uint32_t b_high, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 b;\n setp.ne.b32 p, %5, 0;\n mov.b64 b, {%2, %3};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n}" ::"r"(d),
      "r"(a), "r"(b_low), "r"(b_high), "r"(idesc), "r"(static_cast<uint32_t>(accumulate))
      : "memory");
}

// One lane of a converged warp. (The compiler knows that it is one; with lane == 0 in its place the
// products' operands cost more than the products hide: a long prompt took 1,404 us instead of 1,306.)
__device__ __forceinline__ bool elected() {
  uint32_t one;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(one));
  return one != 0;
}

template <bool FP8>
__device__ __forceinline__ void fewer_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs<FP8>));
}

// A warp's: clears the values of keys that no row of the unit sees, and tells whether one that some
// rows do not see is not finite.
template <int D>
__device__ __forceinline__ bool finite_values(unsigned char* tile, int key0, const ChunkUnit& u) {
  constexpr int kPieces = D / 8, kLoads = 4;  // 16-byte pieces of a key; loads in flight
  // keys before `before` and from `after` on
  const int before = min(max(u.full_low - key0, 0), TK), after = min(max(u.full_high - key0, before), TK);
  const int n = (TK - (after - before)) * kPieces;
  bool odd = false;
  for (int c0 = threadIdx.x & 31; c0 < n; c0 += 32 * kLoads) {
    uint4 v[kLoads];
    uint4* at[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int c = c0 + 32 * k, piece = c % kPieces;
      int key = c / kPieces;
      key += key < before ? 0 : after - before;
      at[k] = nullptr;
      v[k] = make_uint4(0, 0, 0, 0);
      if (c < n) {
        uint4* from = reinterpret_cast<uint4*>(tile + (key >> 3) * Cfg<D, false>::GROUP + (piece >> 3) * 1024 + (key & 7) * 128 + (piece & 7) * 16);
        if (key0 + key < u.low || key0 + key >= u.high) at[k] = from; else v[k] = *from;
      }
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      if (at[k]) *at[k] = v[k];
      odd |= (__vcmpeq2(v[k].x & 0x7f807f80u, 0x7f807f80u) | __vcmpeq2(v[k].y & 0x7f807f80u, 0x7f807f80u) |
              __vcmpeq2(v[k].z & 0x7f807f80u, 0x7f807f80u) | __vcmpeq2(v[k].w & 0x7f807f80u, 0x7f807f80u)) != 0;
    }
  }
  fence_async_smem();
  __syncwarp();
  return odd;
}

// Part `part` of kConverters warps: a tile of the 8-bit cache as fp16, exactly, in the products'
// layout. With VALUES, keys outside [low, high) are cleared and the result tells whether one that some
// rows do not see is NaN.
template <int D, bool VALUES>
__device__ __forceinline__ bool convert_tile(const unsigned char* raw, unsigned char* tile, const RawTile& t, int part) {
  constexpr int kPieces = D / 16, kItems = TK * kPieces, kLoads = 4;  // 16 values each
  const int lane = threadIdx.x & 31;
  bool odd = false;
  int low = 0, high = TK, full_low = 0, full_high = TK;  // keys of the tile that any and that all rows see
  if constexpr (VALUES) {
    low = t.low - t.key0;
    high = t.high - t.key0;
    full_low = t.full_low - t.key0;
    full_high = t.full_high - t.key0;
  }
  const bool partial = full_low > 0 || full_high < TK;
  // Lane l of a round takes piece l % kPieces of key l / kPieces, the upper half of a row's pieces of the
  // neighbour key: the 16-byte places of 8 lanes then lie in different banks in both stores (522 us; 610 without).
  const int piece = lane % kPieces, key_of = (lane / kPieces) ^ (piece >> 2);
  constexpr int kRounds = kItems / 32, kKeys = 32 / kPieces;  // 32 items a round
  const int from = part * (kRounds / 2), to = from + kRounds / 2;
#pragma unroll 1
  for (int r = from; r < to; r += kLoads) {
    uint4 v[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) v[k] = *reinterpret_cast<const uint4*>(raw + ((r + k) * kKeys + key_of) * D + piece * 16);
    if (VALUES && partial) {
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        const int key = (r + k) * kKeys + key_of;
        if (key < low || key >= high) v[k] = make_uint4(0, 0, 0, 0);
        if (key < full_low || key >= full_high)
          odd |= (__vcmpeq4(v[k].x & 0x7f7f7f7fu, 0x7f7f7f7fu) | __vcmpeq4(v[k].y & 0x7f7f7f7fu, 0x7f7f7f7fu) |
                  __vcmpeq4(v[k].z & 0x7f7f7f7fu, 0x7f7f7f7fu) | __vcmpeq4(v[k].w & 0x7f7f7f7fu, 0x7f7f7f7fu)) != 0;
      }
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int key = (r + k) * kKeys + key_of;
      const uint32_t in[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
      uint32_t o[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[2 * e] = e4m3x2_to_f16x2(in[e] & 0xffffu);
        o[2 * e + 1] = e4m3x2_to_f16x2(in[e] >> 16);
      }
      unsigned char* row = tile + (key >> 3) * Cfg<D, true>::GROUP + (piece >> 2) * 1024 + (key & 7) * 128;
      const int p0 = 2 * (piece & 3), x = key & 7;
      *reinterpret_cast<uint4*>(row + ((p0 ^ x) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
      *reinterpret_cast<uint4*>(row + (((p0 + 1) ^ x) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
    }
  }
  fence_async_smem();
  __syncwarp();
  return odd;
}

template <int D, bool FP8>
__global__ void __launch_bounds__(kThreads, 1)
    chunk_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ CUtensorMap map_q, const __grid_constant__ ChunkParams p) {
  using C = Cfg<D, FP8>;
  constexpr int KST = C::KST, VST = C::VST, DH = C::DH;
  extern __shared__ __align__(1024) unsigned char smem[];  // at a fixed address: offsets cost no registers
  const uint32_t sbase = smem_u32(smem);
  if ((sbase & 1023u) != 0) {  // (the swizzle needs it; dynamic shared memory starts there)
    if (threadIdx.x == 0) set_status(p.status, SPEC_FLAG_TIMEOUT);
    return;
  }
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
  const uint32_t q_full = bar0 + 8u * (B0 + 6), q_free = bar0 + 8u * (B0 + 7);
  const uint32_t drain = bar0 + 8u * (B0 + 8);
  auto joined = [&](uint32_t j) { return bar0 + 8u * (B0 + 9 + (j & 1)); };  // twin j has joined its halves
  auto raw_full = [&](int kind) { return bar0 + 8u * (B0 + 11 + kind); };
  auto raw_empty = [&](int kind) { return bar0 + 8u * (B0 + 13 + kind); };
  uint32_t* misc = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NBAR; ++i) {
      const int at = i - static_cast<int>(B0);
      const bool made = FP8 && (i < KST || (i >= 2 * KST + 2 * VST && at < 0) || at >= 13);
      // k_full, v_ready, raw_empty of the 8-bit cache: the converters; p_full: the warps of an M tile;
      // joined: of both
      const int n = made ? kConverters : at == 2 || at == 3 ? kSoftWarps / 2 : at == 9 || at == 10 ? kSoftWarps : 1;
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

  if (FP8 && (warp == kSoftWarps || warp == kSoftWarps + 1 || warp == kSoftWarps + 3)) {
    // ============================ producer and converters of the 8-bit cache ============================
    // A tile of K, then of V: 16 brings them, each as soon as the one before is read, and leaves notes,
    // 17 and 19 make half of its values fp16 each: 522 us for two chunks of 2,048 tokens. A third converter
    // leaves the softmax 80 registers (536); one that also brings the tiles is late with them (780 where two
    // took 610).
    fewer_registers<FP8>();
    const int part = warp == kSoftWarps ? -1 : warp == kSoftWarps + 1 ? 0 : 1;  // -1: the producer
    RawTile* const notes = reinterpret_cast<RawTile*>(smem + C::OFF_RAWS);
    // tiles converted; stops + 1 of the last unit noted for redoing, by each converter (one word for both, in
    // shared memory: 533 us where two chunks of 2,048 tokens take 527)
    uint32_t made = 0, noted = 0;
    auto convert = [&](int kind) {
      const uint32_t st = made % (kind ? VST : KST), use = made / (kind ? VST : KST);
      wait(raw_full(kind), made & 1);
      if (use > 0) wait(kind ? v_empty(st) : k_empty(st), (use - 1) & 1);
      if (dead) return;
      const RawTile& t = notes[made & 3];
      const unsigned char* raw = smem + C::OFF_RAW + kind * C::RAW;
      if (kind) {
        const bool odd = convert_tile<D, true>(raw, smem + C::OFF_V + st * C::TILE, t, part);
        if (__any_sync(0xffffffffu, odd) && noted != t.stop + 1) {
          noted = t.stop + 1;
          if (lane == 0) {
            const int n = atomicAdd(&p.redo[0].x, 1);
            if (n < p.redo_cap) p.redo[1 + n] = make_int4(t.b, t.g, t.rt, 0);
          }
        }
      } else {
        convert_tile<D, false>(raw, smem + C::OFF_K + st * C::TILE, t, part);
      }
      if (lane == 0) {
        mbar_arrive(raw_empty(kind));
        mbar_arrive(kind ? v_ready(st) : k_full(st));
      }
      __syncwarp();
    };
    bool more = false;
    if (part >= 0) {
      if (!p.starve) {
        ChunkWalk first;
        more = first.begin(p, blockIdx.x);
      }
      while (more && !dead) {
#pragma unroll 1
        for (int kind = 0; kind < 2 && !dead; ++kind) convert(kind);
        if (!dead) more = notes[made & 3].more != 0;
        ++made;
      }
    } else {
      ChunkWalk& w = reinterpret_cast<ChunkWalk*>(smem + C::OFF_WALK)[kSoftWarps];  // (saves registers)
      if (lane == 0) more = !p.starve && w.begin(p, blockIdx.x);
      more = __any_sync(0xffffffffu, more);
      const int psh = __ffs(p.page_size) - 1;
      const uint32_t box = static_cast<uint32_t>(p.page_size) * D;
      const uint32_t qbytes = static_cast<uint32_t>(p.tile_tokens * p.group) * 128u;
      float4* const pages = reinterpret_cast<float4*>(smem + C::OFF_PAGES);
      uint32_t it = 0, copies = 0, seg = 0;  // tiles, and K or V of a tile, brought; stops
      uint32_t joins = 0, twins = 0;         // twins joined, of all whole ones so far
      bool was_twin = false;
      while (more && !dead) {
        __syncwarp();
        const ChunkUnit u = w.unit(p);
        const int b = w.b, g = w.g, rt = w.rt, row = w.row0 + u.token0;
        const int32_t* table = p.page_table + static_cast<int64_t>(b) * p.max_pages;
        const int tiles = w.tiles(u, 0) + (u.twin ? w.tiles(u, 1) : 0);
        int key0 = (u.tile0 + u.step_tiles(w.s0, 0)) * TK;
        const bool whole_twin = u.twin && w.whole(u);
        bool bad = false;
        // the walk goes ahead, so that the last tile can say that it is the last
        __syncwarp();
        more = false;
        if (lane == 0) more = w.next(p);
        more = __any_sync(0xffffffffu, more);
        // pages of the tile at key k with a key that the unit sees, a lane each: the ids of the tile
        // after the next one and the scales of the next one are in flight
        auto load_id = [&](int k) {
          const bool in = lane >= (max(k, u.low) - k >> psh) && lane <= (min(k + TK, u.high) - 1 - k >> psh);
          return in && k < u.high ? __ldg(table + (k >> psh) + lane) : 0;
        };
        auto load_scale = [&](int i) {
          return __ldg(reinterpret_cast<const float2*>(p.kv_scale) + static_cast<int64_t>(i >= 0 && i < p.num_pages ? i : 0) * p.hkv + g);
        };
        int id = load_id(key0), id_next = load_id(key0 + TK);
        float2 scale = load_scale(id);
        for (int x = 0; x < tiles && !dead; ++x, key0 += TK) {
          const int q0 = max(key0, u.low) - key0 >> psh, q1 = (min(key0 + TK, u.high) - 1 - key0 >> psh) + 1;
          const bool in_range = id >= 0 && id < p.num_pages;
          bad |= !in_range;
          const int at = 2 * ((in_range ? id : 0) * p.hkv + g);
          const float2 scale_next = load_scale(id_next);
          const int id_last = load_id(key0 + 2 * TK);
#pragma unroll 1
          for (int kind = 0; kind < 2; ++kind) {
            if (it > 0) wait(raw_empty(kind), (it - 1) & 1);
            if (dead) break;
            if (kind == 0) {
              if (lane == 0) notes[it & 3] = {u.low, u.high, u.full_low, u.full_high, key0, b, g, rt, seg, more || x + 1 < tiles};
              const float sv = clamp_scale(scale.y);
              // what the tile's scores and weights are to be scaled by
              if (lane < 8) pages[it % C::PT * 8 + lane] = make_float4(scale.x, log2f(sv), 1.f / sv, 0.f);
              __syncwarp();
            }
            if (elected()) mbar_arrive_tx(raw_full(kind), static_cast<uint32_t>(q1 - q0) * box);
            __syncwarp();
            if (lane >= q0 && lane < q1)
              tma_load_raw(sbase + C::OFF_RAW + kind * C::RAW + static_cast<uint32_t>(lane) * box, &map_k, at + kind, raw_full(kind));
            ++copies;
          }
          if (dead) break;
          ++it;
          id = id_next;
          id_next = id_last;
          scale = scale_next;
          if (x == 0) {
            // Q follows the first tile of keys, once the stop before is done with its own
            if (seg > 0) wait(q_free, (seg - 1) & 1);
            for (; joins < twins - (was_twin && u.twin ? 1 : 0) && !dead; ++joins) wait(joined(joins), joins >> 1 & 1);
            if (dead) break;
            if (lane == 0) {
              const int m_tiles = u.twin ? 1 : 2;
              mbar_arrive_tx(q_full, static_cast<uint32_t>(m_tiles * DH) * qbytes);
              for (int m = 0; m < m_tiles; ++m)
                for (int half = 0; half < DH; ++half)
                  tma_load_q(sbase + C::OFF_Q + m * C::QTILE + half * C::QHALF, &map_q, half, g * p.group,
                             row + m * p.tile_tokens, q_full);
            }
            __syncwarp();
          }
        }
        if (__any_sync(0xffffffffu, bad) && lane == 0) {  // the sequence is cleared at the end
          p.seq_bad[b] = 1;
          set_status(p.status, SPEC_FLAG_BAD_PAGE);
        }
        was_twin = whole_twin;
        twins += whole_twin ? 1 : 0;
        ++seg;
      }
      if (dead && copies > 0) {  // copies still in flight (bounded)
        const long long c0 = clock64();
        for (uint32_t kind = 0; kind < 2; ++kind) {
          const uint32_t n = (copies + 1 - kind) / 2;
          while (n > 0 && !mbar_try(raw_full(kind), (n - 1) & 1) && clock64() - c0 < kWaitCycles) {
          }
        }
        while (seg > 0 && !mbar_try(q_full, (seg - 1) & 1) && clock64() - c0 < kWaitCycles) {
        }
      }
    }
  } else if (warp == kSoftWarps || warp == kSoftWarps + 1) {
    // ============================ producers ============================
    fewer_registers<FP8>();
    ChunkWalk w;
    const bool is_k = warp == kSoftWarps;
    const uint32_t nst = is_k ? KST : VST, ring = sbase + (is_k ? C::OFF_K : C::OFF_V);
    const CUtensorMap* map = is_k ? &map_k : &map_v;
    const int psh = __ffs(p.page_size) - 1, npg = TK >> psh;
    const uint32_t box = static_cast<uint32_t>(p.page_size) * D * 2;
    const uint32_t qbytes = static_cast<uint32_t>(p.tile_tokens * p.group) * 128u;
    uint32_t it = 0, seg = 0, joins = 0, twins = 0;  // twins joined, of all whole ones so far
    bool was_twin = false;
    auto full = [&](uint32_t s) { return is_k ? k_full(s) : v_full(s); };
    auto empty = [&](uint32_t s) { return is_k ? k_empty(s) : v_empty(s); };
    for (bool more = !p.starve && w.begin(p, blockIdx.x); more && !dead; ++seg) {
      const ChunkUnit u = w.unit(p);
      const int32_t* table = p.page_table + static_cast<int64_t>(w.b) * p.max_pages;
      const int pages = (u.high - 1 >> psh) + 1;  // of the sequence, as far as the unit sees it
      // page ids, 32 at a time, the next 32 in flight
      int base = (u.tile0 + u.step_tiles(w.s0, 0)) * npg;
      auto load_id = [&](int at) { return at + lane < pages ? __ldg(table + at + lane) : 0; };
      int id = load_id(base), id_next = load_id(base + 32);
      bool bad = false, first = true;
      const int per = u.twin ? 2 : 1;
      for (int x = 0; x < w.ns * per && !dead; ++x) {
        const int i = w.s0 + x / per, h = x % per;
        if (!u.has(i, h)) continue;
        const int tile = u.tile0 + u.step_tiles(i, h), key0 = tile * TK, pg0 = tile * npg;
        while (pg0 >= base + 32) {
          base += 32;
          id = id_next;
          id_next = load_id(base + 32);
        }
        const uint32_t st = it % nst;
        if (it >= nst) wait(empty(st), (it / nst - 1) & 1);
        if (dead) break;
        // pages with a key that the unit sees
        const int q0 = max(key0, u.low) - key0 >> psh, q1 = (min(key0 + TK, u.high) - 1 - key0 >> psh) + 1;
        if (elected()) mbar_arrive_tx(full(st), static_cast<uint32_t>(q1 - q0) * box);
        __syncwarp();
        const int q = base + lane - pg0;
        if (q >= q0 && q < q1) {
          const bool in_range = id >= 0 && id < p.num_pages;
          bad |= !in_range;
          tma_load_page(ring + st * C::TILE + static_cast<uint32_t>(q) * box, map, (in_range ? id : 0) * p.hkv + w.g, full(st));
        }
        __syncwarp();
        ++it;
        if (is_k && first) {
          // Q follows the first tile of keys, once the segment before is done with its own
          if (seg > 0) wait(q_free, (seg - 1) & 1);
          // (the last twin joins in the second Q tile's place; its join is awaited a stop later
          // where that place is not needed)
          for (; joins < twins - (was_twin && u.twin ? 1 : 0) && !dead; ++joins) wait(joined(joins), joins >> 1 & 1);
          if (dead) break;
          if (lane == 0) {
            const int tiles = u.twin ? 1 : 2;
            mbar_arrive_tx(q_full, static_cast<uint32_t>(tiles * DH) * qbytes);
            for (int m = 0; m < tiles; ++m)
              for (int half = 0; half < DH; ++half)
                tma_load_q(sbase + C::OFF_Q + m * C::QTILE + half * C::QHALF, &map_q, half, w.g * p.group,
                           w.row0 + u.token0 + m * p.tile_tokens, q_full);
          }
          __syncwarp();
        }
        first = false;
      }
      if (__any_sync(0xffffffffu, bad) && lane == 0) {  // the sequence is cleared at the end
        p.seq_bad[w.b] = 1;
        set_status(p.status, SPEC_FLAG_BAD_PAGE);
      }
      was_twin = u.twin && w.whole(u);
      twins += was_twin ? 1 : 0;
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
    // The tensor core keeps about four products in its queue, so that a turn's waits and
    // book-keeping have to stay within their time: one copy of the code, waits before it, all
    // products and commits of a turn in one block of one lane.
    fewer_registers<FP8>();
    ChunkWalk w;
    // (fp16 operands: both type fields 0)
    constexpr uint32_t kHalf = FP8 ? ~((1u << 7) | (1u << 10)) : ~0u;
    constexpr uint32_t kIdescS = idesc_bf16(MR, TK, false) & kHalf, kIdescO = idesc_bf16(MR, D, true) & kHalf;
    const uint32_t q_low = desc_low(sbase + C::OFF_Q, 16), k_low = desc_low(sbase + C::OFF_K, 16),
                   v_low = desc_low(sbase + C::OFF_V, 1024);
    uint32_t ks = 0, vs = 0;       // stages of the next tiles of K and V
    uint32_t k_par = 0, v_par = 0; // and the parities of their barriers
    uint32_t q_par = 0, p_par = 0; // of Q, and a bit per M tile of its weights
    bool gone = false;             // of a lane; of all after a turn
    auto ready = [&](uint32_t bar, uint32_t parity) {
      if (!mbar_try(bar, parity)) gone = gone || !mbar_wait(bar, parity, abort_flag, p.status);
    };
    for (bool more = w.begin(p, blockIdx.x); more && !gone;) {
      int turns, first_last;  // of both M tiles together; M tile 1 of a twin may have a tile less
      bool twin;
      {
        const ChunkUnit u = w.unit(p);
        twin = u.twin;
        turns = 2 * w.ns;
        first_last = turns - (w.tiles(u, 1) < w.tiles(u, 0) ? 1 : 0);  // turns from here on have no tile
      }
      ready(q_full, q_par);
      q_par ^= 1;
#pragma unroll 1
      for (int x = -2; x < turns && !gone; ++x) {  // M tile x & 1: a step's products, the next step's scores
        const int h = x & 1;
        const bool weighed = x >= 0 && x < first_last, goes_on = x + 2 < first_last;
        const bool own = twin || h == 0, frees = twin || h == 1;  // both M tiles use one tile unless twin
        const uint32_t s_tmem = tmem + C::S_COL + h * TK, o_tmem = tmem + C::O_COL + h * D;
        const uint32_t vb = v_low + vs * (C::TILE >> 4), kb = k_low + ks * (C::TILE >> 4);
        const uint32_t qa = q_low + (twin ? 0 : h) * (C::QTILE >> 4), v_now = vs;
        if (goes_on && own) ready(k_full(ks), k_par);
        if (weighed) {
          if (own) ready(v_ready(vs), v_par);
          ready(p_full(h), p_par >> h & 1);
        }
        gone = __any_sync(0xffffffffu, gone);
        if (gone) break;
        tc_fence_after();
        if (weighed) {
          p_par ^= 1u << h;
          if (frees && ++vs == VST) {
            vs = 0;
            v_par ^= 1;
          }
        }
        if (elected()) {
          if (weighed) {
#pragma unroll
            for (int kk = 0; kk < TK / 16; ++kk)
              mma_ts(o_tmem, s_tmem + (kk / 4) * HK + (kk % 4) * 8u, vb + ((kk * 2u * C::GROUP) >> 4), desc_high(C::GROUP),
                     kIdescO, kk > 0 || x > 1);
            if (!goes_on) mma_commit(o_full(h));
            if (frees) mma_commit(v_empty(v_now));
          }
          if (goes_on) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              mma_ss(s_tmem, qa + (((kk / 4) * C::QHALF + (kk % 4) * 32u) >> 4), desc_high(1024),
                     kb + (((kk / 4) * 1024u + (kk % 4) * 32u) >> 4), desc_high(C::GROUP), kIdescS, kk > 0);
            mma_commit(s_full(h));
            if (frees) mma_commit(k_empty(ks));
          }
          if (x == turns - 3) mma_commit(q_free);  // the stop's last scores are issued
        }
        __syncwarp();
        if (goes_on && frees && ++ks == KST) {
          ks = 0;
          k_par ^= 1;
        }
      }
      more = w.next(p);
    }
    if (gone) {  // products still in flight (bounded)
      if (lane == 0) mma_commit(drain);
      __syncwarp();
      const long long c0 = clock64();
      while (!mbar_try(drain, 0) && clock64() - c0 < kWaitCycles) {
      }
    }
  } else if (!FP8 && warp == kSoftWarps + 3) {
    // ============================ finite values ============================
    fewer_registers<FP8>();
    ChunkWalk w;
    uint32_t vc = 0;
    for (bool more = w.begin(p, blockIdx.x); more && !dead;) {
      const ChunkUnit u = w.unit(p);
      bool odd = false;
      int key0 = (u.tile0 + u.step_tiles(w.s0, 0)) * TK;
      for (int n = w.tiles(u, 0) + (u.twin ? w.tiles(u, 1) : 0); n > 0; --n, key0 += TK, ++vc) {
        const uint32_t st = vc % VST;
        wait(v_full(st), (vc / VST) & 1);
        if (dead) break;
        if (key0 < u.full_low || key0 + TK > u.full_high) odd |= finite_values<D>(smem + C::OFF_V + st * C::TILE, key0, u);
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
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs<FP8>));
    // A thread's registers are the scarce thing here (spilled ones miss the little L1 that is left
    // beside the shared memory): the walk is kept in shared memory, by a warp's first lane, and
    // what a stop's ends need is worked out there anew.
    ChunkWalk& w = reinterpret_cast<ChunkWalk*>(smem + C::OFF_WALK)[warp];
    // M tile, half of a tile's keys (and of the outputs' columns), row of the M tile
    const int h = warp >> 3, ch = warp >> 2 & 1, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_col = tmem + lanes + C::S_COL + h * TK + ch * HK, o_col = tmem + lanes + C::O_COL + h * D + ch * (D / 2);
    float* const xch = reinterpret_cast<float*>(smem + C::OFF_XCH) + h * MR + row;
    const int pbar = 1 + h * 4 + (warp & 3), allbar = 9;
    float c = p.scale_log2;  // what a score is multiplied by (8-bit cache: of this row, before its key's scale)
    const float4* const pages = reinterpret_cast<const float4*>(smem + C::OFF_PAGES);
    const int psh = __ffs(p.page_size) - 1;
    uint32_t tiles = 0;  // of the block before the stop
    uint32_t sc = 0, oc = 0, joins = 0;  // tiles weighed, units ended, twins joined
    // f(own, the other thread's) of a row, in both of its threads
    auto joint = [&](float own, auto f) {
      if (ch == 1) *xch = own;
      bar_sync(pbar, 64);
      if (ch == 0) *xch = own = f(own, *xch);
      bar_sync(pbar, 64);
      return ch == 0 ? own : *xch;
    };
    auto settle = [&](uint32_t bar, uint32_t parity) {
      wait(bar, parity);
      tc_fence_after();
    };
    // this row's token among the unit's, or -1
    auto token_of = [&](bool twin, int tokens) {
      int r = row;
      asm volatile("" : "+r"(r));  // not kept from before
      const int token = (twin ? 0 : h * p.tile_tokens) + r / p.group;
      return r < p.tile_tokens * p.group && token < tokens ? token : -1;
    };
    Ended& ended = reinterpret_cast<Ended*>(smem + C::OFF_LAST)[warp];
    bool more = false;
    if (lane == 0) more = w.begin(p, blockIdx.x);
    for (more = __any_sync(0xffffffffu, more); more;) {
      __syncwarp();
      int n, whole_from, whole_to;  // this M tile's tiles at the stop; those that all rows see fully
      bool twin_stop;
      uint32_t reals;               // rows of a token
      {
        const ChunkUnit u = w.unit(p);
        const int key0 = (u.tile0 + u.step_tiles(w.s0, h)) * TK;
        const int step = u.twin ? 2 * TK : TK;
        twin_stop = u.twin;
        n = w.tiles(u, h);
        whole_from = (max(u.full_low - key0, 0) + step - 1) / step;
        whole_to = u.full_high - key0 >= TK ? (u.full_high - key0 - TK) / step + 1 : 0;
        const int token = token_of(u.twin, u.tokens);
        reals = __ballot_sync(0xffffffffu, token >= 0);
        if constexpr (FP8) {
          if (token >= 0)
            c = p.scale_log2 * __ldg(p.q_scale + (static_cast<int64_t>(w.row0) + u.token0 + token) * p.hq + w.g * p.group + row % p.group);
        }
      }
      float m = -INFINITY, l = 0.f;  // the row's reference, a score; the sum of this thread's weights
      for (int k = 0; k < n; ++k) {
        settle(s_full(h), sc & 1);
        ++sc;
        if (reals) {
          const bool partial = k < whole_from || k >= whole_to;  // some row does not see all
          if (partial) {  // hidden keys' scores become -inf in place
            const ChunkUnit u = w.unit(p);
            // (rows of no token see what the last one sees, nothing stale)
            const int token = token_of(u.twin, u.tokens), at = w.kv_len - w.n + u.token0 + (token < 0 ? u.tokens - 1 : token);
            const int key0 = (u.tile0 + u.step_tiles(w.s0, h) + (u.twin ? 2 * k : k)) * TK + ch * HK;
            const int from = chunk_low(p, at) - key0, to = chunk_high(p, at, w.kv_len) - key0;  // columns that this row sees
#pragma unroll 1
            for (int g = 0; g < HK; g += 32) {
              const uint32_t above = to - g >= 32 ? ~0u : to - g <= 0 ? 0u : (1u << (to - g)) - 1u;
              const uint32_t below = from - g >= 32 ? ~0u : from - g <= 0 ? 0u : (1u << (from - g)) - 1u;
              const uint32_t seen = above & ~below;
              uint32_t r[32];
              tmem_ld32(s_col + g, r);
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 32; ++j) r[j] = (seen >> j & 1) ? r[j] : 0xff800000u;
              tmem_st32(s_col + g, r);
            }
            tmem_wait_st();
          }
          // 8-bit cache: exponents are s a + b, with a and b of the key's page: a the scales of the row, of
          // the keys and of the softmax, b the logarithm of the values' scale, so that the products
          // take the values as they are; a is not 0, so that a * -inf stays -inf
          const float4* const page = pages + (tiles + (twin_stop ? 2 * k + h : k)) % C::PT * 8;
          auto page_of = [&](int g) { return page[(ch * HK + g) >> psh]; };
          auto slope = [&](const float4& q) { return fmaxf(q.x * c, 1.17549435e-38f); };
          // scores are loaded twice, 32 at a time, which leaves registers for four warps a scheduler
          float top = -INFINITY;
#pragma unroll
          for (int g = 0; g < HK; g += 32) {
            float s[32];
            tmem_ld32(s_col + g, reinterpret_cast<uint32_t*>(s));
            tmem_wait_ld();
            if constexpr (FP8) {
#pragma unroll
              for (int e = 0; e < 32; e += 16) {
                float t0 = fmaxf(s[e], s[e + 1]), t1 = fmaxf(s[e + 2], s[e + 3]);
#pragma unroll
                for (int j = 4; j < 16; j += 4) {
                  t0 = max3(t0, s[e + j], s[e + j + 1]);
                  t1 = max3(t1, s[e + j + 2], s[e + j + 3]);
                }
                const float4 q = page_of(g + e);
                top = fmaxf(top, fmaf(fmaxf(t0, t1), slope(q), q.y));
              }
            } else {
              float t0 = fmaxf(s[0], s[1]), t1 = fmaxf(s[2], s[3]);
#pragma unroll
              for (int j = 4; j < 32; j += 4) {
                t0 = max3(t0, s[j], s[j + 1]);
                t1 = max3(t1, s[j + 2], s[j + 3]);
              }
              top = max3(top, t0, t1);
            }
          }
          // raise the row's reference where a weight would pass 2^8 (and at first); 8-bit cache: 2^15, to
          // where the largest is 2^8, because fp16 weights have steps of 2^-24 below 2^-14
          auto raises = [&](float x) {
            return x > m && (m == -INFINITY || (FP8 ? x - m > 15.f : (x - m) * c > 8.f));
          };
          if (pair_any(pbar, raises(top))) {
            const float both = joint(top, [](float x, float y) { return fmaxf(x, y); });
            const float now = raises(both) ? (FP8 ? both - 8.f : both) : m;
            const float alpha = m == -INFINITY ? 0.f : ex2(FP8 ? m - now : (m - now) * c);
            if (k > 0 && __any_sync(0xffffffffu, now != m && m != -INFINITY)) {
              // (the scores are done, so the products before them, which O holds, are too)
#pragma unroll 1
              for (int c0 = 0; c0 < D / 2; c0 += 16) {
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
          float neg = m == -INFINITY ? 0.f : FP8 ? -m : -__fmul_ru(m, c);
          const bool far = fabsf(neg) > kFar;
          if (__any_sync(0xffffffffu, far)) {  // the reference is taken off the scores (exponents) themselves
#pragma unroll 1
            for (int g = 0; g < HK; g += 16) {
              uint32_t r[16];
              tmem_ld16(s_col + g, r);
              const float4 q = FP8 ? page_of(g) : make_float4(0.f, 0.f, 0.f, 0.f);
              const float slope_g = FP8 ? slope(q) : 1.f;
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const float x = __uint_as_float(r[j]), e = FP8 ? fmaf(x, slope_g, q.y) : x;
                r[j] = far ? __float_as_uint(e - m) : r[j];
              }
              tmem_st16(s_col + g, r);
            }
            tmem_wait_st();
            neg = far ? 0.f : neg;
          }
          float a0 = 0.f, a1 = 0.f, a2 = 0.f, a3 = 0.f;
          if constexpr (FP8) {
#pragma unroll
            for (int g = 0; g < HK; g += 16) {
              float s[16];
              tmem_ld16(s_col + g, reinterpret_cast<uint32_t*>(s));
              const float4 q = page_of(g);
              const float a = far ? 1.f : slope(q), b = far ? 0.f : q.y + neg;
              tmem_wait_ld();
              uint32_t pk[8];
#pragma unroll
              for (int j = 0; j < 16; j += 2) {
                fma2(s[j], s[j + 1], a, b);
                const float x = ex2(s[j]), y = ex2(s[j + 1]);
                if (j & 2) addmul2(a2, a3, x, y, q.z); else addmul2(a0, a1, x, y, q.z);
                pk[j / 2] = pack_f16(x, y);
              }
              tmem_st8(s_col + g / 2, pk);
            }
          } else {
#pragma unroll
            for (int g = 0; g < HK; g += 32) {
              float s[32];
              tmem_ld32(s_col + g, reinterpret_cast<uint32_t*>(s));
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 32; j += 2) fma2(s[j], s[j + 1], c, neg);
              uint32_t pk[16];
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                const float x = ex2(s[j]), y = ex2(s[j + 1]);
                if (j & 2) add2(a2, a3, x, y); else add2(a0, a1, x, y);
                pk[j / 2] = pack_bf16(x, y);
              }
              tmem_st16(s_col + g / 2, pk);
            }
          }
          l += (a0 + a1) + (a2 + a3);
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(h));
      }
      if constexpr (FP8) {
        const ChunkUnit u = w.unit(p);
        tiles += w.tiles(u, 0) + (u.twin ? w.tiles(u, 1) : 0);
      }
      // ---- the unit's outputs ----
      if (reals) l = joint(l, [](float x, float y) { return x + y; });
      const bool had = n > 0;
      more = false;
      if (lane == 0) {  // the walk goes on while the last products run
        const ChunkUnit u = w.unit(p);
        ended.row = w.row0 + u.token0;
        ended.what = u.tokens | (u.twin ? kTwin : 0) | (w.whole(u) ? kWhole : 0) | (w.starts_unit() ? kStarts : 0);
        ended.g = w.g;
        more = w.next(p);
      }
      more = __any_sync(0xffffffffu, more);
      if (had) {
        settle(o_full(h), oc & 1);
        ++oc;
      }
      const int what = ended.what;
      const bool twin = what & kTwin, whole = what & kWhole;
      const int token = token_of(twin, what & 0xffff);
      const bool real = token >= 0;
      const float mc = m == -INFINITY ? -INFINITY : FP8 ? m : fabsf(m * c) > kFar ? m * c : __fmul_ru(m, c);
      const int64_t out_row = (static_cast<int64_t>(ended.row) + token) * p.hq + ended.g * p.group + row % p.group;
      __nv_bfloat16* const out = static_cast<__nv_bfloat16*>(p.out);
      // stores 32 columns of the warp's rows, from column c0 of this thread's half
      auto store = [&](const uint32_t* pk, int c0) {
        uint4 q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = make_uint4(pk[4 * k], pk[4 * k + 1], pk[4 * k + 2], pk[4 * k + 3]);
        turn_quad(q, lane);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int from = (lane & ~3) + k;
          const int64_t r = __shfl_sync(0xffffffffu, out_row, from);
          if (reals >> from & 1) *reinterpret_cast<uint4*>(out + r * D + ch * (D / 2) + c0 + (lane & 3) * 8) = q[k];
        }
      };
      if (whole && twin) {
        // the two M tiles hold the same rows: the second hands its part over in shared memory (the
        // second Q tile's, unused here), 16 columns of each half at a time
        constexpr int CP = 16;
        float* const place = reinterpret_cast<float*>(smem + C::OFF_Q + C::QTILE) + ch * CP * MR;
        float2* const other = reinterpret_cast<float2*>(smem + C::OFF_XCH);
        float w0 = 1.f, w1 = 0.f;  // what each part counts for; w1 < 0: it saw no key, and may have left nothing
        bar_sync(allbar, 32 * kSoftWarps);  // both M tiles have their sums
        if (h == 1 && ch == 0) other[row] = make_float2(had ? mc : -INFINITY, had ? l : 0.f);
#pragma unroll 1
        for (int c0 = 0; c0 < D / 2; c0 += CP) {
          uint32_t o[CP];
          if (had) {
            tmem_ld16(o_col + c0, o);
            tmem_wait_ld();
          }
          if (h == 1 && had && reals) {
#pragma unroll
            for (int k = 0; k < CP; ++k) place[k * MR + row] = __uint_as_float(o[k]);
          }
          bar_sync(allbar, 32 * kSoftWarps);
          if (h == 0 && reals) {
            if (c0 == 0) {
              const float2 ml = other[row];
              const float top = fmaxf(mc, ml.x);
              w0 = mc == -INFINITY ? 0.f : ex2(mc - top);
              w1 = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
              const float total = l * w0 + ml.y * w1;
              if (real && p.lse && ch == 0) p.lse[out_row] = (top + log2f(total)) * 0.6931471805599453f;
              const float inv = 1.f / total;
              w0 *= inv;
              w1 = ml.x == -INFINITY && ml.y == 0.f ? -1.f : w1 * inv;
            }
            uint32_t pk[CP / 2];
#pragma unroll
            for (int k = 0; k < CP; k += 2) {
              float x = __uint_as_float(o[k]) * w0, y = __uint_as_float(o[k + 1]) * w0;
              if (!(w1 < 0.f)) {
                x = fmaf(place[k * MR + row], w1, x);
                y = fmaf(place[(k + 1) * MR + row], w1, y);
              }
              pk[k / 2] = pack_bf16(x, y);
            }
            if (real) {
#pragma unroll
              for (int k = 0; k < CP / 8; ++k)
                reinterpret_cast<uint4*>(out + out_row * D + ch * (D / 2) + c0)[k] =
                    make_uint4(pk[4 * k], pk[4 * k + 1], pk[4 * k + 2], pk[4 * k + 3]);
            }
          }
          bar_sync(allbar, 32 * kSoftWarps);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(joined(joins));
        ++joins;
      } else if (whole) {
        const float inv = 1.f / l;  // every row sees a key: a sum of 0 (scores of -inf) is NaN
        if (reals) {
#pragma unroll 1
          for (int c0 = 0; c0 < D / 2; c0 += 32) {
            uint32_t o[32], pk[16];
            tmem_ld32(o_col + c0, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 32; k += 2) pk[k / 2] = pack_bf16(__uint_as_float(o[k]) * inv, __uint_as_float(o[k + 1]) * inv);
            store(pk, c0);
          }
          if (real && p.lse && ch == 0) p.lse[out_row] = (mc + log2f(l)) * 0.6931471805599453f;
        }
      } else if (reals) {
        // a part: its place is the block's second where it starts the unit, else its first
        const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (what & kStarts ? 1 : 0);
        if (had) {
#pragma unroll 1
          for (int c0 = 0; c0 < D / 2; c0 += 32) {
            uint32_t o[32];
            tmem_ld32(o_col + c0, o);
            tmem_wait_ld();
            float4* const part = reinterpret_cast<float4*>(p.partial_o) + (slot * (D / 4) + (ch * (D / 2) + c0) / 4) * (2 * MR) + h * MR + row;
            if (real) {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                part[k * 2 * MR] = make_float4(__uint_as_float(o[4 * k]), __uint_as_float(o[4 * k + 1]),
                                               __uint_as_float(o[4 * k + 2]), __uint_as_float(o[4 * k + 3]));
            }
          }
        }
        if (real && ch == 0) p.partial_ml[slot * (2 * MR) + h * MR + row] = make_float2(had ? mc : -INFINITY, had ? l : 0.f);
      }
      tc_fence_before();
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

// The 8-bit cache viewed as (bytes of a key; keys of a page; page, head and kind), the box the keys or
// the values of one page and KV head, as they are.
bool encode_raw(CUtensorMap* map, const spec_chunk_attn_args_t& a) {
  EncodeTiledFn enc = encoder();
  if (!enc) return false;
  const cuuint64_t D = a.head_dim, P = a.page_size;
  const cuuint64_t dims[3] = {D, P, 2 * static_cast<cuuint64_t>(a.num_pages) * a.num_kv_heads};
  const cuuint64_t strides[2] = {D, D * P};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(D), static_cast<cuuint32_t>(P), 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(a.kv_cache), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Q viewed as (64 columns; column halves; heads; rows), the box one column half of an M tile: the
// group's heads of tile_tokens rows. Rows past the last read zeros.
bool encode_q(CUtensorMap* map, const spec_chunk_attn_args_t& a, const ChunkParams& p) {
  EncodeTiledFn enc = encoder();
  if (!enc) return false;
  const cuuint64_t D = a.head_dim;
  const cuuint64_t dims[4] = {64, D / 64, static_cast<cuuint64_t>(a.num_q_heads), static_cast<cuuint64_t>(a.rows)};
  // the 8-bit cache's queries are the dense fp16 ones
  const int64_t stride = a.kv_cache ? static_cast<int64_t>(a.num_q_heads) * a.head_dim : p.q_stride;
  const cuuint64_t strides[3] = {128, D * 2, static_cast<cuuint64_t>(stride) * 2};
  const cuuint32_t box[4] = {64, 1, static_cast<cuuint32_t>(p.group), static_cast<cuuint32_t>(p.tile_tokens)};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(map, a.kv_cache ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
             a.kv_cache ? p.q_half : const_cast<void*>(a.q), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool FP8>
cudaError_t launch_d(const spec_chunk_attn_args_t& a, const ChunkParams& p, cudaStream_t stream) {
  CUtensorMap mk, mv, mq;
  if (!encode_q(&mq, a, p)) return cudaErrorInvalidValue;
  if (FP8) {
    if (!encode_raw(&mk, a)) return cudaErrorInvalidValue;
    mv = mk;
  } else if (!encode_cache(&mk, a.k_cache, a) || !encode_cache(&mv, a.v_cache, a)) {
    return cudaErrorInvalidValue;
  }
  constexpr size_t smem = Cfg<D, FP8>::SMEM;
  const cudaError_t e = cudaFuncSetAttribute(chunk_tc_kernel<D, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  return launch_overlapped(chunk_tc_kernel<D, FP8>, dim3(p.blocks), kThreads, smem, stream, mk, mv, mq, p);
}

}  // namespace

cudaError_t launch_chunk_tc(const spec_chunk_attn_args_t& a, const ChunkParams& p, cudaStream_t stream) {
  if (a.kv_cache) return a.head_dim == 128 ? launch_d<128, true>(a, p, stream) : launch_d<64, true>(a, p, stream);
  return a.head_dim == 128 ? launch_d<128, false>(a, p, stream) : launch_d<64, false>(a, p, stream);
}

}  // namespace specv
