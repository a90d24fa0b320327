// Internal declarations of the operators that serve ragged batches of new tokens: rotary
// positions with the cache write, attention of chunks over the paged caches, forked sequences
// and page copies.
#pragma once

#include <cmath>

#include "common.cuh"

namespace specv {

cudaError_t launch_rope(const spec_rope_args_t& a, int sms, cudaStream_t stream);
cudaError_t launch_fork(const spec_fork_args_t& a, char* ws, cudaStream_t stream);
size_t fork_smem(int batch);
cudaError_t launch_copy(const spec_copy_args_t& a, cudaStream_t stream);

// --- attention of chunks ---
struct ChunkPlan {
  int path;          // SPEC_ATTN_CUDA_CORES or SPEC_ATTN_TENSOR_CORES
  int fp8;           // the cache is the 8-bit one
  int tile_tokens;   // tensor cores: tokens of an M tile, 128 / group
  int grid;          // tensor cores: blocks
  int max_units;     // units per KV head, at most
  int redo_cap;      // tensor cores: notes of units that have to be computed again, at most
  size_t seqs, bad, cum, work, redo, partial_o, partial_ml, q_half, q_scale, end;
};
bool chunk_tc_fits(const spec_chunk_attn_args_t& a);
ChunkPlan chunk_plan(const spec_chunk_attn_args_t& a, size_t base, int num_sms, int path);
constexpr int kChunkKeyTile = 128;     // keys of a tile on the tensor cores
constexpr int kChunkTileRows = 128;    // query rows of an M tile
constexpr int kChunkConverters = 2;    // warps that convert the 8-bit cache's tiles
// The work list counts in virtual steps: what a step costs (a twin's reads twice the bytes for the same
// products), and what a unit's start costs (its queries, the pipeline's refill, the outputs before).
// 60 requests decoding beside four chunks take 668 us; with a step of either kind at 1 and a start at
// 3 they take 778, with a twin's step at 2 and a start at 4, 745.
constexpr int kChunkCost = 3, kChunkTwinCost = 4;
constexpr int kChunkStart = 12, kChunkTwinStart = 10;
// 8-bit cache: a tile takes its conversion's time whichever unit it is for, so a twin's step takes twice
// another's, and starts weigh a third as much: that batch 964 us, with the weights above 987; four whole
// prompts 586, with starts of 6 and 5 595, of 12 and 8 615.
constexpr int kChunkCost8 = 2;
constexpr int kChunkStart8 = 4, kChunkTwinStart8 = 3;

// One sequence of the batch, as the setup leaves it.
struct ChunkSeq {
  int row0, n;     // its rows of q; n = 0: nothing to do
  int kv_len;
  int first_unit;  // its first unit among all
};
// The work list of the tensor-core kernel, and where each block starts in it: the sequence and what is
// known of it, the KV head, the unit of its tokens, the virtual step in it, and the steps to take.
struct alignas(16) ChunkStart {
  int b, g, rt, off;
  int row0, n, kv_len, left;
};
struct ChunkWork {
  long long total;
  int active, pad;       // blocks with work
  ChunkStart starts[1];  // [blocks], left = 0 without work
};

struct ChunkParams {
  int batch, rows, hq, hkv, group;
  int page_size, max_pages, num_pages, max_keys;
  int causal, window;  // window 0: none
  float scale_log2;    // softmax_scale * log2(e)
  int64_t q_stride;    // elements
  const void* q;
  const void* k_cache;  // the 8-bit cache, if kv_scale is given
  const void* v_cache;
  const float* kv_scale;
  const int32_t* page_table;
  const int32_t* row_start;
  const int32_t* kv_len;
  void* out;
  float* lse;
  uint32_t* status;
  int32_t* seq_bad;  // [batch]: its rows become out = 0, lse = -inf at the end
  ChunkSeq* seqs;    // [batch + 1]
  int max_units;     // there is room for: tensor cores, a ChunkUnit each; CUDA cores, blocks of kSimtRowTile query rows
  // tensor cores (blocks = 0: not used)
  int tile_tokens, blocks;
  long long* cum;      // [max_units + 1]: virtual steps before a unit, for one KV head
  ChunkWork* work;
  int4* redo;          // [0].x: how many; then (sequence, KV head, unit) to compute again
  int redo_cap;
  float* partial_o;    // [2 * blocks][D / 4][2 * kChunkTileRows][4]
  float2* partial_ml;  // [2 * blocks][2 * kChunkTileRows] = (m, l)
  void* q_half;        // 8-bit cache: [rows][Hq][D] fp16, each row scaled by a power of two
  float* q_scale;      // 8-bit cache: [rows][Hq], what its scores are to be multiplied by
  int starve;          // test hook: the producers issue no copies, so the waits run out
};

cudaError_t launch_chunk(const spec_chunk_attn_args_t& a, const ChunkPlan& P, char* ws, cudaStream_t stream,
                         bool starve = false);
cudaError_t launch_chunk_tc(const spec_chunk_attn_args_t& a, const ChunkParams& p, cudaStream_t stream);

#ifdef __CUDACC__
// Whether rows [r0, r1) are rows of q.
__device__ __forceinline__ bool chunk_rows_ok(const ChunkParams& p, int r0, int r1) {
  return r0 >= 0 && r1 >= r0 && r1 <= p.rows;
}
// The keys [low, high) that the token at position `at` of a sequence of n keys sees.
__device__ __forceinline__ int chunk_low(const ChunkParams& p, int at) {
  return p.window > 0 ? max(0, at - p.window + 1) : 0;
}
__device__ __forceinline__ int chunk_high(const ChunkParams& p, int at, int n) { return p.causal ? at + 1 : n; }

// A unit of the tensor-core kernel: the query rows of up to 2 * tile_tokens tokens of a sequence
// and one KV head, in two M tiles; with no more than one tile of tokens both M tiles hold the same
// rows and take every second tile of keys each ("twin"). Its work is counted in steps: a tile of
// keys for both M tiles, or, twin, one for each.
struct ChunkUnit {
  int token0, tokens;  // of the sequence's new tokens
  int low, high;       // keys that any of them sees
  int full_low, full_high;  // keys that all of them see
  int tile0, tiles, steps;
  bool twin, eight;  // of the 8-bit cache
  __device__ __forceinline__ int start() const {
    return eight ? (twin ? kChunkTwinStart8 : kChunkStart8) : (twin ? kChunkTwinStart : kChunkStart);
  }
  __device__ __forceinline__ int length() const { return start() + steps * (twin ? kChunkTwinCost : eight ? kChunkCost8 : kChunkCost); }
  // the first step that begins at or after virtual step v of the unit
  __device__ __forceinline__ int step_at(int v) const {
    const int x = max(v - start(), 0);
    return twin ? (x + kChunkTwinCost - 1) / kChunkTwinCost
                : eight ? (x + kChunkCost8 - 1) / kChunkCost8 : (x + kChunkCost - 1) / kChunkCost;
  }
  __device__ __forceinline__ int step_tiles(int i, int h) const { return twin ? 2 * i + h : i; }
  __device__ __forceinline__ bool has(int i, int h) const { return !twin || 2 * i + h < tiles; }
};
__device__ __forceinline__ int chunk_units(const ChunkParams& p, int n) {
  return (n + 2 * p.tile_tokens - 1) / (2 * p.tile_tokens);
}
__device__ __forceinline__ ChunkUnit chunk_unit(const ChunkParams& p, const ChunkSeq& s, int rt) {
  ChunkUnit u;
  u.token0 = rt * 2 * p.tile_tokens;
  u.tokens = min(2 * p.tile_tokens, s.n - u.token0);
  u.twin = u.tokens <= p.tile_tokens;
  u.eight = p.kv_scale != nullptr;
  const int at0 = s.kv_len - s.n + u.token0, at1 = at0 + u.tokens - 1;
  u.low = chunk_low(p, at0);
  u.full_low = chunk_low(p, at1);
  u.full_high = chunk_high(p, at0, s.kv_len);
  u.high = chunk_high(p, at1, s.kv_len);
  u.tile0 = u.low / kChunkKeyTile;
  u.tiles = (u.high + kChunkKeyTile - 1) / kChunkKeyTile - u.tile0;
  u.steps = u.twin ? (u.tiles + 1) / 2 : u.tiles;
  return u;
}

// A walk over a block's part of the work list: each stop is a run of steps of one unit. All roles
// of a block (and the joining of split units) walk alike. Units follow one another within a KV
// head, then the heads of a sequence, then the sequences. The walk keeps few values, and gives the
// stop's unit anew where it is asked for, because it lives beside loops that need the registers.
struct ChunkWalk {
  int left;          // virtual steps of the range behind the stop
  int b, g, rt;
  int row0, n, kv_len;
  int s0, ns;        // the stop's first step, and how many
  __device__ __forceinline__ void enter(const ChunkParams& p) {
    const ChunkSeq s = p.seqs[b];
    row0 = s.row0;
    n = s.n;
    kv_len = s.kv_len;
  }
  __device__ __forceinline__ ChunkUnit unit(const ChunkParams& p) const {
    int r = rt;
    asm volatile("" : "+r"(r));  // not kept from before
    return chunk_unit(p, {row0, n, kv_len, 0}, r);
  }
  __device__ __forceinline__ void stop(const ChunkParams& p, int off) {
    const ChunkUnit u = chunk_unit(p, {row0, n, kv_len, 0}, rt);
    const int take = min(u.length() - off, left);
    s0 = u.step_at(off);
    ns = u.step_at(off + take) - s0;
    left -= take;
  }
  // The first stop of a range that begins at the very end of a unit has no step, and is passed. A range may
  // lie wholly within a unit's start: it has none at all, and the unit's steps are the next block's.
  __device__ __forceinline__ bool begin(const ChunkParams& p, int block) {
    const int4* at = reinterpret_cast<const int4*>(&p.work->starts[block]);
    const int4 x = at[0], y = at[1];
    b = x.x; g = x.y; rt = x.z;
    row0 = y.x; n = y.y; kv_len = y.z; left = y.w;
    if (left == 0) return false;
    stop(p, x.w);
    return ns > 0 || next(p);
  }
  __device__ __forceinline__ bool next(const ChunkParams& p) {
    // nothing, or no more than a unit's start
    if (left <= (p.kv_scale ? min(kChunkStart8, kChunkTwinStart8) : min(kChunkStart, kChunkTwinStart))) return false;
    if (++rt == chunk_units(p, n)) {
      rt = 0;
      if (++g == p.hkv) {
        g = 0;
        do {
          ++b;
          enter(p);
        } while (n == 0 && b < p.batch);
      }
    }
    stop(p, 0);
    return ns > 0;
  }
  __device__ __forceinline__ bool starts_unit() const { return s0 == 0; }
  __device__ __forceinline__ bool ends_unit(const ChunkUnit& u) const { return s0 + ns == u.steps; }
  __device__ __forceinline__ bool whole(const ChunkUnit& u) const { return ns == u.steps; }
  // tiles of M tile h at this stop
  __device__ __forceinline__ int tiles(const ChunkUnit& u, int h) const {
    return u.twin ? max((min(2 * (s0 + ns), u.tiles) - 2 * s0 + 1 - h) / 2, 0) : ns;
  }
};
#endif

}  // namespace specv
