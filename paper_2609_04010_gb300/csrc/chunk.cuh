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
  int path;        // SPEC_ATTN_CUDA_CORES or SPEC_ATTN_TENSOR_CORES
  int fp8;         // the cache is the 8-bit one
  int tile_tokens; // tensor cores: tokens of an M tile, 128 / group
  int grid;        // tensor cores: blocks
  int max_units;   // tensor cores: token tiles of all sequences, at most
  int64_t slots;   // tensor cores: partial results
  size_t seqs, cum, starts, redo, partial_o, partial_ml, end;
};
ChunkPlan chunk_plan(const spec_chunk_attn_args_t& a, size_t base, int num_sms, int path);
constexpr int kChunkSlotRows = 256;

// One sequence of the batch, as the setup leaves it.
struct ChunkSeq {
  int row0, n;     // its rows of q; n = 0: nothing to do
  int kv_len;
  int first_unit;  // its first token tile among all (tensor cores)
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
  ChunkSeq* seqs;    // [batch]
  // tensor cores
  int tile_tokens, tile_rows, max_units, blocks, overhead;
  int64_t* cum;      // [max_units + 1]: steps before a token tile, per KV head
  int4* starts;      // [blocks + 1]
  int4* redo;        // [0].x: how many; then units whose values have to be taken apart
  int redo_cap;
  float* partial_o;    // [slot][kChunkSlotRows][D]
  float2* partial_ml;  // [slot][kChunkSlotRows] = (m, l)
  int starve;          // test hook: the producers issue no copies, so the waits run out
};

ChunkParams make_chunk_params(const spec_chunk_attn_args_t& a, const ChunkPlan& P, char* ws);
cudaError_t launch_chunk(const spec_chunk_attn_args_t& a, const ChunkPlan& P, char* ws, cudaStream_t stream);
cudaError_t launch_chunk_tc(const spec_chunk_attn_args_t& a, const ChunkPlan& P, const ChunkParams& p,
                            cudaStream_t stream, bool starve);

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
#endif

}  // namespace specv
