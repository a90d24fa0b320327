// The C ABI of the operators that serve ragged batches (include/spec_verify.h): host-side
// argument checks, workspace layout and launches.
#include <climits>
#include <initializer_list>

#include "chunk.cuh"

using namespace specv;

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool bad_ws(const void* ws) { return !ws || !aligned(ws, kWsAlign); }
bool head_dim_ok(int d) { return d == 64 || d == 128; }
bool page_size_ok(int p) { return p == 16 || p == 32 || p == 64; }
// a row stride: 0 for dense rows, else at least a row and a multiple of 8 elements
bool stride_ok(int64_t s, int64_t dense) { return s == 0 || (s >= dense && s % 8 == 0); }

spec_status_t check_rope(const spec_rope_args_t* a) {
  if (!a || a->rows < 0 || a->num_q_heads < 0 || a->num_kv_heads < 0 || a->head_dim < 1 || a->rot_dim < 1)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (a->interleaved != 0 && a->interleaved != 1) return SPEC_ERR_INVALID_ARGUMENT;
  if (!(a->factor >= 0.f && a->factor < 1e30f)) return SPEC_ERR_INVALID_ARGUMENT;
  if (!head_dim_ok(a->head_dim)) return SPEC_ERR_UNSUPPORTED;
  if (a->rot_dim > a->head_dim) return SPEC_ERR_INVALID_ARGUMENT;
  if (a->rot_dim % 16 != 0) return SPEC_ERR_UNSUPPORTED;
  const int64_t heads = static_cast<int64_t>(a->num_q_heads) + 2 * static_cast<int64_t>(a->num_kv_heads);
  if (heads * (a->head_dim / 16) > (1 << 20)) return SPEC_ERR_UNSUPPORTED;
  const int64_t dq = static_cast<int64_t>(a->num_q_heads) * a->head_dim, dk = static_cast<int64_t>(a->num_kv_heads) * a->head_dim;
  if (!stride_ok(a->q_row_stride, dq) || !stride_ok(a->k_row_stride, dk) || !stride_ok(a->v_row_stride, dk) ||
      !stride_ok(a->q_out_row_stride, dq) || !stride_ok(a->k_out_row_stride, dk))
    return SPEC_ERR_INVALID_ARGUMENT;
  for (const void* p : {a->q, a->k, a->v, static_cast<const void*>(a->q_out), static_cast<const void*>(a->k_out),
                        static_cast<const void*>(a->k_cache), static_cast<const void*>(a->v_cache)})
    if (!aligned(p, 16)) return SPEC_ERR_INVALID_ARGUMENT;
  if (!aligned(a->turns, 8) || !aligned(a->positions, 4) || !aligned(a->slots, 4) || !aligned(a->status, 4))
    return SPEC_ERR_INVALID_ARGUMENT;
  if (a->slots) {
    if (!a->k_cache || !a->v_cache || a->num_kv_heads < 1 || a->num_pages < 1 || a->page_size < 1)
      return SPEC_ERR_INVALID_ARGUMENT;
    if (!page_size_ok(a->page_size) || static_cast<int64_t>(a->num_pages) * a->page_size > INT32_MAX)
      return SPEC_ERR_UNSUPPORTED;
  }
  if (a->rows == 0) return SPEC_OK;
  if (!a->positions || !a->turns) return SPEC_ERR_INVALID_ARGUMENT;
  // what is given goes somewhere, and what goes somewhere is given
  if ((a->q != nullptr) != (a->q_out != nullptr) || (a->q && a->num_q_heads < 1)) return SPEC_ERR_INVALID_ARGUMENT;
  if ((a->k != nullptr) != (a->k_out != nullptr || a->slots != nullptr) || (a->k && a->num_kv_heads < 1))
    return SPEC_ERR_INVALID_ARGUMENT;
  if ((a->v != nullptr) != (a->slots != nullptr)) return SPEC_ERR_INVALID_ARGUMENT;
  if (!a->q && !a->k) return SPEC_ERR_INVALID_ARGUMENT;
  return SPEC_OK;
}

spec_status_t check_chunk(const spec_chunk_attn_args_t* a) {
  if (!a || a->batch < 1 || a->rows < 0 || a->num_q_heads < 1 || a->num_kv_heads < 1 || a->max_pages_per_seq < 1 ||
      a->num_pages < 1 || a->page_size < 1 || a->head_dim < 1 || a->num_q_heads % a->num_kv_heads != 0 || a->window < 0)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (a->causal != 0 && a->causal != 1) return SPEC_ERR_INVALID_ARGUMENT;
  const bool fp8 = a->kv_cache != nullptr;
  if (fp8 ? (!a->kv_scale || a->k_cache || a->v_cache) : (!a->k_cache || !a->v_cache || a->kv_scale))
    return SPEC_ERR_INVALID_ARGUMENT;
  if (!a->page_table || !a->row_start || !a->kv_len || (a->rows > 0 && (!a->q || !a->out))) return SPEC_ERR_INVALID_ARGUMENT;
  if (!aligned(a->q, 16) || !aligned(a->k_cache, 16) || !aligned(a->v_cache, 16) || !aligned(a->kv_cache, 16) ||
      !aligned(a->kv_scale, 8) || !aligned(a->out, 16) || !aligned(a->lse, 4) || !aligned(a->page_table, 4) ||
      !aligned(a->row_start, 4) || !aligned(a->kv_len, 4))
    return SPEC_ERR_INVALID_ARGUMENT;
  if (!(a->softmax_scale == 0.f || (a->softmax_scale > 0.f && a->softmax_scale < 1e30f))) return SPEC_ERR_INVALID_ARGUMENT;
  if (!stride_ok(a->q_row_stride, static_cast<int64_t>(a->num_q_heads) * a->head_dim)) return SPEC_ERR_INVALID_ARGUMENT;
  if (a->path != SPEC_ATTN_AUTO && a->path != SPEC_ATTN_CUDA_CORES && a->path != SPEC_ATTN_TENSOR_CORES)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (!head_dim_ok(a->head_dim) || !page_size_ok(a->page_size)) return SPEC_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(a->max_pages_per_seq) * a->page_size > (1 << 30) ||
      static_cast<int64_t>(a->num_pages) * a->page_size > INT32_MAX || a->num_kv_heads > 65535)
    return SPEC_ERR_UNSUPPORTED;
  const int64_t group = a->num_q_heads / a->num_kv_heads;
  if (group * (static_cast<int64_t>(a->rows) + 1) > INT32_MAX - 256 ||
      group * a->rows / kSimtRowTile + a->batch > INT32_MAX)
    return SPEC_ERR_UNSUPPORTED;
  if (a->path == SPEC_ATTN_TENSOR_CORES && !chunk_tc_fits(*a)) return SPEC_ERR_UNSUPPORTED;
  return SPEC_OK;
}

// The most that a call may need on any device: the grid is one block per SM.
size_t chunk_bytes(const spec_chunk_attn_args_t& a) {
  int dev = 0, sms = 160;
  if (cudaGetDevice(&dev) == cudaSuccess) {
    const int n = device_sm_count(dev);
    if (n > sms) sms = n;
  } else {
    cudaGetLastError();
  }
  return chunk_plan(a, kWsHeader, sms, a.path).end;
}

spec_status_t run_chunk(const spec_chunk_attn_args_t* a, void* ws, size_t ws_bytes, spec_stream_t stream, bool starve) {
  const spec_status_t st = check_chunk(a);
  if (st != SPEC_OK) return st;
  if (bad_ws(ws)) return SPEC_ERR_INVALID_ARGUMENT;
  if (starve && (a->path == SPEC_ATTN_CUDA_CORES || !chunk_tc_fits(*a) || a->rows == 0)) return SPEC_ERR_UNSUPPORTED;
  if (chunk_plan(*a, kWsHeader, 1, a->path).end > ws_bytes) return SPEC_ERR_WORKSPACE_TOO_SMALL;
  if (a->rows == 0) return SPEC_OK;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  if (!scope.ok) return SPEC_ERR_CUDA;
  (void)cudaGetLastError();
  const ChunkPlan P = chunk_plan(*a, kWsHeader, scope.sms, a->path);
  if (P.end > ws_bytes) return SPEC_ERR_WORKSPACE_TOO_SMALL;
  return launch_chunk(*a, P, static_cast<char*>(ws), s, starve) == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

spec_status_t check_fork(const spec_fork_args_t* a) {
  if (!a || a->batch < 1 || a->page_size < 1 || a->max_pages_per_seq < 1 || a->num_pages < 1 || a->reserved < 0)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (a->free_capacity < a->num_pages) return SPEC_ERR_INVALID_ARGUMENT;
  if (!a->parent || !a->kv_len || !a->new_kv_len || !a->page_table || !a->new_table || !a->shares || !a->new_shares ||
      !a->free_pages || !a->new_free_pages || !a->free_count || !a->new_free_count || !a->copies)
    return SPEC_ERR_INVALID_ARGUMENT;
  for (const void* p : std::initializer_list<const void*>{
           a->parent, a->kv_len, a->new_kv_len, a->page_table, a->new_table, a->shares, a->new_shares, a->free_pages,
           a->new_free_pages, a->free_count, a->new_free_count, a->copies, a->flags})
    if (!aligned(p, 4)) return SPEC_ERR_INVALID_ARGUMENT;
  if (a->batch > SPEC_SLOTS_MAX_BATCH || a->reserved > (1 << 30) ||
      static_cast<int64_t>(a->max_pages_per_seq) * a->page_size > (1 << 30) ||
      static_cast<int64_t>(a->max_pages_per_seq) * a->batch > (1 << 30) ||
      static_cast<int64_t>(a->num_pages) * a->page_size > INT32_MAX)
    return SPEC_ERR_UNSUPPORTED;
  return SPEC_OK;
}
size_t fork_bytes(const spec_fork_args_t& a) {
  const size_t rows = sizeof(int32_t) * static_cast<size_t>(a.batch);
  return kWsHeader + ws_round(rows) + (a.new_table == a.page_table ? ws_round(rows * a.max_pages_per_seq) : 0);
}

spec_status_t check_copy(const spec_copy_args_t* a) {
  if (!a || a->num_pairs < 0 || a->num_pages < 1 || a->num_buffers < 1) return SPEC_ERR_INVALID_ARGUMENT;
  if (a->num_buffers > SPEC_COPY_MAX_BUFFERS) return SPEC_ERR_UNSUPPORTED;
  if (!a->buffers || !a->page_bytes || (a->num_pairs > 0 && !a->pairs)) return SPEC_ERR_INVALID_ARGUMENT;
  if (!aligned(a->pairs, 4) || !aligned(a->status, 4)) return SPEC_ERR_INVALID_ARGUMENT;
  for (int i = 0; i < a->num_buffers; ++i) {
    if (!a->buffers[i] || !aligned(a->buffers[i], 4) || a->page_bytes[i] < 4 || a->page_bytes[i] % 4 != 0)
      return SPEC_ERR_INVALID_ARGUMENT;
    if (a->page_bytes[i] > (int64_t{1} << 40)) return SPEC_ERR_UNSUPPORTED;
  }
  return SPEC_OK;
}

}  // namespace

namespace specv {

// Virtual steps of a unit that sees all the keys that a table row holds, at most.
static int64_t chunk_longest(const spec_chunk_attn_args_t& a) {
  return static_cast<int64_t>(a.max_pages_per_seq) * a.page_size / kChunkKeyTile * kChunkTwinCost + 32;
}

bool chunk_tc_fits(const spec_chunk_attn_args_t& a) {
  const int group = a.num_q_heads / a.num_kv_heads;
  if (group > kChunkTileRows) return false;
  const int64_t per_unit = 2 * (kChunkTileRows / group);
  const int64_t units = a.rows / per_unit + a.batch;
  // 32-bit counts: units, and the steps of a block (of at least 64)
  return units * a.num_kv_heads <= INT32_MAX / 4 && units * a.num_kv_heads <= (static_cast<int64_t>(INT32_MAX) * 32) / chunk_longest(a) && static_cast<int64_t>(a.num_pages) * a.num_kv_heads <= INT32_MAX / 4;
}

ChunkPlan chunk_plan(const spec_chunk_attn_args_t& a, size_t base, int num_sms, int path) {
  ChunkPlan P{};
  P.fp8 = a.kv_cache != nullptr;
  P.path = path != SPEC_ATTN_CUDA_CORES && chunk_tc_fits(a) ? SPEC_ATTN_TENSOR_CORES : SPEC_ATTN_CUDA_CORES;
  P.seqs = base;
  P.bad = ws_round(P.seqs + sizeof(ChunkSeq) * (static_cast<size_t>(a.batch) + 1));
  P.end = ws_round(P.bad + sizeof(int32_t) * static_cast<size_t>(a.batch));
  if (P.path != SPEC_ATTN_TENSOR_CORES) {
    P.max_units = a.rows * (a.num_q_heads / a.num_kv_heads) / kSimtRowTile + a.batch;
    return P;
  }
  P.tile_tokens = kChunkTileRows / (a.num_q_heads / a.num_kv_heads);
  P.max_units = a.rows / (2 * P.tile_tokens) + a.batch;
  // a block per SM, or as many as the longest sequences could give work
  const int64_t work = static_cast<int64_t>(P.max_units) * a.num_kv_heads * chunk_longest(a) / kChunkTwinCost;
  P.grid = static_cast<int>(work < num_sms ? (work < 1 ? 1 : work) : num_sms);
  // one note a stop of a block, of each warp that notes
  P.redo_cap = (P.max_units * a.num_kv_heads + P.grid) * (P.fp8 ? kChunkConverters : 1);
  const size_t rows = static_cast<size_t>(P.grid) * 2 * 2 * kChunkTileRows;
  P.cum = P.end;
  P.work = ws_round(P.cum + sizeof(long long) * (static_cast<size_t>(P.max_units) + 1));
  P.redo = ws_round(P.work + sizeof(ChunkWork) + sizeof(ChunkStart) * static_cast<size_t>(P.grid));
  P.partial_o = ws_round(P.redo + sizeof(int4) * (static_cast<size_t>(P.redo_cap) + 1));
  P.partial_ml = ws_round(P.partial_o + rows * a.head_dim * sizeof(float));
  P.q_half = ws_round(P.partial_ml + rows * sizeof(float2));
  const size_t heads = P.fp8 ? static_cast<size_t>(a.rows) * a.num_q_heads : 0;
  P.q_scale = ws_round(P.q_half + heads * a.head_dim * 2);
  P.end = ws_round(P.q_scale + heads * sizeof(float));
  return P;
}

}  // namespace specv

extern "C" {

spec_status_t spec_rope_kv(const spec_rope_args_t* a, spec_stream_t stream) {
  const spec_status_t st = check_rope(a);
  if (st != SPEC_OK) return st;
  if (a->rows == 0) return SPEC_OK;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  if (!scope.ok) return SPEC_ERR_CUDA;
  return launch_rope(*a, scope.sms, s) == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

size_t spec_chunk_attn_workspace_size(const spec_chunk_attn_args_t* a) {
  return check_chunk(a) == SPEC_OK ? chunk_bytes(*a) : 0;
}

spec_status_t spec_chunk_attention(const spec_chunk_attn_args_t* a, void* ws, size_t ws_bytes, spec_stream_t stream) {
  return run_chunk(a, ws, ws_bytes, stream, false);
}

spec_status_t spec_test_chunk_attention_wait_timeout(const spec_chunk_attn_args_t* a, void* ws, size_t ws_bytes,
                                                     spec_stream_t stream) {
  return run_chunk(a, ws, ws_bytes, stream, true);
}

size_t spec_fork_workspace_size(const spec_fork_args_t* a) { return check_fork(a) == SPEC_OK ? fork_bytes(*a) : 0; }

spec_status_t spec_fork_sequences(const spec_fork_args_t* a, void* ws, size_t ws_bytes, spec_stream_t stream) {
  const spec_status_t st = check_fork(a);
  if (st != SPEC_OK) return st;
  if (bad_ws(ws)) return SPEC_ERR_INVALID_ARGUMENT;
  if (ws_bytes < fork_bytes(*a)) return SPEC_ERR_WORKSPACE_TOO_SMALL;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  if (!scope.ok) return SPEC_ERR_CUDA;
  return launch_fork(*a, static_cast<char*>(ws), s) == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

spec_status_t spec_copy_pages(const spec_copy_args_t* a, spec_stream_t stream) {
  const spec_status_t st = check_copy(a);
  if (st != SPEC_OK) return st;
  if (a->num_pairs == 0) return SPEC_OK;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  if (!scope.ok) return SPEC_ERR_CUDA;
  return launch_copy(*a, s) == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

}  // extern "C"
