// The C ABI of the 8-bit KV cache and the logit constraints (include/spec_verify.h):
// host-side argument checks, workspace layout and launches.
#include <climits>

#include "kv_fp8.cuh"

using namespace specv;

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool bad_ws(const void* ws) { return !ws || !aligned(ws, kWsAlign); }
bool head_dim_ok(int d) { return d == 64 || d == 128; }
bool page_size_ok(int p) { return p == 16 || p == 32 || p == 64; }

spec_status_t check_slots(const spec_slot_args_t* a) {
  if (!a || a->batch < 1 || a->page_size < 1 || a->max_pages_per_seq < 1 || a->num_pages < 1 ||
      a->reserved < 0 || a->max_rows < 1 || a->free_capacity < 0)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (!a->num_new || !a->kv_len || !a->new_len || !a->page_table || !a->free_pages ||
      !a->free_count || !a->new_free_count || !a->row_start || !a->slots)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (a->batch > SPEC_SLOTS_MAX_BATCH || a->reserved > (1 << 30) ||
      static_cast<int64_t>(a->max_pages_per_seq) * a->page_size > (1 << 30) ||
      static_cast<int64_t>(a->num_pages) * a->page_size > INT32_MAX)
    return SPEC_ERR_UNSUPPORTED;
  return SPEC_OK;
}

spec_status_t check_append(const spec_append_fp8_args_t* a) {
  if (!a || a->rows < 0 || a->num_kv_heads < 1 || a->num_pages < 1 || a->head_dim < 1 ||
      a->page_size < 1)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (!a->kv_cache || !a->kv_scale || (a->rows > 0 && (!a->k || !a->v || !a->slots)))
    return SPEC_ERR_INVALID_ARGUMENT;
  if (!head_dim_ok(a->head_dim) || !page_size_ok(a->page_size) || a->num_kv_heads > 65535 ||
      static_cast<int64_t>(a->num_pages) * a->page_size > INT32_MAX)
    return SPEC_ERR_UNSUPPORTED;
  const int64_t dense = static_cast<int64_t>(a->num_kv_heads) * a->head_dim;
  for (int64_t s : {a->k_row_stride, a->v_row_stride})
    if (s != 0 && (s < dense || s % 8 != 0)) return SPEC_ERR_INVALID_ARGUMENT;
  if (!aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->kv_cache, 16) || !aligned(a->kv_scale, 4) ||
      !aligned(a->status, 4))
    return SPEC_ERR_INVALID_ARGUMENT;
  return SPEC_OK;
}

// The tensor-core form of a call. A block serves two sub-units of query rows: two adjacent KV
// heads where each fits one (a page of both is one copy of twice the size; 66 to 128 rows as
// two halves of one head instead: 189 against 127 us at batch 64 / block 20), else two halves
// of one KV head's rows, in tiles. Up to 32 rows a sub-unit the keys are on the MMA's M side,
// from 33 the rows (batch 64 / block 8, 32 rows a KV head: 90 us, with the rows on M 102; block 10:
// 108, as two halves with the keys on M 142). Sequences are taken kFp8TcBatch at a time, because a block keeps their first tiles.
struct TcForm {
  int rows_on_m, heads, sub_rows, row_tiles, batch;
  bool fits;
};
TcForm tc_form(const spec_attn_fp8_args_t& a) {
  const int rows = (a.num_q_heads / a.num_kv_heads) * a.gamma;
  TcForm f;
  f.heads = rows <= 128 && a.num_kv_heads % 2 == 0 ? 2 : 1;
  f.row_tiles = f.heads == 2 ? 1 : (rows + 255) / 256;
  f.sub_rows = f.heads == 2 ? rows : (rows > 256 ? 128 : (rows + 1) / 2);
  f.rows_on_m = f.sub_rows > 32;
  f.batch = a.batch < kFp8TcBatch ? a.batch : kFp8TcBatch;
  const int64_t tiles = (static_cast<int64_t>(a.max_pages_per_seq) * a.page_size + kFp8KeyTile - 1) / kFp8KeyTile + 8;
  const int64_t units = static_cast<int64_t>(f.batch) * (a.num_kv_heads / f.heads) * f.row_tiles;
  f.fits = tiles * units <= INT32_MAX && 2 * static_cast<int64_t>(a.num_pages) * a.num_kv_heads <= INT32_MAX;
  return f;
}

spec_status_t check_attn_fp8(const spec_attn_fp8_args_t* a) {
  if (!a || a->batch < 1 || a->gamma < 1 || a->num_q_heads < 1 || a->num_kv_heads < 1 ||
      a->max_pages_per_seq < 1 || a->num_pages < 1 || a->page_size < 1 || a->head_dim < 1 ||
      a->num_q_heads % a->num_kv_heads != 0)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (!a->q || !a->kv_cache || !a->kv_scale || !a->page_table || !a->kv_len || !a->out)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (!aligned(a->q, 16) || !aligned(a->kv_cache, 16) || !aligned(a->out, 16) || !aligned(a->kv_scale, 8))
    return SPEC_ERR_INVALID_ARGUMENT;
  if (!(a->softmax_scale == 0.f || (a->softmax_scale > 0.f && a->softmax_scale < 1e30f)))
    return SPEC_ERR_INVALID_ARGUMENT;
  if (a->path != SPEC_ATTN_AUTO && a->path != SPEC_ATTN_CUDA_CORES && a->path != SPEC_ATTN_TENSOR_CORES)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (a->gamma > 64 || !head_dim_ok(a->head_dim) || !page_size_ok(a->page_size))
    return SPEC_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(a->max_pages_per_seq) * a->page_size > (1 << 30) ||
      static_cast<int64_t>(a->num_pages) * a->page_size > INT32_MAX)
    return SPEC_ERR_UNSUPPORTED;
  const int64_t rows = static_cast<int64_t>(a->num_q_heads / a->num_kv_heads) * a->gamma;
  if (rows > kFp8MaxRows) return SPEC_ERR_UNSUPPORTED;
  const int64_t z = static_cast<int64_t>(a->batch) * ((rows + kSimtRowTile - 1) / kSimtRowTile);
  const bool tc = tc_form(*a).fits;
  if (a->path == SPEC_ATTN_TENSOR_CORES && !tc) return SPEC_ERR_UNSUPPORTED;
  if ((a->path == SPEC_ATTN_CUDA_CORES || !tc) && (z > 65535 || a->num_kv_heads > 65535))
    return SPEC_ERR_UNSUPPORTED;
  return SPEC_OK;
}

spec_status_t check_adjust(const spec_adjust_args_t* a) {
  if (!a || a->batch < 1 || a->gamma < 1 || a->vocab < 1 || a->max_history < 0 || a->max_bias < 0)
    return SPEC_ERR_INVALID_ARGUMENT;
  if (a->logits_dtype != SPEC_F32 && a->logits_dtype != SPEC_BF16) return SPEC_ERR_INVALID_ARGUMENT;
  if (a->block_shift != 0 && a->block_shift != 1) return SPEC_ERR_INVALID_ARGUMENT;
  if (!a->logits || !a->out || (a->history && !a->history_len) || (a->max_history > 0 && !a->history) ||
      (a->bias_tokens && !a->bias_values) || (a->max_bias > 0 && !a->bias_tokens))
    return SPEC_ERR_INVALID_ARGUMENT;
  const uintptr_t esz = a->logits_dtype == SPEC_BF16 ? 2 : 4;
  if (!aligned(a->logits, esz) || !aligned(a->out, esz)) return SPEC_ERR_INVALID_ARGUMENT;
  if (a->gamma > 64 || a->batch > 65535 || (a->vocab - 1) / kAdjustSlice >= 65535) return SPEC_ERR_UNSUPPORTED;
  return SPEC_OK;
}

size_t attn_fp8_bytes(const spec_attn_fp8_args_t& a, int sms) {
  return attn_fp8_plan(a, kWsHeader, sms, a.path).end;
}

}  // namespace

namespace specv {

AttnFp8Plan attn_fp8_plan(const spec_attn_fp8_args_t& a, size_t base, int num_sms, int path) {
  AttnFp8Plan P{};
  P.rows = (a.num_q_heads / a.num_kv_heads) * a.gamma;
  const TcForm f = tc_form(a);
  P.path = path != SPEC_ATTN_CUDA_CORES && f.fits ? SPEC_ATTN_TENSOR_CORES : SPEC_ATTN_CUDA_CORES;
  int64_t units;
  if (P.path == SPEC_ATTN_TENSOR_CORES) {
    // persistent grid; a block's range begins inside one unit at most and ends inside one
    P.rows_on_m = f.rows_on_m;
    P.heads = f.heads;
    P.sub_rows = f.sub_rows;
    P.row_tiles = f.row_tiles;
    P.batch = f.batch;
    units = static_cast<int64_t>(P.batch) * (a.num_kv_heads / P.heads) * P.row_tiles;
    P.grid = num_sms;
    P.splits = static_cast<int>(units < P.grid ? units : P.grid);
    P.nsplit = 1;
    P.slot_rows = 2 * P.sub_rows;
    P.slots = 2 * P.grid;
  } else {
    P.row_tiles = (P.rows + kSimtRowTile - 1) / kSimtRowTile;
    const int max_tiles = (a.max_pages_per_seq * a.page_size + kSimtKeyTile - 1) / kSimtKeyTile;
    units = static_cast<int64_t>(a.batch) * a.num_kv_heads * P.row_tiles;
    int64_t nsplit = static_cast<int64_t>(num_sms) * 4 / units;  // two blocks fit an SM
    nsplit = nsplit < 1 ? 1 : (nsplit > max_tiles ? max_tiles : nsplit);
    P.tiles_per_split = static_cast<int>((max_tiles + nsplit - 1) / nsplit);
    P.nsplit = (max_tiles + P.tiles_per_split - 1) / P.tiles_per_split;
    P.slot_rows = kSimtRowTile;
    P.slots = P.nsplit > 1 ? units * P.nsplit : 0;
  }
  // (room for the CUDA cores' tickets on either path: they must stay zero)
  P.tickets = base;
  P.partial_o = ws_round(P.tickets + sizeof(uint32_t) * a.batch * a.num_kv_heads *
                                            static_cast<size_t>((P.rows + kSimtRowTile - 1) / kSimtRowTile));
  P.partial_ml = ws_round(P.partial_o + static_cast<size_t>(P.slots) * P.slot_rows * a.head_dim * 4);
  P.split_notes = ws_round(P.partial_ml + static_cast<size_t>(P.slots) * P.slot_rows * sizeof(float2));
  P.end = ws_round(P.split_notes + 2 * sizeof(int4) * P.splits);
  return P;
}

}  // namespace specv

namespace {

spec_status_t run_attn_fp8(const spec_attn_fp8_args_t* a, void* ws, size_t ws_bytes, spec_stream_t stream,
                           bool starve) {
  const spec_status_t st = check_attn_fp8(a);
  if (st != SPEC_OK) return st;
  if (bad_ws(ws)) return SPEC_ERR_INVALID_ARGUMENT;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  if (!scope.ok) return SPEC_ERR_CUDA;
  (void)cudaGetLastError();
  const AttnFp8Plan P = attn_fp8_plan(*a, kWsHeader, scope.sms, a->path);
  if (P.end > ws_bytes) return SPEC_ERR_WORKSPACE_TOO_SMALL;
  char* w = static_cast<char*>(ws);
  if (P.path == SPEC_ATTN_TENSOR_CORES) {
    for (int b0 = 0; b0 < a->batch; b0 += P.batch) {
      spec_attn_fp8_args_t part = *a;
      part.batch = a->batch - b0 < P.batch ? a->batch - b0 : P.batch;
      const int64_t rows = static_cast<int64_t>(b0) * a->gamma, heads = rows * a->num_q_heads;
      part.q = static_cast<const char*>(a->q) + heads * a->head_dim * 2;
      part.out = static_cast<char*>(a->out) + heads * a->head_dim * 2;
      part.page_table = a->page_table + static_cast<int64_t>(b0) * a->max_pages_per_seq;
      part.kv_len = a->kv_len + b0;
      if (a->lse) part.lse = a->lse + heads;
      if (a->tree_mask) part.tree_mask = a->tree_mask + rows;
      if ((P.rows_on_m ? launch_attn_fp8_rows(part, P, w, s, starve) : launch_attn_fp8_keys(part, P, w, s, starve)) !=
          cudaSuccess)
        return SPEC_ERR_CUDA;
    }
    return SPEC_OK;
  }
  if (starve) return SPEC_ERR_UNSUPPORTED;
  return launch_attn_fp8_simt(*a, P, w, s) == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t spec_slot_workspace_size(const spec_slot_args_t* a) {
  return check_slots(a) == SPEC_OK ? kWsHeader + kWsAlign : 0;
}

spec_status_t spec_map_slots(const spec_slot_args_t* a, void* ws, size_t ws_bytes, spec_stream_t stream) {
  const spec_status_t st = check_slots(a);
  if (st != SPEC_OK) return st;
  if (bad_ws(ws)) return SPEC_ERR_INVALID_ARGUMENT;
  if (ws_bytes < kWsHeader + kWsAlign) return SPEC_ERR_WORKSPACE_TOO_SMALL;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  if (!scope.ok) return SPEC_ERR_CUDA;
  return launch_map_slots(*a, static_cast<char*>(ws), s) == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

spec_status_t spec_append_kv_fp8(const spec_append_fp8_args_t* a, spec_stream_t stream) {
  const spec_status_t st = check_append(a);
  if (st != SPEC_OK) return st;
  if (a->rows == 0) return SPEC_OK;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  if (!scope.ok) return SPEC_ERR_CUDA;
  return launch_append_fp8(*a, scope.sms, s) == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

size_t spec_attn_fp8_workspace_size(const spec_attn_fp8_args_t* a) {
  if (check_attn_fp8(a) != SPEC_OK) return 0;
  // the split count depends on the SM count: size for every device it may meet
  int dev = 0, sms = 160;
  if (cudaGetDevice(&dev) == cudaSuccess) {
    const int n = device_sm_count(dev);
    if (n > sms) sms = n;
  } else {
    cudaGetLastError();
  }
  size_t need = 0;
  for (int s : {148, 152, sms}) {
    const size_t x = attn_fp8_bytes(*a, s);
    if (x > need) need = x;
  }
  return need;
}

spec_status_t spec_verify_attention_fp8(const spec_attn_fp8_args_t* a, void* ws, size_t ws_bytes,
                                        spec_stream_t stream) {
  return run_attn_fp8(a, ws, ws_bytes, stream, false);
}

spec_status_t spec_test_attention_fp8_wait_timeout(const spec_attn_fp8_args_t* a, void* ws, size_t ws_bytes,
                                                   spec_stream_t stream) {
  return run_attn_fp8(a, ws, ws_bytes, stream, true);
}

spec_status_t spec_adjust_logits(const spec_adjust_args_t* a, spec_stream_t stream) {
  const spec_status_t st = check_adjust(a);
  if (st != SPEC_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  DeviceScope scope(s);
  if (!scope.ok) return SPEC_ERR_CUDA;
  return launch_adjust(*a, scope.sms, s) == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

}  // extern "C"
