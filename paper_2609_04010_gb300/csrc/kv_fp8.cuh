// Internal declarations of the 8-bit KV cache and the logit constraints, and the e4m3
// conversions of its kernels.
#pragma once

#include "common.cuh"

namespace specv {

cudaError_t launch_map_slots(const spec_slot_args_t& a, char* ws, cudaStream_t stream);
size_t slot_smem(int batch);  // dynamic shared memory of a block
cudaError_t launch_append_fp8(const spec_append_fp8_args_t& a, int sms, cudaStream_t stream);
constexpr int kAdjustSlice = 2048;  // tokens of a block, whose ranges are the grid's second index
cudaError_t launch_adjust(const spec_adjust_args_t& a, int sms, cudaStream_t stream);

// The launch plan of the attention over the 8-bit cache.
struct AttnFp8Plan {
  int path;             // SPEC_ATTN_CUDA_CORES or SPEC_ATTN_TENSOR_CORES
  int rows_on_m;        // tensor cores: attn_fp8_rows.cu, else attn_fp8_keys.cu
  int heads;            // tensor cores: KV heads per block (2: adjacent ones)
  int batch;            // tensor cores: sequences per launch
  int sub_rows;         // tensor cores: query rows of one of a block's two sub-units
  int grid, splits;     // tensor cores: blocks, and places for units to merge
  int rows, row_tiles;  // (Hq/Hkv) * gamma query rows per KV head, in tiles
  int nsplit, tiles_per_split;  // CUDA cores: KV splits per unit and key tiles of a split
  int64_t slots;        // partial results
  int slot_rows;        // rows of one
  size_t tickets, partial_o, partial_ml, split_notes, end;
};
AttnFp8Plan attn_fp8_plan(const spec_attn_fp8_args_t& a, size_t base, int num_sms, int path);
constexpr int kFp8MaxRows = 2147483647 - 255;  // query rows of a KV head: 32-bit counts, in tiles of 256
constexpr int kFp8KeyTile = 128;   // keys per tile of the tensor-core kernels
constexpr int kFp8TcBatch = 2048;  // sequences they take in a launch
// starve (test hook only): the producers issue no copies, so the bounded waits run out.
cudaError_t launch_attn_fp8_keys(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws,
                                 cudaStream_t stream, bool starve = false);
cudaError_t launch_attn_fp8_rows(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws,
                                 cudaStream_t stream, bool starve = false);
cudaError_t launch_attn_fp8_simt(const spec_attn_fp8_args_t& a, const AttnFp8Plan& P, char* ws,
                                 cudaStream_t stream);

#ifdef __CUDACC__
// A launch that may start while the kernel before it on the stream still runs. Every thread of
// such a kernel calls pdl_wait_prior() before it touches global memory, which waits for that
// kernel's end; what the launch itself and a block's set-up take is hidden (1.5 to 2 us a call).
// No kernel lets the next one start before its own blocks end: blocks that wait took the places
// of working ones (the slots of 512 requests: 12 us against 9).
template <typename... Params, typename... Args>
cudaError_t launch_overlapped(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t stream,
                              Args... args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

constexpr float kScaleMin = 2.3283064365386963e-10f;  // 2^-32
constexpr float kScaleMax = 4294967296.f;             // 2^32

// A scale as the kernels use it: within the range that spec_append_kv_fp8 writes.
__device__ __forceinline__ float clamp_scale(float s) { return fminf(fmaxf(s, kScaleMin), kScaleMax); }

// The smallest power of two s in range with the magnitude whose bf16 bits are m <= 448 s.
// With m = f * 2^e, f in [0.5, 1), and 448 = 0.875 * 2^9 it is 2^(e-9), or 2^(e-8) if
// f > 0.875.
__device__ __forceinline__ float fp8_scale_of(uint32_t m) {
  const int e = static_cast<int>(m >> 7) - 126;
  const int k = min(32, max(-32, e - 9 + ((m & 0x7fu) > 0x60u ? 1 : 0)));
  return __uint_as_float(static_cast<uint32_t>(k + 127) << 23);
}

// Two e4m3 values, a in the low byte (ties to even, saturating at +-448, NaN stays NaN).
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
// The two e4m3 values of the low 16 bits (exact), low byte first.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t v) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(v)));
  return r;
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t v) {
  const uint32_t h = e4m3x2_to_f16x2(v);
  float2 f;
  asm("{ .reg .f16 lo, hi; mov.b32 {lo, hi}, %2; cvt.f32.f16 %0, lo; cvt.f32.f16 %1, hi; }"
      : "=f"(f.x), "=f"(f.y)
      : "r"(h));
  return f;
}
#endif

}  // namespace specv
