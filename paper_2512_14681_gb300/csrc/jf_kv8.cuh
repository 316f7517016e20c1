// What the kernels of the 8-bit paged cache share (jf_ops.h: jf_kv8_cache): blocks, bounds, conversions.
#pragma once
#include "../../include/jf_ops.h"
#include "jf_device.cuh"
#include "jf_internal.h"

namespace jf {

constexpr int kKv8MaxSeqs = 1024, kKv8MaxHeads = 32767;  // (append's grid is twice as high as the KV heads with queries)
constexpr int kKv8ExpMin = -120, kKv8ExpMax = 119;

// 2^e in fp32 for -126 <= e <= 127
JF_DEV float pow2i(int e) { return __int_as_float((e + 127) << 23); }

// The smallest e with amax <= 448 2^e (448 = 1.75 * 2^8), for a finite amax >= 0, within the format's range.
JF_DEV int kv8_exponent(float amax) {
  const int bits = __float_as_int(amax), x = (bits >> 23) - 127;  // amax = 1.m * 2^x (subnormals: x = -127, clamped below)
  const int e = (bits & 0x7fffff) <= 0x600000 ? x - 8 : x - 7;
  return min(max(e, kKv8ExpMin), kKv8ExpMax);
}

// Two e4m3 codes (low byte first) as fp16 (exact), and two fp32 values as codes (nearest, ties to even;
// beyond +-448: +-448).
JF_DEV uint32_t e4m3x2_to_f16x2(uint32_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
  return r;
}
JF_DEV uint32_t f32x2_to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// Rows of sequence b: how many (0 where they are not inside the batch and the page table: reported), the first
// one, the tokens before them.
struct Kv8Seq {
  int n, row0, len;
};
JF_DEV Kv8Seq kv8_seq(const jf_kv8_cache& c, const jf_kv8_rows& r, int b, int* err) {
  const int s0 = r.row_start[b], s1 = r.row_start[b + 1], len = r.len[b];
  Kv8Seq s = {0, s0, len};
  if (s0 < 0 || s1 < s0 || s1 > r.n_rows || len < 0 || (long long)len + (s1 - s0) > (long long)c.pages_per_seq * kPage) {
    jf_set_error(err, JF_DERR_BOUNDS);
    return s;
  }
  s.n = s1 - s0;
  return s;
}

// Page of tokens 16 i .. of sequence b, or -1 (reported) where the table names none of the pool.
JF_DEV int kv8_page(const jf_kv8_cache& c, int b, int i, int* err) {
  const int id = c.page_table[(long long)b * c.pages_per_seq + i];
  if (id >= 0 && id < c.n_pages) return id;
  jf_set_error(err, JF_DERR_BOUNDS);
  return -1;
}

// Host checks shared by the entry points.
inline jf_status kv8_check(const jf_kv8_cache* c, const jf_kv8_rows* r) {
  if (!c || !r || !c->k || !c->v || !c->k_exp || !c->v_exp || !c->page_table || !r->row_start || !r->len) return JF_EINVAL;
  if (c->n_seqs < 1 || c->n_pages < 1 || c->pages_per_seq < 1 || c->n_kv_heads < 1 || r->n_rows < 0 || r->max_rows < 0)
    return JF_EINVAL;
  if (r->n_rows > 0 && (r->max_rows < 1 || r->max_rows > r->n_rows)) return JF_EINVAL;
  if (c->pages_per_seq > (1 << 26)) return JF_EUNSUPPORTED;  // slots are 32-bit numbers
  if (((uintptr_t)c->k & 15) || ((uintptr_t)c->v & 15)) return JF_EINVAL;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->n_seqs > kKv8MaxSeqs || c->n_kv_heads > kKv8MaxHeads) return JF_EUNSUPPORTED;
  return JF_OK;
}

// A launch that may start while the kernel before it on the stream drains: every kernel here waits for it
// (pdl_wait) before it reads or writes anything of the caller's.
template <typename K, typename... Args>
cudaError_t kv8_launch(K kernel, dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace jf
