// The 8-bit paged cache (jf_ops.h: jf_kv8_cache): rows appended with the rotary embedding on the way, and the
// values that it stands for read back.
//
// Append. A block of the cache (one page of 16 tokens, one KV head) takes one CTA, and the page's rows of
// queries one more for each KV head's group. With c, s the cosine and sine of the row's position,
//   x'_i = x_i c_i - x_{i+hd/2} s_i,   x'_{i+hd/2} = x_{i+hd/2} c_i + x_i s_i
// for keys and queries; then, for keys and values alike, e = the smallest exponent with max |x'| <= 448 2^e
// (not below the block's own where it holds earlier tokens) and code = e4m3(x' 2^-e). One thread holds 16 values
// of one row (8 pairs), so the block's new values stay in registers between the maximum and the rounding, and
// what the block held before is read once, and written only where its exponent grew.
//
// Queries are rotated by CTAs of their own in the same launch, so that they neither wait for a block's maximum nor for
// its page. Both kinds wait for memory, so what counts is how many are resident: at 5 CTAs of 256 threads (48
// registers) 8,192 rows of 28 + 2 x 4 bf16 heads of 128 (143 MB in and out) take 30 us, 4.8 TB/s; with the queries
// behind the keys in the same CTA 34 us, with two heads in a thread's registers (4 CTAs) 35 us, with 8 CTAs (and
// spills) 47 us. One row: 2.3 us, the length of the chain row -> sequence -> page -> block.
#include "jf_kv8.cuh"

namespace jf {
namespace {

// CTA i of a batch's page grid -> sequence b and the i'th page that its rows touch. Sequence b owns CTAs
// row_start[b] / 16 + 2 b ..: its rows touch at most floor(n / 16) + 2 pages. Called by whole warps.
JF_DEV int kv8_find_seq(const jf_kv8_rows& r, int n_seqs, int i, int lane) {
  int lo = 0, n = n_seqs;  // the last b of [lo, lo + n) whose first CTA is <= i
  while (n > 1) {
    const int step = (n + 31) / 32, b = lo + lane * step;
    const bool at = lane * step < n && r.row_start[b] / kPage + 2 * b <= i;
    const unsigned hits = __ballot_sync(0xffffffffu, at);
    const int k = hits ? 31 - __clz(hits) : 0;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}
inline int kv8_page_grid(const jf_kv8_cache& c, const jf_kv8_rows& r) { return r.n_rows / kPage + 2 * c.n_seqs; }

struct AppendArgs {
  const void *q, *k, *v;
  long long ld_q, ld_k, ld_v;
  int n_heads;
  const int32_t* positions;
  const float* rope;
  int rope_len;
  void* q_out;
  int* err;
};

// 8 consecutive values as fp32. VEC: 16-byte aligned.
template <bool VEC>
JF_DEV void load8(const float* p, float (&x)[8]) {
  if constexpr (VEC) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i];
  }
}
template <bool VEC>
JF_DEV void load8(const bf16* p, float (&x)[8]) {
  if constexpr (VEC) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __bfloat162float(p[i]);
  }
}
// (outputs are allocations of their own: 16-byte aligned where VEC, else of their type)
template <bool VEC>
JF_DEV void store8(float* p, const float (&x)[8]) {
  if constexpr (VEC) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = x[i];
  }
}
template <bool VEC>
JF_DEV void store8(bf16* p, const float (&x)[8]) {
  if constexpr (VEC) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __float2bfloat16_rn(x[i]);
  }
}

// (cos, sin) of 8 pairs.
template <bool VEC>
JF_DEV void load_turns(const float* p, float (&c)[8], float (&s)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    if constexpr (VEC) {
      const float4 t = *reinterpret_cast<const float4*>(p + 2 * i);
      c[i] = t.x, s[i] = t.y, c[i + 1] = t.z, s[i + 1] = t.w;
    } else {
      const float2 t = *reinterpret_cast<const float2*>(p + 2 * i), u = *reinterpret_cast<const float2*>(p + 2 * i + 2);
      c[i] = t.x, s[i] = t.y, c[i + 1] = u.x, s[i + 1] = u.y;
    }
  }
}
// a, b: 8 pairs of a head. Products and sum rounded one by one (no fma), so that the rotated key, and with it its
// code, is the same wherever the formula is evaluated in fp32.
JF_DEV void rotate8(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = a[i], y = b[i];
    a[i] = __fsub_rn(__fmul_rn(x, c[i]), __fmul_rn(y, s[i]));
    b[i] = __fadd_rn(__fmul_rn(y, c[i]), __fmul_rn(x, s[i]));
  }
}

JF_DEV uint2 encode8(const float (&x)[8], float inv) {
  const uint32_t lo = f32x2_to_e4m3x2(x[0] * inv, x[1] * inv) | f32x2_to_e4m3x2(x[2] * inv, x[3] * inv) << 16;
  const uint32_t hi = f32x2_to_e4m3x2(x[4] * inv, x[5] * inv) | f32x2_to_e4m3x2(x[6] * inv, x[7] * inv) << 16;
  return make_uint2(lo, hi);
}
JF_DEV void decode4(uint32_t w, float unit, float* x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t f = e4m3x2_to_f16x2(w >> (16 * h));
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&f));
    x[2 * h] = v.x * unit;
    x[2 * h + 1] = v.y * unit;
  }
}

// Position of a row in the table; one that it does not have is reported and read as 0.
JF_DEV long long turn_at(const AppendArgs& a, int row, int at) {
  int pos = a.positions ? a.positions[row] : at;
  if (pos < 0 || pos >= a.rope_len) {
    jf_set_error(a.err, JF_DERR_BOUNDS);
    pos = 0;
  }
  return pos;
}

// T: type of q, k, v; TO: of q_out. blockIdx.y: a KV head, first of its blocks, then (with queries) of its query heads.
template <typename T, typename TO, int HD, bool VEC>
__global__ void __launch_bounds__(4 * HD / 2, 640 / HD) k_kv8_append(const jf_kv8_cache c, const jf_kv8_rows r, const AppendArgs a) {
  constexpr int TPR = HD / 16;           // threads per row of a block
  constexpr int HALF_THREADS = 16 * TPR; // the first half of the CTA holds keys, the second values
  __shared__ uint32_t s_amax[2 * HALF_THREADS / 32];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31;
  const bool turning = blockIdx.y >= c.n_kv_heads;
  const int b = kv8_find_seq(r, c.n_seqs, blockIdx.x, lane), h = turning ? blockIdx.y - c.n_kv_heads : blockIdx.y;
  const Kv8Seq sq = kv8_seq(c, r, b, a.err);
  const int nth = (int)blockIdx.x - (sq.row0 / kPage + 2 * b);  // of the pages that the rows touch
  const int page = sq.len / kPage + nth, slot0 = page * kPage;
  if (sq.n == 0 || nth < 0 || slot0 >= sq.len + sq.n) return;
  const int old = max(0, sq.len - slot0), last = min(kPage, sq.len + sq.n - slot0);  // new slots: old .. last - 1
  const int row_first = sq.row0 + slot0 + old - sq.len;                              // of slot `old`

  const bool is_k = tid < HALF_THREADS;
  const int t = is_k ? tid : tid - HALF_THREADS, slot = t / TPR, d = t % TPR * 8;
  const bool fresh = slot >= old && slot < last;
  const int row = row_first + slot - old;
  float cs[8], sn[8];
  if (turning) {
    // Even heads by the first half of the CTA, odd ones by the second.
    if (!fresh) return;
    const int G = a.n_heads / c.n_kv_heads;
    const T* src = reinterpret_cast<const T*>(a.q) + row * a.ld_q + (long long)h * G * HD + d;
    TO* dst = reinterpret_cast<TO*>(a.q_out) + ((long long)row * a.n_heads + h * G) * HD + d;
    if (a.rope) load_turns<VEC>(a.rope + (turn_at(a, row, slot0 + slot) * (HD / 2) + d) * 2, cs, sn);
    for (int g = is_k ? 0 : 1; g < G; g += 2) {
      float x[8], y[8];
      load8<VEC>(src + g * HD, x);
      load8<VEC>(src + g * HD + HD / 2, y);
      if (a.rope) rotate8(x, y, cs, sn);
      store8<VEC>(dst + g * HD, x);
      store8<VEC>(dst + g * HD + HD / 2, y);
    }
    return;
  }
  const int id = kv8_page(c, b, page, a.err);
  if (id < 0) return;
  const long long block = (long long)id * c.n_kv_heads + h;
  uint8_t* codes = reinterpret_cast<uint8_t*>(is_k ? c.k : c.v) + (block * kPage + slot) * HD + d;
  int8_t* exps = (is_k ? c.k_exp : c.v_exp) + block;
  float x[8], y[8];
  uint32_t amax = 0;
  bool odd = false;  // met a value that is no finite number
  if (fresh) {
    const T* src = reinterpret_cast<const T*>(is_k ? a.k : a.v) + row * (is_k ? a.ld_k : a.ld_v) + h * HD + d;
    load8<VEC>(src, x);
    load8<VEC>(src + HD / 2, y);
    if (is_k && a.rope) {
      load_turns<VEC>(a.rope + (turn_at(a, row, slot0 + slot) * (HD / 2) + d) * 2, cs, sn);
      rotate8(x, y, cs, sn);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float* const v2[2] = {&x[i], &y[i]};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float& v = *v2[j];
        const uint32_t m = __float_as_uint(v) & 0x7fffffffu;
        if (m < 0x7f800000u) amax = max(amax, m);
        else odd = true;
        if (m > 0x7f800000u) v = 0.f;
      }
    }
  }
  if (odd) jf_set_error(a.err, JF_DERR_NONFINITE);
  amax = __reduce_max_sync(0xffffffffu, amax);
  if (lane == 0) s_amax[tid >> 5] = amax;
  const int e_old = old > 0 ? (int)*exps : kKv8ExpMin;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < HALF_THREADS / 32; ++w) amax = max(amax, s_amax[(is_k ? 0 : HALF_THREADS / 32) + w]);
  const int e = max(e_old, kv8_exponent(__uint_as_float(amax)));
  if (t == 0) *exps = (int8_t)e;
  if (fresh) {
    const float inv = pow2i(-e);
    *reinterpret_cast<uint2*>(codes) = encode8(x, inv);
    *reinterpret_cast<uint2*>(codes + HD / 2) = encode8(y, inv);
  } else if (slot < old && e > e_old) {
    // (a difference beyond 2^-126 leaves nothing of any code)
    const float shrink = pow2i(max(e_old - e, -126));
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint2* p = reinterpret_cast<uint2*>(codes + j * (HD / 2));
      const uint2 w = *p;
      decode4(w.x, 1.f, x);
      decode4(w.y, 1.f, x + 4);
      *p = encode8(x, shrink);
    }
  }
}

// A CTA per block; a thread decodes 16 codes and writes them out. Bound by latency: 8,192 rows of 2 x 4 heads of 128
// (8 MB in, 34 MB out in bf16, held by L2) take 5.8 us, one row 1.9 us.
template <typename TO, int HD, bool VEC>
__global__ void __launch_bounds__(4 * HD / 2)
    k_kv8_read(const jf_kv8_cache c, const jf_kv8_rows r, TO* k_out, TO* v_out, int* err) {
  constexpr int TPR = HD / 16, HALF_THREADS = 16 * TPR;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x;
  const int b = kv8_find_seq(r, c.n_seqs, blockIdx.x, tid & 31), h = blockIdx.y;
  const Kv8Seq sq = kv8_seq(c, r, b, err);
  const int nth = (int)blockIdx.x - (sq.row0 / kPage + 2 * b);
  const int page = sq.len / kPage + nth, slot0 = page * kPage;
  if (sq.n == 0 || nth < 0 || slot0 >= sq.len + sq.n) return;
  const int id = kv8_page(c, b, page, err);
  if (id < 0) return;
  const bool is_k = tid < HALF_THREADS;
  TO* out = is_k ? k_out : v_out;
  const int t = is_k ? tid : tid - HALF_THREADS, slot = t / TPR, d = t % TPR * 16, i = slot0 + slot - sq.len;
  if (!out || i < 0 || i >= sq.n) return;
  const long long block = (long long)id * c.n_kv_heads + h;
  const float unit = pow2i((is_k ? c.k_exp : c.v_exp)[block]);
  const uint4 w = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(is_k ? c.k : c.v) +
                                                  (block * kPage + slot) * HD + d);
  TO* dst = out + ((long long)(sq.row0 + i) * c.n_kv_heads + h) * HD + d;
  float x[8];
  decode4(w.x, unit, x);
  decode4(w.y, unit, x + 4);
  store8<VEC>(dst, x);
  decode4(w.z, unit, x);
  decode4(w.w, unit, x + 4);
  store8<VEC>(dst + 8, x);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <typename T, typename TO>
cudaError_t launch_append(const jf_kv8_cache& c, const jf_kv8_rows& r, const AppendArgs& a, cudaStream_t st) {
  constexpr int per16 = 16 / (int)sizeof(T);
  const bool vec = aligned16(a.k) && aligned16(a.v) && aligned16(a.q) && aligned16(a.q_out) && aligned16(a.rope) &&
                   a.ld_k % per16 == 0 && a.ld_v % per16 == 0 && (!a.q || a.ld_q % per16 == 0);
  const dim3 grid(kv8_page_grid(c, r), a.q ? 2 * c.n_kv_heads : c.n_kv_heads);
  if (c.head_dim == 128)
    return vec ? kv8_launch(k_kv8_append<T, TO, 128, true>, grid, dim3(256), 0, st, c, r, a)
               : kv8_launch(k_kv8_append<T, TO, 128, false>, grid, dim3(256), 0, st, c, r, a);
  return vec ? kv8_launch(k_kv8_append<T, TO, 64, true>, grid, dim3(128), 0, st, c, r, a)
             : kv8_launch(k_kv8_append<T, TO, 64, false>, grid, dim3(128), 0, st, c, r, a);
}

template <typename TO>
cudaError_t launch_read(const jf_kv8_cache& c, const jf_kv8_rows& r, void* k_out, void* v_out, int* err, cudaStream_t st) {
  const bool vec = aligned16(k_out) && aligned16(v_out);
  const dim3 grid(kv8_page_grid(c, r), c.n_kv_heads);
  TO *ko = reinterpret_cast<TO*>(k_out), *vo = reinterpret_cast<TO*>(v_out);
  if (c.head_dim == 128)
    return vec ? kv8_launch(k_kv8_read<TO, 128, true>, grid, dim3(256), 0, st, c, r, ko, vo, err)
               : kv8_launch(k_kv8_read<TO, 128, false>, grid, dim3(256), 0, st, c, r, ko, vo, err);
  return vec ? kv8_launch(k_kv8_read<TO, 64, true>, grid, dim3(128), 0, st, c, r, ko, vo, err)
             : kv8_launch(k_kv8_read<TO, 64, false>, grid, dim3(128), 0, st, c, r, ko, vo, err);
}

bool is_dtype(int d) { return d == JF_F32 || d == JF_BF16; }
bool aligned_to(const void* p, int dtype) { return ((uintptr_t)p & (dtype == JF_BF16 ? 1 : 3)) == 0; }

}  // namespace
}  // namespace jf

using namespace jf;

extern "C" jf_status jf_op_kv8_append(const jf_kv8_cache* cache, const jf_kv8_rows* rows, int dtype, const void* q,
                                      long long ld_q, const void* k, long long ld_k, const void* v, long long ld_v,
                                      int n_heads, const int32_t* positions, const float* rope, int rope_len,
                                      int out_dtype, void* q_out, int* err_word, void* cuda_stream) {
  const jf_status s = kv8_check(cache, rows);
  if (s != JF_OK) return s;
  if (!is_dtype(dtype) || !is_dtype(out_dtype) || !err_word || !q != !q_out) return JF_EINVAL;
  if (rows->n_rows > 0 && (!k || !v)) return JF_EINVAL;
  if (!aligned_to(k, dtype) || !aligned_to(v, dtype) || !aligned_to(q, dtype) || !aligned_to(q_out, out_dtype)) return JF_EINVAL;
  const long long kv_width = (long long)cache->n_kv_heads * cache->head_dim;
  if (ld_k < kv_width || ld_v < kv_width) return JF_EINVAL;
  if (q && (n_heads < 1 || n_heads % cache->n_kv_heads || ld_q < (long long)n_heads * cache->head_dim)) return JF_EINVAL;
  if (rope && (rope_len < 1 || ((uintptr_t)rope & 7))) return JF_EINVAL;
  if (rows->n_rows == 0) return JF_OK;
  const AppendArgs a = {q, k, v, ld_q, ld_k, ld_v, n_heads, positions, rope, rope_len, q_out, err_word};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const bool in_bf16 = dtype == JF_BF16, out_bf16 = out_dtype == JF_BF16;
  const cudaError_t e = in_bf16 ? (out_bf16 ? launch_append<bf16, bf16>(*cache, *rows, a, st)
                                            : launch_append<bf16, float>(*cache, *rows, a, st))
                                : (out_bf16 ? launch_append<float, bf16>(*cache, *rows, a, st)
                                            : launch_append<float, float>(*cache, *rows, a, st));
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}

extern "C" jf_status jf_op_kv8_read(const jf_kv8_cache* cache, const jf_kv8_rows* rows, int out_dtype, void* k_out,
                                    void* v_out, int* err_word, void* cuda_stream) {
  const jf_status s = kv8_check(cache, rows);
  if (s != JF_OK) return s;
  if (!is_dtype(out_dtype) || !err_word || !aligned_to(k_out, out_dtype) || !aligned_to(v_out, out_dtype)) return JF_EINVAL;
  if (rows->n_rows == 0 || (!k_out && !v_out)) return JF_OK;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = out_dtype == JF_BF16 ? launch_read<bf16>(*cache, *rows, k_out, v_out, err_word, st)
                                             : launch_read<float>(*cache, *rows, k_out, v_out, err_word, st);
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}
