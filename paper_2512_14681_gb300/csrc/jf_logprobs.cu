// Log probabilities of given tokens with entropy and top alternatives, and their gradient (jf_ops.h).
//
// One pass over the logits x. Against a running maximum m, with d = x - m,
//   S = sum e^(scale d),  T = sum e^(scale d) d,   lse = scale m + ln S,   entropy = ln S - scale T / S,
// and when m grows, T takes the step times S before both shrink. (The difference comes first: where every logit is
// the type's lowest value, as in a row that a mask has emptied, x log2 e would overflow.) Every thread keeps its own (m, S, T); they are joined in
// thread order. The top list is kept per warp: a buffer of candidates that exceed the warp's n_top'th best so
// far, ordered by (value, lower index) as one 64-bit key, and cut back to n_top whenever it fills, so the list does
// not depend on the order in which candidates arrive. Few rows are cut into segments (one CTA each), whose states
// and lists a second kernel joins in segment order.
#include "../../include/jf_ops.h"
#include "jf_device.cuh"
#include "jf_internal.h"

namespace jf {
namespace {

constexpr int LP_THREADS = 256, LP_WARPS = LP_THREADS / 32;
constexpr int LP_BUF = 512;         // candidates a warp holds
constexpr int LP_SEG_MIN = 4096;    // fewest logits of a segment
constexpr int LP_CTAS = 608;        // CTAs that fill the GPU (152 SMs x 4)
constexpr float LOG2E = 1.4426950408889634f;
constexpr int NO_TOKEN = 0x7fffffff;

JF_DEV float ex2_ftz(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Order of candidates: larger value first, then the lower index. Never 0 for a number above -infinity.
JF_DEV unsigned long long lp_key(float v, int idx) {
  const uint32_t b = __float_as_uint(v + 0.f);  // (-0 counts as 0)
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (unsigned long long)o << 32 | (uint32_t)~idx;
}
JF_DEV float lp_key_value(unsigned long long k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
JF_DEV int lp_key_index(unsigned long long k) { return (int)~(uint32_t)k; }

struct LpStat {
  float m, s, t;  // largest logit; sums relative to it
};
JF_DEV LpStat lp_join(LpStat a, LpStat b, float c) {  // c = scale log2 e
  LpStat r;
  r.m = fmaxf(a.m, b.m);
  // (an empty side has m = -inf and sums 0 or, where it met NaN only, NaN)
  const float da = a.m == -INFINITY ? 0.f : a.m - r.m, db = b.m == -INFINITY ? 0.f : b.m - r.m;
  const float wa = exp2f(da * c), wb = exp2f(db * c);
  // (a weight of 0 would meet d = -inf: keep 0 * d finite)
  r.s = wa * a.s + wb * b.s;
  r.t = wa * fmaf(fmaxf(da, -1e30f), a.s, a.t) + wb * fmaf(fmaxf(db, -1e30f), b.s, b.t);
  return r;
}

template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static JF_DEV void load(const float* p, float (&x)[4]) {
    const float4 v = __ldcs(reinterpret_cast<const float4*>(p));
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  }
  static JF_DEV void store(float* p, const float (&x)[4]) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));
  }
};
template <>
struct Vec<bf16> {
  static constexpr int N = 8;
  static JF_DEV void load(const bf16* p, float (&x)[8]) {
    const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static JF_DEV void store(bf16* p, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
  }
};

// A row as 16-byte vectors from the boundary at or before its first element: vector v holds elements
// v N - skew .. v N - skew + N - 1, of which those in [0, V) exist.
template <typename T>
struct Row {
  const T* p;
  int skew, n_vec, V;
  JF_DEV Row(const T* base, int V_) : p(base), V(V_) {
    skew = (int)(((uintptr_t)base & 15) / sizeof(T));
    n_vec = (int)(((long long)V + skew + Vec<T>::N - 1) / Vec<T>::N);
  }
  JF_DEV long long first(int v) const { return (long long)v * Vec<T>::N - skew; }
  JF_DEV bool whole(int v) const { return first(v) >= 0 && first(v) + Vec<T>::N <= V; }
  JF_DEV void load(int v, bool live, float (&x)[Vec<T>::N]) const {
    if (live && whole(v)) {
      Vec<T>::load(p + first(v), x);
    } else {
#pragma unroll
      for (int i = 0; i < Vec<T>::N; ++i) {
        const long long e = first(v) + i;
        x[i] = live && e >= 0 && e < V ? act_to_f32(p[e]) : -INFINITY;
      }
    }
  }
};

// The n largest of buf[0 .. count) (n <= 64, distinct keys but for 0), in falling order into buf[0 .. n), zeros after
// the last; returns the n'th. By one whole warp. CAP: most entries.
template <int CAP>
JF_DEV unsigned long long lp_cut(unsigned long long* buf, int count, int n) {
  constexpr int R = CAP / 32;
  const int lane = threadIdx.x & 31;
  unsigned long long e[R];
  __syncwarp();
#pragma unroll
  for (int i = 0; i < R; ++i) e[i] = i * 32 + lane < count ? buf[i * 32 + lane] : 0ull;
  __syncwarp();
  unsigned long long best = 0;
  for (int k = 0; k < n; ++k) {
    unsigned long long v = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) v = e[i] > v ? e[i] : v;
    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
    best = (unsigned long long)hi << 32 | lo;
    if (lane == 0) buf[k] = best;
#pragma unroll
    for (int i = 0; i < R; ++i) e[i] = e[i] == best ? 0ull : e[i];
  }
  __syncwarp();
  return best;
}

struct LpParams {
  const void* logits;
  long long ld;
  int rows, V, n_top, segs;
  float scale;
  const int32_t* targets;
  float *logprob, *entropy, *lse, *row_stats;
  int32_t* top_ids;
  float* top_logprobs;
  float4* stats;              // [rows][segs] (m, S, T, -)
  unsigned long long* lists;  // [rows][segs][n_top]
  int* err;
};

// Outputs of a row from its joined state and list.
template <typename T>
JF_DEV void lp_finish(const LpParams& a, int row, const LpStat& st, const unsigned long long* list, int tid) {
  const float ls = logf(st.s);
  const bool none = st.m == -INFINITY && st.s == 0.f;  // no token can occur
  const float m = st.m == -INFINITY ? 0.f : st.m;      // (-inf with NaN sums: NaN below)
  if (tid == 0) {
    if (a.lse) a.lse[row] = none ? -INFINITY : fmaf(a.scale, m, ls);
    if (a.row_stats) a.row_stats[2 * (long long)row] = st.m, a.row_stats[2 * (long long)row + 1] = none ? -INFINITY : ls;
    if (a.entropy) a.entropy[row] = none ? 0.f : ls - a.scale * (st.t / st.s);
    if (a.logprob) {
      const int t = a.targets[row];
      float lp = 0.f;
      if (t >= a.V) {
        jf_set_error(a.err, JF_DERR_BOUNDS);
        lp = __int_as_float(0x7fffffff);
      } else if (t >= 0) {
        const float x = act_to_f32(reinterpret_cast<const T*>(a.logits)[row * a.ld + t]);
        lp = none ? -INFINITY : fmaf(x - m, a.scale, -ls);
      }
      a.logprob[row] = lp;
    }
  }
  for (int k = tid; k < a.n_top; k += LP_THREADS) {
    const unsigned long long key = list[k];
    a.top_ids[(long long)row * a.n_top + k] = key ? lp_key_index(key) : NO_TOKEN;
    a.top_logprobs[(long long)row * a.n_top + k] = key ? fmaf(lp_key_value(key) - m, a.scale, -ls) : -INFINITY;
  }
}

// CTA (row, segment). TOP: a list is asked for.
template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_THREADS) k_logprobs(const LpParams a) {
  constexpr int N = Vec<T>::N;
  constexpr int U = 4;  // vectors in flight per thread
  __shared__ unsigned long long s_buf[TOP ? LP_WARPS : 1][TOP ? LP_BUF : 1];
  __shared__ int s_count[LP_WARPS];
  __shared__ LpStat s_stat[LP_WARPS];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x / a.segs, seg = blockIdx.x % a.segs;
  const Row<T> r(reinterpret_cast<const T*>(a.logits) + row * a.ld, a.V);
  const int v_begin = (int)((long long)r.n_vec * seg / a.segs), v_end = (int)((long long)r.n_vec * (seg + 1) / a.segs);
  const float c = a.scale * LOG2E;
  float m = -INFINITY, s = 0.f, t = 0.f;
  unsigned long long thr = 0;  // the n_top'th best key so far
  float thr_v = -INFINITY;
  if (TOP && lane == 0) s_count[warp] = 0;
  if (TOP) __syncwarp();
  for (int v0 = v_begin + warp * 32; v0 < v_end; v0 += LP_THREADS * U) {
    float x[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = v0 + u * LP_THREADS + lane;
      r.load(v, v < v_end, x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float mx = x[u][0];
#pragma unroll
      for (int i = 1; i < N; ++i) mx = fmaxf(mx, x[u][i]);
      if (TOP && __any_sync(0xffffffffu, mx > thr_v)) {
        const long long e0 = r.first(v0 + u * LP_THREADS + lane);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          if (x[u][i] > thr_v) {
            const unsigned long long key = lp_key(x[u][i], (int)(e0 + i));
            if (key > thr) s_buf[warp][atomicAdd(&s_count[warp], 1)] = key;
          }
        }
        __syncwarp();
        const int count = s_count[warp];
        if (count > LP_BUF - 32 * N) {
          thr = lp_cut<LP_BUF>(s_buf[warp], count, a.n_top);
          thr_v = thr ? lp_key_value(thr) : -INFINITY;
          if (lane == 0) s_count[warp] = min(count, a.n_top);
          __syncwarp();
        }
      }
      if (mx > m) {
        if (m > -INFINITY) {  // (before the first number the sums are 0, or NaN)
          const float d = m - mx, al = ex2_ftz(d * c);
          t = al * fmaf(fmaxf(d, -1e30f), s, t);
          s = al * s;
        }
        m = mx;
      }
      const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float d = x[u][i] - base, e = ex2_ftz(d * c);
        s += e;
        t = fmaf(e, fmaxf(d, -1e30f), t);  // (0 where x = -inf)
      }
    }
  }
  LpStat st = {m, s, t};
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    LpStat b = {__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), __shfl_xor_sync(0xffffffffu, st.t, o)};
    st = lane & o ? lp_join(b, st, c) : lp_join(st, b, c);
  }
  if (lane == 0) s_stat[warp] = st;
  if (TOP) lp_cut<LP_BUF>(s_buf[warp], s_count[warp], a.n_top);
  __syncthreads();
  if (warp == 0) {
    st = s_stat[0];
    for (int w = 1; w < LP_WARPS; ++w) st = lp_join(st, s_stat[w], c);
    if (TOP) {  // the warps' lists, one after the other (8 x 64 at most)
      unsigned long long* all = s_buf[0];
      for (int w = 1; w < LP_WARPS; ++w)
        for (int k = lane; k < a.n_top; k += 32) all[w * a.n_top + k] = s_buf[w][k];
      lp_cut<LP_BUF>(all, LP_WARPS * a.n_top, a.n_top);
    }
    if (lane == 0) s_stat[0] = st;
  }
  __syncthreads();
  if (a.segs == 1) {
    lp_finish<T>(a, row, s_stat[0], s_buf[0], tid);
  } else {
    if (tid == 0) a.stats[blockIdx.x] = make_float4(s_stat[0].m, s_stat[0].s, s_stat[0].t, 0.f);
    if (TOP)
      for (int k = tid; k < a.n_top; k += LP_THREADS) a.lists[(long long)blockIdx.x * a.n_top + k] = s_buf[0][k];
  }
}

// Joins a row's segments: one CTA a row.
template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_THREADS) k_logprobs_join(const LpParams a) {
  __shared__ unsigned long long s_buf[TOP ? LP_WARPS : 1][TOP ? LP_BUF : 1];
  __shared__ LpStat s_stat;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, row = blockIdx.x;
  const float c = a.scale * LOG2E;
  if (warp == 0) {
    LpStat st = {-INFINITY, 0.f, 0.f};
    for (int i = lane; i < a.segs; i += 32) {
      const float4 v = a.stats[(long long)row * a.segs + i];
      st = lp_join(st, LpStat{v.x, v.y, v.z}, c);
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      LpStat b = {__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), __shfl_xor_sync(0xffffffffu, st.t, o)};
      st = lane & o ? lp_join(b, st, c) : lp_join(st, b, c);
    }
    if (lane == 0) s_stat = st;
  }
  if (TOP) {
    // a warp takes every 8th run of LP_BUF - 64 entries
    const unsigned long long* list = a.lists + (long long)row * a.segs * a.n_top;
    const int total = a.segs * a.n_top;
    constexpr int RUN = LP_BUF - 64;
    int have = 0;
    for (int i0 = warp * RUN; i0 < total; i0 += LP_WARPS * RUN) {
      const int n = min(RUN, total - i0);
      __syncwarp();
      for (int i = lane; i < n; i += 32) s_buf[warp][have + i] = list[i0 + i];
      lp_cut<LP_BUF>(s_buf[warp], have + n, a.n_top);
      have = a.n_top;
    }
    if (!have)
      for (int i = lane; i < a.n_top; i += 32) s_buf[warp][i] = 0;
  }
  __syncthreads();
  if (TOP && warp == 0) {
    unsigned long long* all = s_buf[0];
    for (int w = 1; w < LP_WARPS; ++w)
      for (int k = lane; k < a.n_top; k += 32) all[w * a.n_top + k] = s_buf[w][k];
    lp_cut<LP_BUF>(all, LP_WARPS * a.n_top, a.n_top);
  }
  __syncthreads();
  lp_finish<T>(a, row, s_stat, s_buf[0], tid);
}

struct LpGradParams {
  const void* logits;
  long long ld, ld_grad;
  int rows, V, segs;
  float scale;
  const int32_t* targets;
  const float *row_stats, *entropy, *g_logprob, *g_entropy;
  void* grad;
  int* err;
};

constexpr int LP_GRAD_VECS = 4;  // vectors per thread

// CTA (row, run of LP_GRAD_VECS x 256 vectors).
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) k_logprobs_grad(const LpGradParams a) {
  constexpr int N = Vec<T>::N;
  pdl_launch_dependents();
  pdl_wait();
  const int row = blockIdx.x / a.segs, seg = blockIdx.x % a.segs;
  const Row<T> r(reinterpret_cast<const T*>(a.logits) + row * a.ld, a.V);
  T* out = reinterpret_cast<T*>(a.grad) + row * a.ld_grad;
  const bool same = (((uintptr_t)out ^ (uintptr_t)r.p) & 15) == 0;  // the row's vectors are vectors of the output too
  const float m = a.row_stats[2 * (long long)row], ls = a.row_stats[2 * (long long)row + 1], gh = a.g_entropy ? a.g_entropy[row] : 0.f, H = a.g_entropy ? a.entropy[row] : 0.f;
  const int target = a.targets[row];
  float g = target >= 0 && a.g_logprob ? a.g_logprob[row] : 0.f;
  if (target >= a.V) {
    if (threadIdx.x == 0 && seg == 0) jf_set_error(a.err, JF_DERR_BOUNDS);
    g = 0.f;
  }
  const bool none = m == -INFINITY && ls == -INFINITY;
  float x[LP_GRAD_VECS][N];
  const int v0 = seg * (LP_GRAD_VECS * LP_THREADS) + threadIdx.x;
#pragma unroll
  for (int u = 0; u < LP_GRAD_VECS; ++u) r.load(v0 + u * LP_THREADS, v0 + u * LP_THREADS < r.n_vec, x[u]);
#pragma unroll
  for (int u = 0; u < LP_GRAD_VECS; ++u) {
    const int v = v0 + u * LP_THREADS;
    if (v >= r.n_vec) break;
    const long long e0 = r.first(v);
    float d[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float lp = fmaf(x[u][i] - m, a.scale, -ls), p = ex2_ftz(lp * LOG2E);
      // -g p - gh p (lp + H), the logit of probability 0 without its infinite lp
      const float share = g + gh * (fmaxf(lp, -1e4f) + H);
      d[i] = none ? 0.f : a.scale * ((e0 + i == target ? g : 0.f) - p * share);
    }
    if (same && r.whole(v)) {
      Vec<T>::store(out + e0, d);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (e0 + i >= 0 && e0 + i < a.V) out[e0 + i] = to_act<T>(d[i]);
    }
  }
}

template <typename K, typename P>
cudaError_t lp_launch(K kernel, long long grid, cudaStream_t st, const P& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(LP_THREADS);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

// Segments of a row: enough CTAs to fill the GPU, none shorter than LP_SEG_MIN logits.
int lp_segments(int rows, int V) {
  const int most = (V + LP_SEG_MIN - 1) / LP_SEG_MIN, want = LP_CTAS / rows;
  return want < 1 ? 1 : (want < most ? want : most);
}

template <typename T>
cudaError_t launch_logprobs(const LpParams& a, cudaStream_t st) {
  const bool top = a.n_top > 0;
  const long long grid = (long long)a.rows * a.segs;
  cudaError_t e = top ? lp_launch(k_logprobs<T, true>, grid, st, a) : lp_launch(k_logprobs<T, false>, grid, st, a);
  if (e != cudaSuccess || a.segs == 1) return e;
  return top ? lp_launch(k_logprobs_join<T, true>, a.rows, st, a) : lp_launch(k_logprobs_join<T, false>, a.rows, st, a);
}

bool lp_shape_ok(int dtype, const void* logits, long long ld, int rows, int vocab, float scale) {
  if ((dtype != JF_F32 && dtype != JF_BF16) || rows < 0 || vocab < 1 || vocab > (1 << 30)) return false;
  if (!(scale > 0.f) || scale > 1e30f || ld < vocab) return false;
  return rows == 0 || (logits && ((uintptr_t)logits & (dtype == JF_BF16 ? 1 : 3)) == 0);
}

}  // namespace
}  // namespace jf

using namespace jf;

extern "C" jf_status jf_op_token_logprobs_workspace_bytes(int rows, int vocab, int n_top, size_t* out_bytes) {
  if (rows < 0 || vocab < 1 || n_top < 0 || n_top > JF_LOGPROBS_MAX_TOP || !out_bytes) return JF_EINVAL;
  const int segs = rows > 0 ? lp_segments(rows, vocab) : 1;
  *out_bytes = segs > 1 ? (size_t)rows * segs * (16 + 8 * (size_t)n_top) : 0;
  return JF_OK;
}

extern "C" jf_status jf_op_token_logprobs(int dtype, const void* logits, long long ld, int rows, int vocab, float scale,
                                          const int32_t* targets, float* logprob, float* entropy, float* lse, float* row_stats,
                                          int n_top, int32_t* top_ids, float* top_logprobs, void* workspace,
                                          size_t workspace_bytes, int* err_word, void* cuda_stream) {
  if (!lp_shape_ok(dtype, logits, ld, rows, vocab, scale) || !err_word || n_top < 0 || n_top > JF_LOGPROBS_MAX_TOP) return JF_EINVAL;
  if (rows == 0) return JF_OK;
  if ((logprob && !targets) || (n_top > 0 && (!top_ids || !top_logprobs))) return JF_EINVAL;
  size_t need = 0;
  jf_op_token_logprobs_workspace_bytes(rows, vocab, n_top, &need);
  if (need > 0 && (!workspace || workspace_bytes < need)) return JF_ENOMEM;
  if ((uintptr_t)workspace & 15) return JF_EINVAL;
  LpParams a = {logits, ld, rows, vocab, n_top, lp_segments(rows, vocab), scale, targets, logprob, entropy, lse, row_stats,
                top_ids, top_logprobs, nullptr, nullptr, err_word};
  if (a.segs > 1) {
    a.stats = reinterpret_cast<float4*>(workspace);
    a.lists = reinterpret_cast<unsigned long long*>(a.stats + (size_t)rows * a.segs);
  }
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == JF_BF16 ? launch_logprobs<bf16>(a, st) : launch_logprobs<float>(a, st);
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}

extern "C" jf_status jf_op_token_logprobs_grad(int dtype, const void* logits, long long ld, int rows, int vocab,
                                               float scale, const int32_t* targets, const float* row_stats,
                                               const float* entropy, const float* grad_logprob,
                                               const float* grad_entropy, void* grad_logits, long long ld_grad,
                                               int* err_word, void* cuda_stream) {
  if (!lp_shape_ok(dtype, logits, ld, rows, vocab, scale) || !err_word || ld_grad < vocab) return JF_EINVAL;
  if (rows == 0) return JF_OK;
  if (!targets || !row_stats || !grad_logits || (grad_entropy && !entropy)) return JF_EINVAL;
  if ((uintptr_t)grad_logits & (dtype == JF_BF16 ? 1 : 3)) return JF_EINVAL;
  if (grad_logits == logits && ld_grad != ld) return JF_EINVAL;
  const int n = dtype == JF_BF16 ? Vec<bf16>::N : Vec<float>::N;
  const int per_cta = LP_GRAD_VECS * LP_THREADS * n;
  const int segs = (int)(((long long)vocab + n - 1 + per_cta - 1) / per_cta);  // (a row may begin n - 1 elements into a vector)
  const LpGradParams a = {logits, ld, ld_grad, rows, vocab, segs, scale, targets, row_stats, entropy, grad_logprob, grad_entropy,
                          grad_logits, err_word};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const long long grid = (long long)rows * segs;
  if (grid > 0x7fffffffll) return JF_EUNSUPPORTED;
  const cudaError_t e = dtype == JF_BF16 ? lp_launch(k_logprobs_grad<bf16>, grid, st, a) : lp_launch(k_logprobs_grad<float>, grid, st, a);
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}
