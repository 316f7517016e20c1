// Log probabilities of given tokens with entropy and top alternatives, and their gradient (jf_ops.h).
//
// One pass over the logits x. Against a running maximum m, with d = x - m,
//   S = sum e^(scale d),  T = sum e^(scale d) d,   lse = scale m + ln S,   entropy = ln S - scale T / S,
// and when m grows, T takes the step times S before both shrink. (The difference comes first: where every logit is
// the type's lowest value, as in a row that a mask has emptied, x log2 e would overflow.) Every thread keeps its own (m, S, T); they are joined in
// thread order. The top list is kept per CTA: a buffer of candidates that exceed its n_top'th best so far, ordered by
// (value, lower index) as one 64-bit key, and cut back to n_top when it fills, so the list does not depend on the
// order in which candidates arrive. A bound comes first, from a sample of the row: some 150 of 152,064 logits then are
// candidates for a list of 20. Few rows are cut into segments (one CTA each), whose states
// and lists a second kernel joins in segment order.
#include <type_traits>

#include "jf_logprobs.cuh"

namespace jf {
namespace {

constexpr int LP_THREADS = 256, LP_WARPS = LP_THREADS / 32;
constexpr int LP_BUF = 2 * LP_THREADS;         // candidates a CTA holds
constexpr int LP_SEG_MIN = 4096;    // fewest logits of a segment
constexpr int LP_CTAS = 608;        // CTAs that fill the GPU (152 SMs x 4)
constexpr int NO_TOKEN = 0x7fffffff;

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

// The largest float below v (v itself at -infinity).
JF_DEV float lp_below(float v) {
  if (v == 0.f) return -1.4e-45f;
  const int b = __float_as_int(v);
  return v == -INFINITY ? v : __int_as_float(v > 0.f ? b - 1 : b + 1);
}

// The n largest of buf[0 .. count) (count <= LP_BUF, distinct keys but for zeros) in falling order into buf[0 .. n), zeros after the
// last: a key's place is the number of larger ones. By the whole CTA, buf ready.
JF_DEV void lp_cut_cta(unsigned long long* buf, int count, int n) {
  constexpr int R = LP_BUF / LP_THREADS;
  unsigned long long e[R];
  int place[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int i = threadIdx.x + k * LP_THREADS;
    e[k] = i < count ? buf[i] : 0ull;
    place[k] = 0;
  }
  if (__any_sync(0xffffffffu, e[1] != 0)) {
#pragma unroll 4
    for (int i = 0; i < count; ++i) {
      const unsigned long long o = buf[i];
      place[0] += o > e[0];
      place[1] += o > e[1];
    }
  } else if (__any_sync(0xffffffffu, e[0] != 0)) {  // (warps without a key have nothing to place)
#pragma unroll 4
    for (int i = 0; i < count; ++i) place[0] += buf[i] > e[0];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += LP_THREADS) buf[i] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < R; ++k)
    if (e[k] && place[k] < n) buf[place[k]] = e[k];
  __syncthreads();
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

// A CTA's candidates.
struct LpTop {
  unsigned long long buf[LP_BUF];
  int count;
};

// CTA (row, segment). TOP: a list is asked for. Bound by the logits' bytes and, at 5 instructions and an exponential a
// logit, by the issue of instructions, about alike: 512 rows of 152,064 bf16 logits (156 MB) take 32 us without a list
// (4.9 TB/s), 46 with 20 alternatives (the sample, 6 us, then a comparison a pair and some 150 candidates a row), 56
// with 64; fp32 (311 MB) 48 and 56. One fp32 row of 151,936: 9.6 us in 38 segments, most of it the chain of two launches.
template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_THREADS, 4) k_logprobs(const LpParams a) {
  constexpr int N = Vec<T>::N;
  constexpr int U = sizeof(T) == 2 ? 2 : 4;  // vectors a thread takes at a time
  __shared__ LpTop top;
  __shared__ int s_first;
  __shared__ LpStat s_stat[LP_WARPS];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x / a.segs, seg = blockIdx.x % a.segs;
  const Row<T> r(reinterpret_cast<const T*>(a.logits) + row * a.ld, a.V);
  const int v_begin = (int)((long long)r.n_vec * seg / a.segs), v_end = (int)((long long)r.n_vec * (seg + 1) / a.segs);
  const float c = a.scale * LOG2E;
  float m = -INFINITY;
  F2 s = {0.f, 0.f}, t = {0.f, 0.f};
  unsigned long long thr = 0;  // the n_top'th best key so far
  float thr_v = -INFINITY;     // candidates exceed it
  // A cut costs the square of what it looks at, and tightens the bound.
  const int cut_at = a.n_top + max(a.n_top, 32);
  if (TOP && tid == 0) top.count = 0;
  if (TOP) __syncthreads();

  auto raise = [&](float mx) {  // the thread's maximum
    if (mx > m) {
      if (m > -INFINITY) {  // (before the first number the sums are 0, or NaN)
        const float d = m - mx, al = ex2_ftz(d * c), dd = fmaxf(d, -1e30f);
        t = {al * fmaf(dd, s.x, t.x), al * fmaf(dd, s.y, t.y)};
        s = {al * s.x, al * s.y};
      }
      m = mx;
    }
  };
  auto add = [&](F2 x, float base) {
    const F2 d = add2(x, {base, base});
    F2 e = mul2(d, {c, c});
    e = {ex2_ftz(e.x), ex2_ftz(e.y)};
    s = add2(s, e);
    t = fma2(e, {fmaxf(d.x, -1e30f), fmaxf(d.y, -1e30f)}, t);  // (0 where x = -inf)
  };
  auto cut = [&]() {  // by the whole CTA, all candidates in place
    const int count = top.count;
    lp_cut_cta(top.buf, count, a.n_top);
    if (tid == 0) top.count = min(count, a.n_top);
    thr = top.buf[a.n_top - 1];
    if (thr) thr_v = fmaxf(thr_v, lp_below(lp_key_value(thr)));  // (an equal value of a lower index may still come)
    __syncthreads();
  };
  // M values of each thread, index(i) that of x[i]; by the whole CTA. One barrier where nothing special happens: after
  // it candidates of the next call may already arrive, so what it decides goes by the places that threads were given.
  auto offer = [&](const auto& x, float mx, auto index, auto m_const) {
    constexpr int M = decltype(m_const)::value;
    int first_at = LP_BUF, last_at = -1;
    if (mx > thr_v) {
#pragma unroll
      for (int i = 0; i < M; ++i) {
        if (x[i] > thr_v) {
          const unsigned long long key = lp_key(x[i], index(i));
          if (key > thr) {
            last_at = atomicAdd(&top.count, 1);
            first_at = min(first_at, last_at);
            if (last_at < LP_BUF) top.buf[last_at] = key;
          }
        }
      }
    }
    if (!__syncthreads_or(last_at >= cut_at)) return;
    if (top.count > LP_BUF) {  // more than fit (a row that climbs): again, one value of each thread at a time
      if (tid == 0) s_first = LP_BUF;
      __syncthreads();
      atomicMin(&s_first, first_at);
      __syncthreads();
      if (tid == 0) top.count = s_first;
      __syncthreads();
#pragma unroll 1
      for (int i = 0; i < M; ++i) {
        if (top.count > LP_BUF - LP_THREADS) cut();
        float xi = x[0];
#pragma unroll
        for (int k = 1; k < M; ++k)
          if (i == k) xi = x[k];
        const unsigned long long key = lp_key(xi, index(i));
        __syncthreads();
        if (xi > thr_v && key > thr) top.buf[atomicAdd(&top.count, 1)] = key;
        __syncthreads();
      }
    }
    cut();
  };

  uint4 next[U];  // the next round's vectors are on their way while one is worked on
  auto ask = [&](int v0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = v0 + u * LP_THREADS + tid;
      next[u] = v < v_end ? Vec<T>::raw(r.vec(v)) : Vec<T>::nothing();
    }
  };
  auto unpack = [&](float (&x)[U * N]) {
#pragma unroll
    for (int u = 0; u < U; ++u) Vec<T>::unpack(next[u], *reinterpret_cast<float(*)[N]>(x + u * N));
  };
  auto largest = [&](const float (&x)[U * N]) {
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < U * N; ++i) mx = fmaxf(mx, x[i]);
    return mx;
  };
  auto index_of = [&](int v0) {
    return [=](int i) { return r.head + (v0 + i / N * LP_THREADS + tid) * N + i % N; };
  };
  const int edge = r.has_edges() ? r.edge(tid) : -1;
  const bool mine = edge >= 0 && seg == (tid < N ? 0 : a.segs - 1);
  const float at_edge[1] = {mine ? act_to_f32(r.p[edge]) : -INFINITY};
  if (TOP) {
    // The bound that the whole segment's candidates have to exceed: n_top logits are at least a value that n_top of the
    // threads' maxima over a sample of rounds reach; a close one by bisection. A sample of 1 / stride leaves some n_top *
    // stride candidates, which fit; each costs about as much as reading 40 vectors. 512 rows of 152,064 logits, 20
    // alternatives, stride 3 / 4 / 6 / 8: bf16 48.1 / 47.3 / 49.1 / 51.5 us, fp32 66.0 / 62.4 / 60.0 / 60.5.
    const int stride = LP_THREADS * U * min(sizeof(T) == 2 ? 4 : 6, max(2, 150 / a.n_top));
    float mx = -INFINITY, x[U * N];
    for (int v0 = v_begin; v0 < v_end; v0 += stride) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int v = v0 + u * LP_THREADS + tid;
        next[u] = v < v_end ? __ldcg(reinterpret_cast<const uint4*>(r.vec(v))) : Vec<T>::nothing();  // (read again soon: kept in L2)
      }
      unpack(x);
      mx = fmaxf(mx, largest(x));
    }
    const uint32_t ours = mx > -INFINITY ? (uint32_t)(lp_key(mx, 0) >> 32) : 0u;
    uint32_t lo = 0u, hi = 0xffffffffu;
    for (int k = 0; k < 32; ++k) {
      const uint32_t mid = lo + (hi - lo) / 2 + 1;
      const int n = __syncthreads_count(ours >= mid);
      if (n >= a.n_top) lo = mid;
      else hi = mid - 1;
      if (lo == hi || (n >= a.n_top && n <= a.n_top + a.n_top / 4)) break;
    }
    if (lo > 0u) thr_v = lp_below(lp_key_value((unsigned long long)lo << 32));
  }
  // candidates, without a barrier; whether they fitted is seen at the end
  auto push = [&](const auto& x, float mx, auto index, auto m_const) {
    constexpr int M = decltype(m_const)::value;
    if (mx > thr_v) {
#pragma unroll
      for (int i = 0; i < M; ++i)
        if (x[i] > thr_v) {
          const int at = atomicAdd(&top.count, 1);
          if (at < LP_BUF) top.buf[at] = lp_key(x[i], index(i));
        }
    }
  };
  using One = std::integral_constant<int, 1>;
  using All = std::integral_constant<int, U * N>;
  if (r.has_edges()) {
    if (TOP) push(at_edge, at_edge[0], [&](int) { return edge; }, One{});
    raise(at_edge[0]);
    if (mine) add({at_edge[0], -INFINITY}, m == -INFINITY ? 0.f : -m);
  }
  ask(v_begin);
  for (int v0 = v_begin; v0 < v_end; v0 += LP_THREADS * U) {
    float x[U * N];
    unpack(x);
    ask(v0 + LP_THREADS * U);
    const float mx = largest(x);
    if (TOP) push(x, mx, index_of(v0), All{});
    raise(mx);
    const float base = m == -INFINITY ? 0.f : -m;
#pragma unroll
    for (int i = 0; i < U * N; i += 2) add({x[i], x[i + 1]}, base);
  }
  if (TOP) {
    __syncthreads();
    if (top.count > LP_BUF) {  // more than fit (many equal values, a row that climbs between sampled rounds): once more,
      __syncthreads();         // with cuts on the way
      if (tid == 0) top.count = 0;
      __syncthreads();
      offer(at_edge, at_edge[0], [&](int) { return edge; }, One{});
      for (int v0 = v_begin; v0 < v_end; v0 += LP_THREADS * U) {
        float x[U * N];
        ask(v0);
        unpack(x);
        offer(x, largest(x), index_of(v0), All{});
      }
    }
  }
  LpStat st = {m, s.x + s.y, t.x + t.y};
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    LpStat b = {__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), __shfl_xor_sync(0xffffffffu, st.t, o)};
    st = lane & o ? lp_join(b, st, c) : lp_join(st, b, c);
  }
  if (lane == 0) s_stat[warp] = st;
  __syncthreads();
  if (TOP) cut();
  st = s_stat[0];
  for (int w = 1; w < LP_WARPS; ++w) st = lp_join(st, s_stat[w], c);
  if (a.segs == 1) {
    lp_finish<T>(a, row, st, top.buf, tid);
  } else {
    if (tid == 0) a.stats[blockIdx.x] = make_float4(st.m, st.s, st.t, 0.f);
    if (TOP)
      for (int k = tid; k < a.n_top; k += LP_THREADS) a.lists[(long long)blockIdx.x * a.n_top + k] = top.buf[k];
  }
}

// Joins a row's segments: one CTA a row.
template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_THREADS) k_logprobs_join(const LpParams a) {
  __shared__ unsigned long long s_buf[LP_BUF], s_bound;
  __shared__ int s_count;
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
    // The n_top best keys are among those that reach the largest of the lists' last keys; where these do not fit, the
    // lists go in runs.
    const unsigned long long* list = a.lists + (long long)row * a.segs * a.n_top;
    const int total = a.segs * a.n_top;
    if (tid == 0) s_bound = 0, s_count = 0;
    __syncthreads();
    for (int i = tid; i < a.segs; i += LP_THREADS) atomicMax(&s_bound, list[(long long)i * a.n_top + a.n_top - 1]);
    __syncthreads();
    const unsigned long long bound = max(s_bound, 1ull);
    for (int i = tid; i < total; i += LP_THREADS) {
      const unsigned long long key = list[i];
      if (key >= bound) {
        const int at = atomicAdd(&s_count, 1);
        if (at < LP_BUF) s_buf[at] = key;
      }
    }
    __syncthreads();
    if (s_count <= LP_BUF) {
      lp_cut_cta(s_buf, s_count, a.n_top);
    } else {
      for (int i0 = 0, have = 0; i0 < total; have = a.n_top) {
        const int n = min(LP_BUF - have, total - i0);
        for (int i = tid; i < n; i += LP_THREADS) s_buf[have + i] = list[i0 + i];
        __syncthreads();
        lp_cut_cta(s_buf, have + n, a.n_top);
        i0 += n;
      }
    }
  }
  __syncthreads();
  lp_finish<T>(a, row, s_stat, s_buf, tid);
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

// d/dx_i of g logprob + h entropy = scale ((i = target) g - p_i (g + h (ln p_i + H))), from the row's (m, ln S) and entropy H.
// CTA (row, run of LP_GRAD_VECS x 256 vectors); the first run's CTA takes the row's edges too. Bound by the bytes, each
// logit read and each gradient written once with four vectors of a thread in flight: 512 rows of 152,064 fp32 logits
// (623 MB) take 94 us, 6.6 TB/s.
// POLICY: g and h may be infinite, and a row whose g and h are 0 holds anything.
template <typename T, bool POLICY>
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
  const bool none = (m == -INFINITY && ls == -INFINITY) || (POLICY && g == 0.f && gh == 0.f);
  auto of = [&](float x, int i) {
    const float lp = fmaf(x - m, a.scale, -ls), p = ex2_ftz(lp * LOG2E);
    if (POLICY) return none ? 0.f : a.scale * policy_grad(p, lp, H, g, gh, i == target);
    // -g p - gh p (lp + H), the logit of probability 0 without its infinite lp
    const float share = g + gh * (fmaxf(lp, -1e4f) + H);
    return none ? 0.f : a.scale * ((i == target ? g : 0.f) - p * share);
  };
  float x[LP_GRAD_VECS][N];
  const int v0 = seg * (LP_GRAD_VECS * LP_THREADS) + threadIdx.x;
#pragma unroll
  for (int u = 0; u < LP_GRAD_VECS; ++u)
    if (v0 + u * LP_THREADS < r.n_vec) Vec<T>::unpack(Vec<T>::raw(r.vec(v0 + u * LP_THREADS)), x[u]);
  if (seg == 0) {
    const int e = r.edge(threadIdx.x);
    if (e >= 0) out[e] = to_act<T>(of(act_to_f32(r.p[e]), e));
  }
#pragma unroll
  for (int u = 0; u < LP_GRAD_VECS; ++u) {
    const int v = v0 + u * LP_THREADS;
    if (v >= r.n_vec) break;
    const int e0 = r.head + v * N;
    float d[N];
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = of(x[u][i], e0 + i);
    if (same) {
      Vec<T>::store(out + e0, d);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) out[e0 + i] = to_act<T>(d[i]);
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

template <bool POLICY>
static jf_status logprobs_grad(int dtype, const void* logits, long long ld, int rows, int vocab, float scale, const int32_t* targets, const float* row_stats,
                               const float* entropy, const float* grad_logprob, const float* grad_entropy, void* grad_logits, long long ld_grad,
                               int* err_word, cudaStream_t st) {
  if (!lp_shape_ok(dtype, logits, ld, rows, vocab, scale) || !err_word || ld_grad < vocab) return JF_EINVAL;
  if (rows == 0) return JF_OK;
  if (!targets || !row_stats || !grad_logits || (grad_entropy && !entropy)) return JF_EINVAL;
  if ((uintptr_t)grad_logits & (dtype == JF_BF16 ? 1 : 3)) return JF_EINVAL;
  if (grad_logits == logits && ld_grad != ld) return JF_EINVAL;
  const int n = dtype == JF_BF16 ? Vec<bf16>::N : Vec<float>::N;
  const int per_cta = LP_GRAD_VECS * LP_THREADS * n;
  const int segs = (vocab + per_cta - 1) / per_cta;
  const LpGradParams a = {logits, ld, ld_grad, rows, vocab, segs, scale, targets, row_stats, entropy, grad_logprob, grad_entropy,
                          grad_logits, err_word};
  const long long grid = (long long)rows * segs;
  if (grid > 0x7fffffffll) return JF_EUNSUPPORTED;
  const cudaError_t e = dtype == JF_BF16 ? lp_launch(k_logprobs_grad<bf16, POLICY>, grid, st, a) : lp_launch(k_logprobs_grad<float, POLICY>, grid, st, a);
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}

extern "C" jf_status jf_op_token_logprobs_grad(int dtype, const void* logits, long long ld, int rows, int vocab,
                                               float scale, const int32_t* targets, const float* row_stats,
                                               const float* entropy, const float* grad_logprob,
                                               const float* grad_entropy, void* grad_logits, long long ld_grad,
                                               int* err_word, void* cuda_stream) {
  return logprobs_grad<false>(dtype, logits, ld, rows, vocab, scale, targets, row_stats, entropy, grad_logprob, grad_entropy, grad_logits, ld_grad,
                              err_word, reinterpret_cast<cudaStream_t>(cuda_stream));
}

jf_status jf::policy_long_grad(int dtype, const void* logits, long long ld, int rows, int vocab, float scale, const int32_t* targets, const float* row_stats,
                               const float* entropy, const float* g, const float* gh, void* grad_logits, long long ld_grad, int* err_word, cudaStream_t st) {
  return logprobs_grad<true>(dtype, logits, ld, rows, vocab, scale, targets, row_stats, entropy, g, gh, grad_logits, ld_grad, err_word, st);
}
