// The clipped policy loss of given tokens with KL and entropy terms, and its gradient by the logits (jf_ops.h).
//
// With lp = z_target - lse over z = scale * logits, ratio = e^(lp - old), A the advantage, d = ref - lp:
//   loss = w (-min(ratio A, clip(ratio) A) + beta (e^d - 1 - d) - eta H)
//   dloss/dlp = w (-ratio A [ratio A <= clip(ratio) A] + beta (1 - e^d)) = g
//   dloss/dlogit_i = scale (g (1{i = target} - p_i) + w eta p_i (ln p_i + H))
// Loss and gradient are one pass: a cluster of CTAs holds a row in registers between its sums and its gradient, so that every
// logit is read once and every gradient written once. Rows longer than a cluster of eight holds take the log probabilities'
// two kernels, with one for the rows between them.
#include "jf_logprobs.cuh"

namespace jf {
namespace {

struct PolicyParams {
  jf_policy_terms t;
  const void* logits;
  long long ld, ld_grad;
  int rows, V;
  float scale;
  const int32_t* targets;
  const float *old_lp, *ref_lp, *adv, *weight;
  const float *lp_in, *H_in;  // of the rows, where another kernel has found them
  float *loss, *lp, *H, *ratio, *kl;
  void* grad;
  float *g, *gh;  // gradients by the log probability and by the entropy, for another kernel
  int* err;
};

struct PolicyRow {
  float loss, ratio, kl, g, gh;
};
// A row's terms; target: as given, old, ref, A, w: its inputs (old, ref only where there are any).
JF_DEV PolicyRow policy_row(const PolicyParams& a, int target, float lp, float H, float old, float ref, float A, float w) {
  PolicyRow r;
  const bool on = target >= 0;
  r.ratio = a.old_lp ? expf(lp - old) : 1.f;
  const float free = A == 0.f ? 0.f : r.ratio * A, held = A == 0.f ? 0.f : fminf(fmaxf(r.ratio, 1.f - a.t.below), 1.f + a.t.above) * A;
  float sum = free <= held ? -free : -held;
  r.g = free <= held ? -free : 0.f;
  if (!(free <= held) && !(held < free)) sum = free - held;  // (not a number)
  r.kl = 0.f;
  if (a.ref_lp) {
    const float d = ref - lp, e = expm1f(d);
    const bool out = d == INFINITY;
    r.kl = out ? INFINITY : e - d;
    if (a.t.kl != 0.f) {
      sum = fmaf(a.t.kl, r.kl, sum);
      if (!out) r.g = fmaf(-a.t.kl, e, r.g);
    }
  }
  if (a.t.entropy != 0.f) sum = fmaf(-a.t.entropy, H, sum);
  const bool counts = on && w != 0.f, moves = counts && target < a.V;
  r.loss = counts ? w * sum : 0.f;
  r.ratio = on ? r.ratio : 0.f;
  r.kl = on ? r.kl : 0.f;
  r.g = moves ? w * r.g : 0.f;
  r.gh = moves ? -w * a.t.entropy : 0.f;
  return r;
}

// ---------------------------------------------------------------------------------------------
// One pass: cluster (row), each CTA a run of the row's vectors, U a thread.
// ---------------------------------------------------------------------------------------------
constexpr int PL_THREADS = 512, PL_WARPS = PL_THREADS / 32, PL_MOST = 10, PL_CLUSTER = 8;

// (m, S, T) of a warp's lanes, joined in lane order.
JF_DEV LpStat join_lanes(LpStat st, int lanes, int lane, float c) {
  for (int o = 1; o < lanes; o <<= 1) {
    const LpStat b = {__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), __shfl_xor_sync(0xffffffffu, st.t, o)};
    st = lane & o ? lp_join(b, st, c) : lp_join(st, b, c);
  }
  return st;
}
JF_DEV float ld_cluster(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

// 16 bytes from byte `skip` (2 .. 14, even) on of two pieces that lie one behind the other.
JF_DEV uint4 straddle(const uint4& x, const uint4& y, int skip) {
  const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  const int sh = (skip & 2) * 8;
  uint32_t o[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t lo = w[k], hi = w[k + 1];
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      lo = skip >> 2 == i ? w[k + i] : lo;
      if (k + i + 1 < 8) hi = skip >> 2 == i ? w[k + i + 1] : hi;
    }
    o[k] = __funnelshift_r(lo, hi, sh);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

template <typename T, int U>
__global__ void __launch_bounds__(PL_THREADS, 2) k_policy(const PolicyParams a) {
  constexpr int N = Vec<T>::N;
  __shared__ LpStat s_warp[PL_WARPS], s_cta;
  __shared__ float s_row[5];  // m, ln S, H, g, gh
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t parts;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  const int rank = (int)cluster_rank(), row = blockIdx.x / parts;
  const Row<T> r(reinterpret_cast<const T*>(a.logits) + row * a.ld, a.V);
  const int v_begin = (int)((long long)r.n_vec * rank / (int)parts), v_end = (int)((long long)r.n_vec * (rank + 1) / (int)parts);
  const float c = a.scale * LOG2E;
  uint4 raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int v = v_begin + u * PL_THREADS + tid;
    raw[u] = v < v_end ? Vec<T>::raw(r.vec(v)) : Vec<T>::nothing();
  }
  const int e = r.edge(tid);
  const bool edge = e >= 0 && rank == (tid < N ? 0 : (int)parts - 1);
  const float at_edge = edge ? act_to_f32(r.p[e]) : -INFINITY;
  const int target = a.targets[row];
  const float x_t = target >= 0 && target < a.V ? act_to_f32(r.p[target]) : 0.f;  // (before a gradient in its place)

  float m = at_edge;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float x[N];
    Vec<T>::unpack(raw[u], x);
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
  }
  LpStat st;
  {
    const float base = m == -INFINITY ? 0.f : -m;
    F2 s = {0.f, 0.f}, t = {0.f, 0.f};
    auto add = [&](F2 x) {
      const F2 d = add2(x, {base, base});
      F2 p = mul2(d, {c, c});
      p = {ex2_ftz(p.x), ex2_ftz(p.y)};
      s = add2(s, p);
      t = fma2(p, {fmaxf(d.x, -1e30f), fmaxf(d.y, -1e30f)}, t);  // (0 where x = -inf)
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[N];
      Vec<T>::unpack(raw[u], x);
#pragma unroll
      for (int i = 0; i < N; i += 2) add({x[i], x[i + 1]});
    }
    if (edge) add({at_edge, -INFINITY});
    st = join_lanes({m, s.x + s.y, t.x + t.y}, 32, lane, c);
  }
  if (lane == 0) s_warp[warp] = st;
  __syncthreads();
  if (warp == 0) {
    st = join_lanes(s_warp[lane & (PL_WARPS - 1)], PL_WARPS, lane, c);
    if (lane == 0) s_cta = st;
    __syncwarp();
  }
  if (parts > 1) cluster_sync();
  if (warp == 0) {
    if (parts > 1) {
      const uint32_t from = map_to_rank(smem_u32(&s_cta), (uint32_t)lane & (parts - 1));
      st = join_lanes({ld_cluster(from), ld_cluster(from + 4), ld_cluster(from + 8)}, (int)parts, lane, c);
    }
    const bool none = st.m == -INFINITY && st.s == 0.f;  // no token can occur
    const float base = st.m == -INFINITY ? 0.f : st.m, ls = logf(st.s), H = none ? 0.f : ls - a.scale * (st.t / st.s);
    float lp = 0.f;
    if (target >= a.V) lp = __int_as_float(0x7fffffff);
    else if (target >= 0) lp = none ? -INFINITY : fmaf(x_t - base, a.scale, -ls);
    const PolicyRow p = policy_row(a, target, lp, H, a.old_lp ? a.old_lp[row] : 0.f, a.ref_lp ? a.ref_lp[row] : 0.f, a.adv[row],
                                   a.weight ? a.weight[row] : 1.f);
    if (lane == 0) {
      // a row without a token that can occur has no gradient
      s_row[0] = st.m, s_row[1] = ls, s_row[2] = H, s_row[3] = p.g, s_row[4] = p.gh;
      if (rank == 0) {
        if (target >= a.V) jf_set_error(a.err, JF_DERR_BOUNDS);
        if (a.loss) a.loss[row] = p.loss;
        if (a.lp) a.lp[row] = lp;
        if (a.H) a.H[row] = H;
        if (a.ratio) a.ratio[row] = p.ratio;
        if (a.kl) a.kl[row] = p.kl;
      }
    }
  }
  __syncthreads();
  // a peer's sums have been read; its memory is there until all have
  if (parts > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  if (a.grad) {
    const float mx = s_row[0], ls = s_row[1], H = s_row[2], g = s_row[3], gh = s_row[4];
    const bool none = mx == -INFINITY && ls == -INFINITY, still = none || (g == 0.f && gh == 0.f);
    const float k = a.scale;
    // -scale p (g + gh (ln p + H)) of a logit; a probability of 0 without its infinite logarithm
    auto of = [&](float x, float hot) {
      const float lp = fmaf(x - mx, k, -ls), p = ex2_ftz(lp * LOG2E);
      const float share = gh == 0.f ? g : fmaf(gh, fmaxf(lp, -1e4f) + H, g);
      return still ? 0.f : k * fmaf(-p, share, hot);
    };
    T* out = reinterpret_cast<T*>(a.grad) + row * a.ld_grad;
    if (edge) out[e] = to_act<T>(of(at_edge, e == target ? g : 0.f));
    const int skip = (int)((16 - ((uintptr_t)(out + r.head) & 15)) & 15);  // bytes of a vector before its output's next 16-byte boundary
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = v_begin + u * PL_THREADS + tid, e0 = r.head + v * N;
      float x[N], d[N];
      Vec<T>::unpack(raw[u], x);
      if (target >= e0 && target < e0 + N) {
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] = of(x[i], e0 + i == target ? g : 0.f);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] = of(x[i], 0.f);
      }
      if (skip == 0) {
        if (v < v_end) Vec<T>::store(out + e0, d);
      } else {
        // whole 16-byte pieces of the output, each of two neighbours' elements; a warp's ends go one by one
        uint4 w, n;
        if constexpr (N == 8) {
          uint32_t q[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(d[2 * i], d[2 * i + 1]);
            q[i] = *reinterpret_cast<const uint32_t*>(&b);
          }
          w = make_uint4(q[0], q[1], q[2], q[3]);
        } else {
          w = make_uint4(__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3]));
        }
        n.x = __shfl_down_sync(0xffffffffu, w.x, 1), n.y = __shfl_down_sync(0xffffffffu, w.y, 1);
        n.z = __shfl_down_sync(0xffffffffu, w.z, 1), n.w = __shfl_down_sync(0xffffffffu, w.w, 1);
        const int own = skip / (int)sizeof(T);
        const bool whole = lane < 31 && v + 1 < v_end;
        if (whole) __stcs(reinterpret_cast<uint4*>(out + e0 + own), straddle(w, n, skip));
        if (v < v_end && (lane == 0 || !whole)) {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (i < own ? lane == 0 : !whole) out[e0 + i] = to_act<T>(d[i]);
        }
      }
    }
  }
  if (parts > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---------------------------------------------------------------------------------------------
// Rows longer than that: the terms of each row from its log probability and entropy.
// ---------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(128) k_policy_rows(const PolicyParams a) {
  const int r = blockIdx.x * 128 + threadIdx.x;
  if (r >= a.rows) return;
  const PolicyRow p = policy_row(a, a.targets[r], a.lp_in[r], a.H_in[r], a.old_lp ? a.old_lp[r] : 0.f, a.ref_lp ? a.ref_lp[r] : 0.f, a.adv[r],
                                 a.weight ? a.weight[r] : 1.f);
  if (a.loss) a.loss[r] = p.loss;
  if (a.ratio) a.ratio[r] = p.ratio;
  if (a.kl) a.kl[r] = p.kl;
  a.g[r] = p.g;
  a.gh[r] = p.gh;
}

size_t align16(size_t n) { return (n + 15) / 16 * 16; }

// CTAs of a row's cluster and vectors of a thread; parts 0: a cluster does not hold the row. More CTAs than it takes where
// rows are few.
struct PolicyForm {
  int parts, vecs;
};
PolicyForm policy_form(int dtype, int rows, int vocab) {
  const int n = dtype == JF_BF16 ? Vec<bf16>::N : Vec<float>::N, vecs = vocab / n;
  int parts = 1;
  while (parts < PL_CLUSTER && (vecs + parts - 1) / parts > PL_MOST * PL_THREADS) parts *= 2;
  if ((vecs + parts - 1) / parts > PL_MOST * PL_THREADS) return {0, 0};
  while (parts < PL_CLUSTER && (long long)rows * parts * 2 <= 152 && vecs / parts > 2 * PL_THREADS) parts *= 2;
  const int each = (vecs + parts - 1) / parts;
  return {parts, each <= 2 * PL_THREADS ? 2 : (each <= 5 * PL_THREADS ? 5 : 10)};
}

template <typename T, int U>
cudaError_t policy_launch(const PolicyParams& a, int parts, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.rows * parts);
  cfg.blockDim = dim3(PL_THREADS);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)parts, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_policy<T, U>, a);
}
template <typename T>
cudaError_t policy_launch(const PolicyParams& a, PolicyForm f, cudaStream_t st) {
  return f.vecs == 2 ? policy_launch<T, 2>(a, f.parts, st) : (f.vecs == 5 ? policy_launch<T, 5>(a, f.parts, st) : policy_launch<T, 10>(a, f.parts, st));
}

}  // namespace
}  // namespace jf

using namespace jf;

extern "C" jf_status jf_op_policy_loss_workspace_bytes(int dtype, int rows, int vocab, size_t* out_bytes) {
  if ((dtype != JF_F32 && dtype != JF_BF16) || rows < 0 || vocab < 1 || !out_bytes) return JF_EINVAL;
  *out_bytes = 0;
  if (rows == 0 || policy_form(dtype, rows, vocab).parts > 0) return JF_OK;
  size_t n = 0;
  const jf_status s = jf_op_token_logprobs_workspace_bytes(rows, vocab, 0, &n);
  if (s != JF_OK) return s;
  *out_bytes = align16(n) + (size_t)rows * 6 * 4;  // logprob, entropy, row_stats, g, gh
  return JF_OK;
}

extern "C" jf_status jf_op_policy_loss(const jf_policy_terms* terms, int dtype, const void* logits, long long ld, int rows,
                                       int vocab, float scale, const int32_t* targets, const float* old_logprob,
                                       const float* ref_logprob, const float* advantage, const float* weight, float* loss,
                                       float* logprob, float* entropy, float* ratio, float* kl, void* grad_logits,
                                       long long ld_grad, void* workspace, size_t workspace_bytes, int* err_word,
                                       void* cuda_stream) {
  auto finite = [](float v) { return v - v == 0.f; };
  if (!terms || !(terms->below >= 0.f && terms->below <= 1.f) || !(terms->above >= 0.f) || !finite(terms->kl) || !finite(terms->entropy) ||
      (!ref_logprob && terms->kl != 0.f) || (dtype != JF_F32 && dtype != JF_BF16) || rows < 0 || vocab < 1 || vocab > (1 << 30) || !err_word)
    return JF_EINVAL;
  if (!(scale > 0.f) || scale > 1e30f || ld < vocab) return JF_EINVAL;
  if (rows == 0) return JF_OK;
  const uintptr_t type_mask = dtype == JF_BF16 ? 1 : 3;
  if (!logits || ((uintptr_t)logits & type_mask) || !targets || !advantage) return JF_EINVAL;
  if (grad_logits && (ld_grad < vocab || ((uintptr_t)grad_logits & type_mask) || (grad_logits == logits && ld_grad != ld))) return JF_EINVAL;
  size_t need = 0;
  jf_status s = jf_op_policy_loss_workspace_bytes(dtype, rows, vocab, &need);
  if (s != JF_OK) return s;
  if (need > 0 && (!workspace || workspace_bytes < need)) return JF_ENOMEM;
  if ((uintptr_t)workspace & 15) return JF_EINVAL;
  PolicyParams a = {*terms, logits, ld, ld_grad, rows, vocab, scale, targets, old_logprob, ref_logprob, advantage, weight, nullptr, nullptr,
                    loss, logprob, entropy, ratio, kl, grad_logits, nullptr, nullptr, err_word};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const PolicyForm f = policy_form(dtype, rows, vocab);
  if (f.parts > 0) {
    if ((long long)rows * f.parts > 0x7fffffffll) return JF_EUNSUPPORTED;
    const cudaError_t e = dtype == JF_BF16 ? policy_launch<bf16>(a, f, st) : policy_launch<float>(a, f, st);
    return e == cudaSuccess ? JF_OK : JF_ECUDA;
  }
  size_t scores = 0;
  jf_op_token_logprobs_workspace_bytes(rows, vocab, 0, &scores);
  float* at = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + align16(scores));
  float *lp = logprob ? logprob : at, *H = entropy ? entropy : at + rows, *stats = at + 2 * (size_t)rows;
  s = jf_op_token_logprobs(dtype, logits, ld, rows, vocab, scale, targets, lp, H, nullptr, stats, 0, nullptr, nullptr, workspace,
                           scores, err_word, cuda_stream);
  if (s != JF_OK) return s;
  a.lp_in = lp, a.H_in = H, a.g = at + 4 * (size_t)rows, a.gh = at + 5 * (size_t)rows;
  k_policy_rows<<<(rows + 127) / 128, 128, 0, st>>>(a);
  if (cudaGetLastError() != cudaSuccess) return JF_ECUDA;
  if (!grad_logits) return JF_OK;
  return jf_op_token_logprobs_grad(dtype, logits, ld, rows, vocab, scale, targets, stats, H, a.g, a.gh, grad_logits, ld_grad, err_word,
                                   cuda_stream);
}
