// The clipped policy loss of given tokens with KL and entropy terms, and its gradient by the logits (jf_ops.h).
//
// With lp = z_target - lse over z = scale * logits, ratio = e^(lp - old), A the advantage, d = ref - lp:
//   loss = w (-min(ratio A, clip(ratio) A) + beta (e^d - 1 - d) - eta H)
//   dloss/dlp = w (-ratio A [ratio A <= clip(ratio) A] + beta (1 - e^d)) = g
//   dloss/dlogit_i = scale (g (1{i = target} - p_i) + w eta p_i (ln p_i + H))
// Loss and gradient are one pass: a cluster of CTAs holds a row in shared memory between its sums and its gradient, so that every
// logit is read once and every gradient written once. Rows longer than a cluster of eight holds take the log probabilities'
// two kernels, with one for the rows between them.
#include "jf_logprobs.cuh"
#include "jf_once.h"

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
  if (!(free <= held) && !(held < free)) sum = r.g = free - held;  // (not a number: neither is the gradient)
  r.kl = 0.f;
  if (a.ref_lp) {
    const float d = ref - lp, e = expm1f(d);
    const bool out = e == INFINITY;  // (beyond fp32's range: no gradient)
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
// One pass: cluster (row), each CTA a run of the row's 16-byte vectors, which bulk copies bring to shared memory.
//
// In the log2 domain, with c = scale log2 e and a reference b = c m rounded (m the thread's largest logit): y = x c - b comes
// rounded once from a fused product, S = sum 2^y, T = sum 2^y y; states are joined by their b. Then
//   lp = scale (x_t - m) - ln 2 (log2 S + b - c m),  H = ln 2 (log2 S - T / S),  p = 2^y / S,
//   dloss/dx = -scale / S 2^y (g + gh (H - ln S) + gh ln 2 y), + scale g at the target.
// b is off from c m by up to 2^-24 of it, which every 2^y of the thread takes as a factor: within 2 where |c m| is below 2^24 (PL_NEAR; beyond
// 2^31 S would leave fp32's range). Sums of a row whose largest logit lies further out (or is beyond 1e38, or has a c above 1e6) are taken
// again from differences x - m. A logit so far below the largest that 2^y is 0 (PL_BELOW) counts as one at that distance, so that y, and its
// products with what an entropy term gives, stay in fp32's range whatever the mask and the scale are.
//
// Bound by bytes where rows are many: 2,048 fp32 rows of 152,064 in 441 us (5.65 TB/s of logits in and gradients out, 0.84 of a copy);
// bf16 ones, whose pairs take as many instructions for half the bytes, by waits between the three walks over a row (barriers 2.1, loads 1.9 warps
// an issue; 55% of issue slots): 512 rows in 68 us (4.6 TB/s), at an odd distance 71. Without a gradient 41 us, 2,048 fp32
// rows 297. A row in registers instead of shared memory: 516 us; more CTAs a row than it takes to hold: 80 for 71.
// ---------------------------------------------------------------------------------------------
constexpr int PL_THREADS = 256, PL_WARPS = PL_THREADS / 32, PL_CLUSTER = 8;
constexpr int PL_FIT[3] = {56832, 76288, 115200};  // bytes of a CTA's run with which four, three, two are resident on an SM
constexpr int PL_MOST = PL_FIT[2];
constexpr int PL_ROWS = 1 << 30;  // (a row and the step to the next fit 31 bits)
constexpr float PL_FAR = 1e30f, PL_BELOW = 400.f, PL_LARGE = 1e38f, PL_STEEP = 1e6f, PL_NEAR = 16777216.f, LN2 = 0.69314718055994531f;
constexpr float LOG2E_LO = 1.9259630e-8f;  // log2 e beyond LOG2E

JF_DEV float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
// (b, S, T) of groups of `lanes` lanes, joined: every lane gets its group's. S and T of a lane without a reference (b = -infinity)
// are 0, or NaN.
JF_DEV LpStat join_lanes(LpStat st, int lanes) {
  float b = st.m;
  for (int o = lanes >> 1; o > 0; o >>= 1) b = fmaxf(b, __shfl_xor_sync(0xffffffffu, b, o));
  const float d = st.m == -INFINITY ? 0.f : st.m - b, f = ex2_ftz(d);
  st.t = f * (st.t + d * st.s);
  st.s = f * st.s;
  for (int o = lanes >> 1; o > 0; o >>= 1) {
    st.s += __shfl_xor_sync(0xffffffffu, st.s, o);
    st.t += __shfl_xor_sync(0xffffffffu, st.t, o);
  }
  return {b, st.s, st.t};
}
// The largest of a vector's values (NaN ignored) and `most`.
JF_DEV float largest(const uint4& v, float most, float) {
  return fmaxf(fmaxf(most, fmaxf(__uint_as_float(v.x), __uint_as_float(v.y))), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
}
JF_DEV float largest(const uint4& v, float most, bf16) {
  const __nv_bfloat162* w = reinterpret_cast<const __nv_bfloat162*>(&v);
  const __nv_bfloat162 m = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
  return fmaxf(most, fmaxf(__low2float(m), __high2float(m)));
}
// Whether sums relative to c m hold where m is the largest logit, of a row (by 1) or of a thread (by 2, so that one whose sums are left
// out lies at least PL_NEAR below the row's largest, if the row's sums hold).
JF_DEV bool holds(float c, float m, float by) { return c <= PL_STEEP && fabsf(m) < PL_LARGE * by && fabsf(c * m) < PL_NEAR * by; }
JF_DEV float max_nan(float x, float y) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
// Two fp32 values as one register pair: constants are packed once, and vectors from shared memory are pairs already.
typedef unsigned long long Pair;
JF_DEV Pair pair(float x, float y) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
JF_DEV F2 halves(Pair p) {
  F2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
  return r;
}
JF_DEV Pair fma_pair(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
JF_DEV Pair add_pair(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
JF_DEV Pair mul_pair(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
JF_DEV Pair ex2_pair(Pair y) {
  const F2 v = halves(y);
  return pair(ex2_ftz(v.x), ex2_ftz(v.y));
}
// A vector's values, none below `low` (bf16: rounded down; NaN kept).
JF_DEV void raised(const uint4& v, Pair (&x)[2], float low) {
  x[0] = pair(max_nan(__uint_as_float(v.x), low), max_nan(__uint_as_float(v.y), low));
  x[1] = pair(max_nan(__uint_as_float(v.z), low), max_nan(__uint_as_float(v.w), low));
}
JF_DEV void raised(const uint4& v, Pair (&x)[4], float low) {
  const __nv_bfloat162 far = __bfloat162bfloat162(__float2bfloat16_rd(low));
  const __nv_bfloat162* w = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 m = __hmax2_nan(w[i], far);
    const uint32_t u = *reinterpret_cast<const uint32_t*>(&m);
    x[i] = pair(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  }
}

// 16 bytes from byte `skip` (2 .. 14, even) on of two pieces that lie one behind the other.
JF_DEV uint4 straddle(const uint4& x, const uint4& y, int skip) {
  const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  uint32_t p[6], q[5], o[4];
#pragma unroll
  for (int k = 0; k < 6; ++k) p[k] = skip & 8 ? w[k + 2] : w[k];
#pragma unroll
  for (int k = 0; k < 5; ++k) q[k] = skip & 4 ? p[k + 1] : p[k];
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = __funnelshift_r(q[k], q[k + 1], (skip & 2) * 8);
  return make_uint4(o[0], o[1], o[2], o[3]);
}
// A row's inputs beside its logits.
struct PolicyInputs {
  int target;
  float old, ref, A, w;
};

// Clusters walk over rows. (Asking for the next row's first half while the second half's gradient leaves took 1 to 3% longer: a
// row is split finely enough that the SM's other CTAs have copies under way.)
template <typename T>
__global__ void __launch_bounds__(PL_THREADS, 4) k_policy(const PolicyParams a) {
  constexpr int N = Vec<T>::N;
  extern __shared__ __align__(128) uint4 s_run[];
  __shared__ __align__(8) uint64_t b_there;
  __shared__ LpStat s_warp[PL_WARPS];
  __shared__ float s_max[PL_WARPS], s_cta[2][4], s_far[2][2];  // by turns (peers read them): the CTA's b, S, T and largest logit; S, T from differences
  __shared__ float s_row[8];                                    // b, log2 S, S, H, g, gh, m, whether far
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    mbar_init(smem_u32(&b_there), 1);
    fence_mbar_init();
  }
  pdl_launch_dependents();
  pdl_wait();
  __syncthreads();
  const uint32_t parts = cluster_ctas();
  const int rank = (int)cluster_rank(), lg = 31 - __clz(parts), rows_apart = gridDim.x >> lg;  // (parts: a power of two)
  const T* logits = reinterpret_cast<const T*>(a.logits);
  // (y is at least -PL_BELOW less what rounding takes: a step of fp32 at PL_NEAR, of bf16 2^17)
  const float c = a.scale * LOG2E, below = PL_BELOW / c;
  // a row's run
  auto ask = [&](int row) {
    const Row<T> r(logits + row * a.ld, a.V);
    const int v_begin = r.n_vec * rank >> lg, bytes = ((r.n_vec * (rank + 1) >> lg) - v_begin) * 16;
    mbar_arrive_expect_tx(smem_u32(&b_there), (uint32_t)bytes);
    if (bytes > 0) bulk_load(smem_u32(s_run), r.vec(v_begin), (uint32_t)bytes, smem_u32(&b_there));
  };
  auto inputs = [&](int row) {  // (asked for a row ahead)
    PolicyInputs q = {-1, 0.f, 0.f, 0.f, 0.f};
    if (row < a.rows) {
      q.target = a.targets[row];
      if (a.old_lp) q.old = a.old_lp[row];
      if (a.ref_lp) q.ref = a.ref_lp[row];
      q.A = a.adv[row];
      q.w = a.weight ? a.weight[row] : 1.f;
    }
    return q;
  };
  int row = blockIdx.x >> lg, turn = 0;
  if (tid == 0 && row < a.rows) ask(row);
  PolicyInputs next = inputs(row);
  for (; row < a.rows; row += rows_apart, turn ^= 1) {
    const Row<T> r(logits + row * a.ld, a.V);
    const int v_begin = r.n_vec * rank >> lg, n = (r.n_vec * (rank + 1) >> lg) - v_begin;
    const PolicyInputs in = next;
    next = inputs(row + rows_apart);
    const int e = r.edge(tid), target = in.target;
    const bool edge = e >= 0 && rank == (tid < N ? 0 : (int)parts - 1);
    const float at_edge = edge ? act_to_f32(r.p[e]) : -INFINITY;
    const float x_t = target >= 0 && target < a.V ? act_to_f32(r.p[target]) : 0.f;  // (before a gradient in its place)

    float m = at_edge;
    if (!mbar_wait_bounded(smem_u32(&b_there), (uint32_t)turn, kWaitLimitDefaultNs)) jf_set_error(a.err, JF_DERR_TIMEOUT_TMA);
#pragma unroll 4
    for (int v = tid; v < n; v += PL_THREADS) m = largest(s_run[v], m, T{});
    LpStat st;
    {
      const float b = holds(c, m, 2.f) ? c * m : -INFINITY;  // (-inf: the thread's sums do not count, or are taken again)
      const float minus = b == -INFINITY ? 0.f : -b, low = b == -INFINITY ? -PL_FAR : m - below;
      const Pair cc = pair(c, c), nb = pair(minus, minus);
      Pair s = 0, t = 0;
      auto add = [&](Pair x) {
        const Pair y = fma_pair(x, cc, nb), p = ex2_pair(y);
        s = add_pair(s, p);
        t = fma_pair(p, y, t);
      };
      // (the vectors that the thread has looked at)
#pragma unroll 2
      for (int v = tid; v < n; v += PL_THREADS) {
        Pair x[N / 2];
        raised(s_run[v], x, low);
#pragma unroll
        for (int k = 0; k < N / 2; ++k) add(x[k]);
      }
      if (edge) add(pair(max_nan(at_edge, low), low));
      st = {b, halves(s).x + halves(s).y, halves(t).x + halves(t).y};
      if (b == -INFINITY && st.s == st.s) st.s = st.t = 0.f;  // (a NaN among them counts)
      st = join_lanes(st, 32);
      m = warp_max(m);
    }
    if (lane == 0) s_warp[warp] = st, s_max[warp] = m;
    __syncthreads();
    if (warp == 0) {
      st = join_lanes(s_warp[lane & (PL_WARPS - 1)], PL_WARPS);
      m = warp_max(s_max[lane & (PL_WARPS - 1)]);
      if (lane == 0) s_cta[turn][0] = st.m, s_cta[turn][1] = st.s, s_cta[turn][2] = st.t, s_cta[turn][3] = m;
      __syncwarp();
    }
    if (parts > 1) cluster_sync();
    bool none = false, far = false;
    if (warp == 0) {
      if (parts > 1) {
        const uint32_t from = map_to_rank(smem_u32(s_cta[turn]), (uint32_t)lane & (parts - 1));
        const float peer_m = ld_cluster(from + 12);
        st = join_lanes({ld_cluster(from), ld_cluster(from + 4), ld_cluster(from + 8)}, (int)parts);
        m = warp_max(peer_m);
      }
      none = m == -INFINITY, far = !none && !holds(c, m, 1.f);
    }
    auto finish = [&]() {  // by warp 0
      const bool empty = none && st.s == 0.f;  // no token can occur
      const float l2 = log2f(st.s), H = empty ? 0.f : LN2 * (l2 - st.t / st.s);
      float lp = 0.f;
      if (target >= a.V) {
        lp = __int_as_float(0x7fffffff);
      } else if (target >= 0) {
        // With c (1 + d) = scale log2 e before c's rounding: log2 of the sum of 2^(c (1 + d) (x - m)) is log2 S + (b - c m) + d T / S
        // but for d's square. (KL is small where lp is near ref_logprob, and would show the rounding.)
        const float d = fmaf(a.scale, LOG2E_LO, fmaf(a.scale, LOG2E, -c)) / c;
        const float apart = far ? 0.f : fmaf(d, st.t / st.s, -fmaf(m, c, -st.m));
        lp = empty ? -INFINITY : fmaf(0.5f * x_t - 0.5f * m, 2.f * a.scale, -LN2 * (l2 + apart));  // (x_t - m may pass fp32's range)
      }
      const PolicyRow p = policy_row(a, target, lp, H, in.old, in.ref, in.A, in.w);
      if (lane == 0) {
        s_row[0] = st.m, s_row[1] = l2, s_row[2] = st.s, s_row[3] = H, s_row[4] = empty ? 0.f : p.g, s_row[5] = empty ? 0.f : p.gh;
        if (rank == 0) {
          if (target >= a.V) jf_set_error(a.err, JF_DERR_BOUNDS);
          if (a.loss) a.loss[row] = p.loss;
          if (a.lp) a.lp[row] = lp;
          if (a.H) a.H[row] = H;
          if (a.ratio) a.ratio[row] = p.ratio;
          if (a.kl) a.kl[row] = p.kl;
        }
      }
      __syncwarp();
    };
    if (warp == 0) {
      if (lane == 0) s_row[6] = m, s_row[7] = far ? 1.f : 0.f;
      if (!far) finish();
      __syncwarp();
    }
    __syncthreads();
    m = s_row[6];
    far = s_row[7] != 0.f;
    if (far) {  // (uniform in the cluster)
      float s = 0.f, t = 0.f;
      auto add = [&](float x) {
        const float d = fmaxf(x - m, -PL_FAR) * c, p = x - m != x - m ? x - m : ex2_ftz(d);  // (a NaN stays one)
        s += p;
        t += p == 0.f ? 0.f : p * d;
      };
      const T* run = reinterpret_cast<const T*>(s_run);
#pragma unroll 1
      for (int v = tid; v < n * N; v += PL_THREADS) add(act_to_f32(run[v]));
      if (edge) add(at_edge);
      s = warp_sum(s), t = warp_sum(t);
      if (lane == 0) s_warp[warp] = {0.f, s, t};
      __syncthreads();
      if (tid == 0) {
        s = t = 0.f;
        for (int w = 0; w < PL_WARPS; ++w) s += s_warp[w].s, t += s_warp[w].t;
        s_far[turn][0] = s, s_far[turn][1] = t;
      }
      __syncthreads();
      if (parts > 1) cluster_sync();
      if (warp == 0) {
        st = {0.f, 0.f, 0.f};
        for (uint32_t k = 0; k < parts; ++k) {
          const uint32_t from = map_to_rank(smem_u32(s_far[turn]), k);
          st.s += ld_cluster(from), st.t += ld_cluster(from + 4);
        }
        finish();
      }
      __syncthreads();
    }
    const float b = s_row[0], l2 = s_row[1], S = s_row[2], H = s_row[3], g = s_row[4], gh = s_row[5], k = a.scale;
    // -scale / S times (g + gh (H - ln S) + gh ln 2 y)
    const float f = -k / S, share0 = f * fmaf(gh, H - LN2 * l2, g), share1 = f * (gh * LN2), hot = k * g;
    const float low = m - below;
    const bool still = g == 0.f && gh == 0.f;  // (also a row without a token that can occur)
    T* out = reinterpret_cast<T*>(a.grad) + (a.grad ? row * a.ld_grad : 0);
    // Whether a 2^y of 0 times its share is 0 (-y < 2^18): not where a term is infinite, or nearly so, or no number. Such rows and those of
    // sums from differences are taken a value at a time.
    const bool plain = !far && fabsf(share0) < 1e38f && fabsf(share1) < 1e32f;
    auto of1 = [&](float x, bool is_target) {
      const float y = far ? (x - m) * c : fmaf(max_nan(x, low), c, -b), p = ex2_ftz(y);
      if (still) return 0.f;
      if (plain) return p * fmaf(y, share1, share0) + (is_target ? hot : 0.f);
      return k * policy_grad(p / S, LN2 * (y - l2), H, g, gh, is_target);
    };
    auto single = [&](int i, float x) { out[i] = to_act<T>(of1(x, i == target)); };
    // Vectors of the output: where it lies otherwise than the logits, each is of two neighbours' elements, and the first and the
    // last of the run's are stored one by one.
    const int skip = (int)((16 - ((uintptr_t)(out + r.head) & 15)) & 15), own = skip / (int)sizeof(T), n_out = skip ? n - 1 : n;
    const int e0 = r.head + v_begin * N;  // the run's first element
    if (a.grad) {
      if (edge) single(e, at_edge);
      if (skip && n > 0 && tid < N) {
        const int i = tid < own ? tid : (n - 1) * N + tid;
        single(e0 + i, act_to_f32(reinterpret_cast<const T*>(s_run)[i]));
      }
    }
    const Pair cc = pair(c, c), nb = pair(-b, -b), k0 = pair(share0, share0), k1 = pair(share1, share1);
    auto vector = [&](int v, bool entropy) {
      const uint4 w = skip ? straddle(s_run[v], s_run[v + 1], skip) : s_run[v];
      const int i0 = e0 + v * N + own;
      Pair x[N / 2];
      float d[N];
      raised(w, x, low);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const Pair y = fma_pair(x[i], cc, nb);
        Pair p = ex2_pair(y);
        p = mul_pair(p, entropy ? fma_pair(y, k1, k0) : k0);
        d[2 * i] = halves(p).x, d[2 * i + 1] = halves(p).y;
      }
      if (target >= i0 && target < i0 + N) {
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] += i0 + i == target ? hot : 0.f;
      }
      Vec<T>::store(out + i0, d);
    };
    const int end = a.grad ? n_out : 0;
    if (still) {
      const float zeros[N] = {};
#pragma unroll 2
      for (int v = tid; v < end; v += PL_THREADS) Vec<T>::store(out + e0 + v * N + own, zeros);
    } else if (!plain) {
#pragma unroll 1
      for (int v = tid; v < end; v += PL_THREADS)
#pragma unroll 1
        for (int h = 0; h < N; ++h) {
          const int at = v * N + own + h;
          single(e0 + at, act_to_f32(reinterpret_cast<const T*>(s_run)[at]));
        }
    } else if (gh != 0.f) {
#pragma unroll 2
      for (int v = tid; v < end; v += PL_THREADS) vector(v, true);
    } else {
#pragma unroll 2
      for (int v = tid; v < end; v += PL_THREADS) vector(v, false);
    }
    __syncthreads();  // (s_row; the run has been read by all: the next row's takes its place)
    if (tid == 0 && row + rows_apart < a.rows) {
      fence_proxy_async_smem();
      ask(row + rows_apart);
    }
  }
  if (parts > 1) cluster_sync();  // peers may still read this CTA's sums
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

// CTAs of a row's cluster; 0: a cluster does not hold the row. More CTAs than it takes where rows are few and long: 16 bf16 rows of
// 152,064 8.3 us instead of 9.3 (16 fp32 rows of 4,096 lose by it, 5.7 instead of 4.8: a CTA has too little to do).
int policy_parts(int dtype, int rows, int vocab) {
  const int vecs = vocab / (dtype == JF_BF16 ? Vec<bf16>::N : Vec<float>::N);
  int parts = 1;
  while (parts < PL_CLUSTER && (vecs + parts - 1) / parts > PL_MOST / 16) parts *= 2;
  if ((vecs + parts - 1) / parts > PL_MOST / 16) return 0;
  while (parts < PL_CLUSTER && (long long)rows * parts * 2 <= 152 && vecs / parts > 4 * PL_THREADS) parts *= 2;
  return parts;
}

// Clusters that are resident at a time, by type, log2 of their CTAs, and place in PL_FIT.
struct PolicyDevice {
  int clusters[2][4][3];
};
PerDeviceOnce g_once;
PolicyDevice g_policy[PerDeviceOnce::kMaxDevices];

struct PolicyLaunch {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  PolicyLaunch(int clusters, int parts, size_t smem, cudaStream_t st) {
    cfg.gridDim = dim3((unsigned)(clusters * parts));
    cfg.blockDim = dim3(PL_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)parts, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
  }
};
template <typename T>
cudaError_t policy_prepare(int (&clusters)[4][3]) {
  cudaError_t e = cudaFuncSetAttribute(k_policy<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, PL_MOST);
  for (int i = 0; i < 12 && e == cudaSuccess; ++i) {
    PolicyLaunch l(1, 1 << i / 3, PL_FIT[i % 3], nullptr);
    l.cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&clusters[i / 3][i % 3], k_policy<T>, &l.cfg);
    if (e == cudaSuccess && clusters[i / 3][i % 3] < 1) e = cudaErrorInvalidConfiguration;
  }
  return e;
}
const PolicyDevice* policy_device() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return nullptr;
  const int rc = g_once.run(dev, [&]() -> int {
    const cudaError_t e = policy_prepare<float>(g_policy[dev].clusters[0]);
    return (int)(e == cudaSuccess ? policy_prepare<bf16>(g_policy[dev].clusters[1]) : e);
  });
  return rc == 0 ? &g_policy[dev] : nullptr;
}

template <typename T>
cudaError_t policy_launch(const PolicyParams& a, int parts, const int (&resident)[4][3], cudaStream_t st) {
  const int smem = (a.V / Vec<T>::N + parts - 1) / parts * 16;
  const int most = resident[parts == 1 ? 0 : (parts == 2 ? 1 : (parts == 4 ? 2 : 3))][smem <= PL_FIT[0] ? 0 : (smem <= PL_FIT[1] ? 1 : 2)];
  PolicyLaunch l(a.rows < most ? a.rows : most, parts, (size_t)smem, st);
  return cudaLaunchKernelEx(&l.cfg, k_policy<T>, a);
}

}  // namespace
}  // namespace jf

using namespace jf;

extern "C" jf_status jf_op_policy_loss_workspace_bytes(int dtype, int rows, int vocab, size_t* out_bytes) {
  if ((dtype != JF_F32 && dtype != JF_BF16) || rows < 0 || vocab < 1 || !out_bytes) return JF_EINVAL;
  *out_bytes = 0;
  if (rows == 0 || policy_parts(dtype, rows, vocab) > 0) return JF_OK;
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
  if (rows > PL_ROWS) return JF_EUNSUPPORTED;
  if (!(scale >= 1e-28f) || scale > 1e30f || ld < vocab) return JF_EINVAL;  // (2^(-1e30 scale log2 e) is 0: differences are cut there)
  if (rows == 0) return JF_OK;
  const uintptr_t type_mask = dtype == JF_BF16 ? 1 : 3;
  if (!logits || ((uintptr_t)logits & type_mask) || !targets || !advantage) return JF_EINVAL;
  if (grad_logits && (ld_grad < vocab || ((uintptr_t)grad_logits & type_mask))) return JF_EINVAL;
  const int size = dtype == JF_BF16 ? 2 : 4;  // (a gradient in its logit's place is written after it was read, any other is not)
  if (grad_logits && (grad_logits != logits || ld_grad != ld) &&
      rows_overlap({logits, ld * size, (long long)vocab * size}, {grad_logits, ld_grad * size, (long long)vocab * size}, rows))
    return JF_EINVAL;
  size_t need = 0;
  jf_status s = jf_op_policy_loss_workspace_bytes(dtype, rows, vocab, &need);
  if (s != JF_OK) return s;
  if (need > 0 && (!workspace || workspace_bytes < need)) return JF_ENOMEM;
  if ((uintptr_t)workspace & 15) return JF_EINVAL;
  PolicyParams a = {*terms, logits, ld, ld_grad, rows, vocab, scale, targets, old_logprob, ref_logprob, advantage, weight, nullptr, nullptr,
                    loss, logprob, entropy, ratio, kl, grad_logits, nullptr, nullptr, err_word};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const int parts = policy_parts(dtype, rows, vocab);
  if (parts > 0) {
    const PolicyDevice* d = policy_device();
    if (!d) return JF_ECUDA;
    const cudaError_t e = dtype == JF_BF16 ? policy_launch<bf16>(a, parts, d->clusters[1], st) : policy_launch<float>(a, parts, d->clusters[0], st);
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
  return policy_long_grad(dtype, logits, ld, rows, vocab, scale, targets, stats, H, a.g, a.gh, grad_logits, ld_grad, err_word, st);
}
