// The clipped policy loss of given tokens with KL and entropy terms, and its gradient by the logits (jf_ops.h).
//
// With lp = z_target - lse over z = scale * logits, ratio = e^(lp - old), A the advantage, d = ref - lp:
//   loss = w (-min(ratio A, clip(ratio) A) + beta (e^d - 1 - d) - eta H)
//   dloss/dlp = w (-ratio A [ratio A <= clip(ratio) A] + beta (1 - e^d)) = g
//   dloss/dlogit_i = scale (g (1{i = target} - p_i) + w eta p_i (ln p_i + H))
#include "../../include/jf_ops.h"
#include "jf_device.cuh"
#include "jf_internal.h"

namespace jf {
namespace {

struct PolicyParams {
  jf_policy_terms t;
  int rows;
  const int32_t* targets;
  const float *old_lp, *ref_lp, *adv, *weight;
  const float *lp, *H;  // of the rows
  float *loss, *ratio, *kl;
  float *g, *gh;        // gradients by the log probability and by the entropy
};

JF_DEV void policy_row(const PolicyParams& a, int r) {
  const bool on = a.targets[r] >= 0;
  const float lp = a.lp[r], A = a.adv[r], w = a.weight ? a.weight[r] : 1.f;
  const float ratio = a.old_lp ? expf(lp - a.old_lp[r]) : 1.f;
  const float free = A == 0.f ? 0.f : ratio * A, held = A == 0.f ? 0.f : fminf(fmaxf(ratio, 1.f - a.t.below), 1.f + a.t.above) * A;
  float sum = free <= held ? -free : -held, g = free <= held ? -free : 0.f, kl = 0.f;
  if (!(free <= held) && !(held < free)) sum = free - held;  // (not a number)
  if (a.ref_lp) {
    const float d = a.ref_lp[r] - lp;
    const bool out = d == INFINITY;
    const float e = expm1f(d);
    kl = out ? INFINITY : e - d;
    if (a.t.kl != 0.f) {
      sum = fmaf(a.t.kl, kl, sum);
      if (!out) g = fmaf(-a.t.kl, e, g);
    }
  }
  if (a.t.entropy != 0.f) sum = fmaf(-a.t.entropy, a.H[r], sum);
  const bool counts = on && w != 0.f;
  if (a.loss) a.loss[r] = counts ? w * sum : 0.f;
  if (a.ratio) a.ratio[r] = on ? ratio : 0.f;
  if (a.kl) a.kl[r] = on ? kl : 0.f;
  if (a.g) a.g[r] = counts ? w * g : 0.f;
  if (a.gh) a.gh[r] = counts ? -w * a.t.entropy : 0.f;
}

__global__ void __launch_bounds__(128) k_policy_rows(const PolicyParams a) {
  const int r = blockIdx.x * 128 + threadIdx.x;
  if (r < a.rows) policy_row(a, r);
}

size_t align16(size_t n) { return (n + 15) / 16 * 16; }

}  // namespace
}  // namespace jf

using namespace jf;

extern "C" jf_status jf_op_policy_loss_workspace_bytes(int dtype, int rows, int vocab, size_t* out_bytes) {
  if ((dtype != JF_F32 && dtype != JF_BF16) || rows < 0 || vocab < 1 || !out_bytes) return JF_EINVAL;
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
      (!ref_logprob && terms->kl != 0.f) || (dtype != JF_F32 && dtype != JF_BF16) || rows < 0 || vocab < 1 || !err_word)
    return JF_EINVAL;
  if (rows == 0) return JF_OK;
  if (!targets || !advantage) return JF_EINVAL;
  if (grad_logits && (ld_grad < vocab || ((uintptr_t)grad_logits & (dtype == JF_BF16 ? 1 : 3)) || (grad_logits == logits && ld_grad != ld))) return JF_EINVAL;
  size_t need = 0, scores = 0;
  jf_status s = jf_op_policy_loss_workspace_bytes(dtype, rows, vocab, &need);
  if (s != JF_OK) return s;
  if (!workspace || workspace_bytes < need) return JF_ENOMEM;
  if ((uintptr_t)workspace & 15) return JF_EINVAL;
  jf_op_token_logprobs_workspace_bytes(rows, vocab, 0, &scores);
  float* at = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + align16(scores));
  float *lp = logprob ? logprob : at, *H = entropy ? entropy : at + rows, *stats = at + 2 * (size_t)rows;
  s = jf_op_token_logprobs(dtype, logits, ld, rows, vocab, scale, targets, lp, H, nullptr, stats, 0, nullptr, nullptr, workspace,
                           scores, err_word, cuda_stream);
  if (s != JF_OK) return s;
  PolicyParams a = {*terms, rows, targets, old_logprob, ref_logprob, advantage, weight, lp, H, loss, ratio, kl, at + 4 * (size_t)rows, at + 5 * (size_t)rows};
  k_policy_rows<<<(rows + 127) / 128, 128, 0, reinterpret_cast<cudaStream_t>(cuda_stream)>>>(a);
  if (cudaGetLastError() != cudaSuccess) return JF_ECUDA;
  if (!grad_logits) return JF_OK;
  return jf_op_token_logprobs_grad(dtype, logits, ld, rows, vocab, scale, targets, stats, H, a.g, a.gh, grad_logits, ld_grad, err_word,
                                   cuda_stream);
}
