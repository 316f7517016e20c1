// What the kernels over rows of logits share: rows as 16-byte vectors, sums of exponentials, packed arithmetic.
#pragma once
#include "../../include/jf_ops.h"
#include "jf_device.cuh"
#include "jf_internal.h"

namespace jf {

constexpr float LOG2E = 1.4426950408889634f;

JF_DEV float ex2_ftz(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// dloss/dz of a token of probability p, ln p = lp, where dloss/dlogprob = g, dloss/dentropy = gh and the row's entropy is H. What cannot
// occur has no share, and what is certain is moved by nothing, also where a term is infinite.
JF_DEV float policy_grad(float p, float lp, float H, float g, float gh, bool is_target) {
  float d = is_target ? (p == 1.f ? 0.f : g * (1.f - p)) : (p == 0.f ? 0.f : -g * p);
  if (gh != 0.f && p != 0.f) d -= gh * p * (lp + H);
  return d;
}

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
  static JF_DEV uint4 raw(const float* p) { return __ldcs(reinterpret_cast<const uint4*>(p)); }
  static JF_DEV void unpack(uint4 v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
  }
  static JF_DEV uint4 nothing() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }  // -infinities
  static JF_DEV void store(float* p, const float (&x)[4]) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));
  }
};
template <>
struct Vec<bf16> {
  static constexpr int N = 8;
  static JF_DEV uint4 raw(const bf16* p) { return __ldcs(reinterpret_cast<const uint4*>(p)); }
  static JF_DEV uint4 nothing() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }  // -infinities
  static JF_DEV void unpack(uint4 v, float (&x)[8]) {
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

// A row as `n_vec` whole 16-byte vectors of the memory it lies in, the elements before them (fewer than a vector) and
// those behind.
template <typename T>
struct Row {
  const T* p;
  int head, n_vec, V;
  JF_DEV Row(const T* base, int V_) : p(base), V(V_) {
    const int skew = (int)(((uintptr_t)base & 15) / sizeof(T));
    head = min(V, skew ? Vec<T>::N - skew : 0);
    n_vec = (V - head) / Vec<T>::N;
  }
  JF_DEV const T* vec(int v) const { return p + head + (long long)v * Vec<T>::N; }
  // Index of edge element t (0 .. 2 N - 1: the head's, then the tail's), or -1.
  JF_DEV int edge(int t) const {
    constexpr int N = Vec<T>::N;
    const int tail = head + n_vec * N + t - N;
    return t < N ? (t < head ? t : -1) : (t < 2 * N && tail < V ? tail : -1);
  }
  JF_DEV bool has_edges() const { return n_vec * Vec<T>::N < V; }
};

// x - m, x * c and sums on two values at a time.
struct F2 {
  float x, y;
};
JF_DEV F2 add2(F2 a, F2 b) {
  F2 r;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
JF_DEV F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
JF_DEV F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\t"
      "mov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}

// jf_op_token_logprobs_grad (jf_logprobs.cu) for g and gh of any size; rows where both are 0 get 0 whatever their logits hold.
jf_status policy_long_grad(int dtype, const void* logits, long long ld, int rows, int vocab, float scale, const int32_t* targets, const float* row_stats,
                           const float* entropy, const float* g, const float* gh, void* grad_logits, long long ld_grad, int* err_word, cudaStream_t st);

}  // namespace jf
