// Causal attention of packed texts and its backward pass (jf_ops.h: jf_op_packed_attention*): entry points, and the
// kernels on CUDA cores, for fp32 and for bf16 rows that tensor copies cannot read.
//
// For a query row i of a text, s_ij = scale q_i . k_j over its rows j <= i, lse_i = log sum_j e^s_ij, p_ij = e^(s_ij - lse_i):
//   out_i = sum_j p_ij v_j
//   delta_i = d_out_i . out_i,  ds_ij = p_ij (d_out_i . v_j - delta_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij d_out_i
// where a KV head's sums run over the rows of all query heads that read it. Forward: one pass over the keys with the running
// maximum and sum. Backward: p is computed again from lse; one kernel holds a tile of keys and walks over the queries for
// dk and dv, another holds queries and walks over the keys for dq, so that every sum has one owner and one order.
#include "jf_once.h"
#include "jf_packed.cuh"

namespace jf {
namespace {

// Rows that a CTA owns (of queries, or of keys in dk and dv) and rows of the other kind that it takes at a time.
//
// What bounds a step is the shared memory that feeds the FMAs: a 16-byte load of a warp takes 2 to 4 wavefronts, so what counts is
// how many products a loaded value gets. 16 x 8 threads have 4 x 4 scores each, 8 loads to 64 FMAs; with 16 x 16 of 2 x 4, 6 to 32, and
// the next step's rows in registers instead of more CTAs on an SM, 777 rows among others (4 heads of 64) took 73 us instead of 60.
//
// What bounds a small batch is the longest text's last tile, a chain of all its keys. Clusters of up to PF_PARTS CTAs share a tile's
// steps where the grid has fewer than PF_CTAS CTAs, and add up through their shared memory. fp32, CTAs of a cluster 1, 2, 4, 8:
//   forward, 777 rows among others, 4 heads of 64: 60, 45, 33, 33 us; 8 texts of 200 rows, 12 heads of 128 (grid of 672): 72, 90, 89, 90
//   backward, 301 rows among others, 4 heads of 64: 128, 71, 48, 46 us; 1,000 rows, 12 heads of 128: 1,216, 718, 471, 538
constexpr int PF_OWN = 32, PF_T = 64, PF_THREADS = 128;
constexpr int PF_Y = PF_THREADS / 16, PF_R = PF_OWN / PF_Y;  // threads along a tile's rows, owned rows of one
constexpr int PF_PARTS = 4, PF_CTAS = 608;

// Values of `rows` rows from p on (row `ld` apart, HD long) as fp32 rows of HD + 4 in shared memory, where rows up to ALL are zeros.
template <typename T, int HD, int ALL>
JF_DEV void pf_load(float* dst, const T* p, long long ld, int rows, bool by16) {
  constexpr int N = 16 / sizeof(T), C = HD / N, IT = ALL * C / PF_THREADS, AT = IT < 8 ? IT : 8;  // 8 loads in flight
#pragma unroll 1
  for (int k0 = 0; k0 < IT; k0 += AT) {
    uint4 w[AT];
#pragma unroll
    for (int k = 0; k < AT; ++k) {
      const int i = threadIdx.x + (k0 + k) * PF_THREADS, r = i / C, c = i % C * N;
      w[k] = by16 && r < rows ? *reinterpret_cast<const uint4*>(p + r * ld + c) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < AT; ++k) {
      const int i = threadIdx.x + (k0 + k) * PF_THREADS, r = i / C, c = i % C * N;
      float x[N];
      const T* t = reinterpret_cast<const T*>(&w[k]);
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = act_to_f32(t[j]);
      if (!by16 && r < rows) {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = act_to_f32(p[r * ld + c + j]);
      }
#pragma unroll
      for (int j = 0; j < N; j += 4) *reinterpret_cast<float4*>(dst + r * (HD + 4) + c + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
    }
  }
}

// s[i][j] = a row (ty + PF_Y i) . b row (tx + 16 j)
template <int HD, int I, int J>
JF_DEV void pf_dots(const float* a, const float* b, int ty, int tx, float (&s)[I][J]) {
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int j = 0; j < J; ++j) s[i][j] = 0.f;
#pragma unroll 4
  for (int d = 0; d < HD; d += 4) {
    float4 x[I], y[J];
#pragma unroll
    for (int i = 0; i < I; ++i) x[i] = *reinterpret_cast<const float4*>(a + (ty + PF_Y * i) * (HD + 4) + d);
#pragma unroll
    for (int j = 0; j < J; ++j) y[j] = *reinterpret_cast<const float4*>(b + (tx + 16 * j) * (HD + 4) + d);
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j)
        s[i][j] = fmaf(x[i].x, y[j].x, fmaf(x[i].y, y[j].y, fmaf(x[i].z, y[j].z, fmaf(x[i].w, y[j].w, s[i][j]))));
  }
}

// o[i][.] += sum_c w[ty + PF_Y i][c] b[c][dims 4 tx + 64 j ..] over PF_T columns c, w in rows of PF_T + 4
template <int HD, int I>
JF_DEV void pf_rows_by(const float* w, const float* b, int ty, int tx, float (&o)[I][HD / 16]) {
#pragma unroll 2
  for (int c = 0; c < PF_T; c += 4) {
    float4 x[I];
#pragma unroll
    for (int i = 0; i < I; ++i) x[i] = *reinterpret_cast<const float4*>(w + (ty + PF_Y * i) * (PF_T + 4) + c);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < HD / 64; ++j) {
        const float4 y = *reinterpret_cast<const float4*>(b + (c + k) * (HD + 4) + 4 * tx + 64 * j);
#pragma unroll
        for (int i = 0; i < I; ++i) {
          const float f = k == 0 ? x[i].x : (k == 1 ? x[i].y : (k == 2 ? x[i].z : x[i].w));
          o[i][4 * j] = fmaf(f, y.x, o[i][4 * j]);
          o[i][4 * j + 1] = fmaf(f, y.y, o[i][4 * j + 1]);
          o[i][4 * j + 2] = fmaf(f, y.z, o[i][4 * j + 2]);
          o[i][4 * j + 3] = fmaf(f, y.w, o[i][4 * j + 3]);
        }
      }
  }
}

// o[i][.] += sum_r w[r][PF_R ty + i] b[r][dims 4 tx + 64 j ..] over PF_T rows r, w in rows of PF_OWN + 4
template <int HD>
JF_DEV void pf_columns_by(const float* w, const float* b, int ty, int tx, float (&o)[PF_R][HD / 16]) {
  static_assert(PF_R == 4);
#pragma unroll 4
  for (int r = 0; r < PF_T; ++r) {
    const float4 f4 = *reinterpret_cast<const float4*>(w + r * (PF_OWN + 4) + 4 * ty);
    const float f[4] = {f4.x, f4.y, f4.z, f4.w};
#pragma unroll
    for (int j = 0; j < HD / 64; ++j) {
      const float4 y = *reinterpret_cast<const float4*>(b + r * (HD + 4) + 4 * tx + 64 * j);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[i][4 * j] = fmaf(f[i], y.x, o[i][4 * j]);
        o[i][4 * j + 1] = fmaf(f[i], y.y, o[i][4 * j + 1]);
        o[i][4 * j + 2] = fmaf(f[i], y.z, o[i][4 * j + 2]);
        o[i][4 * j + 3] = fmaf(f[i], y.w, o[i][4 * j + 3]);
      }
    }
  }
}

template <typename T>
JF_DEV void pf_store4(T* p, float a, float b, float c, float d) {
  p[0] = to_act<T>(a), p[1] = to_act<T>(b), p[2] = to_act<T>(c), p[3] = to_act<T>(d);
}

struct PfTile {
  int row0, n, first;  // the text's first row and length; the tile's first row in it. n < 0: no tile
};
// Tile x: text by text, PF_OWN rows each. Rows that belong to no text are cleared by `clear(row)` on the way, each by one CTA of
// the grid.
template <typename Clear>
JF_DEV PfTile pf_tile(const PackedParams& a, int x, Clear clear) {
  __shared__ int s_at[kPackedMaxSeqs], s_bad, s_found;
  if (threadIdx.x == 0) s_bad = 0, s_found = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < a.t.n_seqs; b += PF_THREADS) {
    if (!packed_text_ok(a.t, b)) s_bad = 1;
    s_at[b] = (a.t.row_start[b + 1] - a.t.row_start[b] + PF_OWN - 1) / PF_OWN;
  }
  __syncthreads();
  if (s_bad) {
    if (threadIdx.x == 0) jf_set_error(a.err, JF_DERR_BOUNDS);
    return {0, -1, 0};
  }
  if (threadIdx.x < 32) {
    int base = 0;
    for (int b0 = 0; b0 < a.t.n_seqs; b0 += 32) {
      const int b = b0 + (int)threadIdx.x, n = b < a.t.n_seqs ? s_at[b] : 0;
      int sum = n;
#pragma unroll
      for (int sh = 1; sh < 32; sh <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, sum, sh);
        if ((int)threadIdx.x >= sh) sum += u;
      }
      const int before = base + sum - n;
      if (x >= before && x < before + n) {
        s_found = b;
        s_at[b] = x - before;
      }
      base += __shfl_sync(0xffffffffu, sum, 31);
    }
  }
  const int head = a.t.row_start[0], tail = a.t.row_start[a.t.n_seqs];
  for (int r = blockIdx.x; r < head; r += gridDim.x) clear(r);
  for (int r = tail + blockIdx.x; r < a.t.n_rows; r += gridDim.x) clear(r);
  __syncthreads();
  const int b = s_found;
  if (b < 0) return {0, -1, 0};
  const int s0 = a.t.row_start[b];
  return {s0, a.t.row_start[b + 1] - s0, s_at[b] * PF_OWN};
}

template <typename T>
JF_DEV bool pf_by16(const void* p, long long ld) {
  return ((uintptr_t)p & 15) == 0 && ld % (16 / (int)sizeof(T)) == 0;
}

// The CTAs of a cluster share a tile: each takes every parts'th step, and joins some of the owned rows of all from their shared
// memory, in their order.
JF_DEV void pf_join_begin(int parts) {
  if (parts > 1) cluster_sync();
  else __syncthreads();
}
JF_DEV void pf_join_end(int parts) {
  if (parts > 1) cluster_sync();  // peers may still read this CTA's rows
}
// What a thread has of its owned rows, r0 + apart i, to rows of HD in shared memory.
template <int HD>
JF_DEV void pf_put(float* s, int r0, int apart, int tx, const float (&o)[PF_R][HD / 16]) {
#pragma unroll
  for (int i = 0; i < PF_R; ++i)
#pragma unroll
    for (int j = 0; j < HD / 64; ++j)
      *reinterpret_cast<float4*>(s + (r0 + apart * i) * HD + 4 * tx + 64 * j) = make_float4(o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]);
}
// The sum over the cluster of four values at byte `at` of those rows.
JF_DEV float4 pf_sum4(const float* s, int at, int parts) {
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = 0; k < parts; ++k) {
    const float4 v = ld_cluster4(map_to_rank(smem_u32(s), k) + at);
    o.x += v.x, o.y += v.y, o.z += v.z, o.w += v.w;
  }
  return o;
}

// Grid (tiles x parts, query heads).
template <typename T, int HD>
__global__ void __launch_bounds__(PF_THREADS, HD == 64 ? 4 : 2) k_packed_attn(const PackedParams a) {
  extern __shared__ float sm[];
  constexpr int TILE = PF_T * (HD + 4), OWN = PF_OWN * (HD + 4);
  float *sq = sm, *sk = sm + OWN, *sv = sk + TILE, *sp = sv + TILE;
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16, h = blockIdx.y, kvh = h / (a.Hq / a.Hkv);
  pdl_launch_dependents();
  pdl_wait();
  T* out = reinterpret_cast<T*>(a.out);
  const int parts = (int)cluster_ctas(), part = (int)cluster_rank();
  const PfTile t = pf_tile(a, blockIdx.x / parts, [&](int r) {
    for (int d = tid; d < HD; d += PF_THREADS) out[((long long)r * a.Hq + h) * HD + d] = to_act<T>(0.f);
    if (tid == 0 && a.lse) a.lse[(long long)r * a.Hq + h] = -INFINITY;
  });
  if (t.n < 0) return;
  const int rows = min(PF_OWN, t.n - t.first);
  const bool q16 = pf_by16<T>(a.q, a.ld_q), k16 = pf_by16<T>(a.k, a.ld_k), v16 = pf_by16<T>(a.v, a.ld_v);
  pf_load<T, HD, PF_OWN>(sq, reinterpret_cast<const T*>(a.q) + (t.row0 + t.first) * a.ld_q + h * HD, a.ld_q, rows, q16);
  float m[PF_R], l[PF_R], o[PF_R][HD / 16] = {};
#pragma unroll
  for (int i = 0; i < PF_R; ++i) m[i] = -INFINITY, l[i] = 0.f;
  const float c = a.scale * kLog2e;
  for (int k0 = part * PF_T; k0 < t.first + rows; k0 += parts * PF_T) {
    __syncthreads();
    pf_load<T, HD, PF_T>(sk, reinterpret_cast<const T*>(a.k) + (t.row0 + k0) * a.ld_k + kvh * HD, a.ld_k, min(PF_T, t.n - k0), k16);
    pf_load<T, HD, PF_T>(sv, reinterpret_cast<const T*>(a.v) + (t.row0 + k0) * a.ld_v + kvh * HD, a.ld_v, min(PF_T, t.n - k0), v16);
    __syncthreads();
    float s[PF_R][4];
    pf_dots<HD>(sq, sk, ty, tx, s);
#pragma unroll
    for (int i = 0; i < PF_R; ++i) {
      const int qi = t.first + ty + PF_Y * i;
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = k0 + tx + 16 * j <= qi ? s[i][j] * c : -INFINITY;
        mx = fmaxf(mx, s[i][j]);
      }
#pragma unroll
      for (int sh = 8; sh; sh >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, sh));
      mx = fmaxf(mx, m[i]);
      const float base = mx == -INFINITY ? 0.f : mx, al = exp2f(m[i] - base);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = exp2f(s[i][j] - base);
        sum += s[i][j];
        sp[(ty + PF_Y * i) * (PF_T + 4) + tx + 16 * j] = s[i][j];
      }
#pragma unroll
      for (int sh = 8; sh; sh >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, sh);
      l[i] = l[i] * al + sum;
      m[i] = mx;
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[i][d] *= al;
    }
    __syncthreads();
    pf_rows_by<HD>(sp, sv, ty, tx, o);
  }
  __syncthreads();
  float *so = sk, *s_m = so + PF_OWN * HD, *s_l = s_m + PF_OWN;  // sums, maxima, sums of exponentials
  pf_put<HD>(so, ty, PF_Y, tx, o);
  if (tx == 0) {
#pragma unroll
    for (int i = 0; i < PF_R; ++i) s_m[ty + PF_Y * i] = m[i], s_l[ty + PF_Y * i] = l[i];
  }
  pf_join_begin(parts);
  const int mine = PF_OWN / parts;
  for (int i = tid; i < mine * (HD / 4); i += PF_THREADS) {
    const int r = part * mine + i / (HD / 4), d = i % (HD / 4) * 4;
    if (r >= rows) continue;
    float M = -INFINITY, L = 0.f;
    float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < parts; ++k) {
      const uint32_t from = map_to_rank(smem_u32(so), k);
      const float mk = ld_cluster(from + (PF_OWN * HD + r) * 4), lk = ld_cluster(from + (PF_OWN * HD + PF_OWN + r) * 4);
      const float4 v = ld_cluster4(from + (r * HD + d) * 4);
      if (lk == 0.f) continue;  // (it saw nothing)
      const float top = fmaxf(M, mk), f0 = M == top ? 1.f : exp2f(M - top), f1 = mk == top ? 1.f : exp2f(mk - top);
      M = top;
      L = f0 * L + f1 * lk;
      w.x = f0 * w.x + f1 * v.x, w.y = f0 * w.y + f1 * v.y, w.z = f0 * w.z + f1 * v.z, w.w = f0 * w.w + f1 * v.w;
    }
    const long long at = (long long)(t.row0 + t.first + r) * a.Hq + h;
    const float il = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
    pf_store4<T>(out + at * HD + d, w.x * il, w.y * il, w.z * il, w.w * il);
    if (d == 0 && a.lse) a.lse[at] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
  }
  pf_join_end(parts);
}

// delta[row][head] = d_out . out of fp32 rows, a warp per (row, head); rows of no text as well (their d_out may be anything: not used).
template <typename T, int HD>
__global__ void __launch_bounds__(256) k_packed_delta(const PackedParams a) {
  pdl_launch_dependents();
  pdl_wait();
  const long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (i >= (long long)a.t.n_rows * a.Hq) return;
  const long long r = i / a.Hq;
  const T* x = reinterpret_cast<const T*>(a.out) + i * HD;
  const T* y = reinterpret_cast<const T*>(a.d_out) + r * a.ld_do + (i - r * a.Hq) * HD;
  float s = 0.f;
#pragma unroll
  for (int d = lane; d < HD; d += 32) s = fmaf(act_to_f32(x[d]), act_to_f32(y[d]), s);
  s = warp_sum(s);
  if (lane == 0) a.delta[i] = s;
}

// p and ds of a tile of I x J queries and keys a thread (queries from q0 on, keys from k0 on) into sp and sds, rows 16 J + 4 apart.
template <int HD, int I, int J>
JF_DEV void pf_back_tile(const float* sq, const float* sdo, const float* sk, const float* sv, const float* s_lse, const float* s_delta,
                         int q0, int k0, int n, float c, int ty, int tx, float* sp, float* sds) {
  constexpr int LD = 16 * J + 4;
  float s[I][J], dp[I][J];
  pf_dots<HD>(sq, sk, ty, tx, s);
  pf_dots<HD>(sdo, sv, ty, tx, dp);
#pragma unroll
  for (int i = 0; i < I; ++i) {
    const int r = ty + PF_Y * i;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int kj = k0 + tx + 16 * j;
      const bool sees = kj <= q0 + r && q0 + r < n;
      const float p = sees ? exp2f(fmaf(s[i][j], c, -s_lse[r])) : 0.f;
      if (sp) sp[r * LD + tx + 16 * j] = p;
      sds[r * LD + tx + 16 * j] = sees ? p * (dp[i][j] - s_delta[r]) : 0.f;
    }
  }
}

// Grid (tiles of keys x parts, KV heads): dk and dv.
template <typename T, int HD>
__global__ void __launch_bounds__(PF_THREADS, HD == 64 ? 2 : 1) k_packed_dkv(const PackedParams a) {
  extern __shared__ float sm[];
  constexpr int TILE = PF_T * (HD + 4), OWN = PF_OWN * (HD + 4);
  float *sq = sm, *sdo = sm + TILE, *sk = sm + 2 * TILE, *sv = sk + OWN, *sp = sv + OWN, *sds = sp + PF_T * (PF_OWN + 4);
  __shared__ float s_lse[PF_T], s_delta[PF_T];
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16, kvh = blockIdx.y, G = a.Hq / a.Hkv;
  pdl_launch_dependents();
  pdl_wait();
  T *dk = reinterpret_cast<T*>(a.dk), *dv = reinterpret_cast<T*>(a.dv);
  const int parts = (int)cluster_ctas(), part = (int)cluster_rank();
  const PfTile t = pf_tile(a, blockIdx.x / parts, [&](int r) {
    for (int d = tid; d < HD; d += PF_THREADS) dk[r * a.ld_dk + kvh * HD + d] = dv[r * a.ld_dv + kvh * HD + d] = to_act<T>(0.f);
  });
  if (t.n < 0) return;
  const int rows = min(PF_OWN, t.n - t.first);
  pf_load<T, HD, PF_OWN>(sk, reinterpret_cast<const T*>(a.k) + (t.row0 + t.first) * a.ld_k + kvh * HD, a.ld_k, rows, pf_by16<T>(a.k, a.ld_k));
  pf_load<T, HD, PF_OWN>(sv, reinterpret_cast<const T*>(a.v) + (t.row0 + t.first) * a.ld_v + kvh * HD, a.ld_v, rows, pf_by16<T>(a.v, a.ld_v));
  const bool q16 = pf_by16<T>(a.q, a.ld_q), do16 = pf_by16<T>(a.d_out, a.ld_do);
  float gk[PF_R][HD / 16] = {}, gv[PF_R][HD / 16] = {};
  const int tiles = (t.n - t.first + PF_T - 1) / PF_T, steps = G * tiles;  // (head by head)
  for (int step = part; step < steps; step += parts) {
    const int h = kvh * G + step / tiles, q0 = t.first + step % tiles * PF_T, nq = min(PF_T, t.n - q0);
    __syncthreads();
    pf_load<T, HD, PF_T>(sq, reinterpret_cast<const T*>(a.q) + (t.row0 + q0) * a.ld_q + h * HD, a.ld_q, nq, q16);
    pf_load<T, HD, PF_T>(sdo, reinterpret_cast<const T*>(a.d_out) + (t.row0 + q0) * a.ld_do + h * HD, a.ld_do, nq, do16);
    if (tid < nq) {
      s_lse[tid] = a.lse[(long long)(t.row0 + q0 + tid) * a.Hq + h] * kLog2e;
      s_delta[tid] = a.delta[(long long)(t.row0 + q0 + tid) * a.Hq + h];
    }
    __syncthreads();
    pf_back_tile<HD, PF_T / PF_Y, PF_OWN / 16>(sq, sdo, sk, sv, s_lse, s_delta, q0, t.first, t.n, a.scale * kLog2e, ty, tx, sp, sds);
    __syncthreads();
    pf_columns_by<HD>(sp, sdo, ty, tx, gv);
    pf_columns_by<HD>(sds, sq, ty, tx, gk);
  }
  __syncthreads();
  pf_put<HD>(sq, PF_R * ty, 1, tx, gk);
  pf_put<HD>(sdo, PF_R * ty, 1, tx, gv);
  pf_join_begin(parts);
  const int mine = PF_OWN / parts;
  for (int i = tid; i < mine * (HD / 4); i += PF_THREADS) {
    const int r = part * mine + i / (HD / 4), d = i % (HD / 4) * 4;
    if (r >= rows) continue;
    const long long at = t.row0 + t.first + r;
    const float4 x = pf_sum4(sq, (r * HD + d) * 4, parts), y = pf_sum4(sdo, (r * HD + d) * 4, parts);
    pf_store4<T>(dk + at * a.ld_dk + kvh * HD + d, a.scale * x.x, a.scale * x.y, a.scale * x.z, a.scale * x.w);
    pf_store4<T>(dv + at * a.ld_dv + kvh * HD + d, y.x, y.y, y.z, y.w);
  }
  pf_join_end(parts);
}

// Grid (tiles of queries x parts, query heads): dq. DELTA: delta instead, as sum_j p_ij (d_out_i . v_j), for bf16 outputs: that of a rounded out
// is off by 2^-9 of its terms, which counts where a row sees few keys (texts of two rows: dq off by 3.2e-3 of its norm instead of its
// own rounding's 1.66e-3, dk alike; 300 rows: 1.86e-3). Two more products to the seven of the pass.
template <typename T, int HD, bool DELTA>
__global__ void __launch_bounds__(PF_THREADS, HD == 64 ? 2 : 1) k_packed_dq(const PackedParams a) {
  extern __shared__ float sm[];
  constexpr int TILE = PF_T * (HD + 4), OWN = PF_OWN * (HD + 4);
  float *sq = sm, *sdo = sm + OWN, *sk = sm + 2 * OWN, *sv = sk + TILE, *sds = sv + TILE;
  __shared__ float s_lse[PF_OWN], s_delta[PF_OWN];
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16, h = blockIdx.y, kvh = h / (a.Hq / a.Hkv);
  pdl_launch_dependents();
  pdl_wait();
  T* dq = reinterpret_cast<T*>(a.dq);
  const int parts = (int)cluster_ctas(), part = (int)cluster_rank();
  const PfTile t = pf_tile(a, blockIdx.x / parts, [&](int r) {
    if constexpr (!DELTA)
      for (int d = tid; d < HD; d += PF_THREADS) dq[r * a.ld_dq + h * HD + d] = to_act<T>(0.f);
  });
  if (t.n < 0) return;
  const int rows = min(PF_OWN, t.n - t.first);
  pf_load<T, HD, PF_OWN>(sq, reinterpret_cast<const T*>(a.q) + (t.row0 + t.first) * a.ld_q + h * HD, a.ld_q, rows, pf_by16<T>(a.q, a.ld_q));
  pf_load<T, HD, PF_OWN>(sdo, reinterpret_cast<const T*>(a.d_out) + (t.row0 + t.first) * a.ld_do + h * HD, a.ld_do, rows, pf_by16<T>(a.d_out, a.ld_do));
  if (tid < rows) {
    s_lse[tid] = a.lse[(long long)(t.row0 + t.first + tid) * a.Hq + h] * kLog2e;
    s_delta[tid] = DELTA ? 0.f : a.delta[(long long)(t.row0 + t.first + tid) * a.Hq + h];
  }
  const bool k16 = pf_by16<T>(a.k, a.ld_k), v16 = pf_by16<T>(a.v, a.ld_v);
  float g[PF_R][HD / 16] = {}, sum = 0.f;  // (sum: of 16 columns of row tid / 4)
  for (int k0 = part * PF_T; k0 < t.first + rows; k0 += parts * PF_T) {
    __syncthreads();
    pf_load<T, HD, PF_T>(sk, reinterpret_cast<const T*>(a.k) + (t.row0 + k0) * a.ld_k + kvh * HD, a.ld_k, min(PF_T, t.n - k0), k16);
    pf_load<T, HD, PF_T>(sv, reinterpret_cast<const T*>(a.v) + (t.row0 + k0) * a.ld_v + kvh * HD, a.ld_v, min(PF_T, t.n - k0), v16);
    __syncthreads();
    pf_back_tile<HD, PF_R, PF_T / 16>(sq, sdo, sk, sv, s_lse, s_delta, t.first, k0, t.n, a.scale * kLog2e, ty, tx, nullptr, sds);
    __syncthreads();
    if constexpr (DELTA) {
      static_assert(PF_THREADS == 4 * PF_OWN && PF_T == 64);
#pragma unroll
      for (int x = 0; x < 16; ++x) sum += sds[(tid >> 2) * (PF_T + 4) + 16 * (tid & 3) + x];
    } else {
      pf_rows_by<HD>(sds, sk, ty, tx, g);
    }
  }
  __syncthreads();
  if constexpr (DELTA) {
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    if ((tid & 3) == 0) sk[tid >> 2] = sum;
    pf_join_begin(parts);
    if (part == 0 && tid < rows) {
      sum = 0.f;
      for (int k = 0; k < parts; ++k) sum += ld_cluster(map_to_rank(smem_u32(sk), k) + 4 * tid);
      a.delta[(long long)(t.row0 + t.first + tid) * a.Hq + h] = sum;
    }
    pf_join_end(parts);
    return;
  }
  pf_put<HD>(sk, ty, PF_Y, tx, g);
  pf_join_begin(parts);
  const int mine = PF_OWN / parts;
  for (int i = tid; i < mine * (HD / 4); i += PF_THREADS) {
    const int r = part * mine + i / (HD / 4), d = i % (HD / 4) * 4;
    if (r >= rows) continue;
    const float4 x = pf_sum4(sk, (r * HD + d) * 4, parts);
    pf_store4<T>(dq + (t.row0 + t.first + r) * a.ld_dq + h * HD + d, a.scale * x.x, a.scale * x.y, a.scale * x.z, a.scale * x.w);
  }
  pf_join_end(parts);
}

// Shared memory of owned tiles, other tiles, and floats beside them.
template <int HD>
constexpr int pf_smem(int own, int tiles, int more) {
  return ((own * PF_OWN + tiles * PF_T) * (HD + 4) + more) * 4;
}
template <int HD>
constexpr int pf_smem_attn = pf_smem<HD>(1, 2, PF_OWN * (PF_T + 4));
template <int HD>
constexpr int pf_smem_dkv = pf_smem<HD>(2, 2, 2 * PF_T * (PF_OWN + 4));
template <int HD>
constexpr int pf_smem_dq = pf_smem<HD>(2, 2, PF_OWN * (PF_T + 4));
template <typename T, int HD>
cudaError_t pf_prepare() {
  cudaError_t e = cudaFuncSetAttribute(k_packed_attn<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, pf_smem_attn<HD>);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k_packed_dkv<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, pf_smem_dkv<HD>);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k_packed_dq<T, HD, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, pf_smem_dq<HD>);
  if constexpr (sizeof(T) == 2) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_packed_dq<T, HD, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, pf_smem_dq<HD>);
  }
  return e;
}
PerDeviceOnce g_pf_once;
bool pf_ready() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  return g_pf_once.run(dev, []() -> int {
    cudaError_t e = pf_prepare<float, 64>();
    if (e == cudaSuccess) e = pf_prepare<float, 128>();
    if (e == cudaSuccess) e = pf_prepare<bf16, 64>();
    if (e == cudaSuccess) e = pf_prepare<bf16, 128>();
    return (int)e;
  }) == 0;
}

unsigned pf_tiles(const jf_packed& t) { return (unsigned)((t.n_rows + PF_OWN - 1) / PF_OWN + t.n_seqs); }

// CTAs of a cluster, for a grid of `rows` rows of tiles whose longest chain is `steps`.
int pf_parts(const jf_packed& t, int rows, long long steps) {
  int parts = 1;
  while (parts < PF_PARTS && steps > parts && (long long)pf_tiles(t) * rows * parts < PF_CTAS) parts *= 2;
  return parts;
}
long long pf_steps(const jf_packed& t) { return (t.max_rows + PF_T - 1) / PF_T; }

template <typename T, int HD>
cudaError_t pf_forward(const PackedParams& a, cudaStream_t st) {
  const int parts = pf_parts(a.t, a.Hq, pf_steps(a.t));
  return packed_launch_clusters(k_packed_attn<T, HD>, parts, dim3(pf_tiles(a.t) * parts, a.Hq), dim3(PF_THREADS), pf_smem_attn<HD>, st, a);
}
template <typename T, int HD>
cudaError_t pf_backward(const PackedParams& a, cudaStream_t st) {
  const long long warps = (long long)a.t.n_rows * a.Hq;
  const int kv = pf_parts(a.t, a.Hkv, pf_steps(a.t) * (a.Hq / a.Hkv)), q = pf_parts(a.t, a.Hq, pf_steps(a.t));
  cudaError_t e;
  if constexpr (sizeof(T) == 2) e = packed_launch_clusters(k_packed_dq<T, HD, true>, q, dim3(pf_tiles(a.t) * q, a.Hq), dim3(PF_THREADS), pf_smem_dq<HD>, st, a);
  else e = packed_launch(k_packed_delta<T, HD>, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, st, a);
  if (e == cudaSuccess) e = packed_launch_clusters(k_packed_dkv<T, HD>, kv, dim3(pf_tiles(a.t) * kv, a.Hkv), dim3(PF_THREADS), pf_smem_dkv<HD>, st, a);
  if (e == cudaSuccess) e = packed_launch_clusters(k_packed_dq<T, HD, false>, q, dim3(pf_tiles(a.t) * q, a.Hq), dim3(PF_THREADS), pf_smem_dq<HD>, st, a);
  return e;
}

// Arguments that every call has.
jf_status packed_check(const jf_packed* t, int dtype, int Hq, int Hkv, int hd) {
  if (!t || !t->row_start || t->n_seqs < 1 || t->n_rows < 0 || t->max_rows < 0 || t->max_rows > t->n_rows) return JF_EINVAL;
  if ((dtype != JF_F32 && dtype != JF_BF16) || Hq < 1 || Hkv < 1 || Hq % Hkv) return JF_EINVAL;
  if ((hd != 64 && hd != 128) || t->n_seqs > kPackedMaxSeqs || Hq / Hkv > kPackedMaxGroup || Hq > 65535) return JF_EUNSUPPORTED;
  // rows of a KV head and the steps of a batch's tiles are counted in 32 bits
  const long long group_rows = (long long)t->n_rows * (Hq / Hkv) + 128ll * t->n_seqs;
  if ((long long)t->n_rows * Hq > (1 << 30) || group_rows / 64 * ((long long)t->max_rows / 64 + 2) * Hkv > (1 << 30)) return JF_EUNSUPPORTED;
  return JF_OK;
}
bool packed_rows_ok(const void* p, long long ld, long long width, int dtype) {
  return p && ((uintptr_t)p & (dtype == JF_BF16 ? 1 : 3)) == 0 && ld >= width;
}
// Whether an output shares memory with an input or another output: the kernels read and write in no fixed order.
bool packed_overlap(const RowSpan* in, int n_in, const RowSpan* out, int n_out, int rows) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (rows_overlap(in[j], out[i], rows)) return true;
    for (int j = 0; j < i; ++j)
      if (rows_overlap(out[j], out[i], rows)) return true;
  }
  return false;
}

}  // namespace
}  // namespace jf

using namespace jf;

extern "C" jf_status jf_op_packed_attention_workspace_bytes(const jf_packed* texts, int dtype, int n_heads, int n_kv_heads,
                                                            int head_dim, int backward, size_t* out_bytes) {
  const jf_status s = packed_check(texts, dtype, n_heads, n_kv_heads, head_dim);
  if (s != JF_OK) return s;
  if (!out_bytes) return JF_EINVAL;
  if (dtype == JF_BF16) return packed_tc_workspace(*texts, n_heads, n_kv_heads, head_dim, backward != 0, out_bytes);
  *out_bytes = backward ? (size_t)texts->n_rows * n_heads * 4 : 0;
  return JF_OK;
}

extern "C" jf_status jf_op_packed_attention(const jf_packed* texts, int dtype, const void* q, long long ld_q, const void* k,
                                            long long ld_k, const void* v, long long ld_v, int n_heads, int n_kv_heads,
                                            int head_dim, float scale, void* out, float* lse, void* workspace,
                                            size_t workspace_bytes, int* err_word, void* cuda_stream) {
  jf_status s = packed_check(texts, dtype, n_heads, n_kv_heads, head_dim);
  if (s != JF_OK) return s;
  if (!err_word || !(scale >= -1e30f && scale <= 1e30f)) return JF_EINVAL;
  if (texts->n_rows == 0) return JF_OK;
  const long long wq = (long long)n_heads * head_dim, wkv = (long long)n_kv_heads * head_dim;
  if (!packed_rows_ok(q, ld_q, wq, dtype) || !packed_rows_ok(k, ld_k, wkv, dtype) || !packed_rows_ok(v, ld_v, wkv, dtype) || !out ||
      ((uintptr_t)out & 15) || ((uintptr_t)lse & 3) || ((uintptr_t)workspace & 15))
    return JF_EINVAL;
  const int size = dtype == JF_BF16 ? 2 : 4;
  const RowSpan in[] = {{q, ld_q * size, wq * size}, {k, ld_k * size, wkv * size}, {v, ld_v * size, wkv * size}};
  const RowSpan to[] = {{out, wq * size, wq * size}, {lse, n_heads * 4, n_heads * 4}};
  if (packed_overlap(in, 3, to, 2, texts->n_rows)) return JF_EINVAL;
  size_t need = 0;
  s = jf_op_packed_attention_workspace_bytes(texts, dtype, n_heads, n_kv_heads, head_dim, 0, &need);
  if (s != JF_OK) return s;
  if (need > 0 && (!workspace || workspace_bytes < need)) return JF_ENOMEM;
  if (!pf_ready()) return JF_ECUDA;
  PackedParams a = {};
  a.t = *texts, a.q = q, a.k = k, a.v = v, a.ld_q = ld_q, a.ld_k = ld_k, a.ld_v = ld_v, a.Hq = n_heads, a.Hkv = n_kv_heads;
  a.scale = scale, a.out = out, a.lse = lse, a.err = err_word;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (dtype == JF_BF16 && packed_tc_rows(q, ld_q) && packed_tc_rows(k, ld_k) && packed_tc_rows(v, ld_v)) return packed_tc_forward(a, head_dim, workspace, st);
  if (dtype == JF_BF16) e = head_dim == 128 ? pf_forward<bf16, 128>(a, st) : pf_forward<bf16, 64>(a, st);
  else e = head_dim == 128 ? pf_forward<float, 128>(a, st) : pf_forward<float, 64>(a, st);
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}

extern "C" jf_status jf_op_packed_attention_grad(const jf_packed* texts, int dtype, const void* q, long long ld_q, const void* k,
                                                 long long ld_k, const void* v, long long ld_v, int n_heads, int n_kv_heads,
                                                 int head_dim, float scale, const void* out, const float* lse,
                                                 const void* d_out, long long ld_do, void* dq, long long ld_dq, void* dk,
                                                 long long ld_dk, void* dv, long long ld_dv, void* workspace,
                                                 size_t workspace_bytes, int* err_word, void* cuda_stream) {
  jf_status s = packed_check(texts, dtype, n_heads, n_kv_heads, head_dim);
  if (s != JF_OK) return s;
  if (!err_word || !(scale >= -1e30f && scale <= 1e30f)) return JF_EINVAL;
  if (texts->n_rows == 0) return JF_OK;
  const long long wq = (long long)n_heads * head_dim, wkv = (long long)n_kv_heads * head_dim;
  if (!packed_rows_ok(q, ld_q, wq, dtype) || !packed_rows_ok(k, ld_k, wkv, dtype) || !packed_rows_ok(v, ld_v, wkv, dtype) ||
      !packed_rows_ok(d_out, ld_do, wq, dtype) || !packed_rows_ok(dq, ld_dq, wq, dtype) || !packed_rows_ok(dk, ld_dk, wkv, dtype) ||
      !packed_rows_ok(dv, ld_dv, wkv, dtype) || !out || ((uintptr_t)out & 15) || !lse || ((uintptr_t)lse & 3) || ((uintptr_t)workspace & 15))
    return JF_EINVAL;
  const int size = dtype == JF_BF16 ? 2 : 4;
  const RowSpan in[] = {{q, ld_q * size, wq * size},    {k, ld_k * size, wkv * size},      {v, ld_v * size, wkv * size},
                        {out, wq * size, wq * size},    {lse, n_heads * 4, n_heads * 4},   {d_out, ld_do * size, wq * size}};
  const RowSpan to[] = {{dq, ld_dq * size, wq * size}, {dk, ld_dk * size, wkv * size}, {dv, ld_dv * size, wkv * size}};
  if (packed_overlap(in, 6, to, 3, texts->n_rows)) return JF_EINVAL;
  size_t need = 0;
  s = jf_op_packed_attention_workspace_bytes(texts, dtype, n_heads, n_kv_heads, head_dim, 1, &need);
  if (s != JF_OK) return s;
  if (!workspace || workspace_bytes < need) return JF_ENOMEM;
  if (!pf_ready()) return JF_ECUDA;
  PackedParams a = {};
  a.t = *texts, a.q = q, a.k = k, a.v = v, a.ld_q = ld_q, a.ld_k = ld_k, a.ld_v = ld_v, a.Hq = n_heads, a.Hkv = n_kv_heads;
  a.scale = scale, a.out = const_cast<void*>(out), a.lse = const_cast<float*>(lse), a.d_out = d_out, a.ld_do = ld_do;
  a.dq = dq, a.dk = dk, a.dv = dv, a.ld_dq = ld_dq, a.ld_dk = ld_dk, a.ld_dv = ld_dv;
  a.delta = reinterpret_cast<float*>(workspace), a.err = err_word;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (dtype == JF_BF16 && packed_tc_rows(q, ld_q) && packed_tc_rows(k, ld_k) && packed_tc_rows(v, ld_v) && packed_tc_rows(d_out, ld_do))
    return packed_tc_backward(a, head_dim, workspace, st);
  if (dtype == JF_BF16) e = head_dim == 128 ? pf_backward<bf16, 128>(a, st) : pf_backward<bf16, 64>(a, st);
  else e = head_dim == 128 ? pf_backward<float, 128>(a, st) : pf_backward<float, 64>(a, st);
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}
