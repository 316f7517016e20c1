// Causal attention of packed bf16 texts and its backward pass on tcgen05 (jf_ops.h: jf_op_packed_attention*; the formulas
// stand in jf_packed.cu).
//
// Rows of a KV head. The G query heads that read a KV head meet the same keys, so a tile of query rows is TOK = 128 / G whole
// tokens times G heads (row = token * G + head), loaded as one box of a tensor copy: a short text fills the tensor core's 128
// rows G times sooner, and K and V are read once for G heads.
//
// Work is a line of units, (text, KV head, tile), each as long as its steps (tiles of keys, or of query rows in dk and dv)
// plus a constant for what a unit costs beside them; each CTA takes an equal run of that line. A unit that a run's end cuts leaves a
// partial result a part in the workspace, at most two a CTA, and a kernel behind joins the parts in their order. A cut
// close to a unit's end is moved there.
#include "jf_once.h"
#include "jf_packed.cuh"

namespace jf {
namespace {

constexpr int PT_KEYS = 128;                     // keys of a step (of a tile, in dk and dv)
constexpr int PT_MIN_SHARE = 4;                  // shortest run of a CTA
constexpr int PT_SNAP = 1;                       // a cut moves to a unit's end over this many steps

// ---------------------------------------------------------------------------------------------
// The line of units. Kind says how a text is cut: units(n), steps(n, u) for a text of n rows.
// ---------------------------------------------------------------------------------------------
struct ByQueries {  // tiles of `tok` tokens over the key tiles that they see
  static constexpr int UC = 2;
  int tok;
  JF_DEV int units(int n) const { return (n + tok - 1) / tok; }
  JF_DEV int steps(int n, int u) const { return (min(n, (u + 1) * tok) + PT_KEYS - 1) / PT_KEYS; }
};

struct Cut {        // a place between steps: before step `step` of a unit
  int b, kvh, u, step, n_steps, row0, n;
};

template <typename Kind>
struct Line {
  Kind kind;
  const jf_packed t;
  int Hkv, total;
  const int* pre;   // (shared memory) length of the texts before b, [n_seqs + 1]

  // By the whole CTA. False where the texts do not fit (reported).
  JF_DEV bool build(int* pre_, int* s_bad, int* err) {
    pre = pre_;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if (threadIdx.x == 0) *s_bad = 0, pre_[0] = 0;
    __syncthreads();
    for (int b = warp; b < t.n_seqs; b += warps) {
      const bool ok = packed_text_ok(t, b);
      if (!ok && lane == 0) *s_bad = 1;
      const int n = ok ? t.row_start[b + 1] - t.row_start[b] : 0, units = kind.units(n);
      int sum = 0;
      for (int u = lane; u < units; u += 32) sum += Kind::UC + kind.steps(n, u);
      sum = __reduce_add_sync(0xffffffffu, sum);
      if (lane == 0) pre_[b + 1] = sum * Hkv;
    }
    __syncthreads();
    if (*s_bad) {
      if (threadIdx.x == 0) jf_set_error(err, JF_DERR_BOUNDS);
      return false;
    }
    if (warp == 0) {
      int base = 0;
      for (int b0 = 0; b0 < t.n_seqs; b0 += 32) {
        int v = b0 + lane < t.n_seqs ? pre_[b0 + lane + 1] : 0;
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, v, sh);
          if (lane >= sh) v += u;
        }
        if (b0 + lane < t.n_seqs) pre_[b0 + lane + 1] = base + v;
        base += __shfl_sync(0xffffffffu, v, 31);
      }
    }
    __syncthreads();
    total = pre_[t.n_seqs];
    return true;
  }
  // How many of `most` CTAs have a run.
  JF_DEV int workers(int most) const { return max(1, min(most, total / PT_MIN_SHARE)); }
  // The cut before run i of n, by a whole warp; before the first and behind the last: b = -1 where there is no unit.
  JF_DEV Cut cut(int i, int n) const {
    const int x = (int)((long long)total * i / n), lane = threadIdx.x & 31;
    if (x >= total) return {t.n_seqs, 0, 0, 0, 0, 0, 0};
    int lo = 0, hi = t.n_seqs;  // the last b with pre[b] <= x
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (pre[mid] <= x) lo = mid;
      else hi = mid;
    }
    Cut c;
    c.b = lo;
    c.row0 = t.row_start[lo];
    c.n = t.row_start[lo + 1] - c.row0;
    const int per_head = (pre[lo + 1] - pre[lo]) / Hkv;
    c.kvh = (x - pre[lo]) / per_head;
    int rest = x - pre[lo] - c.kvh * per_head;
    const int units = kind.units(c.n);
    for (int u0 = 0;; u0 += 32) {
      const int mine = u0 + lane < units ? Kind::UC + kind.steps(c.n, u0 + lane) : 0;
      int sum = mine;
#pragma unroll
      for (int sh = 1; sh < 32; sh <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, sh);
        if (lane >= sh) sum += v;
      }
      const unsigned in = __ballot_sync(0xffffffffu, sum > rest);
      if (in) {
        const int l = __ffs(in) - 1;
        c.u = u0 + l;
        rest -= __shfl_sync(0xffffffffu, sum - mine, l);
        break;
      }
      rest -= __shfl_sync(0xffffffffu, sum, 31);
    }
    c.n_steps = kind.steps(c.n, c.u);
    c.step = max(0, rest - Kind::UC);
    if (c.step <= PT_SNAP) c.step = 0;
    if (c.n_steps - c.step <= PT_SNAP && c.step > 0) {
      c.step = 0;
      next(c);
    }
    return c;
  }
  JF_DEV void next(Cut& c) const {  // to the following unit's start
    if (++c.u == kind.units(c.n)) {
      c.u = 0;
      if (++c.kvh == Hkv) {
        c.kvh = 0;
        do {
          if (++c.b >= t.n_seqs) return;
          c.row0 = t.row_start[c.b];
          c.n = t.row_start[c.b + 1] - c.row0;
        } while (c.n == 0);
      }
    }
    c.n_steps = kind.steps(c.n, c.u);
  }
};
JF_DEV bool same_unit(const Cut& x, const Cut& y) { return x.b == y.b && x.kvh == y.kvh && x.u == y.u; }

// A CTA's walk along its run: units from `at` to `end`, steps c0 .. c1 - 1 of each. Uniform.
template <typename Kind>
struct Run {
  Line<Kind> line;
  Cut at, end;
  JF_DEV bool there() const { return at.b < line.t.n_seqs && !(same_unit(at, end) && at.step >= end.step); }
  JF_DEV int c0() const { return at.step; }
  JF_DEV int c1() const { return same_unit(at, end) ? end.step : at.n_steps; }
  JF_DEV bool whole() const { return at.step == 0 && c1() == at.n_steps; }
  JF_DEV int slot(int cta) const { return 2 * cta + (at.step > 0 ? 0 : 1); }  // where a part goes
  JF_DEV bool next() {
    if (same_unit(at, end)) return false;
    at.step = 0;
    line.next(at);
    return there();
  }
};

// ---------------------------------------------------------------------------------------------
// Pieces of the kernels
// ---------------------------------------------------------------------------------------------
JF_DEV float2 fma2(float2 x, float2 y, float2 z) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y), "f"(z.x), "f"(z.y));
  return r;
}
JF_DEV float2 add2(float2 x, float2 y) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
  return r;
}
JF_DEV uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Products and commits by the one lane whose `on` is set, in code that the warp goes through together (descriptors stay in
// uniform registers).
JF_DEV void mma_ss_on(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
JF_DEV void mma_ts_on(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
JF_DEV void commit_on(uint32_t bar, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(on)
      : "memory");
}

// A tile in shared memory: 128 rows of HD values as HD / 64 halves of 128 rows x 128 bytes with the 128-byte swizzle. Read
// K-major (rows are M or N, dims are K) or MN-major (dims are N, rows are K).
template <int HD>
struct Tile {
  static constexpr int BYTES = 128 * HD * 2, HALF = 16384;
  // both products over dims: D[128 rows of a][128 rows of b] = a b^T
  static JF_DEV void dots(uint32_t d, uint32_t a, uint32_t b, uint32_t on) {
    uint64_t da = sdesc_k_sw128(a), db = sdesc_k_sw128(b);
    asm volatile("" : "+l"(da), "+l"(db));  // (the sums below are not kept from step to step)
#pragma unroll
    for (int kk = 0; kk < HD / 16; ++kk)
      mma_ss_on(d, da + (uint64_t)((kk >> 2) * (HALF >> 4) + (kk & 3) * 2), db + (uint64_t)((kk >> 2) * (HALF >> 4) + (kk & 3) * 2),
                idesc_bf16_f32(128, 128), kk > 0 ? 1u : 0u, on);
  }
  // D[128][HD] (+)= w b over b's rows; w: bf16 in tensor memory, 64 columns, rows 64 .. at w + gap
  static JF_DEV void rows(uint32_t d, uint32_t w, uint32_t b, bool fresh, uint32_t on, uint32_t gap = 32) {
    uint64_t db = sdesc_mn_sw128(b, HALF, 1024u);
    asm volatile("" : "+l"(db));
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
      mma_ts_on(d, w + (kk >> 2) * gap + (kk & 3) * 8, db + (uint64_t)(kk * (2048 >> 4)), idesc_bf16_f32(128, HD) | (1u << 16),
                kk > 0 || !fresh ? 1u : 0u, on);
  }
  // Rows from `first` on are cleared, by a warp: what lies behind a text may be anything, and 0 times it nothing.
  static JF_DEV void clear_from(uint32_t tile, int first, int lane) {
    for (int i = first * 8 + lane; i < 128 * 8; i += 32)
#pragma unroll
      for (int h = 0; h < HD / 64; ++h)
        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(tile + h * HALF + i * 16), "r"(0) : "memory");
    fence_proxy_async_smem();
    __syncwarp();
  }
  // One box a half: `bytes` in all, to be expected on `bar` beforehand. By one lane.
  static JF_DEV void load(uint32_t tile, const CUtensorMap* map, uint32_t bar, int head, int row) {
#pragma unroll
    for (int h = 0; h < HD / 64; ++h) tma_load_3d_plain(tile + h * HALF, map, bar, 64 * h, head, row);
  }
};

// A wait that the warp agrees on; completion number `uses` (from 0) of the barrier.
JF_DEV bool warp_wait(uint64_t& bar, int uses) {
  const bool ok = mbar_wait_bounded(smem_u32(&bar), (uint32_t)uses & 1u, kWaitLimitDefaultNs);
  return __all_sync(0xffffffffu, ok) != 0;
}

template <int HD>
JF_DEV void scale_o(uint32_t t_o, float x) {
#pragma unroll 1
  for (int h = 0; h < HD / 16; ++h) {
    float o[16];
    uint32_t u[16];
    tmem_ld16(t_o + 16 * h, o);
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(o[i] * x);
    tmem_st16(t_o + 16 * h, u);
  }
}

// ---------------------------------------------------------------------------------------------
// Forward. A unit is two tiles of query rows (streams 0 and 1) over the key tiles that they see: while one stream's softmax
// runs, the tensor core works for the other. Tensor memory: S and O of each stream, P in bf16 in the place of the S it came
// from. Warps 0-3, 4-7: stream 0, 1, a thread per row; warp 8: copies; warp 9: products (10 and
// 11 give their registers away).
// ---------------------------------------------------------------------------------------------
constexpr int PA_THREADS = 384;
constexpr float PA_LAG = 8.f;  // a row's reference maximum follows its scores when they exceed it by more
template <int HD>
struct FwdLayout {
  static constexpr int Q = Tile<HD>::BYTES, KV = Tile<HD>::BYTES, RING = HD == 128 ? 4 : 8;  // (one CTA an SM: it has all tensor memory)
  static constexpr int OFF_KV = 2 * Q, TOTAL = OFF_KV + RING * KV + 1024;
  static constexpr int STATE = 256 * (HD + 2);  // floats of a part: O by 4 columns [HD / 4][256 rows][4], m, l
};
struct FwdMaps {
  CUtensorMap q, k, v;
};

// Output and lse of rows that belong to no text.
template <int HD>
JF_DEV void clear_rest(const PackedParams& a, int first_thread, int threads) {
  const int head = a.t.row_start[0], tail = a.t.row_start[a.t.n_seqs];
  const int tid = (int)threadIdx.x - first_thread, per_row = a.Hq * (HD / 8);
  for (int r = blockIdx.x; r < head + a.t.n_rows - tail; r += gridDim.x) {
    const long long row = r < head ? r : tail + r - head;
    for (int i = tid; i < per_row; i += threads) reinterpret_cast<uint4*>(a.out)[row * per_row + i] = make_uint4(0u, 0u, 0u, 0u);
    if (a.lse)
      for (int i = tid; i < a.Hq; i += threads) a.lse[row * a.Hq + i] = -INFINITY;
  }
}

template <int HD>
__global__ void __launch_bounds__(PA_THREADS, 1) k_packed_attn_tc(const PackedParams a, const __grid_constant__ FwdMaps maps) {
  using Lay = FwdLayout<HD>;
  using T = Tile<HD>;
  constexpr int RING = Lay::RING;
  extern __shared__ uint8_t sm_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(sm_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sQ = smem_u32(sm), sKV = sQ + Lay::OFF_KV;
  // queries there, read; keys or values there, read; per stream: S ready, P ready, P V done; everything done
  __shared__ __align__(8) uint64_t b_q[2], b_qfree[2], b_kv[RING], b_kvfree[RING], b_s[2], b_p[2], b_o[2], b_all;
  __shared__ uint32_t tmem_slot;
  __shared__ int s_bad;
  __shared__ Cut s_cut[2];
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int G = a.Hq / a.Hkv, tok = 128 / G;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&b_q[i]), 1);
      mbar_init(smem_u32(&b_qfree[i]), 1);
      mbar_init(smem_u32(&b_s[i]), 1);
      mbar_init(smem_u32(&b_p[i]), 4);
      mbar_init(smem_u32(&b_o[i]), 1);
    }
    for (int i = 0; i < RING; ++i) {
      mbar_init(smem_u32(&b_kv[i]), 1);
      mbar_init(smem_u32(&b_kvfree[i]), 1);
    }
    mbar_init(smem_u32(&b_all), 1);
    fence_mbar_init();
  }
  pdl_launch_dependents();
  pdl_wait();
  Run<ByQueries> w = {{{2 * tok}, a.t, a.Hkv, 0, nullptr}, {}, {}};
  if (!w.line.build(reinterpret_cast<int*>(sm), &s_bad, a.err)) return;
  const int workers = w.line.workers(gridDim.x);
  if (warp < 2 && (int)blockIdx.x < workers) {
    const Cut c = w.line.cut(blockIdx.x + warp, workers);
    if (lane == 0) s_cut[warp] = c;
  }
  if (warp == 8) {
    tmem_alloc(smem_u32(&tmem_slot), 512);
    tmem_relinquish();
  }
  fence_proxy_async_smem();  // (the line's place is taken by copies)
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
  const bool works = (int)blockIdx.x < workers && w.line.total > 0;
  w.at = s_cut[0], w.end = s_cut[1];
  bool ok = true, go = works && w.there();
  // steps of stream s of the unit in hand, within the run: from c0 on
  auto stream_steps = [&](int s) {
    const int first = (2 * w.at.u + s) * tok;  // its first token
    if (first >= w.at.n) return 0;
    return max(0, min(w.c1(), (min(w.at.n, first + tok) + PT_KEYS - 1) / PT_KEYS) - w.c0());
  };

  // Registers: 384 x 168 at launch; 128 x 80 + 256 x 208 are fewer.
  if (warp >= 8) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
  if (warp == 8) {
    int tiles = 0, units[2] = {0, 0};
    const uint32_t q_bytes = (uint32_t)(tok * G * HD * 2);
    while (go) {
      const int n = max(stream_steps(0), stream_steps(1));
      for (int s = 0; s < 2 && ok; ++s) {
        if (stream_steps(s) == 0) continue;
        ok = units[s] == 0 || warp_wait(b_qfree[s], units[s] - 1);
        if (ok && elect_one()) {
          mbar_arrive_expect_tx(smem_u32(&b_q[s]), q_bytes);
          T::load(sQ + s * Lay::Q, &maps.q, smem_u32(&b_q[s]), w.at.kvh * G, w.at.row0 + (2 * w.at.u + s) * tok);
        }
        __syncwarp();
        if (ok) ++units[s];
      }
      for (int i = 0; i < 2 * n && ok; ++i) {  // K, V, K, V, ...
        const int place = tiles % RING;
        ok = tiles < RING || warp_wait(b_kvfree[place], tiles / RING - 1);
        if (!ok) break;
        if (elect_one()) {
          mbar_arrive_expect_tx(smem_u32(&b_kv[place]), T::BYTES);
          T::load(sKV + place * Lay::KV, i & 1 ? &maps.v : &maps.k, smem_u32(&b_kv[place]), w.at.kvh, w.at.row0 + (w.c0() + i / 2) * PT_KEYS);
        }
        __syncwarp();
        ++tiles;
      }
      go = ok && w.next();
    }
    // every copy has landed before the CTA may leave, also after a wait that gave up
    for (int i = max(0, tiles - RING); i < tiles; ++i) warp_wait(b_kv[i % RING], i / RING);
    for (int s = 0; s < 2; ++s)
      if (units[s]) warp_wait(b_q[s], units[s] - 1);
    if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
  } else if (warp == 9) {
    int tiles = 0, units[2] = {0, 0}, ns[2] = {0, 0}, np[2] = {0, 0};  // (S and P V issued)
    const uint32_t on = elect_one();
    // S of stream s; its place is P's of the product before, which has been read then
    auto issue_s = [&](int s, int k_tile) {
      if (np[s] > 0) ok = ok && warp_wait(b_o[s], np[s] - 1);
      if (!ok) return;
      tc_fence_after();
      T::dots(tmem + s * 128, sQ + s * Lay::Q, sKV + k_tile % RING * Lay::KV, on);
      commit_on(smem_u32(&b_s[s]), on);
      ++ns[s];
    };
    while (go) {
      const int n_of[2] = {stream_steps(0), stream_steps(1)}, n = max(n_of[0], n_of[1]);
      ok = n == 0 || warp_wait(b_kv[tiles % RING], tiles / RING);
      for (int s = 0; s < 2 && ok; ++s) {
        if (n_of[s] == 0) continue;
        ok = warp_wait(b_q[s], units[s]++);
        if (ok) issue_s(s, tiles);
        if (n_of[s] == 1) commit_on(smem_u32(&b_qfree[s]), on);
      }
      commit_on(smem_u32(&b_kvfree[tiles % RING]), on);
      for (int j = 0; j < n && ok; ++j) {
        const int v_tile = tiles + 2 * j + 1, k_next = v_tile + 1;
        ok = warp_wait(b_kv[v_tile % RING], v_tile / RING);
        const int held = w.at.n - (w.c0() + j) * PT_KEYS;
        if (ok && held < PT_KEYS) T::clear_from(sKV + v_tile % RING * Lay::KV, held, lane);
        if (ok && j + 1 < n) ok = warp_wait(b_kv[k_next % RING], k_next / RING);
        for (int s = 0; s < 2 && ok; ++s) {
          if (j >= n_of[s]) continue;
          ok = warp_wait(b_p[s], np[s]);
          if (!ok) break;
          tc_fence_after();
          T::rows(tmem + 256 + s * 128, tmem + s * 128, sKV + v_tile % RING * Lay::KV, j == 0, on);
          commit_on(smem_u32(&b_o[s]), on);
          ++np[s];
          if (j + 1 < n_of[s]) {
            issue_s(s, k_next);
            if (j + 2 == n_of[s]) commit_on(smem_u32(&b_qfree[s]), on);
          }
        }
        commit_on(smem_u32(&b_kvfree[v_tile % RING]), on);
        if (j + 1 < n) commit_on(smem_u32(&b_kvfree[k_next % RING]), on);
      }
      tiles += 2 * n;
      go = ok && w.next();
    }
    if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_TMA);
    commit_on(smem_u32(&b_all), on);
    __syncwarp();
    warp_wait(b_all, 0);  // every product is complete before the CTA may leave
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    clear_rest<HD>(a, 0, 256);
    const int s = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_s = t_row + s * 128, t_o = t_row + 256 + s * 128;
    const int r_tok = r / G, r_head = r - r_tok * G;
    const bool flip = a.scale < 0.f;
    const float c = fmaxf(fabsf(a.scale) * kLog2e, 7.888609e-31f /* 2^-100: a hidden key's -inf stays one */);
    int steps = 0;
    while (go) {
      const int n = stream_steps(s);
      const int i = (2 * w.at.u + s) * tok + r_tok;  // the row's token in its text
      const bool live = r_tok < tok && i < w.at.n;
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < n; ++j, ++steps) {
        ok = warp_wait(b_s[s], steps);
        if (!ok) break;
        tc_fence_after();
        const int k0 = (w.c0() + j) * PT_KEYS;
        float v[4][32];
#pragma unroll
        for (int h = 0; h < 4; ++h) tmem_ld32(t_s + 32 * h, v[h]);
        if (flip) {
#pragma unroll
          for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int x = 0; x < 32; ++x) v[h][x] = -v[h][x];
        }
        if (k0 + PT_KEYS > (2 * w.at.u + s) * tok) {  // (some row does not see all of them)
          const int see = i - k0;  // columns 0 .. see
#pragma unroll
          for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int x = 0; x < 32; ++x) v[h][x] = 32 * h + x <= see ? v[h][x] : -INFINITY;
        }
        float mx[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          mx[h] = v[h][0];
#pragma unroll
          for (int x = 1; x < 32; ++x) mx[h] = fmaxf(mx[h], v[h][x]);
        }
        const float mc = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c;
        const bool raise = mc > m + PA_LAG;
        if (__any_sync(0xffffffffu, raise)) {
          const float al = raise ? (m == -INFINITY ? 0.f : packed_ex2(m - mc)) : 1.f;
          l *= al;
          if (raise) m = mc;
          if (j > 0) scale_o<HD>(t_o, al);
        }
        const float2 base = make_float2(m == -INFINITY ? 0.f : -m, m == -INFINITY ? 0.f : -m), cc = make_float2(c, c);
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t u[16];
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            float2 p = fma2(make_float2(v[h][2 * x], v[h][2 * x + 1]), cc, base);
            p.x = packed_ex2(p.x);
            p.y = packed_ex2(p.y);
            sum = add2(sum, p);
            u[x] = pack_bf16(p.x, p.y);
          }
          tmem_st16(t_s + 16 * h, u);
        }
        l += sum.x + sum.y;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&b_p[s]));
      }
      if (!ok) break;
      if (n > 0) {
        ok = warp_wait(b_o[s], steps - 1);
        if (!ok) break;
        tc_fence_after();
      }
      const long long at = (long long)(w.at.row0 + i) * a.Hq + w.at.kvh * G + r_head;
      if (w.whole()) {
        if (n > 0) {
          const float il = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
#pragma unroll 1
          for (int d = 0; d < HD; d += 32) {
            float o[32];
            tmem_ld32(t_o + d, o);
            if (live) {
              uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(a.out) + at * HD + d);
#pragma unroll
              for (int h = 0; h < 4; ++h)
                dst[h] = make_uint4(pack_bf16(o[8 * h] * il, o[8 * h + 1] * il), pack_bf16(o[8 * h + 2] * il, o[8 * h + 3] * il),
                                    pack_bf16(o[8 * h + 4] * il, o[8 * h + 5] * il), pack_bf16(o[8 * h + 6] * il, o[8 * h + 7] * il));
            }
          }
          if (live && a.lse) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
        }
      } else {
        float* st = a.states + (long long)w.slot(blockIdx.x) * Lay::STATE;
        const int row = s * 128 + r;
        if (n > 0) {
#pragma unroll 1
          for (int d = 0; d < HD; d += 16) {
            float o[16];
            tmem_ld16(t_o + d, o);
#pragma unroll
            for (int h = 0; h < 4; ++h)
              reinterpret_cast<float4*>(st)[(d / 4 + h) * 256 + row] = make_float4(o[4 * h], o[4 * h + 1], o[4 * h + 2], o[4 * h + 3]);
          }
        }
        st[256 * HD + row] = m;
        st[256 * (HD + 1) + row] = l;  // (0 where the stream had no step: O is not looked at)
      }
      tc_fence_before();
      go = w.next();
      if (!go) break;
    }
    if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 8) tmem_dealloc(tmem, 512);
}

// Joins the parts of the units that several CTAs share: CTA (cut i + 1, 32 of the unit's 256 rows). The unit that cut i lies
// in is joined by the first cut in it: CTAs i - 1, i, ... hold its parts in order.
template <int HD>
__global__ void __launch_bounds__(256) k_packed_attn_join(const PackedParams a, int most) {
  using Lay = FwdLayout<HD>;
  extern __shared__ int s_pre[];
  __shared__ int s_bad;
  __shared__ Cut s_cut[2];
  const int tid = threadIdx.x, warp = tid >> 5, G = a.Hq / a.Hkv, tok = 128 / G;
  pdl_launch_dependents();
  pdl_wait();
  Line<ByQueries> line = {{2 * tok}, a.t, a.Hkv, 0, nullptr};
  if (!line.build(s_pre, &s_bad, a.err)) return;
  const int workers = line.workers(most), i = blockIdx.x + 1;
  if (i >= workers || line.total == 0) return;
  if (warp < 2) {
    const Cut c = line.cut(i - 1 + warp, workers);
    if ((tid & 31) == 0) s_cut[warp] = c;
  }
  __syncthreads();
  const Cut before = s_cut[0], c = s_cut[1];
  if (c.b >= a.t.n_seqs || c.step == 0 || (same_unit(before, c) && before.step > 0)) return;
  int last = i;  // the part of CTA `last` ends the unit
  while (last + 1 < workers) {
    const Cut d = line.cut(last + 1, workers);
    if (!same_unit(d, c)) break;
    ++last;
  }
  const int row = blockIdx.y * 32 + (tid & 31), s = row >> 7, r = row & 127, r_tok = r / G;
  const int token = (2 * c.u + s) * tok + r_tok;
  if (r_tok >= tok || token >= c.n) return;
  // the first part lies in its CTA's second place, the others begin inside the unit
  auto part = [&](int k) { return a.states + (long long)(2 * k + (k == i - 1 ? 1 : 0)) * Lay::STATE; };
  float M = -INFINITY;
  for (int k = i - 1; k <= last; ++k) {
    const float* st = part(k);
    if (st[256 * (HD + 1) + row] != 0.f) M = fmaxf(M, st[256 * HD + row]);
  }
  float L = 0.f;
  float4 o[HD / 32];
#pragma unroll
  for (int x = 0; x < HD / 32; ++x) o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = i - 1; k <= last; ++k) {
    const float* st = part(k);
    const float l = st[256 * (HD + 1) + row], m = st[256 * HD + row];
    if (l == 0.f) continue;
    const float f = m == M ? 1.f : exp2f(m - M);
    L = fmaf(f, l, L);
#pragma unroll
    for (int x = 0; x < HD / 32; ++x) {
      const float4 v = reinterpret_cast<const float4*>(st)[(warp + 8 * x) * 256 + row];
      o[x].x = fmaf(f, v.x, o[x].x), o[x].y = fmaf(f, v.y, o[x].y), o[x].z = fmaf(f, v.z, o[x].z), o[x].w = fmaf(f, v.w, o[x].w);
    }
  }
  const float il = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
  const long long at = (long long)(c.row0 + token) * a.Hq + c.kvh * G + (r - r_tok * G);
#pragma unroll
  for (int x = 0; x < HD / 32; ++x)
    reinterpret_cast<uint2*>(reinterpret_cast<bf16*>(a.out) + at * HD)[warp + 8 * x] =
        make_uint2(pack_bf16(o[x].x * il, o[x].y * il), pack_bf16(o[x].z * il, o[x].w * il));
  if (warp == 0 && a.lse) a.lse[at] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
struct PackedDevice {
  int sms;
};
PerDeviceOnce g_tc_once;
PackedDevice g_tc[PerDeviceOnce::kMaxDevices];
template <int HD>
cudaError_t tc_prepare() {
  return cudaFuncSetAttribute(k_packed_attn_tc<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdLayout<HD>::TOTAL);
}
const PackedDevice* tc_device() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return nullptr;
  const int rc = g_tc_once.run(dev, [&]() -> int {
    cudaError_t e = cudaDeviceGetAttribute(&g_tc[dev].sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = tc_prepare<64>();
    if (e == cudaSuccess) e = tc_prepare<128>();
    return (int)e;
  });
  return rc == 0 ? &g_tc[dev] : nullptr;
}

// Rows of `heads` heads of hd as a tensor whose boxes are 64 dims x box_heads x box_rows.
bool tc_map(CUtensorMap* m, const void* p, long long ld, int heads, int hd, int rows, int box_heads, int box_rows) {
  const unsigned long long dims[3] = {(unsigned long long)hd, (unsigned long long)heads, (unsigned long long)rows};
  const unsigned long long strides[2] = {(unsigned long long)hd * 2, (unsigned long long)ld * 2};
  const unsigned box[3] = {64, (unsigned)box_heads, (unsigned)box_rows};
  return encode_tmap_bf16_3d(m, p, dims, strides, box);
}

// Whether units can be cut: a text of one key tile has units of one step.
bool tc_cuts(const jf_packed& t) { return t.max_rows > PT_KEYS; }

template <int HD>
jf_status tc_forward(const PackedParams& a, int sms, cudaStream_t st) {
  FwdMaps maps;
  const int G = a.Hq / a.Hkv, tok = 128 / G;
  if (!tc_map(&maps.q, a.q, a.ld_q, a.Hq, HD, a.t.n_rows, G, tok) || !tc_map(&maps.k, a.k, a.ld_k, a.Hkv, HD, a.t.n_rows, 1, 128) ||
      !tc_map(&maps.v, a.v, a.ld_v, a.Hkv, HD, a.t.n_rows, 1, 128))
    return JF_ECUDA;
  cudaError_t e = packed_launch(k_packed_attn_tc<HD>, dim3(sms), dim3(PA_THREADS), FwdLayout<HD>::TOTAL, st, a, maps);
  if (e == cudaSuccess && tc_cuts(a.t)) e = packed_launch(k_packed_attn_join<HD>, dim3(sms - 1, 8), dim3(256), (a.t.n_seqs + 1) * 4, st, a, sms);
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}

}  // namespace

bool packed_tc_rows(const void* p, long long ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

jf_status packed_tc_workspace(const jf_packed& t, int, int, int hd, bool, size_t* out_bytes) {
  const PackedDevice* d = tc_device();
  if (!d) return JF_ECUDA;
  *out_bytes = tc_cuts(t) ? (size_t)2 * d->sms * (hd == 128 ? FwdLayout<128>::STATE : FwdLayout<64>::STATE) * 4 : 0;
  return JF_OK;
}

jf_status packed_tc_forward(const PackedParams& p, int hd, void* workspace, cudaStream_t st) {
  const PackedDevice* d = tc_device();
  if (!d) return JF_ECUDA;
  PackedParams a = p;
  a.states = reinterpret_cast<float*>(workspace);
  return hd == 128 ? tc_forward<128>(a, d->sms, st) : tc_forward<64>(a, d->sms, st);
}

}  // namespace jf
