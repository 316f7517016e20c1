// Causal attention of packed bf16 texts and its backward pass on tcgen05 (jf_ops.h: jf_op_packed_attention*; the formulas
// stand in jf_packed.cu).
//
// Rows of a KV head. The G query heads that read a KV head meet the same keys, so a tile of query rows is TOK = 128 / G whole
// tokens times G heads (row = token * G + head), loaded as one box of a tensor copy: a short text fills the tensor core's 128
// rows G times sooner, and K and V are read once for G heads.
//
// What bounds a long text is the tensor core, and before it each stream's chain product -> softmax -> product; a short one, latency.
// Measured with 28 heads of 128 on 4: forward of 16,384 rows 1.33 ms (1.45 PFLOP/s), 4,096 rows 112 us, 16 texts of up to 128 rows
// (12 heads on 2) 10.8 us; backward of 8,192 rows 1.24 ms (0.97 PFLOP/s of the five products' work; seven are multiplied), 4 x 1,024
// rows 151 us. (From run to run by up to 2%, 1,315 to 1,340 us: the figures beside a choice below are of one run each.)
//
// Work is a line of units, (text, KV head, tile), each as long as its steps (tiles of keys, or of query rows in dk and dv)
// plus a constant for what a unit costs beside them; each CTA takes an equal run of that line. A unit that a run's end cuts leaves a
// partial result a part in the workspace, at most two a CTA, and a kernel behind joins the parts in their order. Short units are
// not cut: the cut moves to their nearer end.
#include "jf_once.h"
#include "jf_packed.cuh"

namespace jf {
namespace {

constexpr int PT_KEYS = 128;                     // keys of a step (of a tile, in dk and dv)
// Units of so many steps are not cut: a part that is written, read again and added up costs about as much as two steps, and a batch
// of such units only takes no second kernel. Backward of 16 texts of up to 128 rows (28 heads on 4) 41 us (44 with 6), forward of 1,024
// rows 23 (28 with 6); with 16 the backward pass of 4 x 1,024 rows (28 on 4) takes 158 instead of 149.
constexpr int PT_WHOLE = 8;

// ---------------------------------------------------------------------------------------------
// The line of units. Kind says how a text is cut: units(n), steps(n, u) for a text of n rows.
// ---------------------------------------------------------------------------------------------
// (What a unit costs beside its steps, in steps, times in us: forward of 16,384 rows 1,432, 1,316, 1,342 with 0, 2, 4, a packed batch of 8,246
// 205, 155, 164; backward of 8,192 rows by dq's 1,287, 1,225, 1,240 with 2, 5, 8, by that of dk and dv 1,251, 1,225, 1,237 with 1, 3, 6.)
template <int COST>
struct ByQueries {  // tiles of `tok` tokens over the key tiles that they see; COST: of a unit beside its steps
  static constexpr bool KEYS = false;
  static constexpr int UC = COST;
  int tok;
  JF_DEV int units(int n) const { return (n + tok - 1) / tok; }
  JF_DEV int steps(int n, int u) const { return (min(n, (u + 1) * tok) + PT_KEYS - 1) / PT_KEYS; }
};

using ByFwd = ByQueries<2>;
using ByDq = ByQueries<5>;

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
  // How many of `most` CTAs have a run: none is shorter than a unit of one step.
  JF_DEV int workers(int most) const { return max(1, min(most, total / (Kind::UC + 1))); }
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
    if (c.n_steps <= PT_WHOLE) {  // to the nearer end
      const bool behind = c.step > c.n_steps / 2;
      c.step = 0;
      if (behind) next(c);
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

// A CTA's walk along its run: units from `at` to `end` (in shared memory), steps c0 .. c1 - 1 of each. Uniform.
template <typename Kind>
struct Run {
  Line<Kind> line;
  Cut at;
  const Cut* end;
  JF_DEV bool there() const { return at.b < line.t.n_seqs && !(same_unit(at, *end) && at.step >= end->step); }
  JF_DEV int c0() const { return at.step; }
  JF_DEV int c1() const { return same_unit(at, *end) ? end->step : at.n_steps; }
  JF_DEV bool whole() const { return at.step == 0 && c1() == at.n_steps; }
  JF_DEV int slot(int cta) const { return 2 * cta + (at.step > 0 ? 0 : 1); }  // where a part goes
  JF_DEV bool next() {
    if (same_unit(at, *end)) return false;
    at.step = 0;
    line.next(at);
    return there();
  }
};

// Where CTAs' runs begin, for the kernel that joins parts: two int4 a CTA.
constexpr int NO_UNIT = 0x7fffffff;
JF_DEV void tell_cut(int* cuts, const Cut& c, bool works) {
  if (!cuts) return;
  int4* at = reinterpret_cast<int4*>(cuts) + 2 * blockIdx.x;
  at[0] = make_int4(works ? c.b : NO_UNIT, c.kvh, c.u, c.step);
  at[1] = make_int4(c.n_steps, c.row0, c.n, 0);
}
JF_DEV Cut read_cut(const int* cuts, int cta) {
  const int4 x = reinterpret_cast<const int4*>(cuts)[2 * cta], y = reinterpret_cast<const int4*>(cuts)[2 * cta + 1];
  return {x.x, x.y, x.z, x.w, y.x, y.y, y.z};
}
// The parts of a unit that is cut by the beginning of CTA i's run and by none before: CTAs i - 1 .. last. False: there is no such unit.
JF_DEV bool parts_from(const int* cuts, int ctas, int n_seqs, int i, Cut& c, int& last) {
  c = read_cut(cuts, i);
  if (c.b >= n_seqs || c.step == 0) return false;
  const Cut before = read_cut(cuts, i - 1);
  if (same_unit(before, c) && before.step > 0) return false;
  for (last = i;; last += 32) {  // (a unit may lie in many runs)
    const int k = last + 1 + (threadIdx.x & 31);
    const bool same = k < ctas && same_unit(read_cut(cuts, k), c);
    const unsigned rest = __ballot_sync(0xffffffffu, !same);
    if (rest) {
      last += __ffs(rest) - 1;
      return true;
    }
  }
}

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
// 128 consecutive columns of this warp's 32 lanes, at once.
JF_DEV void tmem_ld128(uint32_t taddr, float (&v)[128]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x128.b32 {"
        "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,"
        "%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
        "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63,"
        "%64,%65,%66,%67,%68,%69,%70,%71,%72,%73,%74,%75,%76,%77,%78,%79,"
        "%80,%81,%82,%83,%84,%85,%86,%87,%88,%89,%90,%91,%92,%93,%94,%95,"
        "%96,%97,%98,%99,%100,%101,%102,%103,%104,%105,%106,%107,%108,%109,%110,%111,"
        "%112,%113,%114,%115,%116,%117,%118,%119,%120,%121,%122,%123,%124,%125,%126,%127}, [%128];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
        "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
        "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]),
        "=f"(v[32]), "=f"(v[33]), "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]),
        "=f"(v[40]), "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), "=f"(v[45]), "=f"(v[46]), "=f"(v[47]),
        "=f"(v[48]), "=f"(v[49]), "=f"(v[50]), "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]),
        "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63]),
        "=f"(v[64]), "=f"(v[65]), "=f"(v[66]), "=f"(v[67]), "=f"(v[68]), "=f"(v[69]), "=f"(v[70]), "=f"(v[71]),
        "=f"(v[72]), "=f"(v[73]), "=f"(v[74]), "=f"(v[75]), "=f"(v[76]), "=f"(v[77]), "=f"(v[78]), "=f"(v[79]),
        "=f"(v[80]), "=f"(v[81]), "=f"(v[82]), "=f"(v[83]), "=f"(v[84]), "=f"(v[85]), "=f"(v[86]), "=f"(v[87]),
        "=f"(v[88]), "=f"(v[89]), "=f"(v[90]), "=f"(v[91]), "=f"(v[92]), "=f"(v[93]), "=f"(v[94]), "=f"(v[95]),
        "=f"(v[96]), "=f"(v[97]), "=f"(v[98]), "=f"(v[99]), "=f"(v[100]), "=f"(v[101]), "=f"(v[102]), "=f"(v[103]),
        "=f"(v[104]), "=f"(v[105]), "=f"(v[106]), "=f"(v[107]), "=f"(v[108]), "=f"(v[109]), "=f"(v[110]), "=f"(v[111]),
        "=f"(v[112]), "=f"(v[113]), "=f"(v[114]), "=f"(v[115]), "=f"(v[116]), "=f"(v[117]), "=f"(v[118]), "=f"(v[119]),
        "=f"(v[120]), "=f"(v[121]), "=f"(v[122]), "=f"(v[123]), "=f"(v[124]), "=f"(v[125]), "=f"(v[126]), "=f"(v[127])
      : "r"(taddr)
      : "memory");
}
JF_DEV uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
JF_DEV float tmem_ld1(uint32_t taddr) {
  float v;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=f"(v) : "r"(taddr) : "memory");
  return v;
}
JF_DEV void tmem_st1(uint32_t taddr, float v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "f"(v) : "memory");
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
  // D[128][HD] (+)= w b over b's rows. w: bf16 in tensor memory in the place of the scores that it came from, those of each PER x 16
  // of b's rows at the beginning of their columns. FIRST, COUNT: which runs of 16 rows.
  template <int PER, int FIRST = 0, int COUNT = PER>
  static JF_DEV void rows(uint32_t d, uint32_t w, uint32_t b, bool fresh, uint32_t on) {
    uint64_t db = sdesc_mn_sw128(b, HALF, 1024u);
    asm volatile("" : "+l"(db));
#pragma unroll
    for (int i = 0; i < 8 / PER * COUNT; ++i) {
      const int kk = i / COUNT * PER + FIRST + i % COUNT;  // runs FIRST .. FIRST + COUNT - 1 of each PER
      mma_ts_on(d, w + kk / PER * (PER * 16) + kk % PER * 8, db + (uint64_t)(kk * (2048 >> 4)), idesc_bf16_f32(128, HD) | (1u << 16),
                FIRST > 0 || i > 0 || !fresh ? 1u : 0u, on);
    }
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

template <int COLUMNS>
JF_DEV void scale_o(uint32_t t_o, float x) {
#pragma unroll 1
  for (int h = 0; h < COLUMNS / 16; ++h) {
    float o[16];
    uint32_t u[16];
    tmem_ld16(t_o + 16 * h, o);
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(o[i] * x);
    tmem_st16(t_o + 16 * h, u);
  }
}

// ---------------------------------------------------------------------------------------------
// Forward: one pass over the keys with a row's running maximum m and sum l, out = O / l. p = 2^(s - m) is rounded to bf16 for its product
// with V (the tensor core takes both operands in one type), l adds the unrounded ones: up to 2^-8 of a key's share, each with a sign of
// its own, beside out's own rounding of up to 2^-8. m follows its row's scores only where they exceed it by 2^PA_LAG, so that O is
// seldom scaled; p then is at most 2^8, which costs bf16 nothing (0 instead of 8: 1,593 us for 16,384 rows, 1,328 with).
//
// A unit is two tiles of query rows (streams 0 and 1) over the key tiles that they see: while one stream's softmax
// runs, the tensor core works for the other. Tensor memory: S and O of each stream, P in bf16 in the place of the S it came
// from. Warps 0-3, 4-7: stream 0, 1, a thread per row; warp 8: copies; 9, 10: the streams' products; 11: values behind a text's end.
// (Two threads a row, in 16 warps, took 1.4 times as long: they have to agree on the row's maximum at every step, and 96 registers
// are too few.) At 8,192 rows the tensor pipe is active 62% of the time, issue slots 34%: the rest is a stream's own chain, read S,
// maximum, exponentials, write P, wait for the product, of which two streams hide a half. (Slower at 16,384 rows, 1,315 us: strict turns between
// the streams' products, 1,329 to 1,366 by what a turn covers; scores read twice from tensor memory instead of kept, 1,448; a quarter of
// the exponentials by a polynomial on the FMA units beside that, 1,499.)
// ---------------------------------------------------------------------------------------------
constexpr int PA_THREADS = 384;  // 168 registers a thread: a row's 128 scores fit
constexpr float PA_LAG = 8.f;  // a row's reference maximum follows its scores when they exceed it by more
template <int HD>
struct FwdLayout {
  static constexpr int Q = Tile<HD>::BYTES, KV = Tile<HD>::BYTES, RING = HD == 128 ? 4 : 8;
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
  // queries there, read; keys or values there (b_raw: with rows to be cleared), read (by both streams); per stream: S ready, P ready (its first 64 keys, all), P V
  // done; everything done
  __shared__ __align__(8) uint64_t b_q[2], b_qfree[2], b_kv[RING], b_raw[RING], b_kvfree[RING], b_s[2], b_p[2][2], b_o[2], b_all[2];
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
      mbar_init(smem_u32(&b_p[i][0]), 4);
      mbar_init(smem_u32(&b_p[i][1]), 4);
      mbar_init(smem_u32(&b_o[i]), 1);
      mbar_init(smem_u32(&b_all[i]), 1);
    }
    for (int i = 0; i < RING; ++i) {
      mbar_init(smem_u32(&b_kv[i]), 1);
      mbar_init(smem_u32(&b_raw[i]), 1);
      mbar_init(smem_u32(&b_kvfree[i]), 2);
    }
    fence_mbar_init();
  }
  pdl_launch_dependents();
  pdl_wait();
  Run<ByFwd> w = {{{2 * tok}, a.t, a.Hkv, 0, nullptr}, {}, &s_cut[1]};
  if (!w.line.build(reinterpret_cast<int*>(sm), &s_bad, a.err)) {
    if (tid == 0) tell_cut(a.cuts, {}, false);
    return;
  }
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
  w.at = s_cut[0];
  bool ok = true, go = (int)blockIdx.x < workers && w.line.total > 0 && w.there();
  if (tid == 0) tell_cut(a.cuts, w.at, (int)blockIdx.x < workers && w.line.total > 0);
  // steps of stream s of the unit in hand, within the run: from c0 on
  auto stream_steps = [&](const Run<ByFwd>& w, int s) {
    const int first = (2 * w.at.u + s) * tok;  // its first token
    if (first >= w.at.n) return 0;
    return max(0, min(w.c1(), (min(w.at.n, first + tok) + PT_KEYS - 1) / PT_KEYS) - w.c0());
  };

  if (warp >= 8) {
    if (warp == 8) {
      int tiles = 0, units[2] = {0, 0};
      const uint32_t q_bytes = (uint32_t)(tok * G * HD * 2);
      while (go) {
        const int n0 = stream_steps(w, 0), n1 = stream_steps(w, 1), n = max(n0, n1);
        for (int s = 0; s < 2 && ok; ++s) {
          if ((s ? n1 : n0) == 0) continue;
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
          const bool raw = i == 2 * n - 1 && w.c1() * PT_KEYS > w.at.n;  // values of a text's last tile
          if (elect_one()) {
            const uint32_t bar = smem_u32(raw ? &b_raw[place] : &b_kv[place]);
            mbar_arrive_expect_tx(bar, T::BYTES);
            T::load(sKV + place * Lay::KV, i & 1 ? &maps.v : &maps.k, bar, w.at.kvh, w.at.row0 + (w.c0() + i / 2) * PT_KEYS);
          }
          __syncwarp();
          ++tiles;
        }
        go = ok && w.next();
      }
      // every copy has landed before the CTA may leave, also after a wait that gave up (b_raw's are forwarded)
      for (int i = max(0, tiles - RING); i < tiles; ++i) warp_wait(b_kv[i % RING], i / RING);
      for (int s = 0; s < 2; ++s)
        if (units[s]) warp_wait(b_q[s], units[s] - 1);
      if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
    } else if (warp < 11) {
      // A stream's products. (A warp of its own for each: what one waits for does not hold up the other.)
      const int s = warp - 9;
      const uint32_t on = elect_one(), t_s = tmem + s * 128, t_o = tmem + 256 + s * 128;
      int tiles = 0, units = 0, products = 0;  // tiles before the unit, units, P V so far
      auto place_of = [&](int tile) { return __shfl_sync(0xffffffffu, tile % RING, 0); };
      // The streams run best half a step apart, one's softmax beside the other's products, and stay so: the second begins when the
      // first's first P is there. (Or after 4 us: nothing depends on it. Without, 4,096 rows 113 us instead of 110, the packed batch 162 instead of 154.)
      if (s == 1 && go && stream_steps(w, 0) > 2) mbar_wait_bounded(smem_u32(&b_p[0][1]), 0u, 4000ull);
      while (go) {
        const int n = stream_steps(w, s), all = max(n, stream_steps(w, 1 - s));
        if (n > 0) ok = warp_wait(b_q[s], units++);
        for (int j = 0; j < n && ok; ++j) {
          const int k_tile = tiles + 2 * j, v_tile = k_tile + 1, kp = place_of(k_tile), vp = place_of(v_tile);
          ok = warp_wait(b_kv[kp], k_tile / RING);
          // S: its place is P's of the product before, which has been read then
          if (products > 0) ok = ok && warp_wait(b_o[s], products - 1);
          if (!ok) break;
          tc_fence_after();
          T::dots(t_s, sQ + s * Lay::Q, sKV + kp * Lay::KV, on);
          commit_on(smem_u32(&b_s[s]), on);
          commit_on(smem_u32(&b_kvfree[kp]), on);
          if (j + 1 == n) commit_on(smem_u32(&b_qfree[s]), on);
          ok = warp_wait(b_kv[vp], v_tile / RING) && warp_wait(b_p[s][0], products);
          if (!ok) break;
          tc_fence_after();
          T::template rows<8, 0, 4>(t_o, t_s, sKV + vp * Lay::KV, j == 0, on);
          ok = warp_wait(b_p[s][1], products);
          if (!ok) break;
          tc_fence_after();
          T::template rows<8, 4, 4>(t_o, t_s, sKV + vp * Lay::KV, false, on);
          commit_on(smem_u32(&b_o[s]), on);
          commit_on(smem_u32(&b_kvfree[vp]), on);
          ++products;
        }
        for (int i = 2 * n; i < 2 * all && ok; ++i) {  // tiles of the other stream's alone: read as soon as they are there
          const int place = place_of(tiles + i);
          ok = warp_wait(b_kv[place], (tiles + i) / RING);
          commit_on(smem_u32(&b_kvfree[place]), on);
        }
        tiles += 2 * all;
        go = ok && w.next();
      }
      if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_TMA);
      commit_on(smem_u32(&b_all[s]), on);
      __syncwarp();
      warp_wait(b_all[s], 0);  // every product is complete before the CTA may leave
    } else {
      // Values behind the end of a text are cleared before the products see the tile.
      int tiles = 0;
      unsigned uses = 0;  // of each place's b_raw, their parities
      while (go) {
        const int n = max(stream_steps(w, 0), stream_steps(w, 1));
        tiles += 2 * n;
        if (w.c1() * PT_KEYS > w.at.n) {
          const int place = (tiles - 1) % RING;
          ok = warp_wait(b_raw[place], (int)(uses >> place & 1u));
          uses ^= 1u << place;
          if (!ok) break;
          T::clear_from(sKV + place * Lay::KV, w.at.n - (w.c1() - 1) * PT_KEYS, lane);
          if (lane == 0) mbar_arrive(smem_u32(&b_kv[place]));
        }
        go = w.next();
      }
      if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_TMA);
    }
  } else {
    clear_rest<HD>(a, 0, 256);
    const int s = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_s = t_row + s * 128, t_o = t_row + 256 + s * 128;
    const int r_tok = r / G, r_head = r - r_tok * G;
    const bool flip = a.scale < 0.f;
    const float c = fmaxf(fabsf(a.scale) * kLog2e, 7.888609e-31f /* 2^-100: a hidden key's -inf stays one */);
    int steps = 0;
    while (go) {
      const int n = stream_steps(w, s);
      const int i = (2 * w.at.u + s) * tok + r_tok;  // the row's token in its text
      const bool live = r_tok < tok && i < w.at.n;
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < n; ++j, ++steps) {
        ok = warp_wait(b_s[s], steps);
        if (!ok) break;
        tc_fence_after();
        const int k0 = (w.c0() + j) * PT_KEYS;
        float v[128];
        tmem_ld128(t_s, v);
        if (flip) {
#pragma unroll
          for (int x = 0; x < 128; ++x) v[x] = -v[x];
        }
        if (k0 + PT_KEYS > (2 * w.at.u + s) * tok) {  // (some row does not see all of them)
          const int see = i - k0;  // columns 0 .. see
#pragma unroll
          for (int x = 0; x < 128; ++x) v[x] = x <= see ? v[x] : -INFINITY;
        }
        float mx[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          mx[h] = v[h];
#pragma unroll
          for (int x = 4; x < 128; x += 4) mx[h] = fmaxf(mx[h], v[x + h]);
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
            float2 p = fma2(make_float2(v[32 * h + 2 * x], v[32 * h + 2 * x + 1]), cc, base);
            p.x = packed_ex2(p.x);
            p.y = packed_ex2(p.y);
            sum = add2(sum, p);
            u[x] = pack_bf16(p.x, p.y);
          }
          tmem_st16(t_s + 16 * h, u);
          if (h & 1) {
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_p[s][h >> 1]));
          }
        }
        l += sum.x + sum.y;
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

// Joins the parts of the units that several CTAs share: CTA (run i + 1, an eighth of the columns of the unit's 256 rows). out = sum_k
// 2^(m_k - M) O_k / sum_k 2^(m_k - M) l_k, in the parts' order. Bound by the latency of its loads: 36 MB in
// 16 us from a cold L2 at 8,192 rows (2.3 TB/s).
template <int HD>
__global__ void __launch_bounds__(256) k_packed_attn_join(const PackedParams a) {
  using Lay = FwdLayout<HD>;
  constexpr int X = HD / 32;  // pieces of 4 columns of a thread
  const int G = a.Hq / a.Hkv, tok = 128 / G, i = blockIdx.x + 1;
  pdl_launch_dependents();
  pdl_wait();
  Cut c;
  int last;
  if (!parts_from(a.cuts, gridDim.x + 1, a.t.n_seqs, i, c, last)) return;
  const int row = threadIdx.x, x0 = blockIdx.y * X, s = row >> 7, r = row & 127, r_tok = r / G;
  const int token = (2 * c.u + s) * tok + r_tok;
  if (r_tok >= tok || token >= c.n) return;
  // the first part lies in its CTA's second place, the others begin inside the unit
  auto part = [&](int k) { return a.states + (long long)(2 * k + (k == i - 1 ? 1 : 0)) * Lay::STATE; };
  float M = -INFINITY, L = 0.f;
  float4 o[X];
#pragma unroll
  for (int x = 0; x < X; ++x) o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
  for (int k = i - 1; k <= last; ++k) {
    const float* st = part(k);
    const float l = st[256 * (HD + 1) + row], m = st[256 * HD + row];
    float4 v[X];
#pragma unroll
    for (int x = 0; x < X; ++x) v[x] = reinterpret_cast<const float4*>(st)[(x0 + x) * 256 + row];
    if (l == 0.f) continue;  // (it saw nothing)
    const float top = fmaxf(M, m), f0 = M == top ? 1.f : exp2f(M - top), f1 = m == top ? 1.f : exp2f(m - top);
    M = top;
    L = f0 * L + f1 * l;
#pragma unroll
    for (int x = 0; x < X; ++x)
      o[x].x = f0 * o[x].x + f1 * v[x].x, o[x].y = f0 * o[x].y + f1 * v[x].y, o[x].z = f0 * o[x].z + f1 * v[x].z, o[x].w = f0 * o[x].w + f1 * v[x].w;
  }
  const float il = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
  const long long at = (long long)(c.row0 + token) * a.Hq + c.kvh * G + (r - r_tok * G);
#pragma unroll
  for (int x = 0; x < X; x += 2)
    reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(a.out) + at * HD + 4 * x0)[x / 2] =
        make_uint4(pack_bf16(o[x].x * il, o[x].y * il), pack_bf16(o[x].z * il, o[x].w * il), pack_bf16(o[x + 1].x * il, o[x + 1].y * il),
                   pack_bf16(o[x + 1].z * il, o[x + 1].w * il));
  if (x0 == 0 && a.lse) a.lse[at] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
}

// ---------------------------------------------------------------------------------------------
// Backward. Two kernels, each with sums of its own and no atomics: dq by tiles of query rows over the keys, dk and dv by
// tiles of keys over the query rows; the scores are multiplied out in both (7 products instead of 5).
//
// p and ds are rounded to bf16 for their products, as P is in the forward pass, sums are fp32. Of dq's norm the rounding of ds takes
// 1.8e-3, dq's own 1.65e-3, out's (through delta) 0.3e-3, for 2,048 random rows; of a text's first rows dq takes ds as two terms (two_terms).
//
// delta = d_out . out loses what out was rounded by, which counts where a row sees few keys. As sum_j ds_ij = 0 for the exact
// delta, the dq kernel adds up its ds (a row lies in one thread, or two) and corrects delta by it for dk; where a row's keys
// are one step it takes delta = sum_j p_ij dp_ij to begin with.
//
// A step's 128 x 128 scores are 16 warps' work, 32 columns of a row a thread; warp 16: copies; 17: products that give scores; 18:
// products with what the scores have become (a warp of its own: a wait of one, which stands behind its products in the tensor
// core's queue, does not hold up the other); 19: row statistics (dk and dv).
// ---------------------------------------------------------------------------------------------
constexpr int PT_THREADS = 640;  // 96 registers a thread (and so one CTA an SM, which has all of its tensor memory)
struct BackMaps {
  CUtensorMap q, k, v, d_out;
};

template <int HD>
struct BackLayout {
  static constexpr int T = Tile<HD>::BYTES, OFF_RING = 2 * T;
  static constexpr int TOTAL = OFF_RING + 4 * T + 1024;
  static constexpr int DQ_STATE = 128 * (HD + 2);  // floats of a part: dq by 4 columns [HD / 4][128 rows][4], sum of ds, delta
  static constexpr int DKV_STATE = 2 * 128 * HD;   // dv, dk, each by 4 columns
};

// Gradients of rows that belong to no text, by `threads` threads.
template <int HD>
JF_DEV void clear_rows(const jf_packed& t, void* p, long long ld, int heads, int tid, int threads) {
  const int head = t.row_start[0], tail = t.row_start[t.n_seqs], width = heads * HD;
  for (int r = blockIdx.x; r < head + t.n_rows - tail; r += gridDim.x) {
    const long long row = r < head ? r : tail + r - head;
    for (int i = tid; i < width; i += threads) reinterpret_cast<bf16*>(p)[row * ld + i] = __float2bfloat16_rn(0.f);
  }
}

// What both kernels begin with: the line's cuts, tensor memory. False: nothing to do for the whole grid.
template <typename Kind>
JF_DEV bool back_begin(Run<Kind>& w, const PackedParams& a, uint8_t* sm, int* s_bad, Cut* s_cut, uint32_t* tmem_slot, bool& go) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_launch_dependents();
  pdl_wait();
  if (!w.line.build(reinterpret_cast<int*>(sm), s_bad, a.err)) {
    if (tid == 0) tell_cut(a.cuts, {}, false);
    return false;
  }
  const int workers = w.line.workers(gridDim.x);
  if (warp < 2 && (int)blockIdx.x < workers) {
    const Cut c = w.line.cut(blockIdx.x + warp, workers);
    if (lane == 0) s_cut[warp] = c;
  }
  if (warp == 16) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  fence_proxy_async_smem();  // (the line's place is taken by copies)
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  w.at = s_cut[0];
  go = (int)blockIdx.x < workers && w.line.total > 0;
  if (tid == 0) tell_cut(a.cuts, w.at, go);
  go = go && w.there();
  return true;
}

// 8 bf16 products of two runs of memory
JF_DEV float dot8(const uint4& x, const uint4& y, float s) {
  const uint32_t a[4] = {x.x, x.y, x.z, x.w}, b[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s = fmaf(__uint_as_float(a[i] << 16), __uint_as_float(b[i] << 16), s);
    s = fmaf(__uint_as_float(a[i] & 0xffff0000u), __uint_as_float(b[i] & 0xffff0000u), s);
  }
  return s;
}

// delta = d_out . out of every row and head, HD / 8 lanes each (rows of no text as well: not used). Bound by its bytes: 117 MB at 8,192
// rows of 28 heads, 19 us from a cold L2 (6.2 TB/s).
template <int HD>
__global__ void __launch_bounds__(256) k_packed_delta_tc(const PackedParams a) {
  constexpr int LPR = HD / 8;
  pdl_launch_dependents();
  pdl_wait();
  const uint32_t i = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, piece = threadIdx.x % LPR;  // (n_rows * Hq is at most 2^30)
  const uint32_t row = i / a.Hq;
  float d = 0.f;
  if ((int)row < a.t.n_rows)
    d = dot8(reinterpret_cast<const uint4*>(a.out)[(long long)i * LPR + piece],
             reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(a.d_out) + row * a.ld_do + (long long)(i - row * a.Hq) * HD)[piece], 0.f);
#pragma unroll
  for (int sh = LPR / 2; sh; sh >>= 1) d += __shfl_xor_sync(0xffffffffu, d, sh);
  if (piece == 0 && (int)row < a.t.n_rows) a.delta[i] = d;
}

// Whether a unit's ds goes into dq as two bf16 terms, the second what the first's rounding leaves: in a text's first quarter, and its first
// 512 rows. Rows that see few keys have the largest gradients, and so the largest part in dq's error: 1.7e-3 (300 rows) to 2.0e-3 (2,000) of its norm
// instead of 2.4e-3, for one more product in a sixteenth of a long text's steps: 1,257 us for the pass over
// 8,192 rows, 1,228 without, others within 1%. (As if those steps were longer by two thirds in the line: 1,275.) (In the
// first 1,024 rows of all texts: 1.9 to 2.0e-3, 4% of the pass for 4 x 1,024 rows.)
JF_DEV bool two_terms(const Cut& c) { return c.n_steps <= max(4, c.n >> 9); }

template <int HD>
struct DqLayout {
  // tiles in shared memory beside Q and d_out: a key tile is held until dQ has read it (two of each: 8,192 rows 1,280 us, 1,230 with three)
  static constexpr int T = Tile<HD>::BYTES, KEYS = 3, VALUES = 2;
  static constexpr int TOTAL = (2 + KEYS + VALUES) * T + 1024;
};

// dq. Tensor memory: S, two dP (ds in bf16 in their places), dQ. S and dP of the next step are multiplied before dQ of this one, so that the
// warps and the tensor core both have work ahead. At 8,192 rows, ds as one term, 508 us (three products, 1.42 PFLOP/s; some 30 more with two), tensor pipe 64%, issue slots 48%: a
// step's exponentials and products of a row's 128 scores take the warps about as long as the tensor core. Slower: Q and d_out as operands
// from tensor memory (no gain), two groups of warps that take steps by turns (96 registers spill, 1.4 times as long).
template <int HD>
__global__ void __launch_bounds__(PT_THREADS, 1) k_packed_dq_tc(const PackedParams a, const __grid_constant__ BackMaps maps) {
  using Lay = DqLayout<HD>;
  using T = Tile<HD>;
  extern __shared__ uint8_t sm_raw[];
  uint8_t* smp = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(sm_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sQ = smem_u32(smp), sdO = sQ + Lay::T, sK = sdO + Lay::T, sV = sK + Lay::KEYS * Lay::T;
  // Q and d_out there, read; keys, values there, read; S ready, read; dP ready; ds ready; dQ of a step done, of a unit; everything
  // done. (Two, for even and odd steps, of those that may complete again before a slow warp has seen them.)
  __shared__ __align__(8) uint64_t b_fix, b_fixfree, b_k[Lay::KEYS], b_kfree[Lay::KEYS], b_v[Lay::VALUES], b_vfree[Lay::VALUES], b_s, b_sread, b_dp[2],
      b_ds[2], b_o[2], b_unit, b_all[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int s_bad;
  __shared__ Cut s_cut[2];
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int G = a.Hq / a.Hkv, tok = 128 / G;
  if (tid == 0) {
    uint64_t* const ones[] = {&b_fix, &b_fixfree, &b_s, &b_dp[0], &b_dp[1], &b_o[0], &b_o[1], &b_unit, &b_all[0], &b_all[1]};
    for (uint64_t* b : ones) mbar_init(smem_u32(b), 1);
    for (int i = 0; i < Lay::KEYS; ++i) mbar_init(smem_u32(&b_k[i]), 1), mbar_init(smem_u32(&b_kfree[i]), 1);
    for (int i = 0; i < Lay::VALUES; ++i) mbar_init(smem_u32(&b_v[i]), 1), mbar_init(smem_u32(&b_vfree[i]), 1);
    mbar_init(smem_u32(&b_sread), 16);
    mbar_init(smem_u32(&b_ds[0]), 16);
    mbar_init(smem_u32(&b_ds[1]), 16);
    fence_mbar_init();
  }
  Run<ByDq> w = {{{tok}, a.t, a.Hkv, 0, nullptr}, {}, &s_cut[1]};
  bool go, ok = true;
  if (!back_begin(w, a, smp, &s_bad, s_cut, &tmem_slot, go)) return;
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0), tS = tmem, tP = tmem + 128, tG = tmem + 384;

  if (warp >= 16) {
    if (warp == 16) {
      int units = 0, nk = 0, nv = 0;  // asked for
      const uint32_t fix_bytes = (uint32_t)(2 * tok * G * HD * 2);
      while (go) {
        ok = units == 0 || warp_wait(b_fixfree, units - 1);
        if (!ok) break;
        if (elect_one()) {
          mbar_arrive_expect_tx(smem_u32(&b_fix), fix_bytes);
          T::load(sQ, &maps.q, smem_u32(&b_fix), w.at.kvh * G, w.at.row0 + w.at.u * tok);
          T::load(sdO, &maps.d_out, smem_u32(&b_fix), w.at.kvh * G, w.at.row0 + w.at.u * tok);
        }
        __syncwarp();
        ++units;
        for (int j = w.c0(); j < w.c1() && ok; ++j) {
          int place = nk % Lay::KEYS;
          ok = nk < Lay::KEYS || warp_wait(b_kfree[place], nk / Lay::KEYS - 1);
          if (!ok) break;
          if (elect_one()) {
            mbar_arrive_expect_tx(smem_u32(&b_k[place]), T::BYTES);
            T::load(sK + place * Lay::T, &maps.k, smem_u32(&b_k[place]), w.at.kvh, w.at.row0 + j * PT_KEYS);
          }
          __syncwarp();
          ++nk;
          place = nv % Lay::VALUES;
          ok = nv < Lay::VALUES || warp_wait(b_vfree[place], nv / Lay::VALUES - 1);
          if (!ok) break;
          if (elect_one()) {
            mbar_arrive_expect_tx(smem_u32(&b_v[place]), T::BYTES);
            T::load(sV + place * Lay::T, &maps.v, smem_u32(&b_v[place]), w.at.kvh, w.at.row0 + j * PT_KEYS);
          }
          __syncwarp();
          ++nv;
        }
        if (!ok) break;
        go = w.next();
      }
      // every copy has landed before the CTA may leave, also after a wait that gave up
      if (units) warp_wait(b_fix, units - 1);
      for (int i = max(0, nk - Lay::KEYS); i < nk; ++i) warp_wait(b_k[i % Lay::KEYS], i / Lay::KEYS);
      for (int i = max(0, nv - Lay::VALUES); i < nv; ++i) warp_wait(b_v[i % Lay::VALUES], i / Lay::VALUES);
      if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
    } else if (warp < 19) {
      const uint32_t on = elect_one();
      int g = 0, units = 0;  // steps, units so far
      auto place_of = [&](int i, int n) { return __shfl_sync(0xffffffffu, i % n, 0); };
      while (go && warp == 17) {  // S and dP
        ok = warp_wait(b_fix, units++);
        for (int j = w.c0(); j < w.c1() && ok; ++j, ++g) {
          int place = place_of(g, Lay::KEYS);
          ok = (g == 0 || warp_wait(b_sread, g - 1)) && warp_wait(b_k[place], g / Lay::KEYS);
          if (!ok) break;
          tc_fence_after();
          T::dots(tS, sQ, sK + place * Lay::T, on);
          commit_on(smem_u32(&b_s), on);
          // dP: its place is ds's of two steps before, which has been read then
          place = place_of(g, Lay::VALUES);
          ok = warp_wait(b_v[place], g / Lay::VALUES) && (g < 2 || warp_wait(b_o[g & 1], (g >> 1) - 1));
          if (!ok) break;
          tc_fence_after();
          T::dots(tP + (g & 1) * 128, sdO, sV + place * Lay::T, on);
          commit_on(smem_u32(&b_dp[g & 1]), on);
          commit_on(smem_u32(&b_vfree[place]), on);
        }
        commit_on(smem_u32(&b_fixfree), on);
        go = ok && w.next();
      }
      while (go && warp == 18) {  // dQ
        for (int j = w.c0(); j < w.c1() && ok; ++j, ++g) {
          const int place = place_of(g, Lay::KEYS), held = w.at.n - j * PT_KEYS;
          ok = warp_wait(b_ds[g & 1], g >> 1);
          if (!ok) break;
          if (held < PT_KEYS) T::clear_from(sK + place * Lay::T, held, lane);  // (S has read it, and so has the copy)
          tc_fence_after();
          T::template rows<2>(tG, tP + (g & 1) * 128, sK + place * Lay::T, j == w.c0(), on);
          if (two_terms(w.at)) T::template rows<2>(tG, tP + (g & 1) * 128 + 16, sK + place * Lay::T, false, on);
          commit_on(smem_u32(&b_o[g & 1]), on);
          commit_on(smem_u32(&b_kfree[place]), on);
        }
        commit_on(smem_u32(&b_unit), on);
        go = ok && w.next();
      }
      if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_TMA);
      commit_on(smem_u32(&b_all[warp - 17]), on);
      __syncwarp();
      warp_wait(b_all[warp - 17], 0);  // every product is complete before the CTA may leave
    }
  } else {
    clear_rows<HD>(a.t, a.dq, a.ld_dq, a.Hq, tid, 512);
    const int quarter = warp >> 2, r = (warp & 3) * 32 + lane, r_tok = r / G, r_head = r - r_tok * G;
    const uint32_t t_row = (uint32_t)((warp & 3) * 32) << 16;
    const float c = a.scale * kLog2e;
    int g = 0, units = 0;
    // The sum of the four threads of a row, through tensor memory that each has read its part of. All 512 threads meet, and learn
    // whether one's wait gave up: it keeps to the meetings until then, so that nobody waits at one alone.
    auto join = [&](uint32_t columns, int apart, float x) {
      tmem_st1(columns + t_row + quarter * apart, x);
      tmem_wait_st();
      tc_fence_before();
      ok = sync_and<1, 512>(ok);
      tc_fence_after();
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) sum += tmem_ld1(columns + t_row + k * apart);
      return sum;
    };
    while (go) {
      int i = w.at.u * tok + r_tok;
      const bool live = r_tok < tok && i < w.at.n;
      auto place = [&]() { return (long long)(w.at.row0 + i) * a.Hq + w.at.kvh * G + r_head; };
      const float nl = live ? -a.lse[place()] * kLog2e : -INFINITY;
      float delta = live && w.at.n_steps > 1 ? a.delta[place()] : 0.f, eps = 0.f;
      bool left = false;  // (after a meeting that ends the run, there is no other)
      for (int j = w.c0(); j < w.c1() && ok; ++j, ++g) {
        const int see = i - j * PT_KEYS - 32 * quarter;  // columns 0 .. see of the 32
        const bool cut = (j + 1) * PT_KEYS > w.at.u * tok;
        ok = warp_wait(b_s, g);
        if (!ok) break;
        tc_fence_after();
        float p[32];
        tmem_ld32(tS + t_row + 32 * quarter, p);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&b_sread));
#pragma unroll
        for (int x = 0; x < 32; x += 2) {
          const float2 e = fma2(make_float2(p[x], p[x + 1]), make_float2(c, c), make_float2(nl, nl));
          p[x] = packed_ex2(e.x), p[x + 1] = packed_ex2(e.y);
        }
        if (cut) {
#pragma unroll
          for (int x = 0; x < 32; ++x) p[x] = x <= see ? p[x] : 0.f;
        }
        ok = warp_wait(b_dp[g & 1], g >> 1);
        if (!ok) break;
        tc_fence_after();
        const uint32_t t_p = tP + t_row + (g & 1) * 128 + 32 * quarter;
        float v[32];
        uint32_t u[16];
        tmem_ld32(t_p, v);
        if (cut) {  // (what lies behind the text may be anything)
#pragma unroll
          for (int x = 0; x < 32; ++x) v[x] = x <= see ? v[x] : 0.f;
        }
        if (w.at.n_steps == 1) {
          float sum = 0.f;
#pragma unroll
          for (int x = 0; x < 32; ++x) sum = fmaf(p[x], v[x], sum);
          delta = join(tP + (g & 1) * 128 + 31, 32, sum);  // (a column that ds takes, once all have read it)
          if (ok) ok = sync_and<1, 512>(ok);
          left = !ok;
          if (left) break;
        }
        float2 sum = make_float2(0.f, 0.f);
        auto ds = [&](int x) {
          float2 d = add2(make_float2(v[2 * x], v[2 * x + 1]), make_float2(-delta, -delta));
          d.x *= p[2 * x], d.y *= p[2 * x + 1];
          sum = add2(sum, d);
          return d;
        };
        if (two_terms(w.at)) {  // what the first rounding leaves is a second term
          uint32_t rest[16];
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const float2 d = ds(x);
            u[x] = pack_bf16(d.x, d.y);
            rest[x] = pack_bf16(d.x - __uint_as_float(u[x] << 16), d.y - __uint_as_float(u[x] & 0xffff0000u));
          }
          tmem_st16(t_p, u);
          tmem_st16(t_p + 16, rest);
        } else {
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const float2 d = ds(x);
            u[x] = pack_bf16(d.x, d.y);
          }
          tmem_st16(t_p, u);
        }
        eps += sum.x + sum.y;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&b_ds[g & 1]));
      }
      if (left) break;
      asm volatile("" : "+r"(i));  // (the row's places are found again: registers)
      ok = ok && warp_wait(b_unit, units++);
      tc_fence_after();
      const bool whole = w.whole();
      float* st = a.states + (long long)w.slot(blockIdx.x) * BackLayout<HD>::DQ_STATE;
      constexpr int DW = HD / 4;  // dims of a thread
      const int d0 = quarter * DW;
      if (ok) {
        float o[DW];
        if constexpr (DW == 32) tmem_ld32(tG + t_row + d0, o);
        else tmem_ld16(tG + t_row + d0, o);
        if (whole) {
          if (live) {
            bf16* dst = reinterpret_cast<bf16*>(a.dq) + (w.at.row0 + i) * a.ld_dq + (w.at.kvh * G + r_head) * HD + d0;
            if (((uintptr_t)dst & 15) == 0) {
#pragma unroll
              for (int h = 0; h < DW / 8; ++h)
                reinterpret_cast<uint4*>(dst)[h] =
                    make_uint4(pack_bf16(o[8 * h] * a.scale, o[8 * h + 1] * a.scale), pack_bf16(o[8 * h + 2] * a.scale, o[8 * h + 3] * a.scale),
                               pack_bf16(o[8 * h + 4] * a.scale, o[8 * h + 5] * a.scale), pack_bf16(o[8 * h + 6] * a.scale, o[8 * h + 7] * a.scale));
            } else {
#pragma unroll
              for (int h = 0; h < DW; ++h) dst[h] = __float2bfloat16_rn(o[h] * a.scale);
            }
          }
        } else {
#pragma unroll
          for (int h = 0; h < DW / 4; ++h)
            reinterpret_cast<float4*>(st)[(d0 / 4 + h) * 128 + r] = make_float4(o[4 * h], o[4 * h + 1], o[4 * h + 2], o[4 * h + 3]);
        }
      }
      eps = join(tG, DW, eps);  // (dQ has been read; all threads have, after this)
      if (!ok) break;
      if (quarter == 0) {
        if (!whole) st[128 * HD + r] = eps, st[128 * (HD + 1) + r] = delta;
        else if (live) a.delta[place()] = w.at.n_steps == 1 ? delta : delta + eps;
      }
      tc_fence_before();
      ok = sync_and<1, 512>(ok);  // ... and what they exchanged
      if (!ok) break;
      go = w.next();
    }
    if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 16) tmem_dealloc(tmem, 512);
}

struct ByKeys {  // tiles of keys over the tiles of `tok` tokens that see them
  static constexpr bool KEYS = true;
  static constexpr int UC = 3;
  int tok;
  JF_DEV int units(int n) const { return (n + PT_KEYS - 1) / PT_KEYS; }
  JF_DEV int first(int u) const { return u * PT_KEYS / tok; }
  JF_DEV int steps(int n, int u) const { return (n + tok - 1) / tok - first(u); }
};

// dk and dv. Rows of the products are keys, columns query rows. Tensor memory: S (P in bf16 in its place), dP (ds), dV, dK. All of it, so
// that a step's S waits until dV has read P of the step before: 704 us at 8,192 rows (four products, 1.37 PFLOP/s), tensor pipe 61%.
//
// Q and d_out come through a ring of four places in pairs. d_out's place is free first and takes the Q of two steps on, Q's place its
// d_out.
JF_DEV int place_q(int j) { return 2 * (j & 1) + (j >> 1 & 1); }
JF_DEV int place_do(int j) { return 2 * (j & 1) + (~j >> 1 & 1); }

template <int HD>
__global__ void __launch_bounds__(PT_THREADS, 1) k_packed_dkv_tc(const PackedParams a, const __grid_constant__ BackMaps maps) {
  using Lay = BackLayout<HD>;
  using T = Tile<HD>;
  extern __shared__ uint8_t sm_raw[];
  uint8_t* smp = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(sm_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sK = smem_u32(smp), sV = sK + Lay::T, ring = sK + Lay::OFF_RING;
  // keys and values there, read; the ring's places there (b_raw: with rows to be cleared), read; S, dP, P, ds ready; dV, dK of a step done; everything done;
  // statistics there, read
  __shared__ __align__(8) uint64_t b_fix, b_fixfree, b_tile[4], b_raw[4], b_free[4], b_s, b_dp, b_p, b_ds, b_o1, b_o2, b_all[2], b_stat[2], b_statfree[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int s_bad;
  __shared__ Cut s_cut[2];
  __shared__ __align__(16) float s_nl[2][128], s_nd[2][128];  // of a step's columns: -lse log2 e, -delta
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int G = a.Hq / a.Hkv, tok = 128 / G;
  if (tid == 0) {
    uint64_t* const ones[] = {&b_fix, &b_fixfree, &b_s, &b_dp, &b_o1, &b_o2, &b_all[0], &b_all[1], &b_stat[0], &b_stat[1]};
    for (uint64_t* b : ones) mbar_init(smem_u32(b), 1);
    for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&b_tile[i]), 1), mbar_init(smem_u32(&b_raw[i]), 1), mbar_init(smem_u32(&b_free[i]), 1);
    uint64_t* const all[] = {&b_p, &b_ds, &b_statfree[0], &b_statfree[1]};
    for (uint64_t* b : all) mbar_init(smem_u32(b), 16);
    fence_mbar_init();
  }
  if (warp == 19 && tok * G < 128)
    for (int i = 0; i < 4; ++i) T::clear_from(ring + i * Lay::T, tok * G, lane);  // rows that no copy writes
  Run<ByKeys> w = {{{tok}, a.t, a.Hkv, 0, nullptr}, {}, &s_cut[1]};
  bool go, ok = true;
  if (!back_begin(w, a, smp, &s_bad, s_cut, &tmem_slot, go)) return;
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0), tS = tmem, tP = tmem + 128, tV = tmem + 256, tK = tmem + 384;

  if (warp >= 16) {
    if (warp == 16) {
      int units = 0, g = 0, asked = 0;  // of the ring's places
      const uint32_t tile_bytes = (uint32_t)(tok * G * HD * 2);
      while (go) {
        ok = units == 0 || warp_wait(b_fixfree, units - 1);
        if (!ok) break;
        if (elect_one()) {
          mbar_arrive_expect_tx(smem_u32(&b_fix), (uint32_t)(2 * T::BYTES));
          T::load(sK, &maps.k, smem_u32(&b_fix), w.at.kvh, w.at.row0 + w.at.u * PT_KEYS);
          T::load(sV, &maps.v, smem_u32(&b_fix), w.at.kvh, w.at.row0 + w.at.u * PT_KEYS);
        }
        __syncwarp();
        ++units;
        for (int j = w.c0(); j < w.c1() && ok; ++j, ++g)
          for (int y = 0; y < 2 && ok; ++y) {
            const int place = y ? place_do(g) : place_q(g);
            ok = g < 2 || warp_wait(b_free[place], (g >> 1) - 1);
            if (!ok) break;
            const int first = (w.line.kind.first(w.at.u) + j) * tok;  // the tile's first token
            if (elect_one()) {
              const uint32_t bar = smem_u32(first + tok > w.at.n ? &b_raw[place] : &b_tile[place]);
              mbar_arrive_expect_tx(bar, tile_bytes);
              T::load(ring + place * Lay::T, y ? &maps.d_out : &maps.q, bar, w.at.kvh * G, w.at.row0 + first);
            }
            __syncwarp();
            ++asked;
          }
        if (!ok) break;
        go = w.next();
      }
      // every copy has landed before the CTA may leave, also after a wait that gave up (b_raw's are forwarded)
      if (units) warp_wait(b_fix, units - 1);
      for (int i = max(0, asked - 4); i < asked; ++i) warp_wait(b_tile[i & 1 ? place_do(i >> 1) : place_q(i >> 1)], i >> 2);
      if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
    } else if (warp < 19) {
      const uint32_t on = elect_one();
      int g = 0, units = 0;
      auto of = [&](int place) { return __shfl_sync(0xffffffffu, place, 0); };
      while (go && warp == 17) {  // S and dP: their places are P's and ds's of the step before, which have been read then
        ok = warp_wait(b_fix, units++);
        for (int j = w.c0(); j < w.c1() && ok; ++j, ++g) {
          const int pq = of(place_q(g)), po = of(place_do(g));
          ok = warp_wait(b_tile[pq], g >> 1) && (g == 0 || warp_wait(b_o1, g - 1));
          if (!ok) break;
          tc_fence_after();
          T::dots(tS, sK, ring + pq * Lay::T, on);
          commit_on(smem_u32(&b_s), on);
          ok = warp_wait(b_tile[po], g >> 1) && (g == 0 || warp_wait(b_o2, g - 1));
          if (!ok) break;
          tc_fence_after();
          T::dots(tP, sV, ring + po * Lay::T, on);
          commit_on(smem_u32(&b_dp), on);
        }
        commit_on(smem_u32(&b_fixfree), on);
        go = ok && w.next();
      }
      while (go && warp == 18) {  // dV and dK
        for (int j = w.c0(); j < w.c1() && ok; ++j, ++g) {
          const int pq = of(place_q(g)), po = of(place_do(g));
          ok = warp_wait(b_tile[po], g >> 1) && warp_wait(b_p, g);
          if (!ok) break;
          tc_fence_after();
          T::template rows<2>(tV, tS, ring + po * Lay::T, j == w.c0(), on);
          commit_on(smem_u32(&b_o1), on);
          ok = warp_wait(b_ds, g);
          if (!ok) break;
          commit_on(smem_u32(&b_free[po]), on);  // (dP, which has read it too, is done)
          tc_fence_after();
          T::template rows<2>(tK, tP, ring + pq * Lay::T, j == w.c0(), on);
          commit_on(smem_u32(&b_o2), on);
          commit_on(smem_u32(&b_free[pq]), on);
        }
        go = ok && w.next();
      }
      if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_TMA);
      commit_on(smem_u32(&b_all[warp - 17]), on);
      __syncwarp();
      warp_wait(b_all[warp - 17], 0);  // every product is complete before the CTA may leave
    } else {
      int g = 0;
      unsigned uses = 0;  // of each place's b_raw, their parities
      while (go) {
        for (int j = w.c0(); j < w.c1() && ok; ++j, ++g) {
          const int q = w.line.kind.first(w.at.u) + j;
          float nl[4], nd[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int col = lane + 32 * x, t = col / G, i = q * tok + t;
            const bool live = t < tok && i < w.at.n;
            const long long at = (long long)(w.at.row0 + i) * a.Hq + w.at.kvh * G + (col - t * G);
            nl[x] = live ? -a.lse[at] * kLog2e : -INFINITY;  // (p = 0)
            nd[x] = live ? -a.delta[at] : 0.f;
          }
          ok = g < 2 || warp_wait(b_statfree[g & 1], (g >> 1) - 1);
          if (!ok) break;
#pragma unroll
          for (int x = 0; x < 4; ++x) s_nl[g & 1][lane + 32 * x] = nl[x], s_nd[g & 1][lane + 32 * x] = nd[x];
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&b_stat[g & 1]));
          const int held = (w.at.n - q * tok) * G;
          if (held < tok * G) {  // rows behind the text: cleared before the products see them
            for (int y = 0; y < 2 && ok; ++y) {
              const int place = y ? place_do(g) : place_q(g);
              ok = warp_wait(b_raw[place], (int)(uses >> place & 1u));
              uses ^= 1u << place;
              if (!ok) break;
              T::clear_from(ring + place * Lay::T, held, lane);
              if (lane == 0) mbar_arrive(smem_u32(&b_tile[place]));
            }
          }
        }
        go = ok && w.next();
      }
      if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
    }
  } else {
    clear_rows<HD>(a.t, a.dk, a.ld_dk, a.Hkv, tid, 512);
    clear_rows<HD>(a.t, a.dv, a.ld_dv, a.Hkv, tid, 512);
    const int quarter = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t t_row = (uint32_t)((warp & 3) * 32) << 16, t_s = tS + t_row + 32 * quarter, t_p = tP + t_row + 32 * quarter;
    const float c = a.scale * kLog2e;
    int g = 0;
    while (go) {
      const int k = w.at.u * PT_KEYS + r, q0 = w.line.kind.first(w.at.u);
      for (int j = w.c0(); j < w.c1() && ok; ++j, ++g) {
        const int first = (k - (q0 + j) * tok) * G - 32 * quarter;  // columns from here on see the key
        const bool cut = (q0 + j) * tok < w.at.u * PT_KEYS + PT_KEYS - 1;
        ok = warp_wait(b_stat[g & 1], g >> 1) && warp_wait(b_s, g);
        if (!ok) break;
        tc_fence_after();
        float p[32];
        uint32_t u[16];
        tmem_ld32(t_s, p);
        const float4* nl = reinterpret_cast<const float4*>(s_nl[g & 1] + 32 * quarter);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const float4 l = nl[x];
          const float2 e = fma2(make_float2(p[4 * x], p[4 * x + 1]), make_float2(c, c), make_float2(l.x, l.y));
          const float2 f = fma2(make_float2(p[4 * x + 2], p[4 * x + 3]), make_float2(c, c), make_float2(l.z, l.w));
          p[4 * x] = packed_ex2(e.x), p[4 * x + 1] = packed_ex2(e.y), p[4 * x + 2] = packed_ex2(f.x), p[4 * x + 3] = packed_ex2(f.y);
        }
        if (cut) {
#pragma unroll
          for (int x = 0; x < 32; ++x) p[x] = x >= first ? p[x] : 0.f;
        }
#pragma unroll
        for (int x = 0; x < 16; ++x) u[x] = pack_bf16(p[2 * x], p[2 * x + 1]);
        tmem_st16(t_s, u);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&b_p));
        ok = warp_wait(b_dp, g);
        if (!ok) break;
        tc_fence_after();
        float v[32];
        tmem_ld32(t_p, v);
        const float4* nd = reinterpret_cast<const float4*>(s_nd[g & 1] + 32 * quarter);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const float4 d = nd[x];
          const float2 e = add2(make_float2(v[4 * x], v[4 * x + 1]), make_float2(d.x, d.y));
          const float2 f = add2(make_float2(v[4 * x + 2], v[4 * x + 3]), make_float2(d.z, d.w));
          u[2 * x] = pack_bf16(p[4 * x] * e.x, p[4 * x + 1] * e.y);
          u[2 * x + 1] = pack_bf16(p[4 * x + 2] * f.x, p[4 * x + 3] * f.y);
        }
        tmem_st16(t_p, u);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(&b_ds));
          mbar_arrive(smem_u32(&b_statfree[g & 1]));
        }
      }
      ok = ok && warp_wait(b_o1, g - 1) && warp_wait(b_o2, g - 1);
      tc_fence_after();
      // the first eight warps take dV, the others dK, half of the dims each
      const bool whole = w.whole(), live = k < w.at.n, is_k = quarter >= 2;
      const float f = is_k ? a.scale : 1.f;
      const int d0 = (quarter & 1) * (HD / 2);
      float* st = a.states + (long long)w.slot(blockIdx.x) * Lay::DKV_STATE + (is_k ? 128 * HD : 0);
      bf16* dst = is_k ? reinterpret_cast<bf16*>(a.dk) + (w.at.row0 + k) * a.ld_dk : reinterpret_cast<bf16*>(a.dv) + (w.at.row0 + k) * a.ld_dv;
      dst += w.at.kvh * HD;
#pragma unroll 1
      for (int d = d0; d < d0 + HD / 2 && ok; d += 32) {
        float o[32];
        tmem_ld32((is_k ? tK : tV) + t_row + d, o);
        if (whole) {
          if (live) {
            if (((uintptr_t)dst & 15) == 0) {
#pragma unroll
              for (int h = 0; h < 4; ++h)
                reinterpret_cast<uint4*>(dst + d)[h] = make_uint4(pack_bf16(o[8 * h] * f, o[8 * h + 1] * f), pack_bf16(o[8 * h + 2] * f, o[8 * h + 3] * f),
                                                                  pack_bf16(o[8 * h + 4] * f, o[8 * h + 5] * f), pack_bf16(o[8 * h + 6] * f, o[8 * h + 7] * f));
            } else {
#pragma unroll
              for (int h = 0; h < 32; ++h) dst[d + h] = __float2bfloat16_rn(o[h] * f);
            }
          }
        } else {
#pragma unroll
          for (int h = 0; h < 8; ++h)
            reinterpret_cast<float4*>(st)[(d / 4 + h) * 128 + r] = make_float4(o[4 * h], o[4 * h + 1], o[4 * h + 2], o[4 * h + 3]);
        }
      }
      tc_fence_before();
      // dV and dK have been read before any warp lets the next unit's products begin. (All 512 threads meet here, and learn whether
      // one's wait gave up.)
      ok = sync_and<1, 512>(ok);
      if (!ok) break;
      go = w.next();
    }
    if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 16) tmem_dealloc(tmem, 512);
}

// Adds up the parts of a unit that several CTAs share, in their order: CTA (run i + 1, 8 pieces of 4 columns of the 128 rows). Kind
// ByDq: dq and delta; ByKeys: dv and dk. Bound by the latency of its loads: 10 and 13 us at 8,192 rows from a cold L2.
template <int HD, typename Kind>
__global__ void __launch_bounds__(256) k_packed_back_join(const PackedParams a) {
  constexpr bool KEYS = Kind::KEYS;
  constexpr int STATE = KEYS ? BackLayout<HD>::DKV_STATE : BackLayout<HD>::DQ_STATE, X = 4;
  const int G = a.Hq / a.Hkv, tok = 128 / G, i = blockIdx.x + 1;
  pdl_launch_dependents();
  pdl_wait();
  Cut c;
  int last;
  if (!parts_from(a.cuts, gridDim.x + 1, a.t.n_seqs, i, c, last)) return;
  const int r = threadIdx.x & 127, x0 = X * (2 * blockIdx.y + (threadIdx.x >> 7)), r_tok = r / G;
  const int index = KEYS ? c.u * PT_KEYS + r : c.u * tok + r_tok;
  if (index >= c.n || (!KEYS && r_tok >= tok)) return;
  const long long row = c.row0 + index;
  auto part = [&](int k) { return a.states + (long long)(2 * k + (k == i - 1 ? 1 : 0)) * STATE; };
  float4 o[X];
#pragma unroll
  for (int x = 0; x < X; ++x) o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
  for (int k = i - 1; k <= last; ++k)
#pragma unroll
    for (int x = 0; x < X; ++x) {
      const float4 v = reinterpret_cast<const float4*>(part(k))[(x0 + x) * 128 + r];
      o[x].x += v.x, o[x].y += v.y, o[x].z += v.z, o[x].w += v.w;
    }
  bf16* dst;
  float f = a.scale;
  if (!KEYS) {
    dst = reinterpret_cast<bf16*>(a.dq) + row * a.ld_dq + (c.kvh * G + r - r_tok * G) * HD + 4 * x0;
  } else if (x0 < HD / 4) {
    dst = reinterpret_cast<bf16*>(a.dv) + row * a.ld_dv + c.kvh * HD + 4 * x0;
    f = 1.f;
  } else {
    dst = reinterpret_cast<bf16*>(a.dk) + row * a.ld_dk + c.kvh * HD + 4 * x0 - HD;
  }
  if (((uintptr_t)dst & 15) == 0) {
#pragma unroll
    for (int x = 0; x < X; x += 2)
      reinterpret_cast<uint4*>(dst)[x / 2] = make_uint4(pack_bf16(o[x].x * f, o[x].y * f), pack_bf16(o[x].z * f, o[x].w * f),
                                                        pack_bf16(o[x + 1].x * f, o[x + 1].y * f), pack_bf16(o[x + 1].z * f, o[x + 1].w * f));
  } else {
#pragma unroll
    for (int x = 0; x < X; ++x) {
      dst[4 * x] = __float2bfloat16_rn(o[x].x * f), dst[4 * x + 1] = __float2bfloat16_rn(o[x].y * f);
      dst[4 * x + 2] = __float2bfloat16_rn(o[x].z * f), dst[4 * x + 3] = __float2bfloat16_rn(o[x].w * f);
    }
  }
  if (!KEYS && x0 == 0) {
    float eps = 0.f;
    for (int k = i - 1; k <= last; ++k) eps += part(k)[128 * HD + r];
    a.delta[row * a.Hq + c.kvh * G + r - r_tok * G] = part(i - 1)[128 * (HD + 1) + r] + eps;
  }
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
  cudaError_t e = cudaFuncSetAttribute(k_packed_attn_tc<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdLayout<HD>::TOTAL);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k_packed_dq_tc<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, DqLayout<HD>::TOTAL);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k_packed_dkv_tc<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, BackLayout<HD>::TOTAL);
  return e;
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

// Whether units can be cut, tile: rows of a step.
bool tc_cuts(const jf_packed& t, int tile) { return t.max_rows > PT_WHOLE * tile; }

template <int HD>
jf_status tc_forward(const PackedParams& a, int sms, cudaStream_t st) {
  FwdMaps maps;
  const int G = a.Hq / a.Hkv, tok = 128 / G;
  if (!tc_map(&maps.q, a.q, a.ld_q, a.Hq, HD, a.t.n_rows, G, tok) || !tc_map(&maps.k, a.k, a.ld_k, a.Hkv, HD, a.t.n_rows, 1, 128) ||
      !tc_map(&maps.v, a.v, a.ld_v, a.Hkv, HD, a.t.n_rows, 1, 128))
    return JF_ECUDA;
  cudaError_t e = packed_launch(k_packed_attn_tc<HD>, dim3(sms), dim3(PA_THREADS), FwdLayout<HD>::TOTAL, st, a, maps);
  if (e == cudaSuccess && tc_cuts(a.t, PT_KEYS)) e = packed_launch(k_packed_attn_join<HD>, dim3(sms - 1, 8), dim3(256), 0, st, a);
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}

template <int HD>
jf_status tc_backward(const PackedParams& a, int sms, cudaStream_t st) {
  BackMaps maps;
  const int G = a.Hq / a.Hkv, tok = 128 / G;
  if (!tc_map(&maps.q, a.q, a.ld_q, a.Hq, HD, a.t.n_rows, G, tok) || !tc_map(&maps.d_out, a.d_out, a.ld_do, a.Hq, HD, a.t.n_rows, G, tok) ||
      !tc_map(&maps.k, a.k, a.ld_k, a.Hkv, HD, a.t.n_rows, 1, 128) || !tc_map(&maps.v, a.v, a.ld_v, a.Hkv, HD, a.t.n_rows, 1, 128))
    return JF_ECUDA;
  cudaError_t e = cudaSuccess;
  if (a.t.max_rows > PT_KEYS)  // (delta is read where a row has several steps)
    e = packed_launch(k_packed_delta_tc<HD>, dim3((unsigned)(((long long)a.t.n_rows * a.Hq * (HD / 8) + 255) / 256)), dim3(256), 0, st, a);
  if (e == cudaSuccess) e = packed_launch(k_packed_dq_tc<HD>, dim3(sms), dim3(PT_THREADS), DqLayout<HD>::TOTAL, st, a, maps);
  if (e == cudaSuccess && tc_cuts(a.t, PT_KEYS)) e = packed_launch(k_packed_back_join<HD, ByDq>, dim3(sms - 1, HD / 32), dim3(256), 0, st, a);
  if (e == cudaSuccess) e = packed_launch(k_packed_dkv_tc<HD>, dim3(sms), dim3(PT_THREADS), BackLayout<HD>::TOTAL, st, a, maps);
  if (e == cudaSuccess && tc_cuts(a.t, tok)) e = packed_launch(k_packed_back_join<HD, ByKeys>, dim3(sms - 1, HD / 16), dim3(256), 0, st, a);
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}

}  // namespace

bool packed_tc_rows(const void* p, long long ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

// The workspace of cuts and parts.
static void tc_parts(PackedParams& a, void* at, int sms) {
  a.cuts = reinterpret_cast<int*>(at);
  a.states = reinterpret_cast<float*>(reinterpret_cast<char*>(at) + (size_t)sms * 32);
}

// Backward: delta (read by the copies' form and by the other one), then the parts.
static size_t delta_bytes(const jf_packed& t, int Hq) { return ((size_t)t.n_rows * Hq * 4 + 15) / 16 * 16; }

jf_status packed_tc_workspace(const jf_packed& t, int Hq, int Hkv, int hd, bool backward, size_t* out_bytes) {
  const PackedDevice* d = tc_device();
  if (!d) return JF_ECUDA;
  const size_t parts = (size_t)2 * d->sms * 4, cuts = (size_t)d->sms * 32;
  if (!backward) {
    *out_bytes = tc_cuts(t, PT_KEYS) ? cuts + parts * (hd == 128 ? FwdLayout<128>::STATE : FwdLayout<64>::STATE) : 0;
  } else {
    *out_bytes = delta_bytes(t, Hq);
    if (tc_cuts(t, 128 / (Hq / Hkv))) *out_bytes += cuts + parts * (hd == 128 ? BackLayout<128>::DKV_STATE : BackLayout<64>::DKV_STATE);
  }
  return JF_OK;
}

jf_status packed_tc_forward(const PackedParams& p, int hd, void* workspace, cudaStream_t st) {
  const PackedDevice* d = tc_device();
  if (!d) return JF_ECUDA;
  PackedParams a = p;
  if (tc_cuts(a.t, PT_KEYS)) tc_parts(a, workspace, d->sms);
  return hd == 128 ? tc_forward<128>(a, d->sms, st) : tc_forward<64>(a, d->sms, st);
}

jf_status packed_tc_backward(const PackedParams& p, int hd, void* workspace, cudaStream_t st) {
  const PackedDevice* d = tc_device();
  if (!d) return JF_ECUDA;
  PackedParams a = p;
  a.delta = reinterpret_cast<float*>(workspace);
  if (tc_cuts(a.t, 128 / (a.Hq / a.Hkv))) tc_parts(a, reinterpret_cast<char*>(workspace) + delta_bytes(a.t, a.Hq), d->sms);
  return hd == 128 ? tc_backward<128>(a, d->sms, st) : tc_backward<64>(a, d->sms, st);
}

}  // namespace jf
