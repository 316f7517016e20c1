// Attention of a batch's new rows over the 8-bit paged cache (jf_ops.h: jf_op_kv8_attention).
//
// With q scaled by a power of two per row so that its largest magnitude lies in [2^14, 2^15), codes c_k, c_v and
// block exponents e_k, e_v, a key's score in the log2 domain is s = (q . c_k) 2^(e_k) f, f the row's factor (the
// scaling undone, the softmax scale, log2 e), and
//   out = sum_j 2^(s_j - m) 2^(e_v_j) c_v_j / sum_j 2^(s_j - m).
// Codes are exact in fp16, so both products run on fp16 operands with fp32 sums. The values' exponents go into
// the probabilities: p' = 2^(s - m) 2^(e_v - E) in fp16, against a running reference E of each row in whose unit its
// output accumulates; E follows e_v only when the difference leaves a range in which fp16 keeps p' as well as it keeps
// p, and only as far as the row's weights and what it has summed allow (unit_down, unit_up).
//
// Work is split evenly whatever the batch: a unit is (sequence, KV head, tile of (token, head) query rows), a
// chunk a run of keys of one unit. Units lie one after the other, each as long as its chunks plus a constant for
// what a unit costs beside them (its queries, its end), and each of N workers takes an N'th of that length. A unit
// whose chunks one worker holds entirely is finished there; of the others each worker leaves a partial state (m, l,
// O) in the workspace, at most two a worker, and k_kv8_combine joins a row's states in their order.
#include <type_traits>

#include "../../include/jf_ops.h"
#include "jf_kv8.cuh"
#include "jf_once.h"

namespace jf {
namespace {

struct Kv8AttnParams {
  jf_kv8_cache c;
  jf_kv8_rows r;
  const void* q;
  long long ld_q;
  int n_heads;
  float scale_log2;  // softmax scale * log2 e
  const uint32_t* mask;
  int mask_words;
  void* out;
  float* lse;
  int* plan;         // [n_seqs + 1]: length of the sequences before b (of more than 32)
  float* states;     // [2 N][tile rows x hd normalised O, then m, then l of the tile's rows]
  int* err;
};

// 2^x by the MUFU ex2 instruction (flushes results below 2^-126 to zero; 2^-inf = 0).
JF_DEV float ex2_ftz(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
JF_DEV uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
JF_DEV float2 unpack_f16(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

// ---------------------------------------------------------------------------------------------
// The plan: which units there are. TR: query rows of a tile, CH: keys of a chunk, UC: what a unit costs beside its
// chunks, in chunks.
// ---------------------------------------------------------------------------------------------
template <int TR, int CH, int UC>
struct Plan {
  // Chunks of one tile of a sequence's rows.
  static JF_DEV int chunks(const Kv8AttnParams& a, const Kv8Seq& s, int G, int tile) {
    const int last = a.mask ? s.n - 1 : min(s.n - 1, ((tile + 1) * TR - 1) / G);  // a masked row may see any new row
    return (s.len + last + CH) / CH;
  }
  static JF_DEV int tiles(const Kv8Seq& s, int G) { return (s.n * G + TR - 1) / TR; }
  // Length of a sequence's units, per KV head.
  static JF_DEV int per_head(const Kv8AttnParams& a, const Kv8Seq& s, int G) {
    const int n = tiles(s, G);
    if (a.mask) return n > 0 ? n * (UC + chunks(a, s, G, 0)) : 0;
    int sum = 0;
    for (int t = 0; t < n; ++t) sum += UC + chunks(a, s, G, t);
    return sum;
  }
  // Up to 32 sequences: a warp finds out by itself, lane b for sequence b, and nothing is read twice or passed on. Returns
  // the batch's length.
  struct Few {
    Kv8Seq s;
    int before, length;  // of the sequences before b, of b
  };
  static JF_DEV int build_few(const Kv8AttnParams& a, int G, int lane, Few& f) {
    f.s = {0, 0, 0};
    f.length = 0;
    if (lane < a.c.n_seqs) {
      f.s = kv8_seq(a.c, a.r, lane, a.err);
      f.length = per_head(a, f.s, G) * a.c.n_kv_heads;
    }
    int sum = f.length;
#pragma unroll
    for (int sh = 1; sh < 32; sh <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, sum, sh);
      if (lane >= sh) sum += u;
    }
    f.before = sum - f.length;
    return __shfl_sync(0xffffffffu, sum, 31);
  }
  // pre[b] = length of the sequences before b, pre[n_seqs] = of all (returned); by the whole CTA. The first CTA leaves it for
  // the combine.
  static JF_DEV int build(const Kv8AttnParams& a, int G, int* pre) {
    for (int b = threadIdx.x; b < a.c.n_seqs; b += blockDim.x)
      pre[b + 1] = per_head(a, kv8_seq(a.c, a.r, b, a.err), G) * a.c.n_kv_heads;
    __syncthreads();
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x;
      int base = 0;
      if (lane == 0) pre[0] = 0;
      for (int b0 = 0; b0 < a.c.n_seqs; b0 += 32) {
        const int b = b0 + lane;
        int v = b < a.c.n_seqs ? pre[b + 1] : 0;
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, v, sh);
          if (lane >= sh) v += u;
        }
        if (b < a.c.n_seqs) pre[b + 1] = base + v;
        base += __shfl_sync(0xffffffffu, v, 31);
      }
    }
    __syncthreads();
    if (blockIdx.x == 0)
      for (int b = threadIdx.x; b <= a.c.n_seqs; b += blockDim.x) a.plan[b] = pre[b];
    return pre[a.c.n_seqs];
  }
};

// The batch's length in n shares, the first `more` of them one longer.
struct Shares {
  int each, more;
  JF_DEV Shares(int total, int n) : each(total / n), more(total - total / n * n) {}
  JF_DEV int begin(int i) const { return i * each + min(i, more); }
  JF_DEV int size(int i) const { return each + (i < more ? 1 : 0); }
  // The worker that holds place x.
  JF_DEV int of(int x) const {
    const int cut = more * (each + 1);
    return x < cut ? x / (each + 1) : more + (x - cut) / each;
  }
  // Where worker i leaves its part of a unit whose chunks begin at place `first`: it has at most one unit whose first
  // chunk lies before its share, and one that goes on after it.
  JF_DEV int slot(int first, int i) const { return 2 * i + (begin(i) > first ? 0 : 1); }
};

// A worker's walk over the units of its share. Uniform over the worker's threads.
template <int TR, int CH, int UC>
struct Walk {
  using P = Plan<TR, CH, UC>;
  int at, end, first;  // places: the next one, the end of the share, the unit's first chunk
  int b, kvh, tile, n_chunks;
  Kv8Seq s;

  JF_DEV void start(const Kv8AttnParams& a, const int* pre, int G, int at_, int end_) {
    at = at_;
    end = end_;
    int lo = 0, hi = a.c.n_seqs;  // the last b with pre[b] <= at (then pre[b + 1] > at)
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (pre[mid] <= at) lo = mid;
      else hi = mid;
    }
    b = lo;
    s = kv8_seq(a.c, a.r, b, a.err);
    enter(a, G, at - pre[b], pre[b + 1] - pre[b]);
  }
  JF_DEV void start_few(const Kv8AttnParams& a, const typename P::Few& f, int G, int at_, int end_) {
    at = at_;
    end = end_;
    b = 31 - __clz(__ballot_sync(0xffffffffu, f.before <= at));  // (lanes without a sequence: before = all)
    s = {__shfl_sync(0xffffffffu, f.s.n, b), __shfl_sync(0xffffffffu, f.s.row0, b), __shfl_sync(0xffffffffu, f.s.len, b)};
    enter(a, G, at - __shfl_sync(0xffffffffu, f.before, b), __shfl_sync(0xffffffffu, f.length, b));
  }
  // At place `off` of sequence b, which is `length` long.
  JF_DEV void enter(const Kv8AttnParams& a, int G, int off, int length) {
    const int head = length / a.c.n_kv_heads;
    kvh = off / head;
    int rest = off - kvh * head;
    tile = 0;
    while (rest >= UC + (n_chunks = P::chunks(a, s, G, tile))) {
      rest -= UC + n_chunks;
      ++tile;
    }
    first = at - rest + UC;
  }
  // The share's chunks of the unit: [c0, c1), none when it holds the unit's constant alone.
  JF_DEV int c0() const { return max(0, at - first); }
  JF_DEV int c1() const { return min(n_chunks, end - first); }
  // To the unit that begins where this one ends; false at the end of the share.
  JF_DEV bool next(const Kv8AttnParams& a, int G) {
    at = first + n_chunks;
    if (at >= end) return false;
    first = at + UC;
    if (++tile == P::tiles(s, G)) {
      tile = 0;
      if (++kvh == a.c.n_kv_heads) {
        kvh = 0;
        do s = kv8_seq(a.c, a.r, ++b, a.err);
        while (s.n == 0);
      }
    }
    n_chunks = P::chunks(a, s, G, tile);
    return true;
  }
};

// Whether new row i of the sequence sees slot kp (>= len). (A sequence may have more rows than a mask row has bits: the host
// sees only what max_rows says.)
JF_DEV bool sees_new(const Kv8AttnParams& a, const Kv8Seq& s, int i, int kp) {
  const int j = kp - s.len;
  if (!a.mask) return j <= i;
  return j < s.n && j >> 5 < a.mask_words && (a.mask[(long long)(s.row0 + i) * a.mask_words + (j >> 5)] >> (j & 31) & 1u);
}

// N consecutive values as fp32 (zeros unless live); by 16-byte loads where the caller's rows allow it.
template <int N>
JF_DEV void load_run(const float* p, bool live, bool by16, float (&x)[N]) {
  if (by16 && live) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p + i);
      x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = live ? p[i] : 0.f;
  }
}
template <int N>
JF_DEV void load_run(const bf16* p, bool live, bool by16, float (&x)[N]) {
  if (by16 && live) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
      const uint4 v = *reinterpret_cast<const uint4*>(p + i);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i + 2 * j] = __uint_as_float(w[j] << 16);
        x[i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = live ? __bfloat162float(p[i]) : 0.f;
  }
}

JF_DEV void store2(float* p, float x, float y) { *reinterpret_cast<float2*>(p) = make_float2(x, y); }
JF_DEV void store2(bf16* p, float x, float y) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(x, y); }

// Power of two that brings a row's largest magnitude into [2^14, 2^15), as an exponent (0 for a row of zeros or
// one that holds an infinity).
JF_DEV int query_shift(float amax) {
  const int x = __float_as_int(amax) >> 23;
  return x == 0 || x == 255 ? (x == 0 && amax > 0.f ? 126 : 0) : min(14 - (x - 127), 126);
}

// The exponent E in whose unit a row's output goes on accumulating when values come that would best be added at R.
// Smaller ones lower it, as far as what is summed (most: its largest magnitude) stays below 2^126; what is added beside it
// afterwards is below 2^54 (2^30 keys, probabilities of 2^15, codes of 2^9). A block of zeros, at the format's smallest
// exponent, is such a case.
JF_DEV int unit_down(int E, int R, float most) {
  return R < E ? min(E, max(R, E - (252 - (__float_as_int(most) >> 23)))) : E;
}
// Larger ones raise it, less far where the row gives them little weight: s is its largest score among them (-inf: it sees
// none, and they leave it as it is), m its reference maximum, and at s = m - x they need R - x only (and R - 122 where the
// probabilities' factor 2^(e_v - E) has to remain a number).
JF_DEV int unit_up(int E, int R, float s, float m) {
  return R > E && s > -INFINITY ? max(max(E, R - (int)fminf(fmaxf(m - s, 0.f), 1000.f)), max(R - 122, -126)) : E;
}
// 2^e as two factors, each a number (what lies beyond them is out of fp32's range in any case).
JF_DEV float2 pow2_pair(int e) {
  const int x = max(-126, min(126, e));
  return make_float2(pow2i(x), pow2i(max(-126, min(126, e - x))));
}

// ---------------------------------------------------------------------------------------------
// Few query rows per KV head (single-token serving; fp32 at any row count): warp-level products.
//
// A worker is one warp, with a tile of 16 query rows and a chunk of two pages (32 keys) a step. It streams its pages
// through a ring of its own in shared memory (cp.async, 16-byte pieces swizzled so that both fragment loads are free
// of bank conflicts), so no barrier stands anywhere between loads, products and the end of a unit, and the cost of
// a unit's ends is hidden by the other warps of the SM.
//
// m16n8k16 fragments, lane = 4 g + t. S = Q K^T contracts over dims, whose order is free as long as Q's follows
// it: lane t's four values of each k-step are four consecutive dims (one 32-bit word of codes) of the 16-byte
// pieces PK t .. PK t + PK - 1 of keys g and g + 8. O = P V: lane (g, t) holds keys 2t, 2t + 1, 2t + 8, 2t + 9 of P
// as it held their scores, and needs these keys' codes at dims NT g + j, j = 0 .. NT - 1, of the n-tiles j.
// NS: fp16 terms of queries and probabilities (1 for bf16 models, 2 for fp32).
//
// Bound by the codes' bytes where there are many: 16 sequences of one token, 28 query heads on 4 KV heads of 128, over
// 301 to 32,768 tokens each (231 MB of codes) take 47 us with the join, 4.9 TB/s,
// with 37% of the issue slots and 31% of the warp-level tensor rate taken by fragments that hold 7 rows of 16.
// One sequence over 1,024 tokens takes 9.7 us, the length of the chain lengths -> page table -> codes -> scores -> sums
// -> join.
// ---------------------------------------------------------------------------------------------
constexpr int W_WARPS = 4, W_TR = 16, W_CH = 2 * kPage, W_UC = 3;
constexpr int W_STAGES = 2;  // chunks in a warp's ring
constexpr float W_LAG = 8.f;             // a row's reference maximum follows its scores when they exceed it by more
constexpr int W_EV_SET = 4, W_EV_MAX = 7;  // e_v - E: where E is set, largest (p' <= 2^15); smallest 0

template <int HD>
constexpr int w_smem() { return W_WARPS * W_STAGES * 2 * W_CH * HD; }

JF_DEV void cp_async16_zfill(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}

// Byte offset of 16-byte piece c of row r of a page in a warp's ring.
template <int HD>
JF_DEV int w_piece(int r, int c) {
  return HD == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ (r >> 1 & 3)) << 4);
}

JF_DEV void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <typename T, int HD, int NS>
__global__ void __launch_bounds__(32 * W_WARPS, 2) k_kv8_attn_rows(const Kv8AttnParams a) {
  constexpr int KS = HD / 16;   // k-steps of S
  constexpr int NT = HD / 8;    // n-tiles of O
  constexpr int PK = HD / 64;   // 16-byte pieces of a key that a lane reads
  constexpr int PAGE_BYTES = kPage * HD, STAGE_BYTES = 4 * PAGE_BYTES;  // K and V of the first page, of the second
  extern __shared__ __align__(128) uint8_t sm[];
  __shared__ int pre[kKv8MaxSeqs + 1];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int G = a.n_heads / a.c.n_kv_heads, Hkv = a.c.n_kv_heads;
  pdl_wait();
  pdl_launch_dependents();  // (after the wait: the combine reads the batch's lengths before its own)
  using W = Walk<W_TR, W_CH, W_UC>;
  const bool few = a.c.n_seqs <= 32;
  typename W::P::Few f;
  const int worker = blockIdx.x * W_WARPS + warp, total = few ? W::P::build_few(a, G, lane, f) : W::P::build(a, G, pre);
  const Shares shares(total, gridDim.x * W_WARPS);
  const int begin = shares.begin(worker), end = begin + shares.size(worker);
  if (begin == end) return;
  W w;
  if (few) w.start_few(a, f, G, begin, end);
  else w.start(a, pre, G, begin, end);
  const uint32_t ring = smem_u32(sm) + warp * (W_STAGES * STAGE_BYTES);
  const bool q16 = ((uintptr_t)a.q & 15) == 0 && a.ld_q * sizeof(T) % 16 == 0;
  const uint8_t *Kc = reinterpret_cast<const uint8_t*>(a.c.k), *Vc = reinterpret_cast<const uint8_t*>(a.c.v);

  while (true) {
    const Kv8Seq s = w.s;
    const int c0 = w.c0(), c1 = w.c1(), n = c1 - c0;
    if (n <= 0) return;  // (the share ends within the unit's constant)
    const int keys = s.len + s.n;  // slots that hold a token
    const int rows = s.n * G, r0 = w.tile * W_TR;

    // ---- loads of the n chunks. Lane j of a group of 32 pages: page j's id and exponents (K's and V's packed; NO_PAGE for one
    // outside the pool, whose keys no row sees)
    constexpr int NO_PAGE = 1 << 16;
    const int n_pages = min(2 * c1, (keys + kPage - 1) / kPage) - 2 * c0;
    int id_l = -1, e_l = 0, e_cur = 0;  // of the pages being loaded; of those in use
    auto issue = [&](int i) {  // chunk i of the share: zeros for slots without a token
      if (i < n) {
        if ((i & 15) == 0) {
          id_l = -1;
          e_l = 0;
          if (2 * i + lane < n_pages) {
            id_l = kv8_page(a.c, w.b, 2 * (c0 + i) + lane, a.err);
            if (id_l >= 0) {
              const long long blk = (long long)id_l * Hkv + w.kvh;
              e_l = (int)(uint8_t)a.c.k_exp[blk] | (int)(uint8_t)a.c.v_exp[blk] << 8;
            } else {
              e_l = NO_PAGE;
            }
          }
        }
        const uint32_t dst = ring + (i % W_STAGES) * STAGE_BYTES;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int id = __shfl_sync(0xffffffffu, id_l, (2 * i + x) & 31);
          const int slot0 = (2 * (c0 + i) + x) * kPage;
          const long long off = ((long long)max(id, 0) * Hkv + w.kvh) * PAGE_BYTES;
#pragma unroll
          for (int j = 0; j < PAGE_BYTES / 512; ++j) {
            const int piece = j * 32 + lane, r = piece / (HD / 16), c = piece % (HD / 16);
            const bool in = id >= 0 && slot0 + r < keys;
            cp_async16_zfill(dst + 2 * x * PAGE_BYTES + w_piece<HD>(r, c), Kc + off + piece * 16, in);
            cp_async16_zfill(dst + (2 * x + 1) * PAGE_BYTES + w_piece<HD>(r, c), Vc + off + piece * 16, in);
          }
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < W_STAGES - 1; ++i) issue(i);

    // ---- queries: fragments of this lane's rows g, g + 8, scaled
    uint32_t qf[NS][KS][4];
    float f[2];
    int tok[2];  // of the lane's rows
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool live = r0 + g + 8 * i < rows;
      const int row = live ? r0 + g + 8 * i : 0;
      tok[i] = row / G;
      const T* src = reinterpret_cast<const T*>(a.q) + (long long)(s.row0 + tok[i]) * a.ld_q +
                     (long long)(w.kvh * G + row - tok[i] * G) * HD + PK * 16 * t;
      float x[4 * KS];
      float amax = 0.f;
      load_run<4 * KS>(src, live, q16, x);
#pragma unroll
      for (int j = 0; j < 4 * KS; ++j) amax = fmaxf(amax, fabsf(x[j]));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      const int sh = query_shift(amax);
      const float up = pow2i(sh);
      f[i] = pow2i(-sh) * a.scale_log2;
#pragma unroll
      for (int j = 0; j < KS; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float lo = x[4 * j + 2 * h] * up, hi = x[4 * j + 2 * h + 1] * up;
#pragma unroll
          for (int y = 0; y < NS; ++y) {
            qf[y][j][2 * h + i] = pack_f16(lo, hi);
            const float2 got = unpack_f16(qf[y][j][2 * h + i]);
            lo -= got.x;
            hi -= got.y;
          }
        }
    }
    float o[NT][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    int E[2] = {0, 0};  // a row's o is in units of 2^E (set by the first page)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[j][i] = 0.f;
    auto rescale = [&](float x0, float x1) {
#pragma unroll
      for (int j = 0; j < NT; ++j) o[j][0] *= x0, o[j][1] *= x0, o[j][2] *= x1, o[j][3] *= x1;
    };

    auto move_to = [&](const int (&to)[2]) {  // to units of 2^to
      const float2 a = pow2_pair(E[0] - to[0]), b = pow2_pair(E[1] - to[1]);
      rescale(a.x, b.x);
      if (__any_sync(0xffffffffu, a.y != 1.f || b.y != 1.f)) rescale(a.y, b.y);
      E[0] = to[0];
      E[1] = to[1];
    };

    for (int i = 0; i < n; ++i) {
      if ((i & 15) == 0) e_cur = e_l;  // (the next 32 pages' are fetched later in this group)
      issue(i + W_STAGES - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(W_STAGES - 1) : "memory");
      __syncwarp();  // every lane's pieces of chunk i
      const uint32_t stage = ring + (i % W_STAGES) * STAGE_BYTES;
      // ---- S: two n-tiles of 8 keys a page
      float sc[2][2][4];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) sc[x][u][k] = 0.f;
#pragma unroll
      for (int pc = 0; pc < PK; ++pc)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            uint32_t wd[4];
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(wd[0]), "=r"(wd[1]), "=r"(wd[2]), "=r"(wd[3])
                         : "r"(stage + 2 * x * PAGE_BYTES + w_piece<HD>(g + 8 * u, PK * t + pc))
                         : "memory");
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t b0 = e4m3x2_to_f16x2(wd[k]), b1 = e4m3x2_to_f16x2(wd[k] >> 16);
#pragma unroll
              for (int y = 0; y < NS; ++y) mma_f16(sc[x][u], qf[y][pc * 4 + k], b0, b1);
            }
          }
      const int kp0 = (c0 + i) * W_CH;
      int ev[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int e2 = __shfl_sync(0xffffffffu, e_cur, (2 * i + x) & 31);
        ev[x] = x == 1 && 2 * i + 1 >= n_pages ? ev[0] : (int)(int8_t)(e2 >> 8);  // (no second page: as the first)
        const float unit = pow2i((int)(int8_t)(e2 & 0xff)), fu[2] = {unit * f[0], unit * f[1]};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) sc[x][u][k] = e2 & NO_PAGE ? -INFINITY : sc[x][u][k] * fu[k >> 1];
      }
      if (kp0 + W_CH > s.len) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int kp = kp0 + 16 * x + 8 * u + 2 * t + (k & 1);
              if (kp >= s.len && !(kp < keys && sees_new(a, s, tok[k >> 1], kp))) sc[x][u][k] = -INFINITY;
            }
      }
      // ---- reference maxima (rows g, g + 8), raised for the whole warp together
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) mx[k >> 1] = fmaxf(mx[k >> 1], sc[x][u][k]);
      if (__any_sync(0xffffffffu, mx[0] > m[0] + W_LAG || mx[1] > m[1] + W_LAG)) {
        float al[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float x = fmaxf(mx[k], __shfl_xor_sync(0xffffffffu, mx[k], 1));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
          const float mn = fmaxf(m[k], x);
          al[k] = m[k] == -INFINITY ? 0.f : ex2_ftz(m[k] - mn);
          m[k] = mn;
          l[k] *= al[k];
        }
        rescale(al[0], al[1]);
      }
      const float nb[2] = {m[0] == -INFINITY ? 0.f : -m[0], m[1] == -INFINITY ? 0.f : -m[1]};
      // ---- the rows' reference exponents, before each page: down (before the first for both, so that one of large values and
      // little weight is added in a unit that holds it when the other, of small values, outweighs it), then up
      const int ev_min = min(ev[0], ev[1]), ev_max = max(ev[0], ev[1]);
      if (i == 0) E[0] = E[1] = ev_min - W_EV_SET;
      const bool apart = __any_sync(0xffffffffu, ev_min < max(E[0], E[1]) || ev_max - min(E[0], E[1]) > W_EV_MAX);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int low = x == 0 ? ev_min : ev[1];
        if (apart && __any_sync(0xffffffffu, low < max(E[0], E[1]))) {
          int to[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float most = 0.f;
#pragma unroll
            for (int j = 0; j < NT; ++j) most = fmaxf(most, fmaxf(fabsf(o[j][2 * k]), fabsf(o[j][2 * k + 1])));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            to[k] = low < E[k] ? unit_down(E[k], low - W_EV_SET, most) : E[k];
          }
          move_to(to);
        }
        if (apart && __any_sync(0xffffffffu, ev[x] - min(E[0], E[1]) > W_EV_MAX)) {
          int to[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float most = fmaxf(fmaxf(sc[x][0][2 * k], sc[x][0][2 * k + 1]), fmaxf(sc[x][1][2 * k], sc[x][1][2 * k + 1]));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            to[k] = ev[x] - E[k] > W_EV_MAX ? unit_up(E[k], ev[x] - W_EV_SET, most, m[k]) : E[k];
          }
          move_to(to);
        }
        // ---- P, then O += P V
        float up[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) up[k] = pow2i(max(-126, min(126, ev[x] - E[k])));
        uint32_t pf[NS][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float p0 = ex2_ftz(sc[x][u][2 * k] + nb[k]), p1 = ex2_ftz(sc[x][u][2 * k + 1] + nb[k]);
            l[k] += p0 + p1;
            float lo = p0 * up[k], hi = p1 * up[k];
#pragma unroll
            for (int y = 0; y < NS; ++y) {
              pf[y][2 * u + k] = pack_f16(lo, hi);
              const float2 got = unpack_f16(pf[y][2 * u + k]);
              lo -= got.x;
              hi -= got.y;
            }
          }
        // codes of the lane's four keys at NT consecutive dims, as pairs of keys
        const uint32_t sv = stage + (2 * x + 1) * PAGE_BYTES;
        uint32_t vw[4][NT / 4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int key = 2 * t + (k & 1) + 8 * (k >> 1);
          if constexpr (HD == 128)
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(vw[k][0]), "=r"(vw[k][1]), "=r"(vw[k][2]), "=r"(vw[k][3])
                         : "r"(sv + w_piece<HD>(key, g))
                         : "memory");
          else
            asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];"
                         : "=r"(vw[k][0]), "=r"(vw[k][1])
                         : "r"(sv + w_piece<HD>(key, g >> 1) + (g & 1) * 8)
                         : "memory");
        }
#pragma unroll
        for (int q = 0; q < NT / 4; ++q)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t sel = h ? 0x7362u : 0x5140u;
            const uint32_t c0w = __byte_perm(vw[0][q], vw[1][q], sel), c1w = __byte_perm(vw[2][q], vw[3][q], sel);
#pragma unroll
            for (int y = 0; y < NS; ++y) {
              mma_f16(o[4 * q + 2 * h], pf[y], e4m3x2_to_f16x2(c0w), e4m3x2_to_f16x2(c1w));
              mma_f16(o[4 * q + 2 * h + 1], pf[y], e4m3x2_to_f16x2(c0w >> 16), e4m3x2_to_f16x2(c1w >> 16));
            }
          }
      }
      __syncwarp();  // every lane is done with the stage that the next round loads
    }

    // ---- the unit's end: normalised here (the sums themselves may be out of fp32's range where the values are near its
    // end). Lane (g, t) holds dims 32 t .. 32 t + 31 (of 128; 16 t .. of 64) of its rows.
    const bool whole = c0 == 0 && c1 == w.n_chunks;
    float* st = a.states + (long long)shares.slot(w.first, worker) * (W_TR * (HD + 2));
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
      l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
      const int r = g + 8 * k;
      if (r0 + r >= rows) continue;
      const float il = l[k] > 0.f ? 1.f / l[k] : (l[k] == 0.f ? 0.f : l[k]), unit = pow2i(E[k]);
      const long long at = (long long)(s.row0 + tok[k]) * a.n_heads + w.kvh * G + (r0 + r - tok[k] * G);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < NT; j += 4) {
          const int d = NT * (2 * t + h) + j;
          float v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = o[j + q][2 * k + h] * il * unit;
          if (whole) {
            T* dst = reinterpret_cast<T*>(a.out) + at * HD + d;
            store2(dst, v[0], v[1]);
            store2(dst + 2, v[2], v[3]);
          } else {
            store2(st + r * HD + d, v[0], v[1]);
            store2(st + r * HD + d + 2, v[2], v[3]);
          }
        }
      if (t == 0) {
        if (!whole) st[W_TR * HD + r] = m[k], st[W_TR * (HD + 1) + r] = l[k];
        else if (a.lse) a.lse[at] = l[k] == 0.f ? -INFINITY : (m[k] + log2f(l[k])) * 0.69314718055994531f;
      }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (!w.next(a, G)) return;
  }
}

// ---------------------------------------------------------------------------------------------
// Many query rows per KV head (drafts, prompt chunks; 16-bit models): tcgen05.
//
// A CTA takes a unit of up to 256 query rows over 128-key chunks as two streams, each with an S and an O accumulator of
// its own in tensor memory (128 lanes x 128 columns; P in fp16 takes the place of the S it came from): rows 0..127
// and 128..255 over every chunk, or, in a unit of up to 128 rows, all rows over the even and the odd chunks, whose
// states are joined at the unit's end. While the softmax of one stream runs, the tensor core works for the other.
//
// Warps 0-3 and 4-7: stream 0 and 1, a thread per row; the stream's first warp also issues its products (a stream has
// nothing else to do until they are complete). Warp 11 asks for codes, page by page as bulk copies up to two chunks ahead
// of the converters; warps 8-10 convert them to fp16 and store them as the images of tensor-core
// operands: per page of 16 keys two 8-key groups, each of HD / 64 halves of 8 rows x 128 bytes with the 128-byte
// swizzle; K is read K-major, V MN-major. Exponents stay out of the operands: K's go into the scores, V's into P as in
// the warp-level form, against the chunk's reference E, which the rows' own units follow where they can. Where a chunk's
// value exponents lie further apart than P can carry, its pages go in groups, one step of the stream each (Kv8Info). A
// warp's rows share their unit unless they differ: decided row by row in every step, 512 rows over 65,536 tokens took 485 us.
//
// K and V of a chunk are converted into a ring of three operands, so that the converters are done with a chunk before its
// products are due. Bound by a stream's chain: of about 4,600 cycles a chunk, 1,900 are the softmax of 128 x 128 scores and the
// rest the products (2 x 8 of 64 cycles each, 300 before the first is complete) and the waits between them; the streams share the
// tensor core, which is busy for half of that time. Neither the exponentials (without them the time is the same), nor
// conversion (half its stores left out: the same), nor the codes' bytes bound it. Times with the join, 28 query heads on 4 KV
// heads of 128: 512 rows over 8,192 tokens (62 GFLOP) 97 us, 0.64 PFLOP/s, over 65,536 463 us, 1.04 PFLOP/s; 32 rows over 32,768
// 36 us, of which about 16 are the launch, the first chunk's loads and the join. Measured and not kept: chunks of 64 keys with
// two score accumulators a stream and a warp of its own for the products, 129 us for the first of these (its other step then
// 110; several tests of many chunks failed, so that the time may be of a wrong kernel); 16 softmax warps, each half of a row's
// keys, the same within 4% and spills at 96 registers; the streams taking turns with their products, the same.
// ---------------------------------------------------------------------------------------------
// (T_UC 2 / 4: 512 rows over 8,192 tokens 99.9 / 97.0 us, four sequences of 32 rows over 4,096 31.0 / 28.5, eight of 16 over 100
// to 2,000 19.5 / 21.7.)
constexpr int T_TR = 256, T_CH = 128, T_UC = 4;
constexpr int T_CONV_WARPS = 3, T_THREADS = 32 * (8 + T_CONV_WARPS + 1);  // 168 registers a thread
constexpr int T_PAGES = T_CH / kPage, T_RAW = 2, T_OPS = 3, T_INFO = 4;  // chunks of codes, operands, chunks of Kv8Info in shared memory
constexpr int TM_COLS = 512;
constexpr int UNITS_DIFFER = -4096;  // in place of the exponent that a warp's rows share
template <int HD>
struct TLayout {
  static constexpr int Q = 128 * HD * 2, KV = T_CH * HD * 2, PAGE = kPage * HD * 2;  // bytes of fp16 operands
  static constexpr int RAW = T_CH * HD;                                                                      // codes of a chunk
  static constexpr int OFF_OPS = 2 * Q, OFF_RAW = OFF_OPS + T_OPS * KV;  // RAW: a stage holds K's, then V's
  static constexpr int TOTAL = OFF_RAW + T_RAW * 2 * RAW + 1024;                 // + alignment
  static constexpr int GROUP = HD * 16;  // 8 keys of a page: HD / 64 halves of 1024 bytes
  // byte offset of 16-byte piece c (8 dims) of key r of a page
  static JF_DEV uint32_t page_piece(int r, int c) {
    return (uint32_t)((r >> 3) * GROUP + (c >> 3) * 1024 + (r & 7) * 128 + (((c & 7) ^ (r & 7)) << 4));
  }
  static JF_DEV uint32_t q_piece(int r, int c) {
    return (uint32_t)((c >> 3) * 16384 + r * 128 + (((c & 7) ^ (r & 7)) << 4));
  }
};

// What the steps of a chunk need beside its operands. page: 2^(e_k), e_v - E, 2^(E - e_v) of a page, E the reference exponent of
// its step (0 to 7 below e_v), which the rows' own follow. held: slots with a token (0: no chunk, the share has
// ended). there: its pages (those outside the pool are left out) as bits. groups: how many steps; pages[j]: pages of step j as bits; E[j]: its reference exponent. T_INFO of them are enough:
// chunk g is asked for when the codes of V of chunk g - 2 are converted, after K of g - 2, into the place of V of g - 4, whose
// chunk is done with.
struct __align__(16) Kv8Info {
  float4 page[T_PAGES];
  int16_t E[T_PAGES];
  uint8_t pages[T_PAGES];
  int groups, held, there;
};

// x * y + z and x + y on two values at a time.
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
// Products and their commit by the one lane whose `on` is set, in code that the warp goes through together: descriptors then
// stay in uniform registers, and a product takes its 64 cycles of the tensor core (in a branch of one lane some 100).
JF_DEV void mma_f16_ss_on(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
JF_DEV void mma_f16_ts_on(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
JF_DEV void commit_on(uint32_t bar, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(on)
      : "memory");
}
// The unit that a row's O (in columns t_o .., in units of 2^was) goes on in, of a step whose reference exponent is another
// one; called by whole warps. Not inlined: seldom needed, and its registers would cost every step.
template <int HD>
__device__ __noinline__ int unit_of_row(uint32_t t_o, int was, int E_step, float mc, float m_ref, float al) {
  float most = 0.f;
  if (__any_sync(0xffffffffu, E_step < was)) {
#pragma unroll 1
    for (int h = 0; h < HD / 16; ++h) {
      float o[16];
      tmem_ld16(t_o + 16 * h, o);
#pragma unroll
      for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(o[i]));
    }
  }
  return E_step < was ? (mc > -INFINITY ? unit_down(was, E_step, most * al) : was) : unit_up(was, E_step, mc, m_ref);
}
// O *= x.x x.y
template <int HD>
__device__ __noinline__ void scale_o(uint32_t t_o, float x, float y) {
#pragma unroll 1
  for (int h = 0; h < HD / 16; ++h) {
    float o[16];
    uint32_t u[16];
    tmem_ld16(t_o + 16 * h, o);
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(o[i] * x * y);
    tmem_st16(t_o + 16 * h, u);
  }
}

template <int HD>
__global__ void __launch_bounds__(T_THREADS, 1) k_kv8_attn_tile(const Kv8AttnParams a) {
  using Lay = TLayout<HD>;
  using W = Walk<T_TR, T_CH, T_UC>;
  extern __shared__ uint8_t sm_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(sm_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sQ = smem_u32(sm), sOps = sQ + Lay::OFF_OPS;
  // a stage of codes: landed, converted; operands K and V (number 2 g and 2 g + 1 of the share, in a ring of T_OPS): there, and
  // a place of the ring read by both streams (a unit of one tile: by its stream, counted twice; that they are there, on one
  // barrier for even and one for odd chunks: a stream that waits for every second one must not meet a barrier a completion
  // ahead or behind); per stream: S ready (the products, and the thread that issued them, which passes on the chunk's
  // Kv8Info), P V done, everything done
  __shared__ __align__(8) uint64_t b_raw[T_RAW], b_rawfree[T_RAW], b_kfull[2], b_vfull[2], b_free[T_OPS], b_s[2], b_o[2], b_all[2];
  __shared__ uint32_t tmem_slot;
  __shared__ Kv8Info s_info[T_INFO];
  __shared__ int16_t s_unit[256];
  int* pre = reinterpret_cast<int*>(sm + Lay::OFF_RAW);  // (until the first codes are asked for)
  // (shuffles tell the compiler that warp numbers and the TMEM address are uniform: operand descriptors then are)
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int G = a.n_heads / a.c.n_kv_heads, Hkv = a.c.n_kv_heads;
  if (tid == 0) {
    for (int i = 0; i < T_RAW; ++i) {
      mbar_init(smem_u32(&b_raw[i]), 1);
      mbar_init(smem_u32(&b_rawfree[i]), T_CONV_WARPS);
    }
    for (int i = 0; i < T_OPS; ++i) mbar_init(smem_u32(&b_free[i]), 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&b_kfull[i]), T_CONV_WARPS);
      mbar_init(smem_u32(&b_vfull[i]), T_CONV_WARPS);
      mbar_init(smem_u32(&b_s[i]), 2);
      mbar_init(smem_u32(&b_o[i]), 1);
      mbar_init(smem_u32(&b_all[i]), 1);
    }
    fence_mbar_init();
  }
  pdl_wait();
  pdl_launch_dependents();  // (after the wait: the combine reads the batch's lengths before its own)
  const bool few = a.c.n_seqs <= 32;
  typename W::P::Few f;
  const Shares shares(few ? W::P::build_few(a, G, lane, f) : W::P::build(a, G, pre), gridDim.x);
  const int begin = shares.begin(blockIdx.x), end = begin + shares.size(blockIdx.x);
  if (begin == end) return;
  if (warp == 8) {
    tmem_alloc(smem_u32(&tmem_slot), TM_COLS);
    tmem_relinquish();
  }
  W w;
  if (few) w.start_few(a, f, G, begin, end);
  else w.start(a, pre, G, begin, end);
  fence_proxy_async_smem();  // the plan's place is taken by copies
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
  const unsigned long long limit = kWaitLimitDefaultNs;
  auto wait = [&](uint64_t& bar, int uses) {  // for completion number `uses` (from 0); the warp agrees
    const bool ok = mbar_wait_bounded(smem_u32(&bar), (uint32_t)uses & 1u, limit);
    return __all_sync(0xffffffffu, ok) != 0;
  };
  auto tile_rows = [&](const W& w) { return min(w.s.n * G - w.tile * T_TR, T_TR); };

  if (warp == 11) {
    // ---- asks for codes: page ids are read two chunks ahead of them, exponents one, so that nothing waits for what has
    // just been asked for. Lane j < 8: page j.
    struct Ahead {
      int id, ek, ev, held, kvh;
    };
    int chunk = w.c0();
    bool more = w.c1() > chunk;
    auto look = [&]() {  // the next chunk of the share
      const int kp0 = chunk * T_CH;
      Ahead n = {0, 0, 0, more ? min(T_CH, w.s.len + w.s.n - kp0) : 0, w.kvh};
      if (more) {
        if (lane * kPage < n.held) n.id = a.c.page_table[(long long)w.b * a.c.pages_per_seq + chunk * T_PAGES + lane];
        if (++chunk >= w.c1()) {
          more = w.next(a, G) && w.c1() > 0;
          chunk = 0;
        }
      }
      return n;
    };
    auto exponents = [&](Ahead& n) {
      if (lane * kPage < n.held) {
        if (n.id >= 0 && n.id < a.c.n_pages) {
          const long long blk = (long long)n.id * Hkv + n.kvh;
          n.ek = a.c.k_exp[blk];
          n.ev = a.c.v_exp[blk];
        } else {  // reported and left out
          jf_set_error(a.err, JF_DERR_BOUNDS);
          n.id = -1;
        }
      }
    };
    Ahead cur = look(), next = look();
    exponents(cur);
    int E_run = -126, g = 0;
    bool ok = true;
    for (;; ++g) {  // (the last round asks for nothing and tells the converters so)
      const int stage = g % T_RAW;
      if (g >= T_RAW && !wait(b_rawfree[stage], g / T_RAW - 1)) {
        ok = false;
        break;
      }
      // the copies first: what describes them has time until they have landed
      const bool mine = lane * kPage < cur.held && cur.id >= 0;
      const uint32_t bar = smem_u32(&b_raw[stage]), dst = sQ + Lay::OFF_RAW + stage * 2 * Lay::RAW + lane * (kPage * HD);
      const long long off = ((long long)cur.id * Hkv + cur.kvh) * (kPage * HD);
      if (mine) {
        bulk_load(dst, reinterpret_cast<const uint8_t*>(a.c.k) + off, kPage * HD, bar);
        bulk_load(dst + Lay::RAW, reinterpret_cast<const uint8_t*>(a.c.v) + off, kPage * HD, bar);
      }
      Kv8Info& info = s_info[g % T_INFO];
      unsigned rest = __ballot_sync(0xffffffffu, mine);
      const int there = (int)rest, bytes = __popc(rest) * (2 * kPage * HD);
      int groups = 0, E_mine = 0;
      if (rest == 0) {  // (a step without a key)
        if (lane == 0) info.pages[0] = 0, info.E[0] = (int16_t)E_run;
        groups = 1;
      }
      while (rest) {
        const bool in = rest >> lane & 1u;
        const int hi = __reduce_max_sync(0xffffffffu, in ? cur.ev : -1000);
        const unsigned now = __ballot_sync(0xffffffffu, in && cur.ev >= hi - W_EV_MAX);
        const int lo = __reduce_min_sync(0xffffffffu, now >> lane & 1u ? cur.ev : 1000);
        if (E_run > lo || hi - E_run > W_EV_MAX) E_run = max(max(min(lo, hi - W_EV_SET), hi - W_EV_MAX), -126);
        if (now >> lane & 1u) E_mine = E_run;
        if (lane == 0) info.pages[groups] = (uint8_t)now, info.E[groups] = (int16_t)E_run;
        ++groups;
        rest &= ~now;
      }
      if (lane < T_PAGES) {
        const int d = mine ? cur.ev - E_mine : 0;
        info.page[lane] = make_float4(pow2i(cur.ek), (float)d, pow2i(-d), 0.f);
      }
      if (lane == 0) info.groups = groups, info.held = cur.held, info.there = there;
      __syncwarp();
      if (lane == 0) mbar_arrive_expect_tx(bar, bytes);
      if (cur.held == 0) break;
      cur = next;
      exponents(cur);
      next = look();
    }
    if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
    // every copy has landed before the CTA may leave, also after a wait that gave up. (The last round has completed its
    // stage's barrier once more; the chunk before it there has been converted.)
    for (int k = max(0, g - T_RAW + (ok ? 1 : 0)); k < g; ++k)
      if (!wait(b_raw[k % T_RAW], k / T_RAW)) break;
  } else if (warp >= 8) {
    // ---- codes to operands. Thread: pieces of 16 dims; a warp has pages 3 cw .. of K and 5 - 3 cw .. of V (three, three
    // and two of 8), a round is 4 (8) keys. The lanes of a quarter warp (8 x 16 bytes) read two rows and write two rows so
    // that neither meets a bank twice.
    const int cw = warp - 8;
    constexpr int PR = HD / 16, ROUNDS = kPage * PR / 32;  // pieces per key; rounds per page
    const int lr = PR == 8 ? 2 * ((lane >> 3) & 1) + ((lane >> 2) & 1) : lane >> 2;
    const int lc = PR == 8 ? (lane & 3) + 4 * (((lane >> 2) & 1) ^ (lane >> 4)) : lane & 3;
    auto put = [&](uint32_t src, uint32_t dst, int first, int held, int there) {
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const int page = first + q;
        if (page < 0 || page >= T_PAGES) continue;
        uint4 x[ROUNDS];
#pragma unroll
        for (int j = 0; j < ROUNDS; ++j)
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(x[j].x), "=r"(x[j].y), "=r"(x[j].z), "=r"(x[j].w)
                       : "r"(src + page * (kPage * HD) + (j * (32 / PR) + lr) * HD + lc * 16)
                       : "memory");
        if (held < T_CH || there != 255) {  // slots without a token, pages outside the pool
#pragma unroll
          for (int j = 0; j < ROUNDS; ++j)
            if (page * kPage + j * (32 / PR) + lr >= held || !(there >> page & 1)) x[j] = make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int j = 0; j < ROUNDS; ++j) {
          const uint32_t wd[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t p = dst + page * Lay::PAGE + Lay::page_piece(j * (32 / PR) + lr, 2 * lc + h);
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(p), "r"(e4m3x2_to_f16x2(wd[2 * h])),
                         "r"(e4m3x2_to_f16x2(wd[2 * h] >> 16)), "r"(e4m3x2_to_f16x2(wd[2 * h + 1])),
                         "r"(e4m3x2_to_f16x2(wd[2 * h + 1] >> 16))
                         : "memory");
          }
        }
      }
      fence_proxy_async_smem();  // this thread's stores -> operand reads; its reads of the codes -> the next copies
      __syncwarp();
    };
    bool ok = true;
    for (int g = 0; ok; ++g) {
      const int stage = g % T_RAW;
      const uint32_t src = sQ + Lay::OFF_RAW + stage * 2 * Lay::RAW;
      ok = wait(b_raw[stage], g / T_RAW);
      const int held = s_info[g % T_INFO].held, there = s_info[g % T_INFO].there;
      if (!ok || held == 0) break;
      const int kn = 2 * g, vn = kn + 1;  // the operands' numbers
      ok = kn < T_OPS || wait(b_free[kn % T_OPS], kn / T_OPS - 1);
      if (!ok) break;
      put(src, sOps + kn % T_OPS * Lay::KV, 3 * cw, held, there);
      if (lane == 0) mbar_arrive(smem_u32(&b_kfull[g & 1]));
      ok = vn < T_OPS || wait(b_free[vn % T_OPS], vn / T_OPS - 1);
      if (!ok) break;
      put(src + Lay::RAW, sOps + vn % T_OPS * Lay::KV, 5 - 3 * cw, held, there);
      if (lane == 0) {
        mbar_arrive(smem_u32(&b_vfull[g & 1]));
        mbar_arrive(smem_u32(&b_rawfree[stage]));
      }
    }
    if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
  } else {
    // ---- stream s: row `lr` of its 128
    const int s = warp >> 2, lr = (warp & 3) * 32 + lane;
    const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_s = t_row + s * 128, t_o = t_row + 256 + s * 128;
    const bool issuer = (warp & 3) == 0;
    constexpr uint32_t idesc_s = idesc_f16_f32(128, T_CH), idesc_pv = idesc_f16_f32(128, HD) | (1u << 16);  // V MN-major
    const uint64_t dq = sdesc_k_sw128(sQ + s * Lay::Q), dk0 = sdesc_k_sw128(sOps, Lay::GROUP), dv0 = sdesc_mn_sw128(sOps, 1024u, Lay::GROUP);
    // S of a step, by the stream's first warp; both = a unit of two tiles
    auto issue_s = [&](int gc, bool last, bool both) {
      const int place = __shfl_sync(0xffffffffu, 2 * gc % T_OPS, 0);
      uint64_t dk = dk0 + (uint64_t)(place * (Lay::KV >> 4)), dqn = dq;
      asm volatile("" : "+l"(dk), "+l"(dqn));  // (the sums below are not kept from step to step)
      tc_fence_after();
      const uint32_t on = elect_one();
#pragma unroll
      for (int kk = 0; kk < HD / 16; ++kk)
        mma_f16_ss_on(tmem + s * 128, dqn + (uint64_t)((kk >> 2) * (16384 >> 4) + (kk & 3) * 2), dk + (uint64_t)((kk >> 2) * 64 + (kk & 3) * 2),
                      idesc_s, kk > 0 ? 1u : 0u, on);
      commit_on(smem_u32(&b_s[s]), on);
      if (lane == 0) mbar_arrive(smem_u32(&b_s[s]));
      commit_on(smem_u32(&b_free[place]), on && last);
      commit_on(smem_u32(&b_free[place]), on && last && !both);
      __syncwarp();
    };
    auto issue_pv = [&](int gc, bool fresh, bool last, bool both) {
      const int place = __shfl_sync(0xffffffffu, (2 * gc + 1) % T_OPS, 0);
      uint64_t dv = dv0 + (uint64_t)(place * (Lay::KV >> 4));
      asm volatile("" : "+l"(dv));
      tc_fence_after();
      const uint32_t on = elect_one();
#pragma unroll
      for (int kk = 0; kk < T_PAGES; ++kk)
        mma_f16_ts_on(tmem + 256 + s * 128, tmem + s * 128 + kk * 8, dv + (uint64_t)(kk * (Lay::PAGE >> 4)), idesc_pv,
                      kk > 0 || !fresh ? 1u : 0u, on);
      commit_on(smem_u32(&b_o[s]), on);
      commit_on(smem_u32(&b_free[place]), on && last);
      commit_on(smem_u32(&b_free[place]), on && last && !both);
      __syncwarp();
    };
    auto stream_and = [&](bool ok) { return s ? sync_and<2, 128>(ok) : sync_and<1, 128>(ok); };
    const bool q16 = ((uintptr_t)a.q & 15) == 0 && a.ld_q % 8 == 0;
    bool ok = true;
    int steps = 0, g = 0;  // steps of the stream so far; chunks of the share so far
    while (true) {
      const int rows = tile_rows(w);
      const bool two = rows > 128;
      const int c0 = w.c0(), n = w.c1() - c0;
      if (n <= 0) break;
      const Kv8Seq sq = w.s;
      const int r = (two ? s * 128 : 0) + lr;  // of the tile
      const bool live = r < rows;
      const int tr = w.tile * T_TR + (live ? r : 0), tok = tr / G;
      const long long at = (long long)(sq.row0 + tok) * a.n_heads + w.kvh * G + (tr - tok * G);
      float f;
      {  // queries: a warp copies its rows whole, HD / 8 lanes a row; then each thread scales its own row in place. The
        // softmax scale's sign goes with them, so that f >= 0. (Rolled loops: the code is new to the instruction cache.)
        constexpr int LPR = HD / 8, RPI = 32 / LPR;
        const bf16* mine = live ? reinterpret_cast<const bf16*>(a.q) + (long long)(sq.row0 + tok) * a.ld_q + (long long)(w.kvh * G + (tr - tok * G)) * HD
                                : nullptr;
        const uint32_t sq_s = sQ + (uint32_t)(s * Lay::Q);
        if (q16) {
#pragma unroll 4
          for (int i = 0; i < LPR; ++i) {
            const int rl = i * RPI + lane / LPR, c = lane % LPR;
            const bf16* src = reinterpret_cast<const bf16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), rl));
            cp_async16_zfill(sq_s + Lay::q_piece((warp & 3) * 32 + rl, c), src ? src + c * 8 : reinterpret_cast<const bf16*>(a.q), src != nullptr);
          }
          asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
          __syncwarp();
        } else {
#pragma unroll 1
          for (int c = 0; c < LPR; ++c) {
            uint32_t h[4] = {0u, 0u, 0u, 0u};
            if (live) {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                h[k] = (uint32_t)__bfloat16_as_ushort(mine[c * 8 + 2 * k]) | (uint32_t)__bfloat16_as_ushort(mine[c * 8 + 2 * k + 1]) << 16;
            }
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(sq_s + Lay::q_piece(lr, c)), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
          }
        }
        constexpr uint32_t mag = 0x7fff7fffu;
        uint32_t most = 0;  // the largest magnitudes as bit patterns
        auto piece = [&](int c, uint32_t (&x)[4]) {
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(sq_s + Lay::q_piece(lr, c)) : "memory");
        };
#pragma unroll 4
        for (int c = 0; c < LPR; ++c) {
          uint32_t x[4];
          piece(c, x);
          most = __vmaxu2(most, __vmaxu2(__vmaxu2(x[0] & mag, x[1] & mag), __vmaxu2(x[2] & mag, x[3] & mag)));
        }
        const int my_shift = query_shift(__uint_as_float(max(most & 0xffffu, most >> 16) << 16));
        const float up = a.scale_log2 < 0.f ? -pow2i(my_shift) : pow2i(my_shift);
#pragma unroll 4
        for (int c = 0; c < LPR; ++c) {
          uint32_t x[4];
          piece(c, x);
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] = pack_f16(__uint_as_float(x[k] << 16) * up, __uint_as_float(x[k] & 0xffff0000u) * up);
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(sq_s + Lay::q_piece(lr, c)), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
        }
        f = pow2i(-my_shift) * fabsf(a.scale_log2);
        fence_proxy_async_smem();
      }
      float m_ref = -INFINITY, l = 0.f;
      int E_all = 0;  // the warp's rows' O are in units of 2^E_all, or each in its own (UNITS_DIFFER: s_unit)
      bool first = true;
      const int c_step = two ? 1 : 2, c_first = two ? 0 : s, g0 = g;  // the stream's chunks c_first, + c_step, ...
      g += n;
      ok = stream_and(ok);  // the stream's queries are there
      if (issuer && c_first < n && ok) {
        ok = wait(b_kfull[(g0 + c_first) & 1], (g0 + c_first) >> 1);
        if (ok) issue_s(g0 + c_first, s_info[(g0 + c_first) % T_INFO].groups == 1, two);
      }
      bool fresh = true;  // no P V of the unit yet
      bool go = true;     // (left by all warps of the stream together)
      for (int c = c_first; c < n && go; c += c_step) {
        const int gc = g0 + c;
        const Kv8Info& info = s_info[gc % T_INFO];
        const int kp0 = (c0 + c) * T_CH;
        // bits of the 32 keys from column 32 h on that the row sees
        const bool cut = kp0 + T_CH > sq.len;
        auto visible = [&](int h) -> uint32_t {
          if (!cut) return 0xffffffffu;
          const int jb = kp0 + 32 * h - sq.len;  // as a new row
          uint32_t v;
          if (a.mask) {
            const uint32_t* mw = a.mask + (long long)(sq.row0 + tok) * a.mask_words;
            auto word = [&](int i) { return i >= 0 && i < a.mask_words ? mw[i] : 0u; };
            const int i = jb >> 5, b = jb & 31;
            v = b ? word(i) >> b | word(i + 1) << (32 - b) : word(i);
            const int left = sq.n - jb;  // new rows from here on
            if (left < 32) v &= left <= 0 ? 0u : (1u << left) - 1u;
          } else {
            const int seen = tok - jb + 1;
            v = seen >= 32 ? 0xffffffffu : (seen <= 0 ? 0u : (1u << seen) - 1u);
          }
          if (jb < 0) v |= jb <= -32 ? 0xffffffffu : (1u << -jb) - 1u;
          return v;
        };
        int groups = 1;
        for (int j = 0; j < groups; ++j) {
          ok = wait(b_s[s], steps) && ok;
          tc_fence_after();
          if (ok) {
          // The row's scores, 32 at a time, for the maximum and again for the exponentials (P of column c goes to c / 2,
          // which has been read by then). What a row does not see, in the few chunks that hold new rows, is written over with
          // -inf beforehand: in the loops themselves it would cost every chunk 6%, and as much what a page's factors are made of.
          // (512 rows over 65,536 tokens: 461 us; with the loops rolled 489; in one pass, P in registers until the maximum is
          // known, 686, for it spills.)
          groups = info.groups;
          const int pages = info.pages[j], E_step = info.E[j];
          if (cut || pages != 255) {
#pragma unroll 1
            for (int h = 0; h < 4; ++h) {
              uint32_t see = visible(h);
              if (!(pages >> (2 * h) & 1)) see &= 0xffff0000u;
              if (!(pages >> (2 * h + 1) & 1)) see &= 0x0000ffffu;
#pragma unroll 1
              for (int y = 0; y < 2; ++y, see >>= 16) {
                float v[16];
                uint32_t u[16];
                tmem_ld16(t_s + 32 * h + 16 * y, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) u[i] = see >> i & 1u ? __float_as_uint(v[i]) : 0xff800000u;
                tmem_st16(t_s + 32 * h + 16 * y, u);
              }
            }
            tmem_wait_st();
          }
          // of a page's scores; above 0, so that a hidden key's -inf stays one
          auto factor = [&](float fk) { return fmaxf(f * fk, 7.888609e-31f /* 2^-100 */); };
          float mc = -INFINITY;
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            float v[32];
            const float fk[2] = {info.page[2 * h].x, info.page[2 * h + 1].x};
            tmem_ld32(t_s + 32 * h, v);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float mx = v[16 * y];
#pragma unroll
              for (int i = 1; i < 16; ++i) mx = fmaxf(mx, v[16 * y + i]);
              mc = fmaxf(mc, mx * factor(fk[y]));
            }
          }
          const bool raise = mc > m_ref + W_LAG;
          const float al = raise ? (m_ref == -INFINITY ? 0.f : ex2_ftz(m_ref - mc)) : 1.f;
          l *= al;
          if (raise) m_ref = mc;
          float nb = m_ref == -INFINITY ? 0.f : -m_ref, l_before = 0.f;
          if (first) E_all = E_step;
          const bool apart = E_step != E_all;  // (seldom)
          if (apart) {
            const int was = E_all == UNITS_DIFFER ? s_unit[tid] : E_all, E = unit_of_row<HD>(t_o, was, E_step, mc, m_ref, al);
            E_all = __all_sync(0xffffffffu, E == E_step) ? E_step : UNITS_DIFFER;
            s_unit[tid] = (int16_t)E;
            if (__any_sync(0xffffffffu, raise || E != was)) {
              const float2 step = pow2_pair(was - E);
              scale_o<HD>(t_o, al * step.x, step.y);
            }
            // Probabilities of the step are 2^(E_step - E) of what the page's exponent makes of them. (What lies 2^60 below the
            // row's unit is nothing in fp16 in any case, but its sum counts.)
            nb += (float)max(-60, min(122, E_step - E));
            l_before = l;
            l = 0.f;
          } else if (__any_sync(0xffffffffu, raise) && !first) {
            scale_o<HD>(t_o, al, 1.f);
          }
          first = false;
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            float v[32];
            uint32_t u[16];
            const float4 page[2] = {info.page[2 * h], info.page[2 * h + 1]};
            tmem_ld32(t_s + 32 * h, v);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const float fx = factor(page[y].x), b = nb + page[y].y;
              float2 ls = make_float2(0.f, 0.f);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                float2 p = fma2(make_float2(v[16 * y + 2 * i], v[16 * y + 2 * i + 1]), make_float2(fx, fx), make_float2(b, b));
                p.x = ex2_ftz(p.x);
                p.y = ex2_ftz(p.y);
                ls = add2(ls, p);
                u[8 * y + i] = pack_f16(p.x, p.y);
              }
              l = fmaf(ls.x + ls.y, page[y].z, l);
            }
            tmem_st16(t_s + 16 * h, u);
          }
          if (apart) l = fmaf(l, pow2i(-max(-60, min(122, E_step - s_unit[tid]))), l_before);
          tmem_wait_st();
          }
          tc_fence_before();
          go = ok = stream_and(ok);  // P of all rows is there
          if (!go) break;
          if (issuer) {
            const bool last = j == groups - 1;
            ok = wait(b_vfull[gc & 1], gc >> 1);
            if (ok) issue_pv(gc, fresh, last, two);
            // the stream's next S, once P (which lies where S will) has been read
            const int gn = last ? gc + c_step : gc, jn = last ? 0 : j + 1;
            if (ok && (!last || c + c_step < n)) {
              ok = wait(b_kfull[gn & 1], gn >> 1);
              const bool last_s = s_info[gn % T_INFO].groups == jn + 1;
              ok = ok && wait(b_o[s], steps);
              if (ok) issue_s(gn, last_s, two);
            }
          }
          fresh = false;
          ++steps;
        }
      }
      if (!first && ok) {  // the unit's last P V of the stream
        ok = wait(b_o[s], steps - 1);
        tc_fence_after();
      }
      const int E = E_all == UNITS_DIFFER ? s_unit[tid] : E_all;
      if (!two) {
        // (where the stream's queries were)
        reinterpret_cast<float2*>(sm + s * Lay::Q)[lr] = make_float2(m_ref, l);
        reinterpret_cast<int*>(sm + s * Lay::Q)[256 + lr] = E;
      }
      ok = sync_and<3, 256>(ok);  // both streams leave a unit together (barrier 0 is __syncthreads)
      if (!ok) break;
      // ---- the unit's end: rows normalised, into out or the state that the CTA leaves
      const bool whole = c0 == 0 && n == w.n_chunks;
      float* st = a.states + (long long)shares.slot(w.first, blockIdx.x) * (T_TR * (HD + 2));
      float M = m_ref, L = l, w0 = 1.f, w1 = 0.f;  // weights of this stream's O (two tiles), or of both streams'
      int Em = E, d0 = 0, d1 = HD;                 // their unit 2^Em; the dims that this thread finishes
      if (!two) {
        const float2 ml0 = reinterpret_cast<const float2*>(sm)[lr], ml1 = reinterpret_cast<const float2*>(sm + Lay::Q)[lr];
        const int E0 = reinterpret_cast<const int*>(sm)[256 + lr], E1 = reinterpret_cast<const int*>(sm + Lay::Q)[256 + lr];
        const float m0 = ml0.x, m1 = ml1.x, l0 = ml0.y, l1 = ml1.y;
        M = fmaxf(m0, m1);
        const float a0 = m0 == -INFINITY ? 0.f : exp2f(m0 - M), a1 = m1 == -INFINITY ? 0.f : exp2f(m1 - M);
        L = (m0 == -INFINITY ? l0 : a0 * l0) + (m1 == -INFINITY ? l1 : a1 * l1);  // (nothing seen: 0, or NaN)
        // (a stream that has no weight, or saw nothing, has no say in the unit)
        Em = max(a0 > 0.f ? E0 : -126, a1 > 0.f ? E1 : -126);
        w0 = a0 * pow2i(max(-126, min(0, E0 - Em)));
        w1 = a1 * pow2i(max(-126, min(0, E1 - Em)));
        d0 = s * (HD / 2);
        d1 = d0 + HD / 2;
      }
      const float il = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L), unit = pow2i(Em);
      const uint32_t t_first = two ? t_o : t_row + 256;
      const bool second = !two && n > 1;  // (a stream without a step holds nothing)
      // A state leaves through shared memory (32 rows x DW dims a warp, 16-byte pieces swizzled, in the upper half of the
      // stream's queries' place), so that a row's pieces are written side by side.
      constexpr int DW = HD / 4, PW = DW / 4;  // dims at a time; pieces of a row
      static_assert(4 * 32 * DW * 4 <= Lay::Q / 2, "four warps' pieces");
      const uint32_t turn_buf = sQ + (uint32_t)(s * Lay::Q + Lay::Q / 2 + (warp & 3) * (32 * DW * 4));
      auto place = [&](int row, int piece) {
        return turn_buf + row * (DW * 4) + ((piece ^ (PW == 8 ? row & 7 : row >> 1 & 3)) << 4);
      };
#pragma unroll 1
      for (int d = d0; d < d1; d += DW) {
        float x[DW], y[DW];
        if constexpr (DW == 32) tmem_ld32(t_first + d, x);
        else tmem_ld16(t_first + d, x);
        if (second) {
          if constexpr (DW == 32) tmem_ld32(t_row + 384 + d, y);
          else tmem_ld16(t_row + 384 + d, y);
        }
#pragma unroll
        for (int i = 0; i < DW; ++i) {
          float v = w0 == 0.f ? 0.f : w0 * x[i];
          if (second && w1 != 0.f) v = fmaf(w1, y[i], v);
          x[i] = v * il * unit;
        }
        if (whole) {
          if (live) {
#pragma unroll
            for (int h = 0; h < PW / 2; ++h) {
              uint32_t u[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(x[8 * h + 2 * i], x[8 * h + 2 * i + 1]);
                u[i] = *reinterpret_cast<const uint32_t*>(&v);
              }
              reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(a.out) + at * HD + d)[h] = make_uint4(u[0], u[1], u[2], u[3]);
            }
          }
        } else {
#pragma unroll
          for (int h = 0; h < PW; ++h)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(place(lane, h)), "f"(x[4 * h]), "f"(x[4 * h + 1]), "f"(x[4 * h + 2]),
                         "f"(x[4 * h + 3])
                         : "memory");
          __syncwarp();
#pragma unroll
          for (int h = 0; h < PW; ++h) {
            const int rl = 32 / PW * h + lane / PW, rt = (two ? s * 128 : 0) + (warp & 3) * 32 + rl;
            float4 v;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                         : "r"(place(rl, lane % PW))
                         : "memory");
            if (rt < rows) reinterpret_cast<float4*>(st + rt * HD + d)[lane % PW] = v;
          }
          __syncwarp();
        }
      }
      if (live && d0 == 0) {
        if (!whole) st[T_TR * HD + r] = M, st[T_TR * (HD + 1) + r] = L;
        else if (a.lse) a.lse[at] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
      }
      tc_fence_before();
      sync_and<3, 256>(true);  // both streams have read both accumulators
      if (!w.next(a, G)) break;
    }
    if (!ok && lane == 0) jf_set_error(a.err, JF_DERR_TIMEOUT_MMA);
    // every product is complete before the CTA may leave, also after a wait that gave up
    if (issuer) {
      __syncwarp();
      if (elect_one()) tc_commit(smem_u32(&b_all[s]));
      __syncwarp();
      mbar_wait_bounded(smem_u32(&b_all[s]), 0u, limit);
    }
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 8) tmem_dealloc(tmem, TM_COLS);
}

// ---------------------------------------------------------------------------------------------
// Joins the partial states of the units that several workers share, by RW warps per (row, query head). n: workers of
// the kernel that left them. Which states there are follows from the batch's lengths, which were complete before
// that kernel let this one in, so with up to 32 sequences only the states are left to read after the wait.
// ---------------------------------------------------------------------------------------------
template <typename T, int HD, int TR, int CH, int UC, int RW>
__global__ void __launch_bounds__(256) k_kv8_combine(const Kv8AttnParams a, int n) {
  using P = Plan<TR, CH, UC>;
  constexpr int D = HD / 32, CB_WARPS = 8;
  __shared__ float s_m[CB_WARPS], s_l[CB_WARPS], s_o[RW > 1 ? CB_WARPS : 1][HD];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % RW;
  pdl_launch_dependents();
  const uint32_t i = blockIdx.x * (CB_WARPS / RW) + warp / RW;  // (n_rows * n_heads is below 2^30)
  const int G = a.n_heads / a.c.n_kv_heads;
  // (a row's warps stay together: they meet at a barrier of their own)
  if (i >= (uint32_t)(a.r.n_rows * a.n_heads)) {
    pdl_wait();
    return;
  }
  const int row = (int)(i / (uint32_t)a.n_heads), head = (int)i - row * a.n_heads;
  // the sequence of the row
  int lo = 0, m = a.c.n_seqs;
  while (m > 1) {
    const int step = (m + 31) / 32, b = lo + lane * step;
    const unsigned hits = __ballot_sync(0xffffffffu, lane * step < m && a.r.row_start[b] <= row);
    const int k = hits ? 31 - __clz(hits) : 0;
    lo += k * step;
    m = min(step, m - k * step);
  }
  const Kv8Seq s = kv8_seq(a.c, a.r, lo, a.err);
  const bool live = row >= s.row0 && row < s.row0 + s.n;
  const int tr = (row - s.row0) * G + head % G, tile = tr / TR, r = tr % TR;
  int before = 0;
  for (int t = lane; live && t < tile; t += 32) before += UC + P::chunks(a, s, G, t);
  before = __reduce_add_sync(0xffffffffu, before);
  int base, per_seq, total;
  if (a.c.n_seqs <= 32) {
    const int mine = lane < a.c.n_seqs ? P::per_head(a, kv8_seq(a.c, a.r, lane, a.err), G) * a.c.n_kv_heads : 0;
    total = __reduce_add_sync(0xffffffffu, mine);
    base = __reduce_add_sync(0xffffffffu, lane < lo ? mine : 0);
    per_seq = __shfl_sync(0xffffffffu, mine, lo);
    pdl_wait();
  } else {
    pdl_wait();
    base = a.plan[lo];
    per_seq = a.plan[lo + 1] - base;
    total = a.plan[a.c.n_seqs];
  }
  if (!live) return;
  const Shares shares(total, n);
  const int first = base + head / G * (per_seq / a.c.n_kv_heads) + before + UC, last = first + P::chunks(a, s, G, tile) - 1;
  const int i0 = shares.of(first), i1 = shares.of(last);
  if (i0 == i1) return;  // finished by the one worker that held it
  auto state = [&](int c) { return a.states + (long long)shares.slot(first, c) * (TR * (HD + 2)); };
  // this warp's states c = i0 + part, + RW, ...: 32 at a time, lane j the statistics of the j'th, and of these B at a
  // time in flight
  constexpr int B = 16;
  const int mine = i1 - i0 - part >= 0 ? (i1 - i0 - part) / RW + 1 : 0;
  float M = -INFINITY, L = 0.f, o[D];  // O as the weighted mean of what was joined so far, of weight L 2^M
#pragma unroll
  for (int j = 0; j < D; ++j) o[j] = 0.f;
  for (int k0 = 0; k0 < mine; k0 += 32) {
    const float* st = k0 + lane < mine ? state(i0 + part + (k0 + lane) * RW) : nullptr;
    float ov[B][D];
    auto fetch = [&](int k) {
#pragma unroll
      for (int x = 0; x < B; ++x) {
        const float* sx = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(st), k + x));
        if constexpr (D == 4) {
          const float4 v = sx ? __ldcg(reinterpret_cast<const float4*>(sx + r * HD) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
          ov[x][0] = v.x, ov[x][1] = v.y, ov[x][2] = v.z, ov[x][3] = v.w;
        } else {
          const float2 v = sx ? __ldcg(reinterpret_cast<const float2*>(sx + r * HD) + lane) : make_float2(0.f, 0.f);
          ov[x][0] = v.x, ov[x][1] = v.y;
        }
      }
    };
    const float mc = st ? st[TR * HD + r] : -INFINITY, lc = st ? st[TR * (HD + 1) + r] : 0.f;
    fetch(0);
    float mn = mc;
#pragma unroll
    for (int sh = 16; sh > 0; sh >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, sh));
    mn = fmaxf(M, mn);
    float w = mc == -INFINITY ? lc : exp2f(mc - mn) * lc;  // (nothing seen: 0, or NaN)
    const float was = M == -INFINITY ? L : exp2f(M - mn) * L;
    float Ln = w;
#pragma unroll
    for (int sh = 16; sh > 0; sh >>= 1) Ln += __shfl_xor_sync(0xffffffffu, Ln, sh);
    Ln += was;
    const float il = Ln == 0.f ? 0.f : 1.f / Ln;
    w *= il;
#pragma unroll
    for (int j = 0; j < D; ++j) o[j] *= was * il;
    for (int k = 0; k < 32 && k0 + k < mine; k += B) {
      if (k > 0) fetch(k);
#pragma unroll
      for (int x = 0; x < B; ++x) {
        const float wx = __shfl_sync(0xffffffffu, w, k + x);
        if (wx != 0.f) {
#pragma unroll
          for (int j = 0; j < D; ++j) o[j] = fmaf(wx, ov[x][j], o[j]);
        }
      }
    }
    M = mn;
    L = Ln;
  }
  if constexpr (RW > 1) {  // the row's warps, in order
    if (lane == 0) s_m[warp] = M, s_l[warp] = L;
#pragma unroll
    for (int j = 0; j < D; ++j) s_o[warp][D * lane + j] = o[j];
    const int w0 = warp - part;
    if (RW == CB_WARPS || w0 == 0) sync_and<1, 32 * RW>(true);
    else sync_and<2, 32 * RW>(true);  // (two rows a CTA)
    if (part > 0) return;
    float mn = s_m[w0];
    for (int q = 1; q < RW; ++q) mn = fmaxf(mn, s_m[w0 + q]);
    float w[RW], Ln = 0.f;
#pragma unroll
    for (int q = 0; q < RW; ++q) {
      w[q] = s_m[w0 + q] == -INFINITY ? s_l[w0 + q] : exp2f(s_m[w0 + q] - mn) * s_l[w0 + q];
      Ln += w[q];
    }
    const float il = Ln == 0.f ? 0.f : 1.f / Ln;
#pragma unroll
    for (int j = 0; j < D; ++j) o[j] = 0.f;
#pragma unroll
    for (int q = 0; q < RW; ++q)
      if (w[q] != 0.f) {
#pragma unroll
        for (int j = 0; j < D; ++j) o[j] = fmaf(w[q] * il, s_o[w0 + q][D * lane + j], o[j]);
      }
    M = mn;
    L = Ln;
  }
  T* dst = reinterpret_cast<T*>(a.out) + (long long)i * HD + D * lane;
#pragma unroll
  for (int j = 0; j < D; j += 2) store2(dst + j, o[j], o[j + 1]);
  if (a.lse && lane == 0) a.lse[i] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
}

// Warps a row, by the states that a row may have (workers over units, of which there are at least the tiles of all rows
// together for each KV head): what a warp does before its first state costs as much as some 30 states, so more than one
// pays where states are many and rows few. All of the attention, us with 1 / 4 / 8 / 16 warps a row: 28 rows (heads of
// one token) of up to 304 states 49.5 / 23.5 / 19.2 / 21.6 over 32,768 tokens, 12.7 / 9.7 / 9.9 / 11.1 over 1,024; 448 rows of up to 43
// 50.4 / 47.4; 896 rows of up to 38 17.9 / 20.4 over 128 tokens, 40.1 / 40.3 over 32,768.
template <typename T, int HD, int TR, int CH, int UC>
cudaError_t launch_combine(const Kv8AttnParams& a, int workers, cudaStream_t st) {
  const long long rows = (long long)a.r.n_rows * a.n_heads, group_rows = (long long)a.r.n_rows * (a.n_heads / a.c.n_kv_heads);
  const long long tiles = (group_rows + TR - 1) / TR;
  const long long states = workers / (tiles * a.c.n_kv_heads);
  if (states > 192)
    return kv8_launch(k_kv8_combine<T, HD, TR, CH, UC, 8>, dim3((unsigned)rows), dim3(256), 0, st, a, workers);
  if (states > 16 && rows <= 512) return kv8_launch(k_kv8_combine<T, HD, TR, CH, UC, 4>, dim3((unsigned)((rows + 1) / 2)), dim3(256), 0, st, a, workers);
  return kv8_launch(k_kv8_combine<T, HD, TR, CH, UC, 1>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, a, workers);
}

struct DeviceInfo {
  int sms, rows_ctas[4];  // resident CTAs of k_kv8_attn_rows per SM: bf16 64 / 128, fp32 64 / 128
};
PerDeviceOnce g_once;
DeviceInfo g_info[PerDeviceOnce::kMaxDevices];

template <typename T, int HD, int NS>
cudaError_t prepare_rows(int* per_sm) {
  cudaError_t e = cudaFuncSetAttribute(k_kv8_attn_rows<T, HD, NS>, cudaFuncAttributeMaxDynamicSharedMemorySize, w_smem<HD>());
  if (e != cudaSuccess) return e;
  e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(per_sm, k_kv8_attn_rows<T, HD, NS>, 32 * W_WARPS, w_smem<HD>());
  return e == cudaSuccess && *per_sm < 1 ? cudaErrorInvalidConfiguration : e;
}

template <int HD>
cudaError_t prepare_tile() {
  return cudaFuncSetAttribute(k_kv8_attn_tile<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, TLayout<HD>::TOTAL);
}

// Kernel attributes and sizes of the current device (set once per device).
const DeviceInfo* device_info() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return nullptr;
  const int rc = g_once.run(dev, [&]() -> int {
    DeviceInfo& d = g_info[dev];
    cudaError_t e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = prepare_rows<bf16, 64, 1>(&d.rows_ctas[0]);
    if (e == cudaSuccess) e = prepare_rows<bf16, 128, 1>(&d.rows_ctas[1]);
    if (e == cudaSuccess) e = prepare_rows<float, 64, 2>(&d.rows_ctas[2]);
    if (e == cudaSuccess) e = prepare_rows<float, 128, 2>(&d.rows_ctas[3]);
    if (e == cudaSuccess) e = prepare_tile<64>();
    if (e == cudaSuccess) e = prepare_tile<128>();
    return (int)e;
  });
  return rc == 0 ? &g_info[dev] : nullptr;
}

struct Form {
  bool tile;  // k_kv8_attn_tile
  int ctas, workers, tile_rows;
};
// The warp-level form where a KV head's query rows of a sequence fit its tile: it starts faster and wastes fewer rows. With
// more rows it reads the codes again for every 16, and the tile form leads as soon as there is much to read (which only the
// device knows). us of tile / warp-level form, 28 query heads on 4: one sequence of 3 rows (21 of a KV head) over 100 tokens
// 11.1 / 10.4, over 1,000 14.0 / 11.6, over 30,000 23.0 / 25.8; of 32 rows over 30,000 34.8 / 66.5; four of 18 rows over 30,000 55.1 /
// 129.6; sixteen of 3 rows over 1,000 21.3 / 18.1, of 8 rows 25.0 / 25.4. fp32 has the warp-level form alone: its two-term
// products are not what a cache of 8-bit codes is served with.
Form choose(const DeviceInfo& d, const jf_kv8_cache& c, const jf_kv8_rows& r, int dtype, int n_heads) {
  if (dtype == JF_BF16 && (long long)r.max_rows * (n_heads / c.n_kv_heads) > W_TR) return {true, d.sms, d.sms, T_TR};
  const int ctas = d.sms * d.rows_ctas[(dtype == JF_F32 ? 2 : 0) + (c.head_dim == 128 ? 1 : 0)];
  return {false, ctas, ctas * W_WARPS, W_TR};
}
size_t plan_bytes(const jf_kv8_cache& c) { return ((size_t)(c.n_seqs + 1) * 4 + 255) / 256 * 256; }

template <typename T, int HD, int NS>
cudaError_t launch_rows(const Kv8AttnParams& a, int ctas, cudaStream_t st) {
  cudaError_t e = kv8_launch(k_kv8_attn_rows<T, HD, NS>, dim3(ctas), dim3(32 * W_WARPS), w_smem<HD>(), st, a);
  if (e != cudaSuccess) return e;
  return launch_combine<T, HD, W_TR, W_CH, W_UC>(a, ctas * W_WARPS, st);
}

template <int HD>
cudaError_t launch_tile(const Kv8AttnParams& a, int ctas, cudaStream_t st) {
  const cudaError_t e = kv8_launch(k_kv8_attn_tile<HD>, dim3(ctas), dim3(T_THREADS), TLayout<HD>::TOTAL, st, a);
  return e != cudaSuccess ? e : launch_combine<bf16, HD, T_TR, T_CH, T_UC>(a, ctas, st);
}

}  // namespace
}  // namespace jf

using namespace jf;

extern "C" jf_status jf_op_kv8_attention_workspace_bytes(const jf_kv8_cache* cache, const jf_kv8_rows* rows, int dtype,
                                                         int n_heads, size_t* out_bytes) {
  const jf_status s = kv8_check(cache, rows);
  if (s != JF_OK) return s;
  if (!out_bytes || (dtype != JF_F32 && dtype != JF_BF16) || n_heads < 1 || n_heads % cache->n_kv_heads) return JF_EINVAL;
  const DeviceInfo* d = device_info();
  if (!d) return JF_ECUDA;
  const Form f = choose(*d, *cache, *rows, dtype, n_heads);
  *out_bytes = plan_bytes(*cache) + (size_t)2 * f.workers * f.tile_rows * (cache->head_dim + 2) * 4;
  return JF_OK;
}

extern "C" jf_status jf_op_kv8_attention(const jf_kv8_cache* cache, const jf_kv8_rows* rows, int dtype, const void* q,
                                         long long ld_q, int n_heads, float scale, const uint32_t* mask, int mask_words,
                                         void* out, float* lse, void* workspace, size_t workspace_bytes, int* err_word,
                                         void* cuda_stream) {
  jf_status s = kv8_check(cache, rows);
  if (s != JF_OK) return s;
  if ((dtype != JF_F32 && dtype != JF_BF16) || !err_word || n_heads < 1 || n_heads % cache->n_kv_heads) return JF_EINVAL;
  if (ld_q < (long long)n_heads * cache->head_dim || !(scale == scale)) return JF_EINVAL;
  if (rows->n_rows == 0) return JF_OK;
  const uintptr_t type_mask = dtype == JF_BF16 ? 1 : 3;
  if (!q || !out || ((uintptr_t)q & type_mask) || ((uintptr_t)out & 15) || ((uintptr_t)workspace & 15)) return JF_EINVAL;
  if (mask && (mask_words < 1 || (long long)mask_words * 32 < rows->max_rows)) return JF_EINVAL;
  {  // chunks and rows are counted in 32 bits
    const long long group_rows = (long long)rows->n_rows * (n_heads / cache->n_kv_heads);
    const long long units = (group_rows / W_TR + cache->n_seqs) * cache->n_kv_heads;
    const long long chunks = (long long)cache->pages_per_seq * kPage / W_CH + 1 + W_UC;
    if (group_rows * cache->n_kv_heads > 0x3fffffffll || units > 0x7fffffffll / chunks) return JF_EUNSUPPORTED;
  }
  size_t need = 0;
  s = jf_op_kv8_attention_workspace_bytes(cache, rows, dtype, n_heads, &need);
  if (s != JF_OK) return s;
  if (!workspace || workspace_bytes < need) return JF_ENOMEM;
  const DeviceInfo* d = device_info();
  if (!d) return JF_ECUDA;
  const Form f = choose(*d, *cache, *rows, dtype, n_heads);
  Kv8AttnParams a = {*cache, *rows, q, ld_q, n_heads, scale * 1.4426950408889634f, mask, mask_words, out, lse,
                     reinterpret_cast<int*>(workspace),
                     reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + plan_bytes(*cache)), err_word};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (f.tile)
    e = cache->head_dim == 128 ? launch_tile<128>(a, f.ctas, st) : launch_tile<64>(a, f.ctas, st);
  else if (dtype == JF_BF16)
    e = cache->head_dim == 128 ? launch_rows<bf16, 128, 1>(a, f.ctas, st) : launch_rows<bf16, 64, 1>(a, f.ctas, st);
  else
    e = cache->head_dim == 128 ? launch_rows<float, 128, 2>(a, f.ctas, st) : launch_rows<float, 64, 2>(a, f.ctas, st);
  return e == cudaSuccess ? JF_OK : JF_ECUDA;
}
