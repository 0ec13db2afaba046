// Attention of a batch of requests over the prefix they share and each one's paged tail.
//
// A query head's rows of one key-value head h are numbered rho = (token) * G + (head in its
// group), so that all rows that read head h stand side by side: those of the whole batch for
// the prefix, those of one request for its tail.  Both parts are cut into runs of tokens, each
// run keeps a reference m near the largest score (in units of log2), the sum l of exp2(s - m) and
// the sum of exp2(s - m) v, and the last kernel joins the runs of a row.
//
//  * few:  at most 16 NQ rows.  Reading the keys and values bounds it, so the four waves of a
//    workgroup take different tokens of the run, keys go from memory straight into the matrix
//    operand, and only the values pass through LDS (a region of the wave's own) to be transposed.
//  * many: 64 NQ rows a workgroup, which share the tiles of keys and values in LDS: the
//    prefix is read once per row tile instead of once per request, and the matrix cores bound it.
//  * k_join: the runs of a row.
// k_runs holds few and many, for the prefix and for the tails, in one launch.  A short call is one
// launch altogether: k_whole is few on a request's prefix and tail, and ends with its output.
//
// Products are formed transposed, S^T = K Q^T and O^T = V^T P^T: the matrix instruction then
// leaves the scores of 4 neighbouring tokens of one query in a lane, which are the weights that
// the second product's operand wants there, so no weight ever moves between lanes.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace {

constexpr int NT = 256, WAVES = NT / 64;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef short s4_t __attribute__((ext_vector_type(4)));

// Geometry in bytes: a row of D elements is CH pieces of 16 bytes; piece 4 s + g belongs to the
// s-th matrix step and to lanes 16 g .. 16 g + 15.
template <int D, class T>
struct Geo {
  static constexpr int RB = D * (int)sizeof(T), CH = RB / 16, KS = RB / 64, FT = D / 16;
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int SUB = BF ? 2 : 1, TPW = 16 * SUB;   // groups of 16 tokens, tokens, of a wave's step
  static constexpr int TILE = BF ? 64 : 32;                // tokens of a shared tile
  // Bytes of a row in LDS, padded so that what one instruction reads falls in distinct banks and
  // every address is a lane's base plus a constant: 16 rows x 16 bytes of keys; of values 8 rows x
  // 32 bytes by the transposed reads (bf16), rows 4 apart x 64 bytes (fp32).
  static constexpr int KP = RB + 32, VP = RB + (BF ? 32 : 16);
};

template <class T>
JOLT_DEV f4_t product_step(ju4 a, ju4 b, f4_t c) {
  if constexpr (sizeof(T) == 2) {
    b8_t x, y;
    __builtin_memcpy(&x, &a, 16);
    __builtin_memcpy(&y, &b, 16);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    return c;
  }
}

JOLT_DEV float max4(f4_t x) { return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])); }
// over the four lanes that hold one query (n16, n16 + 16, ...)
JOLT_DEV float over_groups_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
JOLT_DEV float over_groups_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// ------------------------------------------------------------------------------- rows and runs
// Packed rows of a request and the tokens of its tail.  Lengths and starts are device data:
// whatever they hold, 0 <= q0 <= q1 <= n_tok and 0 <= len <= max_pages * page_size, and a
// request with more rows than the call's bound has none.
struct Req { int q0, n, len; };
JOLT_DEV Req request(const PrefixAttendArgs &a, int r) {
  Req x;
  x.q0 = min(max(a.q_start[r], 0), a.n_tok);
  x.n = min(max(a.q_start[r + 1], x.q0), a.n_tok) - x.q0;
  if (x.n > a.max_new) x.n = 0;
  x.len = a.table ? min(max(a.kv_len[r], 0), a.max_pages << a.tail.shift) : 0;
  return x;
}

// Runs of the requests that few() serves: of equal length (a multiple of a wave's step), about
// FEW_WAVES runs of a head over all heads besides one a request, in the requests' order.  Every
// workgroup forms the sums for itself, from one read of the lengths.  2048 waves, two a SIMD, and
// runs down to one step: with 512, 1024, 2048 and 4096 waves the tails of 256 requests of 148
// tokens take 82, 60, 56 and 54 us, 12 of 1700 tokens 34, 35, 31 and 38; with runs of at least 128
// tokens 32 fp32 requests of 45 take 22 us a call, 14 with runs of 32.  A run of the prefix is
// four waves' (RUN_PREFIX): of 512 tokens instead, 4096 tokens under 16 rows take 16 us, not 12.
constexpr int FEW_WAVES = 2048, RUN_MIN = 32, RUN_STEP = 32, RUN_PREFIX = 128;
JOLT_DEV int few_run(int64_t total, int heads) {
  const int64_t c = (total * heads + FEW_WAVES - 1) / FEW_WAVES;
  const int64_t in_range = min(max(c, (int64_t)RUN_MIN), (int64_t)1 << 30);   // no tail is longer
  return (int)((in_range + RUN_STEP - 1) / RUN_STEP * RUN_STEP);
}

// What the join needs to know of a packed row: its place in its request, whose runs are items
// first .. first + count - 1 of few() (kind 0) or the splits of many() (kind 1); kind -1: the row
// is of no request.
struct RowEntry { int first, count, place, kind; };

struct Found { int r, idx, run; Req x; };
template <int W>
struct FindLds {
  int64_t sum[WAVES];
  int cnt[WAVES];
  Found at[W];
};
// Items want[0 .. W - 1] of the call (kind 0: runs of few's requests, kind 1: row tiles of
// many's): their requests and places there, or r = -1 past the last.
template <int KIND, int W>
JOLT_DEV void find_items(const PrefixAttendArgs &a, const int (&want)[W], int limit, int rows_tile, RowEntry *entries, FindLds<W> &sm) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.n_req + NT - 1) / NT, r0 = min(tid * per, a.n_req), r1 = min(r0 + per, a.n_req);
  Req x0{0, 0, 0};
  if (r0 < r1) x0 = request(a, r0);
  auto at = [&](int r) { return r == r0 ? x0 : request(a, r); };
  int run = RUN_MIN;
  if constexpr (KIND == 0) {
    int64_t total = 0;
    for (int r = r0; r < r1; ++r) {
      const Req x = at(r);
      if (x.n > 0 && x.n * a.group <= limit) total += x.len;
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) total += __shfl_xor(total, m, 64);
    if (lane == 0) sm.sum[wave] = total;
    __syncthreads();
    total = 0;
    for (int i = 0; i < WAVES; ++i) total += sm.sum[i];
    run = few_run(total, a.heads);
  }
  auto count = [&](const Req &x) {
    const int rows = x.n * a.group;
    if constexpr (KIND == 0) return x.n > 0 && rows <= limit ? (x.len + run - 1) / run : 0;
    else return rows > limit ? (rows + rows_tile - 1) / rows_tile : 0;
  };
  int mine = 0;
  for (int r = r0; r < r1; ++r) mine += count(at(r));
  int incl = mine;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int u = __shfl_up(incl, m, 64);
    if (lane >= m) incl += u;
  }
  if (lane == 63) sm.cnt[wave] = incl;
  if (tid < W) sm.at[tid].r = -1;
  __syncthreads();
  int before = incl - mine;
  for (int w = 0; w < wave; ++w) before += sm.cnt[w];
  bool here = false;
#pragma unroll
  for (int w = 0; w < W; ++w) here |= want[w] >= before && want[w] < before + mine;
  if (here) {
    int b = before;
    for (int r = r0; r < r1; ++r) {
      const Req x = at(r);
      const int c = count(x);
#pragma unroll
      for (int w = 0; w < W; ++w)
        if (want[w] >= b && want[w] < b + c) sm.at[w] = Found{r, want[w] - b, run, x};
      b += c;
    }
  }
  if (entries) {
    // rows outside q_start[0] .. q_start[n_req], then every request's: a lane its own where they
    // are few, the wave together where they are many
    const int s0 = min(max(a.q_start[0], 0), a.n_tok), s1 = min(max(a.q_start[a.n_req], 0), a.n_tok);
    for (int t = tid; t < s0; t += NT) entries[t].kind = -1;
    for (int t = s1 + tid; t < a.n_tok; t += NT) entries[t].kind = -1;
    for (int i = 0; i < per; ++i) {
      const int r = r0 + i;
      Req x{0, 0, 0};
      int n_all = 0, c = 0;
      if (r < r1) {
        x = at(r);
        n_all = min(max(a.q_start[r + 1], x.q0), a.n_tok) - x.q0;   // with those past the bound
        c = count(x);
      }
      RowEntry e{before, c, 0, n_all > x.n ? -1 : x.n * a.group <= limit ? 0 : 1};
      before += c;
      if (n_all <= 8)
        for (int k = 0; k < n_all; ++k) { e.place = k; entries[x.q0 + k] = e; }
      for (uint64_t m = __ballot(n_all > 8); m; m &= m - 1) {
        const int src = __builtin_ctzll(m);
        const int q0 = __shfl(x.q0, src, 64), nn = __shfl(n_all, src, 64);
        RowEntry f{__shfl(e.first, src, 64), __shfl(e.count, src, 64), 0, __shfl(e.kind, src, 64)};
        for (int k = lane; k < nn; k += 64) { f.place = k; entries[q0 + k] = f; }
      }
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------------------------- one wave's rows
// 16 NQ rows of a wave: query operands, and the running softmax and output.  A lane holds for
// query n16 of each group the features 16 ft + 4 g .. + 3.
template <int D, class T, int NQ>
struct Rows {
  using G = Geo<D, T>;
  ju4 q[NQ][G::KS];
  f4_t o[G::FT][NQ];
  float m[NQ], l[NQ];        // reference in units of log2 (all lanes of the query), this lane's part of the sum
  int seen[NQ];              // tail: tokens the lane's query sees

  JOLT_DEV void clear() {
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      m[x] = -INFINITY;
      l[x] = 0.f;
#pragma unroll
      for (int f = 0; f < G::FT; ++f) o[f][x] = f4_t{0, 0, 0, 0};
    }
  }
  // rows rho0 + 16 x + n16 below n_rows, of the packed rows from t0 on; others are zero
  JOLT_DEV void load(const PrefixAttendArgs &a, int h, int t0, int rho0, int n_rows, int n16, int g) {
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      const int rho = rho0 + 16 * x + n16;
      if (rho < n_rows) {
        const int t = t0 + rho / a.group, j = h * a.group + rho % a.group;
        const uint8_t *p = static_cast<const uint8_t *>(a.Q) + ((int64_t)t * a.q_stride + (int64_t)j * D) * sizeof(T) + 16 * g;
#pragma unroll
        for (int s = 0; s < G::KS; ++s) q[x][s] = gload_u4(p + 64 * s);
      } else {
#pragma unroll
        for (int s = 0; s < G::KS; ++s) q[x][s] = ju4{0, 0, 0, 0};
      }
    }
  }
  // Scores s (16 SUBS tokens) into weights, in place.  The reference m of exp2(s c - m) need not
  // be the running maximum, only near it: it is kept while a lane's weights of a step sum to at most
  // 1 (a weight's precision does not depend on its size), so that most tiles need no maximum, no
  // exchange between lanes and no rescaling.  The first tile (m = -inf gives an infinite sum) and
  // one that outgrows m set it HEAD above the maximum and rescale: weights then start at 2^-8, and
  // what follows may score 8 higher before m moves again.  No weight is ever above 1, so that sums
  // of values overflow only where those of the plain softmax could; with the maximum itself as
  // reference and weights of up to 2^16, values of 1e37 gave infinite sums.  Values below 2^-118 meet
  // weights small enough to lose bits of fp32 (never those of bf16); with 2^-16 those below 2^-110 did.
  static constexpr float HEAD = 8.f;
  template <int SUBS>
  JOLT_DEV void softmax(f4_t (&s)[SUBS][NQ], float c) {
    f4_t p[SUBS][NQ];
    float sum[NQ];
    bool far = false;
    auto weigh = [&](int x) {
      const float base = m[x] == -INFINITY ? 0.f : m[x];
      sum[x] = 0.f;
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[u][x][i] = __builtin_amdgcn_exp2f(fmaf(s[u][x][i], c, -base));
          sum[x] += p[u][x][i];
        }
    };
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      weigh(x);
      far |= !(sum[x] <= 1.f) || m[x] == -INFINITY;
    }
    if (__builtin_expect(__any(far), 0)) {
#pragma unroll
      for (int x = 0; x < NQ; ++x) {
        // only where this query's own lanes say so: no row's rounding depends on another's values
        const bool mine = !(sum[x] <= 1.f) || m[x] == -INFINITY;
        float mx = max4(s[0][x]);
#pragma unroll
        for (int u = 1; u < SUBS; ++u) mx = fmaxf(mx, max4(s[u][x]));
        mx = fmaxf(m[x], over_groups_max(mx) * c + HEAD);
        if (over_groups_max(mine ? 1.f : 0.f) == 0.f) mx = m[x];
        // nothing seen so far: both are -inf, and nothing is there to rescale
        const float al = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[x] - mx);
        l[x] *= al;
#pragma unroll
        for (int f = 0; f < G::FT; ++f) o[f][x] *= al;
        m[x] = mx;
        weigh(x);
      }
    }
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      l[x] += sum[x];
#pragma unroll
      for (int u = 0; u < SUBS; ++u) s[u][x] = p[u][x];
    }
  }
  // o += V^T P^T for 16 SUBS tokens whose values stand in LDS.  For the bf16 product (values are
  // bf16 already) a weight is the sum of two bf16 terms, its upper half and the rest, right to 2^-15: the
  // output's error is that of its own rounding.  One term, the weight rounded, makes it 1.2 .. 1.4
  // times that, and takes 196 us for 256 requests on 32768 tokens, not 224, and 115 for 1025 prompt
  // rows on 4096, not 133; calls that memory bounds take the same (64 requests on 4096 tokens 24.3 us).
  // ABOVE_ONE adds 2^-23 of the weight to the rest, so that it is above zero wherever the weight is and
  // times an infinite value no NaN.
  static constexpr float ABOVE_ONE = 1.f + 0x1p-23f;
  template <int SUBS>
  JOLT_DEV void values(const f4_t (&p)[SUBS][NQ], const uint8_t *v, int n16, int g) {
    if constexpr (G::BF) {
#pragma unroll
      for (int u = 0; u < SUBS; u += 2) {
        b8_t w[NQ], rest[NQ];
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
          uint32_t d[4], r[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float y = p[u + i / 2][x][2 * (i % 2)], z = p[u + i / 2][x][2 * (i % 2) + 1];
            const uint32_t yb = __float_as_uint(y), zb = __float_as_uint(z);
            d[i] = __builtin_amdgcn_perm(zb, yb, 0x07060302u);   // the upper halves
            r[i] = pack_bf16(fmaf(y, ABOVE_ONE, -__uint_as_float(yb & 0xffff0000u)), fmaf(z, ABOVE_ONE, -__uint_as_float(zb & 0xffff0000u)));
          }
          __builtin_memcpy(&w[x], d, 16);
          __builtin_memcpy(&rest[x], r, 16);
        }
        const uint8_t *base = v + (4 * g + (n16 >> 2)) * G::VP + 8 * (n16 & 3);
#pragma unroll
        for (int f = 0; f < G::FT; ++f) {
          auto *pa = base + 16 * u * G::VP + 32 * f;
          auto *pb = pa + 16 * G::VP;
          const s4_t xa = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t *)pa);
          const s4_t xb = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t *)pb);
          const auto xv = __builtin_shufflevector(xa, xb, 0, 1, 2, 3, 4, 5, 6, 7);
          b8_t va;
          __builtin_memcpy(&va, &xv, 16);
#pragma unroll
          for (int x = 0; x < NQ; ++x) o[f][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, w[x], o[f][x], 0, 0, 0);
#pragma unroll
          for (int x = 0; x < NQ; ++x) o[f][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, rest[x], o[f][x], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint8_t *base = v + 4 * g * G::VP + 4 * n16;
#pragma unroll
          for (int f = 0; f < G::FT; ++f) {
            const float va = *reinterpret_cast<const float *>(base + (16 * u + i) * G::VP + 64 * f);
#pragma unroll
            for (int x = 0; x < NQ; ++x) o[f][x] = __builtin_amdgcn_mfma_f32_16x16x4f32(va, p[u][x][i], o[f][x], 0, 0, 0);
          }
        }
    }
  }
  // Values that are not finite, in a tile that some rows see in part only: a weight of zero
  // would not keep them out of the product of a row that does not see them.  They are added
  // here to the rows that do, and replaced by zero for the product.
  template <int ROWS>
  JOLT_DEV void add_nonfinite(const uint8_t *v, int x0, int n16, int g) {
    for (int k = 0; k < ROWS; ++k)
#pragma unroll
      for (int f = 0; f < G::FT; ++f) {
        const int e0 = 16 * f + 4 * g;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int byte = (e0 + i) * (int)sizeof(T);
          const T raw = *reinterpret_cast<const T *>(v + k * G::VP + byte);
          float val;
          if constexpr (G::BF) val = bf16_to_f32(raw); else val = raw;
#pragma unroll
          for (int x = 0; x < NQ; ++x)
            if (!(fabsf(val) < INFINITY) && x0 + k < seen[x]) o[f][x][i] += val;
        }
      }
  }
};

// whether the 16 bytes hold a value that is not finite; and the same with those replaced by zero
template <class T>
JOLT_DEV bool nonfinite(ju4 v) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2)
      bad |= (v[i] & 0x7f80u) == 0x7f80u || (v[i] & 0x7f800000u) == 0x7f800000u;
    else
      bad |= (v[i] & 0x7f800000u) == 0x7f800000u;
  }
  return bad;
}
template <class T>
JOLT_DEV ju4 finite_or_zero(ju4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
      if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0xffffu;
    } else {
      if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] = 0;
    }
  }
  return v;
}

// Byte offset of token x's row of head h, and whether it is there (x < end and its page in the
// pool); a token that is not reads a row that is.
struct RowAt { int64_t off; bool ok; };
JOLT_DEV int page_of(const PrefixSource &s, const int32_t *row, int x, int end) {
  return row ? row[min(x, end - 1) >> s.shift] : 0;
}
JOLT_DEV RowAt row_at(const PrefixSource &s, int page, int h, int x, int end, int esz) {
  const bool in = (uint32_t)page < (uint32_t)s.n_pages;
  const int at = min(x, end - 1) & ((1 << s.shift) - 1);
  return RowAt{((in ? page : 0) * s.s_page + (int64_t)at * s.s_tok + h * s.s_head) * esz, in && x < end};
}

// Where the runs' results go: [run][row] of D floats, and m and l of each.
struct Parts {
  float *o;
  float2 *ml;
};

// ------------------------------------------------------------------------------- few rows
// A workgroup takes one run of the prefix, its waves every fourth step of it, and joins their
// results; of the tails, which are short, every wave takes a run of its own.
struct FewArgs {
  Parts out;
  RowEntry *entries;        // tails: [n_tok]
  int32_t rows;             // rows kept per run and head: row rho of head h at (item * heads + h) * rows + rho
  int32_t limit;            // tails: requests of at most this many rows per head
  int32_t run;              // prefix: tokens of a run
};

template <int D, class T, int NQ>
struct FewLds {
  static constexpr int VB = Geo<D, T>::TPW * Geo<D, T>::VP, OB = 16 * NQ * D * 4;   // a wave's values, its output
  static constexpr int WB = VB > OB ? VB : OB;
  uint8_t w[WAVES][WB];
  float m[WAVES][16 * NQ], l[WAVES][16 * NQ];
  FindLds<WAVES> f;
};

// Features e .. e + 3 of row t, query head j, from the joined sum o, reference M and sum l.
template <int D, class T>
JOLT_DEV void write_row(const PrefixAttendArgs &a, int t, int j, int e, f4_t o, float M, float l, bool first) {
  T *O = static_cast<T *>(a.O) + (int64_t)t * a.o_stride + (int64_t)j * D + e;
  o *= l == 0.f ? 0.f : 1.f / l;
  if constexpr (sizeof(T) == 4) gstore_f4(O, o);
  else *reinterpret_cast<uint2 *>(O) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
  if (a.lse && first) a.lse[(int64_t)t * a.n_q + j] = l == 0.f ? -INFINITY : (M + log2f(l)) * LN2;
}

// What few() takes: runs of the prefix, runs of the tails, or requests as a whole, the prefix and
// then the tail, with their output.
enum { FEW_PREFIX = 0, FEW_TAIL, FEW_WHOLE };

template <int D, class T, int NQ, int MODE>
JOLT_DEV void few(const PrefixAttendArgs &a, const FewArgs &p, int block, FewLds<D, T, NQ> &sm) {
  using G = Geo<D, T>;
  constexpr bool TAIL = MODE != FEW_PREFIX, OWN = MODE == FEW_TAIL, WHOLE = MODE == FEW_WHOLE;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n16 = lane & 15, g = lane >> 4;
  const int id = OWN ? block * WAVES + wave : block;       // item (WHOLE: request) * heads + h
  const int h = id % a.heads, item = id / a.heads;
  constexpr int STRIDE = OWN ? G::TPW : WAVES * G::TPW;    // tokens from a wave's step to its next
  int t0, n, first, end, len = 0;
  int tail0 = 0;                     // the tail's token 0 in the run's count: WHOLE, after the prefix's last step
  const int32_t *pages = nullptr;
  if constexpr (OWN) {
    int want[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) want[w] = (block * WAVES + w) / a.heads;
    find_items<0, WAVES>(a, want, p.limit, 0, block == 0 ? p.entries : nullptr, sm.f);
    const Found f = sm.f.at[wave];
    if (f.r < 0) return;
    t0 = f.x.q0;
    n = f.x.n;
    len = f.x.len;
    first = f.idx * f.run;
    end = min(len, first + f.run);
    pages = a.table + (int64_t)f.r * a.max_pages;
  } else if constexpr (WHOLE) {
    const Req x = request(a, item);
    if (x.n == 0) return;
    t0 = x.q0;
    n = x.n;
    len = x.len;
    first = 0;
    tail0 = (a.T + G::TPW - 1) / G::TPW * G::TPW;
    end = tail0 + len;
    pages = a.table + (int64_t)item * a.max_pages;
  } else {
    t0 = 0;
    n = a.n_tok;
    first = item * p.run;
    end = min(a.T, first + p.run);
  }
  const int n_rows = n * a.group;
  Rows<D, T, NQ> R;
  R.load(a, h, t0, 0, n_rows, n16, g);
  R.clear();
  int seen_all = 0x7fffffff;         // tokens that every row sees
  if constexpr (TAIL) {
#pragma unroll
    for (int c = 0; c < NQ; ++c) {
      const int rho = 16 * c + n16;
      R.seen[c] = rho < n_rows ? max(0, len - n + rho / a.group + 1) : 0x7fffffff;
    }
    seen_all = max(0, len - n + 1);
  }
  const float c = a.scale * LOG2E;
  uint8_t *vl = sm.w[wave];
  ju4 kr[G::SUB][G::KS], vr[G::SUB][G::KS];
  RowAt at[G::SUB];
  int pg[G::SUB];
  const int x0 = first + (OWN ? 0 : wave * G::TPW);
  // whether the step at x is of the tail; it is of one part as a whole
  auto of_tail = [&](int x) { return OWN || (WHOLE && x >= tail0); };
  auto ask_pages = [&](int x) {
    if (of_tail(x))
#pragma unroll
      for (int u = 0; u < G::SUB; ++u) pg[u] = page_of(a.tail, pages, x - tail0 + 16 * u + n16, OWN ? end : len);
  };
  auto place = [&](int x) {
    const bool tail = of_tail(x);
#pragma unroll
    for (int u = 0; u < G::SUB; ++u)
      at[u] = tail ? row_at(a.tail, pg[u], h, x - tail0 + 16 * u + n16, OWN ? end : len, sizeof(T))
                   : row_at(a.prefix, 0, h, x + 16 * u + n16, WHOLE ? a.T : end, sizeof(T));
  };
  auto load = [&](bool values, int x, ju4 (&d)[G::SUB][G::KS]) {
    const PrefixSource &src = of_tail(x) ? a.tail : a.prefix;
    const uint8_t *base = static_cast<const uint8_t *>(values ? src.V : src.K);
#pragma unroll
    for (int u = 0; u < G::SUB; ++u)
#pragma unroll
      for (int s = 0; s < G::KS; ++s) d[u][s] = gload_u4(base + at[u].off + 64 * s + 16 * g);
  };
  if (x0 < end) {
    ask_pages(x0);
    place(x0);
    load(false, x0, kr);
    load(true, x0, vr);
    if (x0 + STRIDE < end) ask_pages(x0 + STRIDE);
  }
  for (int x = x0; x < end; x += STRIDE) {
    f4_t s[G::SUB][NQ];
#pragma unroll
    for (int u = 0; u < G::SUB; ++u)
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        s[u][q] = f4_t{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < G::KS; ++k) s[u][q] = product_step<T>(kr[u][k], R.q[q][k], s[u][q]);
      }
    uint32_t okm[G::SUB];           // bit k: token 16 u + k is there
    bool whole = true;
#pragma unroll
    for (int u = 0; u < G::SUB; ++u) {
      okm[u] = (uint32_t)__ballot(at[u].ok) & 0xffffu;
      whole &= okm[u] == 0xffffu;
    }
    const bool tail = of_tail(x), partly = tail && x - tail0 + G::TPW > seen_all;   // some row does not see all of it
    bool mine[G::SUB];
#pragma unroll
    for (int u = 0; u < G::SUB; ++u) mine[u] = at[u].ok;
    const int xn = x + STRIDE;
    const bool more = xn < end;
    if (more) {
      place(xn);
      load(false, xn, kr);
      if (xn + STRIDE < end) ask_pages(xn + STRIDE);
    }
    if (!whole || partly) {
#pragma unroll
      for (int u = 0; u < G::SUB; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 4 * g + i;
          const bool there = (okm[u] >> k) & 1;
#pragma unroll
          for (int q = 0; q < NQ; ++q)
            if (!there || (TAIL && tail && x - tail0 + 16 * u + k >= R.seen[q])) s[u][q][i] = -INFINITY;
        }
      // a value that is not there must not be NaN either
#pragma unroll
      for (int u = 0; u < G::SUB; ++u)
        if (!mine[u])
#pragma unroll
          for (int k = 0; k < G::KS; ++k) vr[u][k] = ju4{0, 0, 0, 0};
    }
    R.softmax(s, c);
    // the wave's LDS operations run in order: the fences only keep the compiler from moving them
    auto put = [&]() {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int u = 0; u < G::SUB; ++u)
#pragma unroll
        for (int k = 0; k < G::KS; ++k) {
          *reinterpret_cast<ju4 *>(vl + (16 * u + n16) * G::VP + 64 * k + 16 * g) = vr[u][k];
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    put();
    if (TAIL && partly) {
      bool bad = false;
#pragma unroll
      for (int u = 0; u < G::SUB; ++u)
#pragma unroll
        for (int k = 0; k < G::KS; ++k) bad |= nonfinite<T>(vr[u][k]);
      if (__any(bad)) {
        R.template add_nonfinite<G::TPW>(vl, x - tail0, n16, g);
#pragma unroll
        for (int u = 0; u < G::SUB; ++u)
#pragma unroll
          for (int k = 0; k < G::KS; ++k) vr[u][k] = finite_or_zero<T>(vr[u][k]);
        put();
      }
    }
    if (more) load(true, xn, vr);
    R.values(s, vl, n16, g);
  }
  const int64_t base = (int64_t)id * p.rows;
  if constexpr (OWN) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const float l = over_groups_sum(R.l[q]);
      const int rho = 16 * q + n16;
      if (rho < n_rows) {
#pragma unroll
        for (int f = 0; f < G::FT; ++f) *reinterpret_cast<f4_t *>(p.out.o + (base + rho) * D + 16 * f + 4 * g) = R.o[f][q];
        if (g == 0) p.out.ml[base + rho] = make_float2(R.m[q], l);
      }
    }
    return;
  }
  // the waves' results join in LDS
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const float l = over_groups_sum(R.l[q]);
    if (g == 0) { sm.m[wave][16 * q + n16] = R.m[q]; sm.l[wave][16 * q + n16] = l; }
#pragma unroll
    for (int f = 0; f < G::FT; ++f)
      *reinterpret_cast<f4_t *>(vl + ((16 * q + n16) * D + 16 * f + 4 * g) * 4) = R.o[f][q];
  }
  __syncthreads();
  for (int i = tid; i < n_rows * (D / 4); i += NT) {
    const int row = i / (D / 4), e = (i % (D / 4)) * 4;
    float M = sm.m[0][row];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sm.m[w][row]);
    f4_t o = {0, 0, 0, 0};
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float al = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm.m[w][row] - M);
      if (sm.m[w][row] != -INFINITY || sm.l[w][row] != 0.f) {
        l = fmaf(sm.l[w][row], al, l);
        o += *reinterpret_cast<const f4_t *>(sm.w[w] + (row * D + e) * 4) * al;
      }
    }
    if constexpr (WHOLE) {
      const int t = t0 + row / a.group, j = h * a.group + row % a.group;
      write_row<D, T>(a, t, j, e, o, M, l, e == 0);
    } else {
      *reinterpret_cast<f4_t *>(p.out.o + (base + row) * D + e) = o;
      if (e == 0) p.out.ml[base + row] = make_float2(M, l);
    }
  }
}

// ------------------------------------------------------------------------------- many rows
// The prefix's work of a head, (row tile, tile of keys and values) pairs in that order, is cut into
// equal pieces of `share` pairs, a workgroup each: a workgroup ends one row tile and starts the
// next, so that all have the same work whatever the row tiles are.  A row tile's run from its
// s-th workgroup goes to slab s.  The tails' row tiles are cut into `splits` runs each.
struct ManyArgs {
  Parts out;                // [slab][packed row][query head]
  int32_t splits, tiles;    // tails: runs of a row tile, most row tiles of the call; prefix: row tiles
  int32_t limit;            // tails: requests of more rows per head than this
  int64_t share;            // prefix
};

template <int D, class T>
struct ManyLds {
  uint8_t k[2][Geo<D, T>::TILE * Geo<D, T>::KP], v[2][Geo<D, T>::TILE * Geo<D, T>::VP];   // [buffer]
  int there[2][Geo<D, T>::TILE];
  int flag[2];
  FindLds<1> f;
};

template <int D, class T, int NQ, bool TAIL>
JOLT_DEV void many(const PrefixAttendArgs &a, const ManyArgs &p, int block, ManyLds<D, T> &sm) {
  using G = Geo<D, T>;
  constexpr int RT = 64 * NQ, SUBS = G::TILE / 16;
  constexpr int PASS = NT / G::CH, LOADS = G::TILE / PASS;   // rows of a load, loads of a tile
  static_assert(G::TILE % PASS == 0, "a tile is whole loads");
  const PrefixSource &src = TAIL ? a.tail : a.prefix;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n16 = lane & 15, g = lane >> 4;
  const int h = block % a.heads, rest = block / a.heads;
  // prefix: pairs at .. pairs_end - 1; tails: one run
  const int kv_tiles = TAIL ? 1 : (a.T + G::TILE - 1) / G::TILE;
  int64_t at = TAIL ? 0 : rest * p.share;
  const int64_t pairs_end = TAIL ? 1 : min(at + p.share, (int64_t)p.tiles * kv_tiles);
  Found found{};
  if constexpr (TAIL) {
    const int want[1] = {rest % p.tiles};
    find_items<1, 1>(a, want, p.limit, RT, nullptr, sm.f);
    found = sm.f.at[0];
    if (found.r < 0) return;
  }
  while (at < pairs_end) {
    int t0, n, len, tail_len = 0, rho0, slab, first, end, seen_all = 0x7fffffff;
    const int32_t *pages = nullptr;
    if constexpr (TAIL) {
      t0 = found.x.q0;
      n = found.x.n;
      tail_len = found.x.len;
      rho0 = found.idx * RT;
      // the tile's last row sees most, its first least
      len = max(0, tail_len - n + min(n, (rho0 + RT - 1) / a.group + 1));
      seen_all = max(0, tail_len - n + rho0 / a.group + 1);
      pages = a.table + (int64_t)found.r * a.max_pages;
      const int run = ((len + p.splits - 1) / p.splits + G::TILE - 1) / G::TILE * G::TILE;
      slab = rest / p.tiles;
      first = slab * run;
      end = min(len, first + run);
      at = pairs_end;
    } else {
      t0 = 0;
      n = a.n_tok;
      const int tile = (int)(at / kv_tiles), k0 = (int)(at - (int64_t)tile * kv_tiles);
      const int k1 = (int)min((int64_t)kv_tiles, k0 + (pairs_end - at));
      rho0 = tile * RT;
      slab = rest - (int)((int64_t)tile * kv_tiles / p.share);
      first = k0 * G::TILE;
      end = min(a.T, k1 * G::TILE);
      at += k1 - k0;
    }
    const int n_rows = n * a.group;
    Rows<D, T, NQ> R;
    const int rho_w = rho0 + wave * 16 * NQ;
    R.load(a, h, t0, rho_w, n_rows, n16, g);
    R.clear();
    if constexpr (TAIL) {
#pragma unroll
      for (int c = 0; c < NQ; ++c) {
        const int rho = rho_w + 16 * c + n16;
        R.seen[c] = rho < n_rows ? max(0, tail_len - n + rho / a.group + 1) : 0x7fffffff;
      }
    }
    const float c = a.scale * LOG2E;
    const uint8_t *Kb = static_cast<const uint8_t *>(src.K), *Vb = static_cast<const uint8_t *>(src.V);
    const int lrow = tid / G::CH, piece = tid % G::CH;
    ju4 kr[LOADS], vr[LOADS];
    int pg[LOADS];
    bool ok[LOADS];
    int64_t off[LOADS];                // prefix: the next tile's rows
    const int64_t tile_step = (int64_t)G::TILE * src.s_tok * (int)sizeof(T);
    if constexpr (!TAIL) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) off[i] = row_at(src, 0, h, first + i * PASS + lrow, 0x7fffffff, sizeof(T)).off + piece * 16;
    }
    auto ask_pages = [&](int x) {
      if constexpr (TAIL)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) pg[i] = page_of(src, pages, x + i * PASS + lrow, end);
    };
    auto load = [&](int x) {
      if constexpr (!TAIL)
        if (x + G::TILE <= end) {
#pragma unroll
          for (int i = 0; i < LOADS; ++i) {
            ok[i] = true;
            kr[i] = gload_u4(Kb + off[i]);
            vr[i] = gload_u4(Vb + off[i]);
            off[i] += tile_step;
          }
          return;
        }
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const RowAt at = row_at(src, TAIL ? pg[i] : 0, h, x + i * PASS + lrow, end, sizeof(T));
        ok[i] = at.ok;
        kr[i] = gload_u4(Kb + at.off + piece * 16);
        vr[i] = gload_u4(Vb + at.off + piece * 16);
      }
    };
    auto put = [&](int b, int x) {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int row = i * PASS + lrow;
        if ((TAIL || x + G::TILE > end) && !ok[i]) vr[i] = ju4{0, 0, 0, 0};
        *reinterpret_cast<ju4 *>(&sm.k[b][row * G::KP + piece * 16]) = kr[i];
        *reinterpret_cast<ju4 *>(&sm.v[b][row * G::VP + piece * 16]) = vr[i];
        if constexpr (TAIL) {
          if (piece == 0) sm.there[b][row] = ok[i];
          bad |= nonfinite<T>(vr[i]);
        }
      }
      if (TAIL && x + G::TILE > seen_all && bad) sm.flag[b] = 1;
    };
    if (TAIL && tid < 2) sm.flag[tid] = 0;
    if (first < end) {
      ask_pages(first);
      load(first);
      ask_pages(first + G::TILE);
      if (TAIL) __syncthreads();
      put(0, first);
      __syncthreads();
    }
    for (int x = first, b = 0; x < end; x += G::TILE, b ^= 1) {
      const bool more = x + G::TILE < end;
      if (more) {
        load(x + G::TILE);
        ask_pages(x + 2 * G::TILE);
      }
      const uint8_t *kl = sm.k[b] + n16 * G::KP + 16 * g;
      uint8_t *vl = sm.v[b];
      // a step's products of all tokens one after the other: no product waits for the one before it
      f4_t s[SUBS][NQ];
#pragma unroll
      for (int k = 0; k < G::KS; ++k)
#pragma unroll
        for (int u = 0; u < SUBS; ++u) {
          const ju4 ka = *reinterpret_cast<const ju4 *>(kl + 16 * u * G::KP + 64 * k);
#pragma unroll
          for (int q = 0; q < NQ; ++q) s[u][q] = product_step<T>(ka, R.q[q][k], k == 0 ? f4_t{0, 0, 0, 0} : s[u][q]);
        }
      if (TAIL || x + G::TILE > end) {
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = 16 * u + 4 * g + i;
            const bool in = TAIL ? sm.there[b][k] != 0 : x + k < end;
#pragma unroll
            for (int q = 0; q < NQ; ++q)
              if (!in || (TAIL && x + k >= R.seen[q])) s[u][q][i] = -INFINITY;
          }
      }
      R.softmax(s, c);
      if (TAIL && sm.flag[b]) {          // the same for all threads: written before the last barrier
        R.template add_nonfinite<G::TILE>(vl, x, n16, g);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int row = i * PASS + lrow;
          ju4 *at = reinterpret_cast<ju4 *>(vl + row * G::VP + piece * 16);
          *at = finite_or_zero<T>(*at);
        }
        if (tid == 0) sm.flag[b] = 0;
        __syncthreads();
      }
      R.values(s, vl, n16, g);
      if (more) put(b ^ 1, x + G::TILE);
      __syncthreads();
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const float l = over_groups_sum(R.l[q]);
      const int rho = rho_w + 16 * q + n16;
      if (rho < n_rows) {
        const int t = t0 + rho / a.group, j = h * a.group + rho % a.group;
        const int64_t row = ((int64_t)slab * a.n_tok + t) * a.n_q + j;
#pragma unroll
        for (int f = 0; f < G::FT; ++f) *reinterpret_cast<f4_t *>(p.out.o + row * D + 16 * f + 4 * g) = R.o[f][q];
        if (g == 0) p.out.ml[row] = make_float2(R.m[q], l);
      }
    }
  }
}

// ------------------------------------------------------------------------------- all runs
// One launch for the runs of the prefix and of the tails: the first fill the matrix cores while
// the others wait for memory, and no part waits for the last workgroup of another.
enum { ROLE_NONE = 0, ROLE_FEW1, ROLE_FEW2, ROLE_MANY1, ROLE_MANY2 };
struct RunArgs {
  PrefixAttendArgs a;
  FewArgs pre_few, few;
  ManyArgs pre_many, many;
  int32_t pre_role, few_role, many_role;
  int32_t n_pre, n_many, n_few;        // workgroups, in this order
};

template <int D, class T>
union RunLds {
  FewLds<D, T, 1> f1;
  FewLds<D, T, 2> f2;
  ManyLds<D, T> m;
};

template <int D, class T>
__global__ void __launch_bounds__(NT, 2) k_runs(const RunArgs p) {
  __shared__ __attribute__((aligned(16))) RunLds<D, T> sm;
  int b = blockIdx.x;
  if (b < p.n_pre) {
    if (p.pre_role == ROLE_FEW1) few<D, T, 1, FEW_PREFIX>(p.a, p.pre_few, b, sm.f1);
    else if (p.pre_role == ROLE_FEW2) few<D, T, 2, FEW_PREFIX>(p.a, p.pre_few, b, sm.f2);
    else if (p.pre_role == ROLE_MANY1) many<D, T, 1, false>(p.a, p.pre_many, b, sm.m);
    else many<D, T, 2, false>(p.a, p.pre_many, b, sm.m);
    return;
  }
  b -= p.n_pre;
  if (b < p.n_many) {
    if (p.many_role == ROLE_MANY1) many<D, T, 1, true>(p.a, p.many, b, sm.m);
    else many<D, T, 2, true>(p.a, p.many, b, sm.m);
    return;
  }
  b -= p.n_many;
  if (p.few_role == ROLE_FEW1) few<D, T, 1, FEW_TAIL>(p.a, p.few, b, sm.f1);
  else few<D, T, 2, FEW_TAIL>(p.a, p.few, b, sm.f2);
}

// Short calls in one launch: a workgroup a request and key-value head, from the prefix to the output.
template <int D, class T, int NQ>
__global__ void __launch_bounds__(NT, 2) k_whole(const PrefixAttendArgs a) {
  __shared__ __attribute__((aligned(16))) FewLds<D, T, NQ> sm;
  few<D, T, NQ, FEW_WHOLE>(a, FewArgs{}, blockIdx.x, sm);
}

// ------------------------------------------------------------------------------- join
struct JoinArgs {
  PrefixAttendArgs a;
  Parts prefix, few, many;
  const RowEntry *entries;
  int32_t n_prefix, prefix_few;   // runs of the prefix; laid out as few's
  int32_t prefix_rt, kv_tiles;    // or as many's: rows of a row tile, pairs of it and of a workgroup
  int64_t share;
  int32_t few_rows, prefix_rows, few_items;
  int32_t n_many;                 // splits of the tails of many's requests
};

// LW lanes of a wave per row and query head or, BLOCK, the four waves of a workgroup, each a share
// of its runs.  A lane takes one run's reference and sum, so that the weights of LW runs are known
// at once, and the rows that they weigh (D / 4 lanes each, several under way) are read without
// waiting for them.
template <int D, class T, int LW, bool BLOCK>
__global__ void __launch_bounds__(NT) k_join(const JoinArgs p) {
  constexpr int LR = D / 4, RL = LW / LR, AHEAD = RL == 1 ? 8 : 4;   // lanes of a run's row, rows of a load, loads under way
  static_assert(!BLOCK || LW == 64, "whole waves share a row");
  __shared__ float part[BLOCK ? WAVES : 1][D + 2];
  const PrefixAttendArgs &a = p.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, gl = lane % LW, sub = gl / LR, col = 4 * (gl % LR);
  const int block = blockIdx.y * gridDim.x + blockIdx.x;
  const int id = BLOCK ? block : block * (NT / LW) + (int)threadIdx.x / LW;
  if (id >= a.n_tok * a.n_q) return;
  const int t = id / a.n_q, j = id - t * a.n_q, h = j / a.group, jj = j - h * a.group;
  RowEntry e = p.entries[t];
  // starts that do not rise leave entries unwritten or written twice: nothing is read by an entry
  // that is out of bounds
  if (e.kind != 0 && e.kind != 1) return;
  e.first = min(max(e.first, 0), p.few_items);
  e.count = min(max(e.count, 0), p.few_items - e.first);
  // the runs: 0 .. n1 - 1 of the prefix, n1 .. n - 1 of the tail
  const int64_t step_all = (int64_t)a.n_tok * a.n_q;
  const int64_t base1 = p.prefix_few ? (int64_t)h * p.prefix_rows + t * a.group + jj : id;
  const int64_t step1 = p.prefix_few ? (int64_t)a.heads * p.prefix_rows : step_all;
  const Parts p2 = e.kind == 0 ? p.few : p.many;
  const int64_t step2 = e.kind == 0 ? (int64_t)a.heads * p.few_rows : step_all;
  const int64_t base2 = e.kind == 0 ? ((int64_t)e.first * a.heads + h) * p.few_rows + min(max(e.place, 0) * a.group + jj, p.few_rows - 1) : id;
  int n1 = p.n_prefix;
  if (!p.prefix_few && n1 > 0) {
    const int64_t at = (int64_t)((t * a.group + jj) / p.prefix_rt) * p.kv_tiles;
    n1 = (int)((at + p.kv_tiles - 1) / p.share - at / p.share) + 1;
  }
  const int n = n1 + (e.kind == 0 ? e.count : p.n_many);
  const int share = BLOCK ? (n + WAVES - 1) / WAVES : n, i0 = BLOCK ? wave * share : 0, i1 = min(n, i0 + share);
  float M = -INFINITY, l = 0.f;
  f4_t o = {0, 0, 0, 0};
  for (int i = i0; i < i1; i += LW) {
    const int c = min(LW, i1 - i), mine = i + gl;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (gl < c) ml = mine < n1 ? p.prefix.ml[base1 + mine * step1] : p2.ml[base2 + (mine - n1) * step2];
    f4_t v[AHEAD];
    auto rows = [&](int k) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (k + u * RL < c) {
          const int q = i + min(k + u * RL + sub, c - 1);
          v[u] = gload_f4((q < n1 ? p.prefix.o + (base1 + q * step1) * D : p2.o + (base2 + (q - n1) * step2) * D) + col);
        }
    };
    rows(0);
    float mn = ml.x;
#pragma unroll
    for (int k = LW / 2; k >= 1; k >>= 1) mn = fmaxf(mn, __shfl_xor(mn, k, 64));
    mn = fmaxf(mn, M);
    // an empty run weighs nothing, whatever its row holds
    const float w = ml.x == -INFINITY && ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - mn);
    const float al = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);
    M = mn;
    float sum = ml.y * w;
#pragma unroll
    for (int k = LW / 2; k >= 1; k >>= 1) sum += __shfl_xor(sum, k, 64);
    l = fmaf(l, al, sum);
    o *= al;
    for (int k = 0; k < c; k += AHEAD * RL) {
      if (k) rows(k);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int r = k + u * RL + sub;
        const float wk = __shfl(w, (lane & ~(LW - 1)) + (r & (LW - 1)), 64);
        if (r < c && wk != 0.f) o += v[u] * wk;
      }
    }
  }
#pragma unroll
  for (int k = LR; k < LW; k <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], k, 64);
  if constexpr (BLOCK) {
    if (sub == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[wave][col + i] = o[i];
    if (lane == 0) { part[wave][D] = M; part[wave][D + 1] = l; }
    __syncthreads();
    if (wave) return;
    M = part[0][D];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) M = fmaxf(M, part[w][D]);
    l = 0.f;
    o = f4_t{0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float mw = part[w][D], lw = part[w][D + 1];
      if (mw == -INFINITY && lw == 0.f) continue;
      const float al = __builtin_amdgcn_exp2f(mw - M);
      l = fmaf(lw, al, l);
      if (al != 0.f)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(part[w][col + i], al, o[i]);
    }
  }
  if (sub == 0) write_row<D, T>(a, t, j, col, o, M, l, gl == 0);
}

// ------------------------------------------------------------------------------- launches
constexpr int BLOCKS = 512;        // workgroups that fill the chip: two a CU

int64_t ceil_div(int64_t x, int64_t y) { return (x + y - 1) / y; }

// Row tiles of the prefix for many() and the workgroups of a head: the cheapest by a model in us.  A
// workgroup that has its CU to itself takes about `tile` us a tile of keys and values (the matrix
// work, and a part that waits for memory and LDS) and 4 us to start and end a row tile; two on a
// CU take 1.5 times as long as one; every run's output is written and read once more, at about
// 4 MB a us and 0.1 us a run of a row.  Measured against it (prefix alone, us): 256 rows a head on
// 4096 tokens, 64-row tiles in 4, 8 and 16 runs 29, 20 and 20, 128-row tiles in 8, 16 and 32 runs 25,
// 21 and 25; 1024 rows on 32768 tokens by 64 workgroups a head 243 and 193.
void cut_prefix(PrefixCut &c, const PrefixAttendArgs &a, int d, bool bf16) {
  const int64_t rows = (int64_t)a.n_tok * a.group, tokens = bf16 ? 64 : 32;
  const double out = (double)a.n_tok * a.n_q * d * 8 / 4e6;
  const int most = std::max(1, BLOCKS / a.heads);      // workgroups of a head
  double best = 0;
  c.n_prefix = 0;
  c.kv_tiles = (int)ceil_div(a.T, tokens);
  for (int nq = 1; nq <= 2; ++nq) {
    const int64_t tiles = ceil_div(rows, 64 * nq), pairs = tiles * c.kv_tiles;
    const double tile = 0.3 + (bf16 ? 0.9 : 3.4) * d / 128 * nq / 2;
    // past a sixteenth of the chip only a call with nothing to share out is left
    for (int of = most; of >= std::max(1, most / 16); of = of * 3 / 4) {
      const int64_t share = ceil_div(pairs, of), n = a.heads * ceil_div(pairs, share);
      const double slabs = share >= c.kv_tiles ? 1 + (double)(c.kv_tiles - 1) / share : (double)c.kv_tiles / share;
      const double rounds = 1.5 * (n / BLOCKS) + (n % BLOCKS == 0 ? 0 : n % BLOCKS <= BLOCKS / 2 ? 1 : 1.5);
      const double cost = rounds * (tile * share + 4 * (1 + (double)(share - 1) / c.kv_tiles)) + slabs * (out + 0.1);
      if (c.n_prefix == 0 || cost < best) {
        best = cost;
        c.prefix_nq = nq;
        c.prefix_tiles = (int)tiles;
        c.share = share;
        c.prefix_groups = (int)ceil_div(pairs, share);
        c.n_prefix = (int)ceil_div(c.kv_tiles - 1, share) + 1;   // most workgroups of a row tile
      }
    }
  }
}

template <int D, class T>
hipError_t run(const PrefixAttendArgs &a, const PrefixCut &c, uint8_t *ws, hipStream_t st) {
  auto parts = [&](size_t o, size_t m) { return Parts{reinterpret_cast<float *>(ws + o), reinterpret_cast<float2 *>(ws + m)}; };
  const Parts pp = parts(c.off_po, c.off_pm), pf = parts(c.off_fo, c.off_fm), pm = parts(c.off_mo, c.off_mm);
  RowEntry *entries = reinterpret_cast<RowEntry *>(ws + c.off_entries);
  if (c.whole) {
    if (c.few_nq == 1) k_whole<D, T, 1><<<a.n_req * a.heads, NT, 0, st>>>(a);
    else k_whole<D, T, 2><<<a.n_req * a.heads, NT, 0, st>>>(a);
    return hipGetLastError();
  }
  RunArgs p{};
  p.a = a;
  if (a.T > 0 && c.prefix_few) {
    p.pre_few = FewArgs{pp, nullptr, a.n_tok * a.group, 0, c.prefix_run};
    p.pre_role = c.prefix_nq == 1 ? ROLE_FEW1 : ROLE_FEW2;
    p.n_pre = c.n_prefix * a.heads;
  } else if (a.T > 0) {
    p.pre_many = ManyArgs{pp, 1, c.prefix_tiles, 0, c.share};
    p.pre_role = c.prefix_nq == 1 ? ROLE_MANY1 : ROLE_MANY2;
    p.n_pre = c.prefix_groups * a.heads;
  }
  if (c.tails_many) {
    p.many = ManyArgs{pm, c.n_many, c.many_tiles, c.limit, 1};
    p.many_role = c.many_nq == 1 ? ROLE_MANY1 : ROLE_MANY2;
    p.n_many = c.n_many * c.many_tiles * a.heads;
  }
  // the first workgroup of these schedules, also where there are no tails
  p.few = FewArgs{pf, entries, c.few_rows, c.limit, 0};
  p.few_role = c.few_nq == 1 ? ROLE_FEW1 : ROLE_FEW2;
  p.n_few = (int)std::max<int64_t>(1, ceil_div((int64_t)c.few_items * a.heads, WAVES));
  k_runs<D, T><<<p.n_pre + p.n_many + p.n_few, NT, 0, st>>>(p);
  const JoinArgs j{a, pp, pf, pm, entries, c.n_prefix, c.prefix_few, 64 * c.prefix_nq, c.kv_tiles, c.share, c.few_rows, a.n_tok * a.group, c.few_items, c.n_many};
  const dim3 grid = grid_of(ceil_div((int64_t)a.n_tok * a.n_q * c.join_lanes, NT));
  if (c.join_lanes == NT) k_join<D, T, 64, true><<<grid, NT, 0, st>>>(j);
  else if (c.join_lanes == 64) k_join<D, T, 64, false><<<grid, NT, 0, st>>>(j);
  else k_join<D, T, D / 4, false><<<grid, NT, 0, st>>>(j);
  return hipGetLastError();
}

}  // namespace

PrefixCut prefix_attend_cut(const PrefixAttendArgs &a, int d, int dtype) {
  PrefixCut c;
  const int64_t rows = (int64_t)a.n_tok * a.group;     // rows of a key-value head
  const int64_t most = (int64_t)a.max_new * a.group;   // rows of a request
  // Requests as a whole save the join and its launch, but read the prefix once a request and leave
  // all of a request and head to one workgroup: for those of few rows and up to 3 steps of its
  // waves (128 tokens each, fp32 64), at most 4 steps counted once for every 256 workgroups.  In one
  // launch and in two (us; d 128, bf16 and fp32):
  //     32 workgroups, 3 steps 10.6 and 12.3, 11.1 and 13.8;  4 steps 12.8 and 12.8, 13.4 and 14.1
  //    512 workgroups, 2 steps 13.1 and 13.5, 13.3 and 13.2;  3 steps 16.2 and 13.2, 17.5 and 16.1
  //   1024 workgroups, 1 step  16.2 and 16.6, 15.2 and 17.1;  2 steps 23.2 and 15.8, 24.3 and 18.0
  const int64_t steps = ceil_div(a.T + ((int64_t)a.max_pages << a.tail.shift), WAVES * (dtype == JOLT_BF16 ? 32 : 16));
  const int64_t whole = (int64_t)a.n_req * a.heads;    // workgroups that takes
  if (most <= 32 && steps <= 3 && steps * ceil_div(whole, BLOCKS / 2) <= 4) {
    c.whole = true;
    c.few_nq = most <= 16 ? 1 : 2;
    c.ws_bytes = 256;
    return c;
  }
  if (a.T > 0) {
    // Up to 32 rows few() reads the prefix at the rate of memory: 32 rows on 32768 tokens of 8 heads
    // take 31 us, 33 by many(); 17 rows on 4001 tokens of 40 heads 25 and 24.
    c.prefix_few = rows <= 32;
    if (c.prefix_few) {
      c.prefix_nq = rows <= 16 ? 1 : 2;
      const int64_t runs = std::max<int64_t>(1, std::min<int64_t>(ceil_div(a.T, RUN_PREFIX), BLOCKS / a.heads));
      c.prefix_run = (int)(ceil_div(ceil_div(a.T, runs), RUN_PREFIX) * RUN_PREFIX);
      c.n_prefix = (int)ceil_div(a.T, c.prefix_run);
    } else {
      cut_prefix(c, a, d, dtype == JOLT_BF16);
    }
  }
  // A workgroup a row, a wave a row or D / 4 lanes a row: as many lanes as fill the chip, since the
  // chain of reads bounds a row and the lanes that join at its end lengthen it (8192 rows of 10
  // runs: 11 us by D / 4 lanes, 14 by waves; 2048 rows of 11: 7.3 and 6.0; 384 rows of 171: 9 us by
  // waves, 6 by workgroups).
  const int64_t out_rows = (int64_t)a.n_tok * a.n_q;
  c.join_lanes = out_rows <= 2 * BLOCKS ? NT : out_rows <= 8 * BLOCKS ? 64 : d / 4;
  // without tails every request is one of few rows and no runs
  c.limit = 0x7fffffff;
  if (a.max_pages > 0) {
    // Requests of up to 32 rows by few(), also where that takes two groups of rows a wave: 64 requests
    // of up to 32 rows and 100 to 500 tokens take 31 us, 32 with those past 16 rows by many() (fp32 57
    // and 74).
    c.few_nq = most <= 16 ? 1 : 2;
    c.limit = 16 * c.few_nq;
    c.few_rows = (int)std::min<int64_t>(most, c.limit);
    c.few_items = FEW_WAVES / a.heads + a.n_req;
    c.tails_many = most > c.limit;
    if (c.tails_many) {
      c.many_nq = most <= 64 ? 1 : 2;
      // a request of more than `limit` rows has at most one tile that is not full
      c.many_tiles = (int)(rows / (64 * c.many_nq) + std::min<int64_t>(a.n_req, rows / (c.limit + 1)));
      const int64_t want = BLOCKS / ((int64_t)a.heads * c.many_tiles);
      c.n_many = (int)std::max<int64_t>(1, std::min<int64_t>(want, 16));
    }
  }
  auto take = [&](size_t n) {
    const size_t at = c.ws_bytes;
    c.ws_bytes += (n + 255) / 256 * 256;
    return at;
  };
  // Room for the most that the cut of this batch or of any smaller one takes (fewer requests, rows,
  // rows of a request, tokens of prefix and tails), so that the size only grows with them, as those
  // cuts need not: runs times rows of a head.
  //   prefix, few():  n_prefix <= RUN_PREFIX-token runs, workgroups of a head; at most 32 rows.
  //   prefix, many(): with of <= BLOCKS / heads workgroups and tiles >= rows / (64 nq),
  //                   n_prefix < of / tiles + 2, and n_prefix <= kv_tiles.
  //   tails, many():  n_many <= max(1, BLOCKS / (heads many_tiles)), many_tiles > rows / (64 many_nq).
  const int64_t of = std::max(1, BLOCKS / a.heads);
  int64_t most_prefix = 0, most_many = 0;
  if (a.T > 0) {
    most_prefix = std::min<int64_t>(ceil_div(a.T, RUN_PREFIX), of) * std::min<int64_t>(rows, 32);
    if (rows > 32) most_prefix = std::max(most_prefix, std::min((int64_t)c.kv_tiles * rows, 128 * of + 2 * rows));
  }
  if (c.tails_many) most_many = std::max(rows, std::min<int64_t>(16 * rows, ceil_div(128 * BLOCKS, a.heads)));
  const size_t np = (size_t)most_prefix * a.heads, nf = (size_t)c.few_items * c.few_rows * a.heads, nm = (size_t)most_many * a.heads;
  c.off_po = take(np * d * 4); c.off_pm = take(np * 8);
  c.off_fo = take(nf * d * 4); c.off_fm = take(nf * 8);
  c.off_mo = take(nm * d * 4); c.off_mm = take(nm * 8);
  c.off_entries = take((size_t)a.n_tok * sizeof(RowEntry));
  return c;
}

hipError_t launch_prefix_attend(const PrefixAttendArgs &a, const PrefixCut &c, int d, int dtype, void *ws, hipStream_t st) {
  uint8_t *w = static_cast<uint8_t *>(ws);
  if (dtype == JOLT_BF16)
    return d == 32 ? run<32, bf16_t>(a, c, w, st) : d == 64 ? run<64, bf16_t>(a, c, w, st) : run<128, bf16_t>(a, c, w, st);
  return d == 32 ? run<32, float>(a, c, w, st) : d == 64 ? run<64, float>(a, c, w, st) : run<128, float>(a, c, w, st);
}
