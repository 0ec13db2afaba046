// Attention of a batch of requests over the prefix they share and each one's paged tail.
//
// A query head's rows of one key-value head h are numbered rho = (token) * G + (head in its
// group), so that all rows that read head h stand side by side: those of the whole batch for
// the prefix, those of one request for its tail.  Both parts are cut into runs of tokens, each
// run keeps the running maximum m (in units of log2) and sum l of its softmax and the sum of
// exp2(s - m) v, and the last kernel joins the runs of a row.
//
//  * k_few:  at most 16 NQ rows.  Reading the keys and values bounds it, so the four waves of a
//    workgroup take different tokens of the run, keys go from memory straight into the matrix
//    operand, and only the values pass through LDS (a region of the wave's own) to be transposed.
//  * k_many: 64 NQ rows a workgroup, which share the tiles of keys and values in LDS: the
//    prefix is read once per row tile instead of once per request, and the matrix cores bound it.
//  * k_join: the runs of a row.
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
  // Pieces of an LDS row are permuted in pairs by row, so that the 16 rows that one transposed
  // read touches (32 bytes each) fall in distinct banks.
  static JOLT_DEV int swz(int row, int piece) {
    constexpr int RL = RB >= 256 ? 1 : 256 / RB, PM = (RB >= 256 ? 256 : RB) / 32 - 1;
    return piece ^ (((row / RL) & PM) << 1);
  }
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

// The request of packed row t, or -1: the last one that starts at or before t, found by the
// whole wave (64 candidates a step, two steps at most).
JOLT_DEV int request_of(const PrefixAttendArgs &a, int t, int lane) {
  int lo = 0, step = a.n_req > 64 ? 64 : 1;
  for (;; step = 1) {
    const int r = lo + lane * step;
    const bool in = r < a.n_req && a.q_start[r] <= t;
    const int c = __popcll(__ballot(in));
    if (c == 0) return -1;
    lo += (c - 1) * step;
    if (step == 1) break;
  }
  const Req x = request(a, lo);
  return t >= x.q0 && t < x.q0 + x.n ? lo : -1;
}

// Runs of the requests that k_few serves: at most FEW_ITEMS / heads runs besides one a request,
// of equal length (a multiple of the tokens a workgroup takes a step), in the requests' order.
// Every workgroup forms the sums for itself; the result is in LDS.
constexpr int FEW_ITEMS = 1024, RUN_STEP = 128;
struct Item { int r, first, last; };   // request, tokens first .. last - 1
JOLT_DEV int few_run(int64_t total, int heads) {
  const int64_t c = (total * heads + FEW_ITEMS - 1) / FEW_ITEMS;
  return (int)((max(c, (int64_t)RUN_STEP) + RUN_STEP - 1) / RUN_STEP * RUN_STEP);
}

JOLT_DEV int64_t wave_scan(int64_t v, int lane) {   // inclusive
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int64_t u = __shfl_up(v, m, 64);
    if (lane >= m) v += u;
  }
  return v;
}

struct FindLds { int64_t sum[WAVES]; int cnt[WAVES]; int r, idx; };
// Item `want` of the call (kind 0: runs of k_few's requests, kind 1: row tiles of k_many's), or
// r = -1 past the last; item_first (workgroups that write it): [n_req + 1] first run of each.
template <int KIND>
JOLT_DEV void find_item(const PrefixAttendArgs &a, int want, int limit, int rows_tile, int32_t *item_first, int &run, FindLds &sm) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.n_req + NT - 1) / NT, r0 = min(tid * per, a.n_req), r1 = min(r0 + per, a.n_req);
  run = 0;
  if constexpr (KIND == 0) {
    int64_t total = 0;
    for (int r = r0; r < r1; ++r) {
      const Req x = request(a, r);
      if (x.n > 0 && x.n * a.group <= limit) total += x.len;
    }
    const int64_t w = wave_scan(total, lane);
    if (lane == 63) sm.sum[wave] = w;
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
  for (int r = r0; r < r1; ++r) mine += count(request(a, r));
  int incl = mine;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int u = __shfl_up(incl, m, 64);
    if (lane >= m) incl += u;
  }
  if (lane == 63) sm.cnt[wave] = incl;
  if (tid == 0) sm.r = -1;
  __syncthreads();
  int before = incl - mine;
  for (int w = 0; w < wave; ++w) before += sm.cnt[w];
  if (item_first || (want >= before && want < before + mine)) {
    for (int r = r0; r < r1; ++r) {
      const int c = count(request(a, r));
      if (item_first) item_first[r] = before;
      if (want >= before && want < before + c) { sm.r = r; sm.idx = want - before; }
      before += c;
    }
    if (item_first && r1 == a.n_req && r0 < r1) item_first[a.n_req] = before;
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
  float m[NQ], l[NQ];        // maximum in units of log2 (all lanes of the query), this lane's part of the sum
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
  // Scores s (16 SUBS tokens) into weights, in place, with the running maximum and sum and the
  // output rescaled where the maximum moved.
  template <int SUBS>
  JOLT_DEV void softmax(f4_t (&s)[SUBS][NQ], float c) {
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      float mx = max4(s[0][x]);
#pragma unroll
      for (int u = 1; u < SUBS; ++u) mx = fmaxf(mx, max4(s[u][x]));
      mx = fmaxf(m[x], over_groups_max(mx) * c);
      if (__any(mx > m[x])) {
        // nothing seen so far: both are -inf, and nothing is there to rescale
        const float al = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[x] - mx);
        l[x] *= al;
#pragma unroll
        for (int f = 0; f < G::FT; ++f) o[f][x] *= al;
        m[x] = mx;
      }
      const float base = mx == -INFINITY ? 0.f : mx;
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[u][x][i], c, -base));
          s[u][x][i] = p;
          sum += p;
        }
      l[x] += sum;
    }
  }
  // o += V^T P^T for 16 SUBS tokens whose values stand in LDS rows row0 ..; the weights are
  // rounded to bf16 for the bf16 product (values are bf16 already): half a step each, which
  // averages out over the tokens, for half of the matrix work of two terms.
  template <int SUBS>
  JOLT_DEV void values(const f4_t (&p)[SUBS][NQ], const uint8_t *v, int row0, int n16, int g) {
    if constexpr (G::BF) {
#pragma unroll
      for (int u = 0; u < SUBS; u += 2) {
        b8_t w[NQ];
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
          const uint32_t d[4] = {pack_bf16(p[u][x][0], p[u][x][1]), pack_bf16(p[u][x][2], p[u][x][3]),
                                 pack_bf16(p[u + 1][x][0], p[u + 1][x][1]), pack_bf16(p[u + 1][x][2], p[u + 1][x][3])};
          __builtin_memcpy(&w[x], d, 16);
        }
        const int ra = row0 + 16 * u + 4 * g + (n16 >> 2), rb = ra + 16;
#pragma unroll
        for (int f = 0; f < G::FT; ++f) {
          const int piece = 2 * f + ((n16 >> 1) & 1), low = 8 * (n16 & 1);
          auto *pa = v + ra * G::RB + G::swz(ra, piece) * 16 + low;
          auto *pb = v + rb * G::RB + G::swz(rb, piece) * 16 + low;
          const s4_t xa = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t *)pa);
          const s4_t xb = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t *)pb);
          const auto xv = __builtin_shufflevector(xa, xb, 0, 1, 2, 3, 4, 5, 6, 7);
          b8_t va;
          __builtin_memcpy(&va, &xv, 16);
#pragma unroll
          for (int x = 0; x < NQ; ++x) o[f][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, w[x], o[f][x], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = row0 + 16 * u + 4 * g + i;
#pragma unroll
          for (int f = 0; f < G::FT; ++f) {
            const float va = *reinterpret_cast<const float *>(v + r * G::RB + G::swz(r, 4 * f + (n16 >> 2)) * 16 + 4 * (n16 & 3));
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
          const T raw = *reinterpret_cast<const T *>(v + k * G::RB + G::swz(k, byte >> 4) * 16 + (byte & 15));
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
struct FewArgs {
  PrefixAttendArgs a;
  Parts out;
  int32_t *item_first;      // tails: first run of each request
  int32_t rows;             // rows kept per run and head: row rho of head h at (item * heads + h) * rows + rho
  int32_t limit;            // tails: requests of at most this many rows per head
  int32_t run;              // prefix: tokens of a run
};

template <int D, class T, int NQ, bool TAIL>
__global__ void __launch_bounds__(NT) k_few(const FewArgs p) {
  using G = Geo<D, T>;
  constexpr int VB = G::TPW * G::RB;                     // a wave's values
  constexpr int OB = 16 * NQ * D * 4;                    // a wave's output
  constexpr int WB = VB > OB ? VB : OB;
  __shared__ __attribute__((aligned(16))) uint8_t lds[WAVES * WB];
  __shared__ float sm_m[WAVES][16 * NQ], sm_l[WAVES][16 * NQ];
  __shared__ FindLds fl;
  const PrefixAttendArgs &a = p.a;
  const PrefixSource &src = TAIL ? a.tail : a.prefix;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.x % a.heads, item = blockIdx.x / a.heads;
  int t0, n, first, end;
  const int32_t *pages = nullptr;
  if constexpr (TAIL) {
    int run;
    find_item<0>(a, item, p.limit, 0, blockIdx.x == 0 ? p.item_first : nullptr, run, fl);
    const int r = fl.r;
    if (r < 0) return;
    const Req x = request(a, r);
    t0 = x.q0;
    n = x.n;
    first = fl.idx * run;
    end = min(x.len, first + run);
    pages = a.table + (int64_t)r * a.max_pages;
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
    const Req x = request(a, fl.r);
#pragma unroll
    for (int c = 0; c < NQ; ++c) {
      const int rho = 16 * c + n16;
      R.seen[c] = rho < n_rows ? max(0, x.len - x.n + rho / a.group + 1) : 0x7fffffff;
    }
    seen_all = max(0, x.len - x.n + 1);
  }
  const float c = a.scale * LOG2E;
  uint8_t *vl = lds + wave * WB;
  const uint8_t *Kb = static_cast<const uint8_t *>(src.K), *Vb = static_cast<const uint8_t *>(src.V);
  ju4 kr[G::SUB][G::KS], vr[G::SUB][G::KS];
  RowAt at[G::SUB];
  int pg[G::SUB];
  const int x0 = first + wave * G::TPW;
  auto ask_pages = [&](int x) {
#pragma unroll
    for (int u = 0; u < G::SUB; ++u) pg[u] = page_of(src, pages, x + 16 * u + n16, end);
  };
  auto place = [&](int x) {
#pragma unroll
    for (int u = 0; u < G::SUB; ++u) at[u] = row_at(src, pg[u], h, x + 16 * u + n16, end, sizeof(T));
  };
  auto load = [&](const uint8_t *base, ju4 (&d)[G::SUB][G::KS]) {
#pragma unroll
    for (int u = 0; u < G::SUB; ++u)
#pragma unroll
      for (int s = 0; s < G::KS; ++s) d[u][s] = gload_u4(base + at[u].off + 64 * s + 16 * g);
  };
  if (x0 < end) {
    ask_pages(x0);
    place(x0);
    load(Kb, kr);
    load(Vb, vr);
    ask_pages(x0 + WAVES * G::TPW);
  }
  for (int x = x0; x < end; x += WAVES * G::TPW) {
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
    const bool partly = x + G::TPW > seen_all;   // some row does not see all of it
    bool mine[G::SUB];
#pragma unroll
    for (int u = 0; u < G::SUB; ++u) mine[u] = at[u].ok;
    const int xn = x + WAVES * G::TPW;
    const bool more = xn < end;
    if (more) {
      place(xn);
      load(Kb, kr);
      ask_pages(xn + WAVES * G::TPW);
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
            if (!there || (TAIL && x + 16 * u + k >= R.seen[q])) s[u][q][i] = -INFINITY;
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
          const int row = 16 * u + n16;
          *reinterpret_cast<ju4 *>(vl + row * G::RB + G::swz(row, 4 * k + g) * 16) = vr[u][k];
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
        R.template add_nonfinite<G::TPW>(vl, x, n16, g);
#pragma unroll
        for (int u = 0; u < G::SUB; ++u)
#pragma unroll
          for (int k = 0; k < G::KS; ++k) vr[u][k] = finite_or_zero<T>(vr[u][k]);
        put();
      }
    }
    if (more) load(Vb, vr);
    R.values(s, vl, 0, n16, g);
  }
  // the waves' results join in LDS
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const float l = over_groups_sum(R.l[q]);
    if (g == 0) { sm_m[wave][16 * q + n16] = R.m[q]; sm_l[wave][16 * q + n16] = l; }
#pragma unroll
    for (int f = 0; f < G::FT; ++f)
      *reinterpret_cast<f4_t *>(vl + ((16 * q + n16) * D + 16 * f + 4 * g) * 4) = R.o[f][q];
  }
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * p.rows;     // (item * heads + h) * rows
  for (int i = tid; i < n_rows * (D / 4); i += NT) {
    const int row = i / (D / 4), e = (i % (D / 4)) * 4;
    float M = sm_m[0][row];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sm_m[w][row]);
    f4_t o = {0, 0, 0, 0};
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float al = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm_m[w][row] - M);
      if (sm_m[w][row] != -INFINITY || sm_l[w][row] != 0.f) {
        l = fmaf(sm_l[w][row], al, l);
        o += *reinterpret_cast<const f4_t *>(lds + w * WB + (row * D + e) * 4) * al;
      }
    }
    *reinterpret_cast<f4_t *>(p.out.o + (base + row) * D + e) = o;
    if (e == 0) p.out.ml[base + row] = make_float2(M, l);
  }
}

// ------------------------------------------------------------------------------- many rows
struct ManyArgs {
  PrefixAttendArgs a;
  Parts out;                // [split][packed row][query head]
  int32_t splits, tiles;    // prefix: row tiles; tails: most row tiles of the call
  int32_t limit;            // tails: requests of more rows per head than this
};

template <int D, class T, int NQ, bool TAIL>
__global__ void __launch_bounds__(NT) k_many(const ManyArgs p) {
  using G = Geo<D, T>;
  constexpr int RT = 64 * NQ, SUBS = G::TILE / 16;
  constexpr int PASS = NT / G::CH, LOADS = G::TILE / PASS;   // rows of a load, loads of a tile
  static_assert(G::TILE % PASS == 0, "a tile is whole loads");
  constexpr int TB = G::TILE * G::RB;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][TB];
  __shared__ int there[2][G::TILE];
  __shared__ int flag[2];
  __shared__ FindLds fl;
  const PrefixAttendArgs &a = p.a;
  const PrefixSource &src = TAIL ? a.tail : a.prefix;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.x % a.heads, rest = blockIdx.x / a.heads;
  const int tile = rest % p.tiles, split = rest / p.tiles;
  int t0, n, len, rho0, seen_all = 0x7fffffff;
  const int32_t *pages = nullptr;
  if constexpr (TAIL) {
    int run;
    find_item<1>(a, tile, p.limit, RT, nullptr, run, fl);
    const int r = fl.r;
    if (r < 0) return;
    const Req x = request(a, r);
    t0 = x.q0;
    n = x.n;
    rho0 = fl.idx * RT;
    // the tile's last row sees most, its first least
    len = max(0, x.len - x.n + min(x.n, (rho0 + RT - 1) / a.group + 1));
    seen_all = max(0, x.len - x.n + rho0 / a.group + 1);
    pages = a.table + (int64_t)r * a.max_pages;
  } else {
    t0 = 0;
    n = a.n_tok;
    rho0 = tile * RT;
    len = a.T;
  }
  const int n_rows = n * a.group;
  const int run = ((len + p.splits - 1) / p.splits + G::TILE - 1) / G::TILE * G::TILE;
  const int first = split * run, end = min(len, first + run);
  Rows<D, T, NQ> R;
  const int rho_w = rho0 + wave * 16 * NQ;
  R.load(a, h, t0, rho_w, n_rows, n16, g);
  R.clear();
  if constexpr (TAIL) {
    const Req x = request(a, fl.r);
#pragma unroll
    for (int c = 0; c < NQ; ++c) {
      const int rho = rho_w + 16 * c + n16;
      R.seen[c] = rho < n_rows ? max(0, x.len - x.n + rho / a.group + 1) : 0x7fffffff;
    }
  }
  const float c = a.scale * LOG2E;
  const uint8_t *Kb = static_cast<const uint8_t *>(src.K), *Vb = static_cast<const uint8_t *>(src.V);
  const int lrow = tid / G::CH, piece = tid % G::CH;
  ju4 kr[LOADS], vr[LOADS];
  int pg[LOADS];
  bool ok[LOADS];
  auto ask_pages = [&](int x) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) pg[i] = page_of(src, pages, x + i * PASS + lrow, end);
  };
  auto load = [&](int x) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const RowAt at = row_at(src, pg[i], h, x + i * PASS + lrow, end, sizeof(T));
      ok[i] = at.ok;
      kr[i] = gload_u4(Kb + at.off + piece * 16);
      vr[i] = gload_u4(Vb + at.off + piece * 16);
    }
  };
  auto put = [&](int b, int x) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = i * PASS + lrow, at = row * G::RB + G::swz(row, piece) * 16;
      if (!ok[i]) vr[i] = ju4{0, 0, 0, 0};
      *reinterpret_cast<ju4 *>(&lds[b][0][at]) = kr[i];
      *reinterpret_cast<ju4 *>(&lds[b][1][at]) = vr[i];
      if (piece == 0) there[b][row] = ok[i];
      if constexpr (TAIL) bad |= nonfinite<T>(vr[i]);
    }
    if (TAIL && x + G::TILE > seen_all && bad) flag[b] = 1;
  };
  if (TAIL && tid < 2) flag[tid] = 0;
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
    const uint8_t *kl = lds[b][0];
    uint8_t *vl = lds[b][1];
    f4_t s[SUBS][NQ];
#pragma unroll
    for (int u = 0; u < SUBS; ++u) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) s[u][q] = f4_t{0, 0, 0, 0};
      const int row = 16 * u + n16;
#pragma unroll
      for (int k = 0; k < G::KS; ++k) {
        const ju4 ka = *reinterpret_cast<const ju4 *>(kl + row * G::RB + G::swz(row, 4 * k + g) * 16);
#pragma unroll
        for (int q = 0; q < NQ; ++q) s[u][q] = product_step<T>(ka, R.q[q][k], s[u][q]);
      }
    }
    if (TAIL || x + G::TILE > end) {
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 16 * u + 4 * g + i;
          const bool in = there[b][k] != 0;
#pragma unroll
          for (int q = 0; q < NQ; ++q)
            if (!in || (TAIL && x + k >= R.seen[q])) s[u][q][i] = -INFINITY;
        }
    }
    R.softmax(s, c);
    if (TAIL && flag[b]) {          // the same for all threads: written before the last barrier
      R.template add_nonfinite<G::TILE>(vl, x, n16, g);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int row = i * PASS + lrow;
        ju4 *at = reinterpret_cast<ju4 *>(vl + row * G::RB + G::swz(row, piece) * 16);
        *at = finite_or_zero<T>(*at);
      }
      if (tid == 0) flag[b] = 0;
      __syncthreads();
    }
    R.values(s, vl, 0, n16, g);
    if (more) put(b ^ 1, x + G::TILE);
    __syncthreads();
  }
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const float l = over_groups_sum(R.l[q]);
    const int rho = rho_w + 16 * q + n16;
    if (rho < n_rows) {
      const int t = t0 + rho / a.group, j = h * a.group + rho % a.group;
      const int64_t row = ((int64_t)split * a.n_tok + t) * a.n_q + j;
#pragma unroll
      for (int f = 0; f < G::FT; ++f) *reinterpret_cast<f4_t *>(p.out.o + row * D + 16 * f + 4 * g) = R.o[f][q];
      if (g == 0) p.out.ml[row] = make_float2(R.m[q], l);
    }
  }
}

// ------------------------------------------------------------------------------- join
struct JoinArgs {
  PrefixAttendArgs a;
  Parts prefix, few, many;
  const int32_t *item_first;
  int32_t n_prefix, prefix_few;   // runs of the prefix; laid out as k_few's
  int32_t few_rows, prefix_rows, limit;
  int32_t n_many;                 // splits of the tails of k_many's requests
};

// One wave per row and query head.
template <int D, class T>
__global__ void __launch_bounds__(NT) k_join(const JoinArgs p) {
  constexpr int E = D >= 128 ? 2 : 1;
  const PrefixAttendArgs &a = p.a;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
  if (id >= (int64_t)a.n_tok * a.n_q) return;
  const int t = (int)(id / a.n_q), j = (int)(id % a.n_q), h = j / a.group, jj = j % a.group;
  const int r = request_of(a, t, lane);
  if (r < 0) return;
  const Req x = request(a, r);
  float M = -INFINITY, l = 0.f, o[E] = {};
  const bool has = lane * E < D;
  auto add = [&](const Parts &s, int64_t row) {
    const float2 ml = s.ml[row];
    if (ml.x == -INFINITY && ml.y == 0.f) return;   // an empty run
    const float mn = fmaxf(M, ml.x);
    const float al = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);
    const float be = __builtin_amdgcn_exp2f(ml.x - mn);
    M = mn;
    l = fmaf(l, al, ml.y * be);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], al, has ? s.o[row * D + lane * E + e] * be : 0.f);
  };
  for (int s = 0; s < p.n_prefix; ++s)
    add(p.prefix, p.prefix_few ? ((int64_t)s * a.heads + h) * p.prefix_rows + t * a.group + jj : ((int64_t)s * a.n_tok + t) * a.n_q + j);
  if (a.table) {
    if (x.n * a.group <= p.limit) {
      const int i1 = p.item_first[r + 1];
      for (int i = p.item_first[r]; i < i1; ++i) add(p.few, ((int64_t)i * a.heads + h) * p.few_rows + (t - x.q0) * a.group + jj);
    } else {
      for (int s = 0; s < p.n_many; ++s) add(p.many, ((int64_t)s * a.n_tok + t) * a.n_q + j);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (has) {
    T *O = static_cast<T *>(a.O) + (int64_t)t * a.o_stride + (int64_t)j * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float v = o[e] * inv;
      if constexpr (sizeof(T) == 2) O[e] = f32_to_bf16(v); else O[e] = v;
    }
  }
  if (a.lse && lane == 0) a.lse[id] = l == 0.f ? -INFINITY : (M + log2f(l)) * LN2;
}

// ------------------------------------------------------------------------------- launches
// How a call is cut, from its sizes alone (the workspace depends on it too).
struct Cut {
  bool prefix_few = false, tails_few = false, tails_many = false;
  int prefix_nq = 1, prefix_run = 0, n_prefix = 0, prefix_tiles = 0;   // of k_few / k_many
  int few_nq = 1, few_items = 0, few_rows = 0, limit = 0;
  int many_nq = 1, many_tiles = 0, n_many = 0;
  size_t off_po, off_pm, off_fo, off_fm, off_mo, off_mm, off_items, total;
};
constexpr int BLOCKS = 512;        // workgroups that fill the chip: two a CU

int64_t ceil_div(int64_t x, int64_t y) { return (x + y - 1) / y; }

Cut cut(const PrefixAttendArgs &a, int d, bool tails) {
  Cut c;
  const int64_t rows = (int64_t)a.n_tok * a.group;     // rows of a key-value head
  if (a.T > 0) {
    c.prefix_few = rows <= 32;
    c.prefix_nq = c.prefix_few ? (rows <= 16 ? 1 : 2) : (rows <= 64 ? 1 : 2);
    if (c.prefix_few) {
      const int64_t runs = std::max<int64_t>(1, std::min<int64_t>(ceil_div(a.T, RUN_STEP), BLOCKS / a.heads));
      c.prefix_run = (int)(ceil_div(ceil_div(a.T, runs), RUN_STEP) * RUN_STEP);
      c.n_prefix = (int)ceil_div(a.T, c.prefix_run);
    } else {
      c.prefix_tiles = (int)ceil_div(rows, 64 * c.prefix_nq);
      const int64_t want = BLOCKS / ((int64_t)a.heads * c.prefix_tiles);
      c.n_prefix = (int)std::max<int64_t>(1, std::min<int64_t>(want, ceil_div(a.T, 256)));
    }
  }
  if (tails) {
    const int64_t most = (int64_t)a.max_new * a.group; // rows of a request
    c.few_nq = most <= 16 ? 1 : 2;
    c.limit = 16 * c.few_nq;
    c.tails_few = true;
    c.few_rows = (int)std::min<int64_t>(most, c.limit);
    c.few_items = FEW_ITEMS / a.heads + a.n_req;
    c.tails_many = most > c.limit;
    if (c.tails_many) {
      c.many_nq = most <= 64 ? 1 : 2;
      // a request of more than `limit` rows has at most one tile that is not full
      c.many_tiles = (int)(rows / (64 * c.many_nq) + std::min<int64_t>(a.n_req, rows / (c.limit + 1)));
      const int64_t want = BLOCKS / ((int64_t)a.heads * c.many_tiles);
      c.n_many = (int)std::max<int64_t>(1, std::min<int64_t>(want, 16));
    }
  }
  size_t off = 0;
  auto take = [&](size_t n) {
    const size_t at = off;
    off += (n + 255) / 256 * 256;
    return at;
  };
  const size_t np = c.prefix_few ? (size_t)c.n_prefix * a.heads * rows : (size_t)c.n_prefix * a.n_tok * a.n_q;
  const size_t nf = (size_t)c.few_items * a.heads * c.few_rows;
  const size_t nm = (size_t)c.n_many * a.n_tok * a.n_q;
  c.off_po = take(np * d * 4); c.off_pm = take(np * 8);
  c.off_fo = take(nf * d * 4); c.off_fm = take(nf * 8);
  c.off_mo = take(nm * d * 4); c.off_mm = take(nm * 8);
  c.off_items = take(((size_t)a.n_req + 1) * 4);
  c.total = off;
  return c;
}

template <int D, class T>
hipError_t run(const PrefixAttendArgs &a, const Cut &c, uint8_t *ws, hipStream_t st) {
  auto parts = [&](size_t o, size_t m) { return Parts{reinterpret_cast<float *>(ws + o), reinterpret_cast<float2 *>(ws + m)}; };
  const Parts pp = parts(c.off_po, c.off_pm), pf = parts(c.off_fo, c.off_fm), pm = parts(c.off_mo, c.off_mm);
  int32_t *items = reinterpret_cast<int32_t *>(ws + c.off_items);
  if (a.T > 0 && c.prefix_few) {
    const FewArgs p{a, pp, nullptr, a.n_tok * a.group, 0, c.prefix_run};
    const int grid = c.n_prefix * a.heads;
    if (c.prefix_nq == 1) k_few<D, T, 1, false><<<grid, NT, 0, st>>>(p);
    else k_few<D, T, 2, false><<<grid, NT, 0, st>>>(p);
  } else if (a.T > 0) {
    const ManyArgs p{a, pp, c.n_prefix, c.prefix_tiles, 0};
    const int grid = c.n_prefix * c.prefix_tiles * a.heads;
    if (c.prefix_nq == 1) k_many<D, T, 1, false><<<grid, NT, 0, st>>>(p);
    else k_many<D, T, 2, false><<<grid, NT, 0, st>>>(p);
  }
  if (c.tails_few) {
    const FewArgs p{a, pf, items, c.few_rows, c.limit, 0};
    const int grid = c.few_items * a.heads;
    if (c.few_nq == 1) k_few<D, T, 1, true><<<grid, NT, 0, st>>>(p);
    else k_few<D, T, 2, true><<<grid, NT, 0, st>>>(p);
  }
  if (c.tails_many) {
    const ManyArgs p{a, pm, c.n_many, c.many_tiles, c.limit};
    const int grid = c.n_many * c.many_tiles * a.heads;
    if (c.many_nq == 1) k_many<D, T, 1, true><<<grid, NT, 0, st>>>(p);
    else k_many<D, T, 2, true><<<grid, NT, 0, st>>>(p);
  }
  const JoinArgs j{a, pp, pf, pm, items, c.n_prefix, c.prefix_few, c.few_rows, a.n_tok * a.group, c.limit, c.n_many};
  k_join<D, T><<<(int)ceil_div((int64_t)a.n_tok * a.n_q, WAVES), NT, 0, st>>>(j);
  return hipGetLastError();
}

}  // namespace

size_t prefix_attend_workspace(const PrefixAttendArgs &a, int d) { return cut(a, d, a.max_pages > 0).total; }

hipError_t launch_prefix_attend(const PrefixAttendArgs &a, int d, int dtype, void *ws, hipStream_t st) {
  const Cut c = cut(a, d, a.max_pages > 0);
  uint8_t *w = static_cast<uint8_t *>(ws);
  if (dtype == JOLT_BF16)
    return d == 32 ? run<32, bf16_t>(a, c, w, st) : d == 64 ? run<64, bf16_t>(a, c, w, st) : run<128, bf16_t>(a, c, w, st);
  return d == 32 ? run<32, float>(a, c, w, st) : d == 64 ? run<64, float>(a, c, w, st) : run<128, float>(a, c, w, st);
}
