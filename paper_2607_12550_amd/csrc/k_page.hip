// Page plans and paged appends of a batch of requests that add tokens to their tails.
#include "common.h"
#include "kernels.h"

namespace {

constexpr int NT = 256, WAVES = NT / 64;

// ------------------------------------------------------------------------------- plan
// Running sums over the requests give each request's first packed row and its first new page;
// then every packed row finds its request by bisection and its slot from its position.  A page
// that is new is entered by the row of its first token (such a row always exists, and only one),
// so no row needs to know about another.
//
// Latency bounds it: the sums are short (at most 4096 requests) and every workgroup forms them
// for itself, which takes one launch instead of a scan and a second kernel that waits for it.
// Workgroup 0 writes the per-request outputs.
//
// A thread takes STEP rows in a row: one bisection for the first, the others step on from it, and
// their page reads are under way together.  Four where one each would take more workgroups than
// the chip has CUs to repeat the sums (131,000 rows of 500 requests: 6.2 us, 7.8 by one each); one
// where rows are few (64 rows: 3.5 us, 4.7 by four).

JOLT_DEV int64_t wave_scan(int64_t v, int lane) {   // inclusive
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int64_t u = __shfl_up(v, m, 64);
    if (lane >= m) v += u;
  }
  return v;
}

template <int STEP>
__global__ void __launch_bounds__(NT) k_page_plan(const PagePlanArgs a) {
  extern __shared__ int32_t lds[];
  int32_t *start = lds;                    // [n_req + 1] first packed row
  int32_t *first = lds + a.n_req + 1;      // [n_req] first new page of the call
  int32_t *held = first + a.n_req;         // [n_req] have
  __shared__ int64_t tot[2][WAVES];
  __shared__ int bad[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int sh = a.page_shift, mask = (1 << sh) - 1;
  const int per = (a.n_req + NT - 1) / NT;
  const int r0 = min(tid * per, a.n_req), r1 = min(r0 + per, a.n_req);
  int64_t rows = 0, pages = 0;
  int why = 0;
  for (int r = r0; r < r1; ++r) {
    const int64_t h = a.have[r], n = a.add[r];
    if (h < 0 || n < 0) { why |= JOLT_PLAN_BAD_LENGTH; continue; }
    const int64_t after = (h + n + mask) >> sh;
    if (after > a.max_pages) why |= JOLT_PLAN_TABLE_FULL;
    rows += n;
    pages += after - ((h + mask) >> sh);
  }
  const int64_t srow = wave_scan(rows, lane), spage = wave_scan(pages, lane);
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) why |= __shfl_xor(why, m, 64);
  if (lane == 63) { tot[0][wave] = srow; tot[1][wave] = spage; bad[wave] = why; }
  __syncthreads();
  int64_t row0 = srow - rows, page0 = spage - pages, all_rows = 0, all_pages = 0;
  why = 0;
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) { row0 += tot[0][w]; page0 += tot[1][w]; }
    all_rows += tot[0][w];
    all_pages += tot[1][w];
    why |= bad[w];
  }
  const int n_free = max(0, min(a.n_free[0], a.free_cap));
  if (all_pages > n_free) why |= JOLT_PLAN_NO_PAGES;
  if (all_rows > a.n_tok) why |= JOLT_PLAN_NO_TOKENS;
  const bool lead = blockIdx.x == 0;
  for (int r = r0; r < r1; ++r) {
    const int h = a.have[r], n = a.add[r];
    if (lead) {
      a.kv_len[r] = why ? h : h + n;
      a.q_start[r] = why ? 0 : (int)row0;
    }
    if (!why) {
      start[r] = (int)row0;
      first[r] = (int)page0;
      held[r] = h;
      row0 += n;
      page0 += (((int64_t)h + n + mask) >> sh) - (((int64_t)h + mask) >> sh);
    }
  }
  if (lead && tid == 0) {
    a.q_start[a.n_req] = why ? 0 : (int)all_rows;
    a.n_free_out[0] = why ? a.n_free[0] : n_free - (int)all_pages;
    a.info[0] = why ? 0 : (int)all_rows;
    a.info[1] = why ? 0 : (int)all_pages;
    a.info[2] = why;
    a.info[3] = (int)min(all_pages, (int64_t)0x7fffffff);
  }
  if (!why && tid == 0) start[a.n_req] = (int)all_rows;
  __syncthreads();
  const int t0 = (blockIdx.x * NT + tid) * STEP;
  if (t0 >= a.n_tok) return;
  int slot[STEP], pos[STEP], req[STEP], page[STEP];
  int lo = 0;
  if (!why && t0 < all_rows) {
    int hi = a.n_req;                      // start[lo] <= t0 < start[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= t0) lo = mid; else hi = mid;
    }
  }
#pragma unroll
  for (int i = 0; i < STEP; ++i) {
    const int t = t0 + i;
    slot[i] = pos[i] = -1;
    req[i] = -1;
    if (why || t >= all_rows) continue;
    while (start[lo + 1] <= t) ++lo;       // ends: t < all_rows = start[n_req]
    const int have = held[lo];
    req[i] = lo;
    pos[i] = have + (t - start[lo]);
    const int j = pos[i] >> sh, fresh = j - (int)(((int64_t)have + mask) >> sh);
    page[i] = fresh >= 0 ? a.free_pages[n_free - 1 - (first[lo] + fresh)] : a.table[(int64_t)lo * a.max_pages + j];
  }
#pragma unroll
  for (int i = 0; i < STEP; ++i)
    if (req[i] >= 0) {
      if ((pos[i] & mask) == 0) a.table[(int64_t)req[i] * a.max_pages + (pos[i] >> sh)] = page[i];
      if ((uint32_t)page[i] < (uint32_t)a.n_pages) slot[i] = (page[i] << sh) + (pos[i] & mask);
    }
#pragma unroll
  for (int i = 0; i < STEP; ++i)
    if (t0 + i < a.n_tok) {
      a.slots[t0 + i] = slot[i];
      a.positions[t0 + i] = pos[i];
    }
}

// ------------------------------------------------------------------------------- append
// One workgroup per packed row.  A row's rotation is the same for all its heads: one thread per
// feature pair forms its cosine and sine, and all heads take them from LDS.
//
// The angle in turns, (pos + offset) base^(-2 j / d) / (2 pi), is exact to fp64 rounding; its
// distance to the nearest quarter turn, at most pi / 4 in radians, is split into a float and the
// rest, which enters to first order, so that cosine and sine are right to about one fp32 ulp.
JOLT_DEV float2 cos_sin_turns(double u) {
  const double q = rint(4.0 * u);
  const double x = (u - 0.25 * q) * 6.283185307179586477;
  const float hi = (float)x, lo = (float)(x - (double)hi);
  float s0, c0;
  sincosf(hi, &s0, &c0);
  const float s = fmaf(c0, lo, s0), c = fmaf(-s0, lo, c0);
  const int k = (int)((int64_t)q & 3);
  const float cc = (k & 1) ? s : c, ss = (k & 1) ? c : s;
  return make_float2((k == 1 || k == 2) ? -cc : cc, (k & 2) ? -ss : ss);
}

template <int D, class T>
__global__ void __launch_bounds__(NT) k_page_append(const PageAppendArgs a) {
  constexpr int E = 16 / sizeof(T);        // elements of a 16-byte piece
  constexpr int C = D / E, HALF = D / 2;
  __shared__ float2 cs[HALF];
  const uint32_t t = blockIdx.y * gridDim.x + blockIdx.x;
  const int tid = threadIdx.x;
  if (t >= (uint32_t)a.n_tok) return;
  const int slot = a.slots[t];
  if (slot < 0 || slot >= a.n_slots) return;
  const int64_t at = (int64_t)(slot >> a.page_shift) * a.s_page + (int64_t)(slot & ((1 << a.page_shift) - 1)) * a.s_tok;
  const T *K = static_cast<const T *>(a.K) + t * a.k_tok, *V = static_cast<const T *>(a.V) + t * a.v_tok;
  T *Kp = static_cast<T *>(a.Kp) + at, *Vp = static_cast<T *>(a.Vp) + at;
  if (a.rope) {
    if (tid < HALF) cs[tid] = cos_sin_turns(((double)a.positions[t] + (double)a.offset) * a.turns[tid]);
    __syncthreads();
    for (int i = tid; i < a.n_heads * (C / 2); i += NT) {
      const int h = i / (C / 2), c = (i % (C / 2)) * E;
      const T *src = K + h * a.k_head + c;
      T x[2][E], y[2][E];
      *reinterpret_cast<ju4 *>(x[0]) = gload_u4(src);
      *reinterpret_cast<ju4 *>(x[1]) = gload_u4(src + HALF);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 w = cs[c + e];
        if constexpr (sizeof(T) == 2) {
          const float p = bf16_to_f32(x[0][e]), q = bf16_to_f32(x[1][e]);
          y[0][e] = f32_to_bf16(fmaf(-q, w.y, p * w.x));
          y[1][e] = f32_to_bf16(fmaf(p, w.y, q * w.x));
        } else {
          const float p = x[0][e], q = x[1][e];
          y[0][e] = fmaf(-q, w.y, p * w.x);
          y[1][e] = fmaf(p, w.y, q * w.x);
        }
      }
      T *dst = Kp + h * a.s_head + c;
      *reinterpret_cast<ju4 *>(dst) = *reinterpret_cast<ju4 *>(y[0]);
      *reinterpret_cast<ju4 *>(dst + HALF) = *reinterpret_cast<ju4 *>(y[1]);
    }
  } else {
    for (int i = tid; i < a.n_heads * C; i += NT) {
      const int h = i / C, c = (i % C) * E;
      *reinterpret_cast<ju4 *>(Kp + h * a.s_head + c) = gload_u4(K + h * a.k_head + c);
    }
  }
  for (int i = tid; i < a.n_heads * C; i += NT) {
    const int h = i / C, c = (i % C) * E;
    *reinterpret_cast<ju4 *>(Vp + h * a.s_head + c) = gload_u4(V + h * a.v_head + c);
  }
}

template <int D>
hipError_t append(const PageAppendArgs &a, int dtype, hipStream_t st) {
  const dim3 grid = grid_of(a.n_tok);
  if (dtype == JOLT_BF16)
    k_page_append<D, bf16_t><<<grid, NT, 0, st>>>(a);
  else
    k_page_append<D, float><<<grid, NT, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_plan(const PagePlanArgs &a, hipStream_t st) {
  const size_t lds = (3 * a.n_req + 1) * sizeof(int32_t);
  auto grid = [&](int step) { return (uint32_t)(((int64_t)a.n_tok + step * NT - 1) / (step * NT)); };
  if (a.n_tok <= 256 * NT) k_page_plan<1><<<grid(1), NT, lds, st>>>(a);
  else k_page_plan<4><<<grid(4), NT, lds, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_page_append(const PageAppendArgs &a, int d, int dtype, hipStream_t st) {
  return d == 32 ? append<32>(a, dtype, st) : d == 64 ? append<64>(a, dtype, st) : append<128>(a, dtype, st);
}
