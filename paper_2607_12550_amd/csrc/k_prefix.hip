// Attention of a batch of requests over the prefix they share and each one's paged tail.
#include "common.h"
#include "kernels.h"

namespace {

constexpr int NT = 256, WAVES = NT / 64;

// The request of packed row t: the last r with q_start[r] <= t, if t < q_start[r + 1]; else -1.
JOLT_DEV int request_of(const int32_t *q_start, int n_req, int t) {
  int lo = 0, hi = n_req;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (q_start[mid] <= t) lo = mid; else hi = mid;
  }
  return q_start[lo] <= t && t < q_start[lo + 1] ? lo : -1;
}

// Tail tokens that packed row t of a request sees: the request's rows end before q_end > t, its
// tail holds `len` tokens and the table has room for `cap`.  With q_end - t >= 1, whatever the
// device arrays hold, the result is at most cap: every index formed from it is in the table.
JOLT_HD int tail_seen(int q_end, int t, int len, int cap) {
  const int64_t have = len < 0 ? 0 : len < cap ? len : cap;
  const int64_t seen = have - ((int64_t)q_end - t) + 1;
  return seen < 0 ? 0 : (int)seen;
}

template <class T> JOLT_DEV float to_f32(T x);
template <> JOLT_DEV float to_f32<bf16_t>(bf16_t x) { return bf16_to_f32(x); }
template <> JOLT_DEV float to_f32<float>(float x) { return x; }

// One workgroup per row and query head; each wave takes every fourth token and keeps its own
// running maximum, sum and output, joined at the end.
template <int D, class T>
__global__ void __launch_bounds__(NT) k_prefix_rows(const PrefixAttendArgs a) {
  constexpr int F = (D + 63) / 64;
  const int t = blockIdx.x, j = blockIdx.y, h = j / a.group;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = request_of(a.q_start, a.n_req, t);
  if (r < 0) return;
  __shared__ float sm[WAVES], sl[WAVES], so[WAVES][D];
  const float c = a.scale * 1.4426950408889634f;
  float q[F], o[F] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
  for (int f = 0; f < F; ++f) {
    const int x = lane + 64 * f;
    q[f] = x < D ? to_f32<T>(static_cast<const T *>(a.Q)[t * a.q_stride + (int64_t)j * D + x]) : 0.f;
  }
  auto token = [&](const PrefixSource &s, int64_t off) {
    float v[F], dot = 0.f;
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const int x = lane + 64 * f;
      const bool in = x < D;
      dot = fmaf(in ? to_f32<T>(static_cast<const T *>(s.K)[off + x]) : 0.f, q[f], dot);
      v[f] = in ? to_f32<T>(static_cast<const T *>(s.V)[off + x]) : 0.f;
    }
    const float z = wave_sum(dot) * c, mn = fmaxf(m, z);
    if (mn == -INFINITY) return;
    const float al = exp2f(m - mn), p = exp2f(z - mn);
    m = mn;
    l = fmaf(l, al, p);
#pragma unroll
    for (int f = 0; f < F; ++f) o[f] = fmaf(o[f], al, p * v[f]);
  };
  for (int x = wave; x < a.T; x += WAVES) token(a.prefix, h * a.prefix.s_head + x * a.prefix.s_tok);
  if (a.table) {
    const int seen = tail_seen(a.q_start[r + 1], t, a.kv_len[r], a.max_pages << a.tail.shift);
    for (int x = wave; x < seen; x += WAVES) {
      const int page = a.table[(int64_t)r * a.max_pages + (x >> a.tail.shift)];
      if ((uint32_t)page >= (uint32_t)a.tail.n_pages) continue;
      token(a.tail, page * a.tail.s_page + h * a.tail.s_head + (x & ((1 << a.tail.shift) - 1)) * a.tail.s_tok);
    }
  }
  if (lane == 0) { sm[wave] = m; sl[wave] = l; }
#pragma unroll
  for (int f = 0; f < F; ++f)
    if (lane + 64 * f < D) so[wave][lane + 64 * f] = o[f];
  __syncthreads();
  float M = sm[0];
  for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sm[w]);
  float L = 0.f, sum = 0.f;
  for (int w = 0; w < WAVES; ++w) {
    const float al = sm[w] == -INFINITY ? 0.f : exp2f(sm[w] - M);
    L = fmaf(sl[w], al, L);
    if (threadIdx.x < D && al != 0.f) sum = fmaf(so[w][threadIdx.x], al, sum);
  }
  if (threadIdx.x < D) {
    const float v = L > 0.f ? sum / L : L == 0.f ? 0.f : NAN;
    T *O = static_cast<T *>(a.O) + t * a.o_stride + (int64_t)j * D + threadIdx.x;
    if constexpr (sizeof(T) == 2) *O = f32_to_bf16(v); else *O = v;
  }
  if (a.lse && threadIdx.x == 0) a.lse[(int64_t)t * a.n_q + j] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

template <int D>
hipError_t run(const PrefixAttendArgs &a, int dtype, hipStream_t st) {
  const dim3 grid(a.n_tok, a.n_q);
  if (dtype == JOLT_BF16)
    k_prefix_rows<D, bf16_t><<<grid, NT, 0, st>>>(a);
  else
    k_prefix_rows<D, float><<<grid, NT, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t prefix_attend_workspace(const PrefixAttendArgs &a, int d) { return 256; }

hipError_t launch_prefix_attend(const PrefixAttendArgs &a, int d, int dtype, void *ws, hipStream_t st) {
  return d == 32 ? run<32>(a, dtype, st) : d == 64 ? run<64>(a, dtype, st) : run<128>(a, dtype, st);
}
