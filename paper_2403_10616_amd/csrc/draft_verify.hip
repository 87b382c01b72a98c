// Which drafted tokens stay, and the token behind them (include/dipaco_kernels.h has the rule): a workgroup walks a document's tree from row 0.
//
// A token hangs on a border (u q < r, a running sum above v times the whole), so exponentials, sums and what is left of the target are 64-bit numbers: then the
// order of a sum decides nothing but one draw in 10^10.
#include "draft.h"
#include "kernels.h"

namespace dipaco {

namespace {

constexpr int DV_THREADS = 1024, DV_WAVES = DV_THREADS / 64;

__device__ __forceinline__ double wave_total(double v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, WAVE);
  return v;
}
// VEC scores from y0 on, which any address may hold; -inf behind the last
template <typename T> __device__ __forceinline__ void load_scores(const T* row, int y0, int V, float (&x)[Vec16<T>::N]) {
  constexpr int VEC = Vec16<T>::N;
  if (y0 + VEC <= V) {
    T e[VEC];
    __builtin_memcpy(e, row + y0, sizeof(e));
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = to_f32(e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = y0 + i < V ? to_f32(row[y0 + i]) : -INFINITY;
  }
}

struct RowStat {
  float top;      // largest score
  int at;         // its first place
  double total;   // sum of exp((x - top) scale)
  bool ok;        // whether the row is a distribution: no NaN, no +inf, something above -inf
};

template <typename T> struct Walk {
  static constexpr int VEC = Vec16<T>::N;
  const VerifyArgs<T>& a;
  double* const sums;           // [2 DV_WAVES]
  uint32_t* const refused;      // [V bits] tokens of this row that were tried and not taken
  const int tid, lane, wave;
  __device__ __forceinline__ Walk(const VerifyArgs<T>& a, double* sums, uint32_t* refused)
      : a(a), sums(sums), refused(refused), tid(threadIdx.x), lane(threadIdx.x & 63), wave(threadIdx.x >> 6) {}
  __device__ __forceinline__ bool is_refused(int y) const { return (refused[y >> 5] >> (y & 31)) & 1; }
  // over the workgroup, in every thread, waves added in order
  __device__ __forceinline__ double total(double v) const {
    v = wave_total(v);
    __syncthreads();
    if (lane == 0) sums[wave] = v;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int w = 0; w < DV_WAVES; ++w) t += sums[w];
    return t;
  }
  __device__ RowStat stat(const T* row, double scale) const {
    float top = -INFINITY;
    bool nan = false;
    for (int y0 = tid * VEC; y0 < a.V; y0 += DV_THREADS * VEC) {
      float x[VEC];
      load_scores(row, y0, a.V, x);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        top = fmaxf(top, x[i]);
        nan |= x[i] != x[i];
      }
    }
    top = wave_max(top);
    const bool bad = __syncthreads_or(nan);
    float* const tops = reinterpret_cast<float*>(sums);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < DV_WAVES; ++w) top = fmaxf(top, tops[w]);
    RowStat s{top, a.V, 0.0, !bad && top != INFINITY && top != -INFINITY};
    if (!s.ok) return s;
    double e = 0.0;
    int at = a.V;
    for (int y0 = tid * VEC; y0 < a.V; y0 += DV_THREADS * VEC) {
      float x[VEC];
      load_scores(row, y0, a.V, x);
#pragma unroll
      for (int i = VEC - 1; i >= 0; --i) {
        if (x[i] == top) at = min(at, y0 + i);
        if (scale != 0.0) e += exp(((double)x[i] - top) * scale);
      }
    }
    s.total = scale != 0.0 ? total(e) : 1.0;
    // the first place: the smallest index, an exact maximum of 64-bit numbers
    double first = (double)-at;
#pragma unroll
    for (int d = 32; d; d >>= 1) first = fmax(first, __shfl_xor(first, d, WAVE));
    __syncthreads();
    if (lane == 0) sums[wave] = first;
    __syncthreads();
    for (int w = 0; w < DV_WAVES; ++w) first = fmax(first, sums[w]);
    s.at = (int)-first;
    return s;
  }
  // not normalised: divided by total it is the probability of y, whose score is x
  __device__ __forceinline__ double weight(const RowStat& s, double scale, float x, int y) const {
    return scale != 0.0 ? exp(((double)x - s.top) * scale) : y == s.at ? 1.0 : 0.0;
  }
  // The first y whose running sum of weights is above v of them all; per(y0, w) fills VEC weights from y0 on.  -1 where there is none.
  template <typename F> __device__ int sample(double v, F per) const {
    int lo = 0, n = a.V;              // the answer lies in [lo, lo + n)
    double before = 0.0, target = 0.0;
    for (bool first = true;; first = false) {
      const int part = ((n + DV_WAVES - 1) / DV_WAVES + VEC - 1) / VEC * VEC;   // of a wave
      double e = 0.0;
      for (int y0 = lo + wave * part + lane * VEC; y0 < min(lo + (wave + 1) * part, lo + n); y0 += 64 * VEC) {
        double w[VEC];
        per(y0, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) e += y0 + i < lo + n ? w[i] : 0.0;
      }
      e = wave_total(e);
      __syncthreads();
      if (lane == 0) sums[wave] = e;
      __syncthreads();
      if (first) {
        double all = 0.0;
        for (int w = 0; w < DV_WAVES; ++w) all += sums[w];
        if (!(all > 0.0)) return -1;
        target = v * all;
      }
      int at = -1;
      double here = before, base = before;
      for (int w = 0; w < DV_WAVES; ++w) {
        if (sums[w] > 0.0) {
          at = w;                     // rounding may leave the target above every sum: the last part that holds any
          base = here;
        }
        here += sums[w];
        if (at == w && here > target) break;
      }
      if (at < 0) return -1;
      lo += at * part;
      n = min(part, n - at * part);
      before = base;
      if (n <= 64) break;
    }
    __syncthreads();
    // one wave, a weight a lane
    double w[VEC], mine = 0.0;
    if (lane < n) {
      const int y0 = lo + lane / VEC * VEC;
      per(y0, w);
#pragma unroll
      for (int i = 0; i < VEC; ++i) mine = lane % VEC == i ? w[i] : mine;
    }
    double upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const double x = __shfl_up(upto, d, WAVE);
      if (lane >= d) upto += x;
    }
    const unsigned long long any = __builtin_amdgcn_ballot_w64(mine > 0.0), over = __builtin_amdgcn_ballot_w64(mine > 0.0 && before + upto > target);
    if (any == 0) return -1;
    return lo + (over ? __builtin_ctzll(over) : 63 - __builtin_clzll(any));
  }
};

template <typename T> __global__ void __launch_bounds__(DV_THREADS) draft_verify_walk(VerifyArgs<T> a, int b0) {
  constexpr int VEC = Vec16<T>::N;
  __shared__ double sums[2 * DV_WAVES];
  __shared__ int parent[DRAFT_MOST_ROWS];
  extern __shared__ __attribute__((aligned(16))) uint32_t dv_refused[];   // V bits
  const int tid = threadIdx.x, b = b0 + blockIdx.x;
  const RowRange r = ragged_rows(a.row_start, b, a.T_rows);
  const int n = min(r.count, a.max_new);
  int* const path = a.path + (long)b * a.max_new;
  if (tid < n) parent[tid] = draft_parent(a.parent[r.first + tid], tid);
  for (int i = tid; i < (a.V + 31) / 32; i += DV_THREADS) dv_refused[i] = 0;
  const Walk<T> walk(a, sums, dv_refused);
  double* const rest = a.rest + (long)b * a.V;
  int node = 0, kept = n > 0 ? 1 : 0, next = -1;
  if (tid == 0 && n > 0) path[0] = 0;
  __syncthreads();
  while (n > 0) {
    const T* const target = a.target + (long)(r.first + node) * a.V;
    const T* const draft = a.draft ? a.draft + (long)(r.first + node) * a.V : nullptr;
    const RowStat P = walk.stat(target, a.scale);
    if (!P.ok) break;   // no next token
    RowStat Q{};
    int child = node, taken = -1, tried = 0;
    double left = 1.0, q_left = 0.0, r_inv = 1.0;   // what the refused tokens have left of the target (no draft scores), of the draft, and of `rest`
    bool dead = false;                              // the target has nothing left
    while (!dead) {
      // the next child
      int mine = DRAFT_MOST_ROWS;
      const int i = tid;
      const bool is_child = i < n && i > child && parent[i] == node;
      const unsigned long long m = __builtin_amdgcn_ballot_w64(is_child);
      if (m) mine = (tid & ~63) + __builtin_ctzll(m);
      __syncthreads();
      int* const firsts = reinterpret_cast<int*>(sums);
      if ((tid & 63) == 0) firsts[tid >> 6] = mine;
      __syncthreads();
      child = DRAFT_MOST_ROWS;
      for (int w = 0; w < DV_WAVES; ++w) child = min(child, firsts[w]);
      __syncthreads();
      if (child >= n) break;
      if (draft && !tried && Q.total == 0.0) {
        Q = walk.stat(draft, a.draft_scale);
        if (!Q.ok) break;   // what was drawn from no distribution is not taken
        q_left = Q.total;
      }
      const int x = a.tokens[r.first + child];
      if (x < 0 || x >= a.V) continue;
      const bool before = walk.is_refused(x);
      const double q = !draft ? 1.0 : before && a.distinct ? 0.0 : walk.weight(Q, a.draft_scale, to_f32(draft[x]), x) / q_left;
      if (!(q > 0.0)) continue;
      double rx;
      if (!draft) rx = before ? 0.0 : walk.weight(P, a.scale, to_f32(target[x]), x) / P.total / left;
      else rx = tried ? rest[x] * r_inv : walk.weight(P, a.scale, to_f32(target[x]), x) / P.total;
      if ((double)a.u[r.first + child] * q < rx) {
        taken = child;
        break;
      }
      __syncthreads();
      if (tid == 0) dv_refused[x >> 5] |= 1u << (x & 31);
      __syncthreads();
      if (!draft) {
        if (!before) left -= walk.weight(P, a.scale, to_f32(target[x]), x) / P.total;
        dead = !(left > 0.0);
      } else {
        double all = 0.0, q_all = 0.0;
        for (int y0 = tid * VEC; y0 < a.V; y0 += DV_THREADS * VEC) {
          float xt[VEC], xd[VEC];
          if (!tried) load_scores(target, y0, a.V, xt);
          load_scores(draft, y0, a.V, xd);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const int y = y0 + i;
            if (y >= a.V) break;
            const double w = walk.weight(Q, a.draft_scale, xd[i], y);
            // of the tokens refused before this one the draft has nothing left, and the target neither
            const bool gone = a.distinct && walk.is_refused(y);
            const double p = tried ? rest[y] * r_inv : walk.weight(P, a.scale, xt[i], y) / P.total;
            const double now = fmax(p - (gone && y != x ? 0.0 : w / q_left), 0.0);
            rest[y] = now;
            all += now;
            if (!gone) q_all += w;
          }
        }
        all = walk.total(all);
        if (a.distinct) q_left = walk.total(q_all);
        dead = !(all > 0.0);
        r_inv = 1.0 / all;
      }
      ++tried;
    }
    if (taken < 0) {
      const double v = (double)a.v[b];
      auto target_weights = [&](int y0, double (&w)[VEC], bool without) {
        float xt[VEC];
        load_scores(target, y0, a.V, xt);
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[i] = y0 + i < a.V && !(without && walk.is_refused(y0 + i)) ? walk.weight(P, a.scale, xt[i], y0 + i) : 0.0;
      };
      if (tried && !dead) {
        if (draft) next = walk.sample(v, [&](int y0, double (&w)[VEC]) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) w[i] = y0 + i < a.V ? rest[y0 + i] : 0.0;
        });
        else next = walk.sample(v, [&](int y0, double (&w)[VEC]) { target_weights(y0, w, true); });
      }
      if (next < 0) next = walk.sample(v, [&](int y0, double (&w)[VEC]) { target_weights(y0, w, false); });
      break;
    }
    __syncthreads();
    if (tried)   // tokens refused here are children of this row
      for (int i = node + 1 + tid; i < n; i += DV_THREADS) {
        const int x = a.tokens[r.first + i];
        if (parent[i] == node && x >= 0 && x < a.V) dv_refused[x >> 5] = 0;
      }
    node = taken;
    if (tid == 0) path[kept] = node;
    ++kept;
    __syncthreads();
  }
  for (int i = kept + tid; i < a.max_new; i += DV_THREADS) path[i] = -1;
  if (tid == 0) {
    a.kept[b] = kept;
    a.next[b] = next;
  }
}

}  // namespace

size_t draft_verify_workspace_bytes(int B, int V) { return (size_t)B * V * sizeof(double) + 256; }
template <typename T> dipaco_status launch_draft_verify(const VerifyArgs<T>& a, hipStream_t s) {
  const int lds = (a.V + 31) / 32 * 4;
  launch_parts(a.B, [&](long long first, unsigned count) { draft_verify_walk<T><<<count, DV_THREADS, lds, s>>>(a, (int)first); });
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}
template dipaco_status launch_draft_verify<float>(const VerifyArgs<float>&, hipStream_t);
template dipaco_status launch_draft_verify<bf16>(const VerifyArgs<bf16>&, hipStream_t);

}  // namespace dipaco
