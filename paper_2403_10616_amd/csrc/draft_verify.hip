// Which drafted tokens stay, and the token behind them (include/dipaco_kernels.h has the rule): a workgroup walks a document's tree from row 0.
//
// A token hangs on a border (u q < r, a running sum above v times the whole), so exponentials, sums and what is left of the target are 64-bit numbers: then
// neither the order of a sum nor an exponential's last digits (2^-36 here) decide more than one draw in a million.
//
// A row of scores is cut into up to 32 parts of whole 1024 scores, a wave each: largest score, sum of exponentials against it.  From these the row's
// sum is formed, and the part that a drawn token lies in is found without reading the others again; only parts that hold refused tokens are summed anew.
//
// Bound: a document's walk is a chain of decisions in one compute unit.  There a row of 32000 scores takes 10 us, of which its 64-bit exponentials, 18 instructions
// each, are most, and a refusal by draft scores, which forms two of them for every token, 15.  So few rows' sums are formed by a launch of the whole chip ahead
// of the walks, whose decisions then cost 1.3 us each, reads of LDS one behind the other.  Us, 32000 tokens: one chain of 6, bf16, 4 + 12; 64 chains of up to 8,
// fp32, draft scores, 16 + 28; 32 trees of 64, bf16, 46; 24 trees of up to 40 with distinct siblings, 20011 tokens fp32, 13 + 51.
#include <algorithm>
#include <type_traits>

#include "draft.h"
#include "kernels.h"

namespace dipaco {

namespace {

constexpr int DV_THREADS = 512, DV_WAVES = DV_THREADS / 64, DV_PARTS = 32, DV_CHUNK = 1024;
constexpr double DV_LEAST_LEFT = 1.0 / 1024;   // of a row: what differences of probabilities, right to 2^-36 of the row, may leave, to 2^-26 of itself

// 2^t for t <= 0, to 2^-36 of it: 2^f = sum of (f ln 2)^k / k! for |f| <= 1/2, up to k = 9 (those left out are below 2^-37 together, 2^-36.6 of the least 2^f; each
// further one, 2^-5 of that, is an instruction more of 18)
__device__ __forceinline__ double power_of_two(double t) {
  t = fmax(t, -1100.0);   // what is far below, -inf and NaN: 0 in 64 bits
  const double n = rint(t), f = t - n;
  double p = 1.0178086009239696e-07;
  p = fma(p, f, 1.3215486790144305e-06);
  p = fma(p, f, 1.5252733804059838e-05);
  p = fma(p, f, 1.5403530393381606e-04);
  p = fma(p, f, 1.3333558146428441e-03);
  p = fma(p, f, 9.618129107628477e-03);
  p = fma(p, f, 5.5504108664821576e-02);
  p = fma(p, f, 2.402265069591007e-01);
  p = fma(p, f, 6.931471805599453e-01);
  p = fma(p, f, 1.0);
  return ldexp(p, (int)n);
}
template <int CTRL, int ROW_MASK> __device__ __forceinline__ double dpp_fetch64(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROW_MASK, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROW_MASK, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double lane_value(double v, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// lane i: the sum of lanes 0 .. i, in a fixed order
__device__ __forceinline__ double wave_upto(double v) {
  v += dpp_fetch64<0x111, 0xf>(v);   // row_shr 1, 2, 4, 8
  v += dpp_fetch64<0x112, 0xf>(v);
  v += dpp_fetch64<0x114, 0xf>(v);
  v += dpp_fetch64<0x118, 0xf>(v);
  v += dpp_fetch64<0x142, 0xa>(v);   // row_bcast15 into rows 1 and 3
  v += dpp_fetch64<0x143, 0xc>(v);   // row_bcast31 into rows 2 and 3
  return v;
}
__device__ __forceinline__ double wave_total(double v) { return lane_value(wave_upto(v), 63); }

// VEC scores from y0 on, which any address may hold; -inf behind the last
template <typename T> __device__ __forceinline__ void load_scores(const T* row, int y0, int V, float* x) {
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

// 2^((x - top) rate), 0 where x is -inf.  The difference first: it is 0 for x = top, and else off by 2^-53 of itself, however large both are (a mask's lowest value) and
// however large the rate.  x rate - top rate in one fma saves an instruction, and leaves the rounding of top rate, which passes 2^10 where that passes 2^63.
__device__ __forceinline__ double exponential(float x, double top, double rate) { return power_of_two(((double)x - top) * rate); }

// rate: log2(e) / temperature; 0: all probability at the first maximum
__device__ __forceinline__ double weight(double rate, float top, int at, float x, int y) {
  return rate != 0.0 ? exponential(x, top, rate) : y == at ? 1.0 : 0.0;
}

struct PartStat {
  float top;      // largest score
  int at;         // its first place (formed where rate is 0)
  double total;   // sum of 2^((x - top) rate); NaN where a score is NaN or +inf
};
struct Cut {
  int len, count;   // scores of a part, parts
  __host__ __device__ explicit Cut(int V) : len(((V + DV_PARTS - 1) / DV_PARTS + DV_CHUNK - 1) / DV_CHUNK * DV_CHUNK), count((V + len - 1) / len) {}
};

// 1024 scores of a row in a wave, 16 a lane
template <typename T> struct Scores {
  static constexpr int VEC = Vec16<T>::N;
  float x[16];
  __device__ __forceinline__ void load(const T* row, int base, int hi, int lane) {
#pragma unroll
    for (int i = 0; i < 16; i += VEC) load_scores(row, base + 64 * i + lane * VEC, hi, x + i);
  }
  static __device__ __forceinline__ int place(int base, int i, int lane) { return base + 64 * (i / VEC * VEC) + lane * VEC + i % VEC; }
};
// A part of a row, by a wave.  x: its first scores
template <typename T> __device__ __forceinline__ PartStat part_stat(const T* row, int lo, int hi, double rate, Scores<T>& x, int lane) {
  float top = -INFINITY;
  int at = 0x7fffffff;
  bool nan = false;
  double sum = 0.0;
  for (int base = lo;;) {
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      most = fmaxf(most, x.x[i]);
      nan |= x.x[i] != x.x[i];
    }
    if (rate == 0.0) {
      if (most > top) {
#pragma unroll
        for (int i = 15; i >= 0; --i)
          if (x.x[i] == most) at = Scores<T>::place(base, i, lane);
      }
      top = fmaxf(top, most);
    } else {
      if (most > top) {
        sum *= exponential(top, most, rate);
        top = most;
      }
      const double from = top;
      double s0 = 0.0, s1 = 0.0;
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        s0 += exponential(x.x[i], from, rate);
        s1 += exponential(x.x[i + 1], from, rate);
      }
      sum += s0 + s1;
    }
    base += DV_CHUNK;
    if (base >= hi) break;
    x.load(row, base, hi, lane);
  }
  PartStat p;
  p.top = wave_max(top);
  p.at = -1;
  if (rate == 0.0) {
    if (top != p.top) at = 0x7fffffff;
#pragma unroll
    for (int d = 32; d; d >>= 1) at = min(at, __shfl_xor(at, d, WAVE));
    p.at = at;
    p.total = 1.0;
  } else {
    p.total = wave_total(sum * exponential(top, p.top, rate));
  }
  if (__any(nan) || p.top == INFINITY) p.total = NAN;
  return p;
}

// A row, from its parts
struct RowStat {
  float top;
  int at;
  double inv;   // one over the sum; 0 where the row is no distribution
};
// of a part's sum against the row's largest score
__device__ __forceinline__ double part_total(const PartStat& p, float top, double rate) {
  return rate != 0.0 ? p.total * exponential(p.top, top, rate) : p.total;
}
// Two rows by a wave, a part a lane: lanes 0 .. 31 hold `p` and `rate` of one, lanes 32 .. 63 of the other (no part: top -inf, total 0).  Every lane gets its half's.
__device__ __forceinline__ RowStat join(const PartStat& p, double rate, int lane) {
  RowStat r;
  float top = p.top;
  top = fmaxf(top, dpp_fetch<0xb1, 0xf>(top, -INFINITY));
  top = fmaxf(top, dpp_fetch<0x4e, 0xf>(top, -INFINITY));
  top = fmaxf(top, dpp_fetch<0x141, 0xf>(top, -INFINITY));
  top = fmaxf(top, dpp_fetch<0x140, 0xf>(top, -INFINITY));
  top = fmaxf(top, dpp_fetch<0x142, 0xa>(top, -INFINITY));
  r.top = __shfl(top, lane | 31, WAVE);
  double total = p.total == 0.0 ? 0.0 : part_total(p, r.top, rate);
  total += dpp_fetch64<0x111, 0xf>(total);
  total += dpp_fetch64<0x112, 0xf>(total);
  total += dpp_fetch64<0x114, 0xf>(total);
  total += dpp_fetch64<0x118, 0xf>(total);
  total += dpp_fetch64<0x142, 0xa>(total);
  total = __shfl(total, lane | 31, WAVE);   // NaN stays
  const unsigned long long first = __builtin_amdgcn_ballot_w64(p.top == r.top) & (lane < 32 ? 0xffffffffull : 0xffffffffull << 32);
  r.at = __shfl(p.at, first ? __builtin_ctzll(first) : lane, WAVE);
  r.inv = total > 0.0 && r.top > -INFINITY ? rate != 0.0 ? 1.0 / total : 1.0 : 0.0;
  return r;
}

// Which rows' parts are formed ahead of the walks, by a launch of their own: [T rows][parts] of the target, then of the draft
enum Ahead { NO_ROWS, PARENTS, ALL_ROWS };

template <typename T> __device__ __forceinline__ void form_part(const VerifyArgs<T>& a, const Cut& cut, PartStat* parts, int row, int part, int lane) {
  const bool of_draft = row >= a.T_rows;
  const T* const scores = of_draft ? a.draft + (long)(row - a.T_rows) * a.V : a.target + (long)row * a.V;
  const int lo = part * cut.len, hi = min(lo + cut.len, a.V);
  Scores<T> x;
  x.load(scores, lo, hi, lane);
  const PartStat p = part_stat(scores, lo, hi, of_draft ? a.draft_rate : a.rate, x, lane);
  if (lane == 0) parts[(long)row * cut.count + part] = p;
}
// A part a wave
template <typename T> __global__ void __launch_bounds__(256) draft_verify_parts(VerifyArgs<T> a, PartStat* parts, int n_rows, Divisor count) {
  const int item = blockIdx.x * 4 + (threadIdx.x >> 6), row = count(item), part = item - row * (int)count.d;
  if (row < n_rows) form_part(a, Cut(a.V), parts, row, part, threadIdx.x & 63);
}
// Only parts of rows that have children: two thirds or so of a tree's rows are leaves, of which a walk ends at one at most
template <typename T> __global__ void __launch_bounds__(256) draft_verify_parents(VerifyArgs<T> a, PartStat* parts, int n_rows, Divisor count) {
  const int lane = threadIdx.x & 63, item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), row = count(item);
  if (row >= n_rows) return;
  const int at = row >= a.T_rows ? row - a.T_rows : row, b = __builtin_amdgcn_readfirstlane(find_document(a.row_start, a.B, at, lane));
  const RowRange r = ragged_rows(a.row_start, b, a.T_rows);
  const int n = min(r.count, a.max_new), i = at - r.first;
  bool has_child = false;
  for (int c = i + 1 + lane; c < n; c += 64) has_child |= draft_parent(a.parent[r.first + c], c) == i;
  if (i < 0 || i >= n || !__any(has_child)) return;
  form_part(a, Cut(a.V), parts, row, item - row * (int)count.d, lane);
}

// LDS of a walk: arrays of `rows`, then the bits of refused tokens
struct WalkRows {
  RowStat *p, *q;           // the row's own distributions (formed ahead, PARENTS: of rows that are)
  double *target, *draft;   // probabilities of the row's token behind its parent (formed ahead)
  float* u;
  int *parent, *token;
  uint32_t* refused;
  static constexpr int ROW_BYTES = 2 * (int)sizeof(RowStat) + 2 * 8 + 4 + 2 * 4;
  __device__ __forceinline__ WalkRows(char* at, int rows) {
    p = reinterpret_cast<RowStat*>(at);
    q = p + rows;
    target = reinterpret_cast<double*>(q + rows);
    draft = target + rows;
    u = reinterpret_cast<float*>(draft + rows);
    parent = reinterpret_cast<int*>(u + rows);
    token = parent + rows;
    refused = reinterpret_cast<uint32_t*>(token + rows);
  }
};

// AHEAD: whose parts have been formed; another row's are formed when the walk comes to it.  GREEDY: temperature 0.  Both are the
// kernel's because a branch at every score keeps the compiler from holding the series' coefficients: two copies a score where there is one now.
template <typename T, Ahead AHEAD, bool GREEDY>
__global__ void __launch_bounds__(DV_THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) draft_verify_walk(VerifyArgs<T> a, const PartStat* parts, int b0) {
  constexpr int VEC = Vec16<T>::N;
  __shared__ PartStat stats[2][DV_PARTS];   // of the walk's row: target, draft
  __shared__ double sums[DV_PARTS];
  __shared__ int drawn;
  extern __shared__ __attribute__((aligned(16))) char dv_smem[];
  const WalkRows rows(dv_smem, a.max_new);
  uint32_t* const refused = rows.refused;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = b0 + blockIdx.x;
  const Cut cut(a.V);
  const RowRange r = ragged_rows(a.row_start, b, a.T_rows);
  const int n = min(r.count, a.max_new);
  int* const path = a.path + (long)b * a.max_new;
  const double rate = GREEDY ? 0.0 : a.rate, draft_rate = a.draft_rate;
  const PartStat nothing{-INFINITY, -1, 0.0};
  if (AHEAD) {
    const bool of_draft = lane >= 32;
    const int part = lane & 31;
    const PartStat* const at = parts + (long)(r.first + (of_draft ? a.T_rows : 0)) * cut.count + part;
    const bool held = part < cut.count && (a.draft || !of_draft);
#pragma unroll 2
    for (int i = wave; i < n; i += DV_WAVES) {
      const RowStat x = join(held ? at[(long)i * cut.count] : nothing, of_draft ? draft_rate : rate, lane);
      if (lane == 0) rows.p[i] = x;
      if (lane == 32) rows.q[i] = x;
    }
  }
  for (int i = tid; i < n; i += DV_THREADS) {
    const int parent = draft_parent(a.parent[r.first + i], i), token = a.tokens[r.first + i];
    rows.parent[i] = parent;
    rows.token[i] = token;
    rows.u[i] = a.u[r.first + i];
    if (AHEAD && parent >= 0 && token >= 0 && token < a.V) {   // scores, until all rows' sums are in LDS
      const long at = (long)(r.first + parent) * a.V + token;
      rows.target[i] = to_f32(a.target[at]);
      if (a.draft) rows.draft[i] = to_f32(a.draft[at]);
    }
  }
  for (int i = tid; i < (a.V + 31) / 32; i += DV_THREADS) refused[i] = 0;
  __syncthreads();
  if (AHEAD)
    for (int i = tid; i < n; i += DV_THREADS) {
      const int parent = rows.parent[i], token = rows.token[i];
      if (parent < 0 || token < 0 || token >= a.V) continue;
      const RowStat p = rows.p[parent], q = rows.q[parent];
      rows.target[i] = weight(rate, p.top, p.at, (float)rows.target[i], token) * p.inv;
      if (a.draft) rows.draft[i] = weight(draft_rate, q.top, q.at, (float)rows.draft[i], token) * q.inv;
    }
  if (AHEAD) __syncthreads();
  auto is_refused = [&](int y) { return (refused[y >> 5] >> (y & 31)) & 1; };
  // bit i: token y0 + i has been refused; y0 is a multiple of VEC
  auto refused_from = [&](int y0) { return refused[y0 >> 5] >> (y0 & 31); };
  auto part_end = [&](int part) { return min((part + 1) * cut.len, a.V); };
  // a row's distribution, its parts left in stats[which]
  auto stat = [&](const T* row, double row_rate, int which) {
    __syncthreads();
    for (int part = wave; part < cut.count; part += DV_WAVES) {
      Scores<T> x;
      x.load(row, part * cut.len, part_end(part), lane);
      const PartStat p = part_stat(row, part * cut.len, part_end(part), row_rate, x, lane);
      if (lane == 0) stats[which][part] = p;
    }
    __syncthreads();
    return join((lane & 31) < cut.count ? stats[which][lane & 31] : nothing, row_rate, lane);   // the same in both halves
  };
  double* const rest = a.rest + (long)b * a.V;
  int node = 0, kept = n > 0 ? 1 : 0, next = -1;
  if (tid == 0 && n > 0) path[0] = 0;
  while (n > 0) {
    const T* const target = a.target + (long)(r.first + node) * a.V;
    const T* const draft = a.draft ? a.draft + (long)(r.first + node) * a.V : nullptr;
    auto next_child = [&](int after) {
      for (int i0 = (after + 1) & ~63; i0 < n; i0 += 64) {
        const int i = i0 + lane;
        const unsigned long long m = __builtin_amdgcn_ballot_w64(i < n && i > after && rows.parent[i] == node);
        if (m) return i0 + __builtin_ctzll(m);
      }
      return n;
    };
    int child = next_child(node);
    const bool formed = AHEAD == ALL_ROWS || (AHEAD == PARENTS && child < n);
    RowStat P;
    if (AHEAD != ALL_ROWS && !formed) P = stat(target, rate, 0);
    else P = rows.p[node];
    if (P.inv == 0.0) break;   // no next token
    RowStat Q{-INFINITY, -1, 0.0};
    if (AHEAD && draft) Q = rows.q[node];
    bool have_q = AHEAD != NO_ROWS;
    int taken = -1, tried = 0;
    // One over what the refused tokens have left: of the target (no draft scores), of the draft; of `rest`
    double left = 1.0, left_inv = 1.0, q_scale = 1.0, r_inv = 1.0;
    bool dead = false;   // the target has nothing left
    for (; !dead && child < n; child = next_child(child)) {
      if (draft && !have_q) {
        Q = stat(draft, draft_rate, 1);
        have_q = true;
      }
      if (draft && Q.inv == 0.0) break;   // what was drawn from no distribution is not taken
      const int x = rows.token[child];
      if (x < 0 || x >= a.V) continue;
      const bool before = tried && is_refused(x);
      const double px = AHEAD ? rows.target[child] : weight(rate, P.top, P.at, to_f32(target[x]), x) * P.inv;
      double q = 1.0, rx;
      if (draft) {
        const double qx = AHEAD ? rows.draft[child] : weight(draft_rate, Q.top, Q.at, to_f32(draft[x]), x) * Q.inv;
        q = before && a.distinct ? 0.0 : qx * q_scale;
        if (!(q > 0.0)) continue;
        rx = tried ? rest[x] * r_inv : px;
      } else {
        rx = before ? 0.0 : px * left_inv;
      }
      if ((double)rows.u[child] * q < rx) {
        taken = child;
        break;
      }
      __syncthreads();
      if (tid == 0) refused[x >> 5] |= 1u << (x & 31);
      __syncthreads();
      if (!draft) {
        if (!before) left -= px;
        // What is left after large shares is lost in their roundings: its own tokens' sum then.  A row comes to that once in 1/LEAST_LEFT times, and the sum's cost is no matter
        if (!GREEDY && left < DV_LEAST_LEFT) {
          const double top = P.top;
          double e = 0.0;
          for (int y = tid; y < a.V; y += DV_THREADS) e += is_refused(y) ? 0.0 : exponential(to_f32(target[y]), top, rate);
          e = wave_total(e);
          if (lane == 0) sums[wave] = e;
          __syncthreads();
          left = wave_total(lane < DV_WAVES ? sums[lane] : 0.0) * P.inv;
        }
        left_inv = 1.0 / left;
        dead = !(left > 0.0);
      } else {
        // rest <- max(what is left of the target - the draft, 0), and the sums of both
        const double q_inv = Q.inv * q_scale, p_top = P.top, q_top = Q.top;
        auto refuse = [&](auto FIRSTc, auto DISTINCTc) {
          constexpr bool FIRST = decltype(FIRSTc)::value, DISTINCT = decltype(DISTINCTc)::value;
          Scores<T> xd, xt, then_d, then_t;   // a 1024 of scores, and the next, on their way meanwhile
          if (wave < cut.count) {
            xd.load(draft, wave * cut.len, part_end(wave), lane);
            if (FIRST) xt.load(target, wave * cut.len, part_end(wave), lane);
          }
          for (int part = wave; part < cut.count; part += DV_WAVES) {
            const int lo = part * cut.len, hi = part_end(part);
            double all = 0.0, q_all = 0.0;
            for (int base = lo; base < hi; base += DV_CHUNK) {
              const bool same = base + DV_CHUNK < hi;
              const int then_part = same ? part : min(part + DV_WAVES, cut.count - 1), then_base = same ? base + DV_CHUNK : then_part * cut.len;
              then_d.load(draft, then_base, part_end(then_part), lane);
              if (FIRST) then_t.load(target, then_base, part_end(then_part), lane);
              double before[16];
              if (!FIRST)
#pragma unroll
                for (int i = 0; i < 16; ++i) before[i] = rest[min(Scores<T>::place(base, i, lane), hi - 1)];
#pragma unroll
              for (int j = 0; j < 16; j += VEC) {
                const int y0 = Scores<T>::place(base, j, lane);
                const uint32_t gone = DISTINCT && y0 < hi ? refused_from(y0) : 0;
                double now[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {   // a score of -inf behind the part's end: 0
                  double w = exponential(xd.x[j + i], q_top, draft_rate), p;
                  if (!FIRST) p = before[j + i] * r_inv;
                  else if (GREEDY) p = y0 + i == P.at ? 1.0 : 0.0;
                  else p = exponential(xt.x[j + i], p_top, rate) * P.inv;
                  if (DISTINCT) {   // of the tokens refused before this one the draft has nothing left, and the target neither
                    const bool is_gone = gone & (1u << i);
                    q_all += is_gone ? 0.0 : w;
                    w = is_gone && y0 + i != x ? 0.0 : w;
                  }
                  now[i] = fmax(fma(w, -q_inv, p), 0.0);
                }
                if (y0 + VEC <= hi) {
                  __builtin_memcpy(rest + y0, now, sizeof(now));
#pragma unroll
                  for (int i = 0; i < VEC; ++i) all += now[i];
                } else {
#pragma unroll
                  for (int i = 0; i < VEC; ++i)
                    if (y0 + i < hi) {
                      rest[y0 + i] = now[i];
                      all += now[i];
                    }
                }
              }
              xd = then_d;
              if (FIRST) xt = then_t;
            }
            all = wave_total(all);
            if (DISTINCT) q_all = wave_total(q_all);
            if (lane == 0) {
              sums[part] = all;
              stats[1][part].total = q_all;
            }
          }
        };
        if (tried) a.distinct ? refuse(std::false_type{}, std::true_type{}) : refuse(std::false_type{}, std::false_type{});
        else a.distinct ? refuse(std::true_type{}, std::true_type{}) : refuse(std::true_type{}, std::false_type{});
        __syncthreads();
        const double all = wave_total(lane < cut.count ? sums[lane] : 0.0);
        if (a.distinct) q_scale = 1.0 / (wave_total(lane < cut.count ? stats[1][lane].total : 0.0) * Q.inv);   // inf: the draft has nothing left
        dead = !(all > 0.0);
        r_inv = 1.0 / all;
      }
      ++tried;
    }
    if (taken < 0) {
      // The next token: from `rest`, whose parts' sums are in place, or from the target's row without the refused tokens, or from all of it
      const bool from_rest = draft && tried && !dead;
      bool without = !draft && tried && !dead;
      const double top = P.top;
      auto of_target = [&](float x, int y, uint32_t gone) { return gone & 1 ? 0.0 : GREEDY ? (y == P.at && x > -INFINITY ? 1.0 : 0.0) : exponential(x, top, rate); };   // x = -inf: behind what is summed
      // sum over lo .. hi - 1, by a wave; lo is a multiple of VEC
      auto weights = [&](int lo, int hi) {
        double e = 0.0;
        for (int base = lo; base < hi; base += DV_CHUNK) {
          if (from_rest) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int y = Scores<T>::place(base, i, lane);
              const double w = rest[min(y, hi - 1)];
              e += y < hi ? w : 0.0;
            }
          } else {
            Scores<T> x;
            x.load(target, base, hi, lane);
#pragma unroll
            for (int j = 0; j < 16; j += VEC) {
              const int y0 = Scores<T>::place(base, j, lane);
              const uint32_t gone = without && y0 < hi ? refused_from(y0) : 0;
#pragma unroll
              for (int i = 0; i < VEC; ++i) e += of_target(x.x[j + i], y0 + i, gone >> i);
            }
          }
        }
        return wave_total(e);
      };
      double all = 0.0;
      for (;;) {
        if (!from_rest) {
          constexpr int PER = DV_PARTS / DV_WAVES;
          const int part = wave + DV_WAVES * (lane % PER);   // a lane each of the wave's parts
          double of_part = 0.0;
          if (part < cut.count) {
            const PartStat p = formed ? parts[(long)(r.first + node) * cut.count + part] : stats[0][part];
            of_part = rate != 0.0 ? part_total(p, P.top, rate) : P.at >= part * cut.len && P.at < part_end(part) ? 1.0 : 0.0;
          }
          if (without)
            for (int i = 0; i < PER && wave + DV_WAVES * i < cut.count; ++i) {
              const int lo = (wave + DV_WAVES * i) * cut.len, hi = part_end(wave + DV_WAVES * i);
              bool anew = false;
              for (int w = (lo >> 5) + lane; w < (hi + 31) >> 5; w += 64) anew |= refused[w] != 0;
              if (__any(anew)) {
                const double e = weights(lo, hi);
                if (lane % PER == i) of_part = e;
              }
            }
          __syncthreads();
          if (lane < PER && part < cut.count) sums[part] = of_part;
          __syncthreads();
        }
        all = wave_total(lane < cut.count ? sums[lane] : 0.0);
        if (all > 0.0 || !without) break;
        without = false;   // random numbers outside their range may have refused every token
      }
      const double aim = (double)a.v[b] * all;
      // the first part whose running sum is above the aim; rounding may leave it above them all: the last that holds any
      int lo = 0, len = a.V;
      double before = 0.0;
      auto first_above = [&](double mine, double upto) {   // a lane each; -1: none holds any
        const unsigned long long any = __builtin_amdgcn_ballot_w64(mine > 0.0), over = __builtin_amdgcn_ballot_w64(mine > 0.0 && upto > aim);
        return any == 0 ? -1 : over ? __builtin_ctzll(over) : 63 - __builtin_clzll(any);
      };
      auto choose = [&](int n_parts, int part_len) {   // of sums[0 .. n_parts - 1]
        const double mine = lane < n_parts ? sums[lane] : 0.0, upto = before + wave_upto(mine);
        const int at = max(first_above(mine, upto), 0);
        if (at > 0) before = lane_value(upto, at - 1);
        lo += at * part_len;
        len = min(part_len, len - at * part_len);
        return at;
      };
      choose(cut.count, cut.len);
      if (len > DV_CHUNK) {   // then 1024 of it: cut.len is at most 8192
        const double e = lo + DV_CHUNK * wave < lo + len ? weights(lo + DV_CHUNK * wave, min(lo + DV_CHUNK * (wave + 1), lo + len)) : 0.0;
        __syncthreads();
        if (lane == 0) sums[wave] = e;
        __syncthreads();
        choose(DV_WAVES, DV_CHUNK);
      }
      // then two scores a thread
      static_assert(2 * DV_THREADS >= DV_CHUNK, "");
      double two[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int y = lo + 2 * tid + i, at = min(y, lo + len - 1);
        const double w = from_rest ? rest[at] : of_target(to_f32(target[at]), at, without ? is_refused(at) : 0);
        two[i] = y < lo + len ? w : 0.0;
      }
      const double both = two[0] + two[1], upto = wave_upto(both);
      __syncthreads();
      if (lane == 63) sums[wave] = upto;
      if (tid == 0) drawn = -1;
      __syncthreads();
      const int of_wave = choose(DV_WAVES, 128);
      if (wave == of_wave) {
        const int at = first_above(both, before + upto);
        if (lane == at) drawn = lo + 2 * lane + (two[0] > 0.0 && (before + (upto - both) + two[0] > aim || !(two[1] > 0.0)) ? 0 : 1);
      }
      __syncthreads();
      next = drawn;
      break;
    }
    if (tried) {   // tokens refused here are children of this row
      __syncthreads();
      for (int i = tid; i < n; i += DV_THREADS)
        if (rows.parent[i] == node && rows.token[i] >= 0 && rows.token[i] < a.V) refused[rows.token[i] >> 5] = 0;
      __syncthreads();
    }
    node = taken;
    if (tid == 0) path[kept] = node;
    ++kept;
  }
  for (int i = kept + tid; i < a.max_new; i += DV_THREADS) path[i] = -1;
  if (tid == 0) {
    a.kept[b] = kept;
    a.next[b] = next;
  }
}

// Parts that are formed ahead of the walks: all rows' up to DV_ALL_PARTS, then parents' up to DV_DRAWN_PARTS, or DV_PICKED_PARTS where there are no draft scores: a
// walk then forms a row once, not twice, and has no pass at a refusal, so that there is less to gain.  A parent is found by loads of 2 us.  32000 tokens, bf16 (f: fp32), chains or
// trees ("level"), us in the walk | parents ahead | all ahead, both launches:
//   draft scores, chains: 8 x 6, 116 | 33.5 | 32.2;  16 x 8, 8192 parts, 149 | 40.4 | 38.6;  8 x 40, 20480, 172 | 59 | 57;  64 x 8 f, 32768, 157 | 64 | 61;
//     16 x 40, 40960, 230 | 84 | 78;  128 x 8, 65536, 168 | 99 | 90;  256 x 8, 131072, 171 | 163 | 151;  512 x 4, 131072, 174 | 185 | 174
//   draft scores, trees: 24 x up to 40 f, distinct, 20011 tokens, 19080, 67 | 63 | 70;  8 x 64, 32768, 164 | 155 | 169;  32 x 16, 32768, 146 | 151 | 164;  16 x 64, 65536, 147 | 153 | 177
//   picked, trees: 2 x 64, 4096, 58 | 33.5 | 25.4;  4 x 64, 8192, 32 | 28 | 31;  8 x 64, 16384, 46 | 34 | 41;  16 x 64, 32768, 53 | 43 | 55;  64 x 16, 32768, 39 | 41 | 52;
//     32 x 64, 65536, 45 | 57 | 81;  128 x 16, 65536, 42 | 57 | 78
constexpr int64_t DV_ALL_PARTS = 1 << 12, DV_PICKED_PARTS = 1 << 15, DV_DRAWN_PARTS = 1 << 16;

}  // namespace

// [documents][V] of what the target has left, then the parts: as many as a row of V scores or fewer may have (their number falls where they get longer)
size_t draft_verify_workspace_bytes(int T_rows, int B, int V) {
  const int most = std::min(DV_PARTS, (V + DV_CHUNK - 1) / DV_CHUNK);
  return (size_t)B * V * sizeof(double) + 16 + (size_t)std::min<int64_t>(2 * (int64_t)T_rows * most, DV_DRAWN_PARTS) * sizeof(PartStat);
}
template <typename T> dipaco_status launch_draft_verify(const VerifyArgs<T>& a, hipStream_t s) {
  const Cut cut(a.V);
  const int n_rows = a.T_rows * (a.draft ? 2 : 1), lds = a.max_new * WalkRows::ROW_BYTES + (a.V + 31) / 32 * 4;
  const int64_t n = (int64_t)n_rows * cut.count;
  PartStat* const parts = reinterpret_cast<PartStat*>((reinterpret_cast<uintptr_t>(a.rest + (size_t)a.B * a.V) + 15) & ~(uintptr_t)15);
  auto walk = [&](auto AHEADc) -> dipaco_status {
    auto run = [&](auto GREEDYc) -> dipaco_status {
      constexpr Ahead AHEAD = decltype(AHEADc)::value;
      constexpr bool GREEDY = decltype(GREEDYc)::value;
      static std::atomic<unsigned long long> lds_set{0};
      if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(draft_verify_walk<T, AHEAD, GREEDY>), 128 << 10, lds_set)) return st;
      launch_parts(a.B, [&](long long first, unsigned count) { draft_verify_walk<T, AHEAD, GREEDY><<<count, DV_THREADS, lds, s>>>(a, parts, (int)first); });
      DIPACO_LAUNCH_CHECK();
      return DIPACO_OK;
    };
    return a.rate == 0.0 ? run(std::true_type{}) : run(std::false_type{});
  };
  using std::integral_constant;
  if (n == 0 || n > (a.draft ? DV_DRAWN_PARTS : DV_PICKED_PARTS)) return walk(integral_constant<Ahead, NO_ROWS>{});
  if (n <= DV_ALL_PARTS) {
    draft_verify_parts<T><<<(int)((n + 3) / 4), 256, 0, s>>>(a, parts, n_rows, Divisor(cut.count));
    DIPACO_LAUNCH_CHECK();
    return walk(integral_constant<Ahead, ALL_ROWS>{});
  }
  draft_verify_parents<T><<<(int)((n + 3) / 4), 256, 0, s>>>(a, parts, n_rows, Divisor(cut.count));
  DIPACO_LAUNCH_CHECK();
  return walk(integral_constant<Ahead, PARENTS>{});
}
template dipaco_status launch_draft_verify<float>(const VerifyArgs<float>&, hipStream_t);
template dipaco_status launch_draft_verify<bf16>(const VerifyArgs<bf16>&, hipStream_t);

}  // namespace dipaco
