// Sampling rules: a row of logits, a request's temperature, min-p, top-k and
// top-p, the distribution they leave and a token drawn from it.
//
// Definitions.  m = max l; e_j = exp((l_j - m) / T) in 64 bits; the integer
// mass of j is W_j = floor(e_j 2^43).  Candidates: l_j > -inf, e_j >= min_p.
// They are ordered by l (descending), the lower index first on ties; top_k
// keeps the first k; top_p keeps the shortest prefix of those whose mass is at
// least max(1, ceil(p * mass of the k)).  Every rule keeps a prefix of one
// order, so the result is one border: the key of the last candidate kept.
// prob_j = fl32(e_j 2^43 / mass of the kept), the draw is the fixed-point one
// of the other samplers.  Masses are integers: no border depends on how the
// sums are split.
//
// No sort: up to four launches, each over (chunk, row).
//   max    per chunk: maximum, its lowest index, NaN / +inf; maxima of each thread's
//          entries, and of groups of them where the row has a top-k
//   scan   rows with a top-k: the k-th largest group maximum, rounded down, bounds the
//          k-th largest logit from below, so the entries above it, little more than k
//          of them, are all that matters; they go to a list and the last workgroup of
//          the row selects the border in it, and the token where no probabilities are
//          wanted.  Exponentials of listed entries alone.
//          Rows with a top-p alone: masses in buckets of the distance from the
//          maximum, monotone in l; the last workgroup finds the border's bucket.
//          Rows with neither: the mass.
//   pick   (where a top-p is given) the border bucket's candidates go to the list; the
//          last workgroup selects the border in it
//   out    probabilities, and the draw: weights summed by 256 entries, the last
//          workgroup finds t's 256 and the token in them
// From scan on, threads whose maximum lies below the border (the bound) read nothing:
// a row with a border is read once or twice, not four times.  Lists of at most 256
// are ranked by comparing all pairs, longer ones by digits; a list that overflows
// is replaced by passes over the row itself, by one workgroup: slow, and right.  That
// takes thousands of equal logits; or a top-k past about 2400 (1 x 32000: 40 us at 2300,
// 157 at 2500); or one near the row's groups, 256 a chunk, or above, where there are
// so many rows that each has few chunks (640 rows of 32000, three chunks each: 117 us at
// 500, 507 at 760; 1536 rows, one each: 181 us at 200, 556 at 250).
//
// What bounds it.  Few rows: launches and the chains inside them (loads of the words
// before, one counter a row): 1 x 32000, top-k 50 17.5 us, 1000 31 us (a list past 256);
// 16 x 128256, top-p 37 to 42 us, in kernels of 6 + 13 + 13 + 11 us.  Many rows: the
// exponentials of rows without a top-k (64-bit, 25 instructions) and the bytes.
// 112 x 128256 with probabilities (57 MB read once, 57 MB written): top-k 50 62 us,
// 1.9 TB/s; top-k 1000 94 us; neither 96 us (read three times); top-p 105 us; greedy 31 us.
// Six workgroups a CU (kGridTarget): with four the scan of 112 mixed rows is 32 us, not
// 35, but the last launch 33, not 28.  No kernel may spill, for one that uses scratch
// memory starts late (scan of 16 x 128256: 22 us with 16 spilled registers, 12 us with
// none).  One workgroup of 1024 threads a row, all in one launch, was 34 us on
// 1 x 32000 (one CU issues every instruction of the row) and 194 us on 112 x 128256.
// A row's chunks have at least a quad a thread: half as much left half the groups
// empty (top-k 1000 of 32000 listed 1800 entries, not 1330).
#include <algorithm>

#include "device_common.h"
#include "internal.h"
#include "sampling_common.h"

namespace specdec {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kBuckets = 2304;                  // of distances below 44 powers of two (no mass past them)
constexpr int kList = 4096;                     // border candidates kept in LDS
constexpr int kPairs = kList / 2;               // with their masses
constexpr int kGroups = 4096;                   // group maxima of a row, at most
constexpr int kGridTarget = 1536;               // workgroups: six a CU
constexpr int kMaxChunks = 64;                  // per row (one per lane)
constexpr double kTwo43 = 8796093022208.0;

enum { ROW_GREEDY = 1, ROW_BAD = 2, ROW_ALL = 3, ROW_K = 4, ROW_P = 5 };

struct ChunkMax {
  float m;
  int i, bad, pad;
};
// A row's rules, as the launches use them.
struct Rules {
  double c;       // log2(e) / T: distances in powers of two
  double mp;
  double in, off; // distances below `in` pass min_p, above `off` fail it (between them the exponential decides)
  float p;
  int k, kind;    // kind: of a row without NaN, +inf, or only -inf
  int pad;
};
// One row's progress: the counters, which a launch's workgroups on any XCD add to,
// in a cache line of their own; then words that one workgroup of one launch writes
// and the next launches read.
struct RowWork {
  uint32_t done;    // workgroups of the present launch that have finished (the last resets it)
  uint32_t listed;  // candidates in the list
  uint32_t line[30];
  Rules rules;
  int kind, amax;
  float m;
  int drawn;        // the token is out
  int bucket, pad;  // ROW_P: the border's bucket, the mass of those before it and of all
  unsigned long long before, total;
  // result: the key of the last candidate kept (0: all), and the kept mass
  unsigned long long key, mass;
  uint32_t line2[6];
};
static_assert(sizeof(RowWork) == 256, "two lines a row");

// Buckets to a power of two over the first 16 of them, 8 to one from there: few,
// for each workgroup adds all of its own to the row's; enough that the border's,
// 0.4 V ln 2 / rate entries where the logits are normal and T is their deviation,
// goes into the list.
__host__ __device__ __forceinline__ int bucket_rate(int V) { return V <= 262144 ? 32 : 128; }
__host__ __device__ __forceinline__ int buckets_of(int rate) { return 16 * rate + 28 * 8; }
static_assert(16 * 128 + 28 * 8 <= kBuckets, "every rate's buckets");

// Rows' arrays, strides by the call's rows, vocabulary and chunks a row (NC).
struct RuleScratch {
  ChunkMax* cmax;              // [rows][NC]
  unsigned long long* draw;    // [rows][segments_of(V)] weights of the draw in 256 consecutive entries of a chunk
  RowWork* work;               // [rows]
  unsigned long long* mass;    // [rows][buckets_of(V's rate)]
  uint32_t* group;             // [rows][groups_of(NC)] ordered group maxima
  float* top;                  // [rows][NC][kThreads] maximum of each thread's entries
  unsigned long long* list;    // [rows][list_of(V)]
};
// (a chunk's last segment may be short)
__host__ __device__ __forceinline__ int segments_of(int V) { return (V + 255) / 256 + 2 * kMaxChunks; }
__host__ __device__ __forceinline__ int groups_of(int NC) { return NC * kThreads < kGroups ? NC * kThreads : kGroups; }
__host__ __device__ __forceinline__ int list_of(int V) { return V < kList ? V : kList; }
__host__ __device__ inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
// Grows with rows and V: a workspace of the largest call holds every call's.
__host__ __device__ inline size_t carve_rules(void* base, size_t rows, int V, RuleScratch* s) {
  size_t off = 0;
  char* p = (char*)base;
  auto take = [&](size_t n) { const size_t at = off; off = up256(off + n); return p + at; };
  // (chunks of all rows together: rows * ceil(kGridTarget / rows) at most)
  const size_t most = rows + kGridTarget - 1, chunks = rows * kMaxChunks < most ? rows * kMaxChunks : most;
  const size_t groups = rows * kGroups < chunks * kThreads ? rows * kGroups : chunks * kThreads;
  s->cmax = (ChunkMax*)take(chunks * sizeof(ChunkMax));
  s->draw = (unsigned long long*)take(rows * segments_of(V) * 8);
  s->work = (RowWork*)take(rows * sizeof(RowWork));
  s->mass = (unsigned long long*)take(rows * buckets_of(bucket_rate(V)) * 8);
  s->group = (uint32_t*)take(groups * 4);
  s->top = (float*)take(chunks * kThreads * 4);
  s->list = (unsigned long long*)take(rows * list_of(V) * 8);
  return off;
}

// ---------------------------------------------------------------- one row's rules
__device__ __forceinline__ int kind_of(const RulesArgs& a, int b) {
  const float T = a.temperature ? a.temperature[b] : 1.f, mp = a.min_p ? a.min_p[b] : 0.f;
  const float p = a.top_p ? a.top_p[b] : 1.f;
  const int k = a.top_k ? a.top_k[b] : 0;
  return !(T >= 0.f) || mp != mp || p != p ? ROW_BAD
         : T == 0.f                        ? ROW_GREEDY
         : k > 0 && k < a.V                ? ROW_K
         : p < 1.f                         ? ROW_P
                                           : ROW_ALL;
}
__device__ __forceinline__ Rules rules_of(const RulesArgs& a, int b) {
  const float T = a.temperature ? a.temperature[b] : 1.f, mp = a.min_p ? a.min_p[b] : 0.f;
  Rules r;
  r.p = a.top_p ? a.top_p[b] : 1.f;
  r.k = a.top_k ? a.top_k[b] : 0;
  r.c = 1.4426950408889634 / (double)T;
  r.mp = mp > 1.f ? 1.0 : (double)mp;  // (the most likely token always stays)
  const double d = r.mp > 0.0 ? -log2(r.mp) : 1e300;
  r.in = d * (1.0 - 1e-12) - 1e-12;
  r.off = d * (1.0 + 1e-12) + 1e-12;
  r.kind = kind_of(a, b);
  r.pad = 0;
  return r;
}
// Order of the logits as integers (-0 and 0 alike), and back.
__device__ __forceinline__ uint32_t ordered(float l) {
  const uint32_t u = __float_as_uint(l);
  const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return o == 0x7fffffffu ? 0x80000000u : o;
}
__device__ __forceinline__ float logit_of(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
// Order of the candidates: a larger key comes first.
__device__ __forceinline__ unsigned long long key_of(float l, int j) {
  return ((unsigned long long)ordered(l) << 32) | (uint32_t)~(uint32_t)j;
}
// 2^-t for 0 <= t < 2^20: 2^f = sum (f ln 2)^k / k! on |f| <= 1/2, the first
// term left out below 2^-52.
__device__ __forceinline__ double pow2_neg(double t) {
  constexpr double kC[12] = {6.93147180559945286e-01, 2.40226506959100722e-01, 5.55041086648215831e-02,
                             9.61812910762847688e-03, 1.33335581464284433e-03, 1.54035303933816088e-04,
                             1.52527338040598411e-05, 1.32154867901443095e-06, 1.01780860092396999e-07,
                             7.05491162080112336e-09, 4.44553827187081162e-10, 2.56784359934882055e-11};
  const double n = rint(t), f = n - t;
  double p = kC[11];
#pragma unroll
  for (int i = 10; i >= 0; --i) p = fma(p, f, kC[i]);
  return ldexp(fma(p, f, 1.0), -(int)n);
}
// Distance of l from the maximum in powers of two: e = 2^-distance.
__device__ __forceinline__ double distance(const Rules& r, float m, float l) { return ((double)m - (double)l) * r.c; }
__device__ __forceinline__ bool candidate(const Rules& r, float l, double t) {
  if (!(l > -INFINITY) || t > r.off) return false;
  return t < r.in || pow2_neg(t) >= r.mp;
}
// floor(e 2^43) (x < 2^52: the sum with 2^52 holds floor(x) in its low bits).
__device__ __forceinline__ unsigned long long mass_at(double t) {
  if (!(t < 44.0)) return 0ull;
  const double x = floor(pow2_neg(t) * kTwo43) + 4503599627370496.0;
  return (unsigned long long)__double_as_longlong(x) & 0xfffffffffffffull;
}
__device__ __forceinline__ int bucket_of(double t, int rate) {  // (rounding keeps the order; t < 44)
  const float x = (float)t;
  return x < 16.f ? (int)(x * (float)rate) : min(16 * rate + (int)((x - 16.f) * 8.f), buckets_of(rate) - 1);
}
// The least distance of a bucket.
__device__ __forceinline__ double bucket_edge(int i, int rate) {
  return i < 16 * rate ? (double)i / rate : 16.0 + (i - 16 * rate) / 8.0;
}
__device__ __forceinline__ float prob_at(double t, double scale) {
  return t < 150.0 ? (float)(pow2_neg(t) * scale) : 0.f;  // (past 2^-149 a float32 is 0)
}

// Entries of a chunk.
__host__ __device__ __forceinline__ int chunk_of(int V, int NC) { return ((V + NC - 1) / NC + 3) / 4 * 4; }
struct Where {
  int c, r, b, NC, j0, j1;
  const float* row;
};
__device__ __forceinline__ Where where(const RulesArgs& a) {
  Where w;
  w.c = blockIdx.x;
  w.r = blockIdx.y;
  w.b = w.r / a.rows;
  w.NC = gridDim.x;
  const int cs = chunk_of(a.V, w.NC);
  w.j0 = min(a.V, w.c * cs);
  w.j1 = min(a.V, w.j0 + cs);
  w.row = a.logits + (size_t)w.r * a.ld;
  return w;
}
// f(j, l) for the entries [j0, j1) of a row: Q quads a thread and round, loaded before the first is used.
template <int Q = 2, typename F>
__device__ __forceinline__ void each(const float* row, int j0, int j1, F f) {
  for (int base = j0 + 4 * threadIdx.x; base < j1; base += 4 * Q * kThreads) {
    float v[Q][4];
#pragma unroll
    for (int q = 0; q < Q; ++q) load_quad(row, base + 4 * q * kThreads, j1, 1, -INFINITY, v[q]);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = base + 4 * q * kThreads + e;
        if (j < j1) f(j, v[q][e]);
      }
      __builtin_amdgcn_sched_barrier(0);  // (the quads' exponentials one after the other: fewer registers, more waves)
    }
  }
}

// The row's word of the draw.
__device__ __forceinline__ uint32_t row_word(const RulesArgs& a, const Where& w) {
  if (a.rand) return a.rand[w.r];
  return draw_word(a.seed, w.b, a.step_dev ? *a.step_dev : a.step, a.purpose, a.index + w.r % a.rows);
}

template <typename T>
__device__ __forceinline__ void put(T* p, T v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T>
__device__ __forceinline__ T get(const T* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Whether this is the last workgroup of the row to get here (then the counter is
// back at zero).  Each wave's stores and atomics have completed before it counts.
__device__ __forceinline__ bool last_here(uint32_t* done, int n) {
  __shared__ int s_last;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t old = __hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = old == (uint32_t)(n - 1);
    if (s_last) put(done, 0u);
  }
  __syncthreads();
  return s_last;
}

// Exclusive prefix of v over the workgroup, and the total.
__device__ __forceinline__ unsigned long long block_prefix(unsigned long long v, unsigned long long& total,
                                                           unsigned long long* sh) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  unsigned long long incl = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const unsigned long long n = shfl_up_u64(incl, o);
    if (lane >= o) incl += n;
  }
  __syncthreads();
  if (lane == kWave - 1) sh[w] = incl;
  __syncthreads();
  unsigned long long before = 0;
  total = 0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    if (k < w) before += sh[k];
    total += sh[k];
  }
  return before + incl - v;
}

// Sum of v over the workgroup (every thread).
__device__ __forceinline__ unsigned long long block_total(unsigned long long v, unsigned long long* sh) {
  v = wave_sum_u64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  unsigned long long t = 0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) t += sh[k];
  return t;
}
// ceil(p * mass), at least 1.
__device__ __forceinline__ unsigned long long needed(float p, unsigned long long mass) {
  return max(1ull, (unsigned long long)ceil(max(0.0, (double)p) * (double)mass));
}

// A lower bound of the k-th largest of a wave's values: the largest prefix that k
// of them reach, bit by bit, until little more than k do.
template <int E>
__device__ __forceinline__ uint32_t wave_bound(const uint32_t (&v)[E], int k) {
  uint32_t x = 0u;
  for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
    int c = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) c += __popcll(__ballot(v[e] >= (x | bit)));
    if (c < k) continue;
    x |= bit;
    if (c <= k + k / 8 + 4) break;
  }
  return x;
}

// ---------------------------------------------------------------- max
// Groups of a row with a top-k, at most: one, four or sixteen maxima a thread of the
// scan.  (G groups leave G ln(G / (G - k)) entries above their k-th largest maximum
// where the logits' order is random: 1.15 k at G = 4 k, 1.4 k at 2 k.)
__host__ __device__ __forceinline__ int group_limit(int k) { return k <= 64 ? kThreads : k <= 256 ? 4 * kThreads : kGroups; }
// Lanes to a group.
__host__ __device__ __forceinline__ int group_lanes(int NC, int k) {
  int n = 1;
  while (n < kWave && NC * kThreads / n > group_limit(k)) n *= 2;
  return n;
}
__global__ __launch_bounds__(kThreads) void rules_max_kernel(RulesArgs a) {
  __shared__ float sm[kWaves];
  __shared__ int si[kWaves], sb[kWaves];
  RuleScratch sc;
  carve_rules(a.scratch, (size_t)a.B * a.rows, a.V, &sc);
  const Where w = where(a);
  const int kind = kind_of(a, w.b);
  float m = -INFINITY;
  int at = 0x7fffffff, bad = 0;
  each<4>(w.row, w.j0, w.j1, [&](int j, float l) {
    bad |= !(l < INFINITY);  // (NaN or +inf)
    if (l > m) { m = l; at = j; }
  });
  sc.top[((size_t)w.r * w.NC + w.c) * kThreads + threadIdx.x] = m;
  if (kind == ROW_K) {
    const int gl = group_lanes(w.NC, a.top_k[w.b]);
    float gm = m;
    for (int o = 1; o < gl; o <<= 1) gm = fmaxf(gm, __shfl_xor(gm, o, kWave));
    if (threadIdx.x % gl == 0) sc.group[(size_t)w.r * groups_of(w.NC) + (w.c * kThreads + threadIdx.x) / gl] = ordered(gm);
  } else if (kind == ROW_P) {
    for (int i = w.c * kThreads + threadIdx.x; i < buckets_of(bucket_rate(a.V)); i += w.NC * kThreads) sc.mass[(size_t)w.r * buckets_of(bucket_rate(a.V)) + i] = 0ull;
  }
  const float wm = wave_max(m);
  at = m == wm ? at : 0x7fffffff;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) at = min(at, __shfl_xor(at, o, kWave));
  bad = __any(bad);
  if ((threadIdx.x & 63) == 0) {
    sm[threadIdx.x >> 6] = wm;
    si[threadIdx.x >> 6] = at;
    sb[threadIdx.x >> 6] = bad;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    ChunkMax t{sm[0], si[0], sb[0], 0};
    for (int k = 1; k < kWaves; ++k) {
      if (sm[k] > t.m || (sm[k] == t.m && si[k] < t.i)) { t.m = sm[k]; t.i = si[k]; }
      t.bad |= sb[k];
    }
    sc.cmax[(size_t)w.r * w.NC + w.c] = t;
    if (w.c == 0) {
      sc.work[w.r].done = 0u;
      sc.work[w.r].listed = 0u;
      sc.work[w.r].drawn = 0;
      sc.work[w.r].rules = rules_of(a, w.b);
    }
  }
}

// The row's maximum from its chunks (every wave, the same result).
__device__ __forceinline__ ChunkMax row_max(const ChunkMax* parts, int NC) {
  const int lane = threadIdx.x & 63;
  ChunkMax t{-INFINITY, 0x7fffffff, 0, 0};
  if (lane < NC) t = parts[lane];
  const float m = wave_max(t.m);
  int i = t.m == m ? t.i : 0x7fffffff;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) i = min(i, __shfl_xor(i, o, kWave));
  return ChunkMax{m, i, __any(t.bad), 0};
}

// ---------------------------------------------------------------- selection
constexpr int kFew = 128;
struct Select {
  alignas(16) unsigned long long hist_m[2 * kFew];
  uint32_t hist_c[256];
  unsigned long long sum[kWaves], lo[kWaves], hi[kWaves];
  int digit;
  uint32_t left, n_few;
  unsigned long long before, result;
};

// Extremes of lo and hi over the workgroup (every thread).
__device__ __forceinline__ void block_extremes(unsigned long long& lo, unsigned long long& hi, Select& sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, (unsigned long long)__shfl_xor(lo, o, kWave));
    hi = max(hi, (unsigned long long)__shfl_xor(hi, o, kWave));
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    sh.lo[threadIdx.x >> 6] = lo;
    sh.hi[threadIdx.x >> 6] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    lo = min(lo, sh.lo[k]);
    hi = max(hi, sh.hi[k]);
  }
}

// At most a workgroup's width of entries, by 1, 2 or 4 threads an entry (`parts`;
// thread t: entry t / parts): how many of them come before `key`, and their mass.
// pair: {key, mass}, zeros behind the last up to a multiple of 8.
__device__ __forceinline__ int parts_of(int n) { return 4 * n <= kThreads ? 4 : 2 * n <= kThreads ? 2 : 1; }
__device__ __forceinline__ int rank_pairs(const ulonglong2* pair, int n, int parts, unsigned long long key,
                                          unsigned long long& before) {
  int rank = 0;
  before = 0;
  for (int i = 8 * (threadIdx.x & (parts - 1)); i < n; i += 8 * parts) {
    ulonglong2 p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = pair[i + e];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool first = p[e].x > key;
      rank += first;
      before += first ? p[e].y : 0ull;
    }
  }
  for (int o = 1; o < parts; o <<= 1) {
    rank += __shfl_xor(rank, o, kWave);
    before += (unsigned long long)__shfl_xor(before, o, kWave);
  }
  return rank;
}

// The key of the last kept when the first `rest` of src's entries (by_mass: the
// fewest whose mass reaches `rest`) are kept, larger keys first.  src(f):
// f(key, mass) for every entry, keys distinct.  Radix selection from the highest bit
// in which the keys differ, 8 bits a pass, until few entries share the prefix: these
// are ranked.
template <typename SRC>
__device__ __forceinline__ unsigned long long select_border(SRC src, unsigned long long rest, bool by_mass, Select& sh) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  unsigned long long lo = ~0ull, hi = 0ull;
  src([&](unsigned long long key, unsigned long long) {
    lo = min(lo, key);
    hi = max(hi, key);
  });
  block_extremes(lo, hi, sh);
  int top = lo == hi ? 0 : 64 - __clzll((long long)(lo ^ hi));  // differing bits: [0, top)
  unsigned long long prefix = top >= 64 ? 0ull : hi >> top << top;
  while (top > 0) {
    const int shift = top > 8 ? top - 8 : 0, bits = top - shift;
    for (int i = threadIdx.x; i < 256; i += kThreads) {
      sh.hist_m[i] = 0ull;
      sh.hist_c[i] = 0u;
    }
    __syncthreads();
    src([&](unsigned long long key, unsigned long long m) {
      if (top < 64 && (key >> top) != (prefix >> top)) return;
      const int d = (int)((key >> shift) & ((1u << bits) - 1u));
      atomicAdd(&sh.hist_c[d], 1u);
      if (by_mass) atomicAdd(&sh.hist_m[d], m);
    });
    __syncthreads();
    if (w == 0) {  // larger keys first: lane i looks at digits 255 - 4i and the three below
      unsigned long long v[4], sum = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = 255 - 4 * lane - e;
        v[e] = by_mass ? sh.hist_m[d] : sh.hist_c[d];
        sum += v[e];
      }
      unsigned long long before = sum;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const unsigned long long n = shfl_up_u64(before, o);
        if (lane >= o) before += n;
      }
      before -= sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (before < rest && rest <= before + v[e]) {
          sh.digit = 255 - 4 * lane - e;
          sh.before = before;
          sh.left = sh.hist_c[255 - 4 * lane - e];
        }
        before += v[e];
      }
    }
    __syncthreads();
    rest -= sh.before;
    prefix |= (unsigned long long)sh.digit << shift;
    top = shift;
    if (sh.left <= (uint32_t)kFew) break;
  }
  // the entries that share the prefix, in the histogram's place
  ulonglong2* few = (ulonglong2*)sh.hist_m;
  if (threadIdx.x < kFew) few[threadIdx.x] = make_ulonglong2(0ull, 0ull);
  if (threadIdx.x == 0) sh.n_few = 0u;  // (not `left`, which other waves may not have read yet)
  __syncthreads();
  src([&](unsigned long long key, unsigned long long m) {
    if (top >= 64 || (key >> top) == (prefix >> top)) few[atomicAdd(&sh.n_few, 1u)] = make_ulonglong2(key, by_mass ? m : 1ull);
  });
  __syncthreads();
  const int n = (int)sh.n_few, parts = parts_of(n), at = threadIdx.x / parts;
  const ulonglong2 own = at < n ? few[at] : make_ulonglong2(0ull, 0ull);
  unsigned long long before;
  rank_pairs(few, n, parts, own.x, before);
  if (before < rest && rest <= before + own.y) sh.result = own.x;  // (one entry)
  __syncthreads();
  return sh.result;
}
// The mass of src's entries from `key` on.
template <typename SRC>
__device__ __forceinline__ unsigned long long mass_from(SRC src, unsigned long long key, Select& sh) {
  unsigned long long sum = 0;
  src([&](unsigned long long k, unsigned long long m) {
    if (k >= key) sum += m;
  });
  return block_total(sum, sh.sum);
}
// A row with a top-k (and a top-p), from entries that hold its first k: the border, the mass kept.
template <typename SRC>
__device__ __forceinline__ void border_k(const Rules& r, SRC src, unsigned long long& key, unsigned long long& mass,
                                         Select& sh) {
  unsigned long long count = 0, lo = ~0ull, hi = 0;
  mass = 0;
  src([&](unsigned long long k, unsigned long long m) {
    ++count;
    mass += m;
    lo = min(lo, k);
  });
  count = block_total(count, sh.sum);
  if (count > (unsigned long long)r.k) {
    key = select_border(src, (unsigned long long)r.k, false, sh);
    mass = mass_from(src, key, sh);
  } else {  // (min_p or -inf leaves no more)
    mass = block_total(mass, sh.sum);
    block_extremes(lo, hi, sh);
    key = lo;
  }
  if (r.p < 1.f) {
    key = select_border(src, needed(r.p, mass), true, sh);
    mass = mass_from(src, key, sh);
  }
}
// The bucket of a top-p row's border, the mass before it, the mass of all: get_mass(i) of the buckets.
struct Border {
  int bucket;
  unsigned long long before, total;
};
template <typename GET>
__device__ __forceinline__ void find_bucket(float p, int nb, GET get_mass, Border* out, unsigned long long* sh) {
  constexpr int PT = kBuckets / kThreads;  // thread t holds PT buckets from PT t
  unsigned long long tm[PT], sum = 0, total;
#pragma unroll
  for (int i = 0; i < PT; ++i) tm[i] = (int)threadIdx.x * PT + i < nb ? get_mass(threadIdx.x * PT + i) : 0ull;
#pragma unroll
  for (int i = 0; i < PT; ++i) sum += tm[i];
  unsigned long long mm = block_prefix(sum, total, sh);
  const unsigned long long need = needed(p, total);
#pragma unroll
  for (int i = 0; i < PT; ++i) {
    if (mm < need && need <= mm + tm[i]) *out = Border{(int)threadIdx.x * PT + i, mm, total};  // (one thread)
    mm += tm[i];
  }
}
// Whether a logit lies in a bucket.  Those that do lie within [lo, hi]: its edges
// in powers of two, widened past every rounding; the exact test decides.
struct Inside {
  float lo, hi;
  int bucket, rate;
  __device__ __forceinline__ Inside(const Rules& r, float m, int b, int rt) : lo(-INFINITY), hi(INFINITY), bucket(b), rate(rt) {
    if (r.c > 0.0 && r.c < 1e30) {
      const double t0 = bucket_edge(b, rt), t1 = bucket_edge(b + 1, rt);
      const double slack = 1e-5 * (fabs((double)m) + t1 / r.c) + 1e-40;
      hi = (float)((double)m - t0 / r.c + slack);
      lo = (float)((double)m - t1 / r.c - slack);
    }
  }
  __device__ __forceinline__ bool operator()(const Rules& r, float m, float l, double& t) const {
    if (!(l >= lo && l <= hi)) return false;
    t = distance(r, m, l);
    return t < 44.0 && candidate(r, l, t) && bucket_of(t, rate) == bucket;
  }
};
// What the rules leave of an entry.
struct Kept {
  unsigned long long key;
  float edge;
  double scale;
  __device__ __forceinline__ Kept(unsigned long long key_, unsigned long long mass)
      : key(key_), edge(key_ ? logit_of((uint32_t)(key_ >> 32)) : -INFINITY), scale(kTwo43 / (double)mass) {}
  __device__ __forceinline__ float operator()(const Rules& r, float m, int j, float l) const {
    if (key) {  // (a known border settles it without an exponential; what is above it passes min_p)
      if (!(l >= edge) || key_of(l, j) < key) return 0.f;
      return prob_at(distance(r, m, l), scale);
    }
    const double t = distance(r, m, l);
    return candidate(r, l, t) ? prob_at(t, scale) : 0.f;
  }
};
__device__ __forceinline__ void store4(float* p, int j, int end, const float (&v)[4]) {
  if (j + 4 <= end) *(f32x4_a4*)(p + j) = f32x4{v[0], v[1], v[2], v[3]};
  else
    for (int e = 0; j + e < end; ++e) p[j + e] = v[e];
}

// A row's list.  Entries go to the workgroup's own first (LDS), then with one
// reservation to the row's.
struct Gather {
  uint32_t n, at;
};
__device__ __forceinline__ void gather_add(Gather& g, unsigned long long* keys, unsigned long long key) {
  const uint32_t at = atomicAdd(&g.n, 1u);
  if (at < (uint32_t)kList) keys[at] = key;
}
__device__ __forceinline__ void gather_flush(Gather& g, const unsigned long long* keys, RowWork* work, unsigned long long* list) {
  __syncthreads();
  const uint32_t n = g.n;
  if (n == 0) return;  // (workgroup-uniform)
  if (threadIdx.x == 0) g.at = __hip_atomic_fetch_add(&work->listed, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  const uint32_t at = g.at;
  for (uint32_t i = threadIdx.x; i < min(n, (uint32_t)kList) && at + i < (uint32_t)kList; i += kThreads) put(&list[at + i], keys[i]);
}

// f(i, key) for the row's list, its loads in flight eight at a time.
template <typename F>
__device__ __forceinline__ void read_list(const unsigned long long* list, uint32_t n, F f) {
  constexpr int E = 8;
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += E * kThreads) {
    unsigned long long k[E];
#pragma unroll
    for (int e = 0; e < E; ++e) k[e] = get(&list[min(i0 + e * kThreads, n - 1)]);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (i0 + e * kThreads < n) f(i0 + e * kThreads, k[e]);
  }
}

// ---------------------------------------------------------------- scan
__global__ __launch_bounds__(kThreads, 4) void rules_scan_kernel(RulesArgs a) {
  __shared__ union {
    unsigned long long key[kList];
    unsigned long long mass[kBuckets];
    uint32_t hist[256];
    ulonglong2 pair[kPairs];
  } sh;
  __shared__ Select sel;
  __shared__ Gather gather;
  __shared__ Border s_border;
  __shared__ struct {
    float m;
    int kind;
    uint32_t bound[kWaves];
  } s_row;
  RuleScratch sc;
  carve_rules(a.scratch, (size_t)a.B * a.rows, a.V, &sc);
  const Where w = where(a);
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const uint32_t* group = sc.group + (size_t)w.r * groups_of(w.NC);
  const uint32_t first = group[lane * kWaves + wv];  // (of use where the row has a top-k)
  const Rules r = sc.work[w.r].rules;
  RowWork* work = sc.work + w.r;
  const float top = sc.top[((size_t)w.r * w.NC + w.c) * kThreads + threadIdx.x];
  if (r.kind == ROW_K) {
    // A lower bound of the k-th largest logit: each wave's of the (k / 4)-th largest of
    // every fourth group maximum, and the least of these (fewer groups than k: none).
    const int n = w.NC * kThreads / group_lanes(w.NC, r.k), k = (r.k + kWaves - 1) / kWaves, at0 = lane * kWaves + wv;
    uint32_t bound = 0u;
    auto of = [&](auto& v) {
      constexpr int E = sizeof(v) / sizeof(uint32_t);
      v[0] = at0 < n ? first : 0u;
#pragma unroll
      for (int i = 1; i < E; ++i) v[i] = i * kThreads + at0 < n ? group[i * kThreads + at0] : 0u;
      return wave_bound(v, k);
    };
    uint32_t v1[1], v4[4], v16[kGroups / kThreads];
    if (n >= r.k + kWaves) bound = n <= kThreads ? of(v1) : n <= 4 * kThreads ? of(v4) : of(v16);
    if (lane == 0) s_row.bound[wv] = bound;
  }
  if (wv == 0) {
    const ChunkMax mx = row_max(sc.cmax + (size_t)w.r * w.NC, w.NC);
    const int kind = mx.bad || mx.m == -INFINITY ? ROW_BAD : r.kind;
    if (lane == 0) {
      s_row.m = mx.m;
      s_row.kind = kind;
      gather.n = 0u;
      if (w.c == 0) {  // (for the launches after this one)
        work->kind = kind;
        work->amax = mx.i;
        work->m = mx.m;
        if (kind == ROW_BAD) set_status(a.status, kStatusNonFinite);
      }
    }
  }
  __syncthreads();
  const int kind = s_row.kind;
  const float m = s_row.m;
  if (kind == ROW_BAD || kind == ROW_GREEDY) return;  // (workgroup-uniform, as all that follows from the row's words)

  if (kind == ROW_ALL) {
    unsigned long long sum = 0;
    each(w.row, w.j0, w.j1, [&](int, float l) {
      const double t = distance(r, m, l);
      if (candidate(r, l, t)) sum += mass_at(t);
    });
    sum = block_total(sum, sel.sum);
    unsigned long long* parts = sc.draw + (size_t)w.r * segments_of(a.V);
    if (threadIdx.x == 0) put(&parts[w.c], sum);
    if (!last_here(&work->done, w.NC)) return;
    const unsigned long long all = wave_sum_u64(lane < w.NC ? get(&parts[lane]) : 0ull);
    if (threadIdx.x == 0) {
      work->key = 0ull;
      work->mass = all;
    }
    return;
  }

  if (kind == ROW_P) {
    const int rate = bucket_rate(a.V), nb = buckets_of(rate);
    for (int i = threadIdx.x; i < nb; i += kThreads) sh.mass[i] = 0ull;
    __syncthreads();
    each(w.row, w.j0, w.j1, [&](int, float l) {
      const double t = distance(r, m, l);
      if (!candidate(r, l, t)) return;
      const unsigned long long W = mass_at(t);
      if (W) atomicAdd(&sh.mass[bucket_of(t, rate)], W);
    });
    __syncthreads();
    unsigned long long* mass = sc.mass + (size_t)w.r * buckets_of(bucket_rate(a.V));
    for (int i = threadIdx.x; i < nb; i += kThreads)
      if (sh.mass[i]) __hip_atomic_fetch_add(&mass[i], sh.mass[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!last_here(&work->done, w.NC)) return;
    find_bucket(r.p, nb, [&](int i) { return get(&mass[i]); }, &s_border, sel.sum);
    __syncthreads();
    if (threadIdx.x == 0) {
      work->bucket = s_border.bucket;
      work->before = s_border.before;
      work->total = s_border.total;
    }
    return;
  }

  // ROW_K
  uint32_t bound = s_row.bound[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) bound = min(bound, s_row.bound[i]);
  unsigned long long* list = sc.list + (size_t)w.r * list_of(a.V);
  // (nor are those whose probability is 0: a mask of the lowest value fills no list)
  const float low = (float)((double)m - 151.0 / r.c);
  if (ordered(top) >= bound && top >= low)  // (few of the threads have anything to read)
    each(w.row, w.j0, w.j1, [&](int j, float l) {
      if (ordered(l) >= bound && l >= low && l > -INFINITY) gather_add(gather, sh.key, key_of(l, j));
    });
  gather_flush(gather, sh.key, work, list);
  if (!last_here(&work->done, w.NC)) return;

  const uint32_t n = get(&work->listed);
  const bool draw = a.out && !a.probs && n <= (uint32_t)kThreads;  // (longer lists: as rows without one)
  unsigned long long mass = 0, key = ~0ull;
  if (n <= (uint32_t)kThreads) {
    const int parts = parts_of(n), at = threadIdx.x / parts;
    const bool own = threadIdx.x % parts == 0;
    unsigned long long k0 = 0, m0 = 0;  // the thread's candidate, its mass
    if (at < (int)n) {
      k0 = get(&list[at]);
      const float l = logit_of((uint32_t)(k0 >> 32));
      const double t = distance(r, m, l);
      if (candidate(r, l, t)) m0 = mass_at(t);
      else k0 = 0;
    }
    sh.pair[threadIdx.x] = make_ulonglong2(0ull, 0ull);
    __syncthreads();
    if (own) sh.pair[at] = make_ulonglong2(k0, m0);
    const int count = __syncthreads_count(own && k0 != 0);
    unsigned long long before;
    const int rank = rank_pairs(sh.pair, n, parts, k0, before);
    const bool kept = k0 && rank < r.k;
    mass = block_total(own && kept ? m0 : 0ull, sel.sum);
    const unsigned long long need = r.p < 1.f ? needed(r.p, mass) : 0ull;
    if (kept && (need ? before < need && need <= before + m0 : rank == min(r.k, count) - 1)) {  // (one entry)
      sel.lo[0] = k0;
      sel.hi[0] = need ? before + m0 : mass;
    }
    __syncthreads();
    key = sel.lo[0];
    mass = sel.hi[0];
    if (draw) {  // (the lower index first: by the low words, which hold its complement)
      const uint32_t low = (uint32_t)k0;
      const unsigned long long R =
          k0 >= key ? fp_weight(prob_at(distance(r, m, logit_of((uint32_t)(k0 >> 32))), kTwo43 / (double)mass)) : 0ull;
      if (own) sh.pair[at] = make_ulonglong2(low, R);
      const unsigned long long S = block_total(own ? R : 0ull, sel.sum);
      const unsigned long long t = scale_word(row_word(a, w), S);
      rank_pairs(sh.pair, n, parts, low, before);
      if (before <= t && t < before + R) a.out[(size_t)w.r * a.ld_out] = (int32_t)~low;
    }
  } else {
    const bool listed = n <= (uint32_t)kList;
    // The candidates among them (those that fail min_p get the key 0): f(key, mass).
    const bool paired = n <= (uint32_t)kPairs;
    if (listed)
      read_list(list, n, [&](uint32_t i, unsigned long long k) {
        const float l = logit_of((uint32_t)(k >> 32));
        const double t = distance(r, m, l);
        if (!candidate(r, l, t)) k = 0ull;
        if (paired) sh.pair[i] = make_ulonglong2(k, mass_at(t));
        else sh.key[i] = k;
      });
    __syncthreads();
    auto src = [&](auto f) {
      if (paired) {
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
          const ulonglong2 p = sh.pair[i];
          if (p.x) f(p.x, p.y);
        }
      } else if (listed) {
        for (uint32_t i = threadIdx.x; i < n; i += kThreads)
          if (sh.key[i]) f(sh.key[i], mass_at(distance(r, m, logit_of((uint32_t)(sh.key[i] >> 32)))));
      } else {
        each(w.row, 0, a.V, [&](int j, float l) {
          if (ordered(l) < bound) return;
          const double t = distance(r, m, l);
          if (candidate(r, l, t)) f(key_of(l, j), mass_at(t));
        });
      }
    };
    border_k(r, src, key, mass, sel);
  }
  if (threadIdx.x == 0) {
    work->key = key;
    work->mass = mass;
    work->drawn = draw;
  }
}

// ---------------------------------------------------------------- pick
__global__ __launch_bounds__(kThreads) void rules_pick_kernel(RulesArgs a) {
  __shared__ union {
    unsigned long long key[kList];
    ulonglong2 pair[kPairs];
  } sh;
  __shared__ Select sel;
  __shared__ Gather gather;
  RuleScratch sc;
  carve_rules(a.scratch, (size_t)a.B * a.rows, a.V, &sc);
  const Where w = where(a);
  RowWork* work = sc.work + w.r;
  if (work->kind != ROW_P) return;  // (workgroup-uniform, as all that follows from the row's words)
  const Rules r = work->rules;
  const float m = work->m;
  const Inside inside(r, m, work->bucket, bucket_rate(a.V));
  unsigned long long* list = sc.list + (size_t)w.r * list_of(a.V);
  if (threadIdx.x == 0) gather.n = 0u;
  __syncthreads();
  if (sc.top[((size_t)w.r * w.NC + w.c) * kThreads + threadIdx.x] >= inside.lo)
    each(w.row, w.j0, w.j1, [&](int j, float l) {
      double t;
      if (inside(r, m, l, t)) gather_add(gather, sh.key, key_of(l, j));
    });
  gather_flush(gather, sh.key, work, list);
  if (!last_here(&work->done, w.NC)) return;

  const uint32_t n = get(&work->listed);
  const unsigned long long rest = needed(r.p, work->total) - work->before;
  unsigned long long mass, key;
  if (n <= (uint32_t)kThreads) {
    const int parts = parts_of(n), at = threadIdx.x / parts;
    unsigned long long k0 = 0, m0 = 0, before;
    if (at < (int)n) {
      k0 = get(&list[at]);
      m0 = mass_at(distance(r, m, logit_of((uint32_t)(k0 >> 32))));
    }
    sh.pair[threadIdx.x] = make_ulonglong2(0ull, 0ull);
    __syncthreads();
    if (threadIdx.x % parts == 0) sh.pair[at] = make_ulonglong2(k0, m0);
    __syncthreads();
    rank_pairs(sh.pair, n, parts, k0, before);
    if (before < rest && rest <= before + m0) {  // (one entry)
      sel.lo[0] = k0;
      sel.hi[0] = before + m0;
    }
    __syncthreads();
    key = sel.lo[0];
    mass = sel.hi[0];
  } else {
    const bool listed = n <= (uint32_t)kList;
    const bool paired = n <= (uint32_t)kPairs;
    if (listed)
      read_list(list, n, [&](uint32_t i, unsigned long long k) {
        if (paired) sh.pair[i] = make_ulonglong2(k, mass_at(distance(r, m, logit_of((uint32_t)(k >> 32)))));
        else sh.key[i] = k;
      });
    __syncthreads();
    auto src = [&](auto f) {
      if (paired) {
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
          const ulonglong2 p = sh.pair[i];
          f(p.x, p.y);
        }
      } else if (listed) {
        for (uint32_t i = threadIdx.x; i < n; i += kThreads)
          f(sh.key[i], mass_at(distance(r, m, logit_of((uint32_t)(sh.key[i] >> 32)))));
      } else {
        each(w.row, 0, a.V, [&](int j, float l) {
          double t;
          if (inside(r, m, l, t)) f(key_of(l, j), mass_at(t));
        });
      }
    };
    key = select_border(src, rest, true, sel);
    mass = mass_from(src, key, sel);
  }
  if (threadIdx.x == 0) {
    work->key = key;
    work->mass = work->before + mass;
  }
}

// ---------------------------------------------------------------- out
__global__ __launch_bounds__(kThreads) void rules_out_kernel(RulesArgs a) {
  __shared__ unsigned long long s_sum[kWaves];
  __shared__ int s_segment;
  __shared__ unsigned long long s_t;
  RuleScratch sc;
  carve_rules(a.scratch, (size_t)a.B * a.rows, a.V, &sc);
  const Where w = where(a);
  RowWork* work = sc.work + w.r;
  float* probs = a.probs ? a.probs + (size_t)w.r * a.ld_probs : nullptr;
  int32_t* out = a.out ? a.out + (size_t)w.r * a.ld_out : nullptr;
  const int kind = work->kind, amax = work->amax;
  if (work->drawn) return;
  if (kind == ROW_BAD || kind == ROW_GREEDY) {
    if (probs)
      for (int j = w.j0 + 4 * threadIdx.x; j < w.j1; j += 4 * kThreads) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = kind == ROW_BAD ? __uint_as_float(0x7fc00000u) : (j + e == amax ? 1.f : 0.f);
        store4(probs, j, w.j1, v);
      }
    if (out && w.c == 0 && threadIdx.x == 0) *out = kind == ROW_GREEDY ? amax : -1;
    return;
  }
  const Rules r = work->rules;
  const float m = work->m;
  const Kept prob(work->key, work->mass);
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int spc = (chunk_of(a.V, w.NC) + 255) / 256;  // segments of a chunk
  unsigned long long* parts = sc.draw + (size_t)w.r * segments_of(a.V);
  constexpr int Q = 2;
  // (a thread whose entries all lie below the border reads nothing)
  const bool any = sc.top[((size_t)w.r * w.NC + w.c) * kThreads + threadIdx.x] >= prob.edge;
  for (int base = w.j0; base < w.j1; base += 4 * Q * kThreads) {
    float v[Q][4];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = base + 4 * (q * kThreads + (int)threadIdx.x);
      load_quad(w.row, j, any ? w.j1 : j, 1, -INFINITY, v[q]);
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = base + 4 * (q * kThreads + (int)threadIdx.x);
      unsigned long long sum = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[q][e] = prob(r, m, j + e, v[q][e]);
        if (v[q][e] > 0.f) sum += fp_weight(v[q][e]);
      }
      if (probs && j < w.j1) store4(probs, j, w.j1, v[q]);
      const int seg = (base - w.j0) / 256 + q * kWaves + wv;
      if (out && seg < spc) {
        if (__any(sum != 0)) sum = wave_sum_u64(sum);
        if (lane == 0) put(&parts[w.c * spc + seg], sum);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (!out) return;
  // (a last chunk may be shorter, or empty: its segments weigh nothing)
  for (int seg = (w.j1 - w.j0 + 4 * Q * kThreads - 1) / (4 * Q * kThreads) * (Q * kWaves) + threadIdx.x; seg < spc; seg += kThreads)
    put(&parts[w.c * spc + seg], 0ull);
  if (!last_here(&work->done, w.NC)) return;
  // the segment that holds t, then the token in it
  const int n = w.NC * spc, per = (n + kThreads - 1) / kThreads;  // thread t holds `per` segments
  unsigned long long sum = 0, S;
  for (int i = 0; i < per; ++i) {
    const int at = threadIdx.x * per + i;
    sum += at < n ? get(&parts[at]) : 0ull;
  }
  unsigned long long cum = block_prefix(sum, S, s_sum);
  const unsigned long long t = scale_word(row_word(a, w), S);
  if (cum <= t && t < cum + sum) {  // (one thread: S > 0, the most likely token has prob >= 2^-20)
    for (int i = 0; i < per; ++i) {
      const int at = threadIdx.x * per + i;
      const unsigned long long one = at < n ? get(&parts[at]) : 0ull;
      if (t < cum + one) {
        s_segment = at;
        s_t = t - cum;
        break;
      }
      cum += one;
    }
  }
  __syncthreads();
  if (wv) return;
  const int c = s_segment / spc, end = min(a.V, (c + 1) * chunk_of(a.V, w.NC));
  const int j = c * chunk_of(a.V, w.NC) + (s_segment - c * spc) * 256 + 4 * lane;
  float v[4];
  unsigned long long q[4], four = 0;
  load_quad(w.row, j, end, 1, -INFINITY, v);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    q[e] = fp_weight(prob(r, m, j + e, v[e]));
    four += q[e];
  }
  cum = four;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const unsigned long long before = shfl_up_u64(cum, o);
    if (lane >= o) cum += before;
  }
  cum -= four;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (cum <= s_t && s_t < cum + q[e]) *out = j + e;
    cum += q[e];
  }
}

// Chunks of a row: enough workgroups for the card, at least 1024 entries each (a quad a thread).
int chunks_of(int rows, int V) { return std::max(1, std::min({kMaxChunks, (V + 1023) / 1024, (kGridTarget + rows - 1) / rows})); }

}  // namespace

size_t rules_scratch_bytes(int n_rows, int V) {
  RuleScratch s;
  return carve_rules(nullptr, (size_t)n_rows, V, &s);
}

hipError_t launch_rules(const RulesArgs& a, hipStream_t s) {
  const int n = a.B * a.rows;
  const dim3 grid(chunks_of(n, a.V), n), block(kThreads);
  hipLaunchKernelGGL(rules_max_kernel, grid, block, 0, s, a);
  hipLaunchKernelGGL(rules_scan_kernel, grid, block, 0, s, a);
  if (a.top_p) hipLaunchKernelGGL(rules_pick_kernel, grid, block, 0, s, a);
  hipLaunchKernelGGL(rules_out_kernel, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace specdec
