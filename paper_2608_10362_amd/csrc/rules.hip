// Sampling rules: a row of logits, a request's temperature, min-p, top-k and
// top-p, the distribution they leave and a token drawn from it.
//
// Definitions.  m = max l; e_j = exp((l_j - m) / T) in 64 bits; the integer
// mass of j is W_j = floor(e_j 2^43).  Candidates: l_j > -inf, e_j >= min_p.
// They are ordered by l (descending), the lower index first on ties; top_k
// keeps the first k; top_p keeps the shortest prefix of those whose mass is at
// least max(1, ceil(p * mass of the k)).  Every rule keeps a prefix of one
// order, so the result is one border: (bucket, key) below.  prob_j = fl32(e_j
// 2^43 / mass of the kept), the draw is the fixed-point one of the other
// samplers.  Masses are integers: no border depends on how the sums are split,
// and a 64-bit exponential costs nothing here that its reading does not.
//
// No sort: four launches, each over (chunk, row).
//   max      per chunk: maximum, its lowest index, NaN / +inf; clears the row's histogram
//   hist     candidates' counts and masses in buckets of (m - l) / T, monotone in
//            l: 1/64 wide to 16, then 8 to an octave; the last workgroup of the row
//            finds the buckets that hold the borders
//   pick     the border buckets' candidates go to a list (a few hundred of 128k
//            entries); the last workgroup selects the border keys in it
//   out      probabilities, and the draw (the last workgroup scans one chunk)
// A border bucket too full for the list (many equal logits) is selected by
// passes over the row itself, by one workgroup: slow, and right.
#include <algorithm>

#include "device_common.h"
#include "internal.h"
#include "sampling_common.h"

namespace specdec {

namespace {

constexpr int kThreads = 256;
constexpr int kWavesR = kThreads / kWave;
constexpr int kBuckets = 2048, kLinear = 1024;  // linear ones cover (m - l) / T < 16
constexpr int kList = 4096;                     // border candidates kept in LDS
constexpr int kMaxChunks = 64;                  // per row (one per lane)
constexpr double kTwo43 = 8796093022208.0;

enum { ROW_OK = 0, ROW_GREEDY = 1, ROW_BAD = 2 };

struct ChunkMax {
  float m;
  int i, bad, pad;
};
// One row's progress.  Words written by one launch and read by the next, except
// the counters (a launch's workgroups count themselves; the last resets them).
struct RowWork {
  uint32_t done;       // workgroups of the present launch that have finished
  uint32_t listed;     // candidates in the list
  int kind, amax;
  float m;
  int pick;            // 1: border buckets to select in
  int k_bucket;        // bucket of the top-k border, -1: whole buckets (or no such rule)
  uint32_t k_rest;     // candidates of it inside
  int p_lo, p_hi;      // buckets that may hold the top-p border, p_lo > p_hi: no such rule
  // result: kept are the candidates of buckets below `bucket` and those in it with key >= `key`
  int bucket, pad;
  unsigned long long key, mass, k_before;  // k_before: mass of the buckets above k_bucket
};

struct RuleScratch {
  ChunkMax* cmax;              // [rows][kMaxChunks]
  unsigned long long* draw;    // [rows][kMaxChunks]
  RowWork* work;               // [rows]
  unsigned long long* mass;    // [rows][kBuckets]
  uint32_t* count;             // [rows][kBuckets]
  unsigned long long* list;    // [rows][kList]
};
__host__ __device__ inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
__host__ __device__ inline size_t carve_rules(void* base, size_t rows, RuleScratch* s) {
  size_t off = 0;
  char* p = (char*)base;
  auto take = [&](size_t n) { const size_t at = off; off = up256(off + n); return p + at; };
  s->cmax = (ChunkMax*)take(rows * kMaxChunks * sizeof(ChunkMax));
  s->draw = (unsigned long long*)take(rows * kMaxChunks * 8);
  s->work = (RowWork*)take(rows * sizeof(RowWork));
  s->mass = (unsigned long long*)take(rows * kBuckets * 8);
  s->count = (uint32_t*)take(rows * kBuckets * 4);
  s->list = (unsigned long long*)take(rows * kList * 8);
  return off;
}

// ---------------------------------------------------------------- one row's rules
struct Rules {
  double T, mp;
  float p;
  int k;
  bool ok;
};
__device__ __forceinline__ Rules rules_of(const RulesArgs& a, int b) {
  const float T = a.temperature ? a.temperature[b] : 1.f, mp = a.min_p ? a.min_p[b] : 0.f;
  Rules r;
  r.p = a.top_p ? a.top_p[b] : 1.f;
  r.k = a.top_k ? a.top_k[b] : 0;
  r.T = T;
  r.mp = mp > 1.f ? 1.0 : (double)mp;  // (the most likely token always stays)
  r.ok = T >= 0.f && mp == mp && r.p == r.p;
  return r;
}
// Order of the candidates: a larger key comes first.
__device__ __forceinline__ unsigned long long key_of(float l, int j) {
  uint32_t u = __float_as_uint(l);
  u = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  if (u == 0x7fffffffu) u = 0x80000000u;  // (-0 and 0 are equal)
  return ((unsigned long long)u << 32) | (uint32_t)~(uint32_t)j;
}
__device__ __forceinline__ float logit_of(unsigned long long key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u);
}
__device__ __forceinline__ int bucket_of(double z) {
  if (z < 16.0) return (int)(z * 64.0);
  return kLinear + (int)((__float_as_uint((float)z) - 0x41800000u) >> 20);
}
// Whether l is a candidate; its distance z = (m - l) / T and e = exp(-z) (0 where
// neither the mass nor the min-p test can see the difference).
__device__ __forceinline__ bool candidate(const Rules& r, float m, float l, double& z, double& e) {
  if (!(l > -INFINITY)) return false;
  z = ((double)m - (double)l) / r.T;
  e = z < 30.0 || (r.mp > 0.0 && z < 746.0) ? exp(-z) : 0.0;  // (2^-43 = exp(-29.8))
  return e >= r.mp;
}
__device__ __forceinline__ unsigned long long mass_of(double e) { return (unsigned long long)(e * kTwo43); }

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
  const int cs = ((a.V + w.NC - 1) / w.NC + 3) / 4 * 4;
  w.j0 = min(a.V, w.c * cs);
  w.j1 = min(a.V, w.j0 + cs);
  w.row = a.logits + (size_t)w.r * a.ld;
  return w;
}
// f(j, l) for the entries [j0, j1) of a row: two quads a thread and round, loaded before the first is used.
template <typename F>
__device__ __forceinline__ void each(const float* row, int j0, int j1, F f) {
  constexpr int Q = 2;
  for (int base = j0 + 4 * threadIdx.x; base < j1; base += 4 * Q * kThreads) {
    float v[Q][4];
#pragma unroll
    for (int q = 0; q < Q; ++q) load_quad(row, base + 4 * q * kThreads, j1, 1, -INFINITY, v[q]);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = base + 4 * q * kThreads + e;
        if (j < j1) f(j, v[q][e]);
      }
  }
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

// Exclusive prefix of v over the workgroup (256 threads), and the total.
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
  for (int k = 0; k < kWavesR; ++k) {
    if (k < w) before += sh[k];
    total += sh[k];
  }
  return before + incl - v;
}

// ---------------------------------------------------------------- max
__global__ __launch_bounds__(kThreads) void rules_max_kernel(RulesArgs a) {
  __shared__ float sm[kWavesR];
  __shared__ int si[kWavesR], sb[kWavesR];
  RuleScratch sc;
  carve_rules(a.scratch, (size_t)a.B * a.rows, &sc);
  const Where w = where(a);
  for (int i = w.c * kThreads + threadIdx.x; i < kBuckets; i += w.NC * kThreads) {
    sc.mass[(size_t)w.r * kBuckets + i] = 0ull;
    sc.count[(size_t)w.r * kBuckets + i] = 0u;
  }
  float m = -INFINITY;
  int at = 0x7fffffff, bad = 0;
  each(w.row, w.j0, w.j1, [&](int j, float l) {
    bad |= !(l < INFINITY);  // (NaN or +inf)
    if (l > m) { m = l; at = j; }
  });
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
    for (int k = 1; k < kWavesR; ++k) {
      if (sm[k] > t.m || (sm[k] == t.m && si[k] < t.i)) { t.m = sm[k]; t.i = si[k]; }
      t.bad |= sb[k];
    }
    sc.cmax[(size_t)w.r * kMaxChunks + w.c] = t;
    if (w.c == 0) {
      sc.work[w.r].done = 0u;
      sc.work[w.r].listed = 0u;
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

// ---------------------------------------------------------------- hist
__global__ __launch_bounds__(kThreads) void rules_hist_kernel(RulesArgs a) {
  __shared__ unsigned long long s_mass[kBuckets];
  __shared__ uint32_t s_count[kBuckets];
  __shared__ unsigned long long s_sum[kWavesR];
  __shared__ unsigned long long s_kb;      // mass of the buckets before the top-k border's, of it included
  __shared__ unsigned long long s_ki;
  __shared__ int s_kbucket, s_plo, s_phi;
  __shared__ uint32_t s_krest, s_kwhole;
  RuleScratch sc;
  carve_rules(a.scratch, (size_t)a.B * a.rows, &sc);
  const Where w = where(a);
  const Rules r = rules_of(a, w.b);
  const ChunkMax mx = row_max(sc.cmax + (size_t)w.r * kMaxChunks, w.NC);
  RowWork* work = sc.work + w.r;
  const int kind = mx.bad || mx.m == -INFINITY || !r.ok ? ROW_BAD : (r.T == 0.0 ? ROW_GREEDY : ROW_OK);
  if (kind != ROW_OK) {  // (workgroup-uniform)
    if (w.c == 0 && threadIdx.x == 0) {
      work->kind = kind;
      work->amax = mx.i;
      work->pick = 0;
      if (kind == ROW_BAD) set_status(a.status, kStatusNonFinite);
    }
    return;
  }
  for (int i = threadIdx.x; i < kBuckets; i += kThreads) {
    s_mass[i] = 0ull;
    s_count[i] = 0u;
  }
  __syncthreads();
  each(w.row, w.j0, w.j1, [&](int, float l) {
    double z, e;
    if (!candidate(r, mx.m, l, z, e)) return;
    const int i = bucket_of(z);
    atomicAdd(&s_count[i], 1u);
    const unsigned long long W = mass_of(e);
    if (W) atomicAdd(&s_mass[i], W);
  });
  __syncthreads();
  unsigned long long* mass = sc.mass + (size_t)w.r * kBuckets;
  uint32_t* count = sc.count + (size_t)w.r * kBuckets;
  for (int i = threadIdx.x; i < kBuckets; i += kThreads) {
    if (s_count[i]) __hip_atomic_fetch_add(&count[i], s_count[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (s_mass[i]) __hip_atomic_fetch_add(&mass[i], s_mass[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (!last_here(&work->done, w.NC)) return;

  // The borders' buckets.  Thread t holds buckets 8t .. 8t+7.
  constexpr int PT = kBuckets / kThreads;
  unsigned long long tm[PT], msum = 0, csum = 0, mtotal, ctotal;
  uint32_t tc[PT];
#pragma unroll
  for (int i = 0; i < PT; ++i) {
    tm[i] = get(&mass[threadIdx.x * PT + i]);
    tc[i] = get(&count[threadIdx.x * PT + i]);
  }
#pragma unroll
  for (int i = 0; i < PT; ++i) {
    msum += tm[i];
    csum += tc[i];
  }
  const unsigned long long mbefore = block_prefix(msum, mtotal, s_sum);
  const unsigned long long cbefore = block_prefix(csum, ctotal, s_sum);
  const bool by_k = r.k > 0 && (unsigned long long)r.k < ctotal;
  if (threadIdx.x == 0) {
    s_kbucket = -1;
    s_kb = s_ki = mtotal;
    s_krest = 0u;
    s_kwhole = 1u;
    s_plo = 1;
    s_phi = 0;
  }
  __syncthreads();
  if (by_k) {
    unsigned long long cc = cbefore, mm = mbefore;
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      if (cc < (unsigned long long)r.k && (unsigned long long)r.k <= cc + tc[i]) {  // (one bucket of one thread)
        s_kbucket = threadIdx.x * PT + i;
        s_krest = (uint32_t)(r.k - cc);
        s_kwhole = (unsigned long long)r.k == cc + tc[i];
        s_kb = mm;
        s_ki = mm + tm[i];
      }
      cc += tc[i];
      mm += tm[i];
    }
    __syncthreads();
  }
  const bool by_p = r.p < 1.f;
  if (by_p) {
    // The mass of the top k lies in (s_kb, s_ki] (exactly s_ki for whole buckets): so do the border's.
    const unsigned long long lo = s_kwhole ? s_ki : s_kb, hi = s_ki;
    const unsigned long long nlo = max(1ull, (unsigned long long)ceil(max(0.0, (double)r.p) * (double)lo));
    const unsigned long long nhi = max(1ull, (unsigned long long)ceil(max(0.0, (double)r.p) * (double)hi));
    unsigned long long mm = mbefore;
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      if (mm < nlo && nlo <= mm + tm[i]) s_plo = threadIdx.x * PT + i;
      if (mm < nhi && nhi <= mm + tm[i]) s_phi = threadIdx.x * PT + i;
      mm += tm[i];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    work->kind = ROW_OK;
    work->amax = mx.i;
    work->m = mx.m;
    const bool split = by_k && !s_kwhole;
    work->pick = split || by_p;
    work->k_bucket = split ? s_kbucket : -1;
    work->k_rest = s_krest;
    work->k_before = split ? s_kb : s_ki;
    work->p_lo = s_plo;
    work->p_hi = s_phi;
    work->bucket = by_k ? s_kbucket : kBuckets;
    work->key = 0ull;
    work->mass = s_ki;
  }
}

// ---------------------------------------------------------------- pick
struct Select {
  unsigned long long hist_m[256];
  uint32_t hist_c[256];
  unsigned long long sum[kWavesR];
  unsigned long long lo[kWavesR], hi[kWavesR];
  int digit;
  unsigned long long before_m, before_c;
};

// The border in bucket `want`: the key of the last candidate kept, when the
// first `rest` (by_mass: the fewest whose mass reaches `rest`) are; `mass`
// receives theirs.  src(f): f(key, bucket, W) for every listed candidate.
// Radix selection from the highest bit in which the keys differ, 8 bits a
// pass; keys are distinct, so the last pass leaves one.
template <typename SRC>
__device__ unsigned long long select_border(SRC src, int want, unsigned long long rest, bool by_mass,
                                            unsigned long long& mass, Select& sh) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  unsigned long long lo = ~0ull, hi = 0ull;
  src([&](unsigned long long key, int bucket, double) {
    if (bucket != want) return;
    lo = min(lo, key);
    hi = max(hi, key);
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, (unsigned long long)__shfl_xor(lo, o, kWave));
    hi = max(hi, (unsigned long long)__shfl_xor(hi, o, kWave));
  }
  __syncthreads();
  if (lane == 0) {
    sh.lo[w] = lo;
    sh.hi[w] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWavesR; ++k) {
    lo = min(lo, sh.lo[k]);
    hi = max(hi, sh.hi[k]);
  }
  int top = lo == hi ? 0 : 64 - __clzll((long long)(lo ^ hi));  // differing bits: [0, top)
  unsigned long long prefix = top >= 64 ? 0ull : hi >> top << top;
  unsigned long long inside = 0;  // mass of the candidates before the prefix's
  while (top > 0) {
    const int shift = top > 8 ? top - 8 : 0, bits = top - shift;
    __syncthreads();
    sh.hist_m[threadIdx.x] = 0ull;
    sh.hist_c[threadIdx.x] = 0u;
    __syncthreads();
    src([&](unsigned long long key, int bucket, double e) {
      if (bucket != want || (top < 64 && (key >> top) != (prefix >> top))) return;
      const int d = (int)((key >> shift) & ((1u << bits) - 1u));
      atomicAdd(&sh.hist_c[d], 1u);
      atomicAdd(&sh.hist_m[d], mass_of(e));
    });
    __syncthreads();
    // larger keys first: thread t looks at digit 255 - t
    const int d = 255 - (int)threadIdx.x;
    const unsigned long long m = sh.hist_m[d], c = sh.hist_c[d];
    unsigned long long mt, ct;
    const unsigned long long mb = block_prefix(m, mt, sh.sum), cb = block_prefix(c, ct, sh.sum);
    const unsigned long long before = by_mass ? mb : cb, here = by_mass ? m : c;
    if (before < rest && rest <= before + here) {
      sh.digit = d;
      sh.before_m = mb;
      sh.before_c = before;
    }
    __syncthreads();
    inside += sh.before_m;
    rest -= sh.before_c;
    prefix |= (unsigned long long)sh.digit << shift;
    top = shift;
  }
  // (one candidate has this key: its mass)
  __syncthreads();
  if (threadIdx.x == 0) sh.before_m = 0;
  __syncthreads();
  src([&](unsigned long long key, int bucket, double e) {
    if (bucket == want && key == prefix) sh.before_m = mass_of(e);
  });
  __syncthreads();
  mass = inside + sh.before_m;
  return prefix;
}

__global__ __launch_bounds__(kThreads) void rules_pick_kernel(RulesArgs a) {
  __shared__ unsigned long long s_key[kList];
  __shared__ Select sh;
  RuleScratch sc;
  carve_rules(a.scratch, (size_t)a.B * a.rows, &sc);
  const Where w = where(a);
  RowWork* work = sc.work + w.r;
  if (work->kind != ROW_OK || !work->pick) return;  // (workgroup-uniform, as all that follows from the row's words)
  const Rules r = rules_of(a, w.b);
  const float m = work->m;
  const int kb = work->k_bucket, plo = work->p_lo, phi = work->p_hi;
  auto border = [&](int i) { return i == kb || (i >= plo && i <= phi); };
  unsigned long long* list = sc.list + (size_t)w.r * kList;
  each(w.row, w.j0, w.j1, [&](int j, float l) {
    double z, e;
    if (!candidate(r, m, l, z, e) || !border(bucket_of(z))) return;
    const uint32_t at = __hip_atomic_fetch_add(&work->listed, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (at < (uint32_t)kList) put(&list[at], key_of(l, j));
  });
  if (!last_here(&work->done, w.NC)) return;

  const uint32_t n = get(&work->listed);
  const bool listed = n <= (uint32_t)kList;
  if (listed)
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) s_key[i] = get(&list[i]);
  __syncthreads();
  auto src = [&](auto f) {
    if (listed) {
      for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
        double z, e;
        const unsigned long long key = s_key[i];
        candidate(r, m, logit_of(key), z, e);
        f(key, bucket_of(z), e);
      }
    } else {
      each(w.row, 0, a.V, [&](int j, float l) {
        double z, e;
        if (!candidate(r, m, l, z, e)) return;
        const int i = bucket_of(z);
        if (border(i)) f(key_of(l, j), i, e);
      });
    }
  };
  int bucket = work->bucket;
  unsigned long long key = 0ull, mass = work->mass;
  if (kb >= 0) {
    unsigned long long part;
    key = select_border(src, kb, work->k_rest, false, part, sh);
    mass = work->k_before + part;
  }
  if (plo <= phi) {
    const unsigned long long need = max(1ull, (unsigned long long)ceil(max(0.0, (double)r.p) * (double)mass));
    // the bucket of [plo, phi] in which the running mass reaches `need`
    const unsigned long long* hm = sc.mass + (size_t)w.r * kBuckets;
    constexpr int PT = kBuckets / kThreads;
    unsigned long long tm[PT], sum = 0, total;
#pragma unroll
    for (int i = 0; i < PT; ++i) sum += tm[i] = hm[threadIdx.x * PT + i];
    unsigned long long mm = block_prefix(sum, total, sh.sum);
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      if (mm < need && need <= mm + tm[i]) {
        sh.digit = threadIdx.x * PT + i;
        sh.before_m = mm;
      }
      mm += tm[i];
    }
    __syncthreads();
    const int pb = sh.digit;
    const unsigned long long before = sh.before_m;
    unsigned long long part;
    key = select_border(src, pb, need - before, true, part, sh);
    mass = before + part;
    bucket = pb;
  }
  if (threadIdx.x == 0) {
    work->bucket = bucket;
    work->key = key;
    work->mass = mass;
  }
}

// ---------------------------------------------------------------- out
__global__ __launch_bounds__(kThreads) void rules_out_kernel(RulesArgs a) {
  __shared__ unsigned long long s_sum[kWavesR];
  __shared__ int s_chunk;
  __shared__ unsigned long long s_t;
  RuleScratch sc;
  carve_rules(a.scratch, (size_t)a.B * a.rows, &sc);
  const Where w = where(a);
  RowWork* work = sc.work + w.r;
  float* probs = a.probs ? a.probs + (size_t)w.r * a.ld_probs : nullptr;
  int32_t* out = a.out ? a.out + (size_t)w.r * a.ld_out : nullptr;
  const int kind = work->kind, amax = work->amax;
  auto store4 = [&](int j, const float (&v)[4]) {
    if (j + 4 <= w.j1) *(f32x4_a4*)(probs + j) = f32x4{v[0], v[1], v[2], v[3]};
    else
      for (int e = 0; j + e < w.j1; ++e) probs[j + e] = v[e];
  };
  if (kind != ROW_OK) {
    if (probs)
      for (int j = w.j0 + 4 * threadIdx.x; j < w.j1; j += 4 * kThreads) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = kind == ROW_BAD ? __uint_as_float(0x7fc00000u) : (j + e == amax ? 1.f : 0.f);
        store4(j, v);
      }
    if (out && w.c == 0 && threadIdx.x == 0) *out = kind == ROW_GREEDY ? amax : -1;
    return;
  }
  const Rules r = rules_of(a, w.b);
  const float m = work->m;
  const int bucket = work->bucket;
  const unsigned long long key = work->key;
  const double inv = kTwo43, total = (double)work->mass;
  auto prob = [&](int j, float l) {
    if (key && key_of(l, j) < key) return 0.f;  // (a known border key settles it without an exponential)
    double z, e;
    if (!candidate(r, m, l, z, e)) return 0.f;
    if (!key && bucket < kBuckets && bucket_of(z) > bucket) return 0.f;
    if (e == 0.0) e = z < 110.0 ? exp(-z) : 0.0;  // (past it a float32 probability is 0)
    return (float)(e * inv / total);
  };
  unsigned long long sum = 0;
  constexpr int Q = 2;
  for (int base = w.j0 + 4 * threadIdx.x; base < w.j1; base += 4 * Q * kThreads) {
    float v[Q][4];
#pragma unroll
    for (int q = 0; q < Q; ++q) load_quad(w.row, base + 4 * q * kThreads, w.j1, 1, -INFINITY, v[q]);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = base + 4 * q * kThreads;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[q][e] = j + e < w.j1 ? prob(j + e, v[q][e]) : 0.f;
        sum += fp_weight(v[q][e]);
      }
      if (probs && j < w.j1) store4(j, v[q]);
    }
  }
  if (!out) return;
  unsigned long long mine;
  block_prefix(sum, mine, s_sum);
  unsigned long long* parts = sc.draw + (size_t)w.r * kMaxChunks;
  if (threadIdx.x == 0) put(&parts[w.c], mine);
  if (!last_here(&work->done, w.NC)) return;
  // the chunk that holds t (lane k: chunk k), then the token in it
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  if (wv == 0) {
    const unsigned long long pk = lane < w.NC ? get(&parts[lane]) : 0ull;
    const unsigned long long S = wave_sum_u64(pk);
    uint32_t x;
    if (a.rand) x = a.rand[w.r];
    else x = draw_word(a.seed, w.b, a.step_dev ? *a.step_dev : a.step, a.purpose, a.index + w.r % a.rows);
    const unsigned long long t = scale_word(x, S);
    unsigned long long incl = pk;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const unsigned long long n = shfl_up_u64(incl, o);
      if (lane >= o) incl += n;
    }
    if (t < incl && t >= incl - pk) {  // (one lane: S > 0, the most likely token has prob >= 2^-20)
      s_chunk = lane;
      s_t = t - (incl - pk);
    }
  }
  __syncthreads();
  const int cs = ((a.V + w.NC - 1) / w.NC + 3) / 4 * 4;
  const int j0 = min(a.V, s_chunk * cs), j1 = min(a.V, j0 + cs);
  unsigned long long t = s_t;
  for (int base = j0; base < j1; base += 4 * kThreads) {
    const int jj = base + 4 * threadIdx.x;
    float v[4];
    unsigned long long q[4], four = 0, round;
    load_quad(w.row, jj, j1, 1, -INFINITY, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      q[e] = fp_weight(jj + e < j1 ? prob(jj + e, v[e]) : 0.f);
      four += q[e];
    }
    unsigned long long cum = block_prefix(four, round, s_sum);
    if (cum <= t && t < cum + four) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        cum += q[e];
        if (cum > t) {
          *out = jj + e;
          break;
        }
      }
    }
    if (t < round) break;  // (uniform)
    t -= round;
  }
}

// Chunks of a row: enough workgroups for the card, at least 512 entries each
// (every one adds its histogram to the row's).
int chunks_of(int rows, int V) { return std::max(1, std::min({kMaxChunks, (V + 511) / 512, (2048 + rows - 1) / rows})); }

}  // namespace

size_t rules_scratch_bytes(int n_rows, int V) {
  (void)V;
  RuleScratch s;
  return carve_rules(nullptr, (size_t)n_rows, &s);
}

hipError_t launch_rules(const RulesArgs& a, hipStream_t s) {
  const int n = a.B * a.rows;
  const dim3 grid(chunks_of(n, a.V), n), block(kThreads);
  hipLaunchKernelGGL(rules_max_kernel, grid, block, 0, s, a);
  hipLaunchKernelGGL(rules_hist_kernel, grid, block, 0, s, a);
  if (a.top_k || a.top_p) hipLaunchKernelGGL(rules_pick_kernel, grid, block, 0, s, a);
  hipLaunchKernelGGL(rules_out_kernel, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace specdec
