// Norm and position rotation of queries and keys, head by head, in one pass; for an FP8
// cache the rotated keys and the values go to its ring in that pass too.
//
//   y = gain x / sqrt(mean(x^2) + eps)            (per row and head; optional)
//   (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position freq_j
//
// for the pairs j < rotary / 2 of a head: dims (j, j + rotary / 2) or (2j, 2j + 1).
//
// Every element is read once and written once: the bytes are the bound.  A lane holds 8
// dims of a row's head, 16 bytes of bf16; the half that a pair's other dim lies in comes
// from the lane rotary / 16 further.  The angles depend on the row alone: a workgroup takes
// 8 rows and some heads, computes the rows' cosines and sines once (the angle in turns in
// 64 bits, where a far position keeps its fraction, the functions in 32) and keeps them in
// LDS.  Squares are summed in 64 bits and the factor 1 / sqrt is applied there, before gain and rotation: no
// float32 input overflows or vanishes on the way, and a head's bits depend on the head alone.  (Sums in 32 bits, with
// these beside them for heads that they do not hold, took 1.1 us less of 8189 rows' 60, 1.4 less of 2048 rows' 33 into
// the cache.)
//
// The 8 rows are 8 positions of one sequence from a multiple of 8 on: a lane then holds a
// whole piece of V's operand order (8 positions of a dim, 16 bytes), turned in registers,
// and K's pieces of neighbouring positions leave from one CU.
//
// Measured.  7B-like (32 + 32 heads of 128), bf16: 8189 rows 60 us, 4.5 TB/s (a copy of as many bytes: 50), float32 111,
// 4.8 TB/s; one row 4.1 us (10 with the host's call).  Into the cache, 2048 rows 33 us, 100 MB: K and V leave in pieces
// of 16 bytes, 64 and 256 bytes of them side by side (5 us more with the lanes' own order); float32 40.  1.1B-like, 96
// rows 5 us.
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "fp8.h"
#include "internal.h"

namespace specdec {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 8;

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4 a = *(const f32x4_a4*)p, b = *(const f32x4_a4*)(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = a[e];
    x[4 + e] = b[e];
  }
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
  const u32x4 a = *(const u32x4_a2*)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(a[e] << 16);
    x[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
  }
}
// (nearest even, by the conversion instruction)
__device__ __forceinline__ u32x4 to_bf16x8(const float (&x)[8]) {
  u32x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    o[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * e], x[2 * e + 1]}, bf16x2));
  return o;
}
// (`stream`: past the caches)
__device__ __forceinline__ void store8(float* p, const float (&x)[8], bool stream) {
  const f32x4 lo = {x[0], x[1], x[2], x[3]}, up = {x[4], x[5], x[6], x[7]};
  if (stream) {
    __builtin_nontemporal_store(lo, (f32x4_a4*)p);
    __builtin_nontemporal_store(up, (f32x4_a4*)(p + 4));
  } else {
    *(f32x4_a4*)p = lo;
    *(f32x4_a4*)(p + 4) = up;
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8], bool stream) {
  if (stream) __builtin_nontemporal_store(to_bf16x8(x), (u32x4_a2*)p);
  else *(u32x4_a2*)p = to_bf16x8(x);
}

// 8 dims of a value row as bf16.
__device__ __forceinline__ u32x4 bf16_row(const float* p) {
  float x[8];
  load8(p, x);
  return to_bf16x8(x);
}
__device__ __forceinline__ u32x4 bf16_row(const uint16_t* p) { return *(const u32x4_a2*)p; }

// 1 / sqrt(m) in 64 bits: the instruction's 2^-23 squared by one step.
__device__ __forceinline__ double inv_sqrt(double m) {
  const double y = __builtin_amdgcn_rsq(m);
  return isinf(m) ? 0.0 : y * (1.5 - 0.5 * m * y * y);
}

// Between LDS stores of a wave's lanes and loads of them by others: a wave's LDS operations take place
// in the order they are issued in, and this keeps the compiler from another.
__device__ __forceinline__ void lanes_meet() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// x of the lane `far` further (the low half of a pair of halves) or nearer: inside a row of 16 lanes
// without LDS where far is a power of two.
template <int CTRL, int BANKS = 15>
__device__ __forceinline__ float dpp(float x, float old) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(old), __float_as_uint(x), CTRL, 0xf, BANKS, false));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double x) {
  const u32x2 w = __builtin_bit_cast(u32x2, x);
  return __builtin_bit_cast(double, u32x2{(uint32_t)__builtin_amdgcn_update_dpp(w[0], w[0], CTRL, 0xf, 0xf, false),
                                          (uint32_t)__builtin_amdgcn_update_dpp(w[1], w[1], CTRL, 0xf, 0xf, false)});
}
// Sum over the LPH lanes of a head (4, 8 or 16 of a row of 16).
template <int LPH>
__device__ __forceinline__ double head_sum(double v) {
  constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140;
  v += dpp<kXor1>(v);
  v += dpp<kXor2>(v);
  if (LPH >= 8) v += dpp<kHalfMirror>(v);
  if (LPH >= 16) v += dpp<kMirror>(v);
  return v;
}
__device__ __forceinline__ void exchange(const float (&x)[8], int far, int from, float (&y)[8]) {
  constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kShl4 = 0x104, kShr4 = 0x114, kRor8 = 0x128;
  if (far == 8) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = dpp<kRor8>(x[e], x[e]);
  } else if (far == 4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = dpp<kShr4, 10>(x[e], dpp<kShl4, 5>(x[e], x[e]));
  } else if (far == 2) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = dpp<kXor2>(x[e], x[e]);
  } else if (far == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = dpp<kXor1>(x[e], x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = __shfl(x[e], from, kWave);
  }
}

// Workgroup: kRopeRows rows (CACHE: positions of a sequence from a multiple of 8 on, those of
// the call's), and `per` of the units of HPW heads: queries, then keys, then values.
template <int HD, typename TI, typename TO, bool CACHE>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
  constexpr int LPH = HD / 8, HPW = kWave / LPH, NW = kRopeThreads / kWave;
  __shared__ alignas(16) float cs[2][kRopeRows][HD / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int chunk = blockIdx.x % a.chunks, grp = blockIdx.x / a.chunks;
  int r0, T, first = 0, at0 = 0, b = 0;  // first row; rows; the first row's place among the 8, its position
  bool stored = true;
  if constexpr (CACHE) {
    b = grp / a.groups;
    const int len = a.f8.len[b];
    const int lo = max(len, (len >> 3) * 8 + (grp - b * a.groups) * 8), hi = min((lo & ~7) + 8, len + a.n);
    T = hi - lo;
    if (T <= 0) return;  // (workgroup-uniform)
    r0 = b * a.n + lo - len;
    first = lo & 7;
    at0 = lo;
    stored = lo >= 0 && hi <= a.pos_limit;
    if (!stored && threadIdx.x == 0) set_status(a.status, kStatusKvCapacity);  // (the host's bound was wrong)
  } else {
    r0 = grp * kRopeRows;
    T = min(kRopeRows, a.rows - r0);
  }
  const int rot = a.rotary, half = rot >> 1;
  for (int e = threadIdx.x; e < T * half; e += kRopeThreads) {
    const int t = e / half, j = e - t * half;
    const int64_t base = a.positions ? a.positions[r0 + t] : CACHE ? at0 + t : (r0 + t) % a.n;
    const double turns = (double)(base + a.offset) * a.turns[j];
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    cs[0][t][j] = c;
    cs[1][t][j] = s;
  }
  const int H = a.n_heads, G = a.n_kv_heads, n_q = (H + HPW - 1) / HPW, n_k = (G + HPW - 1) / HPW, n_qk = n_q + n_k;
  const int n_v = CACHE ? n_k : 0;
  const int u0 = chunk * a.per, u1 = min(u0 + a.per, n_qk + n_v);
  const int hl = lane / LPH, l = lane % LPH, d0 = 8 * l;
  const int window = CACHE ? a.f8.ring.capacity : 0;
  __syncthreads();

  // Waves over rows first (their angles stay in registers), over units where there are fewer rows.
  const int across = T >= 4 ? 4 : T >= 2 ? 2 : 1;
  const int far = rot / 16;  // lanes of a half
  const bool low = l < far, in = a.interleaved ? d0 < rot : l < 2 * far;
  const int from = lane + (in ? (low ? far : -far) : 0);
  const int j0 = !in ? 0 : a.interleaved ? d0 / 2 : (low ? l : l - far) * 8;
  // Units [from, to) of the queries (or keys): heads of n, norm by `gain` or not.
  auto turn = [&](auto queries, int from_unit, int to_unit, int n, const void* gain, const void* in_rows, int64_t ld) {
    if (from_unit >= to_unit) return;
    float g[8], pg[8];  // this lane's gains, its partner's
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = 1.f;
    if (gain) {
      if (a.gain_bf16) load8((const uint16_t*)gain + d0, g);
      else load8((const float*)gain + d0, g);
    }
    if (!a.interleaved) exchange(g, far, from, pg);
    // out = x c + y s of the normalised x, y: the gains are in c and s (interleaved: c, s of 4 pairs, the gains apart)
    float c[8], s[8];
    auto angles = [&](int t) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        c[e] = 1.f;
        s[e] = 0.f;
      }
      if (in) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (k == 1 && a.interleaved) break;
          const f32x4 cv = *(const f32x4*)&cs[0][t][j0 + 4 * k], sv = *(const f32x4*)&cs[1][t][j0 + 4 * k];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            c[4 * k + e] = cv[e];
            s[4 * k + e] = low && !a.interleaved ? -sv[e] : sv[e];
          }
        }
      }
      if (!a.interleaved)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          c[e] *= g[e];
          s[e] *= pg[e];
        }
    };
    auto head_of = [&](int t, int head) {
      const bool valid = head < n;
      const int row = r0 + t;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.f;
      if (valid) load8((const TI*)in_rows + (int64_t)row * ld + (int64_t)head * HD + d0, x);
      if (gain) {
        double m = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = __builtin_fma((double)x[e], (double)x[e], m);
        const double rs = inv_sqrt(head_sum<LPH>(m) * (1.0 / HD) + (double)a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)((double)x[e] * rs);
      }
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= g[e];
        if (in)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = x[2 * e], r = x[2 * e + 1];
            x[2 * e] = p * c[e] - r * s[e];
            x[2 * e + 1] = r * c[e] + p * s[e];
          }
      } else {
        float y[8];
        exchange(x, far, from, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = x[e] * c[e];
          x[e] = in ? __builtin_fmaf(y[e], s[e], z) : z;
        }
      }
      if (!valid) return;
      if constexpr (queries) {
        store8((TO*)a.q_out + (int64_t)row * a.ld_qo + (int64_t)head * HD + d0, x, a.stream);
      } else if constexpr (CACHE) {
        if (stored) {
          uint16_t* blk = k_block<uint16_t>(a.f8.ring, a.layer, b, head);
          *(u32x4*)(blk + KvIndex<uint16_t>::k((at0 + t) % window, d0, HD, window)) = to_bf16x8(x);
        }
      } else {
        store8((TO*)a.k_out + (int64_t)row * a.ld_ko + (int64_t)head * HD + d0, x, a.stream);
      }
    };
    if (CACHE && !queries && T == kRopeRows) {
      // (positions of one head side by side: K's order has 16 bytes of each in a row)
      const int m0 = from_unit * HPW * kRopeRows + hl, m1 = min(to_unit * HPW, n) * kRopeRows;
      for (int m = m0 + wave * HPW; m - hl < m1; m += NW * HPW) {
        angles(m % kRopeRows);
        head_of(m % kRopeRows, m / kRopeRows);
      }
      return;
    }
    for (int t = wave % across; t < T; t += across) {
      angles(t);
#pragma unroll 4
      for (int u = from_unit + wave / across; u < to_unit; u += NW / across) head_of(t, u * HPW + hl);
    }
  };
  turn(std::true_type{}, u0, min(u1, n_q), H, a.q_gain, a.q, a.ld_q);
  turn(std::false_type{}, max(u0 - n_q, 0), min(u1, n_qk) - n_q, G, a.k_gain, a.k, a.ld_k);

  if constexpr (CACHE) {
    if (!stored) return;
    __shared__ u32x4 turned[NW][8 * kWave];
    const int p0 = (at0 & ~7) % window;
    for (int u = max(u0, n_qk) + wave; u < u1; u += NW) {
      const int g0 = (u - n_qk) * HPW, g = g0 + hl;
      const TI* src = (const TI*)a.v + (int64_t)r0 * a.ld_v + (int64_t)g * HD + d0;
      if (T == kRopeRows) {
        if (g < G) {
          u32x4 x[kRopeRows];
#pragma unroll
          for (int t = 0; t < kRopeRows; ++t) x[t] = bf16_row(src + (int64_t)t * a.ld_v);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            u32x4 y;
#pragma unroll
            for (int w = 0; w < 4; ++w)  // (the e-th 16 bits of two rows)
              y[w] = __builtin_amdgcn_perm(x[2 * w + 1][e >> 1], x[2 * w][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
            turned[wave][8 * lane + (e ^ (lane & 7))] = y;
          }
        }
        lanes_meet();
        // (out through LDS, so that lanes store the dims' pieces side by side: 16 of them are 256 bytes)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int at = k * kWave + lane, head = g0 + at / HD;
          if (head < G)
            *(u32x4*)(k_block<uint16_t>(a.f8.ring, a.layer, b, head) + KvIndex<uint16_t>::v(p0, at % HD, HD, window)) =
                turned[wave][(at & ~7) + ((at & 7) ^ (at >> 3 & 7))];
        }
        lanes_meet();  // (before the next unit's)
      } else if (g < G) {
        uint16_t* dst = k_block<uint16_t>(a.f8.ring, a.layer, b, g) + KvIndex<uint16_t>::v(p0, d0, HD, window);
        for (int t = 0; t < T; ++t) {
          const u32x4 x = bf16_row(src + (int64_t)t * a.ld_v);
#pragma unroll
          for (int e = 0; e < 8; ++e) dst[8 * e + first + t] = (uint16_t)(x[e >> 1] >> (16 * (e & 1)));
        }
      }
    }
  }
}

template <int HD>
hipError_t launch_hd(const RopeArgs& a, bool in_f32, bool out_f32, bool cache, dim3 grid, hipStream_t s) {
#define SD_ROPE(TI, TO)                                                                                     \
  if (cache) hipLaunchKernelGGL((rope_kernel<HD, TI, TO, true>), grid, dim3(kRopeThreads), 0, s, a);        \
  else hipLaunchKernelGGL((rope_kernel<HD, TI, TO, false>), grid, dim3(kRopeThreads), 0, s, a);
  if (in_f32) {
    if (out_f32) { SD_ROPE(float, float) }
    else { SD_ROPE(float, uint16_t) }
  } else {
    if (out_f32) { SD_ROPE(uint16_t, float) }
    else { SD_ROPE(uint16_t, uint16_t) }
  }
#undef SD_ROPE
  return hipGetLastError();
}

// Groups of rows of a launch.
int64_t groups_of(int batch, int n, bool cache) {
  return cache ? (int64_t)batch * ((n + kRopeRows - 2) / kRopeRows + 1)
               : ((int64_t)batch * n + kRopeRows - 1) / kRopeRows;
}

}  // namespace

// (a grid of at most 2^24 workgroups of 256 threads, one at least for a group of rows)
bool rope_fits(int batch, int n, bool cache) {
  return (int64_t)batch * n <= 0x7fffffff && groups_of(batch, n, cache) < 1 << 22;
}

hipError_t launch_rope(RopeArgs a, int head_dim, int batch, bool in_f32, bool out_f32, bool cache, hipStream_t s) {
  const int hpw = 512 / head_dim;
  const int units = (a.n_heads + hpw - 1) / hpw + (cache ? 2 : 1) * ((a.n_kv_heads + hpw - 1) / hpw);
  const int64_t groups = groups_of(batch, a.n, cache);
  a.rows = batch * a.n;
  a.groups = (int)(groups / batch);
  // Results far larger than the caches go past them (134 MB: 60 -> 58 us).
  a.stream = (int64_t)a.rows * (a.n_heads + a.n_kv_heads) * head_dim * (out_f32 ? 4 : 2) > 64 << 20;
  // Heads are split over workgroups until the card is full twice, each wave with a row's unit at least.  (8189
  // rows of 64 heads: 66 us with half as many workgroups, 65 with twice as many.)
  const int64_t slots = 16L * device_compute_units();
  const int rows = std::min(a.n * (cache ? 1 : batch), kRopeRows);
  const int64_t least = (kRopeThreads / kWave + rows - 1) / rows;
  a.per = (int)std::min<int64_t>(units, std::max<int64_t>({least, (units * groups + slots - 1) / slots, (int64_t)1}));
  a.chunks = (units + a.per - 1) / a.per;
  if (groups * a.chunks >= 1 << 24) {  // (few heads a workgroup: as many as the grid takes)
    a.per = units;
    a.chunks = 1;
  }
  const dim3 grid((unsigned)(groups * a.chunks));
  switch (head_dim) {
    case 32: return launch_hd<32>(a, in_f32, out_f32, cache, grid, s);
    case 64: return launch_hd<64>(a, in_f32, out_f32, cache, grid, s);
    case 128: return launch_hd<128>(a, in_f32, out_f32, cache, grid, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace specdec
