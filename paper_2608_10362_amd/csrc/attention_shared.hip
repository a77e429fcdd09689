// Attention of a batch whose sequences begin with the same text, held once as a sequence of an FP8
// cache of its own.
//
// The softmax over a row's keys is taken in two sets, the prefix's and the row's own:
// with (M, L, O) the maximum, the sum of exp(s - M) and the sum of those times the
// values of each set, the result is sum_i e^(M_i - M) O_i / sum_i e^(M_i - M) L_i.
// First launch: all rows of the batch against the prefix as if they were one sequence's,
// split over its keys, (M, L, O) of every part to the workspace; second launch: every
// sequence's rows over its own cache, which joins the parts to its own.
// The prefix's codes are read once for 16 to 64 rows of a kv head, not once a sequence.
//
//  prefix: float32 queries, or bf16 ones of at most 16 rows a kv head: attn8_kernel; bf16: wide_kernel;
//  own texts: at most 64 rows, not long: own_kernel; more than 16 bf16 rows that fill the card or are short: wide_kernel
//  (see wide_takes); else attn8_kernel.
//
// Measured (both launches).  7B-like (32 kv heads of 128): 16 bf16 rows over 8192 shared and 64 to 700 own keys
// 32 us (two streams, 17 and 16 us, 3.9 and 3.4 TB/s), 128 rows over 16384 and up to 256 own 91 us (the prefix 50 us,
// 690 TFLOP/s, own texts 45), 6 x 170 rows over 3500 92 us (650 TFLOP/s; the prefix 80 to 82, 710), 16 x 5 float32 rows
// over 4001 and up to 512 36 us (25 and 14), 6 x 170 over 3500 183.  1.1B-like (4 kv heads of 64, 8 query heads each): 64
// bf16 rows over 65553 and 30 to 300 own keys 48 us (710 TFLOP/s), 2 float32 rows over 200 and 40 11 us (two launches of 5).
#include <type_traits>

#include "attention8.h"

namespace specdec {

namespace {

// ---------------------------------------------------------------- few rows over short texts
// Bound by the stream of the own codes and of the ring's rows, twice as large (128 rows over up to 256 own keys:
// 167 MB, 45 us, 3.7 TB/s; attn8_kernel 308: its eight waves a unit wait for each other's start and merge).
// A wave's part of a unit (a sequence's kv head, 16 query rows): chunks wave, wave + NW, ... of the
// row's own keys, on top of the prefix's parts wave, wave + NW, ..., from which its
// running maximum, sum and outputs start.  Unlike attn8_kernel's, a unit is one
// workgroup's, and nothing is shared by its waves but the merge at the end: queries in
// registers, ring rows to registers before the codes.  So a wave is a unit where there are
// many of them, and its start (length, then descriptors, then codes) hides under
// the other waves' streams instead of a barrier's.
//
// Queries of float32: three bf16 parts, as attn8_kernel's; of bf16: themselves, and the scores are
// scaled.  Probabilities: three bf16 parts, or two (what is left, 2^-17, is far below the result's
// own rounding); the products are few.
template <typename T> struct OwnParts;
template <> struct OwnParts<float> { static constexpr int kQ = 3, kP = 3; };
template <> struct OwnParts<uint16_t> { static constexpr int kQ = 1, kP = 2; };

template <int N>
__device__ __forceinline__ void split_parts(const float (&v)[8], bf16x8 (&part)[N]) {
  float r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = v[j];
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const __bf16 h = (__bf16)r[j];
      part[k][j] = h;
      r[j] -= (float)h;
    }
}

// Waves of a SIMD: what the registers allow (128 dims: outputs, codes, a ring's sub-chunk, queries).
__host__ __device__ constexpr int own_resident(int head_dim) { return head_dim == 128 ? 2 : 3; }

// ONCE: a sequence's codes are read by one unit.
template <int HD, typename T, int NW, bool ONCE>
__global__ __launch_bounds__(64 * NW, own_resident(HD)) void own_kernel(AttnArgs a, SharedParts pre, int n_tiles) {
  constexpr int KST = HD / 32, DT = HD / 16, FS = HD / 32, SP = steps_of(HD), OS = HD + 4;
  constexpr int NQ = OwnParts<T>::kQ, NP = OwnParts<T>::kP;
  constexpr bool F32 = NQ == 3;
  __shared__ float so[NW > 1 ? NW : 1][16][NW > 1 ? OS : 1];
  __shared__ float sml[NW][16][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, grp = lane >> 4;
  const int H = a.n_heads, G = a.n_kv_heads, group = H / G, rps = a.rps, nq = rps * group, window = a.f8.ring.capacity;
  const int g = blockIdx.x % G, bt = blockIdx.x / G, tile = bt % n_tiles, b = bt / n_tiles;
  const float qscale = 1.44269504088896341f / sqrtf((float)HD);  // (scores in powers of two)
  const float factor = F32 ? 1.f : qscale;
  const int qa = tile * 16 + c16, qr = min(qa, nq - 1) / group, head = g * group + min(qa, nq - 1) - qr * group;
  const int row = b * rps + qr, n_here = min(16, nq - tile * 16);

  // This lane's query, in the products' order.
  f32x4 qv[KST][2];
#pragma unroll
  for (int s = 0; s < KST; ++s) {
    const int d = HD >= 64 ? 64 * (s >> 1) + 16 * grp + 8 * (s & 1) : 32 * s + 8 * grp;
    qv[s][0] = qv[s][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (c16 < n_here) load8((const T*)a.qr + ((size_t)row * H + head) * HD + d, qv[s]);
  }
  const int len = __builtin_amdgcn_readfirstlane(a.f8.len[b]);
  const int sealed = len / kF8Block * (kF8Block / kF8Sub / SP);
  const int most = (a.max_ctx + chunk_of(HD) - 1) / chunk_of(HD);
  const int k_end = max(1, min(most, (len + rps - 1) / chunk_of(HD) + 1));
  const int j_sealed = min(k_end, sealed);

  // Codes: loads past the sealed ones read nothing.  (Of large batches, where one unit reads them: past the caches; 64
  // rows of 7B-like heads over 400 to 500 own keys 56 -> 49 us; 16 over 64 to 700, four waves a unit, 32 -> 34 us.  Where
  // units of several tiles read them, not: 256 x 7 rows of 1.1B-like heads, four tiles, over 550 to 600 48 and 36 us;
  // 256 x 4 of 64 heads of 128 over 8 kv heads, two tiles, 68 and 71.)
  constexpr int kCodes = NW == 1 && ONCE ? kNonTemporal : 0;
  const __amdgpu_buffer_rsrc_t cr = make_rsrc(a.f8.code_base(a.layer, b, g), (uint32_t)j_sealed * SP * 2 * kF8Sub * HD);
  const __amdgpu_buffer_rsrc_t sr = make_rsrc(a.f8.scale_base(a.layer, b, g), (uint32_t)((j_sealed * SP + 1) & ~1) * 4);
  u32x4 kc[SP][FS], vc[SP][FS];
  float ks, vs;
  auto load_codes = [&](int j) {
    const uint32_t at = (uint32_t)j * SP * 2 * kF8Sub * HD + lane * 16;
#pragma unroll
    for (int i = 0; i < SP * FS; ++i) {
      const uint32_t k = at + i / FS * 2 * kF8Sub * HD + i % FS * 1024;
      kc[i / FS][i % FS] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(cr, k, 0, kCodes));
      vc[i / FS][i % FS] =
          __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(cr, k + kF8Sub * HD, 0, kCodes));
    }
    ks = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sr, (j * SP & ~1) * 4, 0, 0));
    vs = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sr, (j * SP | 1) * 4, 0, 0));
  };
  const uint16_t* ring = k_block<uint16_t>(a.f8.ring, a.layer, b, g);
  const __amdgpu_buffer_rsrc_t rr = make_rsrc(ring, (uint32_t)window * HD * 4u);
  u32x4 rk[2 * KST], rv[DT];
  // (rows behind the newest are not asked for: most of a short text's 32)
  const int newest = len + min(rps, (tile * 16 + n_here - 1) / group + 1) - 1;
  auto load_ring = [&](int sub) {
    const int w0 = sub * kF8Sub % window, rows = newest - sub * kF8Sub;  // (rows: of the last one)
#pragma unroll
    for (int i = 0; i < 2 * KST; ++i) {
      const int t = i / KST, s = i % KST, d = HD >= 64 ? 64 * (s >> 1) + 16 * grp + 8 * (s & 1) : 32 * s + 8 * grp;
      const int pos = 8 * (c16 >> 2) + 4 * t + (c16 & 3);
      const uint32_t at = (uint32_t)KvIndex<uint16_t>::k(w0 + pos, d, HD, window) * 2u;
      rk[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, pos <= rows ? at : kOutOfRange, 0, 0));
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const uint32_t at = (uint32_t)KvIndex<uint16_t>::v(w0 + 8 * grp, 16 * dt + c16, HD, window) * 2u;
      rv[dt] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, 8 * grp <= rows ? at : kOutOfRange, 0, 0));
    }
  };

  // This wave's chunks, the ring's first.
  int j = wave, jr = max(j, j + (sealed - j + NW - 1) / NW * NW);
  if (jr < k_end) load_ring(jr * SP);
  load_codes(j);

  // The prefix's parts: where this wave's softmax starts.
  f32x4 of[DT];
  float mx = kLeast, sm = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) of[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int plen = __builtin_amdgcn_readfirstlane(*pre.len);
  const int n_pre = (min(plen, pre.max_len) + pre.keys - 1) / pre.keys;
#pragma unroll 2
  for (int p = wave; p < n_pre; p += NW) {  // (two parts' loads in flight: 94 -> 92 us, 128 rows over 16384 keys)
    const size_t slot = ((size_t)row * H + head) * pre.stride + p;
    float2 ml = make_float2(kLeast, 0.f);
    f32x4 v[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) v[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (c16 < n_here) {
      ml = *(const float2*)(pre.ml + 2 * slot);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) v[dt] = *(const f32x4*)(pre.o + slot * HD + 16 * dt + 4 * grp);
    }
    const float m = fmaxf(mx, ml.x), own = __builtin_amdgcn_exp2f(mx - m), w = __builtin_amdgcn_exp2f(ml.x - m);
    sm = sm * own + (grp == 0 ? w * ml.y : 0.f);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) of[dt] = of[dt] * own + w * v[dt];
    mx = m;
  }

  bf16x8 qq[KST][NQ];
#pragma unroll
  for (int s = 0; s < KST; ++s) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = qv[s][e >> 2][e & 3] * (F32 ? qscale : 1.f);
    split_parts<NQ>(v, qq[s]);
  }

  // kk(t, s): K rows of tile t, dims of step s; scores of this lane's 8 positions.
  auto scores = [&](auto kk, float (&p)[8]) {
    floatx4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < KST; ++s) {
      const bf16x8 k0 = kk(0, s), k1 = kk(1, s);
#pragma unroll
      for (int k = NQ - 1; k >= 0; --k) {  // (small parts first)
        acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qq[s][k], acc[0], 0, 0, 0);
        acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qq[s][k], acc[1], 0, 0, 0);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = acc[e >> 2][e & 3] * factor;
  };
  // The running maximum and sum over new scores, which become probabilities (see attn8_kernel).
  auto softmax = [&](auto& p) {
    constexpr int N = sizeof(p) / sizeof(float);
    float m = fmaxf(p[0], p[1]);
#pragma unroll
    for (int e = 2; e < N; ++e) m = fmaxf(m, p[e]);
    const float mnew = fmaxf(mx, groups_max(m));
    if (__any(mnew > mx)) {
      const float alpha = __builtin_amdgcn_exp2f(mx - mnew);
      sm *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) of[dt] *= alpha;
      mx = mnew;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      p[e] = __builtin_amdgcn_exp2f(p[e] - mx);
      sm += p[e];
    }
  };
  auto add = [&](auto vv, const bf16x8 (&pp)[NP]) {  // O^T += V^T P^T
    constexpr int DG = DT < 4 ? DT : 4;
#pragma unroll
    for (int d0 = 0; d0 < DT; d0 += DG) {
      bf16x8 v[DG];
#pragma unroll
      for (int i = 0; i < DG; ++i) v[i] = vv(d0 + i);
#pragma unroll
      for (int k = NP - 1; k >= 0; --k)
#pragma unroll
        for (int i = 0; i < DG; ++i) {
          const floatx4 o = __builtin_bit_cast(floatx4, of[d0 + i]);
          of[d0 + i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[i], pp[k], o, 0, 0, 0));
        }
    }
  };

  if (jr < k_end) {  // (wave-uniform)
    const int qpos = c16 < n_here ? len + qr : -1;
    int vis = qpos + 1, lowest = c16 < n_here ? qpos : 0x7fffffff;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      vis = max(vis, __shfl_xor(vis, o, kWave));
      lowest = min(lowest, __shfl_xor(lowest, o, kWave));
    }
    vis = __builtin_amdgcn_readfirstlane(vis);
    lowest = __builtin_amdgcn_readfirstlane(lowest);
#pragma unroll 1
    for (bool first = true; jr < k_end; jr += NW)
#pragma unroll 1
      for (int sp = 0; sp < SP; ++sp) {
        const int sub = jr * SP + sp, k0 = sub * kF8Sub;
        if (k0 >= vis) break;
        if (!first) load_ring(sub);
        first = false;
        float p[8];
        scores([&](int t, int s) { return __builtin_bit_cast(bf16x8, rk[t * KST + s]); }, p);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = k0 + 8 * grp + e > qpos ? -INFINITY : p[e];
        softmax(p);
        bf16x8 pp[NP];
        split_parts<NP>(p, pp);
        // Where some query does not see all rows: stale entries past the newest row leave the
        // product, and so do NaN and infinities, which are added to the queries that see them.
        const bool diagonal = k0 + kF8Sub - 1 > lowest;
        const int nvalid = vis - (k0 + 8 * grp);
        bool odd = false;
        if (diagonal) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              uint32_t x = rv[dt][w];
              if (2 * w >= nvalid) x = 0u;
              else if (2 * w + 1 >= nvalid) x &= 0xffffu;
              const bool lo = (x & 0x7f80u) == 0x7f80u, up = (x & 0x7f800000u) == 0x7f800000u;
              odd |= lo || up;
              if (lo) x &= 0xffff0000u;
              if (up) x &= 0xffffu;
              rv[dt][w] = x;
            }
        }
        add([&](int dt) { return __builtin_bit_cast(bf16x8, rv[dt]); }, pp);
        if (__any(odd)) {
          for (int i = 0; i < kF8Sub; ++i) {  // (position k0 + i; its probability lies in lane group i / 8)
            float pi = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) pi = (i & 7) == e ? p[e] : pi;
            pi = __shfl(pi, 16 * (i >> 3) + c16, kWave);
            const uint16_t* vrow = ring + KvIndex<uint16_t>::v(k0 % window + i, 0, HD, window);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float v = bf16_bits_to_f32(vrow[(size_t)dt * kWave * 8 + (4 * grp + r) * 8]);
                if (k0 + i <= qpos && !isfinite(v)) of[dt][r] += pi * v;
              }
          }
        }
      }
  }

  for (; j < j_sealed; j += NW) {  // (wave-uniform) codes: every query sees them all
    float p[8 * SP];
#pragma unroll
    for (int sp = 0; sp < SP; ++sp) {
      float x[8];
      scores(
          [&](int t, int s) {
            const u32x4 w = HD >= 64 ? kc[sp][t * (HD / 64) + s / 2] : kc[sp][0];
            const int h = HD >= 64 ? s & 1 : t;
            return fp8x8_to_bf16(w[2 * h], w[2 * h + 1], ks);
          },
          x);
#pragma unroll
      for (int e = 0; e < 8; ++e) p[8 * sp + e] = x[e];
    }
    softmax(p);
#pragma unroll
    for (int sp = 0; sp < SP; ++sp) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = p[8 * sp + e];
      bf16x8 pp[NP];
      split_parts<NP>(x, pp);
      add([&](int dt) { return fp8x8_to_bf16(vc[sp][dt / 2][2 * (dt & 1)], vc[sp][dt / 2][2 * (dt & 1) + 1], vs); }, pp);
    }
    load_codes(j + NW);
  }

  sm += __shfl_xor(sm, 16, kWave);
  sm += __shfl_xor(sm, 32, kWave);
  T* out = (T*)a.o;
  if (threadIdx.x == 0 && (len + rps > a.max_ctx || plen > pre.max_len)) set_status(a.status, kStatusKvCapacity);  // (the host's bound was wrong)
  if constexpr (NW == 1) {
    const float inv = 1.0f / sm;
    if (c16 < n_here)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) store4(out + ((size_t)row * H + head) * HD + 16 * dt + 4 * grp, of[dt] * inv);
  } else {
    if (c16 < n_here) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *(f32x4*)&so[wave][c16][16 * dt + 4 * grp] = of[dt];
      if (grp == 0) {
        sml[wave][c16][0] = mx;
        sml[wave][c16][1] = sm;
      }
    }
    __syncthreads();
    const int d = threadIdx.x % (HD / 4) * 4;
    for (int i = threadIdx.x / (HD / 4); i < n_here; i += 64 * NW / (HD / 4)) {
      float M = kLeast, L = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) M = fmaxf(M, sml[w][i][0]);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float e = __builtin_amdgcn_exp2f(sml[w][i][0] - M);
        L += e * sml[w][i][1];
        o += e * *(const f32x4*)&so[w][i][d];
      }
      const int q = tile * 16 + i, r = q / group;
      store4(out + ((size_t)(b * rps + r) * H + g * group + q - r * group) * HD + d, o * (1.0f / L));
    }
  }
}

// Waves of a unit: a wave a unit where the card is full of them, else as many as fill it; 0: another kernel, for many
// bf16 rows the one that wide_takes says, else attn8_kernel, whose units are split over workgroups.  That is faster from
// 32 chunks a wave on where the card is full (7B-like, 32 sequences: over 1000 own keys 52 us, 60 there; over 2000 108 and
// 100), from the fewer the emptier it is (one sequence: over 1000 14 and 16, over 2000 18 and 17; 1.1B-like, 16: over 2000
// 15 and 18, over 4000 22 both).
int own_waves(int rps, int batch, int n_heads, int n_kv_heads, int head_dim, int max_ctx) {
  const int nq = rps * (n_heads / n_kv_heads);
  if (nq > 64) return 0;
  const int64_t units = (int64_t)batch * n_kv_heads * ((nq + 15) / 16);
  const int64_t slots = 4L * own_resident(head_dim) * device_compute_units();
  const int nb = (max_ctx + chunk_of(head_dim) - 1) / chunk_of(head_dim);
  int nw = 8;
  while (nw > 1 && (units * nw > slots || nw > nb)) nw /= 2;
  const int64_t most = std::max<int64_t>(6, std::min<int64_t>(32, 32 * units * nw / slots));
  return nb <= most * nw && units < 1 << 24 ? nw : 0;
}

template <typename T>
hipError_t launch_own(const AttnArgs& a, const SharedParts& pre, int nw, hipStream_t s) {
  const int nq = a.rps * (a.n_heads / a.n_kv_heads), n_tiles = (nq + 15) / 16;
  const dim3 grid((unsigned)(a.M / a.rps) * a.n_kv_heads * n_tiles);
#define SD_OWN(HD, NW, ONCE) hipLaunchKernelGGL((own_kernel<HD, T, NW, ONCE>), grid, dim3(64 * NW), 0, s, a, pre, n_tiles)
#define SD_OWN_HD(HD)                          \
  switch (nw) {                                \
    case 1:                                    \
      if (n_tiles == 1) SD_OWN(HD, 1, true);   \
      else SD_OWN(HD, 1, false);               \
      break;                                   \
    case 2: SD_OWN(HD, 2, false); break;       \
    case 4: SD_OWN(HD, 4, false); break;       \
    default: SD_OWN(HD, 8, false); break;      \
  }
  switch (a.head_dim) {
    case 32: SD_OWN_HD(32) break;
    case 64: SD_OWN_HD(64) break;
    case 128: SD_OWN_HD(128) break;
    default: return hipErrorInvalidValue;
  }
#undef SD_OWN_HD
#undef SD_OWN
  return hipGetLastError();
}

// ---------------------------------------------------------------- many rows of 16-bit queries
// One workgroup: 16 RT rows of a kv head and a range of keys, its waves every fourth chunk of
// 32 (all rows each), merged at the end as attn8_kernel's are; or 64 RT rows (KW, below).  Queries of bf16 are one
// part of their product, with K's codes as bf16 (exact); probabilities are one fp16 part
// with V's codes as fp16 (exact), off by 2^-11 of each; the sums are taken of the rounded ones,
// by a product with ones.  bf16 rows of the ring take two bf16 parts.
//
// What bounds it is the vector unit beside the matrix unit: a chunk's conversions, 64 of two
// codes each for 32 keys of 128 dims, are shared by RT tiles; a score costs a maximum, a
// multiply-add, an exponential and half a conversion.  Of a chunk of 32 keys and 32 rows of 128 dims the products take
// the matrix unit 544 cycles and the rest the vector unit's issue about 700, which overlap in part (128 rows over 65536
// keys: matrix unit busy 41% of the time).  The running maximum is raised only when a score exceeds it by 2^kSlack (then
// exactly): no value crosses lanes in a chunk that does not.
constexpr float kSlack = 4.f, kWideLift = 11.f;  // (2^(kSlack + kWideLift) is fp16's; held down to 2^-25 in full)

// Maximum of a lane's scores, NaN where one is (fmaxf would quiet each product's value first).
__device__ __forceinline__ float max_of(const float (&p)[8]) {
  float m = p[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) m = __builtin_elementwise_maximum(m, p[e]);
  return m;
}

// KW: waves that take turns at a unit's chunks (the unit is the workgroup's, its waves are merged at
// the end), or 1: each wave has 16 RT rows of its own and all of its unit's keys, so nothing is
// merged, and the codes that four waves read at about the same time come from one cache.  (Own texts' form of it spills
// 49 registers with 64 dims, 28 with 128, outside of the loop over codes whose scales are in range.)
template <int HD, int RT, int KW, class X>
__global__ __launch_bounds__(256, 2) void wide_kernel(AttnArgs a, int n_tiles, int parts, int per, X x) {
  constexpr int KST = HD / 32, DT = HD / 16, FS = HD / 32, OS = HD + 4, NW = KW;
  __shared__ float so[KW > 1 ? KW : 1][16][KW > 1 ? OS : 1];
  __shared__ float sml[KW][16][2];
  typedef uint16_t T;
  const int lane = threadIdx.x & 63;
  const int wave_id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = KW > 1 ? wave_id : 0;
  const int c16 = lane & 15, grp = lane >> 4;
  const int H = a.n_heads, G = a.n_kv_heads, group = H / G, rps = a.rps, nq = rps * group, window = a.f8.ring.capacity;
  const int b = blockIdx.z, u = blockIdx.y, part = blockIdx.x, unit = u / G, g = u - unit * G;
  const int tile = KW > 1 ? unit : unit * 4 + wave_id;  // (of 16 RT rows)
  if (KW == 1 && tile * RT * 16 >= nq) return;
  const float qscale = 1.44269504088896341f / sqrtf((float)HD), inv_group = 1.0f / (float)group;
  int seq = b;
  if constexpr (X::kPrefix) seq = x.b;
  const int nb = __builtin_amdgcn_readfirstlane(chunks_of<kF8Sub>(a, x, b)), k_lo = part * per;
  if (k_lo >= nb) return;  // (workgroup-uniform)
  const int k_hi = min(nb, k_lo + per);

  bf16x8 qq[RT][KST];
#pragma unroll
  for (int q = 0; q < RT; ++q) {
    const int qa = (tile * RT + q) * 16 + c16, qr = div_small(qa, inv_group);
#pragma unroll
    for (int s = 0; s < KST; ++s) {
      const int d = HD >= 64 ? 64 * (s >> 1) + 16 * grp + 8 * (s & 1) : 32 * s + 8 * grp;
      u32x4 v = {0u, 0u, 0u, 0u};
      if (qa < nq) v = *(const u32x4_a2*)((const T*)a.qr + ((size_t)(b * rps + qr) * H + g * group + qa - qr * group) * HD + d);
      qq[q][s] = __builtin_bit_cast(bf16x8, v);
    }
  }
  const int sealed = __builtin_amdgcn_readfirstlane(a.f8.len[seq]) / kF8Block * (kF8Block / kF8Sub);
  const int j_sealed = min(k_hi, sealed);
  const __amdgpu_buffer_rsrc_t cr = make_rsrc(a.f8.code_base(a.layer, seq, g), (uint32_t)j_sealed * 2 * kF8Sub * HD);
  const __amdgpu_buffer_rsrc_t sr = make_rsrc(a.f8.scale_base(a.layer, seq, g), (uint32_t)((j_sealed + 1) & ~1) * 4);
  u32x4 kc[FS], vc[FS];
  float ks, vs;
  auto load_k = [&](int j) {
    const uint32_t at = (uint32_t)j * 2 * kF8Sub * HD + lane * 16;
#pragma unroll
    for (int i = 0; i < FS; ++i)
      kc[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(cr, at + i * 1024, 0, 0));
    ks = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sr, (j & ~1) * 4, 0, 0));
  };
  auto load_v = [&](int j) {
    const uint32_t at = (uint32_t)j * 2 * kF8Sub * HD + kF8Sub * HD + lane * 16;
#pragma unroll
    for (int i = 0; i < FS; ++i)
      vc[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(cr, at + i * 1024, 0, 0));
    vs = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sr, (j | 1) * 4, 0, 0));
  };
  int j = k_lo + wave, jr = max(j, j + (sealed - j + NW - 1) / NW * NW);  // (jr: the first of the ring's)
  load_k(j);
  load_v(j);

  floatx4 of[RT][DT], sums[RT];
  float mx[RT];
#pragma unroll
  for (int q = 0; q < RT; ++q) {
    mx[q] = kLeast;
    sums[q] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) of[q][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  if constexpr (X::kJoin && KW == 1) {  // from the prefix's parts on
    const int n_pre = (min(*x.parts.len, x.parts.max_len) + x.parts.keys - 1) / x.parts.keys;
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      const int qa = (tile * RT + q) * 16 + c16, qr = div_small(min(qa, nq - 1), inv_group);
      const size_t slot = ((size_t)(b * rps + qr) * H + g * group + min(qa, nq - 1) - qr * group) * x.parts.stride;
      for (int p = 0; p < n_pre; ++p) {
        const float2 ml = *(const float2*)(x.parts.ml + 2 * (slot + p));
        const float m = fmaxf(mx[q], ml.x), was = __builtin_amdgcn_exp2f(mx[q] - m);
        const float w = __builtin_amdgcn_exp2f(ml.x - m) * 0x1p11f;  // (2^kWideLift)
        sums[q] = sums[q] * was + w * ml.y;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const f32x4 v = *(const f32x4*)(x.parts.o + (slot + p) * HD + 16 * dt + 4 * grp);
          of[q][dt] = of[q][dt] * was + __builtin_bit_cast(floatx4, v) * w;
        }
        mx[q] = m;
      }
    }
  }
  // Scores (unscaled) of N positions a lane: whether one exceeds its maximum by 2^kSlack; the maxima
  // raised to them.
  auto over = [&](const float (&p)[RT][8]) {
    bool any = false;  // (tile by tile: a NaN says nothing of the other tiles' queries)
#pragma unroll
    for (int q = 0; q < RT; ++q) any |= __builtin_fmaf(max_of(p[q]), qscale, -mx[q]) > kSlack;
    return __any(any);
  };
  auto raise = [&](const float (&p)[RT][8]) {
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      const float mnew = fmaxf(mx[q], groups_max(max_of(p[q])) * qscale), alpha = __builtin_amdgcn_exp2f(mx[q] - mnew);
      sums[q] *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) of[q][dt] *= alpha;
      mx[q] = mnew;
    }
  };
  // Scores become probabilities times 2^kWideLift.
  auto exponentials = [&](float (&p)[RT][8]) {
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      const float off = kWideLift - mx[q];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[q][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[q][e], qscale, off));
    }
  };
  // The codes in hand: scores of this lane's positions.
  auto scores = [&](float (&p)[RT][8]) {
    floatx4 acc[RT][2];
#pragma unroll
    for (int q = 0; q < RT; ++q) acc[q][0] = acc[q][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KST; ++s) {
      bf16x8 kk[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const u32x4 w = HD >= 64 ? kc[t * (HD / 64) + s / 2] : kc[0];
        const int h = HD >= 64 ? s & 1 : t;
        kk[t] = fp8x8_to_bf16(w[2 * h], w[2 * h + 1], ks);
      }
#pragma unroll
      for (int q = 0; q < RT; ++q) {
        acc[q][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[0], qq[q][s], acc[q][0], 0, 0, 0);
        acc[q][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[1], qq[q][s], acc[q][1], 0, 0, 0);
      }
    }
#pragma unroll
    for (int q = 0; q < RT; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) p[q][e] = acc[q][e >> 2][e & 3];
  };
  auto halves = [&](const float (&p)[RT][8], f16x8 (&pp)[RT]) {
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{p[q][2 * e], p[q][2 * e + 1]}, f16x2));
      pp[q] = __builtin_bit_cast(f16x8, w);
    }
  };
  f16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (_Float16)1.f;
  auto add = [&](const f16x8 (&pp)[RT], auto in_range) {
#pragma unroll
    for (int q = 0; q < RT; ++q) sums[q] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, pp[q], sums[q], 0, 0, 0);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const u32x4 w = vc[dt / 2];
      const f16x8 vv = fp8x8_to_f16(w[2 * (dt & 1)], w[2 * (dt & 1) + 1], in_range ? vs : 1.0f);
#pragma unroll
      for (int q = 0; q < RT; ++q) {
        if (in_range) of[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, pp[q], of[q][dt], 0, 0, 0);
        else of[q][dt] += __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, pp[q], floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0) * vs;
      }
    }
  };

  // Codes: every query sees them all.  Where all of V's scales leave fp16's values (2^-15 .. 2^7),
  // a chunk's exponentials and second product run beside the next chunk's scores, which wait
  // for none of them: one block of instructions, that the vector and the matrix unit share.
  bool ranged = true;
  for (int i = k_lo / 2 + lane; 2 * i < j_sealed; i += kWave) {
    const int ve = (int)(__builtin_amdgcn_raw_buffer_load_b32(sr, (2 * i + 1) * 4, 0, 0) >> 23) - 127;
    ranged = ranged && ve >= -15 && ve <= 7;
  }
  if (j < j_sealed) {  // (wave-uniform)
    if (__all(ranged)) {
      // (the maxima are raised outside of the loop over chunks: a branch inside it would cost copies of all outputs)
      float p[RT][8], next[RT][8];
      scores(p);
      load_k(j + NW);
      while (true) {
        raise(p);
        bool more;
        do {
          f16x8 pp[RT];
          // (a wave at its products before one at its maxima: 1.1B-like, 64 rows over 131072 keys 97 -> 92 us, four
          // runs of each; 128 dims, 128 rows: 112 to 119 us with it and without)
          if (HD < 128) __builtin_amdgcn_s_setprio(1);
          scores(next);  // (past the last chunk: of zeros, unused)
          exponentials(p);
          load_k(j + 2 * NW);
          halves(p, pp);
          add(pp, std::true_type{});
          if (HD < 128) __builtin_amdgcn_s_setprio(0);
          load_v(j + NW);
          // (in this order: 4 vector instructions and an exponential to a product of the scores, 2 to one of the
          // values; 51.5 us against 55 in the compiler's, 128 rows over 16384 keys)
#pragma unroll
          for (int i = 0; i < 2 * RT * KST; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          }
#pragma unroll
          for (int i = 0; i < RT * (DT + 1); ++i) {
            __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          }
          j += NW;
          more = j < j_sealed;
#pragma unroll
          for (int q = 0; q < RT; ++q)
#pragma unroll
            for (int e = 0; e < 8; ++e) p[q][e] = next[q][e];
        } while (more && !over(p));
        if (!more) break;
      }
    } else {
#pragma unroll 1
      for (; j < j_sealed; j += NW) {
        float p[RT][8];
        f16x8 pp[RT];
        scores(p);
        load_k(j + NW);
        if (over(p)) raise(p);
        exponentials(p);
        halves(p, pp);
        add(pp, std::false_type{});  // (the codes' products, times the scale)
        load_v(j + NW);
      }
    }
  }

  if (jr < k_hi) {  // (wave-uniform) the ring's rows
    int qpos[RT], vis = 0, lowest = 0x7fffffff;
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      const int qa = (tile * RT + q) * 16 + c16;
      const RowDesc rd = row_of(a, x, b, qa < nq ? div_small(qa, inv_group) : 0);
      qpos[q] = qa < nq && rd.valid ? rd.pos : -1;
      if (qpos[q] >= 0) {
        vis = max(vis, qpos[q] + 1);
        lowest = min(lowest, qpos[q]);
      }
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      vis = max(vis, __shfl_xor(vis, o, kWave));
      lowest = min(lowest, __shfl_xor(lowest, o, kWave));
    }
    vis = __builtin_amdgcn_readfirstlane(vis);
    lowest = __builtin_amdgcn_readfirstlane(lowest);
    const uint16_t* ring = k_block<uint16_t>(a.f8.ring, a.layer, seq, g);
    bf16x8 one;
#pragma unroll
    for (int e = 0; e < 8; ++e) one[e] = (__bf16)1.f;
    // (a sub-chunk's K and V are asked for a sub-chunk ahead; those behind the newest row, not)
    const __amdgpu_buffer_rsrc_t rr = make_rsrc(ring, (uint32_t)window * HD * 4u);
    u32x4 rk[2 * KST], rv[DT];
    auto ring_k = [&](int k0) {
      const int w0 = k0 % window;
#pragma unroll
      for (int i = 0; i < 2 * KST; ++i) {
        const int t = i / KST, s = i % KST, d = HD >= 64 ? 64 * (s >> 1) + 16 * grp + 8 * (s & 1) : 32 * s + 8 * grp;
        const int pos = 8 * (c16 >> 2) + 4 * t + (c16 & 3);
        const uint32_t at = (uint32_t)KvIndex<uint16_t>::k(w0 + pos, d, HD, window) * 2u;
        rk[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, k0 + pos < vis ? at : kOutOfRange, 0, 0));
      }
    };
    auto ring_v = [&](int k0) {
      const int w0 = k0 % window;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint32_t at = (uint32_t)KvIndex<uint16_t>::v(w0 + 8 * grp, 16 * dt + c16, HD, window) * 2u;
        rv[dt] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, k0 + 8 * grp < vis ? at : kOutOfRange, 0, 0));
      }
    };
    ring_k(jr * kF8Sub);
    ring_v(jr * kF8Sub);
#pragma unroll 1
    for (; jr < k_hi; jr += NW) {
      const int k0 = jr * kF8Sub, w0 = k0 % window;
      if (k0 >= vis) break;
      const bool diagonal = k0 + kF8Sub - 1 > lowest;
      floatx4 acc[RT][2];
#pragma unroll
      for (int q = 0; q < RT; ++q) acc[q][0] = acc[q][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KST; ++s) {
#pragma unroll
        for (int q = 0; q < RT; ++q) {
          acc[q][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, rk[s]), qq[q][s], acc[q][0], 0, 0, 0);
          acc[q][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, rk[KST + s]), qq[q][s], acc[q][1], 0, 0, 0);
        }
      }
      ring_k(k0 + NW * kF8Sub);
      float p[RT][8];
      bf16x8 pp[RT][2];
#pragma unroll
      for (int q = 0; q < RT; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) p[q][e] = k0 + 8 * grp + e > qpos[q] ? -INFINITY : acc[q][e >> 2][e & 3];
      if (over(p)) raise(p);
      exponentials(p);
#pragma unroll
      for (int q = 0; q < RT; ++q) {
        split_parts<2>(p[q], pp[q]);
#pragma unroll
        for (int k = 1; k >= 0; --k) sums[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(one, pp[q][k], sums[q], 0, 0, 0);
      }
      // (stale entries, NaN and infinities where some query does not see all rows: see attn8_kernel)
      const int nvalid = vis - (k0 + 8 * grp);
      bool odd = false;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        u32x4 v = rv[dt];
        if (diagonal) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            if (2 * w >= nvalid) v[w] = 0u;
            else if (2 * w + 1 >= nvalid) v[w] &= 0xffffu;
            const bool lo = (v[w] & 0x7f80u) == 0x7f80u, up = (v[w] & 0x7f800000u) == 0x7f800000u;
            odd |= lo || up;
            if (lo) v[w] &= 0xffff0000u;
            if (up) v[w] &= 0xffffu;
          }
        }
#pragma unroll
        for (int k = 1; k >= 0; --k)
#pragma unroll
          for (int q = 0; q < RT; ++q)
            of[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), pp[q][k], of[q][dt], 0, 0, 0);
      }
      if (__any(odd)) {
        for (int i = 0; i < kF8Sub; ++i) {  // (position k0 + i; its probability lies in lane group i / 8)
          const uint16_t* vrow = ring + KvIndex<uint16_t>::v(w0 + i, 0, HD, window);
#pragma unroll
          for (int q = 0; q < RT; ++q) {
            float pi = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) pi = (i & 7) == e ? p[q][e] : pi;
            pi = __shfl(pi, 16 * (i >> 3) + c16, kWave);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float v = bf16_bits_to_f32(vrow[(size_t)dt * kWave * 8 + (4 * grp + r) * 8]);
                if (k0 + i <= qpos[q] && !isfinite(v)) of[q][dt][r] += pi * v;
              }
          }
        }
      }
      ring_v(k0 + NW * kF8Sub);
    }
  }

  if constexpr (KW == 1) {  // a lane's dims of its queries
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      const int qa = (tile * RT + q) * 16 + c16, qr = div_small(qa, inv_group), head = g * group + qa - qr * group;
      if (qa >= nq) continue;
      const size_t row = (size_t)b * rps + qr;
      if constexpr (X::kPrefix) {
        const size_t slot = (row * H + head) * parts + part;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          *(floatx4*)(a.o_part + slot * HD + 16 * dt + 4 * grp) = of[q][dt] * 0x1p-11f;  // (2^-kWideLift)
        if (grp == 0) *(float2*)(a.ml_part + 2 * slot) = make_float2(mx[q], sums[q][0] * 0x1p-11f);
      } else {
        const float inv = 1.0f / sums[q][0];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          store4((T*)a.o + (row * H + head) * HD + 16 * dt + 4 * grp, __builtin_bit_cast(f32x4, of[q][dt]) * inv);
        if (grp == 0 && (a.f8.len[b] + qr >= a.max_ctx || *x.parts.len > x.parts.max_len))
          set_status(a.status, kStatusKvCapacity);  // (the host's bound was wrong)
      }
    }
    return;
  }
  // The waves' results, tile by tile.
#pragma unroll
  for (int q = 0; q < RT; ++q) {
    const int n_here = min(16, nq - (tile * RT + q) * 16);
    if (n_here <= 0) break;
    __syncthreads();
    if (c16 < n_here) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *(floatx4*)&so[wave][c16][16 * dt + 4 * grp] = of[q][dt];
      if (grp == 0) {
        sml[wave][c16][0] = mx[q];
        sml[wave][c16][1] = sums[q][0];
      }
    }
    __syncthreads();
    const int d = threadIdx.x % (HD / 4) * 4;
    for (int i = threadIdx.x / (HD / 4); i < n_here; i += 64 * NW / (HD / 4)) {
      float M = kLeast, L = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) M = fmaxf(M, sml[w][i][0]);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float e = __builtin_amdgcn_exp2f(sml[w][i][0] - M) * 0x1p-11f;  // (2^-kWideLift)
        L += e * sml[w][i][1];
        o += e * *(const f32x4*)&so[w][i][d];
      }
      const int qa = (tile * RT + q) * 16 + i, qr = div_small(qa, inv_group), head = g * group + qa - qr * group;
      if constexpr (X::kPrefix) {
        const size_t slot = ((size_t)(b * rps + qr) * H + head) * parts + part;
        *(f32x4*)(a.o_part + slot * HD + d) = o;
        if (d == 0) *(float2*)(a.ml_part + 2 * slot) = make_float2(M, L);
      } else {
        finish_row(a, x, b, qr, head, d, o, 1.0f, M, L);
      }
    }
  }
}

// Rows of a kv head from which bf16 queries take it, and how the work is split: query tiles of
// 16 RT rows, as many parts of the keys as fill the card twice.
__host__ __device__ constexpr int wide_tiles(int head_dim) { return head_dim == 128 ? 2 : 4; }
bool is_wide(int nq) { return nq > 16; }
// `line` of its plan: whether a wave has rows of its own (KW == 1).
Plan wide_plan(int rps, int batch, int n_heads, int n_kv_heads, int head_dim, int max_ctx, bool prefix) {
  Plan p{};
  const int nq = rps * (n_heads / n_kv_heads), rows = 16 * wide_tiles(head_dim);
  const long slots = 2L * device_compute_units(), nb = (max_ctx + kF8Sub - 1) / kF8Sub;
  // A wave's own rows: a prefix's where they fill the card without a cut of its keys (8 x 512 rows over 2000
  // keys 223 us, 245 else; 6 x 170 rows over 3500, half of that, 99 us, 95 else).  Own texts', whose keys are never cut:
  // where tiles full of rows would fill the card and the texts have at most 32 chunks (7B-like, four waves a tile's keys
  // and rows of their own: 8 x 70 rows over 500 keys 32 and 26 us, over 2000 49 and 58; 8 x 40, half as many, over 250
  // 16 and 19), or the waves that have rows are three quarters of the card's and of their workgroups' (64 x 100 rows of
  // 4 kv heads of 32 dims, 4 query heads each, over 2000 keys 76 and 62; 32 x 70 of 7B-like heads 193 and 178; 64
  // dims: 64 x 65 of 1.1B-like heads over 4000 209 and 251, its registers spill).
  const long groups = (long)n_kv_heads * batch, at_once = groups * ((nq + 4 * rows - 1) / (4 * rows));
  const long live = groups * ((nq + rows - 1) / rows);
  p.line = prefix ? at_once >= slots
                  : groups * nq >= slots * rows &&
                        (nb <= 32 || (head_dim != 64 && live >= 3 * slots && live >= 3 * at_once));
  p.n_tiles = (nq + (p.line ? 4 : 1) * rows - 1) / ((p.line ? 4 : 1) * rows);
  const long units = (long)n_kv_heads * p.n_tiles * batch, all = prefix ? std::max(1L, slots / units) : 1;
  const long per = std::max({(nb + all - 1) / all, (nb + kPartsMax8 - 1) / kPartsMax8, 4L});
  p.per = (int)(prefix ? per : nb);
  p.nwg = (int)((nb + p.per - 1) / p.per);
  p.parts = (int)std::min<long>({nb, all, (long)kPartsMax8});
  return p;
}

// Whether own texts of bf16 rows are wide_kernel's, which is faster at full tiles but does not cut keys, or attn8_kernel's:
// where tiles full of rows would fill a seventh of the card (wide_kernel and attn8_kernel, us: 7B-like, 2 x 40 rows over
// 8000 keys 56 and 72, 32 x 40 over 16000 776 and 2094; 1.1B-like, 16 x 9 over 8000 60 and 53, 16 x 3 56 and 26), or,
// more than 64 rows, at most 128 chunks (4 x 20 rows of 1.1B-like heads: over 2000 keys 20 and 25, 4000 30 and 26, 8000
// 55 and 33; one sequence of 70 7B-like: 4000 33 and 39, 16000 99 and 81).  One sequence of 5 rows, 1.1B-like, over
// 8000 keys: 47 and 13.  The choice is up to a quarter slower than the other near its borders.
bool wide_takes(int rps, int batch, int n_heads, int n_kv_heads, int head_dim, int max_ctx) {
  const int nq = rps * (n_heads / n_kv_heads), nb = (max_ctx + kF8Sub - 1) / kF8Sub;
  if (!is_wide(nq)) return false;
  const int64_t slots = 2L * device_compute_units();
  return 7 * (int64_t)n_kv_heads * batch * nq >= slots * 16 * wide_tiles(head_dim) || (nq > 64 && nb <= 128);
}

template <class X>
hipError_t launch_wide(const AttnArgs& a, const Plan& p, int B, const X& x, hipStream_t s) {
  const dim3 grid(p.nwg, (unsigned)(a.n_kv_heads * p.n_tiles), B);
#define SD_WIDE(HD, KW) \
  hipLaunchKernelGGL((wide_kernel<HD, wide_tiles(HD), KW, X>), grid, dim3(256), 0, s, a, p.n_tiles, p.parts, p.per, x)
#define SD_WIDE_HD(HD)          \
  if (p.line) SD_WIDE(HD, 1);   \
  else SD_WIDE(HD, 4);
  switch (a.head_dim) {
    case 32: SD_WIDE_HD(32) break;
    case 64: SD_WIDE_HD(64) break;
    case 128: SD_WIDE_HD(128) break;
    default: return hipErrorInvalidValue;
  }
#undef SD_WIDE_HD
#undef SD_WIDE
  return hipGetLastError();
}

// float32 queries: two tiles a wave from 17 rows on where the codes' second reading would count (32 rows of
// 7B-like heads over 65536 keys 112 us, 183 with one; over 8192 32 both; over 4000 27 and 24).
Plan prefix_plan(int rows, int n_heads, int n_kv_heads, int head_dim, int max_len, bool bf16) {
  const int nq = rows * (n_heads / n_kv_heads);
  if (bf16 && is_wide(nq)) return wide_plan(rows, 1, n_heads, n_kv_heads, head_dim, max_len, true);
  return plan_of(rows, 1, n_heads, n_kv_heads, head_dim, max_len, nq > 64 || (nq > 16 && max_len > 8192) ? 2 : 1);
}

template <typename T>
hipError_t launch_typed(AttnArgs own, const SharedAttn& sh, hipStream_t s) {
  SharedParts parts{sh.o, sh.ml, sh.prefix.len + sh.b, sh.max_len, 1, 1};
  if (sh.max_len > 0) {
    AttnArgs a = own;
    a.f8 = sh.prefix;
    a.rps = own.M;
    a.max_ctx = sh.max_len;
    a.o_part = sh.o;
    a.ml_part = sh.ml;
    const bool wide = sh.bf16 && is_wide(a.rps * (a.n_heads / a.n_kv_heads));
    const Plan p = prefix_plan(a.rps, a.n_heads, a.n_kv_heads, a.head_dim, a.max_ctx, sh.bf16);
    if (p.parts > sh.parts) return hipErrorInvalidValue;  // (the caller has checked)
    parts.keys = p.per * (wide ? kF8Sub : chunk_of(a.head_dim));
    parts.stride = p.parts;
    hipError_t e;
    if constexpr (sizeof(T) == 2) e = wide ? launch_wide(a, p, 1, PrefixPass<T>{sh.b}, s) : launch_plan(a, p, 1, PrefixPass<T>{sh.b}, s);
    else e = launch_plan(a, p, 1, PrefixPass<T>{sh.b}, s);
    if (e != hipSuccess) return e;
  }
  const int B = own.M / own.rps;
  const int nw = own_waves(own.rps, B, own.n_heads, own.n_kv_heads, own.head_dim, own.max_ctx);
  if (nw > 0) return launch_own<T>(own, parts, nw, s);
  if constexpr (sizeof(T) == 2) {
    if (wide_takes(own.rps, B, own.n_heads, own.n_kv_heads, own.head_dim, own.max_ctx)) {
      const Plan p = wide_plan(own.rps, B, own.n_heads, own.n_kv_heads, own.head_dim, own.max_ctx, false);
      return launch_wide(own, p, B, OwnPass<T>{parts}, s);
    }
  }
  const Plan p = plan_of(own.rps, B, own.n_heads, own.n_kv_heads, own.head_dim, own.max_ctx);
  if (p.parts > own.n_split) return hipErrorInvalidValue;
  return launch_plan(own, p, B, OwnPass<T>{parts}, s);
}

}  // namespace

bool attention_shared_fits(int64_t rows, int n_heads, int n_kv_heads) {
  // (rows of a kv head are numbered below 2^20, see div_small)
  return rows * (n_heads / n_kv_heads) < 1 << 20 && attention8_fits((int)rows, 1, n_heads, n_kv_heads);
}

int attention_shared_parts(int rows, int n_heads, int n_kv_heads, int head_dim, int max_len, bool bf16) {
  return prefix_plan(rows, n_heads, n_kv_heads, head_dim, max_len, bf16).parts;
}

hipError_t launch_attention_shared(const AttnArgs& own, const SharedAttn& sh, hipStream_t s) {
  return sh.bf16 ? launch_typed<uint16_t>(own, sh, s) : launch_typed<float>(own, sh, s);
}

}  // namespace specdec
