// Attention of a batch whose sequences begin with the same text, held once as a sequence of an FP8
// cache of its own.
//
// The softmax over a row's keys is taken in two sets, the prefix's and the row's own:
// with (M, L, O) the maximum, the sum of exp(s - M) and the sum of those times the
// values of each set, the result is sum_i e^(M_i - M) O_i / sum_i e^(M_i - M) L_i.
// First launch: all rows of the batch against the prefix as if they were one sequence's,
// split over its keys, (M, L, O) of every part to the workspace; second launch: every
// sequence's rows over its own cache, which joins the parts as it finishes a row.
// The prefix's codes are read once for 16 or 32 rows of a kv head, not once a sequence.
#include "attention8.h"

namespace specdec {

namespace {

// ---------------------------------------------------------------- few rows over short texts
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

template <int HD, typename T, int NW>
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

  // Codes: loads past the sealed ones read nothing.
  const __amdgpu_buffer_rsrc_t cr = make_rsrc(a.f8.code_base(a.layer, b, g), (uint32_t)j_sealed * SP * 2 * kF8Sub * HD);
  const __amdgpu_buffer_rsrc_t sr = make_rsrc(a.f8.scale_base(a.layer, b, g), (uint32_t)((j_sealed * SP + 1) & ~1) * 4);
  u32x4 kc[SP][FS], vc[SP][FS];
  float ks, vs;
  auto load_codes = [&](int j) {
    const uint32_t at = (uint32_t)j * SP * 2 * kF8Sub * HD + lane * 16;
#pragma unroll
    for (int i = 0; i < SP * FS; ++i) {
      const uint32_t k = at + i / FS * 2 * kF8Sub * HD + i % FS * 1024;
      kc[i / FS][i % FS] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(cr, k, 0, 0));
      vc[i / FS][i % FS] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(cr, k + kF8Sub * HD, 0, 0));
    }
    ks = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sr, (j * SP & ~1) * 4, 0, 0));
    vs = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sr, (j * SP | 1) * 4, 0, 0));
  };
  const uint16_t* ring = k_block<uint16_t>(a.f8.ring, a.layer, b, g);
  const __amdgpu_buffer_rsrc_t rr = make_rsrc(ring, (uint32_t)window * HD * 4u);
  u32x4 rk[2 * KST], rv[DT];
  auto load_ring = [&](int sub) {
    const int w0 = sub * kF8Sub % window;
#pragma unroll
    for (int i = 0; i < 2 * KST; ++i) {
      const int t = i / KST, s = i % KST, d = HD >= 64 ? 64 * (s >> 1) + 16 * grp + 8 * (s & 1) : 32 * s + 8 * grp;
      const int pos = w0 + 8 * (c16 >> 2) + 4 * t + (c16 & 3);
      rk[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                            rr, (uint32_t)KvIndex<uint16_t>::k(pos, d, HD, window) * 2u, 0, 0));
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      rv[dt] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                   rr, (uint32_t)KvIndex<uint16_t>::v(w0 + 8 * grp, 16 * dt + c16, HD, window) * 2u, 0, 0));
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
  for (int p = wave; p < n_pre; p += NW) {
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

// Waves of a unit: a wave a unit where the card is full of them, else as many as
// fill it; 0: attn8_kernel, whose units are split over workgroups.
int own_waves(int rps, int batch, int n_heads, int n_kv_heads, int head_dim, int max_ctx) {
  const int nq = rps * (n_heads / n_kv_heads);
  if (nq > 64) return 0;
  const int64_t units = (int64_t)batch * n_kv_heads * ((nq + 15) / 16), slots = 4L * own_resident(head_dim) * device_compute_units();
  const int nb = (max_ctx + chunk_of(head_dim) - 1) / chunk_of(head_dim);
  int nw = 8;
  while (nw > 1 && (units * nw > slots || nw > nb)) nw /= 2;
  return nb <= 32 * nw && units < 1 << 24 ? nw : 0;
}

template <typename T>
hipError_t launch_own(const AttnArgs& a, const SharedParts& pre, int nw, hipStream_t s) {
  const int nq = a.rps * (a.n_heads / a.n_kv_heads), n_tiles = (nq + 15) / 16;
  const dim3 grid((unsigned)(a.M / a.rps) * a.n_kv_heads * n_tiles);
#define SD_OWN(HD, NW) hipLaunchKernelGGL((own_kernel<HD, T, NW>), grid, dim3(64 * NW), 0, s, a, pre, n_tiles)
#define SD_OWN_HD(HD)                  \
  switch (nw) {                        \
    case 1: SD_OWN(HD, 1); break;      \
    case 2: SD_OWN(HD, 2); break;      \
    case 4: SD_OWN(HD, 4); break;      \
    default: SD_OWN(HD, 8); break;     \
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
    const Plan p = plan_of(a.rps, 1, a.n_heads, a.n_kv_heads, a.head_dim, a.max_ctx);
    if (p.parts > sh.parts) return hipErrorInvalidValue;  // (the caller has checked)
    parts.keys = p.per * chunk_of(a.head_dim);
    parts.stride = p.parts;
    const hipError_t e = launch_plan(a, p, 1, PrefixPass<T>{sh.b}, s);
    if (e != hipSuccess) return e;
  }
  const int B = own.M / own.rps;
  const int nw = own_waves(own.rps, B, own.n_heads, own.n_kv_heads, own.head_dim, own.max_ctx);
  if (nw > 0) return launch_own<T>(own, parts, nw, s);
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
  return plan_of(rows, 1, n_heads, n_kv_heads, head_dim, max_len).parts;
}

hipError_t launch_attention_shared(const AttnArgs& own, const SharedAttn& sh, hipStream_t s) {
  return sh.bf16 ? launch_typed<uint16_t>(own, sh, s) : launch_typed<float>(own, sh, s);
}

}  // namespace specdec
