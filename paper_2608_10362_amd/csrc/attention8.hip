// GQA attention over the FP8 cache (layout: internal.h).
//
// o = softmax(q K^T / sqrt(hd)) V for the newest rows of every sequence, query
// i of a sequence at position pos_i seeing keys 0 .. pos_i.  One pass over the
// keys with a running maximum and sum per query.
//
// The scores are taken as K Q^T: D[4 (l/16) + r][l % 16] is a key row and a
// query column, so a lane holds scores of one query, and with the K rows in the
// cache's order lane group c holds positions 8c .. 8c+7 of a 32-position step,
// the k order of V: the probabilities feed O^T = V^T P^T from the registers
// they were made in, and no value crosses lanes but the row maximum.  Codes
// become bf16 by v_cvt_scalef32_pk_bf16_fp8 (exact); queries and probabilities
// are split into hi + lo bf16 parts (the result is float32: a bf16 probability
// alone would be off by 2^-9), so each product runs twice.
#include <algorithm>

#include "device_common.h"
#include "fp8.h"
#include "internal.h"

namespace specdec {

namespace {

constexpr int kWaves8 = 4;      // per workgroup, each on a 64-position block of its own
constexpr int kPartsMax8 = 64;  // parts of one unit (one per lane of the combining wave)

__device__ __forceinline__ void split8(const float (&v)[8], bf16x8& hi, bf16x8& lo) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const __bf16 h = (__bf16)v[j];
    hi[j] = h;
    lo[j] = (__bf16)(v[j] - (float)h);
  }
}

__device__ __forceinline__ RowDesc row_of(const AttnArgs& a, int r) {
  if (a.rows) return a.rows[r];
  const int b = r / a.rps;
  return RowDesc{b, a.f8.len[b] + r % a.rps, 0, 1};
}
// Blocks of 64 positions sequence b's rows see (its last row bounds them; the
// host's count where that row is invalid).
__device__ __forceinline__ int blocks_of(const AttnArgs& a, int b) {
  const RowDesc last = row_of(a, b * a.rps + a.rps - 1);
  const int most = (a.max_ctx + kF8Block - 1) / kF8Block;
  return last.valid ? max(1, min(most, last.pos / kF8Block + 1)) : most;
}

// The work is a line: sequence by sequence, unit by unit (kv head, query tile),
// block by block; workgroup i takes blocks [i * per, (i + 1) * per).
struct Line {
  int total, per;
};
__device__ __forceinline__ int lane_sum(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ Line line_of(const AttnArgs& a, int B, int U, int nwg, int n0) {
  const int lane = threadIdx.x & 63;
  int t = 0;
  for (int c = 0; c < B; c += kWave) t += lane_sum(c == 0 ? n0 : (c + lane < B ? blocks_of(a, c + lane) : 0));
  const int most = (a.max_ctx + kF8Block - 1) / kF8Block;
  Line l;
  l.total = t * U;
  l.per = max((l.total + nwg - 1) / nwg, (most + kPartsMax8 - 3) / (kPartsMax8 - 2));
  return l;
}
// Blocks before sequence b on the line of one unit.
__device__ __forceinline__ int before_of(const AttnArgs& a, int b, int n0) {
  const int lane = threadIdx.x & 63;
  int t = 0;
  for (int c = 0; c < b; c += kWave) t += lane_sum(c + lane >= b ? 0 : (c == 0 ? n0 : blocks_of(a, c + lane)));
  return t;
}

__device__ __forceinline__ void put_row(const AttnArgs& a, int row, int head, int d, float v) {
  if (a.xs) put_stacked(a.xs, a.stt, row, head * a.head_dim + d, v);
  else a.o[((size_t)row * a.n_heads + head) * a.head_dim + d] = v;
}

template <int HD, int QT>
__global__ __launch_bounds__(64 * kWaves8, QT > 2 ? 1 : 2) void attn8_kernel(AttnArgs a, int n_tiles, int parts) {
  constexpr int KST = HD / 32, DT = HD / 16, F = HD / 16, OS = HD + 4, NW = kWaves8;
  __shared__ float s_o[NW][16][OS];
  __shared__ float s_ml[NW][16][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, grp = lane >> 4;
  const int H = a.n_heads, G = a.n_kv_heads, group = H / G, rps = a.rps, nq = rps * group, B = a.M / rps;
  const int U = G * n_tiles, window = a.f8.ring.capacity;
  const int n0 = lane < B ? blocks_of(a, lane) : 0;  // (the first 64 sequences stay in a register)
  const Line ln = line_of(a, B, U, (int)gridDim.x, n0);
  auto blocks = [&](int s) { return s < kWave ? __builtin_amdgcn_readlane(n0, s) : blocks_of(a, s); };
  int x = (int)blockIdx.x * ln.per;
  const int hi = min(ln.total, x + ln.per);
  const float qscale = 1.44269504088896341f / sqrtf((float)HD);  // (scores in powers of two)

  int b = 0, base = 0, nb = blocks(0);  // the sequence that holds x; base: the line where it starts
  while (x < hi) {
    while (x >= base + nb * U) {
      base += nb * U;
      ++b;
      nb = blocks(b);
    }
    const int u = (x - base) / nb, k_lo = (x - base) % nb, k_hi = min(nb, k_lo + (hi - x));
    const int unit0 = base + u * nb;  // the line where the unit starts
    const int g = u / n_tiles, tile = u % n_tiles;
    x += k_hi - k_lo;
    const int sealed = (a.f8.len[b] + a.c0) / kF8Block;

    // This lane's query of each tile, its position, and the tiles' position range.
    int qpos[QT];
    bf16x8 qhi[QT][KST], qlo[QT][KST];
    int vis = 0, lowest = 0x7fffffff;
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      const int qa = (tile * QT + q) * 16 + c16;
      const bool in = qa < nq;
      const int row = b * rps + (in ? qa / group : 0), head = g * group + (in ? qa % group : 0);
      const RowDesc rd = row_of(a, row);
      qpos[q] = in && rd.valid ? rd.pos : -1;
      if (qpos[q] >= 0) {
        vis = max(vis, qpos[q] + 1);
        lowest = min(lowest, qpos[q]);
      }
      const float* qp = a.qr + ((size_t)row * H + head) * HD;
#pragma unroll
      for (int s = 0; s < KST; ++s) {
        const int d = HD >= 64 ? 64 * (s >> 1) + 16 * grp + 8 * (s & 1) : 32 * s + 8 * grp;
        const f32x4 v0 = *(const f32x4_a4*)(qp + d), v1 = *(const f32x4_a4*)(qp + d + 4);
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[j] = in ? v0[j] * qscale : 0.f;
          v[4 + j] = in ? v1[j] * qscale : 0.f;
        }
        split8(v, qhi[q][s], qlo[q][s]);
      }
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      vis = max(vis, __shfl_xor(vis, o, kWave));
      lowest = min(lowest, __shfl_xor(lowest, o, kWave));
    }
    vis = __builtin_amdgcn_readfirstlane(vis);
    lowest = __builtin_amdgcn_readfirstlane(lowest);

    floatx4 of[QT][DT];
    float mx[QT], sm[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      mx[q] = -INFINITY;
      sm[q] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) of[q][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    // New scores of tile q: the running maximum and sum,
    // then the scores become probabilities relative to it.
    auto softmax = [&](int q, auto& p) {
      constexpr int n = sizeof(p) / sizeof(float);
      float m = p[0];
#pragma unroll
      for (int j = 1; j < n; ++j) m = fmaxf(m, p[j]);
      m = fmaxf(m, __shfl_xor(m, 16, kWave));
      m = fmaxf(m, __shfl_xor(m, 32, kWave));
      const float mnew = fmaxf(mx[q], m);
      if (__any(mnew > mx[q])) {  // (rescaled only where a maximum rose)
        const float alpha = mx[q] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx[q] - mnew);
        sm[q] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) of[q][dt] *= alpha;
        mx[q] = mnew;
      }
#pragma unroll
      for (int j = 0; j < n; ++j) {
        // (a query that has seen no key yet keeps the maximum -inf)
        p[j] = mx[q] == -INFINITY && p[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(p[j] - mx[q]);
        sm[q] += p[j];
      }
    };

    for (int kb = k_lo + wave; kb < k_hi; kb += NW) {  // (wave-uniform)
      if (kb < sealed) {  // codes: every query sees the whole block
        const unsigned char* codes = a.f8.code_base(a.layer, b, g) + (size_t)kb * 2 * kF8Block * HD + lane * 16;
        const float* sc = a.f8.scale_base(a.layer, b, g) + 2 * (size_t)kb;
        u32x4 kc[F], vc[F];
#pragma unroll
        for (int f = 0; f < F; ++f) kc[f] = *(const u32x4*)(codes + f * 1024);
#pragma unroll
        for (int f = 0; f < F; ++f) vc[f] = *(const u32x4*)(codes + kF8Block * HD + f * 1024);
        const float ks = sc[0], vs = sc[1];
        float p[QT][16];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            floatx4 acc[QT];
#pragma unroll
            for (int q = 0; q < QT; ++q) acc[q] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < KST; ++st) {
              bf16x8 kk;
              if constexpr (HD >= 64) {
                const u32x4 w = kc[(2 * s + t) * (HD / 64) + st / 2];
                kk = fp8x8_to_bf16(w[2 * (st & 1)], w[2 * (st & 1) + 1], ks);
              } else {
                kk = fp8x8_to_bf16(kc[s][2 * t], kc[s][2 * t + 1], ks);
              }
#pragma unroll
              for (int q = 0; q < QT; ++q) {
                acc[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qhi[q][st], acc[q], 0, 0, 0);
                acc[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qlo[q][st], acc[q], 0, 0, 0);
              }
            }
#pragma unroll
            for (int q = 0; q < QT; ++q)
#pragma unroll
              for (int r = 0; r < 4; ++r) p[q][8 * s + 4 * t + r] = acc[q][r];
          }
        bf16x8 phi[QT][2], plo[QT][2];
#pragma unroll
        for (int q = 0; q < QT; ++q) {
          softmax(q, p[q]);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p[q][8 * s + j];
            split8(v, phi[q][s], plo[q][s]);
          }
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const bf16x8 vv = fp8x8_to_bf16(vc[dt][2 * s], vc[dt][2 * s + 1], vs);
#pragma unroll
            for (int q = 0; q < QT; ++q) {
              of[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, phi[q][s], of[q][dt], 0, 0, 0);
              of[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, plo[q][s], of[q][dt], 0, 0, 0);
            }
          }
      } else {  // the ring, 32 positions at a time
        const uint16_t* kr = k_block<uint16_t>(a.f8.ring, a.layer, b, g);
        for (int s = 0; s < 2; ++s) {
          const int k0 = kb * kF8Block + 32 * s, w0 = k0 % window;
          if (k0 >= vis) break;
          u32x4 vf[DT];
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
            vf[dt] = *(const u32x4*)(kr + KvIndex<uint16_t>::v(w0 + 8 * grp, 16 * dt + c16, HD, window));
          float p[QT][8];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            floatx4 acc[QT];
#pragma unroll
            for (int q = 0; q < QT; ++q) acc[q] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < KST; ++st) {
              const int d = HD >= 64 ? 64 * (st >> 1) + 16 * grp + 8 * (st & 1) : 32 * st + 8 * grp;
              const int pos = w0 + 8 * (c16 >> 2) + 4 * t + (c16 & 3);
              const bf16x8 kk = __builtin_bit_cast(bf16x8, *(const u32x4*)(kr + KvIndex<uint16_t>::k(pos, d, HD, window)));
#pragma unroll
              for (int q = 0; q < QT; ++q) {
                acc[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qhi[q][st], acc[q], 0, 0, 0);
                acc[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qlo[q][st], acc[q], 0, 0, 0);
              }
            }
#pragma unroll
            for (int q = 0; q < QT; ++q)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                p[q][4 * t + r] = k0 + 8 * grp + 4 * t + r > qpos[q] ? -INFINITY : acc[q][r];
          }
          // Slots past the newest visible position hold stale values: their V
          // entries are zeroed, never multiplied by a zero probability.
          const int nvalid = vis - (k0 + 8 * grp);
          bool odd = false;  // a NaN or infinity among the V entries
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              if (2 * w >= nvalid) vf[dt][w] = 0u;
              else if (2 * w + 1 >= nvalid) vf[dt][w] &= 0xffffu;
              odd |= (vf[dt][w] & 0x7f80u) == 0x7f80u || (vf[dt][w] & 0x7f800000u) == 0x7f800000u;
            }
          // One that only later rows see must not reach the others through
          // 0 * inf: such entries leave the product and are added by themselves
          // to the queries that see them.
          const bool apart = k0 + 31 > lowest && __any(odd);
          if (apart) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                if ((vf[dt][w] & 0x7f80u) == 0x7f80u) vf[dt][w] &= 0xffff0000u;
                if ((vf[dt][w] & 0x7f800000u) == 0x7f800000u) vf[dt][w] &= 0xffffu;
              }
          }
#pragma unroll
          for (int q = 0; q < QT; ++q) {
            softmax(q, p[q]);
            bf16x8 phi, plo;
            split8(p[q], phi, plo);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              const bf16x8 vv = __builtin_bit_cast(bf16x8, vf[dt]);
              of[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, phi, of[q][dt], 0, 0, 0);
              of[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, plo, of[q][dt], 0, 0, 0);
            }
            if (apart) {
              for (int j = 0; j < 32; ++j) {  // (position k0 + j; its probability lies in lane group j / 8)
                float pj = 0.f;
#pragma unroll
                for (int t = 0; t < 8; ++t) pj = (j & 7) == t ? p[q][t] : pj;
                pj = __shfl(pj, 16 * (j >> 3) + c16, kWave);
                if (k0 + j > qpos[q]) continue;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                  for (int r = 0; r < 4; ++r) {
                    const float v = bf16_bits_to_f32(kr[KvIndex<uint16_t>::v(w0 + j, 16 * dt + 4 * grp + r, HD, window)]);
                    if (!isfinite(v)) of[q][dt][r] += pj * v;
                  }
              }
            }
          }
        }
      }
    }

    // Merge the waves of this segment, tile by tile, in LDS (fixed order).
    const bool whole = k_lo == 0 && k_hi == nb;
    const int part = (int)blockIdx.x - unit0 / ln.per;
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      const int n_here = min(16, nq - (tile * QT + q) * 16);
      if (n_here <= 0) break;
      float sum = sm[q];
      sum += __shfl_xor(sum, 16, kWave);
      sum += __shfl_xor(sum, 32, kWave);
      __syncthreads();  // (the tile or segment before is read out)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *(floatx4*)&s_o[wave][c16][16 * dt + 4 * grp] = of[q][dt];
      if (grp == 0) {
        s_ml[wave][c16][0] = mx[q];
        s_ml[wave][c16][1] = sum;
      }
      __syncthreads();
      for (int i = wave; i < n_here; i += NW) {
        float M = -INFINITY, L = 0.f, e[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, s_ml[w][i][0]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          // (a wave without keys: maximum -inf, sum and outputs 0; NaN scores leave the maximum -inf but a NaN sum)
          const float m = s_ml[w][i][0], l = s_ml[w][i][1];
          e[w] = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - M);
          L += e[w] * l;
        }
        const int qa = (tile * QT + q) * 16 + i, row = b * rps + qa / group, head = g * group + qa % group;
        const RowDesc rd = row_of(a, row);
        if (rd.valid && rd.pos + 1 > a.max_ctx && lane == 0) set_status(a.status, kStatusKvCapacity);  // the host's bound was wrong
        const size_t slot = ((size_t)row * H + head) * parts + part;
        for (int d = lane; d < HD; d += kWave) {
          float o = 0.f;
#pragma unroll
          for (int w = 0; w < NW; ++w) o += e[w] * s_o[w][i][d];
          if (whole) put_row(a, row, head, d, rd.valid ? o / L : 0.f);
          else a.o_part[slot * HD + d] = o;
        }
        if (!whole && lane == 0) {
          a.ml_part[2 * slot] = M;
          a.ml_part[2 * slot + 1] = L;
        }
      }
    }
  }
}

// Grid (heads, rows), one wave: adds the parts of a (row, head) whose unit
// spans workgroups.
template <int HD>
__global__ __launch_bounds__(64) void attn8_combine_kernel(AttnArgs a, int n_tiles, int qt, int parts, int nwg) {
  const int head = blockIdx.x, row = blockIdx.y, lane = threadIdx.x;
  const int H = a.n_heads, G = a.n_kv_heads, group = H / G, rps = a.rps, B = a.M / rps, b = row / rps;
  const int n0 = lane < B ? blocks_of(a, lane) : 0;
  const Line ln = line_of(a, B, G * n_tiles, nwg, n0);
  const int nb = b < kWave ? __builtin_amdgcn_readlane(n0, b) : blocks_of(a, b), tile = ((row % rps) * group + head % group) / (16 * qt);
  const int unit0 = before_of(a, b, n0) * G * n_tiles + ((head / group) * n_tiles + tile) * nb;
  const int first = unit0 / ln.per, n = (unit0 + nb - 1) / ln.per - first + 1;
  if (n == 1) return;  // (finished by its workgroup)
  const RowDesc rd = row_of(a, row);
  const size_t slot = ((size_t)row * H + head) * parts;
  const float m = lane < n ? a.ml_part[2 * (slot + lane)] : -INFINITY, l = lane < n ? a.ml_part[2 * (slot + lane) + 1] : 0.f;
  const float M = wave_max(m);
  const float e = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - M);
  const float inv = 1.0f / wave_sum(e * l);
  constexpr int DPL = HD >= 64 ? HD / 64 : 1;
  float acc[DPL] = {};
  for (int p = 0; p < n; ++p) {
    const float w = __shfl(e, p, kWave);
#pragma unroll
    for (int j = 0; j < DPL; ++j)
      if (lane + 64 * j < HD) acc[j] += w * a.o_part[(slot + p) * HD + lane + 64 * j];
  }
#pragma unroll
  for (int j = 0; j < DPL; ++j)
    if (lane + 64 * j < HD) put_row(a, row, head, lane + 64 * j, rd.valid ? acc[j] * inv : 0.f);
}

// Query tiles of 16 a wave takes at once (they share a block's codes).
int query_tiles(int nq) { return nq <= 16 ? 1 : (nq <= 32 ? 2 : 4); }

struct Plan {
  int qt, n_tiles, nwg, parts;
};
Plan plan_of(int rps, int batch, int n_heads, int n_kv_heads, int max_ctx) {
  Plan p;
  const int nq = rps * (n_heads / n_kv_heads);
  p.qt = query_tiles(nq);
  p.n_tiles = (nq + 16 * p.qt - 1) / (16 * p.qt);
  const long nb = (max_ctx + kF8Block - 1) / kF8Block, units = (long)n_kv_heads * p.n_tiles;
  const long most = nb * units * batch;
  // one block a wave until the card is full, then 2 workgroups a CU
  p.nwg = (int)std::max(1L, std::min((most + kWaves8 - 1) / kWaves8, 2L * device_compute_units()));
  // a unit of the longest sequence spans at most this many workgroups, whatever the other lengths
  p.parts = (int)std::min<long>({nb, p.nwg / units + 2, (long)kPartsMax8});
  return p;
}

}  // namespace

int attention8_parts(int rps, int batch, int n_heads, int n_kv_heads, int max_ctx) {
  return plan_of(rps, batch, n_heads, n_kv_heads, max_ctx).parts;
}

hipError_t launch_attention8(const AttnArgs& a, hipStream_t s) {
  const int B = a.M / a.rps;
  const Plan p = plan_of(a.rps, B, a.n_heads, a.n_kv_heads, a.max_ctx);
  if (p.parts > a.n_split || (a.max_ctx + kF8Block - 1L) / kF8Block * a.n_kv_heads * p.n_tiles * B > 1L << 30)
    return hipErrorInvalidValue;
#define SD_A8(HDV)                                                                                              \
  {                                                                                                             \
    if (p.qt == 1) hipLaunchKernelGGL((attn8_kernel<HDV, 1>), dim3(p.nwg), dim3(64 * kWaves8), 0, s, a, p.n_tiles, p.parts); \
    else if (p.qt == 2) hipLaunchKernelGGL((attn8_kernel<HDV, 2>), dim3(p.nwg), dim3(64 * kWaves8), 0, s, a, p.n_tiles, p.parts); \
    else hipLaunchKernelGGL((attn8_kernel<HDV, 4>), dim3(p.nwg), dim3(64 * kWaves8), 0, s, a, p.n_tiles, p.parts); \
    hipLaunchKernelGGL((attn8_combine_kernel<HDV>), dim3(a.n_heads, a.M), dim3(64), 0, s, a, p.n_tiles, p.qt, p.parts, p.nwg); \
  }
  switch (a.head_dim) {
    case 32: SD_A8(32) break;
    case 64: SD_A8(64) break;
    case 128: SD_A8(128) break;
    default: return hipErrorInvalidValue;
  }
#undef SD_A8
  return hipGetLastError();
}

}  // namespace specdec
