// GQA attention over the FP8 cache (layout: internal.h).
//
// o = softmax(q K^T / sqrt(hd)) V for the newest rows of every sequence, query
// i of a sequence at position pos_i seeing keys 0 .. pos_i.  One pass over the
// keys with a running maximum and sum per query.
//
// The scores are taken as K Q^T: D[4 (l/16) + r][l % 16] is a key row and a
// query column, so a lane holds scores of one query, and with the K rows in the
// cache's order lane group c holds positions 8c .. 8c+7 of 32, the k order of V:
// the probabilities feed O^T = V^T P^T from the registers they were made in,
// and no value crosses lanes but the row maximum.  Queries and probabilities are
// float32 and enter their products in parts, so that the result is as good as a
// float32 computation's (3e-7 of it against 1e-6 for the plain form, 7B-like):
//  - one query tile a wave (at most 64 rows a kv head): codes as bf16, times their
//    scale (exact), three bf16 parts, which hold a float32 whole (two leave up to
//    2^-17 of it, 3.5e-6 of the result over 2048 keys; one up to 2^-8).  The products
//    are few and the stream of codes is the bound;
//  - two tiles: codes as fp16 (exact), two fp16 parts (up to 2^-23 left) of the query
//    row times a power of two that brings its largest to 2^13 (parts far below lose
//    bits no float32 sum holds), and of 2^15 p.  K's scale multiplies the scores, V's goes
//    into the conversion where the values are fp16's and into the sums where not.
//    56 -> 49 us against three bf16 parts, which the ring's rows, bf16 values, still take.
//
// Work: a unit is a kv head and a query tile of a sequence; its keys come in chunks of
// 32 or 64, and a workgroup takes a range of them, its NW waves every NW-th.  Each
// wave keeps (max, sum, O) of its own, then they merge in LDS.  A unit inside one
// workgroup is finished there; otherwise each stores its part and the last to count
// itself adds the parts.  Ragged batches of few rows, with more than four chunks a wave,
// put all units' chunks on a line, and workgroup i takes the i-th `per` of them: all stream
// the same bytes whatever the lengths.  Other calls have a workgroup per range.
//
// Measured.  7B-like (32 kv heads of 128): one row over 2048 keys 9.8 us (a chain of
// start 3, codes and products 3, merge 1.5, parts 2.5); 16 ragged rows over 1024 to
// 8191 keys 112 us, 5.4 TB/s of codes (99 us, 6.1 TB/s, where all are 4607 long and
// no unit is cut; a read of as many bytes takes 94); 512 rows over 2048 keys 42 us,
// 358 TFLOP/s of the operator's products, twice that in the matrix unit (half the
// time is conversions and softmax, which its products do not hide, a quarter the
// ring's rows).  1.1B-like (4 kv heads of 64, 8 query heads each): one row over
// 131072 keys 20.7 us, 3.2 TB/s (14 us of stream; 61 parts of one unit by one
// workgroup 5 us), 4 x 5 rows over 301 to 1028 keys 9.8 us, 8 x 5 rows over 8192
// keys 23 us, 1.4 TB/s (each of a kv head's three query tiles reads its codes).
#include <algorithm>

#include "device_common.h"
#include "fp8.h"
#include "gemm_common.h"
#include "internal.h"

namespace specdec {

namespace {

constexpr float kLeast = -3.4028234663852886e38f;  // the least finite float32
constexpr int kPartsMax8 = 64;  // parts of one unit (one per lane of the combining wave)
// Sub-chunks of 32 keys a wave takes at a time, its chunk: 8 KB of codes for 128
// dims as for 64.
__host__ __device__ constexpr int steps_of(int head_dim) { return head_dim == 128 ? 1 : 2; }
__host__ __device__ constexpr int chunk_of(int head_dim) { return kF8Sub * steps_of(head_dim); }

// v as a sum of three bf16 values, each of what the ones before leave (exact: 24 bits
// in three times 8 and two signs).
__device__ __forceinline__ void split8(const float (&v)[8], bf16x8 (&part)[3]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const __bf16 h = (__bf16)v[j];
    const float r = v[j] - (float)h;
    const __bf16 m = (__bf16)r;
    part[0][j] = h;
    part[1][j] = m;
    part[2][j] = (__bf16)(r - (float)m);
  }
}

// v as a sum of two fp16 values (of 24 bits the last may be off: 11 each and a sign).
__device__ __forceinline__ void split8(const float (&v)[8], f16x8 (&part)[2]) {
  u32x4 h, l;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    h[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2 * j], v[2 * j + 1]}, f16x2));
    float r0, r1;  // v - h (exact) without a conversion of h
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r0) : "v"(h[j]), "v"(v[2 * j]));
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r1) : "v"(h[j]), "v"(v[2 * j + 1]));
    l[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{r0, r1}, f16x2));
  }
  part[0] = __builtin_bit_cast(f16x8, h);
  part[1] = __builtin_bit_cast(f16x8, l);
}

// Exponent that brings a query row, whose largest |x| has the bits m, to [2^13, 2^14).
__device__ __forceinline__ int row_shift(uint32_t m) {
  return m == 0u || m >= 0x7f800000u ? 0 : min(100, 13 + 127 - (int)(m >> 23));
}
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// Maximum over the four lane groups of 16 (the same query).
__device__ __forceinline__ float groups_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const float m = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Row i of sequence b.
__device__ __forceinline__ RowDesc row_of(const AttnArgs& a, int b, int i) {
  if (a.rows) return a.rows[b * a.rps + i];
  return RowDesc{b, a.f8.len[b] + i, 0, 1};
}
// Chunks sequence b's rows see (its last row bounds them; the host's count
// where that row is invalid).
template <int C>
__device__ __forceinline__ int chunks_of(const AttnArgs& a, int b) {
  const RowDesc last = row_of(a, b, a.rps - 1);
  const int most = (a.max_ctx + C - 1) / C;
  return last.valid ? max(1, min(most, last.pos / C + 1)) : most;
}

__device__ __forceinline__ int lane_sum(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return __builtin_amdgcn_readfirstlane(v);
}

// Agent-scope accesses of the parts: visible to a combining workgroup on any XCD
// once completed.
__device__ __forceinline__ void put2(float* p, float x, float y) {
  __hip_atomic_store((unsigned long long*)p, ((unsigned long long)__float_as_uint(y) << 32) | __float_as_uint(x),
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float* p) {
  const unsigned long long v =
      __hip_atomic_load((const unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// Four consecutive dims of the output of row i of sequence b, o * inv (0 for an invalid row).
__device__ __forceinline__ void finish_row(const AttnArgs& a, int b, int i, int head, int d, f32x4 o, float inv) {
  const RowDesc rd = row_of(a, b, i);
  const int row = b * a.rps + i;
  if (!rd.valid) o = f32x4{0.f, 0.f, 0.f, 0.f};
  else o *= inv;
  if (rd.valid && rd.pos + 1 > a.max_ctx && d == 0) set_status(a.status, kStatusKvCapacity);  // the host's bound was wrong
  if (a.xs) put_stacked4(a.xs, a.stt, row, head * a.head_dim + d, o);
  else *(f32x4_a4*)(a.o + ((size_t)row * a.n_heads + head) * a.head_dim + d) = o;
}

// n / d for 0 <= n < 2^20 by the reciprocal of d (the quotient plus half a step
// is far from the next whole number compared with the product's rounding).
__device__ __forceinline__ int div_small(int n, float inv) { return (int)(((float)n + 0.5f) * inv); }

// Waves of a workgroup: with two query tiles a wave, two workgroups of 4 share a
// CU, so that one's start and merge run under the other's products.
__host__ __device__ constexpr int waves_of(int query_tiles) { return query_tiles == 1 ? 8 : 4; }

// LDS: the queries' parts; then, one query tile a wave, ring rows (a K fragment
// per tile and step, V's fragments), one slot per sub-chunk; reused by the
// merge.  With at most 64 rows, at most 65 of them not committed, at most 4
// sub-chunks of a sequence lie in the ring (63 + 65 rows from a multiple of
// 64): sub-chunk j in slot j % 4.
template <int HD, int QT>
struct Lds8 {
  static constexpr int KST = HD / 32, DT = HD / 16, OS = HD + 4, NW = waves_of(QT);
  bf16x8 q[QT][KST][3][kWave];
  f16x8 qh[QT > 1 ? QT : 1][QT > 1 ? KST : 1][2][QT > 1 ? kWave : 1];
  uint32_t row_max[QT * 16];
  union {
    u32x4 ring[QT == 1 ? 4 : 1][2 * KST + DT][kWave];
    struct {
      float o[NW][16][OS];
      float ml[NW][16][2];
    } m;
  };
  int last;
};

// Workgroups: LINE: the line of all units' chunks, `per` to a workgroup (x);
// otherwise part x of unit y of sequence z, every part of a sequence `per` long.
template <int HD, int QT, bool LINE, bool ONCE>
__global__ __launch_bounds__(64 * waves_of(QT), QT > 1 ? 2 : 4) void attn8_kernel(AttnArgs a, int n_tiles, int parts, int per0) {
  constexpr int KST = HD / 32, DT = HD / 16, FS = HD / 32, RK = 2 * KST, NW = waves_of(QT), SP = steps_of(HD);
  __shared__ Lds8<HD, QT> sh;
  const int lane0 = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int H = a.n_heads, G = a.n_kv_heads, group = H / G, rps = a.rps, nq = rps * group;
  const int window = a.f8.ring.capacity;
  const float qscale = 1.44269504088896341f / sqrtf((float)HD);  // (scores in powers of two)
  const float inv_group = 1.0f / (float)group;
  constexpr bool F16 = QT > 1;
  constexpr float kLift = F16 ? 15.f : 0.f;  // (probabilities are held times 2^kLift: away from fp16's least values)

  // One segment: chunks [k_lo, k_hi) of unit (b, g, tile), part `part` of its n.
  auto segment = [&](int b, int g, int tile, int k_lo, int k_hi, int part, int n) {
    // (opaque: what a segment derives from it stays in the segment, not in registers across all of them)
    int lane = lane0;
    asm volatile("" : "+v"(lane));
    const int c16 = lane & 15, grp = lane >> 4;
    if (F16) {
      if (threadIdx.x < 16 * QT) sh.row_max[threadIdx.x] = 0u;
      __syncthreads();
    }
    // This wave's 32-dim steps of the query tiles, asked for before the length that
    // everything else needs has arrived.
    constexpr int QW = (QT * KST + NW - 1) / NW;
    f32x4 qv[QW][2];
#pragma unroll
    for (int i = 0; i < QW; ++i) {
      const int st = wave + i * NW, q = st / KST, s = st % KST;
      const int qa = (tile * QT + q) * 16 + c16, qr = div_small(qa, inv_group);
      const int d = HD >= 64 ? 64 * (s >> 1) + 16 * grp + 8 * (s & 1) : 32 * s + 8 * grp;
      qv[i][0] = qv[i][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (st < QT * KST && qa < nq) {
        const float* qp = a.qr + ((size_t)(b * rps + qr) * H + g * group + qa - qr * group) * HD + d;
        qv[i][0] = *(const f32x4_a4*)qp;
        qv[i][1] = *(const f32x4_a4*)(qp + 4);
      }
    }
    // (the same in every lane; told so, the addresses that follow from it stay scalar)
    const int sealed = __builtin_amdgcn_readfirstlane((a.f8.len[b] + a.c0) / kF8Block * (kF8Block / kF8Sub / SP));
    if (QT == 1) k_hi = min(k_hi, sealed + 4 / SP);  // (no valid row is past it: the ring's slots)

    // Codes and scales through buffer descriptors that end with the sealed ones: a
    // wave's loads past its last sub-chunk read nothing, so none needs a branch
    // (with one, the compiler waits for every load at the loop's head).
    const int j_sealed = min(k_hi, sealed);
    const __amdgpu_buffer_rsrc_t cr = make_rsrc(a.f8.code_base(a.layer, b, g), (uint32_t)j_sealed * SP * 2 * kF8Sub * HD);
    const __amdgpu_buffer_rsrc_t sr = make_rsrc(a.f8.scale_base(a.layer, b, g), (uint32_t)((j_sealed * SP + 1) & ~1) * 4);
    constexpr int kCodes = ONCE ? kNonTemporal : 0;
    u32x4 kc[SP][FS], vc[SP][FS];
    float ks, vs;
    auto load_k = [&](int j) {
      const uint32_t at = (uint32_t)j * SP * 2 * kF8Sub * HD + lane * 16;
#pragma unroll
      for (int i = 0; i < SP * FS; ++i)
        kc[i / FS][i % FS] = __builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(cr, at + i / FS * 2 * kF8Sub * HD + i % FS * 1024, 0, kCodes));
      ks = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sr, (j * SP & ~1) * 4, 0, 0));
    };
    auto load_v = [&](int j) {
      const uint32_t at = (uint32_t)j * SP * 2 * kF8Sub * HD + kF8Sub * HD + lane * 16;
#pragma unroll
      for (int i = 0; i < SP * FS; ++i)
        vc[i / FS][i % FS] = __builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(cr, at + i / FS * 2 * kF8Sub * HD + i % FS * 1024, 0, kCodes));
      vs = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sr, (j * SP | 1) * 4, 0, 0));
    };
    // The ring's rows: with one query tile a wave they go to LDS without passing the
    // registers, at the segment's start; with two, to registers, a step ahead.
    const uint16_t* ring = k_block<uint16_t>(a.f8.ring, a.layer, b, g);
    u32x4 rk[QT == 1 ? 1 : RK], rv[QT == 1 ? 1 : DT];
    auto ring_k = [&](int sub) {  // (sub: the sub-chunk, in 32 positions)
      const __amdgpu_buffer_rsrc_t rr = make_rsrc(ring, (uint32_t)window * HD * 4u);
      int l = lane;
      asm volatile("" : "+v"(l));  // (addresses computed here, not kept)
      const int w0 = sub * kF8Sub % window, i = l & 15, c = l >> 4;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int s = 0; s < KST; ++s) {
          const int d = HD >= 64 ? 64 * (s >> 1) + 16 * c + 8 * (s & 1) : 32 * s + 8 * c;
          const int pos = w0 + 8 * (i >> 2) + 4 * t + (i & 3);
          const uint32_t at = (uint32_t)KvIndex<uint16_t>::k(pos, d, HD, window) * 2u;
          if constexpr (QT == 1) {
            const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&sh.ring[sub & 3][0][0];
            load_lds16(lds0 + (t * KST + s) * 1024u, at, rr);
          } else {
            rk[t * KST + s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, at, 0, 0));
          }
        }
    };
    auto ring_v = [&](int sub) {
      const __amdgpu_buffer_rsrc_t rr = make_rsrc(ring, (uint32_t)window * HD * 4u);
      int l = lane;
      asm volatile("" : "+v"(l));
      const int w0 = sub * kF8Sub % window, i = l & 15, c = l >> 4;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint32_t at = (uint32_t)KvIndex<uint16_t>::v(w0 + 8 * c, 16 * dt + i, HD, window) * 2u;
        if constexpr (QT == 1) {
          const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&sh.ring[sub & 3][0][0];
          load_lds16(lds0 + (RK + dt) * 1024u, at, rr);
        } else {
          rv[dt] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, at, 0, 0));
        }
      }
    };

    // This wave's chunks: j, j + NW, ...; the first codes, and the first ring
    // rows, are on their way while the queries are made ready.
    int j = k_lo + wave;
    int jr = max(j, j + (sealed - j + NW - 1) / NW * NW);  // the first of them in the ring
    // (one query tile: each wave has at most one chunk of the ring's)
    const bool has_ring = jr < k_hi;
    if (QT == 1 && has_ring) {
#pragma unroll
      for (int sp = 0; sp < SP; ++sp) {
        ring_k(jr * SP + sp);
        ring_v(jr * SP + sp);
      }
    }
    load_k(j);
    load_v(j);
    // Where this wave has ring rows: this lane's query of each tile, its position; the tiles' range.
    int qpos[QT], vis = 0, lowest = 0x7fffffff;
    if (has_ring) {
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        const int qa = (tile * QT + q) * 16 + c16;
        const RowDesc rd = row_of(a, b, qa < nq ? div_small(qa, inv_group) : 0);
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
    }

#pragma unroll
    for (int i = 0; i < QW; ++i) {
      const int st = wave + i * NW;
      if (st >= QT * KST) break;  // (wave-uniform)
      float v[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = qv[i][0][e] * qscale;
        v[4 + e] = qv[i][1][e] * qscale;
      }
      bf16x8 p3[3];
      split8(v, p3);
#pragma unroll
      for (int k = 0; k < 3; ++k) sh.q[st / KST][st % KST][k][lane] = p3[k];
      if constexpr (F16) {
        uint32_t m = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
        atomicMax(&sh.row_max[st / KST * 16 + c16], m);
      }
    }
    __syncthreads();
    float qinv[QT];  // (F16: what a row's products are multiplied by)
    if constexpr (F16) {
#pragma unroll
      for (int i = 0; i < QW; ++i) {
        const int st = wave + i * NW;
        if (st >= QT * KST) break;
        const float up = qscale * pow2i(row_shift(sh.row_max[st / KST * 16 + c16]));
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = qv[i][0][e] * up;
          v[4 + e] = qv[i][1][e] * up;
        }
        f16x8 p2[2];
        split8(v, p2);
#pragma unroll
        for (int k = 0; k < 2; ++k) sh.qh[st / KST][st % KST][k][lane] = p2[k];
      }
#pragma unroll
      for (int q = 0; q < QT; ++q) qinv[q] = pow2i(-row_shift(sh.row_max[q * 16 + c16]));
      __syncthreads();
    }

    floatx4 of[QT][DT];
    float mx[QT], sm[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      mx[q] = kLeast;
      sm[q] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) of[q][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    // kk(t, s): K rows of tile t, dims of step s; the scores of this lane's 8 positions, tile by tile.
    auto scores = [&](auto kk, floatx4 (&acc)[QT][2]) {
      int ql = lane;
      asm volatile("" : "+v"(ql));  // (the queries stay in LDS: hoisted out of the loop they would fill the registers)
#pragma unroll
      for (int q = 0; q < QT; ++q) acc[q][0] = acc[q][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KST; ++s) {
        const bf16x8 k0 = kk(0, s), k1 = kk(1, s);
#pragma unroll
        for (int k = 2; k >= 0; --k)  // (small parts first)
#pragma unroll
          for (int q = 0; q < QT; ++q) {
            const bf16x8 qq = sh.q[q][s][k][ql];
            acc[q][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qq, acc[q][0], 0, 0, 0);
            acc[q][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qq, acc[q][1], 0, 0, 0);
          }
      }
    };
    // The running maximum and sum of tile q over new scores p f, which become
    // probabilities relative to it.  Scores may be -inf, masked or below float32's
    // range: the maximum starts at the least finite value, so they weigh 0 even where
    // a query has seen no others yet.
    auto softmax = [&](int q, auto& p, float f) {
      constexpr int N = sizeof(p) / sizeof(float);
      float m = fmaxf(p[0], p[1]);
#pragma unroll
      for (int e = 2; e < N; ++e) m = fmaxf(m, p[e]);
      m = groups_max(m) * f;
      const float mnew = fmaxf(mx[q], m);
      if (__any(mnew > mx[q])) {  // (rescaled only where a maximum rose)
        const float alpha = __builtin_amdgcn_exp2f(mx[q] - mnew);
        sm[q] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) of[q][dt] *= alpha;
        mx[q] = mnew;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        p[e] = __builtin_amdgcn_exp2f(F16 ? __builtin_fmaf(p[e], f, kLift - mx[q]) : p[e] - mx[q]);
        sm[q] += p[e];
      }
    };

    if constexpr (F16) {
      for (; j < j_sealed; j += NW) {  // (wave-uniform) codes: every query sees them all
        float p[QT][8 * SP], f[QT];
#pragma unroll
        for (int q = 0; q < QT; ++q) f[q] = fminf(qinv[q] * ks, 3.4028235e38f);
        int ql = lane;
        asm volatile("" : "+v"(ql));
        // (a wave at its products goes before one at its softmax: 51.5 -> 48.7 us, 512 rows over 2048)
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int sp = 0; sp < SP; ++sp) {
          floatx4 acc[QT][2];
#pragma unroll
          for (int q = 0; q < QT; ++q) acc[q][0] = acc[q][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < KST; ++s) {
            f16x8 kk[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const u32x4 w = HD >= 64 ? kc[sp][t * (HD / 64) + s / 2] : kc[sp][0];
              const int h = HD >= 64 ? s & 1 : t;
              kk[t] = fp8x8_to_f16(w[2 * h], w[2 * h + 1], 1.0f);
            }
#pragma unroll
            for (int k = 1; k >= 0; --k)  // (small parts first)
#pragma unroll
              for (int q = 0; q < QT; ++q) {
                const f16x8 qq = sh.qh[q][s][k][ql];
                acc[q][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk[0], qq, acc[q][0], 0, 0, 0);
                acc[q][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk[1], qq, acc[q][1], 0, 0, 0);
              }
          }
#pragma unroll
          for (int q = 0; q < QT; ++q)
#pragma unroll
            for (int e = 0; e < 8; ++e) p[q][8 * sp + e] = acc[q][e >> 2][e & 3];
        }
        __builtin_amdgcn_s_setprio(0);
        load_k(j + NW);
        f16x8 pp[QT][SP][2];
#pragma unroll
        for (int q = 0; q < QT; ++q) {
          softmax(q, p[q], f[q]);
#pragma unroll
          for (int sp = 0; sp < SP; ++sp) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = p[q][8 * sp + e];
            split8(v, pp[q][sp]);
          }
        }
        const int ve = __builtin_amdgcn_readfirstlane((int)__float_as_uint(vs) >> 23) - 127;
        __builtin_amdgcn_s_setprio(1);
        if (ve >= -15 && ve <= 7) {  // (V's values are fp16's)
          constexpr int DG = DT < 4 ? DT : 4;
#pragma unroll
          for (int sp = 0; sp < SP; ++sp)
#pragma unroll
            for (int d0 = 0; d0 < DT; d0 += DG) {
              f16x8 vv[DG];
#pragma unroll
              for (int i = 0; i < DG; ++i) {
                const u32x4 w = vc[sp][(d0 + i) / 2];
                vv[i] = fp8x8_to_f16(w[2 * (i & 1)], w[2 * (i & 1) + 1], vs);
              }
#pragma unroll
              for (int k = 1; k >= 0; --k)
#pragma unroll
                for (int i = 0; i < DG; ++i)
#pragma unroll
                  for (int q = 0; q < QT; ++q)
                    of[q][d0 + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv[i], pp[q][sp][k], of[q][d0 + i], 0, 0, 0);
            }
        } else {  // the codes' products, times the scale
#pragma unroll
          for (int sp = 0; sp < SP; ++sp)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              const u32x4 w = vc[sp][dt / 2];
              const f16x8 vv = fp8x8_to_f16(w[2 * (dt & 1)], w[2 * (dt & 1) + 1], 1.0f);
#pragma unroll
              for (int q = 0; q < QT; ++q) {
                floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 1; k >= 0; --k) x = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, pp[q][sp][k], x, 0, 0, 0);
                of[q][dt] += x * vs;
              }
            }
        }
        __builtin_amdgcn_s_setprio(0);
        load_v(j + NW);
      }
    } else {
      for (; j < j_sealed; j += NW) {  // (wave-uniform) codes: every query sees them all
        float p[QT][8 * SP];
#pragma unroll
        for (int sp = 0; sp < SP; ++sp) {
          floatx4 acc[QT][2];
          scores(
              [&](int t, int s) {
                const u32x4 w = HD >= 64 ? kc[sp][t * (HD / 64) + s / 2] : kc[sp][0];
                const int h = HD >= 64 ? s & 1 : t;
                return fp8x8_to_bf16(w[2 * h], w[2 * h + 1], ks);
              },
              acc);
#pragma unroll
          for (int q = 0; q < QT; ++q)
#pragma unroll
            for (int e = 0; e < 8; ++e) p[q][8 * sp + e] = acc[q][e >> 2][e & 3];
        }
        // (a wave's next K is on its way through the softmax and P V, its next V through the next scores)
        load_k(j + NW);
        bf16x8 pp[QT][SP][3];
#pragma unroll
        for (int q = 0; q < QT; ++q) {
          softmax(q, p[q], 1.f);
#pragma unroll
          for (int sp = 0; sp < SP; ++sp) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = p[q][8 * sp + e];
            split8(v, pp[q][sp]);
          }
        }
        // (DG dimension tiles in turn: a product that waits for its accumulator would leave the matrix unit idle)
        constexpr int DG = DT < 4 ? DT : 4;
#pragma unroll
        for (int sp = 0; sp < SP; ++sp)
#pragma unroll
          for (int d0 = 0; d0 < DT; d0 += DG) {
            bf16x8 vv[DG];
#pragma unroll
            for (int i = 0; i < DG; ++i) {
              const u32x4 w = vc[sp][(d0 + i) / 2];
              vv[i] = fp8x8_to_bf16(w[2 * (i & 1)], w[2 * (i & 1) + 1], vs);
            }
#pragma unroll
            for (int k = 2; k >= 0; --k)
#pragma unroll
              for (int i = 0; i < DG; ++i)
#pragma unroll
                for (int q = 0; q < QT; ++q)
                  of[q][d0 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv[i], pp[q][sp][k], of[q][d0 + i], 0, 0, 0);
          }
        load_v(j + NW);
      }
    }

    if (has_ring) {
      if (QT > 1) {
        ring_k(jr * SP);
        ring_v(jr * SP);
      }
#pragma unroll 1
      for (; jr < k_hi; jr += NW)
#pragma unroll 1
        for (int sp = 0; sp < SP; ++sp) {
          const int sub = jr * SP + sp, k0 = sub * kF8Sub;
          if (QT == 1) {
            wait_vm<0>();  // (the rows are in LDS)
            __builtin_amdgcn_wave_barrier();
          }
          if (k0 >= vis) break;
          const int next = sp + 1 < SP ? sub + 1 : (jr + NW) * SP;
          const u32x4(*rows)[kWave] = sh.ring[QT == 1 ? sub & 3 : 0];
          floatx4 acc[QT][2];
          scores([&](int t, int s) { return __builtin_bit_cast(bf16x8, QT == 1 ? rows[t * KST + s][lane] : rk[QT == 1 ? 0 : t * KST + s]); }, acc);
          if (QT > 1) ring_k(next);
          // Where some query does not see all of them (uniform):
          //  - slots past the newest visible position hold stale values: their V entries
          //    are zeroed, never multiplied by a zero probability;
          //  - a NaN or infinity that only later rows see must not reach the others through
          //    0 * inf: such entries leave the product and are added by themselves to the
          //    queries that see them.
          const bool diagonal = k0 + kF8Sub - 1 > lowest;
          const int nvalid = vis - (k0 + 8 * grp);
          bool odd = false;
          auto strip = [&](u32x4& v) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              if (2 * w >= nvalid) v[w] = 0u;
              else if (2 * w + 1 >= nvalid) v[w] &= 0xffffu;
              const bool lo = (v[w] & 0x7f80u) == 0x7f80u, up = (v[w] & 0x7f800000u) == 0x7f800000u;
              odd |= lo || up;
              if (lo) v[w] &= 0xffff0000u;
              if (up) v[w] &= 0xffffu;
            }
          };
          if (QT > 1 && diagonal) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) strip(rv[QT == 1 ? 0 : dt]);
          }
#pragma unroll
          for (int q = 0; q < QT; ++q) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = k0 + 8 * grp + e > qpos[q] ? -INFINITY : acc[q][e >> 2][e & 3];
            softmax(q, p, 1.f);
            bf16x8 pp[3];
            split8(p, pp);
            constexpr int DG = DT < 4 ? DT : 4;
#pragma unroll
            for (int d0 = 0; d0 < DT; d0 += DG) {
              u32x4 v[DG];
#pragma unroll
              for (int i = 0; i < DG; ++i) {
                v[i] = QT == 1 ? rows[RK + d0 + i][lane] : rv[QT == 1 ? 0 : d0 + i];
                if (QT == 1 && diagonal) strip(v[i]);
              }
#pragma unroll
              for (int k = 2; k >= 0; --k)
#pragma unroll
                for (int i = 0; i < DG; ++i)
                  of[q][d0 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[i]), pp[k], of[q][d0 + i], 0, 0, 0);
            }
            if (diagonal && __any(odd)) {
              for (int i = 0; i < kF8Sub; ++i) {  // (position k0 + i; its probability lies in lane group i / 8)
                float pi = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) pi = (i & 7) == e ? p[e] : pi;
                pi = __shfl(pi, 16 * (i >> 3) + c16, kWave);
                // (V fragment dt: lane 16 (i / 8) + d, entry i % 8)
                const uint16_t* vrow = QT == 1 ? (const uint16_t*)&rows[RK][16 * (i >> 3)] + (i & 7)
                                               : ring + KvIndex<uint16_t>::v(k0 % window + i, 0, HD, window);
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
          if (QT > 1) ring_v(next);
        }
    }

    // Merge the waves of this segment in LDS, tile by tile (fixed order).
    // Thread: 4 dims of a row.
    const bool whole = n == 1;
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      const int n_here = min(16, nq - (tile * QT + q) * 16);
      if (n_here <= 0) break;
      float sum = sm[q];
      sum += __shfl_xor(sum, 16, kWave);
      sum += __shfl_xor(sum, 32, kWave);
      __syncthreads();  // (the ring's rows, or the tile before, are read)
      if (c16 < n_here) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(floatx4*)&sh.m.o[wave][c16][16 * dt + 4 * grp] = of[q][dt];
        if (grp == 0) {
          sh.m.ml[wave][c16][0] = mx[q];
          sh.m.ml[wave][c16][1] = sum;
        }
      }
      __syncthreads();
      const int d = threadIdx.x % (HD / 4) * 4;
      for (int i = threadIdx.x / (HD / 4); i < n_here; i += 64 * NW / (HD / 4)) {
        float M = kLeast, L = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, sh.m.ml[w][i][0]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          // (a wave without keys: the least maximum, sum and outputs 0; NaN scores alone: that and a NaN sum)
          const float e = __builtin_amdgcn_exp2f(sh.m.ml[w][i][0] - M);
          L += e * sh.m.ml[w][i][1];
          o += e * *(const f32x4*)&sh.m.o[w][i][d];
        }
        const int qa = (tile * QT + q) * 16 + i, qr = div_small(qa, inv_group);
        const int row = b * rps + qr, head = g * group + qa - qr * group;
        if (whole) {
          finish_row(a, b, qr, head, d, o, 1.0f / L);
        } else {
          const size_t slot = ((size_t)row * H + head) * parts + part;
          put2(a.o_part + slot * HD + d, o[0], o[1]);
          put2(a.o_part + slot * HD + d + 2, o[2], o[3]);
          if (d == 0) put2(a.ml_part + 2 * slot, M, L);
        }
      }
    }

    // The last workgroup of a unit that spans several adds its parts: one wave a
    // row, lane p the (max, sum) of part p, then LP lanes of 4 dims per part.
    if (!whole) {
      uint32_t* ctr = a.f8.counters + ((size_t)b * G + g) * n_tiles + tile;
      wait_vm<0>();  // (this wave's stores have completed)
      __syncthreads();
      if (threadIdx.x == 0) {
        const uint32_t old = __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sh.last = old == (uint32_t)(n - 1);
        if (sh.last) __hip_atomic_store(ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      if (sh.last) {
        // (two rows a wave at once, their loads in one list: IT of them in flight)
        constexpr int LP = HD / 4, PI = kWave / LP, RW = 2, IT = 12;
        const int n_rows = min(16 * QT, nq - tile * QT * 16), pg = lane / LP, d = lane % LP * 4;
        const int steps = (n + PI - 1) / PI;  // loads of one row
        for (int i0 = wave; i0 < n_rows; i0 += NW * RW) {  // (wave-uniform)
          const int here = i0 + NW < n_rows ? 2 : 1;
          size_t slot[RW];
          int qr[RW], head[RW];
          float2 ml[RW];
          f32x4 acc[RW];
          float wgt[RW], inv[RW];
#pragma unroll
          for (int r = 0; r < RW; ++r) {
            const int qa = tile * QT * 16 + i0 + (r < here ? r * NW : 0);
            qr[r] = div_small(qa, inv_group);
            head[r] = g * group + qa - qr[r] * group;
            slot[r] = ((size_t)(b * rps + qr[r]) * H + head[r]) * parts;
            ml[r] = lane < n ? get2(a.ml_part + 2 * (slot[r] + lane)) : make_float2(kLeast, 0.f);
            acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
          }
          for (int t0 = 0; t0 < here * steps; t0 += IT) {
            float2 lo[IT], up[IT];
#pragma unroll
            for (int k = 0; k < IT; ++k) {
              const int t = t0 + k;
              if (t >= here * steps) break;  // (uniform)
              const int row1 = t >= steps, p = (t - (row1 ? steps : 0)) * PI + pg;
              const float* src = a.o_part + ((row1 ? slot[1] : slot[0]) + min(p, n - 1)) * HD + d;
              lo[k] = get2(src);
              up[k] = get2(src + 2);
            }
            if (t0 == 0) {
#pragma unroll
              for (int r = 0; r < RW; ++r) {
                const float M = wave_max(ml[r].x);
                wgt[r] = __builtin_amdgcn_exp2f(ml[r].x - M);
                inv[r] = 1.0f / wave_sum(wgt[r] * ml[r].y);
              }
            }
#pragma unroll
            for (int k = 0; k < IT; ++k) {
              const int t = t0 + k;
              if (t >= here * steps) break;
              const int row1 = t >= steps, p = (t - (row1 ? steps : 0)) * PI + pg;
              const float wp = __shfl(row1 ? wgt[1] : wgt[0], p & 63, kWave), w = p < n ? wp : 0.f;  // (by every lane)
              const f32x4 v = {lo[k].x, lo[k].y, up[k].x, up[k].y};
              if (row1) acc[1] += w * v;
              else acc[0] += w * v;
            }
          }
#pragma unroll
          for (int r = 0; r < RW; ++r) {
            if (r >= here) break;
#pragma unroll
            for (int o = LP; o < kWave; o <<= 1)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[r][e] += __shfl_xor(acc[r][e], o, kWave);
            if (lane < LP) finish_row(a, b, qr[r], head[r], d, acc[r], inv[r]);
          }
        }
      }
    }
  };

  if constexpr (!LINE) {
    const int b = blockIdx.z, u = blockIdx.y, part = blockIdx.x;
    const int nb = __builtin_amdgcn_readfirstlane(chunks_of<chunk_of(HD)>(a, b)), k_lo = part * per0;
    if (k_lo >= nb) return;  // (workgroup-uniform)
    // (kv heads first, so that an XCD's workgroups read few of them; later tiles, which see
    // more, beside earlier ones)
    const int t = u / G, half = (n_tiles + 1) / 2;
    segment(b, u - t * G, t < half ? n_tiles - 1 - t : t - half, k_lo, min(nb, k_lo + per0), part, (nb + per0 - 1) / per0);
  } else {
    const int B = a.M / rps, U = G * n_tiles;
    // (64 sequences' chunks at a time in a register)
    auto some = [&](int c) { return c + lane0 < B ? chunks_of<chunk_of(HD)>(a, c + lane0) : 0; };
    int n64 = some(0), at64 = 0, total = lane_sum(n64);
    for (int c = kWave; c < B; c += kWave) total += lane_sum(some(c));
    total *= U;
    // (four chunks a wave at least: a cut moves by less than half of that)
    const int per = max(max((total + (int)gridDim.x - 1) / (int)gridDim.x, per0), 4 * NW);
    auto subs = [&](int s) {
      if ((s & ~(kWave - 1)) != at64) {
        at64 = s & ~(kWave - 1);
        n64 = some(at64);
      }
      return __builtin_amdgcn_readlane(n64, s & (kWave - 1));
    };
    // Where a unit of n chunks is cut that a border meets d chunks in: after whole rounds
    // of all waves, and not at all where a round or less would be cut off (16 ragged rows
    // over 1024 to 8191 keys 114.5 us, 118 us with cuts where they fall).
    auto snap = [](int d, int n) {
      const int r = (d + NW / 2) / NW * NW;
      return r <= NW ? 0 : n - r <= NW ? n : r;
    };
    struct At {
      int b, base, nb;  // a sequence, the line where it starts, the chunks of its units
    };
    auto walk = [&](At& at, int x) {  // to the sequence that holds x
      while (x >= at.base + at.nb * U) {
        at.base += at.nb * U;
        ++at.b;
        at.nb = subs(at.b);
      }
      return at.base + (x - at.base) / at.nb * at.nb;  // the line where x's unit starts
    };
    int x = (int)blockIdx.x * per, hi = x + per;
    if (x >= total) return;
    At at{0, 0, subs(0)};
    int unit0 = walk(at, x);
    x = unit0 + snap(x - unit0, at.nb);
    if (hi < total) {
      At end = at;
      unit0 = walk(end, hi);
      hi = unit0 + snap(hi - unit0, end.nb);
    } else {
      hi = total;
    }
    while (x < hi) {
      unit0 = walk(at, x);
      const int nb = at.nb, u = (unit0 - at.base) / nb, g = u / n_tiles, k_lo = x - unit0, k_hi = min(nb, hi - unit0);
      // the first and the last workgroup with a part of the unit: the borders before its
      // start and its end, but for one that was moved across
      int first = unit0 / per, last = (unit0 + nb - 1) / per;
      const int y0 = (first + 1) * per - unit0, y1 = last * per - unit0;
      if (y0 < nb && snap(y0, nb) == 0) ++first;
      if (y1 >= 0 && snap(y1, nb) == nb) --last;
      x = unit0 + k_hi;
      segment(at.b, g, u - g * n_tiles, k_lo, k_hi, (int)blockIdx.x - first, last - first + 1);
      __syncthreads();  // (LDS is free for the next segment)
    }
  }
}

struct Plan {
  int qt, n_tiles, line, nwg, per, parts;
};
int tiles_a_wave(int nq) { return nq <= 64 ? 1 : 2; }
int tiles_of(int nq) { return (nq + 16 * tiles_a_wave(nq) - 1) / (16 * tiles_a_wave(nq)); }
Plan plan_of(int rps, int batch, int n_heads, int n_kv_heads, int head_dim, int max_ctx) {
  Plan p;
  const int nq = rps * (n_heads / n_kv_heads);
  p.qt = tiles_a_wave(nq);
  p.n_tiles = tiles_of(nq);
  const long nb = (max_ctx + chunk_of(head_dim) - 1) / chunk_of(head_dim), units = (long)n_kv_heads * p.n_tiles;
  const long slots = 2L * device_compute_units();  // workgroups resident at once
  // Several sequences of unlike lengths, one query tile, more than four chunks a wave:
  // the line.  (Two tiles cost a cut more than it gives: 4 x 70 rows over 500 to 6000 keys
  // 106 us on the line, 93 us not; over 100, 60000, 100 and 50 keys 437 and 97 us.)
  const long least = (nb + kPartsMax8 - 3) / (kPartsMax8 - 2);
  // (The line is counted in 32 bits.)
  const long most = nb * units * batch;
  p.line = p.qt == 1 && batch > 1 && (most + slots - 1) / slots > 4 * waves_of(p.qt) && most <= 1L << 30;
  // Otherwise as many parts of a unit as let all workgroups be resident (200 rows over
  // 1736 keys, 224 units: 2 parts 36 us, 3, of equal chunks and a rest, 45 us); more where
  // one sequence of a batch may be far longer than the others, 128 chunks to a part, but
  // no more than it would have alone (one of 60000 keys in four: 97 us, without 299 us;
  // 64 chunks to a part make 4 x 70 rows over 4000 keys 101 us, not 80); and at least a
  // chunk a wave: fewer parts to add.  (Half a chunk was 12.9 us, one 10.4 us, two 11.4 us
  // for a row over 2048 keys of 32 heads.)
  const long all = std::max(1L, slots / (units * batch)), alone = std::max(1L, slots / units);
  const long share = std::min((nb + all - 1) / all, batch > 1 ? 128L : nb);
  const long per = std::max({share, (nb + alone - 1) / alone, least, (long)waves_of(p.qt)});
  p.per = (int)(p.line ? least : per);
  p.nwg = (int)(p.line ? slots : (nb + per - 1) / per);
  // Parts of a unit, at most: a workgroup takes at least nb * units / slots of the
  // longest sequence's line, whatever the other lengths.  (Grows with max_ctx:
  // a workspace for the capacity holds every call's.)
  p.parts = (int)std::min<long>({nb, slots / units + 2, (long)kPartsMax8});
  return p;
}

}  // namespace

bool attention8_fits(int rps, int batch, int n_heads, int n_kv_heads) {
  return batch <= kF8MaxBatch && (long)n_kv_heads * tiles_of(rps * (n_heads / n_kv_heads)) <= kF8MaxUnits;
}

int attention8_parts(int rps, int batch, int n_heads, int n_kv_heads, int head_dim, int max_ctx) {
  return plan_of(rps, batch, n_heads, n_kv_heads, head_dim, max_ctx).parts;
}

hipError_t launch_attention8(const AttnArgs& a, hipStream_t s) {
  const int B = a.M / a.rps;
  const Plan p = plan_of(a.rps, B, a.n_heads, a.n_kv_heads, a.head_dim, a.max_ctx);
  if (p.parts > a.n_split || p.n_tiles > kF8TilesPerSlot * a.f8.ring.capacity ||
      !attention8_fits(a.rps, B, a.n_heads, a.n_kv_heads))
    return hipErrorInvalidValue;  // (the callers have checked)
  const dim3 grid = p.line ? dim3(p.nwg) : dim3(p.nwg, (unsigned)(a.n_kv_heads * p.n_tiles), B);
  const dim3 block(64 * waves_of(p.qt));
  // (codes that one unit alone reads need not stay in a cache)
#define SD_A8(HDV, QT, LINE, ONCE) \
  hipLaunchKernelGGL((attn8_kernel<HDV, QT, LINE, ONCE>), grid, block, 0, s, a, p.n_tiles, p.parts, p.per)
#define SD_A8_HD(HDV)                                  \
  if (p.qt == 2) {                                     \
    SD_A8(HDV, 2, false, false);                       \
  } else if (p.n_tiles == 1) {                         \
    if (p.line) SD_A8(HDV, 1, true, true);             \
    else SD_A8(HDV, 1, false, true);                   \
  } else {                                             \
    if (p.line) SD_A8(HDV, 1, true, false);            \
    else SD_A8(HDV, 1, false, false);                  \
  }
  switch (a.head_dim) {
    case 32: SD_A8_HD(32) break;
    case 64: SD_A8_HD(64) break;
    case 128: SD_A8_HD(128) break;
    default: return hipErrorInvalidValue;
  }
#undef SD_A8_HD
#undef SD_A8
  return hipGetLastError();
}

}  // namespace specdec
