// The FP8 KV cache (layout: internal.h): writing whole blocks from bf16 rows,
// reading values back, appending rows to the ring, and sealing the blocks that
// a commit completes.
//
// All are copies: the bound is the stream of bytes.  A block of 64 positions of
// one kv head is one workgroup's: its K and V pass through registers once
// (their maximum, then the codes).  V changes from rows to operand order in LDS,
// K's operand order is that of its rows' pieces; the write asks for K before it
// waits for V (16.0 -> 15.0 us at 2048 positions of 32 heads of 128).
// 32745 positions of that shape: write 173 us, read 136 us, 805 MB each, 4.7 and
// 5.9 TB/s (a copy of that size: 5.2).  Read back, K goes through LDS too: stored from
// operand order, in pieces of 16 bytes, 643 MB were written for 537 (194 against
// 160 us).  Nontemporal rows out: 100 us more; so all accesses are plain ones.
#include <algorithm>

#include "device_common.h"
#include "fp8.h"
#include "internal.h"

namespace specdec {

namespace {

constexpr int kCopyThreads = 256;

// Position (in its block of 64) and first dim of the 8 codes at bytes 8e .. 8e+7
// of lane 16c + i of the block's K fragment f (HD / 32 of its first half, then of
// its second); the dim whose 8 positions from `pos` V's fragment f holds there.
template <int HD>
__device__ __forceinline__ void k_place(int f, int c, int i, int e, int& pos, int& dim) {
  constexpr int FS = HD / 32;
  const int s = f / FS, r = f % FS;
  if constexpr (HD >= 64) {
    pos = 32 * s + 8 * (i >> 2) + 4 * (r / (HD / 64)) + (i & 3);
    dim = 64 * (r % (HD / 64)) + 16 * c + 8 * e;
  } else {
    pos = 32 * s + 8 * (i >> 2) + 4 * e + (i & 3);
    dim = 8 * c;
  }
}
template <int HD>
__device__ __forceinline__ void v_place(int f, int c, int i, int e, int& pos, int& dim) {
  constexpr int FS = HD / 32;
  pos = 32 * (f / FS) + 8 * c;
  dim = 16 * (2 * (f % FS) + e) + i;
}
// Byte of fragment f in the block's codes.
template <int HD>
__device__ __forceinline__ int frag_at(bool is_v, int f) {
  constexpr int FS = HD / 32;
  return (2 * (f / FS) + is_v) * 32 * HD + f % FS * 1024;
}

// Largest |x| among the finite of 8 bf16 values, as its bits.
__device__ __forceinline__ uint32_t amax8(u32x4 v, uint32_t m) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t a = v[q] & 0x7fffu, b = (v[q] >> 16) & 0x7fffu;
    if (a < 0x7f80u && a > m) m = a;
    if (b < 0x7f80u && b > m) m = b;
  }
  return m;
}

// Scale exponent of a block whose largest finite |x| has the bf16 bits m:
// 448 = 1.75 * 2^8, so 2^(E-8) fits mantissas up to 1.75 and 2^(E-7) the rest.
__device__ __forceinline__ int scale_exp(uint32_t m) {
  const int e = (int)(m >> 7) - 127 - 8 + ((m & 0x7fu) > 0x60u ? 1 : 0);
  return e < kF8MinExp ? kF8MinExp : e;
}

// 8 bf16 values times 2^-e as e4m3 codes (nearest, ties to even; non-finite: NaN).
__device__ __forceinline__ u32x2 codes8(u32x4 v, float inv) {
  u32x2 o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float x[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t w = v[2 * h + (q >> 1)];
      const float f = __uint_as_float((q & 1) ? (w & 0xffff0000u) : (w << 16));
      x[q] = isfinite(f) ? f * inv : __uint_as_float(0x7fc00000u);
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
    o[h] = (uint32_t)w;
  }
  return o;
}

// One block's codes and scales (256 threads; waves 0 and 1 K, 2 and 3 V).
// k8(pos, dim): 8 dims of one position; v8(pos, dim): 8 positions of one dim, after
// ready(), which every wave calls once K's loads are under way.
template <int HD, typename KF, typename RF, typename VF>
__device__ __forceinline__ void quantize_block(KF k8, RF ready, VF v8, unsigned char* codes, float* scales) {
  constexpr int F = HD / 16, FW = F / 2;  // fragments of K (as many of V), per wave
  __shared__ uint32_t red[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane >> 4, i = lane & 15;
  const bool is_v = wave >= 2;
  u32x4 x[FW][2];
  uint32_t m = 0;
  auto load = [&](auto place, auto get) {
#pragma unroll
    for (int j = 0; j < FW; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        int pos, dim;
        place((wave & 1) * FW + j, c, i, e, pos, dim);
        x[j][e] = get(pos, dim);
      }
  };
  if (!is_v) load(k_place<HD>, k8);
  ready();
  if (is_v) load(v_place<HD>, v8);
#pragma unroll
  for (int j = 0; j < FW; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) m = amax8(x[j][e], m);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, kWave));
  __syncthreads();  // (a caller's loop: red is free again)
  if (lane == 0) red[wave] = m;
  __syncthreads();
  m = is_v ? max(red[2], red[3]) : max(red[0], red[1]);
  const int ex = scale_exp(m);
  const float inv = __uint_as_float((uint32_t)(127 - ex) << 23);
#pragma unroll
  for (int j = 0; j < FW; ++j) {
    const int f = (wave & 1) * FW + j;
    const u32x2 a = codes8(x[j][0], inv), b = codes8(x[j][1], inv);
    *(u32x4*)(codes + frag_at<HD>(is_v, f) + lane * 16) = u32x4{a[0], a[1], b[0], b[1]};
  }
  if (lane == 0 && (wave & 1) == 0) scales[is_v] = __uint_as_float((uint32_t)(ex + 127) << 23);
}

// One row's K and V (source offset src of k, v [.., h_kv, hd]) into ring slot p.
__device__ __forceinline__ void ring_put(const KvLayout& ring, int layer, int b, int p, size_t src, const uint16_t* k,
                                         const uint16_t* v) {
  const int hd = ring.head_dim, w = ring.n_kv_heads * hd;
  for (int i = 8 * threadIdx.x; i < w; i += 8 * blockDim.x) {
    const int g = i / hd, dd = i % hd;
    uint16_t* blk = k_block<uint16_t>(ring, layer, b, g);
    const u32x4 kk = *(const u32x4_a2*)(k + src + i), vv = *(const u32x4_a2*)(v + src + i);
    *(u32x4*)(blk + KvIndex<uint16_t>::k(p, dd, hd, ring.capacity)) = kk;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      blk[KvIndex<uint16_t>::v(p, dd + e, hd, ring.capacity)] = (uint16_t)(vv[e >> 1] >> (16 * (e & 1)));
  }
}

// Grid x: n_whole * G workgroups, one per (whole block, kv head), then one per
// row that goes to the ring.
template <int HD>
__global__ __launch_bounds__(kCopyThreads) void kv8_write_kernel(Kv8Layout kv, int layer, int b, int pos0, int n,
                                                                 int n_whole, int n_ring, const uint16_t* k,
                                                                 const uint16_t* v) {
  const int G = kv.ring.n_kv_heads;
  if ((int)blockIdx.x >= n_whole * G) {
    const int p = n - n_ring + ((int)blockIdx.x - n_whole * G);
    ring_put(kv.ring, layer, b, (pos0 + p) % kv.ring.capacity, (size_t)p * G * HD, k, v);
    return;
  }
  // V's rows of 64 positions, then read along the positions (row stride HD + 2:
  // the 16 dims of a lane group fall on 8 banks, its 4 position groups on others).
  __shared__ uint16_t sv[kF8Block][HD + 2];
  const int blk = blockIdx.x / G, g = blockIdx.x % G;
  const size_t base = ((size_t)blk * kF8Block * G + g) * HD;
  constexpr int RC = HD / 8, VL = kF8Block * RC / kCopyThreads;  // 16-byte pieces of a row, of a thread
  u32x4 vr[VL];
#pragma unroll
  for (int j = 0; j < VL; ++j) {
    const int t = threadIdx.x + j * kCopyThreads, r = t / RC, d = t % RC * 8;
    vr[j] = *(const u32x4_a2*)(v + base + (size_t)r * G * HD + d);
  }
  const int at = pos0 / kF8Block + blk;
  quantize_block<HD>(
      [&](int pos, int dim) { return (u32x4) * (const u32x4_a2*)(k + base + (size_t)pos * G * HD + dim); },
      [&] {
#pragma unroll
        for (int j = 0; j < VL; ++j) {
          const int t = threadIdx.x + j * kCopyThreads, r = t / RC, d = t % RC * 8;
#pragma unroll
          for (int q = 0; q < 4; ++q) *(uint32_t*)&sv[r][d + 2 * q] = vr[j][q];
        }
        __syncthreads();
      },
      [&](int pos, int dim) {
        u32x4 x;
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] = sv[pos + 2 * q][dim] | (uint32_t)sv[pos + 2 * q + 1][dim] << 16;
        return x;
      },
      kv.code_base(layer, b, g) + (size_t)at * 2 * kF8Block * HD, kv.scale_base(layer, b, g) + 2 * (size_t)at);
}

// Grid: G times the blocks that [pos0, pos0 + n) touches; the block's values as rows.  (Heads
// first, so that whole positions are stored at about the same time: 160 -> 136 us for
// 32745 positions of 32 heads, and 194 -> 171 us for the write of them before it.)
template <int HD>
__global__ __launch_bounds__(kCopyThreads) void kv8_read_kernel(Kv8Layout kv, int layer, int b, int pos0, int n,
                                                                uint16_t* k, uint16_t* v) {
  __shared__ uint16_t sv[kF8Block][HD + 2];
  __shared__ alignas(16) uint16_t sk[kF8Block][HD + 8];
  constexpr int F = HD / 16, FW = F / 4 > 0 ? F / 4 : 1;  // fragments per wave
  const int G = kv.ring.n_kv_heads, g = blockIdx.x % G;
  const int blk = pos0 / kF8Block + blockIdx.x / G, p0 = blk * kF8Block;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane >> 4, i = lane & 15;
  auto at = [&](int pos) { return ((size_t)(p0 + pos - pos0) * G + g) * HD; };
  auto in = [&](int pos) { return p0 + pos >= pos0 && p0 + pos < pos0 + n; };
  if (p0 + kF8Block <= kv.len[b]) {  // sealed
    const unsigned char* codes = kv.code_base(layer, b, g) + (size_t)blk * 2 * kF8Block * HD;
    const float* sc = kv.scale_base(layer, b, g) + 2 * (size_t)blk;
    const float ks = sc[0], vs = sc[1];
    u32x4 kc[FW], vc[FW];
#pragma unroll
    for (int j = 0; j < FW; ++j) {
      const int f = wave * FW + j;
      if (f < F) {
        kc[j] = *(const u32x4*)(codes + frag_at<HD>(false, f) + lane * 16);
        vc[j] = *(const u32x4*)(codes + frag_at<HD>(true, f) + lane * 16);
      }
    }
#pragma unroll
    for (int j = 0; j < FW; ++j) {
      const int f = wave * FW + j;
      if (f >= F) break;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        int pos, dim;
        k_place<HD>(f, c, i, e, pos, dim);
        *(u32x4*)&sk[pos][dim] = __builtin_bit_cast(u32x4, fp8x8_to_bf16(kc[j][2 * e], kc[j][2 * e + 1], ks));
        const u32x4 y = __builtin_bit_cast(u32x4, fp8x8_to_bf16(vc[j][2 * e], vc[j][2 * e + 1], vs));
        v_place<HD>(f, c, i, e, pos, dim);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          sv[pos + 2 * q][dim] = (uint16_t)y[q];
          sv[pos + 2 * q + 1][dim] = (uint16_t)(y[q] >> 16);
        }
      }
    }
  } else {  // the ring's rows
    const uint16_t* src = k_block<uint16_t>(kv.ring, layer, b, g);
    const int w0 = p0 % kv.ring.capacity;
    for (int t = threadIdx.x; t < kF8Block * HD / 8; t += kCopyThreads) {
      const int r = t / (HD / 8), d = t % (HD / 8) * 8;
      *(u32x4*)&sk[r][d] = *(const u32x4*)(src + KvIndex<uint16_t>::k(w0 + r, d, HD, kv.ring.capacity));
      const int dim = t % HD, pos = t / HD * 8;
      const u32x4 y = *(const u32x4*)(src + KvIndex<uint16_t>::v(w0 + pos, dim, HD, kv.ring.capacity));
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        sv[pos + 2 * q][dim] = (uint16_t)y[q];
        sv[pos + 2 * q + 1][dim] = (uint16_t)(y[q] >> 16);
      }
    }
  }
  __syncthreads();
  for (int t = threadIdx.x; t < kF8Block * HD / 8; t += kCopyThreads) {
    const int r = t / (HD / 8), d = t % (HD / 8) * 8;
    if (!in(r)) continue;
    *(u32x4_a2*)(k + at(r) + d) = *(const u32x4*)&sk[r][d];
    u32x4 x;
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = *(const uint32_t*)&sv[r][d + 2 * q];
    *(u32x4_a2*)(v + at(r) + d) = x;
  }
}

// Grid (n, batch).  7B-like (32 kv heads of 128): 1 row 4.8 us (7 with the host's call),
// 512 rows 17 us, 2048 rows 52 us, 1.3 TB/s: V goes out two bytes at a time, 16 apart.
__global__ __launch_bounds__(kCopyThreads) void kv8_append_kernel(Kv8Layout kv, int layer, int n, const uint16_t* k,
                                                                  const uint16_t* v, int32_t* status, int pos_limit) {
  const int b = blockIdx.y, i = blockIdx.x, pos = kv.len[b] + i;
  if (pos < 0 || pos >= pos_limit) {  // (the host's bound was wrong)
    if (threadIdx.x == 0) set_status(status, kStatusKvCapacity);
    return;
  }
  ring_put(kv.ring, layer, b, pos % kv.ring.capacity,
           ((size_t)b * n + i) * kv.ring.n_kv_heads * kv.ring.head_dim, k, v);
}

// Grid (kv heads / kSealHeads, layers, batch).  Most calls complete no block of
// most sequences: such a workgroup ends after reading two words.  A commit over 8 layers,
// 7B-like, takes 3 us longer than over a bf16 cache where no block is completed, 8 where
// one sequence completes one, 30 where 16 do.  Blocks of one call are taken in turn:
// advances by 512 and 2048 rows (8 and 32 blocks, 8 layers) take 82 and 362 us,
// 1.2 and 1.1 TB/s.
constexpr int kSealHeads = 4;
template <int HD>
__global__ __launch_bounds__(kCopyThreads) void kv8_seal_kernel(Kv8Layout kv, int c0, int n, int is_commit,
                                                                CommitArgs cm) {
  const int b = blockIdx.z, layer = blockIdx.y, G = kv.ring.n_kv_heads;
  const int from = kv.len[b] + c0;
  int step = n;
  if (is_commit) step = commit_step(cm, b);
  const int first = from / kF8Block, last = min(from + step, kv.capacity) / kF8Block;
  for (int blk = first; blk < last; ++blk) {
    const int w0 = blk * kF8Block % kv.ring.capacity;
    for (int g = blockIdx.x * kSealHeads; g < min(G, ((int)blockIdx.x + 1) * kSealHeads); ++g) {
      const uint16_t* src = k_block<uint16_t>(kv.ring, layer, b, g);
      quantize_block<HD>(
          [&](int pos, int dim) {
            return *(const u32x4*)(src + KvIndex<uint16_t>::k(w0 + pos, dim, HD, kv.ring.capacity));
          },
          [] {},
          [&](int pos, int dim) {
            return *(const u32x4*)(src + KvIndex<uint16_t>::v(w0 + pos, dim, HD, kv.ring.capacity));
          },
          kv.code_base(layer, b, g) + (size_t)blk * 2 * kF8Block * HD, kv.scale_base(layer, b, g) + 2 * (size_t)blk);
    }
  }
}

__global__ void kv_advance_kernel(int B, int n, int32_t* len) {
  for (int b = threadIdx.x; b < B; b += blockDim.x) len[b] += n;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }
size_t counter_count(int B, int G, int window) { return (size_t)B * G * kF8TilesPerSlot * window; }
size_t ring_bytes(int L, int B, int G, int hd, int window) { return align256((size_t)L * B * G * 2 * window * hd * 2); }
size_t scale_bytes(int L, int B, int G, int cap) { return align256((size_t)L * B * G * 2 * (cap / kF8Block) * 4); }

}  // namespace

size_t kv8_bytes(int n_layers, int batch, int n_kv_heads, int head_dim, int capacity, int window) {
  return align256(counter_count(batch, n_kv_heads, window) * 4) +
         ring_bytes(n_layers, batch, n_kv_heads, head_dim, window) + scale_bytes(n_layers, batch, n_kv_heads, capacity) +
         (size_t)n_layers * batch * n_kv_heads * 2 * (size_t)capacity * head_dim;
}

Kv8Layout kv8_layout(void* data, const int32_t* len, int n_layers, int batch, int n_kv_heads, int head_dim,
                     int capacity, int window) {
  char* p = (char*)data;
  Kv8Layout l{};
  l.counters = (uint32_t*)p;
  p += align256(counter_count(batch, n_kv_heads, window) * 4);
  l.ring = KvLayout{p, batch, window, n_kv_heads, head_dim, SPECDEC_BF16};
  p += ring_bytes(n_layers, batch, n_kv_heads, head_dim, window);
  l.scales = (float*)p;
  p += scale_bytes(n_layers, batch, n_kv_heads, capacity);
  l.codes = (unsigned char*)p;
  l.len = len;
  l.capacity = capacity;
  return l;
}

hipError_t launch_kv8_init(const Kv8Layout& kv, hipStream_t s) {
  return launch_fill_u32(kv.counters, counter_count(kv.ring.batch, kv.ring.n_kv_heads, kv.ring.capacity), 0u, s);
}

#define SD_BY_HEAD_DIM(hd, CALL)              \
  switch (hd) {                               \
    case 32: CALL(32); break;                 \
    case 64: CALL(64); break;                 \
    case 128: CALL(128); break;               \
    default: return hipErrorInvalidValue;     \
  }

hipError_t launch_kv8_write(const Kv8Layout& kv, int layer, int b, int pos0, int n, const void* k, const void* v,
                            hipStream_t s) {
  if (n <= 0) return hipSuccess;
  const int n_whole = n / kF8Block, n_ring = std::min(n, kv.ring.capacity);
  const dim3 grid(n_whole * kv.ring.n_kv_heads + n_ring);
#define SD_W(HD)                                                                                                \
  hipLaunchKernelGGL((kv8_write_kernel<HD>), grid, dim3(kCopyThreads), 0, s, kv, layer, b, pos0, n, n_whole, n_ring, \
                     (const uint16_t*)k, (const uint16_t*)v)
  SD_BY_HEAD_DIM(kv.ring.head_dim, SD_W)
#undef SD_W
  return hipGetLastError();
}

hipError_t launch_kv8_read(const Kv8Layout& kv, int layer, int b, int pos0, int n, void* k, void* v, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  const dim3 grid(((pos0 + n - 1) / kF8Block - pos0 / kF8Block + 1) * kv.ring.n_kv_heads);
#define SD_R(HD)                                                                                                   \
  hipLaunchKernelGGL((kv8_read_kernel<HD>), grid, dim3(kCopyThreads), 0, s, kv, layer, b, pos0, n, (uint16_t*)k, \
                     (uint16_t*)v)
  SD_BY_HEAD_DIM(kv.ring.head_dim, SD_R)
#undef SD_R
  return hipGetLastError();
}

hipError_t launch_kv8_append(const Kv8Layout& kv, int layer, int n, const void* k, const void* v, int32_t* status,
                             int pos_limit, hipStream_t s) {
  hipLaunchKernelGGL(kv8_append_kernel, dim3(n, kv.ring.batch), dim3(kCopyThreads), 0, s, kv, layer, n,
                     (const uint16_t*)k, (const uint16_t*)v, status, pos_limit);
  return hipGetLastError();
}

hipError_t launch_kv8_seal(const Kv8Layout& kv, int n_layers, int c0, int n, const CommitArgs* commit, hipStream_t s) {
  const dim3 grid((kv.ring.n_kv_heads + kSealHeads - 1) / kSealHeads, n_layers, kv.ring.batch);
  const CommitArgs cm = commit ? *commit : CommitArgs{};
#define SD_S(HD) \
  hipLaunchKernelGGL((kv8_seal_kernel<HD>), grid, dim3(kCopyThreads), 0, s, kv, c0, n, commit ? 1 : 0, cm)
  SD_BY_HEAD_DIM(kv.ring.head_dim, SD_S)
#undef SD_S
  return hipGetLastError();
}

hipError_t launch_kv_advance(int batch, int n, int32_t* len, hipStream_t s) {
  hipLaunchKernelGGL(kv_advance_kernel, dim3(1), dim3(256), 0, s, batch, n, len);
  return hipGetLastError();
}

}  // namespace specdec
