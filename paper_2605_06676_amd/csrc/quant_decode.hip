// One decode step of grouped-query attention over the packed cache in 8 bits (lkv_quant.h): decode.hip's operator with half the
// bytes per row.
//
// Work decomposition.  A chunk is up to C rows of one segment, C a multiple of the 32 rows of a scale; chunk j of segment s has number
// cap[s] / C + s + j, which orders them as scale numbers order the blocks, so that a wave finds its segment by a search over
// the segments' first rows and no table has to be made.  A segment always has its number of chunk 0, where an empty one gets its
// zeros.  The four waves of a block take the chunk's tiles of 32 rows in turn and merge their running maximum, denominator and sums in LDS; a
// segment of one chunk is finished there, the others leave partials, numbered as the chunks, to a second kernel.
//
// Arithmetic.  Both products run on the matrix cores in bf16, into which every code converts exactly; the scales never touch
// the operands: the keys' scale multiplies the scores, the values' scale the probabilities.
//   S^T[token, head] = K[token, :] . Q[head, :]^T      (A = K tile, B = Q^T)
//   O[head, ch]     += P[head, token] V[token, ch]     (A = P,      B = V tile)
// Nothing is staged in LDS.  The first product's operand needs 8 channels of a token in a lane: a sum over channels may
// take them in any order, so a lane takes 16 contiguous bytes of its token's row for two steps and Q's operand is read in that
// order.  The second needs 8 tokens of a channel in a lane: it loads 8 bytes, 8 channels, of each of the 8 tokens whose scores the
// first product left with it, and turns the 8 x 8 bytes about with byte permutes (32 for a tile); column c of the m-th
// product then is channel 8 c + m, and a lane ends with 8 contiguous channels of the output.  Softmax runs in fp32 in the
// log2 domain; P is rounded to bf16 and what the rounding left is multiplied too, as in decode.hip.
#include <type_traits>

#include "lkv_kernels.h"

namespace lkv {

constexpr int kQdThreads = 256;
constexpr int kQdWaves = kQdThreads / 64;
constexpr int kQdTile = kQuantBlock;
constexpr int kQdMinChunk = 128;        // rows: a tile for every wave
constexpr int kQdTargetChunks = 1024;   // chunks that a launch wants
constexpr int kQdMergeThreads = kHeadDim;
constexpr float kQdLog2e = 1.4426950408889634f;
constexpr float kQdLn2 = 0.6931471805599453f;

__device__ __forceinline__ float qd_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2_t;

// Eight codes to bf16, exact.
template <int kFormat>
__device__ __forceinline__ bf16x8_t codes_to_bf16(uint32_t lo, uint32_t hi) {
  uint4 w;
  if constexpr (kFormat == kQuantE4m3) {
    w.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
    w.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
    w.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
    w.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
  } else {
    float f[4], g[4];
    unquant4<kFormat>(lo, f);
    unquant4<kFormat>(hi, g);
    w.x = __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)f[0], (__bf16)f[1]});
    w.y = __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)f[2], (__bf16)f[3]});
    w.z = __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)g[0], (__bf16)g[1]});
    w.w = __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)g[2], (__bf16)g[3]});
  }
  return __builtin_bit_cast(bf16x8_t, w);
}

// Bytes of four rows turned about: out[b] holds byte b of a, b, c and d.
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&out)[4]) {
  const uint32_t ab_lo = __builtin_amdgcn_perm(b, a, 0x05010400u), ab_hi = __builtin_amdgcn_perm(b, a, 0x07030602u);
  const uint32_t cd_lo = __builtin_amdgcn_perm(d, c, 0x05010400u), cd_hi = __builtin_amdgcn_perm(d, c, 0x07030602u);
  out[0] = __builtin_amdgcn_perm(cd_lo, ab_lo, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(cd_lo, ab_lo, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(cd_hi, ab_hi, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(cd_hi, ab_hi, 0x07060302u);
}

// What a lane holds of a tile of 32 rows, and the tile's scales.
struct QdTile {
  uint4 k[2][2];   // [16-token half][64-channel half]: token 16 h + c, bytes 64 w + 16 r .. + 15
  uint2 v[2][4];   // token 16 h + 4 r + e, bytes 8 c .. 8 c + 7
  float ks, vs;
};

template <int kFormat>
__global__ void __launch_bounds__(kQdThreads)
quant_decode_kernel(const uint16_t* __restrict__ q, QuantRows rows, const int32_t* __restrict__ cap,
                    const int32_t* __restrict__ lengths /* rows in use, or null: all of them */, int n_segments, int chunk_rows, int G,
                    float scale, float* __restrict__ out, float* __restrict__ lse, float* __restrict__ ws_acc,
                    float* __restrict__ ws_m, float* __restrict__ ws_l) {
  extern __shared__ __align__(16) float merge_lds[];   // [waves][G][128] sums, then [waves][G] maxima, then denominators
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane >> 4, c = lane & 15;
  const int number = blockIdx.x;
  auto first_chunk = [&](int s) { return cap[s] / chunk_rows + s; };
  const int s = wave_upper_key(n_segments, number, lane, first_chunk);
  const int lo = cap[s];
  const int len = max(lengths != nullptr ? lengths[s] : cap[s + 1] - lo, 0);
  const int64_t ahead = (int64_t)(number - first_chunk(s)) * chunk_rows;   // rows of the segment ahead of this chunk
  if (ahead >= len) {
    if (ahead == 0) {   // an empty segment: zero output, lse = -inf
      for (int o = tid; o < G * kHeadDim; o += kQdThreads) out[(size_t)s * G * kHeadDim + o] = 0.f;
      if (lse != nullptr && tid < G) lse[(size_t)s * G + tid] = -INFINITY;
    }
    return;
  }
  const int n_rows = (int)min((int64_t)chunk_rows, len - ahead);
  const int n_tiles = (n_rows + kQdTile - 1) / kQdTile;
  const int64_t row0 = (int64_t)lo + ahead;
  const int scale0 = quant_first_scale(lo, s) + (int)(ahead / kQuantBlock);
  const uint8_t* kbase = rows.k + row0 * kHeadDim;
  const uint8_t* vbase = rows.v + row0 * kHeadDim;

  auto load_tile = [&](QdTile& x, int t) __attribute__((always_inline)) {
    const int last = n_rows - 1;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* p = kbase + (int64_t)min(t * kQdTile + 16 * h + c, last) * kHeadDim + 16 * r;   // past the end: the last row again
      x.k[h][0] = load_stream16(reinterpret_cast<const uint4*>(p));
      x.k[h][1] = load_stream16(reinterpret_cast<const uint4*>(p + 64));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned long long w = __builtin_nontemporal_load(reinterpret_cast<const unsigned long long*>(
            vbase + (int64_t)min(t * kQdTile + 16 * h + 4 * r + e, last) * kHeadDim + 8 * c));
        x.v[h][e] = make_uint2((uint32_t)w, (uint32_t)(w >> 32));
      }
    x.ks = rows.k_scale[scale0 + t];
    x.vs = rows.v_scale[scale0 + t];
  };

  // B operand of the first product, columns past the group repeat its last head and are not used
  bf16x8_t qfrag[2][2];
  {
    const uint4* row = reinterpret_cast<const uint4*>(q + ((size_t)s * G + min(c, G - 1)) * kHeadDim);
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int j = 0; j < 2; ++j) qfrag[w][j] = __builtin_bit_cast(bf16x8_t, row[8 * w + 2 * r + j]);
  }
  float m_run = -INFINITY, l_run = 0.f;   // running maximum of head c (log2 domain) in its four lanes, this lane's share of the denominator
  f32x4_t acc[8];                         // O[head 4 r + e][channel 8 c + m]
#pragma unroll
  for (int m = 0; m < 8; ++m) acc[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const float qscale = scale * kQdLog2e;

  QdTile next;
  if (wave < n_tiles) load_tile(next, wave);
#pragma unroll 1
  for (int t = wave; t < n_tiles; t += kQdWaves) {
    const QdTile x = next;
    if (t + kQdWaves < n_tiles) load_tile(next, t + kQdWaves);
    f32x4_t sacc[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sacc[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        sacc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16<kFormat>(x.k[h][w].x, x.k[h][w].y), qfrag[w][0], sacc[h], 0, 0, 0);
        sacc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16<kFormat>(x.k[h][w].z, x.k[h][w].w), qfrag[w][1], sacc[h], 0, 0, 0);
      }
    }
    const float ts = qscale * x.ks;
    float p[8];
    float mx = m_run;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[4 * h + e] = t * kQdTile + 16 * h + 4 * r + e < n_rows ? sacc[h][e] * ts : -INFINITY;
        mx = fmaxf(mx, p[4 * h + e]);
      }
    mx = max_over_row_blocks(mx);
    const float alpha = qd_exp2(m_run - mx);   // 0 on the first tile
    m_run = mx;
    float psum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) { p[i] = qd_exp2(p[i] - mx); psum += p[i]; }
    l_run = l_run * alpha + psum;
    bf16x8_t phigh, plow;   // the weights of the values' codes: rounded, and what the rounding left
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float w = p[i] * x.vs;
      phigh[i] = (__bf16)w;
      plow[i] = (__bf16)(w - (float)phigh[i]);
    }
    if (__ballot(alpha != 1.f) != 0ull) {   // a maximum moved: the sums' rows are heads 4 r + e
      float al[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) al[e] = __shfl(alpha, 4 * r + e, 64);
#pragma unroll
      for (int m = 0; m < 8; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[m][e] *= al[e];
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {   // channels 8 c + 4 b .. + 3
      uint32_t v0[4], v1[4];
      if (b == 0) {
        transpose4(x.v[0][0].x, x.v[0][1].x, x.v[0][2].x, x.v[0][3].x, v0);
        transpose4(x.v[1][0].x, x.v[1][1].x, x.v[1][2].x, x.v[1][3].x, v1);
      } else {
        transpose4(x.v[0][0].y, x.v[0][1].y, x.v[0][2].y, x.v[0][3].y, v0);
        transpose4(x.v[1][0].y, x.v[1][1].y, x.v[1][2].y, x.v[1][3].y, v1);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x8_t vb = codes_to_bf16<kFormat>(v0[i], v1[i]);
        acc[4 * b + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(phigh, vb, acc[4 * b + i], 0, 0, 0);
        acc[4 * b + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(plow, vb, acc[4 * b + i], 0, 0, 0);
      }
    }
  }
  l_run = sum_over_row_blocks(l_run);

  // the four waves' sums meet in LDS
  const int per_wave = G * kHeadDim;
  float* m_lds = merge_lds + kQdWaves * per_wave;
  float* l_lds = m_lds + kQdWaves * G;
  if (r == 0 && c < G) { m_lds[wave * G + c] = m_run; l_lds[wave * G + c] = l_run; }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int h = 4 * r + e;
    if (h < G) {
      float4* dst = reinterpret_cast<float4*>(merge_lds + wave * per_wave + h * kHeadDim + 8 * c);
      dst[0] = make_float4(acc[0][e], acc[1][e], acc[2][e], acc[3][e]);
      dst[1] = make_float4(acc[4][e], acc[5][e], acc[6][e], acc[7][e]);
    }
  }
  __syncthreads();
  const bool whole = len <= chunk_rows;
  for (int o = tid; o < per_wave; o += kQdThreads) {
    const int h = o / kHeadDim;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < kQdWaves; ++w) mx = fmaxf(mx, m_lds[w * G + h]);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float num = 0.f, den = 0.f;
#pragma unroll
    for (int w = 0; w < kQdWaves; ++w) {
      const float weight = qd_exp2(m_lds[w * G + h] - ref);   // 0 for a wave without a tile
      num = fmaf(merge_lds[w * per_wave + o], weight, num);
      den = fmaf(l_lds[w * G + h], weight, den);
    }
    if (whole) {
      out[(size_t)s * per_wave + o] = num / den;
      if (o % kHeadDim == 0 && lse != nullptr) lse[(size_t)s * G + h] = mx * kQdLn2 + __logf(den);
    } else {
      ws_acc[(size_t)number * per_wave + o] = num;
      if (o % kHeadDim == 0) { ws_m[(size_t)number * G + h] = mx; ws_l[(size_t)number * G + h] = den; }
    }
  }
}

// The partials of a segment of several chunks: a block per segment and query head, a thread per channel, eight chunks' loads
// in flight together.
__global__ void __launch_bounds__(kQdMergeThreads)
quant_decode_merge_kernel(const int32_t* __restrict__ cap, const int32_t* __restrict__ lengths, int chunk_rows, int G,
                          const float* __restrict__ ws_acc, const float* __restrict__ ws_m, const float* __restrict__ ws_l,
                          float* __restrict__ out, float* __restrict__ lse) {
  const int s = blockIdx.x / G, h = blockIdx.x - s * G, ch = threadIdx.x;
  const int lo = cap[s];
  const int len = lengths != nullptr ? lengths[s] : cap[s + 1] - lo;
  if (len <= chunk_rows) return;   // finished, or empty
  const int first = lo / chunk_rows + s, n = (int)(((int64_t)len + chunk_rows - 1) / chunk_rows);
  constexpr int kU = 8;
  float mx = -INFINITY, num = 0.f, den = 0.f;
  for (int i0 = 0; i0 < n; i0 += kU) {
    float mv[kU], lv[kU], av[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const size_t at = (size_t)(first + min(i0 + u, n - 1)) * G + h;
      mv[u] = ws_m[at];
      lv[u] = ws_l[at];
      av[u] = ws_acc[at * kHeadDim + ch];
    }
    float top = mx;
#pragma unroll
    for (int u = 0; u < kU; ++u) top = fmaxf(top, mv[u]);
    const float keep = qd_exp2(mx - top);
    num *= keep;
    den *= keep;
    mx = top;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const float weight = i0 + u < n ? qd_exp2(mv[u] - top) : 0.f;
      num = fmaf(av[u], weight, num);
      den = fmaf(lv[u], weight, den);
    }
  }
  const size_t row = (size_t)s * G + h;
  out[row * kHeadDim + ch] = num / den;
  if (ch == 0 && lse != nullptr) lse[row] = mx * kQdLn2 + __logf(den);
}

// Rows of a chunk: a power of two.
static int quant_decode_chunk_rows(int64_t total_rows) {
  int c = kQdMinChunk;
  while (c < (1 << 20) && total_rows / c > kQdTargetChunks) c *= 2;
  return c;
}

static int64_t quant_decode_chunks(int n_segments, int64_t total_rows) {
  return total_rows / quant_decode_chunk_rows(total_rows) + n_segments;
}

size_t quant_decode_workspace_bytes(int n_segments, int64_t total_rows, int G) {
  const size_t bytes = (size_t)quant_decode_chunks(n_segments, total_rows) * G * (kHeadDim + 2) * sizeof(float);
  return (bytes + 255) & ~(size_t)255;
}

hipError_t launch_quant_decode(int format, int G, const void* q, const QuantRows& rows, const int32_t* cap, const int32_t* lengths,
                               int n_segments, int64_t total_rows, float scale, float* out, float* lse, float* ws, hipStream_t stream) {
  if (G < 1 || G > kDecodeMaxGroup) return hipErrorInvalidValue;
  const int chunk_rows = quant_decode_chunk_rows(total_rows);
  const int64_t chunks = quant_decode_chunks(n_segments, total_rows);
  float* ws_acc = ws;
  float* ws_m = ws + (size_t)chunks * G * kHeadDim;
  float* ws_l = ws_m + (size_t)chunks * G;
  const size_t lds = (size_t)kQdWaves * G * (kHeadDim + 2) * sizeof(float);   // at most 33 KB
  auto launch = [&](auto tag) {
    hipLaunchKernelGGL((quant_decode_kernel<decltype(tag)::value>), dim3((unsigned)chunks), dim3(kQdThreads), lds, stream,
                       static_cast<const uint16_t*>(q), rows, cap, lengths, n_segments, chunk_rows, G, scale, out, lse, ws_acc, ws_m, ws_l);
  };
  if (format == kQuantE4m3) launch(std::integral_constant<int, kQuantE4m3>{});
  else launch(std::integral_constant<int, kQuantInt8>{});
  if (total_rows > chunk_rows)   // else no segment has two chunks
    hipLaunchKernelGGL(quant_decode_merge_kernel, dim3((unsigned)((int64_t)n_segments * G)), dim3(kQdMergeThreads), 0, stream, cap, lengths,
                       chunk_rows, G, ws_acc, ws_m, ws_l, out, lse);
  return hipGetLastError();
}

}  // namespace lkv
