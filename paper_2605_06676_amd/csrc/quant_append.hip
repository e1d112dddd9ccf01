// One generated token joins a packed cache in 8 bits: its key is turned by its position (rope.hip's arithmetic) and rounded
// to bf16, the LKV-T score of key and value is stored as lkv_append stores it, and the row goes to the first spare row of
// every segment.
//
// The row's block of 32 may have rows already.  Its scale becomes the larger of what it is and what the new row needs; where it
// grows, the rows that are there are requantised (at most 31, 4 KB of K or V; lkv_quant.h says what that costs in precision).
// Nobody else writes these rows: a block belongs to one segment and a segment to one wave.
//
// A few hundred bytes per segment, and the scorer's weights: launch-latency sized, a chain of loads that wait for nothing but
// each other.  Linear scorer or none: one wave per segment; lane i holds pair i of the key, which are the channels that turn together, and
// after that channels 2i and 2i + 1 of both.  MLP scorer: one block per segment, whose four waves share the hidden units and ask for
// their weights before anything else (1792 segments, hidden 64, rotation: 15.0 us with a wave per segment that reads its
// weights sixteen units at a time, 8.6 us).
#include <type_traits>

#include "lkv_act.h"
#include "lkv_kernels.h"

namespace lkv {

constexpr int kQaThreads = 256;
constexpr int kQaWaves = kQaThreads / 64;

// Rows row0 .. row0 + n - 1 of one side, n <= 32, from the scale `old` to `scale`; by a whole wave.
template <int kFormat>
__device__ __forceinline__ void requantise_rows(uint8_t* codes, size_t row0, int n, float old, float scale, int lane) {
  const float ratio = old * quant_inverse(scale);
  const int c = lane & 15;
  for (int j = lane >> 4; j < n; j += 4) {
    uint2* p = reinterpret_cast<uint2*>(codes + (row0 + j) * kHeadDim + c * 8);
    const uint2 w = *p;
    float f[4], g[4];
    unquant4<kFormat>(w.x, f);
    unquant4<kFormat>(w.y, g);
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] *= ratio; g[i] *= ratio; }
    *p = make_uint2(quant4<kFormat>(f[0], f[1], f[2], f[3]), quant4<kFormat>(g[0], g[1], g[2], g[3]));
  }
}

__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

// One side of the new row: two channels a lane; `old` is its block's scale, 0 for a block that it opens.
template <int kFormat>
__device__ __forceinline__ void append_side(uint8_t* codes, float* scales, int number, size_t row, int inside, float old, float x0, float x1,
                                            int lane) {
  const float need = quant_scale<kFormat>(__uint_as_float(wave_max_u32(max(finite_bits(x0), finite_bits(x1)))));
  const float scale = fmaxf(old, need);
  const float inv = quant_inverse(scale);
  const uint32_t w = quant4<kFormat>(quant_tame<kFormat>(x0 * inv), quant_tame<kFormat>(x1 * inv), 0.f, 0.f);
  if (old > 0.f && old < scale) requantise_rows<kFormat>(codes, row - inside, inside, old, scale, lane);   // the same in the whole wave
  if (lane == 0) scales[number] = scale;
  *reinterpret_cast<uint16_t*>(codes + row * kHeadDim + lane * 2) = (uint16_t)w;
}

// Where the new row goes.
struct AppendPlace {
  int used, cap;
  bool full;
  __device__ __forceinline__ AppendPlace(const int32_t* __restrict__ cap_offsets, const int32_t* len, int seg) {
    used = len[seg];
    cap = cap_offsets[seg];
    full = used < 0 || (int64_t)cap + used >= (int64_t)cap_offsets[seg + 1];
  }
  __device__ __forceinline__ size_t row() const { return (size_t)cap + (size_t)used; }
  __device__ __forceinline__ int inside() const { return used % kQuantBlock; }
  __device__ __forceinline__ int number(int seg) const { return quant_first_scale(cap, seg) + used / kQuantBlock; }
  // a block's first row finds whatever an earlier use has left there
  __device__ __forceinline__ float scale(const float* scales, int seg) const { return inside() > 0 ? scales[number(seg)] : 0.f; }
};

// The new key, turned, to x (LDS, bf16); by a whole wave.
template <bool kRotary>
__device__ __forceinline__ void stage_key(const uint16_t* __restrict__ key, const RotaryArgs& rot, const int32_t* __restrict__ positions, int seq,
                                          uint16_t* x, int lane) {
  if constexpr (kRotary) {
    const int half = rot.rotary_dim >> 1;
    const bool turned = lane < half;
    const bool split = turned && rot.pairs == 0;
    const int ch0 = split ? lane : 2 * lane, ch1 = split ? lane + half : 2 * lane + 1;
    const uint16_t ka = key[ch0], kb = key[ch1];
    float a = __uint_as_float((uint32_t)ka << 16), b = __uint_as_float((uint32_t)kb << 16);
    float c, s;
    rotary_cos_sin(positions[seq], rot.inv_freq[min(lane, half - 1)], rot.factor, &c, &s);
    rotary_turn(a, b, c, s);
    x[ch0] = turned ? __builtin_bit_cast(uint16_t, (__bf16)a) : ka;
    x[ch1] = turned ? __builtin_bit_cast(uint16_t, (__bf16)b) : kb;
  } else {
    reinterpret_cast<uint32_t*>(x)[lane] = reinterpret_cast<const uint32_t*>(key)[lane];
  }
}

template <int kFormat, bool kRotary>
__global__ void __launch_bounds__(kQaThreads)
quant_append_kernel(int n_segments, int heads_per_seq, int n_kv_heads, AppendScorer sc, RotaryArgs rot,
                    const int32_t* __restrict__ positions, const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new,
                    QuantRows rows, float* __restrict__ up, const int32_t* __restrict__ cap, int32_t* __restrict__ len,
                    int32_t* __restrict__ overflow) {
  __shared__ __align__(16) uint16_t x_lds[kQaWaves][kHeadDim];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int seg = blockIdx.x * kQaWaves + wave;
  if (seg >= n_segments) return;   // the whole wave
  uint16_t* x = x_lds[wave];
  const AppendPlace place(cap, len, seg);
  const uint32_t vw = reinterpret_cast<const uint32_t*>(v_new + (size_t)seg * kHeadDim)[lane];
  stage_key<kRotary>(k_new + (size_t)seg * kHeadDim, rot, positions, seg / heads_per_seq, x, lane);
  if (place.full) {   // nothing is written, the caller must re-evict first
    if (lane == 0 && overflow != nullptr) *overflow = 1;
    return;
  }
  const float k_old = place.scale(rows.k_scale, seg), v_old = place.scale(rows.v_scale, seg);
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const uint32_t kw = reinterpret_cast<const uint32_t*>(x)[lane];
  const float k0 = bf16_lo(kw), k1 = bf16_hi(kw), v0 = bf16_lo(vw), v1 = bf16_hi(vw);
  if (sc.w1 != nullptr) {   // linear: w . [k ; v] + b
    const int lh = seg % heads_per_seq;
    const size_t srow = sc.per_head ? (size_t)lh : (size_t)(lh / n_kv_heads);
    const uint32_t* w = reinterpret_cast<const uint32_t*>(sc.w1 + srow * 2 * kHeadDim);
    const uint32_t wk = w[lane], wv = w[64 + lane];
    float u = fmaf(bf16_hi(wv), v1, fmaf(bf16_lo(wv), v0, fmaf(bf16_hi(wk), k1, bf16_lo(wk) * k0)));
    u = sum_over_row_blocks(row16_allreduce_sum(u)) + sc.b1[srow];
    if (lane == 0) up[place.row()] = u;
  }
  append_side<kFormat>(rows.k, rows.k_scale, place.number(seg), place.row(), place.inside(), k_old, k0, k1, lane);
  append_side<kFormat>(rows.v, rows.v_scale, place.number(seg), place.row(), place.inside(), v_old, v0, v1, lane);
  if (lane == 0) len[seg] = place.used + 1;
}

// MLP scorer: a block per segment, 16 hidden units at a time to a wave.  Sixteen lanes share a unit, whose weights they load as
// 256 contiguous bytes for the key and for the value each (as a matrix product, a lane's 16 bytes are 512 from its neighbour's:
// 12.2 us for the call above); lane (r, c) has units 4 i + r and channels 8 c .. 8 c + 7 of both.
// kQaTiles: of a wave, 64 hidden units of the block each; with the registers of two, fewer waves are resident (64 units 9.3 us).
constexpr int kQaUnits = 16 * kQaWaves;
template <int kFormat, bool kRotary, int kQaTiles>
__global__ void __launch_bounds__(kQaThreads)
quant_append_mlp_kernel(int heads_per_seq, int n_kv_heads, AppendScorer sc, RotaryArgs rot, const int32_t* __restrict__ positions,
                        const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new, QuantRows rows, float* __restrict__ up,
                        const int32_t* __restrict__ cap, int32_t* __restrict__ len, int32_t* __restrict__ overflow) {
  __shared__ __align__(16) uint16_t x[2 * kHeadDim];   // key, then value
  __shared__ float part_lds[kQaWaves];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane >> 4, c = lane & 15;
  const int seg = blockIdx.x;
  const int lh = seg % heads_per_seq;
  const size_t srow = sc.per_head ? (size_t)lh : (size_t)(lh / n_kv_heads);
  const int hidden = sc.hidden;
  uint4 wk[kQaTiles][4], wv[kQaTiles][4];
  float b1[kQaTiles][4], w2[kQaTiles][4];
#pragma unroll
  for (int i = 0; i < kQaTiles; ++i) {
    const int j0 = (wave + i * kQaWaves) * 16;   // units past the last one repeat it and are weighted out
    if (i > 0 && j0 >= hidden) break;            // the same in the whole wave
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const size_t unit = srow * hidden + min(j0 + 4 * e + r, hidden - 1);
      const uint4* wrow = reinterpret_cast<const uint4*>(sc.w1 + unit * 2 * kHeadDim);
      wk[i][e] = wrow[c];
      wv[i][e] = wrow[16 + c];
      b1[i][e] = sc.b1[unit];
      w2[i][e] = sc.w2[unit];
    }
  }
  const AppendPlace place(cap, len, seg);
  if (place.full) {   // nothing is written, the caller must re-evict first
    if (threadIdx.x == 0 && overflow != nullptr) *overflow = 1;
    return;
  }
  float old = 0.f;   // wave 0 has the key, wave 1 the value
  if (wave == 0) {
    old = place.scale(rows.k_scale, seg);
    stage_key<kRotary>(k_new + (size_t)seg * kHeadDim, rot, positions, seg / heads_per_seq, x, lane);
  } else if (wave == 1) {
    old = place.scale(rows.v_scale, seg);
    reinterpret_cast<uint32_t*>(x + kHeadDim)[lane] = reinterpret_cast<const uint32_t*>(v_new + (size_t)seg * kHeadDim)[lane];
  }
  __syncthreads();
  float xk[8], xv[8];
  unpack8(reinterpret_cast<const uint4*>(x)[c], xk);
  unpack8(reinterpret_cast<const uint4*>(x)[16 + c], xv);
  float part = 0.f;
#pragma unroll
  for (int i = 0; i < kQaTiles; ++i) {
    const int j0 = (wave + i * kQaWaves) * 16;
    if (j0 >= hidden) break;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float fk[8], fv[8], z = 0.f;
      unpack8(wk[i][e], fk);
      unpack8(wv[i][e], fv);
#pragma unroll
      for (int k = 0; k < 8; ++k) z = fmaf(fv[k], xv[k], fmaf(fk[k], xk[k], z));
      z = row16_allreduce_sum(z) + b1[i][e];
      const float a = sc.act == kActSilu ? activation<kActSilu>(z) : activation<kActGelu>(z);
      part += j0 + 4 * e + r < hidden ? w2[i][e] * a : 0.f;
    }
  }
  part = sum_over_row_blocks(part);   // the same in the 16 lanes of a unit
  if (lane == 0) part_lds[wave] = part;
  __syncthreads();
  if (wave < 2) {
    const uint32_t xw = reinterpret_cast<const uint32_t*>(x + wave * kHeadDim)[lane];
    append_side<kFormat>(wave == 0 ? rows.k : rows.v, wave == 0 ? rows.k_scale : rows.v_scale, place.number(seg), place.row(), place.inside(), old,
                         bf16_lo(xw), bf16_hi(xw), lane);
  } else if (wave == 2) {
    if (lane == 0) up[place.row()] = (part_lds[0] + part_lds[1]) + (part_lds[2] + part_lds[3]) + (sc.b2 != nullptr ? sc.b2[srow] : 0.f);
  } else if (lane == 0) {
    len[seg] = place.used + 1;
  }
}

void launch_quant_append(int format, int n_segments, int heads_per_seq, int n_kv_heads, const AppendScorer& scorer,
                         const RotaryArgs* rotary, const int32_t* positions, const void* k_new, const void* v_new,
                         const QuantRows& rows, float* up, const int32_t* cap, int32_t* len, int32_t* overflow, hipStream_t stream) {
  const RotaryArgs none = {};
  auto launch = [&](auto format_tag, auto rotary_tag) {
    auto launch_mlp = [&](auto tiles_tag) {
      hipLaunchKernelGGL((quant_append_mlp_kernel<decltype(format_tag)::value, decltype(rotary_tag)::value, decltype(tiles_tag)::value>),
                         dim3(n_segments), dim3(kQaThreads), 0, stream, heads_per_seq, n_kv_heads, scorer,
                         rotary != nullptr ? *rotary : none, positions, static_cast<const uint16_t*>(k_new),
                         static_cast<const uint16_t*>(v_new), rows, up, cap, len, overflow);
    };
    if (scorer.w1 != nullptr && scorer.kind != 0) {
      if (scorer.hidden <= kQaUnits) launch_mlp(std::integral_constant<int, 1>{});
      else launch_mlp(std::integral_constant<int, 2>{});
    } else {
      hipLaunchKernelGGL((quant_append_kernel<decltype(format_tag)::value, decltype(rotary_tag)::value>),
                       dim3((n_segments + kQaWaves - 1) / kQaWaves), dim3(kQaThreads), 0, stream, n_segments, heads_per_seq, n_kv_heads,
                       scorer, rotary != nullptr ? *rotary : none, positions, static_cast<const uint16_t*>(k_new),
                       static_cast<const uint16_t*>(v_new), rows, up, cap, len, overflow);
    }
  };
  auto launch_format = [&](auto format_tag) {
    if (rotary != nullptr) launch(format_tag, std::true_type{}); else launch(format_tag, std::false_type{});
  };
  if (format == kQuantE4m3) launch_format(std::integral_constant<int, kQuantE4m3>{});
  else launch_format(std::integral_constant<int, kQuantInt8>{});
}

}  // namespace lkv
