// One generated token joins a packed cache in 8 bits: its key is turned by its position (rope.hip's arithmetic) and rounded
// to bf16, the LKV-T score of key and value is stored as lkv_append stores it, and the row goes to the first spare row of
// every segment.
//
// The row's block of 32 may have rows already.  Its scale becomes the larger of what it is and what the new row needs; where it
// grows, the rows that are there are requantised (at most 31, 4 KB of K or V; lkv_quant.h says what that costs in precision).
// Nobody else writes these rows: a block belongs to one segment and a segment to one wave.
//
// A few hundred bytes per segment: launch-latency sized.  One wave per segment; lane i holds pair i of the key, which are the channels
// that turn together, and after that channels 2i and 2i + 1 of both.
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

// One side of the new row: two channels a lane.
template <int kFormat>
__device__ __forceinline__ void append_side(uint8_t* codes, float* scales, int number, size_t row, int inside, float x0, float x1, int lane) {
  const float old = inside > 0 ? scales[number] : 0.f;   // a block's first row finds whatever an earlier use has left
  const float need = quant_scale<kFormat>(__uint_as_float(wave_max_u32(max(finite_bits(x0), finite_bits(x1)))));
  const float scale = fmaxf(old, need);
  const float inv = quant_inverse(scale);
  const uint32_t w = quant4<kFormat>(quant_tame<kFormat>(x0 * inv), quant_tame<kFormat>(x1 * inv), 0.f, 0.f);
  if (old < scale) {   // the same in the whole wave
    if (old > 0.f) requantise_rows<kFormat>(codes, row - inside, inside, old, scale, lane);
    if (lane == 0) scales[number] = scale;
  } else if (inside == 0 && lane == 0) {
    scales[number] = scale;   // a row of zeros that opens a block
  }
  *reinterpret_cast<uint16_t*>(codes + row * kHeadDim + lane * 2) = (uint16_t)w;
}

template <int kFormat, bool kRotary>
__global__ void __launch_bounds__(kQaThreads)
quant_append_kernel(int n_segments, int heads_per_seq, int n_kv_heads, AppendScorer sc, RotaryArgs rot,
                    const int32_t* __restrict__ positions, const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new,
                    QuantRows rows, float* __restrict__ up, const int32_t* __restrict__ cap, int32_t* __restrict__ len,
                    int32_t* __restrict__ overflow) {
  __shared__ __align__(16) float x_lds[kQaWaves][2 * kHeadDim];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int seg = blockIdx.x * kQaWaves + wave;
  if (seg >= n_segments) return;   // the whole wave
  float* x = x_lds[wave];
  const int used = len[seg], cap0 = cap[seg], cap1 = cap[seg + 1];

  const uint32_t vw = reinterpret_cast<const uint32_t*>(v_new + (size_t)seg * kHeadDim)[lane];
  const float v0 = bf16_lo(vw), v1 = bf16_hi(vw);
  float k0, k1;
  if constexpr (kRotary) {
    const int half = rot.rotary_dim >> 1;
    const bool turned = lane < half;
    const bool split = turned && rot.pairs == 0;
    const int ch0 = split ? lane : 2 * lane, ch1 = split ? lane + half : 2 * lane + 1;
    float a = __uint_as_float((uint32_t)k_new[(size_t)seg * kHeadDim + ch0] << 16);
    float b = __uint_as_float((uint32_t)k_new[(size_t)seg * kHeadDim + ch1] << 16);
    if (turned) {
      float c, s;
      rotary_cos_sin(positions[seg / heads_per_seq], rot.inv_freq[lane], rot.factor, &c, &s);
      rotary_turn(a, b, c, s);
    }
    x[ch0] = (float)(__bf16)a;
    x[ch1] = (float)(__bf16)b;
  } else {
    const uint32_t kw = reinterpret_cast<const uint32_t*>(k_new + (size_t)seg * kHeadDim)[lane];
    x[2 * lane] = bf16_lo(kw);
    x[2 * lane + 1] = bf16_hi(kw);
  }
  x[kHeadDim + 2 * lane] = v0;
  x[kHeadDim + 2 * lane + 1] = v1;
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  k0 = x[2 * lane];
  k1 = x[2 * lane + 1];

  const int64_t row = (int64_t)cap0 + used;
  if (used < 0 || row >= (int64_t)cap1) {   // the segment is full: nothing is written, the caller must re-evict first
    if (lane == 0 && overflow != nullptr) *overflow = 1;
    return;
  }

  if (sc.w1 != nullptr) {
    const int lh = seg % heads_per_seq;
    const size_t srow = sc.per_head ? (size_t)lh : (size_t)(lh / n_kv_heads);
    float part = 0.f;
    if (sc.kind == 0) {   // linear: w . [k ; v] + b
      const uint32_t* w = reinterpret_cast<const uint32_t*>(sc.w1 + srow * 2 * kHeadDim);
      const uint32_t wk = w[lane], wv = w[64 + lane];
      part = fmaf(bf16_hi(wv), v1, fmaf(bf16_lo(wv), v0, fmaf(bf16_hi(wk), k1, bf16_lo(wk) * k0)));
    } else {
      // lane j evaluates hidden units j and j + 64; lanes past the last one repeat unit 0 and are weighted out
      for (int j0 = 0; j0 < sc.hidden; j0 += 64) {
        const bool on = j0 + lane < sc.hidden;
        const int j = on ? j0 + lane : 0;
        const uint4* wrow = reinterpret_cast<const uint4*>(sc.w1 + (srow * sc.hidden + j) * 2 * kHeadDim);
        float z = sc.b1[srow * sc.hidden + j];
        for (int q = 0; q < 2 * kHeadDim / 8; ++q) {
          float wf[8];
          unpack8(wrow[q], wf);
#pragma unroll
          for (int i = 0; i < 8; ++i) z = fmaf(wf[i], x[q * 8 + i], z);
        }
        const float a = sc.act == kActSilu ? activation<kActSilu>(z) : activation<kActGelu>(z);
        part += on ? sc.w2[srow * sc.hidden + j] * a : 0.f;
      }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) part += __shfl_xor(part, off, 64);
    if (sc.kind == 0) part += sc.b1[srow];
    else if (sc.b2 != nullptr) part += sc.b2[srow];
    if (lane == 0) up[row] = part;
  }

  const int inside = used % kQuantBlock;
  const int number = quant_first_scale(cap0, seg) + used / kQuantBlock;
  append_side<kFormat>(rows.k, rows.k_scale, number, (size_t)row, inside, k0, k1, lane);
  append_side<kFormat>(rows.v, rows.v_scale, number, (size_t)row, inside, v0, v1, lane);
  if (lane == 0) len[seg] = used + 1;
}

void launch_quant_append(int format, int n_segments, int heads_per_seq, int n_kv_heads, const AppendScorer& scorer,
                         const RotaryArgs* rotary, const int32_t* positions, const void* k_new, const void* v_new,
                         const QuantRows& rows, float* up, const int32_t* cap, int32_t* len, int32_t* overflow, hipStream_t stream) {
  const RotaryArgs none = {};
  auto launch = [&](auto format_tag, auto rotary_tag) {
    hipLaunchKernelGGL((quant_append_kernel<decltype(format_tag)::value, decltype(rotary_tag)::value>),
                       dim3((n_segments + kQaWaves - 1) / kQaWaves), dim3(kQaThreads), 0, stream, n_segments, heads_per_seq, n_kv_heads,
                       scorer, rotary != nullptr ? *rotary : none, positions, static_cast<const uint16_t*>(k_new),
                       static_cast<const uint16_t*>(v_new), rows, up, cap, len, overflow);
  };
  auto launch_format = [&](auto format_tag) {
    if (rotary != nullptr) launch(format_tag, std::true_type{}); else launch(format_tag, std::false_type{});
  };
  if (format == kQuantE4m3) launch_format(std::integral_constant<int, kQuantE4m3>{});
  else launch_format(std::integral_constant<int, kQuantInt8>{});
}

}  // namespace lkv
