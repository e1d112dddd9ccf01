// Rotary positions: of the `rotary_dim` channels of every head, pair i of token t is turned by the angle position(t) w_i,
//   y_a = f (x_a cos - x_b sin),  y_b = f (x_b cos + x_a sin),
// the other channels are copied.  The backward pass is the transpose, the same turn by the negative angle (the sine's sign).
//
// The call moves every element once in and once out and is bound by that; what could get in the way are the cosines and sines.
// They are fp64 work (lkv_rotary.h), the same for all heads of a token, so a block takes 8 tokens and many heads: its 256
// threads compute the 8 x 64 cosines and sines of the tokens once, into LDS, and each wave then turns head after head, with the
// 16 of its lanes in registers.  A lane has 8 pairs: 16 channels, which in bf16 are two 16-byte pieces, and 8 lanes make a row.
// Calls too short to fill the chip so are cut along the heads as well.
#include <algorithm>
#include <type_traits>

#include "lkv_kernels.h"

namespace lkv {

constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / 64;
constexpr int kRopeTokens = 8;
constexpr int kRopePairs = kHeadDim / 2;
constexpr int kRopeUnroll = 4;     // heads of a wave whose loads are in flight together
constexpr int kRopeBlocks = 1024;   // blocks that a launch wants: 4 per compute unit

template <typename T> struct RopePiece;   // 8 elements
template <> struct RopePiece<uint16_t> {
  uint4 w;
  __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&f)[8]) const { unpack8(w, f); }
  static __device__ __forceinline__ uint32_t two(float a, float b) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
  __device__ __forceinline__ void set(const float (&f)[8]) { w = make_uint4(two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7])); }
  __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<uint4*>(p) = w; }
};
template <> struct RopePiece<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    a = make_float4(f[0], f[1], f[2], f[3]);
    b = make_float4(f[4], f[5], f[6], f[7]);
  }
  __device__ __forceinline__ void store(float* p) const { reinterpret_cast<float4*>(p)[0] = a; reinterpret_cast<float4*>(p)[1] = b; }
};

__device__ __forceinline__ float rope_get(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float rope_get(float x) { return x; }
template <typename T> __device__ __forceinline__ T rope_put(float f) {
  if constexpr (sizeof(T) == 2) return __builtin_bit_cast(uint16_t, (__bf16)f);
  else return f;
}

// kWide: rotary_dim is a multiple of 16, so that the 8 pairs of a lane are whole pieces.  Else a lane takes one pair at a time.
template <typename T, bool kWide>
__global__ void __launch_bounds__(kRopeThreads)
rope_kernel(RotaryArgs rot, const T* x, RopeStrides xs, T* y, RopeStrides ys, const int32_t* __restrict__ positions,
            int64_t positions_stride, int first_position, int n_tokens, int64_t n_rows /* batch x tokens */, int n_heads,
            int heads_per_block, int head_blocks, float sign) {
  __shared__ __align__(16) float cos_lds[kRopeTokens][kRopePairs];
  __shared__ __align__(16) float sin_lds[kRopeTokens][kRopePairs];
  const int tid = threadIdx.x;
  const int64_t row0 = (int64_t)(blockIdx.x / (unsigned)head_blocks) * kRopeTokens;
  const int h0 = (int)(blockIdx.x % (unsigned)head_blocks) * heads_per_block;
  const int h1 = min(h0 + heads_per_block, n_heads);
  const int half = rot.rotary_dim >> 1;

  for (int i = tid; i < kRopeTokens * kRopePairs; i += kRopeThreads) {
    const int pair = i % kRopePairs;
    const int64_t row = row0 + i / kRopePairs;
    float c = 1.f, s = 0.f;
    if (pair < half && row < n_rows) {
      const int64_t b = row / n_tokens;
      const int t = (int)(row - b * n_tokens);
      const int pos = positions != nullptr ? positions[b * positions_stride + t] : first_position + t;
      rotary_cos_sin(pos, rot.inv_freq[pair], rot.factor, &c, &s);
    }
    cos_lds[i / kRopePairs][pair] = c;
    sin_lds[i / kRopePairs][pair] = s * sign;
  }
  __syncthreads();

  const int wave = tid >> 6, lane = tid & 63;
  if constexpr (kWide) {
    const int token = lane >> 3, octet = lane & 7;
    const int64_t row = row0 + token;
    if (row >= n_rows) return;
    const int64_t b = row / n_tokens;
    const int64_t t = row - b * n_tokens;
    const bool turned = octet * 8 < half;
    // this lane's two pieces of 8 channels
    const bool split = turned && rot.pairs == 0;
    const int ch0 = split ? octet * 8 : octet * 16;
    const int ch1 = split ? octet * 8 + half : octet * 16 + 8;
    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) { c[i] = cos_lds[token][octet * 8 + i]; s[i] = sin_lds[token][octet * 8 + i]; }
    const T* px = x + b * xs.batch + t * xs.token;
    T* py = y + b * ys.batch + t * ys.token;
    // y may be x: the loads of a round go ahead of its stores by hand
    for (int h = h0 + wave; h < h1; h += kRopeWaves * kRopeUnroll) {
      RopePiece<T> p0[kRopeUnroll], p1[kRopeUnroll];
#pragma unroll
      for (int u = 0; u < kRopeUnroll; ++u) {
        const T* p = px + min(h + u * kRopeWaves, h1 - 1) * xs.head;   // past the last head: read, not written
        p0[u].load(p + ch0);
        p1[u].load(p + ch1);
      }
#pragma unroll
      for (int u = 0; u < kRopeUnroll; ++u) {
        if (h + u * kRopeWaves >= h1) break;
        if (turned) {
          float f0[8], f1[8];
          p0[u].get(f0);
          p1[u].get(f1);
          if (rot.pairs == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) rotary_turn(f0[i], f1[i], c[i], s[i]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              rotary_turn(f0[2 * i], f0[2 * i + 1], c[i], s[i]);
              rotary_turn(f1[2 * i], f1[2 * i + 1], c[4 + i], s[4 + i]);
            }
          }
          p0[u].set(f0);
          p1[u].set(f1);
        }
        T* p = py + (h + u * kRopeWaves) * ys.head;
        p0[u].store(p + ch0);
        p1[u].store(p + ch1);
      }
    }
  } else {
    const int ch0 = lane < half && rot.pairs == 0 ? lane : 2 * lane;
    const int ch1 = lane < half && rot.pairs == 0 ? lane + half : 2 * lane + 1;
    for (int token = 0; token < kRopeTokens; ++token) {
      const int64_t row = row0 + token;
      if (row >= n_rows) return;
      const int64_t b = row / n_tokens;
      const int64_t t = row - b * n_tokens;
      const float c = cos_lds[token][lane], s = sin_lds[token][lane];
      const T* px = x + b * xs.batch + t * xs.token;
      T* py = y + b * ys.batch + t * ys.token;
      for (int h = h0 + wave; h < h1; h += kRopeWaves) {
        const T x0 = px[h * xs.head + ch0], x1 = px[h * xs.head + ch1];
        float a0 = rope_get(x0), a1 = rope_get(x1);
        rotary_turn(a0, a1, c, s);
        py[h * ys.head + ch0] = lane < half ? rope_put<T>(a0) : x0;
        py[h * ys.head + ch1] = lane < half ? rope_put<T>(a1) : x1;
      }
    }
  }
}

void launch_rope(const RotaryArgs& rot, bool f32, const void* x, const RopeStrides& xs, void* y, const RopeStrides& ys,
                 const int32_t* positions, int64_t positions_stride, int first_position, int n_batch, int n_heads, int n_tokens,
                 bool backward, hipStream_t stream) {
  const int64_t n_rows = (int64_t)n_batch * n_tokens;
  const int64_t token_blocks = (n_rows + kRopeTokens - 1) / kRopeTokens;
  int head_blocks = (int)std::min<int64_t>((n_heads + kRopeWaves - 1) / kRopeWaves, std::max<int64_t>(1, kRopeBlocks / token_blocks));
  const int per_block = ((n_heads + head_blocks - 1) / head_blocks + kRopeWaves - 1) / kRopeWaves * kRopeWaves;
  head_blocks = (n_heads + per_block - 1) / per_block;
  auto launch = [&](auto tag, auto wide) {
    using T = decltype(tag);
    hipLaunchKernelGGL((rope_kernel<T, decltype(wide)::value>), dim3((unsigned)(token_blocks * head_blocks)), dim3(kRopeThreads), 0,
                       stream, rot, static_cast<const T*>(x), xs, static_cast<T*>(y), ys, positions, positions_stride, first_position,
                       n_tokens, n_rows, n_heads, per_block, head_blocks, backward ? -1.f : 1.f);
  };
  const bool wide = rot.rotary_dim % 16 == 0;
  if (f32) { if (wide) launch(float{}, std::true_type{}); else launch(float{}, std::false_type{}); }
  else { if (wide) launch(uint16_t{}, std::true_type{}); else launch(uint16_t{}, std::false_type{}); }
}

}  // namespace lkv
