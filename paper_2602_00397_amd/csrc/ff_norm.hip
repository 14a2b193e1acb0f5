// Norms around a block with the block's gate and the residual's scale, one pass over the data:
//   s = h + scale * gate * post(y),  h_out = bf16(s),  x = bf16(pre(s))
// A token's row stays in registers (fp32) between its one read and its one write, so the bound is HBM: 2 d bytes of h, 2 or 4 d
// of y, 2 d of each output; gains and gate rows come from L2.  16384 rows of 3584, bf16 y and both outputs: 91 us, 5.2 TB/s; a row or
// a few take 3 us, a launch's latency.
#include "ff_internal.h"

namespace {

// sum over the W wavefronts that share a token; every lane gets it.  Fixed order: a token's bits do not depend on its neighbours.
template <int W>
__device__ __forceinline__ float token_sum(float v, float *part, int wave) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  if (W == 1) return v;
  if ((threadIdx.x & 63) == 0) part[wave] = v;
  __syncthreads();
  float s = part[0];
#pragma unroll
  for (int w = 1; w < W; ++w) s += part[w];
  __syncthreads();
  return s;
}

__device__ __forceinline__ void unpack8(const uint4 &v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    f[2 * j] = __uint_as_float(w[j] << 16);
    f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// v -> its norm; statistics in fp32 over the values in registers (the deviations of a layer norm from the mean that is already
// known, so nothing cancels)
template <int W, int NCH>
__device__ __forceinline__ void apply_norm(float (&v)[NCH][8], const NormSpec &n, int c0, int d_model, float *part, int wave) {
  const float inv_d = 1.0f / (float)d_model;
  float mean = 0.f;
  if (n.kind == FF_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[i][j];       // (channels past the row are 0)
    mean = token_sum<W>(s, part, wave) * inv_d;
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
    if (c0 + i * W * 512 < d_model)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] -= mean;
        ss = fmaf(v[i][j], v[i][j], ss);
      }
  const float inv = 1.0f / sqrtf(token_sum<W>(ss, part, wave) * inv_d + n.eps);
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = c0 + i * W * 512;
    if (c < d_model) {
      float g[8], b[8];
      if (n.gain) {
        unpack8(*reinterpret_cast<const uint4 *>(n.gain + c), g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= inv * (g[j] + n.gain_offset);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= inv;
      }
      if (n.bias) {
        unpack8(*reinterpret_cast<const uint4 *>(n.bias + c), b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += b[j];
      }
    }
  }
}

// W wavefronts to a token (4 / W tokens to a workgroup), NCH chunks of 8 channels to a lane
template <int W, int NCH, bool YF32>
__global__ __launch_bounds__(256) void ff_norm_kernel(NormParams p) {
  __shared__ float part[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const unsigned t = (blockIdx.y * gridDim.x + blockIdx.x) * (4 / W) + wave / W;
  if (t >= (unsigned)p.T) return;                      // (W == 4: the whole workgroup; W == 1: no barriers)
  const int c0 = ((wave % W) * 64 + lane) * 8;
  const size_t row = (size_t)t * p.d_model;
  uint4 hv[NCH];
  float s[NCH][8];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = c0 + i * W * 512;
    hv[i] = c < p.d_model ? *reinterpret_cast<const uint4 *>(p.h + row + c) : make_uint4(0, 0, 0, 0);
  }
  if (p.y) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = c0 + i * W * 512;
#pragma unroll
      for (int j = 0; j < 8; ++j) s[i][j] = 0.f;
      if (c < p.d_model) {
        if (YF32) {
          const float4 *y = reinterpret_cast<const float4 *>(static_cast<const float *>(p.y) + row + c);
          const float4 a = y[0], b = y[1];
          s[i][0] = a.x; s[i][1] = a.y; s[i][2] = a.z; s[i][3] = a.w;
          s[i][4] = b.x; s[i][5] = b.y; s[i][6] = b.z; s[i][7] = b.w;
        } else {
          unpack8(*reinterpret_cast<const uint4 *>(static_cast<const bf16_t *>(p.y) + row + c), s[i]);
        }
      }
    }
    if (p.post.kind) apply_norm<W, NCH>(s, p.post, c0, p.d_model, part, wave);
    const bf16_t *gate = p.gate ? p.gate + (size_t)(t / (unsigned)p.gate_tokens) * p.d_model : nullptr;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = c0 + i * W * 512;
      float h[8], g[8];
      unpack8(hv[i], h);
      if (gate && c < p.d_model) {
        unpack8(*reinterpret_cast<const uint4 *>(gate + c), g);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[i][j] *= g[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) s[i][j] = c < p.d_model ? fmaf(p.scale, s[i][j], h[j]) : 0.f;
    }
    if (p.h_out) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = c0 + i * W * 512;
        if (c < p.d_model) *reinterpret_cast<uint4 *>(p.h_out + row + c) = pack8(s[i]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NCH; ++i) unpack8(hv[i], s[i]);
  }
  if (p.x) {
    apply_norm<W, NCH>(s, p.pre, c0, p.d_model, part, wave);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = c0 + i * W * 512;
      if (c < p.d_model) *reinterpret_cast<uint4 *>(p.x + row + c) = pack8(s[i]);
    }
  }
}

template <int W, int NCH>
void launch(const NormParams &p, hipStream_t s) {
  const unsigned groups = ((unsigned)p.T + 4 / W - 1) / (4 / W), across = groups < 1u << 20 ? groups : 1u << 20;
  const dim3 grid(across, (groups + across - 1) / across);               // (a launch's dimension has 32 bits of threads)
  if (p.y_f32) hipLaunchKernelGGL((ff_norm_kernel<W, NCH, true>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((ff_norm_kernel<W, NCH, false>), grid, dim3(256), 0, s, p);
}

}  // namespace

hipError_t ff_launch_norm(const NormParams &p, hipStream_t s) {
  if (p.d_model > kNormMaxModel) return hipErrorInvalidValue;
  // A wavefront to a token where its row is that short, or nearly and there are many (8192 rows of 1024: 11.8 us, with four wavefronts to
  // a row 13.5; 64 rows of 2048 4.7 and 3.0, 16384 of 3584 127 and 92: the loads of a row on four wavefronts are on their way together).
  if (p.d_model <= 512) launch<1, 1>(p, s);
  else if (p.d_model <= 1024 && p.T >= 2048) launch<1, 2>(p, s);
  else if (p.d_model <= 2048) launch<4, 1>(p, s);
  else if (p.d_model <= 4096) launch<4, 2>(p, s);
  else if (p.d_model <= 8192) launch<4, 4>(p, s);
  else launch<4, 8>(p, s);
  return hipGetLastError();
}
