// Rotary positions on one or several axes, with the keys' and values' way into the paged cache: q, k and v are read once and
// written once (k twice where both outputs are wanted).  HBM-bound for prompts, a launch's latency for single tokens.
#include "ff_internal.h"

namespace {

// One workgroup to kTokens tokens.  First every thread finds the cosine and sine of its (token, pair); then the tokens' heads are
// worked through in units of 16 channels: a unit of turned channels is the eight pairs 8 u .. 8 u + 7, wherever the layout has
// their channels, a unit behind them is copied.  A unit is read before it is written by the thread that owns it alone, so
// outputs may be the inputs.
template <int kTokens>
__global__ __launch_bounds__(256) void ff_rotary_kernel(RotaryParams p) {
  __shared__ float cs[kTokens][2][64];
  const int t0 = blockIdx.x * kTokens;
  const int pairs = p.rot_dim / 2, units = p.head_dim / 16, turned = p.rot_dim / 16;
  for (int i = threadIdx.x; i < kTokens * pairs; i += 256) {
    const int tt = i / pairs, j = i - tt * pairs, t = t0 + tt;
    if (t < p.T) {
      const int axis = (p.axis[j >> 4] >> (2 * (j & 15))) & 3;
      // positions have up to 31 bits and a frequency 24: the angle in float64, less its whole turns, fits into fp32
      const double turns = (double)p.positions[(size_t)axis * p.T + t] * (double)p.inv_freq[j] * 0.15915494309189533577;
      float sn, cn;
      sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cn);
      cs[tt][0][j] = cn;
      cs[tt][1][j] = sn;
    }
  }
  __syncthreads();
  const int n_rows = p.n_heads + (p.v_pages ? 2 : 1) * p.n_kv;      // heads of q, k and v
  const int per_token = n_rows * units;
  const int shift = units == 4 ? 2 : 3;                             // (head_dim 64 or 128)
  for (int i = threadIdx.x; i < kTokens * per_token; i += 256) {
    const int tt = kTokens == 1 ? 0 : i / per_token, t = t0 + tt;
    if (t >= p.T) break;
    const int r = i - tt * per_token, head = r >> shift, u = r & (units - 1);
    const int64_t slot = p.slots ? p.slots[t] : -1;
    const bool cached = slot >= 0 && slot < p.n_slots;
    const bf16_t *src;
    bf16_t *dst = nullptr, *page = nullptr;
    if (head < p.n_heads) {
      src = p.q + t * p.q_stride + head * p.head_dim;
      dst = p.q_out + t * p.q_out_stride + head * p.head_dim;
    } else {
      const bool is_k = head < p.n_heads + p.n_kv;
      const int hk = head - p.n_heads - (is_k ? 0 : p.n_kv);
      src = is_k ? p.k + t * p.k_stride + hk * p.head_dim : p.v + t * p.v_stride + hk * p.head_dim;
      if (is_k && p.k_out) dst = p.k_out + t * p.k_out_stride + hk * p.head_dim;
      if (cached)
        page = (is_k ? p.k_pages : p.v_pages) +
               ((((slot >> p.page_shift) * p.n_kv + hk) << p.page_shift) + (slot & ((1 << p.page_shift) - 1))) * p.head_dim;
      if (!dst && !page) continue;
    }
    const bool turn = u < turned && head < p.n_heads + p.n_kv;
    const bool halves = u < turned && !p.interleaved;
    const int ca = halves ? 8 * u : 16 * u, cb = halves ? pairs + 8 * u : 16 * u + 8;
    uint4 a = *reinterpret_cast<const uint4 *>(src + ca), b = *reinterpret_cast<const uint4 *>(src + cb);
    if (turn) {
      const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
      uint32_t ao[4], bo[4];
      const float *cn = &cs[tt][0][8 * u], *sn = &cs[tt][1][8 * u];
      if (p.interleaved) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x0 = __uint_as_float(aw[j] << 16), x1 = __uint_as_float(aw[j] & 0xffff0000u);
          const float y0 = __uint_as_float(bw[j] << 16), y1 = __uint_as_float(bw[j] & 0xffff0000u);
          ao[j] = pack_bf16x2(x0 * cn[j] - x1 * sn[j], x1 * cn[j] + x0 * sn[j]);
          bo[j] = pack_bf16x2(y0 * cn[4 + j] - y1 * sn[4 + j], y1 * cn[4 + j] + y0 * sn[4 + j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x0 = __uint_as_float(aw[j] << 16), x1 = __uint_as_float(aw[j] & 0xffff0000u);
          const float y0 = __uint_as_float(bw[j] << 16), y1 = __uint_as_float(bw[j] & 0xffff0000u);
          ao[j] = pack_bf16x2(x0 * cn[2 * j] - y0 * sn[2 * j], x1 * cn[2 * j + 1] - y1 * sn[2 * j + 1]);
          bo[j] = pack_bf16x2(y0 * cn[2 * j] + x0 * sn[2 * j], y1 * cn[2 * j + 1] + x1 * sn[2 * j + 1]);
        }
      }
      a = make_uint4(ao[0], ao[1], ao[2], ao[3]);
      b = make_uint4(bo[0], bo[1], bo[2], bo[3]);
    }
    if (dst) {
      *reinterpret_cast<uint4 *>(dst + ca) = a;
      *reinterpret_cast<uint4 *>(dst + cb) = b;
    }
    if (page) {
      *reinterpret_cast<uint4 *>(page + ca) = a;
      *reinterpret_cast<uint4 *>(page + cb) = b;
    }
  }
}

}  // namespace

hipError_t ff_launch_rotary(const RotaryParams &p, hipStream_t s) {
  if (p.T <= 1024) hipLaunchKernelGGL(ff_rotary_kernel<1>, dim3(p.T), dim3(256), 0, s, p);
  else hipLaunchKernelGGL(ff_rotary_kernel<4>, dim3((p.T + 3) / 4), dim3(256), 0, s, p);
  return hipGetLastError();
}
