// Rotary positions on one or several axes, with the keys' and values' way into the paged cache: q, k and v are read once and
// written once (k twice where both outputs are wanted).  HBM-bound for prompts (9001 tokens of 28 + 4 heads of 128, 34 us, 5.1
// TB/s), a launch's latency for single tokens (64 tokens of 32 + 8 heads into the cache 4 us).
#include "ff_internal.h"

namespace {

// One workgroup to a token.  First a thread for each pair finds its cosine and sine; then the token's heads are worked through in units of
// 16 channels, kBatch to a lane with all their loads on their way: a unit of turned channels is the eight pairs 8 u .. 8 u + 7, wherever
// the layout has their channels, a unit behind them is copied.  A unit is read before it is written by the lane that owns it alone,
// so outputs may be the inputs.  (Four tokens to a workgroup, a wavefront each, took 8.9 us for 7.8 with 1500 tokens of 32 + 8 heads of
// 128, and as long with 9001.)
constexpr int kThreads = 256, kBatch = 2;
__global__ __launch_bounds__(kThreads) void ff_rotary_kernel(RotaryParams p) {
  __shared__ float cs[2][64];
  const int t = blockIdx.y * gridDim.x + blockIdx.x, pairs = p.rot_dim / 2;
  if (t >= p.T) return;
  const int64_t slot = p.slots ? p.slots[t] : -1;
  if ((int)threadIdx.x < pairs) {
    const int j = threadIdx.x, axis = (p.axis[j >> 4] >> (2 * (j & 15))) & 3;
    // positions have up to 31 bits and a frequency 24: the angle in float64, less its whole turns, fits into fp32
    const double turns = (double)p.positions[(size_t)axis * p.T + t] * (double)p.inv_freq[j] * 0.15915494309189533577;
    float sn, cn;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cn);
    cs[0][j] = cn;
    cs[1][j] = sn;
  }
  __syncthreads();
  const int shift = p.head_dim == 64 ? 2 : 3, turned = p.rot_dim / 16;        // units of a head, and those of them that turn
  const int n_units = (p.n_heads + (p.v_pages ? 2 : 1) * p.n_kv) << shift;    // of q, k and v
  const bool cached = slot >= 0 && slot < p.n_slots;
  const size_t place = cached ? (((size_t)(slot >> p.page_shift) * p.n_kv << p.page_shift) + (slot & ((1 << p.page_shift) - 1))) * p.head_dim : 0;
  const bf16_t *q = p.q + t * p.q_stride, *k = p.k + t * p.k_stride, *v = p.v_pages ? p.v + t * p.v_stride : nullptr;
  for (int i0 = threadIdx.x; i0 < n_units; i0 += kThreads * kBatch) {
    uint4 a[kBatch], b[kBatch];
    int ca[kBatch], cb[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int r = min(i0 + i * kThreads, n_units - 1), head = r >> shift, u = r & ((1 << shift) - 1);
      const bool halves = u < turned && !p.interleaved;
      ca[i] = halves ? 8 * u : 16 * u;
      cb[i] = halves ? pairs + 8 * u : 16 * u + 8;
      const bf16_t *src = head < p.n_heads ? q + head * p.head_dim
                          : head < p.n_heads + p.n_kv ? k + (head - p.n_heads) * p.head_dim : v + (head - p.n_heads - p.n_kv) * p.head_dim;
      a[i] = *reinterpret_cast<const uint4 *>(src + ca[i]);
      b[i] = *reinterpret_cast<const uint4 *>(src + cb[i]);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int r = i0 + i * kThreads, head = r >> shift, u = r & ((1 << shift) - 1);
      if (r >= n_units) break;
      if (u < turned && head < p.n_heads + p.n_kv) {
        const uint32_t aw[4] = {a[i].x, a[i].y, a[i].z, a[i].w}, bw[4] = {b[i].x, b[i].y, b[i].z, b[i].w};
        uint32_t ao[4], bo[4];
        const float *cn = &cs[0][8 * u], *sn = &cs[1][8 * u];
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
        a[i] = make_uint4(ao[0], ao[1], ao[2], ao[3]);
        b[i] = make_uint4(bo[0], bo[1], bo[2], bo[3]);
      }
      bf16_t *dst = nullptr, *page = nullptr;
      if (head < p.n_heads) {
        dst = p.q_out + t * p.q_out_stride + head * p.head_dim;
      } else {
        const bool is_k = head < p.n_heads + p.n_kv;
        const int hk = head - p.n_heads - (is_k ? 0 : p.n_kv);
        if (is_k && p.k_out) dst = p.k_out + t * p.k_out_stride + hk * p.head_dim;
        if (cached) page = (is_k ? p.k_pages : p.v_pages) + place + ((size_t)hk << p.page_shift) * p.head_dim;
      }
      if (dst) {
        *reinterpret_cast<uint4 *>(dst + ca[i]) = a[i];
        *reinterpret_cast<uint4 *>(dst + cb[i]) = b[i];
      }
      if (page) {
        *reinterpret_cast<uint4 *>(page + ca[i]) = a[i];
        *reinterpret_cast<uint4 *>(page + cb[i]) = b[i];
      }
    }
  }
}

}  // namespace

hipError_t ff_launch_rotary(const RotaryParams &p, hipStream_t s) {
  const unsigned across = (unsigned)p.T < 1u << 20 ? p.T : 1u << 20;     // (a launch's dimension has 32 bits of threads)
  hipLaunchKernelGGL(ff_rotary_kernel, dim3(across, ((unsigned)p.T + across - 1) / across), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}
