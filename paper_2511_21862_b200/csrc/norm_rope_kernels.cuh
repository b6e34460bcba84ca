// Norms of the heads of q and k, rotary positions and the append to the paged cache, in one pass over q, k and v.
#pragma once
#include "cta_util.cuh"

namespace ooco {

struct HeadNormParams {
  const uint16_t *q_weight, *k_weight;  // bf16 [D] or NULL
  float eps, offset;
};

// The work is cut as in rope_append_kernel: a unit is 16 dims of one head of one token, two 16-byte pieces (with the halves
// layout the two members of eight pairs).  Consecutive lanes hold the units of a head, so a head's sum of squares is the sum
// over 16 values of a thread and a butterfly over its D / 16 lanes, in 32 bits; and since a thread keeps its place in the head
// from unit to unit, it finds the weights of its 16 dims at a place of its own.  Bound by HBM and, nearly as much, by issue slots: q, k
// and v are read and written once, sums and rotations run on pairs of fp32 values.  Tokens of 64 q and 8 kv heads of 128: 16384 over
// a bf16 cache 121 us, 5.5 TB/s, and over codes 126 to 135 us, 4.7 to 5.0 TB/s (66 % of the issue slots, ALU pipe 46 %, special
// functions 17 %, fp64, which forms the angles, 0.2 %); over bf16 158 when lanes' weights, cosines and sines met in the banks
// of shared memory, 135 with single operations; 64 tokens 4.3 to 4.6 us, a launch and two trips to memory.
template <int D, bool KV8>
__global__ void __launch_bounds__(kRopeThreads, 4) norm_rope_append_kernel(const RopeParams p, const HeadNormParams hn,
                                                                        const int interleaved) {
  constexpr int UPH = D / 16;  // units (lanes) per head
  // By the place in the head, so that neighbouring lanes read neighbouring vectors (no bank conflicts): the 16 weights with their
  // offset, of q and of k; the cosines and sines of 8 pairs, of each token of the tile.
  __shared__ float4 s_w[2][4][UPH], s_cs[kRopeMaxTile][4][UPH];
  __shared__ int s_pos[kRopeMaxTile], s_slot[kRopeMaxTile];
  grid_dep_wait();
  grid_dep_launch();
  constexpr int GROUPS = kRopeThreads / UPH;  // heads at a time
  const int heads = p.Hq + 2 * p.Hkv, rot_units = p.half / 8;
  const int c = threadIdx.x % UPH;  // (the number of threads is a multiple of UPH)
  const bool turned = c < rot_units, turned_halves = !interleaved && turned;
  const int d_lo = turned_halves ? 8 * c : 16 * c, d_hi = turned_halves ? p.half + 8 * c : 16 * c + 8;
  const uint4 none = make_uint4(0u, 0u, 0u, 0u);
  if (threadIdx.x < 2 * D) {
    const int kind = threadIdx.x / D, place = threadIdx.x % D / 16, e = threadIdx.x % 16;  // element e of a thread's 16
    const bool halves = !interleaved && place < rot_units;
    const int dim = halves ? (e < 8 ? 8 * place + e : p.half + 8 * place + e - 8) : 16 * place + e;
    const uint16_t* w = kind ? hn.k_weight : hn.q_weight;
    reinterpret_cast<float*>(&s_w[kind][e / 4][place])[e % 4] = w ? __uint_as_float((uint32_t)w[dim] << 16) + hn.offset : 1.f;
  }
  for (int t0 = blockIdx.x * p.tile; t0 < p.T; t0 += gridDim.x * p.tile) {
    const int nt = min(p.tile, p.T - t0);
    for (int i = threadIdx.x; i < nt * p.half; i += kRopeThreads) {
      const int tk = i / p.half, j = i - tk * p.half;
      // angle / (2 pi) reduced to [-1/2, 1/2] in 64 bits: far positions lose nothing
      const double turns = (double)p.positions[t0 + tk] * (double)p.inv_freq[j] * 0.15915494309189533577;
      float s, co;
      sincospif((float)(2.0 * (turns - rint(turns))), &s, &co);
      float* cs = reinterpret_cast<float*>(&s_cs[tk][j % 8 / 2][j / 8]);  // cosines of two pairs, sines of both
      cs[j % 2] = co * p.magnitude;
      cs[2 + j % 2] = s * p.magnitude;
    }
    if ((int)threadIdx.x < nt) {
      s_pos[threadIdx.x] = p.positions[t0 + threadIdx.x];
      s_slot[threadIdx.x] = p.slots[t0 + threadIdx.x];
    }
    __syncthreads();
    // the heads of all tokens of the tile in a row, GROUPS at a time (the same trips for every thread: warps stay whole)
    const int n = (nt * heads + GROUPS * kRopeBatch - 1) / (GROUPS * kRopeBatch);
    int tok = 0, next = threadIdx.x / UPH;
    for (int trip = 0; trip < n; ++trip) {
      uint4 a[kRopeBatch], b[kRopeBatch];
      int tk[kRopeBatch], head[kRopeBatch];
#pragma unroll
      for (int i = 0; i < kRopeBatch; ++i) {
        while (next >= heads) {
          next -= heads;
          ++tok;
        }
        a[i] = b[i] = none;
        tk[i] = -1;
        head[i] = next;
        next += GROUPS;
        if (tok >= nt || s_pos[tok] < 0) continue;  // (padding)
        tk[i] = tok;
        const size_t t = (size_t)(t0 + tok);
        const uint16_t* src = head[i] < p.Hq           ? p.q + t * p.q_stride + (size_t)head[i] * D
                              : head[i] < p.Hq + p.Hkv ? p.k + t * p.k_stride + (size_t)(head[i] - p.Hq) * D
                                                       : p.v + t * p.v_stride + (size_t)(head[i] - p.Hq - p.Hkv) * D;
        a[i] = *reinterpret_cast<const uint4*>(src + d_lo);
        b[i] = *reinterpret_cast<const uint4*>(src + d_hi);
      }
#pragma unroll
      for (int i = 0; i < kRopeBatch; ++i) {
        const bool is_q = head[i] < p.Hq, is_v = head[i] >= p.Hq + p.Hkv;
        float x[8], y[8];
        unpack8(a[i], x);
        unpack8(b[i], y);
        // (two values an instruction where the pairs are neighbours)
        float2 xx[4], yy[4], sq = make_float2(0.f, 0.f);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          xx[m] = make_float2(x[2 * m], x[2 * m + 1]);
          yy[m] = make_float2(y[2 * m], y[2 * m + 1]);
          sq = ffma2(xx[m], xx[m], ffma2(yy[m], yy[m], sq));
        }
        float ss = sq.x + sq.y;
#pragma unroll
        for (int o = 1; o < UPH; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);  // (all lanes of a head take part alike)
        if (tk[i] < 0) continue;
        if (!is_v) {
          const float r = __frsqrt_rn(ss * (1.f / D) + hn.eps);
          const float4(*w)[UPH] = s_w[is_q ? 0 : 1];
          const float2 rr = make_float2(r, r);
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const float4 u = w[m][c];
            float2* v = m < 2 ? xx + 2 * m : yy + 2 * (m - 2);
            v[0] = fmul2(fmul2(v[0], rr), make_float2(u.x, u.y));
            v[1] = fmul2(fmul2(v[1], rr), make_float2(u.z, u.w));
          }
          if (turned) {
#pragma unroll
            for (int m = 0; m < 4; ++m) {  // pairs 8 c + 2 m, + 1
              const float4 cs = s_cs[tk[i]][m][c];
              if (interleaved) {
                float2* v = m < 2 ? xx + 2 * m : yy + 2 * (m - 2);
                v[0] = make_float2(v[0].x * cs.x - v[0].y * cs.z, v[0].y * cs.x + v[0].x * cs.z);
                v[1] = make_float2(v[1].x * cs.y - v[1].y * cs.w, v[1].y * cs.y + v[1].x * cs.w);
              } else {
                const float2 x0 = xx[m];
                xx[m] = make_float2(x0.x * cs.x - yy[m].x * cs.z, x0.y * cs.y - yy[m].y * cs.w);
                yy[m] = ffma2(x0, make_float2(cs.z, cs.w), fmul2(yy[m], make_float2(cs.x, cs.y)));
              }
            }
          }
#pragma unroll
          for (int m = 0; m < 4; ++m) x[2 * m] = xx[m].x, x[2 * m + 1] = xx[m].y, y[2 * m] = yy[m].x, y[2 * m + 1] = yy[m].y;
        }
        if (is_q) {
          uint16_t* dst = p.q_out + (size_t)(t0 + tk[i]) * p.q_out_stride + (size_t)head[i] * D;
          *reinterpret_cast<uint4*>(dst + d_lo) = pack8_bf16(x);
          *reinterpret_cast<uint4*>(dst + d_hi) = pack8_bf16(y);
        } else {
          const int slot = s_slot[tk[i]];
          if (slot < 0 || slot >= p.num_slots) continue;
          const int h = head[i] - p.Hq - (is_v ? p.Hkv : 0);
          const int64_t at = (int64_t)(slot >> p.bs_log2) * p.bstr + (int64_t)h * p.hstr +
                             (int64_t)(slot & ((1 << p.bs_log2) - 1)) * p.tstr;
          uint8_t* cache = is_v ? p.v_cache : p.k_cache;
          if (KV8) {
            const float sc = is_v ? p.v_scale : p.k_scale;
            *reinterpret_cast<uint2*>(cache + at + d_lo) = pack8_e4m3(x, sc);
            *reinterpret_cast<uint2*>(cache + at + d_hi) = pack8_e4m3(y, sc);
          } else {
            *reinterpret_cast<uint4*>(cache + 2 * (at + d_lo)) = is_v ? a[i] : pack8_bf16(x);
            *reinterpret_cast<uint4*>(cache + 2 * (at + d_hi)) = is_v ? b[i] : pack8_bf16(y);
          }
        }
      }
    }
    __syncthreads();  // the tile's cosines are consumed before the next tile's are written
  }
}

}  // namespace ooco
