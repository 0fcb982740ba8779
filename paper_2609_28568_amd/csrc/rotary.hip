// Head norm and rotary embedding of queries and keys at positions with several
// axes, forward and backward.
//
//   n = x / sqrt(mean(x^2) + eps) g     (per head; left out without gains)
//   y_i        = n_i cos f_i - n_(i+hd/2) sin f_i
//   y_(i+hd/2) = n_(i+hd/2) cos f_i + n_i sin f_i,   f_i = pos[axis(i)] theta^(-2i/hd)
//
// backward: the turn's transpose, then the norm's derivative (gains frozen),
// its 1/rms computed again from x, which is read anyway.
//
// One wave takes one token (or, with few tokens, some of a token's heads): its
// lanes first compute the token's hd/2 angles, a lane a pair, which all heads
// share, so there is no table to fill or read, and any position costs the same.
// The angle is a number of turns in fp64, reduced there and rounded to fp32
// only as a remainder within half a turn: positions of any size lose nothing.
// Then hd/8 lanes hold a head, 8 elements each, and the wave walks the heads
// with four loads in flight. HBM-bound: 16,384 tokens of 16 + 2 x 8 heads of
// 128, one read and one write of 134 MB, take 47 us (5.7 TB/s), backward, which
// reads the rows again for the norm, 71 (5.2 TB/s; a copy reaches 5.1). Eight
// tokens take 4.6 us, a launch.
#include "common.h"
#include "kernels.h"

namespace {

DEV void unpack8(const uint4& u, float* v) {
  v[0] = lo_f(u.x); v[1] = hi_f(u.x); v[2] = lo_f(u.y); v[3] = hi_f(u.y);
  v[4] = lo_f(u.z); v[5] = hi_f(u.z); v[6] = lo_f(u.w); v[7] = hi_f(u.w);
}
DEV uint4 pack8(const float* v) {
  return make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
}

// over the LANES lanes of a head
template <int LANES>
DEV float head_sum(float v) {
  if constexpr (LANES == 16) return group16_sum(v);
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
// the value of the lane that holds the other element of a pair
template <int LANES>
DEV float other_half(float v) {
  if constexpr (LANES == 16) return xor8(v);
  return __shfl_xor(v, LANES / 2);
}

template <int HD, bool NORM, bool BWD>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, const bf16_t* in, const bf16_t* raw, bf16_t* out) {
  constexpr int HALF = HD / 2, LANES = HD / 8, HEADS = 64 / LANES, FLIGHT = 4;
  __shared__ __attribute__((aligned(16))) float turn[4][2][HALF];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int part = blockIdx.y, parts = gridDim.y;   // of the token's heads
  const int tok = blockIdx.x * 4 + wave;
  const bool on = tok < a.tokens;
  if (on) {
#pragma unroll
    for (int i = lane; i < HALF; i += 64) {
      const double t = a.freq[i] * (double)a.positions[(size_t)a.axis[i] * a.tokens + tok];
      float s, c;
      sincospif((float)(2.0 * (t - rint(t))), &s, &c);
      turn[wave][0][i] = c;
      turn[wave][1][i] = s;
    }
  }
  __syncthreads();
  if (!on) return;
  const int sub = lane % LANES, slots = a.H + 2 * a.Hkv, turned = a.H + a.Hkv;
  const bool first = sub < LANES / 2;
  float c[8], sn[8], gq[8], gk[8];
#pragma unroll
  for (int e = 0; e < 8; e += 4) {
    const int p = 8 * (sub % (LANES / 2)) + e;
    const float4 c4 = *reinterpret_cast<const float4*>(&turn[wave][0][p]);
    const float4 s4 = *reinterpret_cast<const float4*>(&turn[wave][1][p]);
    c[e] = c4.x; c[e + 1] = c4.y; c[e + 2] = c4.z; c[e + 3] = c4.w;
    sn[e] = s4.x; sn[e + 1] = s4.y; sn[e + 2] = s4.z; sn[e + 3] = s4.w;
  }
  // forward turns the first half by -sin, backward the second
#pragma unroll
  for (int e = 0; e < 8; ++e) sn[e] = first != BWD ? -sn[e] : sn[e];
  if constexpr (NORM) {
    unpack8(*reinterpret_cast<const uint4*>(a.q_norm + 8 * sub), gq);
    unpack8(*reinterpret_cast<const uint4*>(a.k_norm + 8 * sub), gk);
  }
  const size_t row = (size_t)tok * slots * HD + 8 * sub;
  const int nsteps = (slots + HEADS - 1) / HEADS;
  const int s0 = nsteps * part / parts, s1 = nsteps * (part + 1) / parts;
  for (int s = s0; s < s1; s += FLIGHT) {
    uint4 u[FLIGHT], r[FLIGHT];
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) {
      const int h = min((min(s + k, s1 - 1)) * HEADS + lane / LANES, slots - 1);
      u[k] = *reinterpret_cast<const uint4*>(in + row + (size_t)h * HD);
      if constexpr (BWD && NORM) r[k] = *reinterpret_cast<const uint4*>(raw + row + (size_t)min(h, turned - 1) * HD);
    }
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) {
      const int h = (s + k) * HEADS + lane / LANES;
      // a head's lanes agree on all of this; exchanges stay within them
      const bool live = s + k < s1 && h < slots;
      if (h < turned) {
        float x[8], y[8];
        unpack8(u[k], x);
        if constexpr (NORM && !BWD) {
          float ss = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
          const float rstd = 1.0f / sqrtf(head_sum<LANES>(ss) / HD + a.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = x[e] * rstd * (h < a.H ? gq[e] : gk[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e] * c[e] + other_half<LANES>(x[e]) * sn[e];
        if constexpr (NORM && BWD) {
          float z[8], ss = 0.0f, dot = 0.0f;
          unpack8(r[k], z);
#pragma unroll
          for (int e = 0; e < 8; ++e) ss += z[e] * z[e];
          const float rstd = 1.0f / sqrtf(head_sum<LANES>(ss) / HD + a.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            z[e] *= rstd;
            y[e] *= h < a.H ? gq[e] : gk[e];
            dot += y[e] * z[e];
          }
          const float m = head_sum<LANES>(dot) / HD;
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = rstd * (y[e] - z[e] * m);
        }
        u[k] = pack8(y);
      }
      if (live && (h < turned || in != out)) *reinterpret_cast<uint4*>(out + row + (size_t)h * HD) = u[k];
    }
  }
}

template <int HD>
void launch_hd(const RotaryArgs& a, const bf16_t* in, const bf16_t* raw, bf16_t* out, bool bwd, hipStream_t s) {
  const bool norm = a.q_norm != nullptr;
  const unsigned blocks = (unsigned)((a.tokens + 3) / 4);
  // with few tokens a token's heads go to several waves, each with the angles
  // again, towards a wave for each SIMD of the chip (1024)
  const int nsteps = (a.H + 2 * a.Hkv + 512 / HD - 1) / (512 / HD);
  const unsigned parts = (unsigned)(a.tokens >= 1024 ? 1 : a.tokens * nsteps <= 1024 ? nsteps : 1024 / a.tokens);
  const dim3 grid(blocks, parts), block(256);
  if (norm && bwd) hipLaunchKernelGGL((rotary_kernel<HD, true, true>), grid, block, 0, s, a, in, raw, out);
  else if (norm) hipLaunchKernelGGL((rotary_kernel<HD, true, false>), grid, block, 0, s, a, in, raw, out);
  else if (bwd) hipLaunchKernelGGL((rotary_kernel<HD, false, true>), grid, block, 0, s, a, in, raw, out);
  else hipLaunchKernelGGL((rotary_kernel<HD, false, false>), grid, block, 0, s, a, in, raw, out);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, const bf16_t* in, const bf16_t* raw, bf16_t* out, int backward,
                         hipStream_t s) {
  if (a.tokens < 1) return hipSuccess;
  switch (a.hd) {
    case 32: launch_hd<32>(a, in, raw, out, backward, s); break;
    case 64: launch_hd<64>(a, in, raw, out, backward, s); break;
    case 128: launch_hd<128>(a, in, raw, out, backward, s); break;
    case 256: launch_hd<256>(a, in, raw, out, backward, s); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}
