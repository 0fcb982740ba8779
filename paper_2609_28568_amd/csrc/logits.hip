// Adjustment of logits before a token is chosen: penalties for repeated tokens,
// biases, grammar masks.
//
// A workgroup takes a piece of one row. It counts the row's history within the
// piece in LDS (whole numbers, so their order does not matter), collects the
// biases that fall into it, and passes over the logits once, its loads under way
// while it counts. HBM-bound with many rows; the history is read again by every
// piece of the row, from L2, so pieces are as long as leaves workgroups for all
// CUs.
#include "../../include/qwen3_decode.h"
#include "common.h"
#include "kernels.h"

namespace {

constexpr int THREADS = 256, VEC = 8, STEP = THREADS * VEC;
constexpr uint32_t PROMPT = 1u << 31;   // seen, whatever the count

// Rows begin at any element.
struct __attribute__((packed, aligned(2))) Bf16s { uint32_t w[4]; };
struct __attribute__((packed, aligned(4))) Floats { float v[4]; };

template <bool BF16>
DEV void load8(const void* base, size_t at, float* x) {
  if constexpr (BF16) {
    const Bf16s u = *reinterpret_cast<const Bf16s*>(static_cast<const bf16_t*>(base) + at);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = lo_f(u.w[k]);
      x[2 * k + 1] = hi_f(u.w[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const Floats u = *reinterpret_cast<const Floats*>(static_cast<const float*>(base) + at + 4 * k);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * k + e] = u.v[e];
    }
  }
}
template <bool BF16>
DEV void store8(void* base, size_t at, const float* x) {
  if constexpr (BF16) {
    Bf16s u;
#pragma unroll
    for (int k = 0; k < 4; ++k) u.w[k] = pack2(x[2 * k], x[2 * k + 1]);
    *reinterpret_cast<Bf16s*>(static_cast<bf16_t*>(base) + at) = u;
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      Floats u;
#pragma unroll
      for (int e = 0; e < 4; ++e) u.v[e] = x[4 * k + e];
      *reinterpret_cast<Floats*>(static_cast<float*>(base) + at + 4 * k) = u;
    }
  }
}
template <bool BF16>
DEV float load1(const void* base, size_t at) {
  if constexpr (BF16) return bf2f(static_cast<const bf16_t*>(base)[at]);
  else return static_cast<const float*>(base)[at];
}
template <bool BF16>
DEV void store1(void* base, size_t at, float x) {
  if constexpr (BF16) static_cast<bf16_t*>(base)[at] = f2bf(x);
  else static_cast<float*>(base)[at] = x;
}

// The biases of a piece in LDS: which tokens have one, and the entries.
constexpr int MAX_BIAS = 1024;
struct Biases {
  int n;
  int token[MAX_BIAS], entry[MAX_BIAS];
  float value[MAX_BIAS];
};

template <bool BF16, int STEPS>
__global__ __launch_bounds__(THREADS) void logits_kernel(qwen3_logits l, const void* in, void* out) {
  constexpr int PIECE = STEPS * STEP;
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  const bool counting = l.d_history || l.d_path, biased = l.n_bias > 0;
  uint32_t* count = lds;
  uint32_t* has_bias = lds + (counting ? PIECE : 0);
  Biases* b = reinterpret_cast<Biases*>(has_bias + PIECE / 32);
  const int tid = threadIdx.x, row = blockIdx.y, v0 = blockIdx.x * PIECE;
  const size_t at = (size_t)row * l.logits_stride + v0, to = (size_t)row * l.out_stride + v0;
  const int n = min(PIECE, l.vocab - v0);

  float x[STEPS][VEC];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int i = k * STEP + tid * VEC;
    if (i + VEC <= n) {
      load8<BF16>(in, at + i, x[k]);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[k][e] = i + e < n ? load1<BF16>(in, at + i + e) : 0.0f;
    }
  }
  const int which = l.d_row_mask ? l.d_row_mask[row] : row;
  const int32_t* mask = l.n_masks > 0 && (unsigned)which < (unsigned)l.n_masks
                            ? l.d_masks + (size_t)which * ((l.vocab + 31) / 32) + v0 / 32 : nullptr;
  const float rep = l.d_repetition ? l.d_repetition[row] : 1.0f;
  const float freq = l.d_frequency ? l.d_frequency[row] : 0.0f;
  const float pres = l.d_presence ? l.d_presence[row] : 0.0f;

  if (counting || biased) {
    if (counting)
      for (int i = tid; i < PIECE / 4; i += THREADS) reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
    if (biased) {
      for (int i = tid; i < PIECE / 32; i += THREADS) has_bias[i] = 0;
      if (tid == 0) b->n = 0;
    }
    __syncthreads();
    const int h = l.d_row_seq ? l.d_row_seq[row] : row;
    if (l.d_history && (unsigned)h < (unsigned)l.n_seq) {
      const int32_t* tokens = l.d_history + (size_t)h * l.history_stride;
      const int len = min(l.d_lens[h], l.history_stride), prompt = l.d_prompt_lens ? l.d_prompt_lens[h] : 0;
#pragma unroll 8
      for (int i = tid; i < len; i += THREADS) {
        const unsigned v = (unsigned)(tokens[i] - v0);
        if (v < (unsigned)n && tokens[i] >= 0) {
          if (i < prompt) atomicOr(count + v, PROMPT);
          else atomicAdd(count + v, 1u);
        }
      }
    }
    if (l.d_path)
      for (int i = tid; i < l.path_len; i += THREADS) {
        const int token = l.d_path[(size_t)row * l.path_len + i];
        if (token >= v0 && token - v0 < n) atomicAdd(count + (token - v0), 1u);
      }
    for (int i = tid; i < l.n_bias; i += THREADS) {
      const int token = l.d_bias_ids[(size_t)row * l.n_bias + i];
      if (token >= v0 && token - v0 < n) {
        atomicOr(has_bias + (token - v0) / 32, 1u << ((token - v0) & 31));
        const int k = atomicAdd(&b->n, 1);
        b->token[k] = token - v0;
        b->entry[k] = i;
        b->value[k] = l.d_bias[(size_t)row * l.n_bias + i];
      }
    }
    __syncthreads();
  }

#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int i = k * STEP + tid * VEC;
    if (i >= n) continue;
    if (counting) {
      const uint4 c0 = reinterpret_cast<const uint4*>(count)[i / 4], c1 = reinterpret_cast<const uint4*>(count)[i / 4 + 1];
      const uint32_t c[VEC] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c[e]) {
          float y = x[k][e];
          y = y > 0.0f ? y / rep : y * rep;
          if (c[e] & ~PROMPT) y -= freq * (float)(c[e] & ~PROMPT) + pres;
          x[k][e] = y;
        }
    }
    if (biased) {
      const uint32_t some = has_bias[i / 32] >> (i & 31) & 0xffu;
      if (some) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (some >> e & 1) {
            int best = -1;
            float value = 0.0f;
            for (int q = 0; q < b->n; ++q)
              if (b->token[q] == i + e && b->entry[q] > best) {
                best = b->entry[q];
                value = b->value[q];
              }
            x[k][e] += value;
          }
      }
    }
    if (mask) {
      const uint32_t allowed = (uint32_t)mask[i / 32] >> (i & 31) & 0xffu;
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[k][e] = allowed >> e & 1 ? x[k][e] : -INFINITY;
    }
    if (i + VEC <= n) {
      store8<BF16>(out, to + i, x[k]);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (i + e < n) store1<BF16>(out, to + i + e, x[k][e]);
    }
  }
}

template <bool BF16, int STEPS>
void launch_pieces(const qwen3_logits& l, const void* in, void* out, hipStream_t s) {
  constexpr int PIECE = STEPS * STEP;
  const size_t lds = (l.d_history || l.d_path ? 4u * PIECE : 0u) + (l.n_bias > 0 ? PIECE / 8 + sizeof(Biases) : 0u);
  hipLaunchKernelGGL((logits_kernel<BF16, STEPS>), dim3((l.vocab + PIECE - 1) / PIECE, l.rows), dim3(THREADS), lds, s, l,
                     in, out);
}

}  // namespace

hipError_t launch_adjust_logits(const qwen3_logits& l, const void* logits, void* out, hipStream_t s) {
  const bool bf = l.dtype == 1;
  const long all = (long)l.rows * l.vocab;
  if (all >= 512l * 4 * STEP) bf ? launch_pieces<true, 4>(l, logits, out, s) : launch_pieces<false, 4>(l, logits, out, s);
  else if (all >= 512l * 2 * STEP) bf ? launch_pieces<true, 2>(l, logits, out, s) : launch_pieces<false, 2>(l, logits, out, s);
  else bf ? launch_pieces<true, 1>(l, logits, out, s) : launch_pieces<false, 1>(l, logits, out, s);
  return hipGetLastError();
}
