// Adjustment of logits before a token is chosen: penalties for repeated tokens,
// biases, grammar masks.
//
// A workgroup takes a piece of one row. It counts the row's history within the
// piece in LDS (whole numbers, so their order does not matter), then passes over
// the logits once, whose loads are under way behind the history's. HBM-bound with
// many rows (64 rows of 151,936 bf16 after 2,048 tokens 13.1 us a pass, 39 MB: 3.0 TB/s,
// most of it the chain of history, counts and logits that every workgroup runs once);
// every piece of a row reads the history again, from L2, so pieces are long where
// histories are (96 rows of 50,257 fp32 after up to 30,000 16.3 us a pass, of which some
// 6 to compare tokens and 3 to count them). One row takes 3.0 us, a launch and two
// dependent loads. (Passes of one launch among others; a launch that is traced takes
// longer.)
#include <algorithm>

#include "../../include/qwen3_decode.h"
#include "common.h"
#include "kernels.h"

namespace {

constexpr int VEC = 8;
// Changed logits of eight that are taken one at a time; with more in some lane, all eight at once. 64 rows of 151,936
// after 2,048 tokens 14.4, 13.1, 13.0 us with 0, 2, 8; 96 of 50,257 after 30,000 17.2, 17.1, 18.7; one row after 200
// 3.2, 3.2, 3.7.
constexpr int FEW = 2;

// A token's count; the highest bit says that it was seen in the prompt.
constexpr uint32_t SEEN = 1u << 31;

// Eight logits as they are in memory, where rows begin at any element.
template <bool BF16>
struct Raw;
template <>
struct __attribute__((packed, aligned(2))) Raw<true> {
  uint32_t w[4];
  DEV float get(int e) const { return e & 1 ? hi_f(w[e / 2]) : lo_f(w[e / 2]); }
  DEV void set(const float* x) {
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = pack2(x[2 * k], x[2 * k + 1]);
  }
};
template <>
struct __attribute__((packed, aligned(4))) Raw<false> {
  float v[8];
  DEV float get(int e) const { return v[e]; }
  DEV void set(const float* x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[e];
  }
};
template <bool BF16>
DEV Raw<BF16> load8(const void* base, size_t at) {
  return *reinterpret_cast<const Raw<BF16>*>(static_cast<const char*>(base) + at * (BF16 ? 2 : 4));
}
template <bool BF16>
DEV void store8(void* base, size_t at, const Raw<BF16>& x) {
  *reinterpret_cast<Raw<BF16>*>(static_cast<char*>(base) + at * (BF16 ? 2 : 4)) = x;
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

struct __attribute__((packed, aligned(4))) Quad { int32_t t[4]; };

// LDS of a workgroup, in words: counts, a bit for each logit with a bias, the
// biases of the piece (how many, then token, entry and value of each).
__host__ DEV int lds_words(const qwen3_logits& l, int piece) {
  return (l.d_history || l.d_path ? piece : 0) + (l.n_bias > 0 ? piece / 32 + 4 + 3 * l.n_bias : 0);
}

// (waves a SIMD, by the registers: four workgroups a CU)
template <bool BF16, int THREADS, int STEPS>
__global__ __launch_bounds__(THREADS, 8) void logits_kernel(qwen3_logits l, const void* in, void* out) {
  constexpr int STEP = THREADS * VEC, PIECE = STEPS * STEP;
  constexpr int AT_ONCE = 4 * THREADS;   // history tokens under way (twice as many: 12.9 -> 13.4 us at 64 rows)
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  const bool counting = l.d_history || l.d_path, biased = l.n_bias > 0;
  uint32_t* count = lds;
  uint32_t* has_bias = lds + (counting ? PIECE : 0);
  int* n_biases = reinterpret_cast<int*>(has_bias + PIECE / 32);
  int *bias_token = n_biases + 4, *bias_entry = bias_token + l.n_bias;
  float* bias_value = reinterpret_cast<float*>(bias_entry + l.n_bias);
  const int tid = threadIdx.x, row = blockIdx.y, v0 = blockIdx.x * PIECE, n = min(PIECE, l.vocab - v0);
  const size_t at = (size_t)row * l.logits_stride + v0, to = (size_t)row * l.out_stride + v0;

  // the history's first tokens, before their number is known
  int h = l.d_row_seq ? l.d_row_seq[row] : row;
  if (!l.d_history || (unsigned)h >= (unsigned)l.n_seq) h = -1;
  const int32_t* tokens = l.d_history + (size_t)max(h, 0) * l.history_stride;
  auto load = [&](int i0) {   // the thread's of those from i0 on, the row's last one behind its end
    Quad q{};
    const int i = i0 + 4 * tid;
    if (i + 4 <= l.history_stride) {
      q = *reinterpret_cast<const Quad*>(tokens + i);
    } else if (i < l.history_stride) {
#pragma unroll
      for (int e = 0; e < 4; ++e) q.t[e] = tokens[min(i + e, l.history_stride - 1)];
    }
    return q;
  };
  Quad quad{};
  int len = 0, prompt = 0;
  if (h >= 0) {
    quad = load(0);
    len = min(l.d_lens[h], l.history_stride);
    prompt = l.d_prompt_lens ? l.d_prompt_lens[h] : 0;
  }
  int bias_id = -1;
  float bias = 0.0f;
  if (tid < l.n_bias) {
    bias_id = l.d_bias_ids[(size_t)row * l.n_bias + tid];
    bias = l.d_bias[(size_t)row * l.n_bias + tid];
  }
  const float rep = l.d_repetition ? l.d_repetition[row] : 1.0f;
  const float freq = l.d_frequency ? l.d_frequency[row] : 0.0f;
  const float pres = l.d_presence ? l.d_presence[row] : 0.0f;
  const int which = l.d_row_mask ? l.d_row_mask[row] : row;
  const int32_t* mask = l.n_masks > 0 && (unsigned)which < (unsigned)l.n_masks
                            ? l.d_masks + (size_t)which * ((l.vocab + 31) / 32) + v0 / 32 : nullptr;
  Raw<BF16> raw[STEPS];
  uint32_t allowed[STEPS];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int i = k * STEP + tid * VEC;
    if (i + VEC <= n) raw[k] = load8<BF16>(in, at + i);
    allowed[k] = mask && i < n ? (uint32_t)mask[i / 32] >> (i & 31) : ~0u;
  }

  if (counting || biased) {
    if (counting) {
#pragma unroll
      for (int i = tid; i < PIECE / 4; i += THREADS) reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
    }
    if (biased) {
      for (int i = tid; i < PIECE / 32; i += THREADS) has_bias[i] = 0;
      if (tid == 0) *n_biases = 0;
    }
    __syncthreads();
    // f(place of a token in the piece, i) of the thread's four
    auto four = [&](const Quad& q, int i, auto f) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned v = (unsigned)q.t[e] - (unsigned)v0;
        if (v < (unsigned)n) f(v, i + e);
      }
    };
    for (int i0 = 0; i0 < len; i0 += AT_ONCE) {
      const Quad now = quad;
      const int next = i0 + AT_ONCE, i = i0 + 4 * tid;
      if (next < len) quad = load(next);
      if (next <= min(len, prompt)) {
        four(now, i, [&](unsigned v, int) { atomicOr(count + v, SEEN); });
      } else if (next <= len && i0 >= prompt) {
        four(now, i, [&](unsigned v, int) { atomicAdd(count + v, 1u); });
      } else {
        four(now, i, [&](unsigned v, int k) {
          if (k < min(len, prompt)) atomicOr(count + v, SEEN);
          else if (k < len) atomicAdd(count + v, 1u);
        });
      }
    }
    auto piece_has = [&](int token) { return token >= v0 && token - v0 < n; };
    if (l.d_path) {
#pragma unroll 1
      for (int i = tid; i < l.path_len; i += THREADS) {
        const int token = l.d_path[(size_t)row * l.path_len + i];
        if (piece_has(token)) atomicAdd(count + token - v0, 1u);
      }
    }
#pragma unroll 1
    for (int i = tid; i < l.n_bias; i += THREADS) {
      if (i >= THREADS) {
        bias_id = l.d_bias_ids[(size_t)row * l.n_bias + i];
        bias = l.d_bias[(size_t)row * l.n_bias + i];
      }
      if (piece_has(bias_id)) {
        atomicOr(has_bias + (bias_id - v0) / 32, 1u << ((bias_id - v0) & 31));
        const int k = atomicAdd(n_biases, 1);
        bias_token[k] = bias_id - v0;
        bias_entry[k] = i;
        bias_value[k] = bias;
      }
    }
    __syncthreads();
  }

  // a logit as its token's count leaves it (both quotient and product: a branch would cost more)
  auto counted = [&](float y, uint32_t c) {
    const float less = y / rep, more = y * rep, seen = y > 0.0f ? less : more;
    const uint32_t times = c & ~SEEN;
    const float off = times ? freq * (float)times + pres : 0.0f;
    return c ? seen - off : y;
  };
  // logit i as its bias leaves it
  auto with_bias = [&](float y, int i) {
    int best = -1;
    float add_on = 0.0f;
#pragma unroll 1
    for (int k = 0; k < *n_biases; ++k)
      if (bias_token[k] == i && bias_entry[k] > best) {
        best = bias_entry[k];
        add_on = bias_value[k];
      }
    return y + add_on;
  };
  // f(element, its value) of x for the elements of `some`, one at a time
  auto each = [&](float* x, uint32_t some, auto f) {
#pragma unroll 1
    while (some) {
      const int e = __builtin_ctz(some);
      some &= some - 1;
      float y = x[0];
#pragma unroll
      for (int q = 1; q < VEC; ++q) y = e == q ? x[q] : y;
      y = f(e, y);
#pragma unroll
      for (int q = 0; q < VEC; ++q) x[q] = e == q ? y : x[q];
    }
  };
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int i0 = k * STEP + tid * VEC;
    if (i0 + VEC > n) continue;
    float x[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = raw[k].get(e);
    if (counting) {
      const uint4 *words = reinterpret_cast<const uint4*>(count + i0), lo = words[0], hi = words[1];
      const uint32_t c[VEC] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      uint32_t some = 0;
#pragma unroll
      for (int e = 0; e < VEC; ++e) some |= c[e] ? 1u << e : 0u;
      if (__ballot(__builtin_popcount(some) > FEW) != 0) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = counted(x[e], c[e]);
      } else {
        each(x, some, [&](int e, float y) { return counted(y, count[i0 + e]); });
      }
    }
    if (biased) each(x, has_bias[i0 / 32] >> (i0 & 31) & 0xffu, [&](int e, float y) { return with_bias(y, i0 + e); });
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = allowed[k] >> e & 1 ? x[e] : -INFINITY;
    raw[k].set(x);
    store8<BF16>(out, to + i0, raw[k]);
  }
  // the columns behind the last eight
  const int i = n / VEC * VEC + tid;
  if (i < n) {
    float y = load1<BF16>(in, at + i);
    if (counting) y = counted(y, count[i]);
    if (biased && has_bias[i / 32] >> (i & 31) & 1) y = with_bias(y, i);
    if (mask && !((uint32_t)mask[i / 32] >> (i & 31) & 1)) y = -INFINITY;
    store1<BF16>(out, to + i, y);
  }
}

template <bool BF16, int THREADS, int STEPS>
void launch_pieces(const qwen3_logits& l, const void* in, void* out, hipStream_t s) {
  constexpr int PIECE = STEPS * THREADS * VEC;
  hipLaunchKernelGGL((logits_kernel<BF16, THREADS, STEPS>), dim3((l.vocab + PIECE - 1) / PIECE, l.rows), dim3(THREADS),
                     sizeof(uint32_t) * lds_words(l, PIECE), s, l, in, out);
}

template <bool BF16>
void launch(const qwen3_logits& l, const void* in, void* out, hipStream_t s) {
  const long all = (long)l.rows * l.vocab;
  const long longest = (l.d_history ? l.history_stride : 0) + (long)l.path_len;
  // Pieces of 8,192 by 512 threads where there is enough work or a long history, of 2,048 by 256 otherwise. 64 rows of
  // 151,936 after 2,048 tokens, with all adjustments: 13.1 us so, 13.3 in pieces of 2,048, 12.9 of 4,096 (256 threads),
  // 14.4 of 8,192 (1,024 threads); 96 rows of 50,257 after 30,000: 16.2, 23.1, 18.6, 15.7; one row after 200: 4.0, 3.0.
  if (all >= 512l * 2048 || longest > 4096) launch_pieces<BF16, 512, 2>(l, in, out, s);
  else launch_pieces<BF16, 256, 1>(l, in, out, s);
}

}  // namespace

hipError_t launch_adjust_logits(const qwen3_logits& l, const void* logits, void* out, hipStream_t s) {
  l.dtype == 1 ? launch<true>(l, logits, out, s) : launch<false>(l, logits, out, s);
  return hipGetLastError();
}
