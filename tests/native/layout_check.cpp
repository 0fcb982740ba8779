// Host check of the layout's entry points where memory runs out: every
// allocation that qwen3_layout_size and qwen3_set_layout make fails in turn (and
// all after it); the call says so and nothing is thrown through the C entry. The
// copy to the device is one in host memory; no GPU is touched.
#include "../../paper_2609_28568_amd/csrc/qwen3.cpp"

#include <cstdio>
#include <cstdlib>
#include <cstring>

static long g_left = -1;   // allocations until one fails; -1: none does

void* operator new(size_t n) {
  if (g_left == 0) throw std::bad_alloc();
  if (g_left > 0) --g_left;
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void* operator new(size_t n, const std::nothrow_t&) noexcept {
  if (g_left == 0) return nullptr;
  if (g_left > 0) --g_left;
  return std::malloc(n ? n : 1);
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }
void operator delete(void* p, const std::nothrow_t&) noexcept { std::free(p); }

extern "C" hipError_t hipMemcpyAsync(void* to, const void* from, size_t n, hipMemcpyKind, hipStream_t) {
  std::memcpy(to, from, n);
  return hipSuccess;
}
extern "C" hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
extern "C" hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
  *s = hipStreamCaptureStatusNone;
  return hipSuccess;
}

int main() {
  qwen3_model* m = new qwen3_model();
  m->d.B = 1;
  m->d.T = 300;
  m->d.H = 4;
  m->d.Hkv = 2;
  m->d.hd = 128;
  m->stream = nullptr;
  const int32_t good[] = {40, 100, 60}, bad[] = {40, -1, 60}, short_of[] = {40, 100, 59};
  static char plan[1 << 22] __attribute__((aligned(256)));
  int wrong = 0, calls = 0;
  for (const int32_t* lens : {good, bad, short_of})
    for (int set = 0; set < 2; ++set) {
      const gpt2_status want = lens == good || (lens == short_of && !set) ? GPT2_OK : GPT2_ERR_INVALID_ARG;
      for (long k = 0;; ++k) {
        gpt2_status st = GPT2_OK;
        size_t bytes = 0;
        bool thrown = false;
        g_left = k;
        try {
          st = set ? qwen3_set_layout(m, 100, 3, lens, plan, sizeof plan) : qwen3_layout_size(m, 100, 3, lens, &bytes);
        } catch (...) {
          thrown = true;
        }
        const bool failed = g_left == 0;   // (an allocation may have been the last to succeed)
        g_left = -1;
        ++calls;
        if (thrown || (st != want && (!failed || st != GPT2_ERR_DEVICE)) || (st != GPT2_OK && !*qwen3_last_error(m))) {
          ++wrong;
          std::printf("lengths %d %d %d, %s, allocation %ld: %s status %d\n", lens[0], lens[1], lens[2],
                      set ? "set_layout" : "layout_size", k, thrown ? "thrown" : "returned", (int)st);
        }
        if (!failed) break;
      }
    }
  std::printf("%d calls, %d wrong\n", calls, wrong);
  return wrong ? 1 : 0;
}
