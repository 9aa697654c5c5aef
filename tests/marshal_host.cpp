// The binding's shortcuts (marshal.cpp) over CPU tensors, for tests without a GPU, and calls of
// the library in their place that wait until another thread lets them go.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <atomic>
#include <chrono>
#include <thread>

#define is_cuda is_cpu
#include "../paper_2606_22968_amd/csrc/marshal.cpp"

namespace {

std::atomic<int> entered{0}, released{0};

template <typename F>
struct Waiting;
template <typename... A>
struct Waiting<mocap_status (*)(A...)> {
  // OK if it was let go within 5 seconds.
  static mocap_status call(A...) {
    entered = 1;
    for (int i = 0; i < 5000 && released == 0; ++i) std::this_thread::sleep_for(std::chrono::milliseconds(1));
    return released != 0 ? MOCAP_OK : MOCAP_ERR_HIP;
  }
};

}  // namespace

#define EXPORTED extern "C" __attribute__((visibility("default")))

EXPORTED int waiting_entered() { return entered; }
EXPORTED void waiting_release() { released = 1; }
EXPORTED void waiting_reset() { entered = released = 0; }
EXPORTED void* waiting_call(const char* name) {
#define MOCAP_WAITING(x) \
  if (std::strcmp(name, "mocap_" #x) == 0) return reinterpret_cast<void*>(&Waiting<decltype(lib.x)>::call);
  MOCAP_WAITING(rope_append)
  MOCAP_WAITING(decode_rope_append)
  MOCAP_WAITING(kv4_append)
  MOCAP_WAITING(kv4_decode_append)
  MOCAP_WAITING(kv4_load)
  MOCAP_WAITING(kv4_decode_attn)
  MOCAP_WAITING(kv4_chunk_attn)
#undef MOCAP_WAITING
  return nullptr;
}
