// trace.cu -- optional per-kernel-class timing with CUDA events recorded on
// the launching stream around every kernel of soma_spsa_step / soma_eval_loss,
// and around every call of the first-order entry points (soma_trace_enable /
// soma_trace_read / soma_trace_read_first_order / soma_trace_read_sequence in
// include/soma_api.h).
#include <mutex>
#include <vector>

#include "soma_api.h"
#include "soma_launch.h"

namespace soma {

namespace {

struct Record {
  int kind;
  cudaEvent_t start, stop;
};

std::mutex g_mu;
bool g_enabled = false;
std::vector<Record> g_pending;
std::vector<cudaEvent_t> g_pool;
Record g_open = {-1, nullptr, nullptr};

cudaEvent_t take_event() {
  if (!g_pool.empty()) {
    cudaEvent_t e = g_pool.back();
    g_pool.pop_back();
    return e;
  }
  cudaEvent_t e = nullptr;
  if (cudaEventCreate(&e) != cudaSuccess) return nullptr;
  return e;
}

// Sums the records of the classes [first, first + count).  Under g_mu.
int read_kinds(int first, int count, double* ms, int64_t* launches, int reset) {
  for (int k = 0; k < count; ++k) {
    ms[k] = 0.0;
    launches[k] = 0;
  }
  int rc = SOMA_OK;
  for (const Record& r : g_pending) {
    if (r.kind < first || r.kind >= first + count) continue;
    if (cudaEventSynchronize(r.stop) != cudaSuccess) {
      rc = SOMA_ERR_CUDA;
      continue;
    }
    float t = 0.f;
    if (cudaEventElapsedTime(&t, r.start, r.stop) != cudaSuccess) {
      rc = SOMA_ERR_CUDA;
      continue;
    }
    ms[r.kind - first] += t;
    launches[r.kind - first] += 1;
  }
  if (reset) {
    std::vector<Record> others;
    for (const Record& r : g_pending) {
      if (r.kind < first || r.kind >= first + count) {
        others.push_back(r);
        continue;
      }
      g_pool.push_back(r.start);
      g_pool.push_back(r.stop);
    }
    g_pending.swap(others);
  }
  return rc;
}

}  // namespace

void trace_begin(int kind, cudaStream_t stream) {
  std::lock_guard<std::mutex> lk(g_mu);
  if (!g_enabled) return;
  g_open.kind = kind;
  g_open.start = take_event();
  g_open.stop = take_event();
  if (g_open.start) cudaEventRecord(g_open.start, stream);
}

void trace_end(int kind, cudaStream_t stream) {
  std::lock_guard<std::mutex> lk(g_mu);
  if (!g_enabled || g_open.kind != kind || !g_open.start || !g_open.stop) return;
  cudaEventRecord(g_open.stop, stream);
  g_pending.push_back(g_open);
  g_open.kind = -1;
}

}  // namespace soma

using namespace soma;

extern "C" {

int soma_trace_enable(int enable) {
  std::lock_guard<std::mutex> lk(g_mu);
  g_enabled = enable != 0;
  return SOMA_OK;
}

int soma_trace_read(soma_kernel_times* out, int reset) {
  if (!out) return SOMA_ERR_INVALID_ARG;
  std::lock_guard<std::mutex> lk(g_mu);
  return read_kinds(0, SOMA_TRACE_KINDS, out->ms, out->launches, reset);
}

int soma_trace_read_first_order(soma_first_order_times* out, int reset) {
  if (!out) return SOMA_ERR_INVALID_ARG;
  std::lock_guard<std::mutex> lk(g_mu);
  return read_kinds(SOMA_TRACE_LINEAR_CE, SOMA_TRACE_FIRST_ORDER, out->ms, out->calls, reset);
}

int soma_trace_read_sequence(soma_sequence_times* out, int reset) {
  if (!out) return SOMA_ERR_INVALID_ARG;
  std::lock_guard<std::mutex> lk(g_mu);
  return read_kinds(SOMA_TRACE_LINEAR_ATTN, SOMA_TRACE_SEQUENCE, out->ms, out->calls, reset);
}

}  // extern "C"
