// Test-only: the launchers' side of the learning calls for the stand-in runtime (fake_hip.cpp, compiled
// with its own emr_launch_net under another name). No kernel runs; what the launches are given is written
// down, so that the CPU tests can look at which buffers a call names. Events recorded under capture cannot be
// waited for, as in HIP.
#include <hip/hip_runtime_api.h>

#include <map>
#include <vector>

#include "../../paper_2608_27612_amd/csrc/learn.h"

namespace {
struct Launch {
  int64_t step, items, joins, step_items, values, partial, state, count, first, at;
};
std::vector<Launch>& log() {
  static std::vector<Launch>* l = new std::vector<Launch>;
  return *l;
}
bool is_capturing() {
  hipStreamCaptureStatus st;
  (void)hipStreamIsCapturing(nullptr, &st);
  return st != hipStreamCaptureStatusNone;
}
std::map<hipEvent_t, bool>& events() {  // whether last recorded under capture
  static std::map<hipEvent_t, bool>* e = new std::map<hipEvent_t, bool>;
  return *e;
}
int64_t address(const void* p) { return (int64_t)(uintptr_t)p; }
}  // namespace

extern "C" {

int64_t fake_launches(void) { return (int64_t)log().size(); }
void fake_launch(int64_t i, int64_t* out) {
  const Launch& l = log()[(size_t)i];
  const int64_t v[] = {l.step, l.items, l.joins, l.step_items, l.values, l.partial, l.state, l.count, l.first, l.at};
  for (int k = 0; k < 10; ++k) out[k] = v[k];
}

int64_t fake_sums(int64_t n, int64_t e) { return emr::learn_sums(n, e); }
uint32_t fake_light_edges(uint32_t edges, uint32_t rows) { return emr::light_edges(edges, rows); }

hipError_t plain_hipEventRecord(hipEvent_t e, hipStream_t s);
hipError_t plain_hipEventSynchronize(hipEvent_t e);
hipError_t hipEventRecord(hipEvent_t e, hipStream_t s) {
  events()[e] = is_capturing();
  return events()[e] ? hipSuccess : plain_hipEventRecord(e, s);
}
hipError_t hipEventSynchronize(hipEvent_t e) {
  return events()[e] ? hipErrorCapturedEvent : plain_hipEventSynchronize(e);
}

hipError_t emr_launch_net(int step, const void* args, hipStream_t) {
  Launch l{};
  l.step = step;
  switch (step) {
    case 9:
      l.state = address(static_cast<const emr::NetStateArgs*>(args)->state);
      break;
    case 24:
    case 25:
    case 26:
    case 31:
    case 32:
    case 33: {
      const auto& A = *static_cast<const emr::LearnArgs*>(args);
      l.items = address(A.items);
      l.joins = address(A.joins);
      l.step_items = address(A.step_items);
      if (step > 30) l.values = address(A.cur < A.nxt ? A.cur : A.nxt);  // (the buffer's first array)
      l.partial = address(A.partial);
      l.count = A.n_items;
      l.first = A.first_item;
      l.at = A.step;
      break;
    }
    default:
      break;
  }
  log().push_back(l);
  return hipSuccess;
}

}  // extern "C"
