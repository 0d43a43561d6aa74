// Host check of csrc/in_flight.h with streams, events and captures played by this
// file: a plan's call on another stream is refused as long as its last eager call
// has not completed, whatever was captured in between.
#include <cstdarg>
#include <cstdio>

#include "in_flight.h"

namespace {
bool captured[4], event_pending;
int index_of(hipStream_t s) { return (int)reinterpret_cast<uintptr_t>(s); }
}  // namespace

extern "C" {
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus* cs) {
  *cs = captured[index_of(s)] ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}
hipError_t hipEventQuery(hipEvent_t) { return event_pending ? hipErrorNotReady : hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) {
  event_pending = true;
  return hipSuccess;
}
const char* hipGetErrorString(hipError_t) { return ""; }
}

int ebag::fail(int code, const char*, ...) { return code; }

int main() {
  using namespace ebag;
  int bad = 0;
  auto expect = [&](int got, int want, const char* what) {
    if (got != want) std::printf("%s: %d, not %d\n", what, got, want), ++bad;
  };
  const hipStream_t a = reinterpret_cast<hipStream_t>(1), b = reinterpret_cast<hipStream_t>(2), c = reinterpret_cast<hipStream_t>(3);
  for (bool capture : {false, true}) {
    InFlight f;
    event_pending = false;
    expect(check_busy(f, a, "call"), EBAG_OK, "the first call");
    expect(note_call(f, a), EBAG_OK, "the first call");
    if (capture) {
      captured[2] = true;
      expect(check_busy(f, b, "call"), EBAG_OK, "a captured call");
      expect(note_call(f, b), EBAG_OK, "a captured call");
      captured[2] = false;
    }
    expect(check_busy(f, c, "call"), EBAG_EBUSY, "another stream while the first call runs");
    expect(check_busy(f, a, "call"), EBAG_OK, "its own stream");
    event_pending = false;
    expect(check_busy(f, c, "call"), EBAG_OK, "another stream behind the first call");
    expect(note_call(f, c), EBAG_OK, "another stream behind the first call");
    expect(check_busy(f, a, "call"), EBAG_EBUSY, "the first stream while the last call runs");
  }
  std::printf("bad=%d\n", bad);
  return bad != 0;
}
