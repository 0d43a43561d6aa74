// The rule that one call of a kind is in flight per plan, for every plan that
// shares device state between its calls.
#pragma once

#include <hip/hip_runtime.h>

#include "common.h"

namespace ebag {

// One kind of call whose device state a plan shares between calls: the
// event recorded after the last one and the stream it was enqueued on.
struct InFlight {
  hipEvent_t done = nullptr;
  hipStream_t stream = nullptr;
  bool pending = false;
};

// Whether `stream` is being captured into a graph.  Work that waits for a
// host-chosen epoch cannot be replayed from a graph: the epoch is fixed at
// capture, so a replay would not wait for the flags of its own producer.
inline bool capturing(hipStream_t stream) {
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  return hipStreamIsCapturing(stream, &cs) == hipSuccess && cs != hipStreamCaptureStatusNone;
}

// One call of each kind in flight per plan: a call on another stream than
// the last one of its kind, while that one has not completed, would share its
// device state.
inline int check_busy(InFlight& f, hipStream_t stream, const char* what) {
  if (!f.pending || stream == f.stream || capturing(stream)) return EBAG_OK;
  const hipError_t e = hipEventQuery(f.done);
  if (e == hipErrorNotReady)
    return fail(EBAG_EBUSY, "a %s of this plan is still running on another stream (the plan's device state for it "
                            "is shared): order them on one stream or wait for it", what);
  if (e != hipSuccess) return fail(EBAG_EHIP, "query the last call: %s", hipGetErrorString(e));
  f.pending = false;
  return EBAG_OK;
}

// Remember the call just enqueued on `stream`.  A captured one runs nothing: the
// last eager call remains the one in flight.
inline int note_call(InFlight& f, hipStream_t stream) {
  if (capturing(stream)) return EBAG_OK;
  const hipError_t e = hipEventRecord(f.done, stream);
  if (e != hipSuccess) return fail(EBAG_EHIP, "record the call's completion: %s", hipGetErrorString(e));
  f.stream = stream;
  f.pending = true;
  return EBAG_OK;
}

}  // namespace ebag
