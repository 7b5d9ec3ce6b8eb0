// Scratch memory of a call: the caller's, or temporaries of the library.
#pragma once

#include "common.h"

namespace gcn {

// With `bytes`, a call's work arguments are: where `work` is null, a question for the
// bytes (asked() is true after the allocations: the call ends there); else memory of so many
// bytes. Without `bytes` the memory comes from the library's temporaries, and not on a
// capturing stream: there they would be memory nodes of the caller's graph.
class Scratch {
 public:
  Scratch(void* work, int64_t* bytes, hipStream_t stream)
      : temps_(stream), work_(static_cast<char*>(work)), bytes_(bytes), left_(0) {
    if (!bytes_) return;
    if (work_)
      left_ = *bytes_;
    else
      *bytes_ = 0;
  }
  bool asked() const { return bytes_ && !work_; }
  template <class T>
  gcn_status alloc(T** p, int64_t count, const char* what) {
    const int64_t need = (count * (int64_t)sizeof(T) + 255) / 256 * 256;
    *p = nullptr;
    if (asked()) {
      *bytes_ += need;
      return GCN_OK;
    }
    if (work_) {
      if (left_ < need) {
        set_error("the work memory is too small for %s", what);
        return GCN_EINVAL;
      }
      *p = reinterpret_cast<T*>(work_);
      work_ += need;
      left_ -= need;
      return GCN_OK;
    }
    if (stream_capturing(temps_.stream)) {
      set_error("a captured call needs work memory for %s", what);
      return GCN_ESTATE;
    }
    return temps_.alloc(p, count, what);
  }

 private:
  TempScope temps_;
  char* work_;
  int64_t* bytes_;
  int64_t left_;
};

}  // namespace gcn
