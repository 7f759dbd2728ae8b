// Host arrays into device memory that work on any stream may read as soon as the call is over.  Plain C++, so that it can be run against a model of the device on the host.
#pragma once

#include <stddef.h>

struct UploadPart {
  void* to;
  const void* from;
  size_t bytes;
};

// A copy from pageable memory may be over for the host once its bytes are staged: that they have arrived is known when the stream that they went by has been waited for, and other streams do not
// wait for it.  Waits behind a copy that failed too: the ones before it may still read their sources.  copy(part) and wait() return an error, 0: none; the first one is returned.
template <class Copy, class Wait>
auto upload(const UploadPart* parts, int count, Copy copy, Wait wait) -> decltype(wait()) {
  decltype(wait()) error = {};
  for (int i = 0; i < count && !error; ++i) error = copy(parts[i]);
  const auto waited = wait();
  return error ? error : waited;
}
