// No exception leaves a C entry (internal; host rules, no device code).
#pragma once
#include <string>

namespace wf {

// call(), or `code` where it throws (the host's records of a search, of a graph or of a message may fail to allocate), with
// the message where a caller looks for it: on the handle, if there is one, and for the thread.
template <typename H, typename Call>
int guarded(H* h, std::string& thread, int code, Call&& call) noexcept {
  try {
    return call();
  } catch (...) {
  }
  for (std::string* to : {h ? &h->err : nullptr, &thread}) {
    if (!to) continue;
    try {
      *to = "out of host memory";
    } catch (...) {
      to->clear();  // no message rather than an older call's
    }
  }
  return code;
}

}  // namespace wf
