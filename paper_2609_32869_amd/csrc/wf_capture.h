// The capture of a stream's work as a graph (internal; host rules, no device code).
#pragma once

namespace wf {

// Ends the capture and gives back what it holds whichever way its scope is left, an exception of
// the work's enqueueing included: a stream left in capture would take no other work.  `on` tells
// the enqueueing that it is captured.  Api: the runtime's calls and types.
template <typename Api>
class Capture {
 public:
  using Error = typename Api::Error;
  Capture(typename Api::Stream st, bool& on) : st_(st), on_(on) {}
  Capture(const Capture&) = delete;
  Capture& operator=(const Capture&) = delete;
  ~Capture() {
    if (on_) (void)end();
    if (graph_) Api::destroy(graph_);
    if (exec_) Api::destroy_exec(exec_);
  }
  Error begin() {
    const Error e = Api::begin(st_);
    on_ = e == Api::ok;
    return e;
  }
  Error end() {
    on_ = false;
    return Api::end(st_, &graph_);
  }
  Error instantiate() { return Api::instantiate(&exec_, graph_); }
  typename Api::Exec exec() const { return exec_; }
  void release() { exec_ = nullptr; }  // exec() has another owner

 private:
  typename Api::Stream st_;
  bool& on_;
  typename Api::Graph graph_ = nullptr;
  typename Api::Exec exec_ = nullptr;
};

}  // namespace wf
