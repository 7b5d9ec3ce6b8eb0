// The routed layer's calls on the CPU as a library (routed.py): the kernels, thread by thread, of
// model.cpp, and arrays between pages that nothing may touch.
#define main typed_layer_main
#include "model.cpp"
#undef main

extern "C" {

void model_start() {
  struct sigaction sa = {};
  static char stack[1 << 16];
  stack_t ss = {};
  ss.ss_sp = stack;
  ss.ss_size = sizeof stack;
  sigaltstack(&ss, nullptr);
  sa.sa_sigaction = model::on_fault;
  sa.sa_flags = SA_SIGINFO | SA_ONSTACK;
  sigaction(SIGSEGV, &sa, nullptr);
  sigaction(SIGBUS, &sa, nullptr);
}
// at_end: arrays end with their pages, else they begin with them
void model_side(int at_end) { model::g_at_end = at_end; }
void* model_array(int64_t bytes) { return model::array((size_t)bytes); }
void model_check() { model::check_margins(); }
void model_release() {
  while (!model::g_arrays.empty()) model::release(model::g_arrays.begin()->first);
}

}  // extern "C"
