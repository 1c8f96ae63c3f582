// The rotation's host code on top of fake_cuda.cpp: what it hands to its kernel.
#include "../../paper_2607_20125_b200/csrc/packed_api.cu"

static RopeParams seen;
extern "C" const void* fake_saw_launch(const char* name, void** args) {
  if (std::strstr(name, "rope_kernel")) seen = *static_cast<const RopeParams*>(args[0]);
  return nullptr;
}
// The frequencies of the last launch, in 2^-64 turns per position; returns how many.
extern "C" int fake_frequencies(uint64_t* out) {
  std::memcpy(out, seen.frequency, sizeof(seen.frequency));
  return seen.pairs;
}
