// The dense layers' entry points with launches that only write down what they were given: which kernels a call takes,
// without a device.  Compiled by tests/dense_launches.py.
#include "../../paper_2507_01676_amd/csrc/dense_api.cpp"

#include <cstdio>
#include <string>

namespace {
std::string g_log;
int g_call = 0;   // of the launches' functions

template <class... V>
void note(const char* format, V... v) {
  char line[512];
  std::snprintf(line, sizeof line, format, v...);
  g_log += line;
}

int product(const char* name, int kind, int variant, const embx::DenseGemm& g) {
  note("%s call=%d kind=%d variant=%d splits=%d slots=%d first=%d row_blocks=%d whole=%d ni=%d nj=%d nr=%d parts=%d lda=%lld ldb0=%lld "
       "ldb1=%lld\n", name, g_call, kind, variant, g.splits, g.slots, g.first, g.row_blocks, g.whole, g.ni, g.nj, g.nr, g.parts, static_cast<long long>(g.lda),
       static_cast<long long>(g.ldb[0]), static_cast<long long>(g.ldb[1]));
  return 0;
}

int both(const embx::DenseGemm& w, const embx::DenseGemm& x, int variant) {
  ++g_call;
  if (w.parts) product("dw", embx::kWeightGrad, variant, w);
  if (x.parts) product("dx", embx::kInputGrad, variant, x);
  return 0;
}

int slopes(const embx::DenseSlope& s) {
  note("slope m=%d n=%d whole=%d copies=%d row_blocks=%d lddz=%lld\n", s.m, s.n, s.whole, s.pack.count, s.row_blocks,
       static_cast<long long>(s.lddz));
  return 0;
}
}  // namespace

namespace embx {
int dense_pack_launch(const DensePack& p, void*) {
  note("pack copies=%d\n", p.count);
  return 0;
}
#define STUBS(NAME)                                                                                                        \
  int dense_forward_##NAME(int kind, const DenseGemm& g, void*) { return ++g_call, product("forward", kind, g.variant, g); }        \
  int dense_grads_##NAME(const DenseGemm& w, const DenseGemm& x, int variant, void*) { return both(w, x, variant); }       \
  int dense_tail_##NAME(const DenseGemm&, const DenseGemm&, const DenseColsum&, void*) { return 0; }                       \
  int dense_slope_##NAME(const DenseSlope& s, void*) { return slopes(s); }
STUBS(f32)
STUBS(f16)
STUBS(bf16)
}  // namespace embx

// what was noted since the last call
extern "C" const char* dense_launches() {
  static std::string out;
  out.swap(g_log);
  g_log.clear();
  return out.c_str();
}
