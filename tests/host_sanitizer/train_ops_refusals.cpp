// What the entry points of the layer norm refuse and what they launch, at the library's own limit of calls in one launch (CPU only; built
// and run by tests/test_host_sanitizer_train_ops.py).  The launchers are counting stand-ins: the device pointers are fake and no
// kernel sees them, whichever way a limit moves.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "decoder.h"
#include "train_ops.h"

#define CHECK(cond)                                                        \
  do {                                                                     \
    if (!(cond)) {                                                         \
      std::fprintf(stderr, "%s:%d: CHECK failed: %s\n", __FILE__, __LINE__, #cond); \
      std::exit(1);                                                        \
    }                                                                      \
  } while (0)

namespace {
int fwd_launches, bwd_launches, few_launches, sum_launches;
template <typename T = void> T* at(uintptr_t p) { return reinterpret_cast<T*>(p); }
}  // namespace

namespace seco {
int norm_blocks(int64_t rows, int64_t, int) { return rows < 1 ? 1 : rows < SECO_NORM_BLOCKS ? (int)rows : SECO_NORM_BLOCKS; }
bool norm_few(int64_t rows, int64_t d) { return rows >= 1 && rows <= kNormFewRows && d <= kNormFewLength; }
int launch_norm_fwd(const NormArgs&, hipStream_t) { fwd_launches++; return SECO_OK; }
int launch_norm_bwd(const NormArgs&, hipStream_t) { bwd_launches++; return SECO_OK; }
int launch_norm_bwd_few(const NormArgs&, bool, bool, hipStream_t) { few_launches++; return SECO_OK; }
int launch_norm_sums(const float*, int, int64_t, void*, void*, int, hipStream_t) { sum_launches++; return SECO_OK; }
int launch_adamw(int, const AdamArgs&, hipStream_t) { return SECO_OK; }
int launch_adamw_count(int64_t*, hipStream_t) { return SECO_OK; }
int launch_rope_axes(const RopeAxesArgs&, bool, bool, bool, hipStream_t) { return SECO_OK; }
}  // namespace seco
using namespace seco;

static layer_norm_desc desc(int64_t rows, int64_t d) {
  layer_norm_desc x{};
  x.rows = rows; x.d = d; x.x_stride = x.residual_stride = x.out_stride = x.y_stride = d;
  x.dtype = x.gain_dtype = SECO_BF16; x.eps = 1e-5f;
  return x;
}
static int bwd(const layer_norm_desc& d, uintptr_t ws, size_t n, uintptr_t dg = 0x3000, uintptr_t dx = 0x90000000) {
  return layer_norm_bwd(&d, at(0x10000000), nullptr, at<float>(0x1000), at<float>(0x2000), at(0x50000000), nullptr, at(dx), at(dg), nullptr, at(ws), n,
                        nullptr);
}

int main() {
  // the workspace: below the limit none, beyond it all of it, from a 16-byte boundary on
  for (const layer_norm_desc& d : {desc(kNormFewRows, 16), desc(1, kNormFewLength), desc(kNormFewRows, kNormFewLength)}) {
    few_launches = bwd_launches = 0;
    CHECK(layer_norm_workspace_bytes(&d) == 0 && bwd(d, 0, 0) == SECO_OK && few_launches == 1 && bwd_launches == 0);
  }
  for (const layer_norm_desc& d : {desc(kNormFewRows + 1, 16), desc(1, kNormFewLength + 1), desc(2000, 16), desc(100000, 5)}) {
    const size_t n = layer_norm_workspace_bytes(&d);
    few_launches = bwd_launches = sum_launches = 0;
    CHECK(n > 0 && n != (size_t)-1);
    CHECK(bwd(d, 0, n) == SECO_ERR_WORKSPACE && bwd(d, 0x40000000, n - 1) == SECO_ERR_WORKSPACE && bwd(d, 0x40000000, 16) == SECO_ERR_WORKSPACE);
    CHECK(bwd(d, 0x40000008, n) == SECO_ERR_WORKSPACE && bwd_launches == 0 && few_launches == 0 && sum_launches == 0);
    CHECK(bwd(d, 0x40000000, n) == SECO_OK && bwd_launches == 1 && sum_launches == 1 && few_launches == 0);
    CHECK(bwd(d, 0, 0, 0) == SECO_OK && bwd_launches == 2 && sum_launches == 1);      // no sums wanted: no workspace
  }
  // nothing is launched by a call that is refused
  fwd_launches = bwd_launches = few_launches = 0;
  const layer_norm_desc d = desc(4, 16);
  CHECK(bwd(d, 0, 0, 0x3001) == SECO_ERR_ALIGN && bwd(d, 0, 0, 0x3000, 0) == SECO_ERR_NULL);
  auto fwd = [&](layer_norm_desc x, uintptr_t in = 0x1000, uintptr_t res = 0, uintptr_t out = 0, uintptr_t mean = 0x2000) {
    return layer_norm_fwd(&x, at(in), at(res), nullptr, nullptr, at(out), at(0x4000), at<float>(mean), at<float>(0x3000), nullptr);
  };
  CHECK(fwd(d, 0) == SECO_ERR_NULL && fwd(d, 0x1000, 0x8000) == SECO_ERR_NULL && fwd(d, 0x1000, 0, 0x8000) == SECO_ERR_NULL);
  CHECK(fwd(d, 0x1001) == SECO_ERR_ALIGN && fwd(d, 0x1000, 0, 0, 0x2002) == SECO_ERR_ALIGN);
  layer_norm_desc bad = d;
  bad.dtype = 3;
  CHECK(fwd(bad) == SECO_ERR_DTYPE && layer_norm_workspace_bytes(&bad) == (size_t)-1);
  bad = d; bad.y_stride = 15;
  CHECK(fwd(bad) == SECO_ERR_SHAPE);
  bad = d; bad.out_stride = 15;
  CHECK(bwd(bad, 0, 0) == SECO_ERR_SHAPE && fwd_launches == 0 && bwd_launches == 0 && few_launches == 0);
  CHECK(fwd(d) == SECO_OK && fwd_launches == 1);
  std::puts("all checks passed");
  return 0;
}
