// Host side of the operators around the training step under AddressSanitizer + UndefinedBehaviorSanitizer (CPU only; built and
// run by tests/test_host_sanitizer_train_ops.py).  The launchers are recording stand-ins, so the device pointers are fake and
// never dereferenced; what runs for real is what the entry points do before a launch.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <vector>

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
struct Log {
  std::vector<seco::NormArgs> fwd, bwd, few;
  std::vector<std::pair<bool, bool>> parts_of;
  int sums = 0, counts = 0;
  std::vector<std::pair<int, seco::AdamArgs>> adam;
  std::vector<seco::RopeAxesArgs> rope;
} log_;
template <typename T = void> T* at(uintptr_t p) { return reinterpret_cast<T*>(p); }
}  // namespace

namespace seco {
int norm_blocks(int64_t rows, int64_t, int) { return rows < 1 ? 1 : rows < SECO_NORM_BLOCKS ? (int)rows : SECO_NORM_BLOCKS; }
bool norm_few(int64_t rows, int64_t d) { return rows >= 1 && rows <= 1024 && d <= 16384; }
int launch_norm_fwd(const NormArgs& a, hipStream_t) { log_.fwd.push_back(a); return SECO_OK; }
int launch_norm_bwd(const NormArgs& a, hipStream_t) { log_.bwd.push_back(a); return SECO_OK; }
int launch_norm_bwd_few(const NormArgs& a, bool rows, bool sums, hipStream_t) {
  log_.few.push_back(a);
  log_.parts_of.emplace_back(rows, sums);
  return SECO_OK;
}
int launch_norm_sums(const float*, int, int64_t, void*, void*, int, hipStream_t) { log_.sums++; return SECO_OK; }
int launch_adamw(int kind, const AdamArgs& a, hipStream_t) { log_.adam.emplace_back(kind, a); return SECO_OK; }
int launch_adamw_count(int64_t*, hipStream_t) { log_.counts++; return SECO_OK; }
int launch_rope_axes(const RopeAxesArgs& a, bool, bool, bool, hipStream_t) { log_.rope.push_back(a); return SECO_OK; }
}  // namespace seco
using namespace seco;

static void layer_norms() {
  layer_norm_desc d{};
  d.rows = 10; d.d = 64; d.x_stride = d.residual_stride = d.out_stride = d.y_stride = 64;
  d.dtype = SECO_BF16; d.gain_dtype = SECO_F32; d.eps = 1e-5f;
  float *m = at<float>(0x1000), *r = at<float>(0x2000);
  CHECK(layer_norm_fwd(&d, at(0x100000), nullptr, nullptr, nullptr, nullptr, at(0x200000), m, r, nullptr) == SECO_OK);
  CHECK(log_.fwd.size() == 1 && log_.fwd[0].rows == 10 && log_.fwd[0].gain_f32 == 1);
  // where the rows of d_x lie: apart, in x, in d_y, across the end of x, behind it
  auto bwd = [&](uintptr_t dx, size_t n = 0) {
    return layer_norm_bwd(&d, at(0x100000), nullptr, m, r, at(0x200000), nullptr, at(dx), at(0x3000), nullptr, n ? at(0x400000) : nullptr, n, nullptr);
  };
  const uintptr_t span = 10 * 64 * 2;
  for (auto [dx, apart] : {std::pair<uintptr_t, bool>{0x300000, true}, {0x100000, false}, {0x200000, false}, {0x100000 + span - 2, false},
                           {0x100000 + span, true}, {0x100000 - span, true}, {0x100000 - span + 2, false}}) {
    log_ = Log{};
    CHECK(bwd(dx) == SECO_OK && log_.few.size() == (apart ? 1u : 2u) && log_.bwd.empty() && log_.sums == 0);
    CHECK(log_.parts_of[0].first == apart && log_.parts_of[0].second && (apart || (log_.parts_of[1].first && !log_.parts_of[1].second)));
  }
  d.rows = 5000;
  log_ = Log{};
  const size_t ws = layer_norm_workspace_bytes(&d);
  CHECK(ws == 2u * 256 * 64 * 4 && bwd(0x300000) == SECO_ERR_WORKSPACE && bwd(0x300000, ws - 1) == SECO_ERR_WORKSPACE);
  CHECK(bwd(0x300000, ws) == SECO_OK && log_.bwd.size() == 1 && log_.sums == 1 && log_.few.empty());
  // extremes: sizes and strides at their limits, and behind them
  d.rows = (int64_t)1 << 31; d.d = (int64_t)1 << 30;
  d.x_stride = d.residual_stride = d.out_stride = d.y_stride = (int64_t)1 << 31;
  CHECK(layer_norm_workspace_bytes(&d) == (size_t)2 * 256 * ((size_t)1 << 30) * 4);
  CHECK(layer_norm_fwd(&d, at(0x100000), nullptr, nullptr, nullptr, nullptr, at(0x200000), m, r, nullptr) == SECO_OK);
  for (int64_t bad : {std::numeric_limits<int64_t>::min(), (int64_t)-1, std::numeric_limits<int64_t>::max()}) {
    layer_norm_desc e = d;
    e.rows = bad; CHECK(layer_norm_workspace_bytes(&e) == (size_t)-1);
    e = d; e.d = bad; CHECK(layer_norm_workspace_bytes(&e) == (size_t)-1);
    e = d; e.out_stride = bad; CHECK(layer_norm_workspace_bytes(&e) == (size_t)-1);
  }
  // in the training step
  log_ = Log{};
  CHECK(dec_add_layer_norm(SECO_F32, at(0x100), nullptr, at(0x200), nullptr, 1e-5f, nullptr, at(0x300), m, r, 7, 9, nullptr) == SECO_OK);
  CHECK(log_.fwd.size() == 1 && log_.fwd[0].out == nullptr && log_.fwd[0].xs == 9);
  CHECK(dec_embed_layer_norm(SECO_BF16, at(0x100), at<int64_t>(0x200), at(0x200), at(0x300), 1e-5f, at(0x300), at(0x400), m, r, 7, 9, 29,
                             m, nullptr) == SECO_OK && log_.fwd[1].table == 29);
  CHECK(dec_embed_layer_norm(SECO_BF16, at(0x100), at<int64_t>(0x200), at(0x200), at(0x300), 1e-5f, at(0x300), at(0x400), m, r, 7, 9, 0,
                             m, nullptr) == SECO_ERR_SHAPE);
  CHECK(dec_layer_norm_bwd(SECO_BF16, at(0x100), at(0x200), m, r, at(0x300), at(0x400), at(0x400), at<float>(0x1000), 0, 9, nullptr) == SECO_OK &&
        log_.bwd.empty());
  CHECK(dec_layer_norm_bwd(SECO_BF16, at(0x100), at(0x200), m, r, at(0x300), at(0x400), at(0x400), at<float>(0x1000), 3, 9, nullptr) == SECO_OK);
  CHECK(log_.few.size() == 1 && log_.few[0].accumulate == 1 && log_.few[0].d_bias == at(0x1000 + SECO_NORM_BLOCKS * 9 * 4) && log_.bwd.empty());
  CHECK(dec_layer_norm_bwd(SECO_BF16, at(0x100), at(0x200), m, r, at(0x300), at(0x400), at(0x400), at<float>(0x1000), 3000, 9, nullptr) == SECO_OK);
  CHECK(log_.bwd.size() == 1 && log_.bwd[0].accumulate == 1 && log_.bwd[0].part_rows == SECO_NORM_BLOCKS && log_.bwd[0].blocks == SECO_NORM_BLOCKS);
}

static adamw_tensor tensor(int64_t n, int param, int grad, bool master) {
  adamw_tensor t{};
  t.param = at(0x1000); t.grad = at(0x2000); t.m = at(0x3000); t.v = at(0x4000);
  t.m_scale = at<float>(0x5000); t.v_scale = at<float>(0x6000); t.master = master ? at<float>(0x7000) : nullptr;
  t.n = n; t.param_dtype = param; t.grad_dtype = grad; t.weight_decay = 0.1f;
  return t;
}
static void adamw() {
  for (int bits : {32, 8})
    for (int n_tensors : {0, 1, 47, 48, 49, 97, 500}) {
      adamw_desc d{};
      d.lr = 1e-3; d.beta1 = 0.9; d.beta2 = 0.95; d.eps = 1e-8; d.state_bits = bits;
      std::vector<adamw_tensor> ts;
      uint64_t x = 88172645463325252ull + (uint64_t)n_tensors;
      int64_t spans = 0;
      const int64_t span = adam_span(bits == 8);
      for (int i = 0; i < n_tensors; ++i) {
        x ^= x << 13; x ^= x >> 7; x ^= x << 17;
        const int64_t n = x % 7 == 0 ? 0 : (int64_t)(x >> 40) % 5000 + 1;
        const bool bf16 = x >> 8 & 1;
        ts.push_back(tensor(n, bf16 ? SECO_BF16 : SECO_F32, x >> 9 & 1 ? SECO_BF16 : SECO_F32, bf16 && (x >> 10 & 1)));
        spans += (n + span - 1) / span;
      }
      log_ = Log{};
      CHECK(adamw_step(&d, ts.data(), n_tensors, at<int64_t>(0x8000), nullptr) == SECO_OK);
      const bool counted = spans > kAdamCounting;
      CHECK(log_.counts == (counted ? 1 : 0));
      int64_t seen = 0, seen_spans = 0;
      int last = 0;
      for (auto& [kind, a] : log_.adam) {
        CHECK(a.count >= 0 && a.count <= kAdamTensors && (a.counted != 0) == counted);
        last += a.last;
        uint32_t next = 0;
        for (int i = 0; i < a.count; ++i) {
          const AdamEntry& e = a.e[i];
          CHECK(e.first == next && e.last >= e.first && e.tail >= 1 && e.tail <= span);
          next = e.last + 1;
          seen += (int64_t)(e.last - e.first) * span + e.tail;
          CHECK((e.master != nullptr) == ((kind & kAdamMaster) != 0));
        }
        CHECK(next == a.spans);
        seen_spans += a.spans;
      }
      int64_t all = 0;
      for (auto& t : ts) all += t.n;
      CHECK(seen == all && seen_spans == spans && last == (counted ? 0 : 1));
      CHECK(counted || (!log_.adam.empty() && log_.adam.back().second.last == 1));
    }
  // the largest tensors: their spans are counted in 32 bits, over several launches
  adamw_desc d{};
  d.state_bits = 8;
  std::vector<adamw_tensor> ts(3, tensor((int64_t)1 << 40, SECO_F32, SECO_F32, false));
  log_ = Log{};
  CHECK(adamw_step(&d, ts.data(), 3, at<int64_t>(0x8000), nullptr) == SECO_OK && log_.adam.size() == 2);
  CHECK(log_.adam[0].second.spans == (uint32_t)1 << 31 && log_.adam[0].second.e[1].last == 0x7fffffffu);
  ts[1].n = ((int64_t)1 << 40) + 1;
  CHECK(adamw_step(&d, ts.data(), 3, at<int64_t>(0x8000), nullptr) == SECO_ERR_TOO_LARGE);
  ts[1].n = std::numeric_limits<int64_t>::min();
  CHECK(adamw_step(&d, ts.data(), 3, at<int64_t>(0x8000), nullptr) == SECO_ERR_SHAPE);
}

static void rope() {
  seco_desc d;
  std::memset(&d, 0, sizeof d);
  d.batch = 2; d.n_q_heads = 4; d.n_kv_heads = 2; d.chunk_len = 16; d.q_start = 48; d.dtype = SECO_BF16;
  const int64_t ps[3] = {64, 32, 1};
  for (int D = 8; D <= 256; D += 8)
    for (int inter = 0; inter < 2; ++inter)
      for (int own = 0; own < 2; ++own)
        for (int n = 1; n <= SECO_ROPE_MAX_AXES; ++n)
          for (int first = 0; first <= D / 2; first += n == 1 ? D / 2 : 1) {
            rope_axes x{};
            x.n_axes = n; x.interleaved = inter; x.own_frequencies = own; x.base = 10000.f;
            if (n == 1 && first == 0) continue;
            x.sections[n - 1] = D / 2;
            x.sections[0] = first;
            if (n > 1) x.sections[n - 1] -= first;
            for (int64_t* s : {d.q_stride, d.o_stride, d.g_stride, d.kv_stride}) s[0] = 1 << 20, s[1] = 1 << 14, s[2] = D;
            d.head_dim = D;
            log_ = Log{};
            CHECK(rope_append_axes(&d, &x, at(0x10000), at(0x20000), at(0x30000), at(0x40000), at(0x50000), at(0x60000), at<int64_t>(0x1000), ps,
                                   nullptr) == SECO_OK && log_.rope.size() == 1);
            const RopeAxesArgs& a = log_.rope[0];
            int count[SECO_ROPE_MAX_AXES] = {};
            for (int i = 0; i < D / 2; ++i) {
              const int axis = a.axis[i];
              CHECK(axis < n);
              const double e = own ? (double)count[axis] / x.sections[axis] : (double)i / (D / 2), want = std::pow(10000.0, -e);
              CHECK(std::fabs(a.frequency[i] - want) <= 1e-14 * want);       // (7 products and a power: 20 roundings of 2^-53)
              ++count[axis];
            }
            for (int i = 0; i < n; ++i) CHECK(count[i] == x.sections[i]);
            CHECK(a.k.out == at(0x50000 + 48 * D * 2) && a.k.heads == 2 && a.v.in == at(0x40000) && a.q.heads == 4);
          }
  rope_axes x{};
  x.n_axes = 4; x.base = 10000.f;
  for (int& s : x.sections) s = std::numeric_limits<int>::max();
  d.head_dim = 256;
  auto call = [&] { return rope_rotate_axes(&d, &x, 4, at(0x10000), at(0x20000), at<int64_t>(0x1000), ps, 0, nullptr); };
  CHECK(call() == SECO_ERR_RANGE);
  x.sections[0] = -128; x.sections[1] = 256; x.sections[2] = x.sections[3] = 0;
  CHECK(call() == SECO_ERR_RANGE);
  x.sections[0] = 128; x.sections[1] = 0;
  d.q_stride[2] = std::numeric_limits<int64_t>::max();
  CHECK(call() == SECO_ERR_TOO_LARGE);
  d.q_start = (1 << 30) - 16;                                   // the last rows of the longest cache, at the largest strides
  for (int64_t* s : {d.q_stride, d.o_stride, d.g_stride, d.kv_stride}) s[0] = s[1] = (int64_t)1 << 40, s[2] = (int64_t)1 << 30;
  log_ = Log{};
  CHECK(rope_readout_axes(&d, &x, at(0x10000), at(0x20000), at<float>(0x30000), at<float>(0x40000), at(0x50000), at(0x60000), 1.f,
                          at<int64_t>(0x1000), ps, nullptr) == SECO_OK);
  CHECK(log_.rope[0].k.in == at(0x30000 + ((uintptr_t)d.q_start << 32)));
  d.g_stride[2] += 16;
  CHECK(rope_readout_axes(&d, &x, nullptr, nullptr, at<float>(0x30000), nullptr, at(0x50000), nullptr, 1.f, at<int64_t>(0x1000), ps, nullptr) ==
        SECO_ERR_TOO_LARGE);
}

int main() {
  layer_norms();
  adamw();
  rope();
  std::puts("all checks passed");
  return 0;
}
