// The entry points of a step of drafted tokens under AddressSanitizer and UndefinedBehaviorSanitizer (host code only; no GPU
// is needed and no kernel is launched).  Every device address below is fake and is only compared, never dereferenced: each
// call fails a host-side check or has nothing to do.  Exit status 0 when every expectation holds.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "kvc.h"

static int failures = 0;
#define EXPECT(cond)                                                 \
  do {                                                               \
    if (!(cond)) {                                                   \
      std::fprintf(stderr, "FAILED line %d: %s\n", __LINE__, #cond); \
      ++failures;                                                    \
    }                                                                \
  } while (0)

template <class T = void>
static T* fake(uintptr_t off) {
  return reinterpret_cast<T*>(0x7F0000001000ull + off);
}

int main() {
  const int64_t far[] = {INT64_MAX, INT64_MAX - 15, INT64_C(1) << 62, INT64_C(3) << 61, INT64_MIN};
  int32_t* a = fake<int32_t>(0);
  kvc_step step = {2, 5, 4, 100, 0, 0, a, a, nullptr, nullptr};

  // rotation: strides that no address reaches, frequencies at their ends
  std::vector<double> freq(64, 0.5);
  kvc_rotary r = {KVC_BF16, 5, 128, KVC_ROPE_HALF, 128, 0, 1.0, freq.data(), a};
  const kvc_heads good = {8, 0, fake(0x1000), 1024, 128, fake(0x9000), 1024, 128};
  for (int64_t s : far) {
    for (int i = 0; i < 4; ++i) {
      kvc_heads h = good;
      (i == 0 ? h.in_token_stride : i == 1 ? h.in_head_stride : i == 2 ? h.out_token_stride : h.out_head_stride) = s;
      EXPECT(kvc_rotate(&r, &h, nullptr, nullptr) == KVC_ERR_SHAPE);
      EXPECT(kvc_rotate(&r, &good, &h, nullptr) == KVC_ERR_SHAPE);
    }
  }
  for (double f : {65537.0, -1e300, HUGE_VAL, std::nan("")}) {
    freq[63] = f;
    EXPECT(kvc_rotate(&r, &good, nullptr, nullptr) == KVC_ERR_SHAPE);
    r.rotary_dim = 126;  // (the last pair is not read)
    r.factor = f;
    EXPECT(kvc_rotate(&r, &good, nullptr, nullptr) == KVC_ERR_SHAPE);
    r.rotary_dim = 128;
    r.factor = 1.0;
  }
  freq.assign(64, 65536.0);
  r.num_rows = 0;
  EXPECT(kvc_rotate(&r, &good, &good, nullptr) == KVC_OK);
  r.rotary_dim = 2;
  std::vector<double> one(1, -65536.0);
  r.inv_freq = one.data();
  EXPECT(kvc_rotate(&r, &good, nullptr, nullptr) == KVC_OK);

  // trees: the ends of the step's ranges
  for (int32_t words : {INT32_MIN, -1, 0}) EXPECT(kvc_tree(&step, a, fake<uint64_t>(0), words, a, nullptr) == KVC_ERR_SHAPE);
  step.num_rows = step.max_new = INT32_MAX;
  EXPECT(kvc_tree(&step, a, fake<uint64_t>(0), INT32_MAX, a, nullptr) == KVC_ERR_UNSUPPORTED);
  step.num_seqs = 1 << 30;
  EXPECT(kvc_verify_workspace_bytes(&step, 1 << 30) < size_t{1} << 62 && kvc_verify_workspace_bytes(&step, 1 << 30) > 0);
  EXPECT(kvc_verify_workspace_bytes(&step, (1 << 30) + 1) == 0 && kvc_verify_workspace_bytes(&step, INT32_MIN) == 0);

  // verification
  step = {2, 5, 4, 100, 0, 0, a, a, nullptr, nullptr};
  const float* f = fake<float>(0);
  const kvc_draft d = {1000, 0, a, a, f, 1000, f, 1000, f, f, a, a, a};
  EXPECT(kvc_verify(&step, &d, nullptr, 0, nullptr) == KVC_ERR_WORKSPACE);
  for (int64_t s : far) {
    kvc_draft x = d;
    x.target_stride = s;
    EXPECT(kvc_verify(&step, &x, nullptr, 0, nullptr) == KVC_ERR_SHAPE);
    x = d;
    x.draft_stride = s;
    EXPECT(kvc_verify(&step, &x, nullptr, 0, nullptr) == KVC_ERR_SHAPE);
  }
  for (int32_t v : {INT32_MIN, 0, INT32_MAX}) {
    kvc_draft x = d;
    x.vocab = v;
    EXPECT(kvc_verify(&step, &x, nullptr, 0, nullptr) == KVC_ERR_SHAPE);
  }

  // masks and moves
  for (kvc_dtype t : {KVC_F32, KVC_BF16, KVC_I8}) {
    std::vector<void*> k(70, fake(0)), v(70, fake(0x1000));
    std::vector<float*> sk(70, fake<float>(0x2000)), sv(70, fake<float>(0x3000));
    kvc_cache c = {t, 70, 2, 128, 16, 64, 16 * 256, 256, 128, k.data(), v.data(), 0, 0, nullptr};
    kvc_scales sc = {sk.data(), sv.data(), 32, 1, 16};
    const kvc_scales* s = t == KVC_I8 ? &sc : nullptr;
    kvc_query q = {t == KVC_F32 ? KVC_F32 : KVC_BF16, 8, 1, 0, 0.1f, 0, fake(0), 1024, 128, fake(0), 1024, 128, nullptr};
    step.max_context = 1 << 30;
    EXPECT(kvc_attend_tree(&c, s, &step, &q, fake<uint64_t>(0), 1, 69, nullptr, 0, nullptr) == KVC_ERR_WORKSPACE);
    EXPECT(kvc_attend_tree(&c, s, &step, &q, fake<uint64_t>(0), 1, 70, nullptr, 0, nullptr) == KVC_ERR_SHAPE);
    EXPECT(kvc_attend_tree(&c, s, &step, &q, fake<uint64_t>(0), INT32_MIN, 0, nullptr, 0, nullptr) == KVC_ERR_SHAPE);
    q.window = INT32_MAX;
    EXPECT(kvc_attend_tree(&c, s, &step, &q, fake<uint64_t>(0), 1, 0, nullptr, 0, nullptr) == KVC_ERR_WORKSPACE);
    kvc_step wide = step;
    wide.num_rows = wide.max_new = INT32_MAX / 8;
    EXPECT(kvc_attend_tree(&c, s, &wide, &q, fake<uint64_t>(0), INT32_MAX / 512, 0, nullptr, 0, nullptr) == KVC_ERR_SHAPE);
    EXPECT(kvc_keep(&c, s, &step, a, a, 0, 71, nullptr) == KVC_ERR_SHAPE);
    EXPECT(kvc_keep(&c, s, &step, a, a, 70, 70, nullptr) == KVC_OK && kvc_keep(&c, s, &step, nullptr, a, 0, 1, nullptr) == KVC_ERR_NULL_ARG);
    v[69] = nullptr;
    EXPECT(kvc_keep(&c, s, &step, a, a, 0, 70, nullptr) == KVC_ERR_NULL_ARG);
    c.block_stride = INT64_MAX;
    EXPECT(kvc_keep(&c, s, &step, a, a, 0, 1, nullptr) == KVC_ERR_SHAPE);
  }
  if (failures) return 1;
  std::puts("all checks of drafted tokens passed");
  return 0;
}
