// The served step's entry points under AddressSanitizer and UndefinedBehaviorSanitizer (host code only; no GPU is needed
// and no kernel is launched).  Every device address below is fake and is only compared, never dereferenced: each call fails
// a host-side check or has nothing to do.  Exit status 0 when every expectation holds.
#include <cstdint>
#include <cstdio>
#include <functional>
#include <vector>

#include "kvc.h"

static int failures = 0;
#define EXPECT(cond)                                                          \
  do {                                                                        \
    if (!(cond)) {                                                            \
      std::fprintf(stderr, "FAILED line %d: %s\n", __LINE__, #cond);          \
      ++failures;                                                             \
    }                                                                         \
  } while (0)

template <class T = void>
static T* fake(uintptr_t off) {
  return reinterpret_cast<T*>(0x7F0000001000ull + off);
}

struct Fixture {
  std::vector<void*> k, v;
  std::vector<float*> ks, vs;
  kvc_cache cache{};
  kvc_scales scales{};
  kvc_step step{};
  kvc_rows rows{};
  kvc_query query{};
  explicit Fixture(kvc_dtype t = KVC_BF16, int L = 70) {
    for (int l = 0; l < L; ++l) {
      k.push_back(fake(0x1000u * l));
      v.push_back(fake(0x800000u + 0x1000u * l));
      ks.push_back(fake<float>(0x900000u + 0x1000u * l));
      vs.push_back(fake<float>(0xA00000u + 0x1000u * l));
    }
    const kvc_dtype r = t == KVC_F32 ? KVC_F32 : KVC_BF16;
    cache = {t, L, 2, 128, 16, 64, 16 * 256, 256, 128, k.data(), v.data(), 0, 0, nullptr};
    scales = {ks.data(), vs.data(), 32, 1, 16};
    step = {2, 5, 4, 100, 7, 0, fake<int32_t>(0), fake<int32_t>(64), fake<int32_t>(128), fake<int32_t>(256)};
    rows = {r, 0, fake(0x10000), fake(0x20000), 5 * 256, 256, 128};
    query = {r, 8, 1, 0, 0.1f, 0, fake(0x30000), 1024, 128, fake(0x40000), 1024, 128, nullptr};
  }
  const kvc_scales* sc() const { return cache.dtype == KVC_I8 ? &scales : nullptr; }
  kvc_status append(int b = 0, int e = 1) const { return kvc_append(&cache, sc(), &step, &rows, b, e, nullptr); }
  kvc_status gather(int b = 0, int e = 1) const { return kvc_gather(&cache, sc(), &step, &rows, b, e, nullptr); }
  kvc_status attend(int layer = 0) const {
    return kvc_attend(&cache, sc(), &step, &query, layer, nullptr, 0, nullptr);
  }
};

using Change = std::function<void(Fixture&)>;

// What all three calls refuse, the moves, and the attention.
static void refused(const Change& change, kvc_status want, bool moves = true, bool attends = true, kvc_dtype t = KVC_BF16) {
  Fixture f(t);
  change(f);
  if (moves) EXPECT(f.append() == want && f.gather() == want);
  if (attends) EXPECT(f.attend() == want);
}

int main() {
  const int64_t far[] = {INT64_MAX, INT64_MAX - 15, INT64_C(1) << 62, INT64_C(1) << 61, INT64_C(3) << 61};
  for (kvc_dtype t : {KVC_F32, KVC_BF16, KVC_I8}) {
    for (int64_t s : far) {  // strides whose bytes no address reaches
      refused([s](Fixture& f) { f.cache.block_stride = s; }, KVC_ERR_SHAPE, true, true, t);
      refused([s](Fixture& f) { f.cache.token_stride = s; }, KVC_ERR_SHAPE, true, true, t);
      refused([s](Fixture& f) { f.cache.head_stride = s; }, KVC_ERR_SHAPE, true, true, t);
      refused([s](Fixture& f) { f.rows.layer_stride = s; }, KVC_ERR_SHAPE, true, false, t);
      refused([s](Fixture& f) { f.rows.token_stride = s; }, KVC_ERR_SHAPE, true, false, t);
      refused([s](Fixture& f) { f.rows.head_stride = s; }, KVC_ERR_SHAPE, true, false, t);
      refused([s](Fixture& f) { f.query.q_token_stride = s; }, KVC_ERR_SHAPE, false, true, t);
      refused([s](Fixture& f) { f.query.q_head_stride = s; }, KVC_ERR_SHAPE, false, true, t);
      refused([s](Fixture& f) { f.query.out_token_stride = s; }, KVC_ERR_SHAPE, false, true, t);
      refused([s](Fixture& f) { f.query.out_head_stride = s; }, KVC_ERR_SHAPE, false, true, t);
      if (t != KVC_I8) continue;
      refused([s](Fixture& f) { f.scales.block_stride = s; }, KVC_ERR_SHAPE, true, true, t);
      refused([s](Fixture& f) { f.scales.token_stride = s; }, KVC_ERR_SHAPE, true, true, t);
      refused([s](Fixture& f) { f.scales.head_stride = s; }, KVC_ERR_SHAPE, true, true, t);
    }
    // the ends of the step's ranges
    refused([](Fixture& f) { f.step.num_rows = INT32_MAX, f.step.max_new = INT32_MAX; }, KVC_ERR_SHAPE, true, true, t);
    refused([](Fixture& f) { f.step.num_seqs = INT32_MAX; }, KVC_ERR_SHAPE, true, true, t);
    refused([](Fixture& f) { f.step.max_context = INT32_MAX; }, KVC_ERR_SHAPE, true, true, t);
    refused([](Fixture& f) { f.step.max_blocks = INT32_MIN; }, KVC_ERR_SHAPE, true, true, t);
    refused([](Fixture& f) { f.query.num_heads = INT32_MAX - 1; }, KVC_ERR_SHAPE, false, true, t);
    refused([](Fixture& f) { f.query.window = INT32_MIN; }, KVC_ERR_SHAPE, false, true, t);
    {
      Fixture f(t);  // many layers, none of them, and layers that are not there
      EXPECT(f.append(70, 70) == KVC_OK && f.gather(0, 0) == KVC_OK);
      EXPECT(f.append(0, 71) == KVC_ERR_SHAPE && f.attend(70) == KVC_ERR_SHAPE && f.attend(INT32_MIN) == KVC_ERR_SHAPE);
      f.k[69] = nullptr;
      EXPECT(f.append(0, 70) == KVC_ERR_NULL_ARG && f.attend(69) == KVC_ERR_NULL_ARG);
      f.step.num_rows = f.step.max_new = 0;
      EXPECT(f.append(0, 69) == KVC_OK && f.gather(0, 69) == KVC_OK && f.attend(0) == KVC_OK);
    }
    {
      Fixture f(t);  // contexts of the greatest length, and a workspace that is missing
      f.step.max_context = 1 << 30;
      f.step.max_blocks = 1 << 30;
      EXPECT(kvc_attend_workspace_bytes(&f.cache, &f.step, 8) > 0);
      EXPECT(f.attend() == KVC_ERR_WORKSPACE);
      f.query.window = INT32_MAX;
      EXPECT(f.attend() == KVC_ERR_WORKSPACE);
      f.step.num_rows = f.step.max_new = INT32_MAX / 8;
      EXPECT(kvc_attend_workspace_bytes(&f.cache, &f.step, 8) < size_t{1} << 62);
      EXPECT(kvc_attend_workspace_bytes(&f.cache, &f.step, 3) == 0);
    }
  }
  if (failures) return 1;
  std::puts("all served-step checks passed");
  return 0;
}
