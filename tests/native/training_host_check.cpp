// Host-side paths of the calls that train device levels by reward under
// AddressSanitizer and UndefinedBehaviorSanitizer: sizes at the limits, range
// checks of many buffers, and the launch lists of up to 65536 tensors (the
// launches that follow them fail without a GPU).  Linked against host-only
// objects of the library.  Prints "ALL OK" when every expectation holds.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "../../include/lr.h"

static int g_fail = 0;
#define EXPECT(c)                                           \
  do {                                                      \
    if (!(c)) {                                             \
      std::printf("FAIL line %d: %s\n", __LINE__, #c);      \
      ++g_fail;                                             \
    }                                                       \
  } while (0)

static char* fake(uint64_t a) { return reinterpret_cast<char*>(a); }
static float* f32(uint64_t a) { return reinterpret_cast<float*>(a); }

// Tensors a terabyte apart would leave the address space: `num` of `count` values, 1 GiB each for every kind.
static std::vector<lr_param> tensors(int num, int64_t count) {
  std::vector<lr_param> v;
  const uint64_t step = (static_cast<uint64_t>(count) * 4 + 4096) / 4096 * 4096;
  uint64_t at = 1 << 20;
  for (int i = 0; i < num; ++i) {
    lr_param p{f32(at), fake(at + step), fake(at + 2 * step), fake(at + 3 * step), f32(at + 4 * step), count};
    at += 5 * step;
    v.push_back(p);
  }
  return v;
}

int main() {
  int devices = 0;
  if (hipGetDeviceCount(&devices) != hipSuccess) devices = 0;
  if (devices > 0) {
    std::printf("(GPU present: nothing is called)\nALL OK\n");
    return 0;
  }
  const uint64_t G = uint64_t(1) << 40;
  // draws and log-probabilities: the largest sizes pass the checks and fail at the launch; beyond them LR_E_SIZE
  for (int32_t k : {1, 3, 16, 1000, 2048, 2049, 65536}) {
    for (int32_t s : {1, 1024}) {
      EXPECT(lr_policy_draw(f32(G), f32(3 * G), f32(2 * G), s, 1000, k, reinterpret_cast<int32_t*>(fake(2 * G + (1 << 30))),
                            f32(2 * G + (3LL << 30)), nullptr, nullptr) == LR_E_HIP);
      EXPECT(lr_policy_logp(f32(G), reinterpret_cast<int32_t*>(fake(2 * G)), s, 1000, k, f32(3 * G), nullptr) == LR_E_HIP);
    }
  }
  EXPECT(lr_policy_logp(f32(G), reinterpret_cast<int32_t*>(fake(2 * G)), 1024, INT64_MAX, 65536, f32(3 * G), nullptr) == LR_E_SIZE);
  EXPECT(lr_policy_logp(f32(G), reinterpret_cast<int32_t*>(fake(2 * G)), INT32_MAX, 1, 1, f32(3 * G), nullptr) == LR_E_SIZE);
  EXPECT(lr_policy_logp(f32(G), reinterpret_cast<int32_t*>(fake(2 * G)), 1, INT64_MIN, 1, f32(3 * G), nullptr) == LR_E_SIZE);
  // the loss: every grid and shared-memory size
  const lr_policy pol{0.2f, 0.2f, 0.1f, 0.01f, 1.f};
  const size_t w = static_cast<size_t>(lr_policy_workspace_size());
  for (int32_t k = 1; k <= 65536; k = k < 2100 ? k + 13 : k * 2 - 7) {
    for (int32_t s : {1, 7, 64, 1024}) {
      for (int64_t n : {int64_t(1), int64_t(999), int64_t(1) << 22}) {
        for (int32_t gt : {0, 1}) {
          EXPECT(lr_policy_loss(&pol, f32(8 * G), reinterpret_cast<int32_t*>(fake(2 * G)), f32(3 * G), f32(4 * G),
                                f32(5 * G), 1, s, n, k, f32(6 * G), f32(6 * G + 64), gt, fake(12 * G), fake(7 * G), w,
                                nullptr) == LR_E_HIP);
        }
      }
    }
  }
  // the optimiser: list building at the limits, every overlap found wherever it stands
  for (int num : {1, 67, 68, 69, 136, 137, 198, 199, 1000, LR_MAX_PARAMS}) {
    std::vector<lr_param> t = tensors(num, 1000);
    const int64_t need = lr_grad_norm_workspace_size(num);
    EXPECT(need > 0);
    EXPECT(lr_grad_norm(t.data(), num, LR_GRAD_BF16, f32(8 * G), fake(9 * G), static_cast<size_t>(need), nullptr) == LR_E_HIP);
    for (int st : {0, 1})
      EXPECT(lr_adamw_update(t.data(), num, LR_GRAD_F32, st, 1, 0.1f, 0.9f, 0.999f, 1e-8f, 0.f, f32(8 * G), 1.f, 7u,
                             nullptr) == LR_E_HIP);
    const int at = num / 2;
    std::vector<lr_param> bad = t;
    bad[at].d_m = fake(reinterpret_cast<uint64_t>(t[num - 1].d_param) + 3999);
    EXPECT(lr_adamw_update(bad.data(), num, LR_GRAD_F32, LR_STATE_F32, 1, 0.1f, 0.9f, 0.999f, 1e-8f, 0.f, nullptr, 1.f, 7u,
                           nullptr) == LR_E_ALIAS);
    bad = t;
    bad[0].d_param = f32(reinterpret_cast<uint64_t>(t[at].d_grad) - 4);
    EXPECT(lr_adamw_update(bad.data(), num, LR_GRAD_F32, LR_STATE_F32, 1, 0.1f, 0.9f, 0.999f, 1e-8f, 0.f, nullptr, 1.f, 7u,
                           nullptr) == LR_E_ALIAS);
    std::vector<float*> m, v;
    for (int i = 0; i < num; ++i) {
      m.push_back(f32(4 * G + static_cast<uint64_t>(i) * 8192));
      v.push_back(f32(5 * G + static_cast<uint64_t>(i) * 8192));
    }
    EXPECT(lr_adamw_moments(t.data(), num, m.data(), v.data(), nullptr) == LR_E_HIP);
    v[at] = reinterpret_cast<float*>(t[0].d_scales);
    EXPECT(lr_adamw_moments(t.data(), num, m.data(), v.data(), nullptr) == LR_E_ALIAS);
  }
  std::vector<lr_param> large = tensors(1, LR_MAX_PARAM_VALUES);
  EXPECT(lr_adamw_update(large.data(), 1, 0, 1, INT32_MAX, 0.1f, 0.9f, 0.999f, 1e-8f, 0.f, nullptr, INFINITY, UINT32_MAX,
                         nullptr) == LR_E_HIP);
  large.push_back(lr_param{f32(1 << 12), fake(1 << 13), fake(1 << 14), fake(1 << 15), f32(1 << 16), 1});
  EXPECT(lr_adamw_update(large.data(), 2, 0, 1, 1, 0.1f, 0.9f, 0.999f, 1e-8f, 0.f, nullptr, 1.f, 0, nullptr) == LR_E_SIZE);
  large[1].count = INT64_MAX;
  EXPECT(lr_grad_norm(large.data(), 2, 0, f32(8 * G), fake(9 * G), size_t(1) << 30, nullptr) == LR_E_SIZE);
  EXPECT(lr_grad_norm(nullptr, 0, 0, f32(8 * G), fake(9 * G), size_t(1) << 30, nullptr) == LR_E_HIP);
  if (g_fail) {
    std::printf("%d failures\n", g_fail);
    return 1;
  }
  std::printf("ALL OK\n");
  return 0;
}
