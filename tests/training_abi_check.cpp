// Host-side driver of the training step's entry points for the sanitizer tier:
// struct layouts ("struct name size offsets..."), workspace sizes over a table of
// shapes ("norm T d status bytes", "loss|back T Nh dh Ne status bytes"), calls that must
// be refused ("FAIL ..." lines) and what AdamW launches (its launcher is a stub
// that looks the arguments over; the others abort).
#include <cstddef>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "mhlmoe.h"
#include "training_launch.hpp"

namespace {
int g_fail = 0;
void expect(const char* what, long long got, long long want) {
  if (got == want) return;
  std::printf("FAIL %s: %lld, expected %lld (%s)\n", what, got, want, mhlmoe_last_error());
  ++g_fail;
}
std::vector<mhl::AdamLaunch> g_launches;
std::vector<unsigned> g_groups;
}  // namespace

namespace mhl {
hipError_t launch_adamw(const AdamLaunch& a, unsigned workgroups, hipStream_t) {
  g_launches.push_back(a);
  g_groups.push_back(workgroups);
  return hipSuccess;
}
}  // namespace mhl

int main() {
  std::printf("struct tensor %zu %zu %zu %zu %zu %zu %zu %zu %zu %zu %zu %zu %zu\n",
              sizeof(mhlmoe_adamw_tensor), offsetof(mhlmoe_adamw_tensor, param),
              offsetof(mhlmoe_adamw_tensor, master), offsetof(mhlmoe_adamw_tensor, grad),
              offsetof(mhlmoe_adamw_tensor, m), offsetof(mhlmoe_adamw_tensor, v),
              offsetof(mhlmoe_adamw_tensor, m_scale), offsetof(mhlmoe_adamw_tensor, v_scale),
              offsetof(mhlmoe_adamw_tensor, n), offsetof(mhlmoe_adamw_tensor, weight_decay),
              offsetof(mhlmoe_adamw_tensor, seed), offsetof(mhlmoe_adamw_tensor, param_dtype),
              offsetof(mhlmoe_adamw_tensor, grad_dtype));
  std::printf("struct step %zu %zu %zu %zu %zu %zu %zu\n", sizeof(mhlmoe_adamw_step),
              offsetof(mhlmoe_adamw_step, lr), offsetof(mhlmoe_adamw_step, beta1),
              offsetof(mhlmoe_adamw_step, beta2), offsetof(mhlmoe_adamw_step, eps),
              offsetof(mhlmoe_adamw_step, step), offsetof(mhlmoe_adamw_step, grad_scale));
  const int64_t Ts[] = {0, 1, 63, 128, 4096, 65537, (int64_t(1) << 30) - 1, int64_t(1) << 30,
                        (int64_t(1) << 31) - 1, int64_t(1) << 31, -1, INT64_MAX, INT64_MIN};
  for (int64_t T : Ts) {
    for (int d : {0, 1, 16, 208, 1001, 4096, 16400, 65536, 65537, INT32_MAX, -16}) {
      size_t b = 0;
      const mhlmoe_status st = mhlmoe_layernorm_backward_workspace(T, d, &b);
      std::printf("norm %lld %d %d %zu\n", (long long)T, d, (int)st, st == MHLMOE_OK ? b : 0);
    }
    for (int Nh : {1, 3, 1024, 1025, 0})
      for (int Ne : {1, 32, 33, 200, 1024, 1025, 0, INT32_MAX})
        for (int dh : {64, 128, 96}) {
          size_t b = 0;
          mhlmoe_status st = mhlmoe_balance_loss_workspace(T, Nh, dh, Ne, &b);
          std::printf("loss %lld %d %d %d %d %zu\n", (long long)T, Nh, dh, Ne, (int)st,
                      st == MHLMOE_OK ? b : 0);
          st = mhlmoe_balance_loss_backward_workspace(T, Nh, dh, Ne, &b);
          std::printf("back %lld %d %d %d %d %zu\n", (long long)T, Nh, dh, Ne, (int)st,
                      st == MHLMOE_OK ? b : 0);
          // every launch is of fewer than 2^32 threads, the partial results' count is T's
          if (st == MHLMOE_OK) {
            const int64_t splits = mhl::balance_splits(T, Nh, dh, Ne);
            const int64_t groups = mhl::ceil_div(mhl::balance_blocks(Ne), mhl::balance_dw_blocks(T, Nh, dh, Ne));
            expect("splits", splits <= 1024 && (T == 0 || splits >= 1), 1);
            expect("dw", (Nh * splits + 7) * groups < (int64_t(1) << 24), 1);
            expect("tokens", Nh * mhl::balance_token_blocks(T, Nh, Ne) < (int64_t(1) << 24), 1);
          }
        }
  }
  // AdamW: 48 tensors to a launch, empty ones left out; the workgroups cover every tensor once
  const uintptr_t base = uintptr_t(1) << 44;
  auto tensor = [&](int64_t n, int at) {
    const uintptr_t a = base + ((uintptr_t)at << 46);
    auto p = [&](int k) { return reinterpret_cast<void*>(a + ((uintptr_t)k << 43)); };
    return mhlmoe_adamw_tensor{p(0), nullptr, p(1), p(2), p(3), static_cast<float*>(p(4)),
                               static_cast<float*>(p(5)), n, 0.1f, 7u, MHLMOE_BF16, MHLMOE_F32};
  };
  const mhlmoe_adamw_step step{1e-3, 0.9, 0.99, 1e-8, 3, nullptr};
  for (int count : {0, 1, 47, 48, 49, 100, 1000}) {
    std::vector<mhlmoe_adamw_tensor> t;
    int64_t full = 0;
    for (int i = 0; i < count; ++i) {
      t.push_back(tensor(i % 6 == 5 ? 0 : 1 + 1000 * i, i));
      full += t.back().n > 0;
    }
    g_launches.clear();
    g_groups.clear();
    expect("adamw", mhlmoe_adamw(t.data(), count, &step, nullptr), MHLMOE_OK);
    expect("launches", (long long)g_launches.size(), (full + 47) / 48);
    size_t k = 0;
    for (size_t l = 0; l < g_launches.size(); ++l) {
      const mhl::AdamLaunch& a = g_launches[l];
      int64_t next = 0;
      for (int j = 0; j < mhl::kAdamTensors; ++j) {
        if (a.first[j] == UINT32_MAX) continue;
        while (t[k].n == 0) ++k;
        expect("tensor", a.t[j].n == t[k].n && a.t[j].param == t[k].param, 1);
        expect("first", a.first[j], next);
        next += (t[k].n + a.chunk - 1) / a.chunk;
        ++k;
      }
      expect("groups", g_groups[l], next);
    }
  }
  for (int64_t n : {(int64_t)1 << 34, ((int64_t)1 << 40) - 1}) {  // larger chunks, not more workgroups
    g_launches.clear();
    g_groups.clear();
    mhlmoe_adamw_tensor t = tensor(n, 0);
    expect("large", mhlmoe_adamw(&t, 1, &step, nullptr), MHLMOE_OK);
    expect("large groups", g_groups[0] < (1u << 23) && g_groups[0] * g_launches[0].chunk >= n, 1);
  }
  mhlmoe_adamw_tensor t = tensor(int64_t(1) << 40, 0);
  expect("n", mhlmoe_adamw(&t, 1, &step, nullptr), MHLMOE_EUNSUPPORTED);
  std::printf("done %d failures\n", g_fail);
  return g_fail == 0 ? 0 : 1;
}
