"""Meetings of warps inside a block: what was written is seen, and nobody waits for a warp that has given up (needs a B200)."""
import ctypes as C

import pytest
import torch

import native_probe

pytestmark = pytest.mark.gpu

SOURCE = r"""
#include "espo_attn_common.cuh"
using namespace espo;
// Four warps meet `rounds` times and pass a number on; in round `leaver` warp 0 gives up instead, as a warp whose wait ran out does.
__global__ void probe(int rounds, int leaver, int* met, int* sum) {
  __shared__ uint64_t bar;
  __shared__ int abort_flag, box[2][4];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    mbar_init(&bar, 4);
    abort_flag = 0;
    mbar_init_fence();
  }
  __syncthreads();
  uint32_t parity = 0;
  int n = 0, s = 0;
  for (; n < rounds; ++n) {
    if (n == leaver && warp == 0) {
      *const_cast<volatile int*>(&abort_flag) = 1;
      break;
    }
    if (lane == 0) box[n & 1][warp] = n + warp;
    if (!warps_meet(&bar, parity, &abort_flag)) break;
    s += box[n & 1][(warp + 1) & 3];
  }
  if (lane == 0) {
    met[warp] = n;
    sum[warp] = s;
  }
}
extern "C" int run(int rounds, int leaver, int* met, int* sum) {
  probe<<<1, 128>>>(rounds, leaver, met, sum);
  return static_cast<int>(cudaDeviceSynchronize());
}
"""


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    return native_probe.compile_probe(SOURCE, tmp_path_factory.mktemp("probe"))


@pytest.mark.parametrize("rounds,leaver", [(1, -1), (1000, -1), (1000, 0), (1000, 1), (1000, 500)])
def test_warps_meet_and_none_is_left_waiting(probe, rounds, leaver):
    met, total = (torch.full((4,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    assert probe.run(rounds, leaver, C.c_void_p(met.data_ptr()), C.c_void_p(total.data_ptr())) == 0
    last = rounds if leaver < 0 else leaver
    assert met.tolist() == [last] * 4
    assert total.tolist() == [last * (last - 1) // 2 + last * ((w + 1) % 4) for w in range(4)]
