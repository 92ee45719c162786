"""Room for the partial results of shared prefixes in contexts of very many heads: one part at least of every (request, head), the plan
of the requests' own rows and their parts."""
import shutil
import subprocess

import pytest
import torch

from paper_2506_15704_amd import build

MAIN = r"""
#include <cstdio>
#include "part_rooms.h"
using namespace lfps;
int main() {                                           // every context that lfps_create takes: batch * heads <= 65535
  long long shapes = 0, least = 1 << 30;
  for (int G = 1; G <= 4; G *= 2)
    for (int kv = 1; kv * G <= 65535; ++kv)
      for (int batch = 1; (long long)batch * kv * G <= 65535; ++batch, ++shapes) {
        const long long heads = (long long)batch * kv * G, rows = attn_part_rows_for(batch, kv * G, kv);
        const long long own = (long long)own_items_for(batch, kv) * kv * G, parts = rows - own - own_plan_rows_for(batch, kv);
        if (parts < heads) return printf("%d %d %d: room for %lld rows of %lld\n", batch, kv * G, kv, parts, heads), 1;
        if (own_plan_rows_for(batch, kv) * kPartFloats * 4 < 16LL * own_items_for(batch, kv) + 4 * (2LL * batch + 1)) return printf("plan\n"), 1;
        const long long usual = (2 * heads > 65536 ? 2 * heads : 65536) + 8192;
        if (rows < usual || (kv <= 1024 && rows != usual)) return printf("%d %d %d: %lld\n", batch, kv * G, kv, rows), 1;
        if (parts - heads < least) least = parts - heads;
      }
  printf("%lld shapes, %lld rows to spare\n", shapes, least);
}
"""


def test_there_is_room_for_one_part_of_every_head_and_the_own_rows(tmp_path):
    (tmp_path / "main.cpp").write_text(MAIN)
    compiler = shutil.which("g++") or build.hipcc()
    subprocess.run([compiler, "-std=c++17", "-O1", "-I", build.CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "rooms")], check=True)
    res = subprocess.run([str(tmp_path / "rooms")], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout
    assert int(res.stdout.split()[0]) > 500000


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,B,Hq,Hkv", [("bf16", 1, 32768, 8192), ("f32", 2, 24600, 12300), ("fp8kv", 1, 30000, 30000)])
def test_prefix_of_very_many_heads(dtype, B, Hq, Hkv):
    """All rows shared, none, some."""
    from tests.cache_case import CacheCase, D, ints
    from tests.harness import DEV, stored_values
    c = CacheCase(dtype, Hq, Hkv, [40 - 7 * i for i in range(B)], seed=1)
    q = c.randn(B, Hq, D)
    K, V = (stored_values(x).double().nan_to_num(0) for x in (c.K, c.V))
    for p in (40, 0, 13):
        out = torch.zeros((B, Hq, D), device=DEV)
        c.ctx.lfps_prefix_attn_decode(q, c.kv, ints([0, B]), ints([p]), out)
        for i in range(B):
            n = c.lens[i]
            k, v = (torch.cat([x[0, :, :min(p, n)], x[i, :, min(p, n):n]], 1) for x in (K, V))
            x = torch.matmul(q[i].double().view(Hkv, c.G, D), k.transpose(1, 2).contiguous()) / D ** 0.5
            w = torch.softmax(x, -1)
            dots = torch.matmul(q[i].double().abs().view(Hkv, c.G, D), k.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True) / D ** 0.5
            # query and weights as sums of 16-bit terms (2^-18 left of bf16 ones), fp32 products and sums, the scores' errors twice, the exponential 2^-21
            left = 0.0 if dtype == "f32" else 2.0 ** -18
            tol = (2 * (left + 260 * 2.0 ** -24) * dots + 2 * left + 2.0 ** -21 + 120 * 2.0 ** -24) * torch.matmul(w, v.abs()) + 1e-7
            assert bool(((out[i].view(Hkv, c.G, D).double() - torch.matmul(w, v)).abs() <= tol).all()), (p, i)
    c.ctx.close()
