"""The forward pass of differential attention on the GPU within what its roundings
cost, each counted once: half a step of every probability of each map (of the type,
relative; in fp16 at least 2^-25), the 32-bit sums, and half a step of the result."""
import math

import pytest
import torch

import token_refs as refs
from paper_2007_09835_amd import build, layers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build(force=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("frame", [0, 9])
@pytest.mark.parametrize("n,lq,lk,hq,hk,d", [(2, 60, 60, 4, 2, 32), (1, 200, 330, 2, 1, 64), (1, 3, 1500, 2, 2, 128),
                                             (1, 100, 100, 1, 1, 104), (1, 33, 700, 3, 1, 16)])
def test_output_and_second_map(n, lq, lk, hq, hk, d, frame, dtype):
    gen = torch.Generator().manual_seed(lk + d)
    r = lambda *s: torch.randn(s, generator=gen)
    q, k = refs.rounded(r(n, lq, hq, 2, d), dtype), refs.rounded(r(n, lk, hk, 2, d), dtype)
    v, lam = refs.rounded(r(n, lk, hk, 2 * d) + 0.3, dtype), r(hq) * 0.2 + 0.6
    o, (_, o2, _) = layers.diff_attention(q[0].cuda(), k[0].cuda(), v[0].cuda(), lam.cuda(), frame, save=True)
    h, half, tiny = (0.0 if dtype == "f32" else refs.HALF[dtype]), max(refs.HALF[dtype], refs.U), refs.TINY[dtype]
    limit = torch.tensor([refs.visible(i, lq, lk, frame) for i in range(lq)])
    seen = torch.arange(lk)[None] < limit[:, None]
    for b in range(n):
        for head in range(hq):
            g, l = head // (hq // hk), float(lam[head])
            vv, maps, errs = v[1][b, :, g], [], []
            for m in range(2):
                qq, kk = q[1][b, :, head, m], k[1][b, :, g, m]
                s = (qq @ kk.T / math.sqrt(d)).masked_fill(~seen, -math.inf)
                p = torch.nan_to_num(torch.softmax(s, 1))
                size = torch.where(seen, qq.abs() @ kk.abs().T / math.sqrt(d), torch.zeros(()).double())
                rel = refs.U * ((d + 8) * size + 16 + (lk / 32 + 16))
                rel = rel + rel.max(1, keepdim=True).values
                maps.append(p @ vv)
                errs.append((p * (h + rel + refs.U * (lk + 8)) + tiny * seen) @ vv.abs())
            want, err = maps[0] - l * maps[1], errs[0] + abs(l) * errs[1]
            refs.within(o[b, :, head], want, err + half * (want.abs() + err) + 4 * tiny + 1e-30, "o")
            refs.within(o2[b, :, head], maps[1], errs[1] + half * (maps[1].abs() + errs[1]) + 4 * tiny + 1e-30, "o2")
