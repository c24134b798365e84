"""Sums of the norm's gradients on the GPU: any of them alone, for vectors of one token and of many, beside all of them.

Tolerances as in test_gpu_block_norm: 4e-5 of the sum of absolute values, and of the largest term for each of the terms' square root."""
import pytest
import torch

import block_reference as ref
import paper_2509_25401_amd as pkg

pytestmark = pytest.mark.gpu
SUMS = ("dshift", "dscale", "dgate", "dweight", "dpost_weight")


# one token to a vector, a few, one chunk and several, more than 32 chunks to a vector (folded first), one vector
@pytest.mark.parametrize("frames,per,C,v32", [(700, 1, 264, False), (3000, 1, 64, True), (2100, 2, 72, False), (300, 7, 1160, True), (16, 129, 520, False),
                                              (3, 700, 1001, False), (1, 9001, 256, True), (1, 1, 40, False)])
@pytest.mark.parametrize("post", [False, True])
def test_each_sum_alone(frames, per, C, v32, post):
    print(f"[case] norm sums {frames} {per} {C} {v32} {post}", flush=True)
    rows, g = frames * per, torch.Generator().manual_seed(frames + C)
    vt = torch.float32 if v32 else torch.bfloat16

    def normal(*shape, dtype=torch.bfloat16, mean=0.0):
        return (torch.randn(*shape, generator=g) * 0.5 + mean).to(dtype)

    dh, dxo, x, y = (normal(rows, C) for _ in range(4))
    scale, gate, weight = normal(frames, C, dtype=vt), normal(frames, C, dtype=vt), normal(C, dtype=vt, mean=1.0)
    post_weight = normal(C, dtype=vt, mean=1.0) if post else None
    names = [n for n in SUMS if post or n != "dpost_weight"]
    gpu = {n: t.cuda() for n, t in dict(scale=scale.view(1, frames, C), gate=gate.view(1, frames, C), weight=weight).items()}
    if post:
        gpu["post_weight"] = post_weight.cuda()

    def call(which):
        out = {n: torch.full((C,) if "weight" in n else (1, frames, C), 7.0, device="cuda") for n in which}
        dx, dy = torch.empty_like(x, device="cuda"), torch.empty_like(y, device="cuda")
        pkg.sparse_block_norm_backward(*(t.cuda().view(1, rows, C) for t in (dh, dxo, x, y)), dx.view(1, rows, C), dy.view(1, rows, C), eps=1e-3, **gpu, **out)
        return out, dx, dy

    all_, dx, dy = call(names)
    want = ref.block_norm_backward(dh, dxo, x, y, True, 1e-3, weight, scale, gate, post_weight, 1e-3, 1.0, per)
    std = ref.moments(x.double(), True, 1e-3)[1]
    size = ((x.double().abs().amax(1, True) / std + 1) * (1 + dh.double().abs().amax(1, True) * 8 / std) + dxo.double().abs().amax(1, True)).max()
    for n, t in all_.items():
        total, of_abs = want[n]
        terms = rows if total.dim() == 1 else per
        assert ((t.cpu().double().view(total.shape) - total).abs() <= 4e-5 * of_abs + 4e-5 * size * terms ** 0.5 * (terms if total.dim() == 1 else 1) ** 0.5).all(), n
    for which in [[n] for n in names] + [[], ["dshift", "dweight"], ["dscale", "dgate"]]:
        some, dx2, dy2 = call(which)
        assert torch.equal(dx2, dx) and torch.equal(dy2, dy)
        assert all(torch.equal(some[n], all_[n]) for n in which), f"{which}: another result than beside the other sums"
