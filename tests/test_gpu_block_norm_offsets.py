"""Block norm and its gradients on the GPU where rows do not start on 16 bytes: every tensor at a shifted address, widths that are
whole runs of eight and others, with one row to a wave and with several waves to a row.  Tolerances are those of test_gpu_block_norm."""
import pytest
import torch

import block_reference as ref
import paper_2509_25401_amd as pkg
from test_gpu_block_norm import _case, _check_bf16_or_f32, _up

pytestmark = pytest.mark.gpu
# rows: few (several waves share one), many (one wave to a row up to 4096 channels); widths: below a run, one unit to a thread and more
ROWS_C = [(9, 5), (9, 8), (9, 64), (9, 1160), (9, 3073), (9, 4104), (9, 9001), (1600, 7), (1600, 64), (1600, 333), (1600, 519), (1600, 1160), (1600, 2109),
          (1600, 3072), (1600, 4095), (5, 16383)]


def _shifted(s, names, offset):
    return {n: _up(s[n], offset) for n in names}


@pytest.mark.parametrize("rows,C", ROWS_C)
@pytest.mark.parametrize("offset,x32,v32,post", [(1, False, False, False), (3, True, True, True), (1, False, True, True), (2, True, False, False)])
def test_forward(rows, C, offset, x32, v32, post):
    print(f"[case] block_norm offset {rows} {C} {offset} {x32} {v32} {post}", flush=True)
    s = _case(C + offset, 1, rows, C, 1, x32, v32, True, post)
    eps, alpha = 1e-5, 0.75
    gpu = _shifted(s, ("x", "y", "weight", "post_weight"), offset)
    vectors = {n: _up(s[n][0], offset) for n in ("scale", "shift", "gate")}
    guard_x, guard_h = (torch.full((rows * C + 2 * offset,), 7.0, dtype=t, device="cuda") for t in (s["x"].dtype, torch.bfloat16))
    xo, h = guard_x[offset:offset + rows * C].view(rows, C), guard_h[offset:offset + rows * C].view(rows, C)
    call = dict(eps=eps, alpha=alpha, weight=gpu["weight"], post_weight=gpu["post_weight"], **vectors)
    pkg.sparse_block_norm(gpu["x"], gpu["y"], h, xo, **call)
    for g in (guard_x, guard_h):
        assert (g[:offset] == 7.0).all() and (g[offset + rows * C:] == 7.0).all(), "written outside"
    want_x, want_h = ref.block_norm(s["x"], s["y"], True, eps, s["weight"], s["scale"], s["shift"], s["gate"], s["post_weight"], eps, alpha, rows)
    std, top = ref.moments(want_x, True, eps)[1], want_x.abs().amax(dim=1, keepdim=True)
    _check_bf16_or_f32(xo, want_x, 2e-5 * top, "x_out")
    size = (want_h - s["shift"].double()).abs().amax(dim=1, keepdim=True)
    _check_bf16_or_f32(h, want_h, 1e-5 * (size + 1) + 6e-6 * top / std * 8 + 4e-5 * top / std * (1 if post else 0), "h")
    alone = torch.empty_like(h)
    pkg.sparse_block_norm(gpu["x"], None, alone, eps=eps, weight=gpu["weight"], scale=vectors["scale"], shift=vectors["shift"])
    want_h = ref.block_norm(s["x"], None, True, eps, s["weight"], s["scale"], s["shift"], per=rows)[1]
    x = s["x"].double()
    std, top = ref.moments(x, True, eps)[1], x.abs().amax(dim=1, keepdim=True)
    size = (want_h - s["shift"].double()).abs().amax(dim=1, keepdim=True)
    _check_bf16_or_f32(alone, want_h, 1e-5 * (size + 1) + 6e-6 * top / std * 8, "h of x alone")
    kept, again = gpu["x"].clone(), torch.empty_like(h)
    moved = _up(kept.cpu(), offset)
    pkg.sparse_block_norm(moved, gpu["y"], again, moved, **call)
    assert torch.equal(moved, xo) and torch.equal(again, h), "in place"


@pytest.mark.parametrize("rows,C", ROWS_C)
@pytest.mark.parametrize("offset,x32,v32,post", [(1, False, False, False), (3, True, True, True), (1, False, True, True)])
def test_backward(rows, C, offset, x32, v32, post):
    print(f"[case] block_norm_backward offset {rows} {C} {offset} {x32} {v32} {post}", flush=True)
    s = _case(C + offset + 1, 1, rows, C, 1, x32, v32, True, post)
    eps, alpha, f32 = 1e-3, 0.75, dict(dtype=torch.float32, device="cuda")
    gpu = _shifted(s, ("dh", "dx_out", "x", "y", "weight", "post_weight"), offset)
    vectors = {n: _up(s[n][0], offset) for n in ("scale", "gate")}
    sums = {n: torch.full((C + 2,), 7.0, **f32)[1:1 + C] for n in ("dscale", "dshift", "dgate", "dweight") + (("dpost_weight",) if post else ())}
    guard_x, guard_y = (torch.full((rows * C + 2 * offset,), 7.0, dtype=t, device="cuda") for t in (s["x"].dtype, torch.bfloat16))
    dx, dy = guard_x[offset:offset + rows * C].view(rows, C), guard_y[offset:offset + rows * C].view(rows, C)
    pkg.sparse_block_norm_backward(gpu["dh"], gpu["dx_out"], gpu["x"], gpu["y"], dx, dy, eps=eps, weight=gpu["weight"], post_weight=gpu["post_weight"],
                                   alpha=alpha, **vectors, **sums)
    for g in (guard_x, guard_y):
        assert (g[:offset] == 7.0).all() and (g[offset + rows * C:] == 7.0).all(), "written outside"
    want = ref.block_norm_backward(s["dh"], s["dx_out"], s["x"], s["y"], True, eps, s["weight"], s["scale"], s["gate"], s["post_weight"], eps, alpha, rows)
    std = ref.moments(s["x"].double(), True, eps)[1]
    size = (s["x"].double().abs().amax(1, True) / std + 1) * (1 + s["dh"].double().abs().amax(1, True) * 8 / std) + s["dx_out"].double().abs().amax(1, True)
    _check_bf16_or_f32(dx, want["dx"], 2e-5 * size, "dx")
    std_y = ref.moments(s["y"].double(), False, eps)[1] if post else torch.ones_like(std)
    _check_bf16_or_f32(dy, want["dy"], 4e-5 * size * 8 / std_y, "dy")
    for name, t in sums.items():
        total, of_abs = (v.reshape(C) for v in want[name])
        err = (t.cpu().double() - total).abs()
        bound = 4e-5 * of_abs + 4e-5 * size.max() * rows + 1e-30
        assert (err <= bound).all(), f"{name}: off by up to {(err / bound).max():.2f} of the bound"
        held = t._base
        assert held[0] == 7.0 and held[-1] == 7.0, "written outside"
