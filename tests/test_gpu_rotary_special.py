"""Rotary heads on the GPU: channels behind the turned ones pass as they are, whatever their neighbours or the position hold.

Tolerances: a turned channel is rounded to bf16 once, 2^-8 of its size, behind fp32 rounding of its pair, 4e-6 of the larger."""
import pytest
import torch

import block_reference as ref
import paper_2509_25401_amd as pkg

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
CASES = [(64, (16, 24, 0), "adjacent"), (32, (2, 4), "adjacent"), (128, (10, 56, 56), "adjacent"), (128, (8, 24), "halves"), (256, (64, 96, 88), "halves"),
         (64, (0,), "adjacent"), (64, (0,), "halves")]


def _equal(got, want, what):
    got = got.cpu().double()
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN in other places"
    assert torch.equal(got.isinf(), want.isinf()), f"{what}: infinities in other places"
    fine = want.isfinite()
    largest = torch.where(fine, want, torch.zeros_like(want)).abs().amax()
    assert torch.equal(got[want.isinf()], want[want.isinf()])
    assert ((got - want)[fine].abs() <= 2.0 ** -8 * want[fine].abs() + 4e-6 * largest).all(), what


def _spoilt(t, R):
    """Non-finite values in some of the channels from R on, others beside them untouched."""
    n = t.shape[-1] - R
    for i, v in enumerate((INF, -INF, NAN)):
        t[:, i::3, ..., R + (2 * i) % n] = v
    t[:, 0, ..., R + n - 1] = INF
    return t


@pytest.mark.parametrize("D,axes,pairs", CASES)
def test_channels_that_are_not_turned_pass_as_they_are(D, axes, pairs):
    print(f"[case] rotary special {D} {axes} {pairs}", flush=True)
    B, L, Hq, Hkv, R, halves = 2, 19, 3, 2, sum(axes), pairs == "halves"
    g = torch.Generator().manual_seed(D + R)
    pos = torch.randint(-40, 4000, (L, len(axes)), generator=g, dtype=torch.int32)
    freq = pkg.sparse_rotary_frequencies(axes, 500.0)
    angle = ref.angles(pos, axes, freq)
    heads = _spoilt(torch.randn(B, L, Hq + 2 * Hkv, D, generator=g).bfloat16(), R)
    qkv = heads.view(B, L, -1)
    call = dict(axes=axes, theta=500.0, pairs=pairs)
    got = [torch.zeros(B, n, L, D, dtype=torch.bfloat16, device="cuda") for n in (Hq, Hkv, Hkv)]
    pkg.sparse_rotary_heads(qkv.cuda(), pos.cuda(), *got, **call)
    for t, w, name in zip(got, ref.rotary(qkv, angle, Hq, Hkv, D, halves, None, None, 1e-6), "QKV"):
        _equal(t, w, name)
        assert torch.equal(t.cpu()[..., R:].float().nan_to_num(7.0), w[..., R:].float().nan_to_num(7.0)), f"{name}: a passing channel has changed"
    grads = [_spoilt(torch.randn(B, n, L, D, generator=g).bfloat16(), R) for n in (Hq, Hkv, Hkv)]
    dqkv = torch.zeros(qkv.shape, dtype=torch.bfloat16, device="cuda")
    pkg.sparse_rotary_heads_backward(*(t.cuda() for t in grads), None, pos.cuda(), dqkv, **call)
    _equal(dqkv, ref.rotary_backward(*grads, None, angle, halves, None, None, 1e-6)[0], "dqkv")


@pytest.mark.parametrize("D,axes,pairs", [c for c in CASES if sum(c[1])])
def test_positions_that_are_no_numbers_reach_the_turned_channels_alone(D, axes, pairs):
    print(f"[case] rotary position special {D} {axes} {pairs}", flush=True)
    B, L, H, R = 1, 9, 2, sum(axes)
    g = torch.Generator().manual_seed(D + R)
    pos = torch.rand(L, len(axes), generator=g) * 50
    pos[2], pos[5, 0], pos[7, -1] = NAN, INF, -INF
    qkv = torch.randn(B, L, 3 * H * D, generator=g).bfloat16()
    call = dict(axes=axes, pairs=pairs)
    got = [torch.zeros(B, H, L, D, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    pkg.sparse_rotary_heads(qkv.cuda(), pos.cuda(), *got, **call)
    heads = qkv.view(B, L, 3 * H, D).transpose(1, 2)
    bad = torch.zeros(L, R // 2, dtype=torch.bool)
    axis = torch.tensor([a for a, d in enumerate(axes) for _ in range(d // 2)])
    for l, a in ((2, None), (5, 0), (7, len(axes) - 1)):
        bad[l] |= torch.ones_like(axis, dtype=torch.bool) if a is None else axis == a
    bad = torch.cat((bad, bad), 1) if pairs == "halves" else bad.repeat_interleave(2, 1)
    for i, t in enumerate(got[:2]):
        t = t.cpu()
        assert torch.equal(t[..., R:], heads[:, i * H:(i + 1) * H, :, R:]), "a passing channel has changed"
        assert torch.equal(t[..., :R].isnan(), bad.expand(B, H, L, R)), "NaN in other places"


@pytest.mark.parametrize("Hq,Hkv", [(6, 2), (5, 1), (2, 3)])
def test_grouped_heads_as_slices_of_one_tensor(Hq, Hkv):
    print(f"[case] rotary slices {Hq} {Hkv}", flush=True)
    B, L, D, axes = 2, 37, 64, (16, 24, 24)
    g = torch.Generator().manual_seed(Hq)
    qkv = torch.randn(B, L, (Hq + 2 * Hkv) * D, generator=g).bfloat16().cuda()
    pos = torch.randint(0, 99, (L, 3), generator=g, dtype=torch.int32).cuda()
    apart = [torch.zeros(B, n, L, D, dtype=torch.bfloat16, device="cuda") for n in (Hq, Hkv, Hkv)]
    pkg.sparse_rotary_heads(qkv, pos, *apart, axes=axes)
    want = torch.cat(apart, dim=1)
    heads = torch.zeros(B, Hq + 2 * Hkv, L, D, dtype=torch.bfloat16, device="cuda")
    tokens = torch.zeros(B, L, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    for whole in (heads, tokens.transpose(1, 2)):
        pkg.sparse_rotary_heads(qkv, pos, whole[:, :Hq], whole[:, Hq:Hq + Hkv], whole[:, Hq + Hkv:], axes=axes)
        assert torch.equal(whole, want)
