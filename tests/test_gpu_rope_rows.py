"""Rotation of natural rows against the formula in 64 bits; its inverse as the gradient; refusals are in test_kv_operators_host.py."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import paper_2503_14153_amd as sd
    sd.lib()
    return sd


def frequencies(r):
    out = []
    for i in range(r.rotary_dim // 2):
        f = r.theta ** (-2.0 * i / r.rotary_dim)
        if r.scaling == "linear":
            f /= r.factor
        elif r.scaling == "by_parts":
            t = r.trained_len * f / (2 * math.pi)
            g = min(1.0, max(0.0, (t - r.low) / (r.high - r.low)))
            f *= g + (1 - g) / r.factor
        out.append(f)
    return torch.tensor(out, dtype=torch.float64)


def rotated(x, pos, r, inverse=False):
    x, rd = x.double().cpu(), r.rotary_dim
    w = pos.cpu().double()[:, None] * frequencies(r) * (-1.0 if inverse else 1.0)
    c, s = (g(w)[:, None, :] * r.magnitude for g in (torch.cos, torch.sin))
    y = x.clone()
    i = torch.arange(rd // 2)
    p, q = (i, i + rd // 2) if r.layout == "half" else (2 * i, 2 * i + 1)
    y[..., p] = x[..., p] * c - x[..., q] * s
    y[..., q] = x[..., p] * s + x[..., q] * c
    return y


def bound(x, want, r, dtype, pos):
    """Cosine and sine in float32: the turn is rounded to 2^-25 (2^-25 * 2 pi < 2^-22 of the pair) and the functions are good to
    2^-22; two products and a sum, 2^-22 of the pair's magnitudes; the angle itself, a float64 product: 2^-52 of it. bfloat16
    rounds the result by 2^-8 of itself."""
    x = x.double().cpu().abs()
    pair = r.magnitude * x.amax(dim=-1, keepdim=True) * 2
    far = float(pos.abs().max()) * 2.0 ** -52 * 4 if pos.numel() else 0.0
    return pair * (3 * 2.0 ** -22 + far) + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0.0) + 1e-38


CASES = [dict(), dict(layout="interleaved"), dict(scaling="linear", factor=4.0), dict(scaling="by_parts", factor=8.0, trained_len=2048),
         dict(layout="interleaved", scaling="by_parts", factor=32.0, trained_len=8192, magnitude=1.25)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("heads,dim,rd", [(1, 64, 64), (8, 128, 128), (5, 128, 32), (3, 96, 48), (2, 64, 20), (7, 10, 6), (4, 256, 256)])
@pytest.mark.parametrize("n", [1, 5, 2100])
def test_rows(sd, dtype, case, heads, dim, rd, n):
    r = sd.Rope(1e4, rd, **case)
    g = torch.Generator().manual_seed(n)
    x = torch.randn((n, heads, dim), generator=g).to(dtype).cuda()
    pos = torch.randint(-100, 200000, (n,), generator=g, dtype=torch.int32).cuda()
    for inverse in (False, True):
        want = rotated(x, pos, r, inverse)
        got = sd.rope_rows(x, pos, r, inverse=inverse)
        assert bool(((got.double().cpu() - want).abs() <= bound(x, want, r, dtype, pos)).all())
        assert torch.equal(got[..., rd:], x[..., rd:])
        here = x.clone()
        assert sd.rope_rows(here, pos, r, inverse=inverse, out=here) is here and torch.equal(here, got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_queries_and_keys_of_a_packed_projection_and_odd_alignments(sd, dtype, layout):
    n, nh, hd = 37, 4, 64
    r = sd.Rope(1e6, hd, layout=layout)
    packed = torch.randn((n, 3 * nh, hd), generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 31
    want = sd.rope_rows(packed[:, :2 * nh].contiguous(), pos, r)
    before = packed.clone()
    assert torch.equal(sd.rope_rows(packed[:, :2 * nh], pos, r), want) and torch.equal(packed, before)
    sd.rope_rows(packed[:, :2 * nh], pos, r, out=packed[:, :2 * nh])
    assert torch.equal(packed[:, :2 * nh], want) and torch.equal(packed[:, 2 * nh:], before[:, 2 * nh:])
    flat = torch.empty(n * 2 * nh * hd + 1, dtype=dtype, device="cuda")[1:].view(n, 2 * nh, hd).copy_(before[:, :2 * nh])
    # (eight at a time or one by one: the same two products and sum)
    assert torch.equal(sd.rope_rows(flat, pos, r), want)


def test_extreme_positions(sd):
    r = sd.Rope(1e4, 64)
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1], dtype=torch.int32, device="cuda")
    x = torch.randn((6, 2, 64), generator=torch.Generator().manual_seed(2)).cuda()
    got, want = sd.rope_rows(x, pos, r), rotated(x, pos, r)
    assert bool(((got.double().cpu() - want).abs() <= bound(x, want, r, torch.float32, pos.double())).all())
    assert torch.equal(got[0], x[0])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_the_inverse_is_the_gradient(sd, layout):
    n, nh, hd, rd = 6, 2, 64, 32
    r = sd.Rope(1e4, rd, layout=layout, scaling="linear", factor=2.0, magnitude=1.5)
    g = torch.Generator().manual_seed(3)
    x, w = (torch.randn((n, nh, hd), generator=g) for _ in range(2))
    pos = torch.arange(n, dtype=torch.int32) * 100
    leaf = x.double().requires_grad_(True)
    c, s = (f(pos.double()[:, None] * frequencies(r))[:, None] * 1.5 for f in (torch.cos, torch.sin))
    if layout == "half":
        a, b = leaf[..., :rd // 2], leaf[..., rd // 2:rd]
        y = torch.cat([a * c - b * s, a * s + b * c, leaf[..., rd:]], dim=-1)
    else:
        a, b = leaf[..., 0:rd:2], leaf[..., 1:rd:2]
        y = torch.cat([torch.stack([a * c - b * s, a * s + b * c], dim=-1).flatten(-2), leaf[..., rd:]], dim=-1)
    (y * w.double()).sum().backward()
    got = sd.rope_rows(w.cuda(), pos.cuda(), r, inverse=True)
    lim = bound(w, leaf.grad, r, torch.float32, pos)
    assert bool(((got.double().cpu() - leaf.grad).abs() <= lim).all())
    # and against differences of the operator itself: it is linear, so a step of any size gives the slope
    for probe in (0, 17, 40):
        e = torch.zeros((n, nh, hd))
        e[:, :, probe] = 1.0
        up = sd.rope_rows((x + e).cuda(), pos.cuda(), r).double().cpu() - sd.rope_rows((x - e).cuda(), pos.cuda(), r).double().cpu()
        slope = (up / 2 * w.double()).sum(-1)
        # a sum of hd differences, each off by twice the bound above of values up to |x| + 1
        tol = hd * float(w.abs().max()) * float(bound(x.abs() + 1, y.detach(), r, torch.float32, pos).max())
        assert float((slope - got[..., probe].double().cpu()).abs().max()) <= tol


def test_nothing_to_rotate(sd):
    r = sd.Rope(1e4, 64)
    x = torch.empty((0, 4, 64), device="cuda")
    assert sd.rope_rows(x, torch.empty(0, dtype=torch.int32, device="cuda"), r).shape == (0, 4, 64)


def test_a_captured_rotation_replays_on_new_rows(sd):
    r = sd.Rope(1e4, 64)
    x = torch.randn((40, 4, 64), device="cuda")
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(x)
    sd.rope_rows(x, pos, r, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.rope_rows(x, pos, r, out=out)
    for i in range(3):
        x.normal_()
        pos += 7
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, sd.rope_rows(x, pos, r))
