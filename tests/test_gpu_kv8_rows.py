"""Rows into and out of a cache of 8 bits, bit for bit against the definition in 64 bits."""
import dataclasses

import pytest
import torch

import workload as wl
from tests import kv8_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import paper_2503_14153_amd as sd
    sd.lib()
    return sd


def model_of(sd, layers=1, heads=4, dim=64, max_rows=64, dtype="bf16", **more):
    shape = dataclasses.replace(wl.preset("tiny").model, n_layers=layers, n_heads=heads, head_dim=dim, d_model=heads * dim, dtype=dtype, **more)
    return sd.Model(shape, {k: v.cuda() for k, v in wl.make_weights(shape).items()}, max_rows)


def rows_of(n, heads, dim, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, dim), generator=g) * scale
    x[:, :, 3] *= 20.0                                 # a dim of large values
    x[:, 0] *= 1e-3                                    # a head of small ones
    return x.to(torch.bfloat16)


def same(got, want):
    got, want = got.double().cpu(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want)), float((got - want).abs().nan_to_num().max())


@pytest.mark.parametrize("heads,dim", [(4, 64), (3, 128), (1, 128)])
@pytest.mark.parametrize("at,n", [(0, 1), (0, 32), (0, 33), (31, 2), (5, 7), (64, 32), (1, 130), (95, 0)])
def test_rows_written_into_an_empty_cache_read_back_as_the_definition_says(sd, heads, dim, at, n):
    model = model_of(sd, heads=heads, dim=dim) if heads * dim % 32 == 0 else pytest.skip("width")
    kv = sd.KVCache(model, 2, 200, rows="e4m3")
    k, v = rows_of(n, heads, dim, 1), rows_of(n, heads, dim, 2, 3.0)
    kv.write_rows(0, 1, at, k.cuda(), v.cuda())
    got = kv.read_rows(0, 1, at, n)
    for x, y in zip((k, v), got):
        whole = torch.cat([torch.zeros((at, heads, dim), dtype=torch.bfloat16), x])
        same(y, ref.held(whole)[at:])
    other = kv.read_rows(0, 0, 0, 200)
    assert float(other[0].abs().max()) == 0.0 and float(other[1].abs().max()) == 0.0


def test_every_bfloat16_number_is_rounded_as_the_definition_says(sd):
    model = model_of(sd, heads=4, dim=64)
    kv = sd.KVCache(model, 1, 64, rows="e4m3")
    bits = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    # blocks whose largest number is fixed by one entry, the others running through the numbers up to it
    for top in (448.0, 449.0, 1.0, 0.875, 0.876953125, 3e38, 2.0 ** -120, 2.0 ** -126, 0.0):
        t = torch.tensor(top).to(torch.bfloat16)
        small = bits[(bits.float().abs() <= t.float()) | ~torch.isfinite(bits.float())]
        for c in range(0, small.numel(), 32 * 4 * 64 - 4):
            part = small[c:c + 32 * 4 * 64 - 4]
            x = torch.zeros(32, 4, 64, dtype=torch.bfloat16)
            x.view(-1)[:part.numel()] = part
            x[31, :, 63] = t
            kv.write_rows(0, 0, 0, x.cuda(), (-x).cuda())
            k, v = kv.read_rows(0, 0, 0, 32)
            same(k, ref.held(x))
            same(v, ref.held(-x))


def test_a_block_that_gets_larger_rows_keeps_its_values(sd):
    model = model_of(sd, heads=4, dim=128)
    kv = sd.KVCache(model, 1, 96, rows="e4m3")
    first, more = rows_of(20, 4, 128, 3), rows_of(30, 4, 128, 4, 100.0)
    kv.write_rows(0, 0, 0, first.cuda(), first.cuda())
    kv.write_rows(0, 0, 20, more.cuda(), more.cuda())
    whole = torch.cat([ref.held(first), more.double()])
    for x in kv.read_rows(0, 0, 0, 50):
        same(x, ref.held(whole))
    # and one that is patched in its middle, by smaller rows
    kv.write_rows(0, 0, 24, first[:3].cuda(), first[:3].cuda())
    again = ref.held(whole)
    again[24:27] = first[:3].double()
    for x in kv.read_rows(0, 0, 0, 50):
        same(x, ref.held(again))


def test_infinities_and_nan_become_nan_and_leave_the_others_alone(sd):
    model = model_of(sd, heads=4, dim=64)
    kv = sd.KVCache(model, 1, 64, rows="e4m3")
    x = rows_of(32, 4, 64, 5)
    x[3, 1, 7], x[9, 2, 0], x[31, 3, 63] = float("inf"), float("nan"), float("-inf")
    kv.write_rows(0, 0, 0, x.cuda(), x.cuda())
    for y in kv.read_rows(0, 0, 0, 32):
        same(y, ref.held(x))
        assert int(torch.isnan(y).sum()) == 3


@pytest.mark.parametrize("rows", ["e4m3", "model"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_all_layers_in_one_call(sd, rows, dtype):
    if rows == "e4m3" and dtype == "f32":
        pytest.skip("8-bit rows need a bfloat16 model")
    L, nh, hd = 3, 4, 64
    model = model_of(sd, layers=L, heads=nh, dim=hd, dtype=dtype)
    kv = sd.KVCache(model, 2, 100, rows=rows)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    k, v = (torch.stack([rows_of(50, nh, hd, s + l) for l in range(L)]).to(t) for s in (10, 20))
    kv.write_layers(1, 17, k.cuda(), v.cuda())
    got = kv.read_layers(1, 17, 50)
    for l in range(L):
        one = kv.read_rows(l, 1, 17, 50)
        for x, y, z in zip((k, v), got, one):
            assert torch.equal(y[l], z)
            whole = torch.cat([torch.zeros((17, nh, hd), dtype=t), x[l]])
            same(z, ref.held(whole)[17:] if rows == "e4m3" else x[l].double())


@pytest.mark.parametrize("n", [1, 40])
def test_arrays_of_any_alignment(sd, n):
    model = model_of(sd, heads=4, dim=64)
    kv = sd.KVCache(model, 1, 64, rows="e4m3")
    x = rows_of(n, 4, 64, 6).cuda()
    off = torch.empty(x.numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view_as(x).copy_(x)
    kv.write_rows(0, 0, 3, off, off)
    k, v = kv.read_rows(0, 0, 3, n)
    out = torch.full((x.numel() + 2,), 7.0, dtype=torch.bfloat16, device="cuda")
    sd.binding._check(sd.lib().sd_kv_read_rows(kv.handle, 0, 0, 3, n, out[1:].data_ptr(), torch.empty_like(x).data_ptr(), sd.binding._stream()))
    want = ref.held(torch.cat([torch.zeros((3, 4, 64), dtype=torch.bfloat16), x.cpu()]))[3:]
    same(k, want)
    same(v, want)
    same(out[1:-1].view_as(x), want)
    assert float(out[0]) == 7.0 and float(out[-1]) == 7.0
