"""The operators round the cache where their launches change: replays beyond the captured lengths, bounds far ahead of them, waves
with more than 64 blocks, as many (layer, head) pairs as fill the chip, caches of more than 2^20 rows and of more than 4 GiB."""
import pytest
import torch

import workload as wl
from tests import kv8_reference as ref
from tests.test_gpu_kv8_rows import model_of, rows_of, same
from tests.test_gpu_kv8_steps import near, twins
from tests.test_gpu_kv_sequences import after_drop, held, layers_of
from tests.test_gpu_tree_attention import check, filled, qkv, tree_of

pytestmark = pytest.mark.gpu

FORMATS = [("f32", "model"), ("bf16", "model"), ("bf16", "e4m3")]


@pytest.fixture(scope="module")
def sd():
    import paper_2503_14153_amd as sd
    sd.lib()
    return sd


# ---------------------------------------------------------------------------------------------- attention
@pytest.mark.parametrize("T", [1, 16, 64])
@pytest.mark.parametrize("captured", [[40, 0], [900, 300]])
def test_replays_follow_the_lengths(sd, T, captured):
    """Captured at some lengths, replayed at others (shorter, empty, the whole cache): the launch stays, the rows are the device's."""
    nh, hd, cap = 4, 64, 1000
    model = model_of(sd, heads=nh, dim=hd, max_rows=128, n_medusa=4, topk=10)
    tree, parent = tree_of(sd, T, 4, 10)
    kv, cached = filled(sd, model, [cap, cap], cap, 30)
    args = qkv(2, T, nh, hd, 2)
    kv.set_len(captured)
    out = torch.zeros_like(args[0])
    sd.tree_attention(model, kv, tree, 0, *args, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.tree_attention(model, kv, tree, 0, *args, out=out)
    sees = ref.ancestors(parent)
    for lens in (captured, [cap, cap], [0, 1], [33, cap], [cap, 0], captured):
        kv.set_len(lens)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        check(sd, model, kv, tree, parent, lens, cached, *args)
        for b, n in enumerate(lens):
            keys = torch.cat([ref.held(cached[b][0])[:n], args[1][b].double().cpu()])
            values = torch.cat([ref.held(cached[b][1])[:n], args[2][b].double().cpu()])
            want, spread, reach = ref.attention(args[0][b].cpu(), keys, values, torch.cat([torch.ones(T, n, dtype=torch.bool), sees], dim=1))
            assert bool(((out[b].double().cpu() - want).abs() <= ref.attention_bound(want, spread, reach, hd, n + T)).all()), (b, n)


@pytest.mark.parametrize("T", [1, 48])
def test_bounds_far_ahead_of_the_lengths(sd, T):
    nh, hd, n = 4, 64, 70
    model = model_of(sd, heads=nh, dim=hd, n_medusa=4, topk=10)
    tree, parent = tree_of(sd, T, 4, 10)
    kv = sd.KVCache(model, 1, 3000, rows="e4m3")
    sd.prefill(model, kv, torch.arange(40, dtype=torch.int32, device="cuda"), [40])     # leaves 40 rows that can be committed
    cached = [(rows_of(n, nh, hd, 1), rows_of(n, nh, hd, 2))]
    kv.set_len([0])
    kv.write_rows(0, 0, 0, cached[0][0].cuda(), cached[0][1].cuda())
    kv.set_len([n])
    slots, none = torch.zeros((1, 40), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(60):
        sd.kv_commit_rows(model, kv, slots, none)      # (each moves the host's bound by 40 rows, the device's length by none)
    check(sd, model, kv, tree, parent, [n], cached, *qkv(1, T, nh, hd, 3))


@pytest.mark.parametrize("T,B,n", [(1, 8, 9000), (16, 8, 8210), (64, 4, 9001)])
def test_waves_with_more_than_64_blocks(sd, T, B, n):
    """Sequences and heads enough that a long sequence is one part: a quarter of it per wave."""
    nh, hd = 64, 64
    model = model_of(sd, heads=nh, dim=hd, max_rows=256, n_medusa=4, topk=10)     # (rows: T in 32s, of every sequence)
    tree, parent = tree_of(sd, T, 4, 10)
    lens = [40 * b for b in range(B - 1)] + [n]
    kv, cached = filled(sd, model, lens, n + 70, 90)
    q, k, v = qkv(B, T, nh, hd, 4)
    out = sd.tree_attention(model, kv, tree, 0, q, k, v)
    sees = ref.ancestors(parent)
    for b, m in enumerate(lens):
        for h in (0, 37, 63):
            pick = slice(h, h + 1)
            keys = torch.cat([ref.held(cached[b][0][:, pick]), k[b, :, pick].double().cpu()])
            values = torch.cat([ref.held(cached[b][1][:, pick]), v[b, :, pick].double().cpu()])
            want, spread, reach = ref.attention(q[b, :, pick].cpu(), keys, values, torch.cat([torch.ones(T, m, dtype=torch.bool), sees], dim=1))
            off = (out[b, :, pick].double().cpu() - want).abs()
            assert bool((off <= ref.attention_bound(want, spread, reach, hd, m + T)).all()), (b, h, float(off.max()))


def test_a_step_whose_waves_have_more_than_64_blocks(sd):
    model = model_of(sd, layers=1, heads=64, dim=64, max_rows=256, n_medusa=4, topk=10)
    lens = [9000, 5, 0, 33, 64, 500, 1, 1200]
    eight, sixteen = sd.KVCache(model, 8, 9100, rows="e4m3"), sd.KVCache(model, 8, 9100)
    for b, n in enumerate(lens):
        if n:
            eight.write_rows(0, b, 0, *(rows_of(n, 64, 64, b + 9 * p).cuda() for p in (0, 1)))
            sixteen.write_rows(0, b, 0, *eight.read_rows(0, b, 0, n))
    for kv in (eight, sixteen):
        kv.set_len(lens)
        kv.set_draft(torch.arange(8), torch.arange(320).reshape(8, 4, 10))
    tree = sd.Tree(*wl.default_tree(16, 4, 10), 4, 10)
    words = torch.from_numpy(wl.pack_mask_words(wl.stop_set(model.shape.vocab, 0.3)).view("int32")).cuda()
    near(*(sd.spec_step(model, kv, tree, words, want_logits=True).logits for kv in (eight, sixteen)), layers=1)


# ---------------------------------------------------------------------------------------------- sequences
MANY = [(100, [(3, 2), (60, 1)]), (1500, [(10, 600)]), (1500, [(10, 30), (100, 600)])]


@pytest.mark.parametrize("dtype,rows", FORMATS)
@pytest.mark.parametrize("layers", [130, 260])
def test_as_many_layers_and_heads_as_fill_the_chip(sd, dtype, rows, layers):
    """More than 1024 and more than 2048 (layer, head, plane) triples: every workgroup walks its blocks alone."""
    heads, dim = 4, 64
    model = model_of(sd, layers=layers, heads=heads, dim=dim, dtype=dtype)
    kv = sd.KVCache(model, 3, 1510, rows=rows)
    for n, ranges in MANY:
        x = [t.repeat(layers // 2, 1, 1, 1) for t in layers_of(2, n, heads, dim, 3, dtype)]       # (layers 0, 1, 0, 1 ...)
        kv.write_layers(1, 0, *(t.cuda() for t in x))
        kv.set_len([5, n, 0])
        kv.fork(1, kv, [2, 0])
        kv.drop_rows(1, ranges)
        left = n - sum(c for _, c in ranges)
        assert kv.len() == [n, left, n]
        got, other = kv.read_layers(1, 0, left), kv.read_layers(2, 0, n)
        for p in (0, 1):
            for l in (0, 1):
                inside = held(x[p][l:l + 1], rows)[0]
                same_rows = torch.equal(other[p][l].double().cpu(), inside)
                assert same_rows
                want = after_drop(inside, n, ranges, 1e4, p, dtype, rows)
                off = (got[p][l].double().cpu() - want).abs()
                assert bool((off <= (2.0 ** -23 * want.abs() + 1e-14 if dtype == "f32" and p == 0 else 0.0 * want)).all()), float(off.max())
            for l in range(2, layers):                 # the others as those two, to the bit
                assert torch.equal(got[p][l], got[p][l % 2]) and torch.equal(other[p][l], other[p][l % 2])


@pytest.mark.parametrize("dtype,rows", FORMATS)
@pytest.mark.parametrize("ranges", [[(100, 600)], [(100, 600), (900, 5), (1200, 300)], [(0, 513), (1023, 1), (1500, 600)], [(5, 1990)]])
def test_gaps_of_many_blocks_are_closed_in_runs(sd, dtype, rows, ranges):
    heads, dim, n = 2, 128, 2000
    model = model_of(sd, heads=heads, dim=dim, dtype=dtype)
    kv = sd.KVCache(model, 1, 2100, rows=rows)
    x = layers_of(1, n, heads, dim, 5, dtype)
    kv.write_layers(0, 0, *(t.cuda() for t in x))
    kv.set_len([n])
    kv.drop_rows(0, ranges)
    left = n - sum(max(0, min(c, n - f)) for f, c in ranges)
    assert kv.len() == [left]
    for p, got in enumerate(kv.read_layers(0, 0, left)):
        want = after_drop(held(x[p], rows)[0], n, ranges, 1e4, p, dtype, rows)
        off = (got[0].double().cpu() - want).abs()
        assert bool((off <= (2.0 ** -23 * want.abs() + 1e-14 if dtype == "f32" and p == 0 else 0.0 * want)).all()), float(off.max())


@pytest.mark.parametrize("rows", ["model", "e4m3"])
def test_graph_mode_steps_go_on_after_forks_drops_and_scaled_positions(sd, rows):
    model = model_of(sd, layers=2, heads=4, dim=64, max_rows=64, n_medusa=4, topk=10)
    tree = sd.Tree(*wl.default_tree(16, 4, 10), 4, 10)
    words = torch.from_numpy(wl.pack_mask_words(wl.stop_set(model.shape.vocab, 0.3)).view("int32")).cuda()
    seen = []
    for graphs in (False, True):
        model.set_graph_mode(graphs)
        model.set_rope(sd.Rope(model.shape.rope_theta, 64))
        eight, sixteen = twins(sd, model, [300, 20], 700, 11)
        kv, log, out = eight if rows == "e4m3" else sixteen, [], None

        def step():
            nonlocal out
            out = sd.spec_step(model, kv, tree, words, want_logits=True, out=out)
            log.append((out.tokens.clone(), out.logits.clone(), kv.len()))
        for _ in range(3):
            step()
        kv.fork(0, kv, [1])
        for _ in range(3):
            step()
        assert torch.equal(out.logits[0], out.logits[1])
        kv.drop_rows(1, [(30, 100)])
        for _ in range(3):
            step()
        model.set_rope(sd.Rope(model.shape.rope_theta, 64, scaling="linear", factor=2.0))
        for _ in range(3):
            step()
        seen.append(log)
    model.set_graph_mode(False)
    for (a, x, n), (b, y, m) in zip(*seen):
        assert torch.equal(a, b) and torch.equal(x, y) and n == m


def test_another_stream(sd):
    heads, dim, n, T = 4, 64, 200, 16
    model = model_of(sd, layers=2, heads=heads, dim=dim)
    tree, parent = tree_of(sd, T)
    k, v = layers_of(2, n, heads, dim, 6, "bf16")
    args = qkv(1, T, heads, dim, 1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        kv = sd.KVCache(model, 2, 300, rows="e4m3")
        kv.write_layers(0, 0, k.cuda(), v.cuda())
        kv.set_len([n, 0])
        kv.fork(0, kv, [1])
        kv.drop_rows(0, [(20, 50)])
        out = sd.tree_attention(model, kv, tree, 1, *(t.repeat(2, 1, 1, 1) for t in args))
    side.synchronize()
    assert kv.len() == [n - 50, n]
    cached = [(after_drop(held(k, "e4m3")[1], n, [(20, 50)], 1e4, 0, "bf16", "e4m3"), after_drop(held(v, "e4m3")[1], n, [(20, 50)], 1e4, 1, "bf16", "e4m3")),
              (held(k, "e4m3")[1], held(v, "e4m3")[1])]
    sees = ref.ancestors(parent)
    for b, m in ((0, n - 50), (1, n)):
        keys, values = (torch.cat([c, t[0].double().cpu()]) for c, t in zip(cached[b], args[1:]))
        want, spread, reach = ref.attention(args[0][0].cpu(), keys, values, torch.cat([torch.ones(T, m, dtype=torch.bool), sees], dim=1))
        assert bool(((out[b].double().cpu() - want).abs() <= ref.attention_bound(want, spread, reach, dim, m + T)).all())


# ---------------------------------------------------------------------------------------------- large caches
def test_more_than_a_million_rows(sd):
    n, heads, dim = 2 ** 20 + 70, 4, 64
    model = model_of(sd, heads=heads, dim=dim)
    kv = sd.KVCache(model, 1, n + 10, rows="e4m3")
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((1, n, heads, dim), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    kv.write_layers(0, 3, k, v)
    got = kv.read_layers(0, 3, n)
    for x, y in zip((k, v), got):
        off = (x.float() - y.float()).abs()
        # half a step of e4m3 (2^-4 of a value), or of its subnormals: 2^-10 units, of which the largest is more than 224
        most = x.float().abs().max()
        assert bool((off <= 2.0 ** -4 * x.float().abs() + 2.0 ** -10 / 224 * most).all())
        for at in (29, 2 ** 20 - 3 - 32, 2 ** 20 - 3, 2 ** 20 + 29):      # whole blocks, to the bit
            same(y[0, at:at + 32], ref.held(x[0, at:at + 32].cpu()))
    kv.set_len([n + 3])
    tree, parent = tree_of(sd, 1)
    args = qkv(1, 1, heads, dim, 1)
    out = sd.tree_attention(model, kv, tree, 0, *args)
    keys, values = (torch.cat([torch.zeros((3, heads, dim), dtype=torch.float64), x[0].cpu().double(), t[0].cpu().double()]) for x, t in zip(got, args[1:]))
    want, spread, reach = ref.attention(args[0][0].cpu(), keys, values, torch.ones((1, n + 4), dtype=torch.bool))
    assert bool(((out[0].double().cpu() - want).abs() <= ref.attention_bound(want, spread, reach, dim, n + 4)).all())


@pytest.mark.parametrize("rows", ["model", "e4m3"])
def test_offsets_past_32_bits(sd, rows):
    heads, dim, cap, n = 8, 128, 620_000 if rows == "e4m3" else 310_000, 300
    model = model_of(sd, layers=2, heads=heads, dim=dim, max_rows=256)
    kv = sd.KVCache(model, 8, cap, rows=rows)          # sequence 7 of layer 0 begins past 4 GiB of keys
    k, v = layers_of(2, n, heads, dim, 8, "bf16")
    kv.write_layers(7, 0, k.cuda(), v.cuda())
    kv.write_layers(6, cap - n, k.cuda(), v.cuda())
    kv.set_len([0] * 7 + [n])
    kv.fork(7, kv, [0])
    kv.drop_rows(7, [(40, 130)])
    assert kv.len() == [n] + [0] * 6 + [n - 130]
    for seq, at in ((0, 0), (6, cap - n)):
        for x, y in zip((k, v), kv.read_layers(seq, at, n)):
            if rows == "model" or at % 32 == 0:
                same(y, held(x, rows))
    for p, y in enumerate(kv.read_layers(7, 0, n - 130)):
        for l in range(2):
            same(y[l], after_drop(held((k, v)[p], rows)[l], n, [(40, 130)], 1e4, p, "bf16", rows))
    if rows == "e4m3":
        tree, parent = tree_of(sd, 16)
        args = qkv(8, 16, heads, dim, 1)
        out = sd.tree_attention(model, kv, tree, 1, *args)
        for b, left in ((0, n), (7, n - 130)):
            cached = [held(x, rows)[1] for x in (k, v)] if b == 0 else [after_drop(held((k, v)[p], rows)[1], n, [(40, 130)], 1e4, p, "bf16", rows) for p in (0, 1)]
            keys, values = (torch.cat([c, t[b].double().cpu()]) for c, t in zip(cached, args[1:]))
            sees = torch.cat([torch.ones(16, left, dtype=torch.bool), ref.ancestors(parent)], dim=1)
            want, spread, reach = ref.attention(args[0][b].cpu(), keys, values, sees)
            assert bool(((out[b].double().cpu() - want).abs() <= ref.attention_bound(want, spread, reach, dim, left + 16)).all())


def test_a_step_needs_a_draft_state_of_every_sequence(sd):
    model = model_of(sd, layers=1, heads=4, dim=64)
    ready, bare = sd.KVCache(model, 1, 100, rows="e4m3"), sd.KVCache(model, 1, 100, rows="e4m3")
    sd.prefill(model, ready, torch.arange(20, dtype=torch.int32, device="cuda"), [20])
    kv = sd.KVCache(model, 2, 100, rows="e4m3")

    def refused():
        with pytest.raises(sd.SpecDecError) as e:
            sd.greedy_step(model, kv)
        assert e.value.name == "SD_ERR_STATE"
    refused()
    ready.fork(0, kv, [1])
    refused()
    ready.fork(0, kv, [0])
    a = sd.greedy_step(model, kv)
    assert kv.len() == [21, 21] and torch.equal(a.tokens[0], a.tokens[1])
    bare.fork(0, kv, [1])
    refused()
    kv.fork(0, kv, [1])
    sd.greedy_step(model, kv)
    assert kv.len() == [22, 22]


def test_more_than_a_million_rows_are_rotated(sd):
    n = 2 ** 20 + 77
    x = torch.randn((n, 1, 64), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") % 5000
    rope = sd.Rope(1e4, 64)
    got = sd.rope_rows(x, pos, rope)
    for at in (0, 2 ** 20 - 50, 2 ** 20 - 1, n - 60):   # the same rows in calls of their own, to the bit
        assert torch.equal(got[at:at + 60], sd.rope_rows(x[at:at + 60].contiguous(), pos[at:at + 60].contiguous(), rope))


@pytest.mark.parametrize("dtype,rows", FORMATS)
@pytest.mark.parametrize("ranges", [[(40, 30)], [(10, 600)]])
def test_nan_stays_in_its_pair(sd, dtype, rows, ranges):
    heads, dim, n = 4, 64, 700
    model = model_of(sd, heads=heads, dim=dim, dtype=dtype)
    kv = sd.KVCache(model, 1, 720, rows=rows)
    x = layers_of(1, n, heads, dim, 13, dtype)
    for t in x:
        for row, head, e in ((5, 0, 3), (39, 1, 40), (50, 2, 0), (71, 3, 63), (650, 0, 31), (699, 2, 32)):
            t[0, row, head, e] = float("nan")
    kv.write_layers(0, 0, *(t.cuda() for t in x))
    kv.set_len([n])
    kv.fork(0, kv2 := sd.KVCache(model, 1, 720, rows=rows), [0])
    for t, got in zip(x, kv2.read_layers(0, 0, n)):
        same(got, held(t, rows))
    kv.drop_rows(0, ranges)
    left = n - ranges[0][1]
    for p, got in enumerate(kv.read_layers(0, 0, left)):
        want = after_drop(held(x[p], rows)[0], n, ranges, 1e4, p, dtype, rows)
        got = got[0].double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and int(torch.isnan(want).sum()) >= 3
        off = (got - want).abs().nan_to_num()
        assert bool((off <= (2.0 ** -23 * want.abs().nan_to_num() + 1e-14 if dtype == "f32" and p == 0 else 0.0)).all()), float(off.max())


def test_attention_over_nan_and_infinite_rows(sd):
    """A cached NaN is seen by every row of its head and by no other head; one in the tree by its descendants alone."""
    nh, hd, T, n = 4, 64, 40, 100
    model = model_of(sd, heads=nh, dim=hd, n_medusa=4, topk=10)
    tree, parent = tree_of(sd, T, 4, 10)
    kv, cached = filled(sd, model, [n], 200, 21)
    q, k, v = qkv(1, T, nh, hd, 22)
    clean = sd.tree_attention(model, kv, tree, 0, q, k, v)
    bad_k, bad_v = cached[0][0].clone(), cached[0][1].clone()
    bad_k[37, 1, 5] = float("inf")
    bad_v[99, 2, 7] = float("nan")
    kv.write_rows(0, 0, 0, bad_k.cuda(), bad_v.cuda())
    out = sd.tree_attention(model, kv, tree, 0, q, k, v)
    assert torch.equal(out[:, :, [0, 3]], clean[:, :, [0, 3]])
    assert bool(torch.isnan(out[:, :, 1]).all())
    assert bool(torch.isnan(out[:, :, 2, 7]).all()) and torch.equal(out[:, :, 2, :7], clean[:, :, 2, :7])
    kv.write_rows(0, 0, 0, cached[0][0].cuda(), cached[0][1].cuda())
    k2 = k.clone()
    k2[0, 3, 0, 0] = float("nan")
    out = sd.tree_attention(model, kv, tree, 0, q, k2, v)
    sees = ref.ancestors(parent)[:, 3].cuda()
    assert torch.equal(torch.isnan(out[0, :, 0]).all(dim=1), sees) and torch.equal(out[0, ~sees], clean[0, ~sees])
    assert torch.equal(out[:, :, 1:], clean[:, :, 1:])


@pytest.mark.parametrize("dtype,rows", FORMATS)
@pytest.mark.parametrize("heads,dim", [(4, 64), (2, 128)])
@pytest.mark.parametrize("ranges", [[(100, 800)], [(31, 770), (1000, 1), (1900, 200)], [(0, 1025), (1200, 900)]])
def test_longer_gaps_are_closed_in_runs(sd, dtype, rows, heads, dim, ranges):
    n = 3500
    model = model_of(sd, layers=2, heads=heads, dim=dim, dtype=dtype)
    kv = sd.KVCache(model, 2, 3600, rows=rows)
    x = layers_of(2, n, heads, dim, 17, dtype)
    kv.write_layers(1, 0, *(t.cuda() for t in x))
    kv.set_len([0, n])
    kv.drop_rows(1, ranges)
    left = n - sum(c for _, c in ranges)
    assert kv.len() == [0, left]
    for p, got in enumerate(kv.read_layers(1, 0, left)):
        for l in range(2):
            want = after_drop(held(x[p], rows)[l], n, ranges, 1e4, p, dtype, rows)
            off = (got[l].double().cpu() - want).abs()
            assert bool((off <= (2.0 ** -23 * want.abs() + 1e-14 if dtype == "f32" and p == 0 else 0.0 * want)).all()), float(off.max())
