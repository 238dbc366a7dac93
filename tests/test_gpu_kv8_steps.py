"""Steps, prompts and commits over a cache in 8 bits, and the operators round the cache used together.

Keys and values of layer 0 hang on tokens and positions alone, not on the cache, so what the 8-bit cache holds of them is known bit
for bit from a bfloat16 cache that ran the same tokens; deeper rows and logits are compared with a bfloat16 cache that holds the
same rounded rows. There the two differ in that queries and probabilities are rounded to bfloat16 (2^-8 each, so an attention
output by up to about 2^-7 of itself per layer, and what follows is added to a residual stream that holds more than that output):
relative errors of the logits stay below layers * 2^-7."""
import pytest
import torch

import workload as wl
from tests import kv8_reference as ref
from tests.test_gpu_kv8_rows import model_of, rows_of, same

pytestmark = pytest.mark.gpu

L, NH, HD = 2, 4, 64


@pytest.fixture(scope="module")
def sd():
    import paper_2503_14153_amd as sd
    sd.lib()
    return sd


def tree_and_stop(sd, model, T):
    s = model.shape
    tree = sd.Tree(*wl.default_tree(T, s.n_medusa, s.topk), s.n_medusa, s.topk)
    words = torch.from_numpy(wl.pack_mask_words(wl.stop_set(s.vocab, 0.3)).view("int32")).cuda()
    return tree, words


def near(a, b, layers=L):
    a, b = a.double(), b.double()
    assert torch.isfinite(a).all()
    assert float((a - b).norm() / b.norm()) <= layers * 2.0 ** -7


def twins(sd, model, lens, cap, seed):
    """Two caches with the same rows: in 8 bits, and their values in bfloat16."""
    eight, sixteen = sd.KVCache(model, len(lens), cap, rows="e4m3"), sd.KVCache(model, len(lens), cap)
    for b, n in enumerate(lens):
        if n:
            k, v = (torch.stack([rows_of(n, NH, HD, seed + 7 * b + l + 50 * p) for l in range(L)]).cuda() for p in (0, 1))
            eight.write_layers(b, 0, k, v)
            sixteen.write_layers(b, 0, *eight.read_layers(b, 0, n))
    g = torch.Generator().manual_seed(seed)
    root = torch.randint(0, model.shape.vocab, (len(lens),), generator=g)
    cand = torch.randint(0, model.shape.vocab, (len(lens), model.shape.n_medusa, model.shape.topk), generator=g)
    for kv in (eight, sixteen):
        kv.set_len(lens)
        kv.set_draft(root, cand)
    return eight, sixteen


@pytest.mark.parametrize("T,lens", [(16, [0]), (16, [100]), (16, [900]), (16, [31, 0, 400, 64]), (16, [1] * 8), (1, [333]), (1, [5, 700]),
                                    (1, [40] * 8), (48, [200]), (64, [500, 90])])
def test_a_step_sees_the_rounded_rows(sd, T, lens):
    model = model_of(sd, layers=L, heads=NH, dim=HD, max_rows=256, n_medusa=4, topk=10)
    eight, sixteen = twins(sd, model, lens, 1000, 3)
    if T == 1:
        a, b = (sd.greedy_step(model, kv, want_logits=True, want_head_logits=True) for kv in (eight, sixteen))
    else:
        tree, words = tree_and_stop(sd, model, T)
        a, b = (sd.spec_step(model, kv, tree, words, want_logits=True, want_head_logits=True, want_argmax=True) for kv in (eight, sixteen))
    near(a.logits, b.logits)
    near(a.head_logits, b.head_logits)
    assert [n + int(x) for n, x in zip(lens, a.n_accept)] == eight.len()


@pytest.mark.parametrize("n,slots", [(0, [0]), (31, [0, 3, 5]), (30, [0, 1, 2]), (64, [0, 2, 4, 9]), (77, [1, 1, 0]), (95, [0])])
def test_committed_rows_are_rounded_once_with_their_block(sd, n, slots):
    model = model_of(sd, layers=L, heads=NH, dim=HD, max_rows=64, n_medusa=4, topk=10)
    eight, sixteen = twins(sd, model, [n, n + 40], 300, 5)
    tree, words = tree_and_stop(sd, model, 16)
    prefix = [[x.clone() for x in eight.read_layers(b, 0, m)] if m else None for b, m in ((0, n), (1, n + 40))]
    src = torch.tensor([slots + [0] * (5 - len(slots)), [0, 1, 2, 3, 4]], dtype=torch.int32, device="cuda")
    count = torch.tensor([len(slots), 0], dtype=torch.int32, device="cuda")     # (sequence 1 gets none)
    huge = torch.full((L, 3, NH, HD), 3e4, dtype=torch.bfloat16, device="cuda")
    for kv in (eight, sixteen):
        sd.spec_step(model, kv, tree, words)           # leaves its tree rows in the model's scratch
        kv.set_len([n, n + 40])
        if kv is eight and n % 32 == 0:                # large rows past the end, in a block of new rows alone, must not count
            eight.write_layers(0, n + len(slots), huge, huge)
        sd.kv_commit_rows(model, kv, src, count)
        assert kv.len() == [n + len(slots), n + 40]
    new = sixteen.read_layers(0, n, len(slots))
    got = eight.read_layers(0, 0, n + len(slots))
    head = n // 32 * 32
    for p in (0, 1):
        whole = torch.cat([prefix[0][p][0].cpu() if n else torch.zeros((0, NH, HD), dtype=torch.bfloat16), new[p][0].cpu()])
        want = torch.cat([whole[:head].double(), ref.held(whole[head:])])
        same(got[p][0, :head], want[:head])
        same(got[p][0, n:], want[n:])
        kept_but_for_low_bits(got[p][0, head:n], want[head:n], whole[head:])
    if n:                                              # sequence 1: its last block has had the step's own rows
        for x, y, z in zip(prefix[1], eight.read_layers(1, 0, n + 40), sixteen.read_layers(1, 0, n + 45)):
            last = (n + 40) // 32 * 32
            same(y[:, :last], x[:, :last].cpu().double())
            for l in range(L):
                kept_but_for_low_bits(y[l, last:], x[l, last:].cpu().double(), z[l, last:].cpu())


def kept_but_for_low_bits(got, want, block):
    """Values of a block that got further rows: a code is a multiple of 2^-9 of the block's unit at the least, so a new unit moves a
    value by 2^-10 of it at most, and the block's largest is more than 224 units."""
    if got.numel():
        most = block.double().abs().amax(dim=(0, 2))[None, :, None] * (1 + 2.0 ** -4)
        assert bool(((got.double().cpu() - want).abs() <= 2.0 ** -10 / 224 * most).all())


@pytest.mark.parametrize("lens", [[1], [20], [64, 33], [300], [700, 5, 90]])
def test_prompts_in_passes_and_appended(sd, lens):
    model = model_of(sd, layers=L, heads=NH, dim=HD, max_rows=256, n_medusa=4, topk=10)
    B = len(lens)
    eight, sixteen = sd.KVCache(model, B, 1200, rows="e4m3"), sd.KVCache(model, B, 1200)
    g = torch.Generator().manual_seed(1)
    tokens = torch.randint(0, model.shape.vocab, (sum(lens),), generator=g, dtype=torch.int32).cuda()
    more = torch.randint(0, model.shape.vocab, (50 * B,), generator=g, dtype=torch.int32).cuda()
    for kv in (eight, sixteen):
        sd.prefill(model, kv, tokens, lens)
        sd.prefill(model, kv, more, [50] * B)
        assert kv.len() == [n + 50 for n in lens]
    for b, n in enumerate(lens):
        for x, y in zip(eight.read_layers(b, 0, n + 50), sixteen.read_layers(b, 0, n + 50)):
            # a block's rows may have come in several passes: each time it is rounded anew, which moves nothing but what lies
            # below 2^-15 of its largest. The bfloat16 cache takes long prompts in other passes (joined ones), whose projections
            # add up in another order: a row's bfloat16 number can fall to the next one, 2^-7 of it away, and that may lie on the
            # other side of a border between two e4m3 numbers, which are 2^-3 of each other apart at most. One number in some
            # 2^24 / 2^8 is so near a border of bfloat16, and an e4m3 step has sixteen of those.
            want = ref.held(y[0].cpu())
            off = (x[0].cpu().double() - want).abs()
            assert bool((off <= 2.0 ** -3 * want.abs() + 2.0 ** -17 * want.abs().max()).all())
            assert float((off > 0).double().mean()) < 1e-3
    out = sd.greedy_step(model, eight, want_logits=True)
    assert torch.isfinite(out.logits).all()


def test_graph_mode_is_the_same_to_the_bit(sd):
    model = model_of(sd, layers=L, heads=NH, dim=HD, max_rows=64, n_medusa=4, topk=10)
    tree, words = tree_and_stop(sd, model, 16)
    seen = []
    for graphs in (False, True):
        model.set_graph_mode(graphs)
        kv, _ = twins(sd, model, [30, 200], 400, 11)
        tokens, out = [], None
        for i in range(6):
            out = sd.spec_step(model, kv, tree, words, want_logits=True, out=out)
            tokens.append((out.tokens.clone(), out.logits.clone(), kv.len()))
            g = sd.greedy_step(model, kv)
            tokens.append((g.tokens.clone(), g.tokens.clone(), kv.len()))
        seen.append(tokens)
    for (a, x, n), (b, y, m) in zip(*seen):
        assert torch.equal(a, b) and torch.equal(x, y) and n == m


def test_bounds_that_run_ahead_of_the_lengths(sd):
    model = model_of(sd, layers=L, heads=NH, dim=HD, max_rows=64, n_medusa=4, topk=10)
    tree, words = tree_and_stop(sd, model, 16)
    a, _ = twins(sd, model, [100], 600, 13)
    b, _ = twins(sd, model, [100], 600, 13)
    for i in range(12):                                # (one of five rows accepted a step: the host's bound of `a` runs ahead)
        x, y = sd.spec_step(model, a, tree, words, want_logits=True), sd.spec_step(model, b, tree, words, want_logits=True)
        b.len()
        if not torch.equal(x.tokens, y.tokens):
            break                                      # (a near tie: the parts differ, and with them the order of sums)
        near(x.logits, y.logits)
    assert i >= 3


def test_the_other_settings_run(sd):
    model = model_of(sd, layers=L, heads=NH, dim=HD, max_rows=256, n_medusa=4, topk=10)
    tree, words = tree_and_stop(sd, model, 16)
    eight, sixteen = twins(sd, model, [300, 20], 500, 17)
    u = torch.tensor([0.3, 0.9], device="cuda")
    ty = dict(temperature=0.8, epsilon=0.09, delta=0.3, want_logits=True)
    near(sd.spec_step_typical(model, eight, tree, words, u, **ty).logits, sd.spec_step_typical(model, sixteen, tree, words, u, **ty).logits)
    model.set_fused(True)                              # has no effect on a cache in 8 bits
    eight2, _ = twins(sd, model, [300, 20], 500, 17)
    model.set_fused(False)
    eight3, _ = twins(sd, model, [300, 20], 500, 17)
    model.set_fused(True)
    x = sd.spec_step(model, eight2, tree, words, want_logits=True)
    model.set_fused(False)
    y = sd.spec_step(model, eight3, tree, words, want_logits=True)
    assert torch.equal(x.logits, y.logits) and torch.equal(x.tokens, y.tokens)
    model.set_draft_schedule("all_nodes")
    z = sd.spec_step(model, eight2, tree, words, want_head_logits=True)
    model.set_draft_schedule("after_accept")
    w = sd.spec_step(model, eight3, tree, words, want_head_logits=True)
    assert torch.equal(z.tokens, w.tokens)
    near(z.head_logits, w.head_logits)
    model.profile_begin()
    sd.spec_step(model, eight2, tree, words)
    p = model.profile_end()
    assert p["attn"]["launches"] == L


def test_head_dim_128(sd):
    model = model_of(sd, layers=L, heads=2, dim=128, max_rows=64, n_medusa=4, topk=10)
    tree, words = tree_and_stop(sd, model, 48)
    eight, sixteen = sd.KVCache(model, 1, 400, rows="e4m3"), sd.KVCache(model, 1, 400)
    k, v = (torch.stack([rows_of(250, 2, 128, l + 9 * p) for l in range(L)]).cuda() for p in (0, 1))
    eight.write_layers(0, 0, k, v)
    sixteen.write_layers(0, 0, *eight.read_layers(0, 0, 250))
    for kv in (eight, sixteen):
        kv.set_len([250])
        kv.set_draft([5], torch.arange(40).reshape(1, 4, 10))
    near(*(sd.spec_step(model, kv, tree, words, want_logits=True).logits for kv in (eight, sixteen)))


def test_scaled_positions_in_the_models_own_steps(sd):
    """sd_set_rope: keys of layer 0 are the unrotated ones (every angle tiny) rotated by the scaled frequencies."""
    n = 60
    for dtype in ("bf16", "f32"):
        model = model_of(sd, layers=1, heads=NH, dim=HD, max_rows=64, dtype=dtype)
        s = model.shape
        tokens = torch.randint(0, s.vocab, (n,), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()

        def keys(rope):
            kv = sd.KVCache(model, 1, 100)
            if rope is not None:
                model.set_rope(rope)
            sd.prefill(model, kv, tokens, [n])
            return kv.read_rows(0, 0, 0, n)[0]
        asis = keys(None)
        assert torch.equal(keys(sd.Rope(s.rope_theta, HD)), asis)
        still = keys(sd.Rope(s.rope_theta, HD, scaling="linear", factor=1e30))
        for rope in (sd.Rope(s.rope_theta, HD), sd.Rope(s.rope_theta, HD, scaling="linear", factor=4.0),
                     sd.Rope(s.rope_theta, HD, scaling="by_parts", factor=8.0, trained_len=32, magnitude=1.5)):
            want = sd.rope_rows(still, torch.arange(n, dtype=torch.int32, device="cuda"), rope).double()
            got = keys(rope).double()
            # bfloat16: `still` was rounded (2^-8 of each of a pair), so was its rotation, and so are the model's keys;
            # float32: the same with the functions' 2^-22
            step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -20
            a, b = still.double().abs().chunk(2, dim=-1)
            pair = torch.cat([a + b, a + b], dim=-1)
            assert bool(((got - want).abs() <= step * (rope.magnitude * pair + 2 * want.abs()) + 1e-6).all())
        with pytest.raises(sd.SpecDecError) as e:
            model.set_rope(sd.Rope(1e4, HD // 2))
        assert e.value.name == "SD_ERR_SHAPE"
        with pytest.raises(sd.SpecDecError):
            model.set_rope(sd.Rope(1e4, HD, layout="interleaved"))


def test_the_operators_together(sd):
    """A prompt; four samples of it; each goes on by itself; one loses a part of its context and goes on: and the same by hand, stage
    by stage, for one layer: rotate, write, attend, accept, append."""
    model = model_of(sd, layers=L, heads=NH, dim=HD, max_rows=256, n_medusa=4, topk=10)
    tree, words = tree_and_stop(sd, model, 16)
    one, four = sd.KVCache(model, 1, 400, rows="e4m3"), sd.KVCache(model, 4, 400, rows="e4m3")
    tokens = torch.randint(0, model.shape.vocab, (150,), generator=torch.Generator().manual_seed(4), dtype=torch.int32).cuda()
    sd.prefill(model, one, tokens, [150])
    one.fork(0, four, range(4))
    u = torch.tensor([0.1, 0.4, 0.6, 0.9], device="cuda")
    ty = dict(temperature=0.8, epsilon=0.09, delta=0.3)
    first = sd.spec_step_typical(model, four, tree, words, u, **ty, want_logits=True)
    # the samples share their prompt: the same logits in the root's row, to the bit, whatever sequence of the batch they are
    for b in range(1, 4):
        assert torch.equal(first.logits[b, 0], first.logits[0, 0])
    lens = four.len()
    four.drop_rows(2, [(4, 60)])
    assert four.len() == [n - (60 if b == 2 else 0) for b, n in enumerate(lens)]
    before = [four.read_layers(b, 0, lens[b])[0].clone() for b in (0, 1, 3)]
    out = sd.spec_step_typical(model, four, tree, words, u.flip(0).contiguous(), **ty, want_logits=True)
    assert torch.isfinite(out.logits).all()
    for x, b in zip(before, (0, 1, 3)):
        head = lens[b] // 32 * 32
        assert torch.equal(four.read_layers(b, 0, lens[b])[0][:, :head], x[:, :head])

    # by hand
    T, n = 16, 90
    parent, depth, rank = wl.default_tree(T, 4, 10)
    rope = sd.Rope(model.shape.rope_theta, HD)
    kv = sd.KVCache(model, 1, 200, rows="e4m3")
    g = torch.Generator().manual_seed(6)
    cached, packed = (torch.randn((m, 3 * NH, HD), generator=g).to(torch.bfloat16).cuda() for m in (n, T))
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    here = torch.tensor([n + int(d) for d in depth], dtype=torch.int32, device="cuda")
    turned = sd.rope_rows(cached[:, :2 * NH], at, rope)
    kv.write_rows(0, 0, 0, turned[:, NH:].contiguous(), cached[:, 2 * NH:].contiguous())
    kv.set_len([n])
    sd.rope_rows(packed[:, :2 * NH], here, rope, out=packed[:, :2 * NH])
    q, k, v = packed.view(1, T, 3, NH, HD).unbind(2)
    got = sd.tree_attention(model, kv, tree, 0, q, k, v)
    keys = torch.cat([ref.held(turned[:, NH:].cpu()), k[0].double().cpu()])
    values = torch.cat([ref.held(cached[:, 2 * NH:].cpu()), v[0].double().cpu()])
    sees = torch.cat([torch.ones(T, n, dtype=torch.bool), ref.ancestors([int(p) for p in parent])], dim=1)
    want, spread, reach = ref.attention(q[0].cpu(), keys, values, sees)
    assert bool(((got[0].double().cpu() - want).abs() <= ref.attention_bound(want, spread, reach, HD, n + T)).all())
    am = torch.zeros((1, T), dtype=torch.int32, device="cuda")
    n_acc, _, _, slots = sd.verify_tree(tree, torch.zeros_like(am), am, words, model.shape.vocab)
    rows = slots[0, :int(n_acc[0])].long()
    kv.write_rows(0, 0, n, k[0, rows].contiguous(), v[0, rows].contiguous())
    kv.set_len([n + len(rows)])
    whole = torch.cat([ref.held(turned[:, NH:].cpu()), k[0, rows].cpu().double()])
    same(kv.read_rows(0, 0, 0, n + len(rows))[0], ref.held(whole))
