"""GPU parity of the packed-batch operators (layout, rotary positions, attention) against the float64 oracle.

Attention: every value within packed_attention_bound(), which is first-order arithmetic for the worst case, and for bf16 the whole tensor to 4e-3 relative L2 as
well, which sees a single missing key among hundreds: a rounding to bf16 has an rms of at most 2^-8 / sqrt(3) = 2.3e-3, probabilities, normaliser and
output are rounded once each, together sqrt(3) 2.3e-3."""
import numpy as np
import pytest
import torch

from oracle import hyb_oracle as O
from oracle import packed_oracle as P
from paper_2602_21760_amd import synth
from gpu_util import dev, host, err, rel_l2, tdt, tol

pytestmark = pytest.mark.gpu

TOL_REL = {"bf16": 4e-3, "f32": 2e-6}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def hb():
    from paper_2602_21760_amd import binding
    binding.lib()
    return binding


def _offsets(lengths, start=0):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]) + start, dtype=torch.int32).cuda()


# ---- layout -------------------------------------------------------------------------------------------------------------------------------

def _run_layout(hb, shapes, capacity, text_after, with_request=True, with_positions=True):
    sh = torch.tensor(shapes, dtype=torch.int32).reshape(-1, 4).cuda()
    offsets = torch.full((len(shapes) + 1,), -9, dtype=torch.int32, device="cuda")
    request = torch.full((capacity,), -7, dtype=torch.int32, device="cuda") if with_request else None
    positions = torch.full((capacity, 3), -8, dtype=torch.int32, device="cuda") if with_positions else None
    hb.hyb_packed_layout(sh, offsets, request, positions, text_after)
    torch.cuda.synchronize()
    return tuple(None if t is None else t.cpu().numpy() for t in (offsets, request, positions))


def _random_shapes(n, seed, top=5):
    rng = np.random.default_rng(seed)
    s = rng.integers(0, top, (n, 4))
    s[rng.random(n) < 0.2] = 0
    s[rng.random(n) < 0.1, 1] = -3
    return s.tolist()


@pytest.mark.parametrize("text_after", [False, True])
@pytest.mark.parametrize("shapes,spare", [
    ([(1, 1, 1, 0)], 0), ([(0, 0, 0, 1)], 3), ([(1, 32, 33, 77)], 5), ([(3, 7, 5, 0), (1, 64, 64, 333), (2, 1, 9, 11)], 1), ([(0, 4, 4, 0), (1, 0, 3, 0)], 8), ([(1, 3, 3, 4)] * 9, -20),
    ([(-1, -2, -3, -4), (1, 2, 2, 1)], 2), (_random_shapes(255, 1), 7), (_random_shapes(2048, 2), 0), (_random_shapes(2049, 3), 13), (_random_shapes(5000, 4), -1000), (_random_shapes(20000, 6, 3), 9)])
def test_layout(hb, shapes, spare, text_after):
    total = int(P.packed_layout(shapes, 10 ** 9)[0][-1])
    capacity = max(total + spare, 0)
    want = P.packed_layout(shapes, capacity, text_after)
    offsets, request, positions = _run_layout(hb, shapes, capacity, text_after)
    rows = int(want[0][-1])
    np.testing.assert_array_equal(offsets, want[0])
    np.testing.assert_array_equal(request[:rows], want[1])
    np.testing.assert_array_equal(positions[:rows], want[2])
    assert (request[rows:] == -7).all() and (positions[rows:] == -8).all()      # rows behind the last request: as they were


@pytest.mark.parametrize("n", [3, 3000])
def test_layout_parts_of_it(hb, n):
    shapes = _random_shapes(n, 5)
    want = P.packed_layout(shapes, 10 ** 9)
    rows = int(want[0][-1])
    for r, p in ((True, False), (False, True), (False, False)):
        offsets, request, positions = _run_layout(hb, shapes, rows, False, r, p)
        np.testing.assert_array_equal(offsets, want[0])
        assert request is None or (request == want[1]).all()
        assert positions is None or (positions == want[2]).all()


def test_layout_of_nothing_and_of_too_much(hb):
    assert _run_layout(hb, [], 4, False)[0].tolist() == [0]
    assert _run_layout(hb, [(1, 2, 2, 2)], 0, False)[0].tolist() == [0, 0]
    big = 2 ** 31 - 1
    offsets, request, positions = _run_layout(hb, [(0, big, big, 3), (big, big, big, big), (1, 1, 1, 1)], 50, False)      # products beyond 64 bits
    assert offsets.tolist() == [0, 3, 50, 50]
    assert request.tolist() == [0] * 3 + [1] * 47
    np.testing.assert_array_equal(positions[:, 2], [0, 0, 0] + list(range(47)))
    assert not positions[:, :2].any()


# ---- rotary -------------------------------------------------------------------------------------------------------------------------------

# (tokens, q heads, k heads, head_dim, axis_dims, farthest position)
ROTARY = [(1, 1, 1, 64, (64,), 1000000), (5, 4, 2, 64, (16, 24, 24), 64), (333, 24, 24, 64, (20, 20, 24), 128), (130, 3, 1, 128, (42, 42, 44), 4096), (77, 12, 12, 64, (24, 24), 45),
          (9, 1, 0, 16, (2, 2, 4, 8), 10), (3, 512, 512, 32, (32,), 100), (4, 2, 3, 256, (256,), 2 ** 31 - 1), (1027, 1, 1, 16, (16,), 9), (40, 5, 5, 80, (32,), 300), (2, 7, 0, 48, (6, 10), 5)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("case", ROTARY, ids=[str(c[:5]).replace(" ", "") for c in ROTARY])
def test_rotary(hb, case, dt, halves, in_place):
    tokens, hq, hk, d, dims, far = case
    if halves and sum(dims) % 16:
        with pytest.raises(hb.HybError) as e:
            q = torch.zeros(tokens, hq, d, device="cuda", dtype=tdt(dt))
            hb.hyb_rotary(hb.rotary_desc(q, None, dims, pairs=hb.HYB_ROTARY_HALVES), torch.zeros(tokens, len(dims), dtype=torch.int32, device="cuda"), q)
        assert e.value.code == 2
        return
    rng = np.random.default_rng(tokens + d)
    pos = rng.integers(-far, far, (tokens, len(dims)))
    pos[0] = far - 1
    x = synth.normal(7, (tokens, hq + 2 * hk + 1, d), 1.0, dt)
    buf = dev(x, tdt(dt))                                  # q, k, v and a head that is not theirs
    q, k = buf[:, :hq], buf[:, hq:hq + hk] if hk else None
    p = torch.tensor(pos, dtype=torch.int32).cuda()
    pairs = hb.HYB_ROTARY_HALVES if halves else hb.HYB_ROTARY_NEIGHBOURS
    for inverse, q_scale, axis_scale in ((False, 1.0, None), (True, 0.18, [0.5] * len(dims))):
        buf.copy_(dev(x, tdt(dt)))
        outs = {} if in_place else {"q_out": torch.full((tokens, hq, d), 9.0, device="cuda", dtype=tdt(dt)),
                                    "k_out": torch.full((tokens, hk + 1, d), 9.0, device="cuda", dtype=tdt(dt))[:, :hk] if hk else None}
        desc = hb.rotary_desc(q, k, dims, 10000.0, pairs, axis_scale, q_scale, inverse, **outs)
        gq, gk = hb.hyb_rotary(desc, p, q, k, **outs)
        for got, ref, scale in ((gq, x[:, :hq], np.float32(q_scale)), (gk, x[:, hq:hq + hk], 1.0)):
            if got is None:
                continue
            want = P.rotary(ref, pos, dims, 10000.0, halves, axis_scale, inverse, float(scale))
            # (fp64 angles of far positions: 2^31 / (2 pi) turns to 2^-53 of themselves, twice: below 2^-20 of a radian)
            bound = P.rotary_bound(ref, HALF_STEP[dt], float(scale), dims, halves)(want) + (far > 2 ** 24) * 2.0 ** -19 * (np.abs(ref).max() * 2)
            assert (np.abs(host(got) - want) <= bound).all(), np.abs(host(got) - want).max()
        rest = buf[:, hq + hk:] if in_place else buf
        assert torch.equal(rest, dev(x, tdt(dt))[:, hq + hk:] if in_place else dev(x, tdt(dt)))        # the values and the neighbour, or everything, untouched


def test_rotary_gradient_is_the_inverse(hb):
    """d <g, rotary(x)> / dx against differences and against the formula."""
    dims, tokens = (16, 24, 24), 6
    x, g, step = (synth.normal(s, (tokens, 2, 64), 1.0, "f32") for s in (1, 2, 3))
    p = torch.arange(tokens * 3, dtype=torch.int32).reshape(tokens, 3).cuda()
    run = lambda t, inverse=False: host(hb.hyb_rotary(hb.rotary_desc(t, None, dims, inverse=inverse), p, t)[0])      # noqa: E731
    grad = run(dev(g), True)
    np.testing.assert_allclose(grad, P.rotary(g, p.cpu().numpy(), dims, inverse=True), atol=1e-5)
    eps = 2.0 ** -6      # the map is linear: a difference is exact but for fp32's rounding, about 2^-24 sqrt(768) 64 = 1e-4
    diff = ((run(dev(x + eps * step)) - run(dev(x - eps * step))) * g).sum() / (2 * eps)
    assert abs(diff - (grad * step).sum()) < 2e-3


def test_rotary_more_workgroups_than_one_grid_dimension_holds(hb):
    """2^28 + 37 tokens of one small head: more than 2^24 workgroups of 256 threads, 8.6 GB."""
    tokens = 2 ** 28 + 37
    q = torch.ones(tokens, 1, 16, device="cuda", dtype=torch.bfloat16)
    p = torch.arange(tokens, device="cuda", dtype=torch.int32).remainder_(1009)[:, None]
    hb.hyb_rotary(hb.rotary_desc(q, None, (16,)), p, q)
    rows = torch.cat([torch.arange(40), torch.tensor([2 ** 27 - 1, 2 ** 27, 2 ** 27 + 1, 123456789]), torch.arange(2 ** 28 - 40, tokens)])
    at = rows.cuda()
    x = np.ones((len(rows), 1, 16))
    want = P.rotary(x, p[at].cpu().numpy(), (16,))
    assert (np.abs(host(q[at]) - want) <= P.rotary_bound(x, 2.0 ** -8, axis_dims=(16,))(want)).all()
    # every row turned once and by its own angle: rows of one position are alike
    same = q[1009 * 7 + 5:1009 * 7 + 5 + 1009 * 266000].view(266000, 1009, 16)
    assert bool((same == same[0]).all())


def test_rotary_binding_refusals(hb):
    q = torch.zeros(8, 2, 64, device="cuda", dtype=torch.bfloat16)
    p = torch.zeros(8, 1, dtype=torch.int32, device="cuda")
    desc = hb.rotary_desc(q, None, (64,))
    for bad in ((p[:7], q), (p.long(), q), (p, q[:7]), (p, q.float()), (p.cpu(), q), (p, q.cpu())):
        with pytest.raises((ValueError, TypeError)):
            hb.hyb_rotary(desc, *bad)


# ---- attention ----------------------------------------------------------------------------------------------------------------------------

def _attention(hb, dt, lq, lk, hq, hk, d, causal=False, std=1.0, prescaled=False, seed=1, hints=True, spare=0, edit=None, layout="fused", scale=None):
    """Runs a packed batch and holds it against the oracle; `spare` rows before and behind the sequences; edit(q, k, v, cu_q, cu_k) changes the data."""
    nq, nk = sum(lq) + 2 * spare, sum(lk) + 2 * spare
    q = synth.normal(seed, (nq, hq, d), std * (d ** -0.5 * 1.4426950408889634 if prescaled else 1.0), dt)
    k, v = synth.normal(seed + 1, (nk, hk, d), 1.0, dt), synth.normal(seed + 2, (nk, hk, d), 1.0, dt)
    cu_q, cu_k = (np.concatenate([[0], np.cumsum(n)]) + spare for n in (lq, lk))
    if edit:
        edit(q, k, v, cu_q, cu_k)
    t = tdt(dt)
    if layout == "fused" and nq == nk:
        buf = torch.cat([dev(x, t) for x in (q, k, v)], 1)
        dq, dk, dv = buf[:, :hq], buf[:, hq:hq + hk], buf[:, hq + hk:]
    elif layout == "heads":        # head-major
        dq, dk, dv = (dev(x, t).transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
    else:                          # keys and values side by side
        kv = torch.cat([dev(k, t), dev(v, t)], 1)
        dq, dk, dv = dev(q, t), kv[:, :hk], kv[:, hk:]
    o = torch.full((nq, hq, d), 7.0, device="cuda", dtype=t)
    if layout == "heads":
        o = torch.full((hq, nq, d), 7.0, device="cuda", dtype=t).transpose(0, 1)
    tq, tk = (torch.tensor(c, dtype=torch.int32).cuda() for c in (cu_q, cu_k))
    desc = hb.packed_attention_desc(dq, dk, dv, o, tq, max(lq, default=0) if hints is True else hints or 0, max(lk, default=0) if hints is True else hints or 0, causal=causal,
                                    prescaled=prescaled, scale=scale or 0.0)
    need = hb.hyb_packed_attention_workspace_bytes(desc)
    ws = torch.full((need,), 255, device="cuda", dtype=torch.uint8)      # NaN wherever it is read before it is written
    hb.hyb_packed_attention(desc, dq, dk, dv, o, tq, tk, ws if need else None)
    got = host(o)
    factor = 0.6931471805599453 if prescaled else scale
    want = P.packed_attention(q, k, v, cu_q, cu_k, causal, factor, np.full((nq, hq, d), 7.0))
    again = torch.full_like(o, 7.0)
    hb.hyb_packed_attention(desc, dq, dk, dv, again, tq, tk, ws if need else None)
    torch.cuda.synchronize()
    return got, want, (q, k, v, cu_q, cu_k, causal, factor), torch.equal(o.contiguous().view(torch.int16 if dt == "bf16" else torch.int32), again.contiguous().view(torch.int16 if dt == "bf16" else torch.int32)), need


def _check(dt, got, want, inputs, same, need=None):
    assert same                                            # twice the same bits
    q, k, v, cu_q, cu_k, causal, factor = inputs
    inside = np.arange(cu_q[0], cu_q[-1])
    outside = np.setdiff1d(np.arange(len(got)), inside)
    assert (got[outside] == 7.0).all()                     # rows of no sequence: as they were
    bound = P.packed_attention_bound(q, k, v, cu_q, cu_k, dt == "bf16", causal, factor)
    assert np.isfinite(got).all()
    assert (np.abs(got - want)[inside] <= bound[inside]).all(), np.abs(got - want).max()
    assert rel_l2(got[inside], want[inside]) < TOL_REL[dt], rel_l2(got[inside], want[inside])


LENGTHS = [([1], [1]), ([5], [5]), ([1, 1, 1], [1, 2, 64]), ([64, 1, 128, 31], [64, 1, 128, 31]), ([129, 33, 65], [129, 33, 65]), ([0, 3, 0, 7, 0], [5, 0, 0, 7, 2]), ([200, 70], [63, 191]),
           ([40, 20, 130], [10, 20, 65]), ([17] * 9, [80] * 9)]
HEADS = [(1, 1, 64), (4, 2, 64), (6, 2, 128), (5, 5, 64), (8, 8, 128), (7, 1, 64)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_lengths(hb, dt, heads, causal):
    for lq, lk in LENGTHS:
        got = _attention(hb, dt, lq, lk, *heads, causal=causal, spare=3, layout="kv")
        if not np.any(got[1][3:-3]):
            assert not got[0][3:-3].any()                  # nobody sees a key
            continue
        _check(dt, *got)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_more_sequences_than_lanes(hb, dt, causal):
    lens = [(7 * i) % 61 for i in range(150)]
    _check(dt, *_attention(hb, dt, lens, [n + i % 3 for i, n in enumerate(lens)], 6, 3, 64, causal=causal, spare=2, layout="kv"))


@pytest.mark.parametrize("new", [0, 1])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_broadcast_keys(hb, dt, new):
    """Keys and values that are one row for all tokens, or one head for all heads (strides of 0): every query gets the mean of what it sees."""
    n = 300
    q = dev(synth.normal(1, (new or n, 4, 64), 1.0, dt), tdt(dt))
    k, v = (dev(synth.normal(s, (n, 1, 64), 1.0, dt), tdt(dt)) for s in (2, 3))
    cu_q, cu_k = _offsets([new or n]), _offsets([n])
    for name, kk, vv in (("tokens", k[:1].expand(n, 2, 64), v[:1].expand(n, 2, 64)), ("heads", k.expand(n, 2, 64), v.expand(n, 2, 64))):
        o = torch.full_like(q, 7.0)
        desc = hb.packed_attention_desc(q, kk, vv, o, cu_q, new or n, n)
        ws = torch.empty(hb.hyb_packed_attention_workspace_bytes(desc), device="cuda", dtype=torch.uint8)
        hb.hyb_packed_attention(desc, q, kk, vv, o, cu_q, cu_k, ws)
        args = host(q), host(kk.contiguous()), host(vv.contiguous()), cu_q.cpu().numpy(), cu_k.cpu().numpy()
        want = P.packed_attention(*args)
        assert (np.abs(host(o) - want) <= P.packed_attention_bound(*args, dt == "bf16")).all(), name


@pytest.mark.parametrize("layout", ["fused", "heads", "kv"])
@pytest.mark.parametrize("prescaled", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_layouts_and_scales(hb, dt, prescaled, layout):
    for d in (64, 128):
        _check(dt, *_attention(hb, dt, [130, 77], [130, 77], 4, 2, d, causal=True, prescaled=prescaled, layout=layout))
        _check(dt, *_attention(hb, dt, [90, 45], [90, 45], 3, 3, d, prescaled=prescaled, layout=layout, scale=None if prescaled else 0.3))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", [([1, 1, 1], [1000, 3000, 65], 8, 2, 128), ([1], [5000], 4, 4, 64), ([2, 5, 1], [700, 1300, 4000], 6, 2, 64), ([100], [3000], 2, 1, 128), ([1, 0, 1], [2000, 900, 0], 4, 1, 128),
                                  ([3, 60, 1], [1, 600, 900], 2, 2, 64)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_few_queries_over_long_keys(hb, dt, case, causal):
    """New tokens at the end of caches: keys are cut into parts."""
    *got, need = _attention(hb, dt, *case, causal=causal)
    assert need > 0
    _check(dt, *got)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_many_caches_of_much_the_same_length(hb, dt):
    """Single tokens whose caches alone fill the chip: not cut."""
    for hq, hk, d in ((16, 8, 64), (8, 8, 128)):
        *got, need = _attention(hb, dt, [1] * 60, [600 - 3 * i for i in range(60)], hq, hk, d, causal=True)
        assert need == 0
        _check(dt, *got)


@pytest.mark.parametrize("sequences", [40, 64, 65])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_many_ragged_caches(hb, d, sequences):
    """Several rounds of pieces: full ones, rests of all sizes, none at all and empty caches; two queries here and there, or none."""
    lk = [(3100, 0, 256, 512, 700, 1, 255, 257, 1024, 60)[i % 10] + i // 10 * (i % 3) for i in range(sequences)]
    lq = [(1, 1, 2, 1, 0, 1, 2)[i % 7] for i in range(sequences)]
    for causal in (False, True):
        *got, need = _attention(hb, "bf16", lq, lk, 16, 16 if d == 64 else 8, d, causal=causal)
        assert need > 0
        _check("bf16", *got)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_cut_keys_without_hints(hb, dt, d):
    """One long cache among short and empty ones: every block deals its own keys out, down to parts of 256."""
    lq, lk = [1, 3, 1, 0, 2, 1, 1, 1, 4], [3000, 40, 0, 9, 700, 257, 256, 255, 513]
    *got, need = _attention(hb, dt, lq, lk, 4, 2, d, causal=True, hints=False)
    assert need > 0
    _check(dt, *got)


@pytest.mark.parametrize("dt,hint", [("bf16", 1), ("bf16", 0), ("f32", 0)])
def test_attention_more_workgroups_than_one_grid_dimension_holds(hb, dt, hint):
    """300000 sequences of one query and one key, 32 heads: 9.6 million units.  The one probability is 1, so o is v but for the rounding of p v / p: none in bf16 (the products of two
    8-bit significands are exact, the quotient is off by 2^-23 at most, far inside half a step), three of 2^-24 in fp32."""
    n = 300000
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(n, 32, 64, generator=g, device="cuda").to(tdt(dt)) for _ in range(3))
    o = torch.full_like(q, 7.0)
    cu = torch.arange(n + 1, device="cuda", dtype=torch.int32)
    desc = hb.packed_attention_desc(q, k, v, o, cu, hint, hint)
    hb.hyb_packed_attention(desc, q, k, v, o, cu, cu, torch.empty(max(hb.hyb_packed_attention_workspace_bytes(desc), 16), device="cuda", dtype=torch.uint8))
    if dt == "bf16":
        assert torch.equal(o, v)
    else:
        assert bool(((o - v).abs() <= 3 * 2.0 ** -24 * v.abs()).all())


@pytest.mark.parametrize("hints", [False, 1, 600, 100000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_hints_do_not_decide_the_result(hb, dt, hints):
    for lq, lk in (([1, 1], [1900, 700]), ([150, 1], [200, 1500])):
        _check(dt, *_attention(hb, dt, lq, lk, 4, 2, 64, causal=True, hints=hints))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", [([300, 200], [300, 200]), ([2], [4000])])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_scores_far_from_zero(hb, dt, d, case, causal):
    """Scores of some hundreds in base 2: the running maximum, in some of the row blocks and parts only."""
    lq, lk = case

    def edit(q, k, v, cu_q, cu_k):
        q[:len(q) // 2 + 1] *= 40.0
        k[3::7] += np.float32(2.0)
        q[-1] = 0.0
        if dt == "bf16":
            for x in (q, k):
                x[...] = synth.round_bf16(x)
    got, want, inputs, same, _ = _attention(hb, dt, lq, lk, 4, 2, d, causal=causal, edit=edit)
    assert same and np.isfinite(got).all()
    bound = P.packed_attention_bound(*inputs[:5], dt == "bf16", inputs[5], inputs[6])
    assert (np.abs(got - want) <= bound).all()
    # (scores of 500 in fp32: off by 500 sqrt(d) 2^-24 or 4e-4, and a probability by as much, against the worst case of the bound)
    assert rel_l2(got, want) < (4e-3 if dt == "bf16" else 1e-3)


# (queries, keys, base-2 score that all pairs are near, exponent of the values): row blocks cut and not, single tokens
SIZES = [([100], [3000], 50, 67), ([100], [3000], -60, -70), ([100], [3000], -20, -80), ([100, 3], [500, 90], -60, -70), ([100, 3], [500, 90], 60, 50), ([100, 3], [500, 90], 20, 90),
         ([1, 1], [3000, 900], 50, 67), ([1, 1], [3000, 900], -60, -70), ([100], [3000], -60, -92), ([100, 3], [500, 90], -60, -92), ([1, 1], [3000, 900], -60, -92)]


@pytest.mark.parametrize("prescaled", [False, True])
@pytest.mark.parametrize("case", SIZES, ids=[str(c).replace(" ", "") for c in SIZES])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_values_of_any_size(hb, dt, d, case, prescaled):
    """Scores all far from zero on one side, and large or small values: what the softmax weighs is their mean, whatever the size of the numbers on the way.  (2^8 x keys x value stays below
    2^128 in all of them, and half a step of every result above 2^-117 x keys.)"""
    lq, lk, near, exponent = case

    def edit(q, k, v, cu_q, cu_k):
        # the first feature makes the common part of the score, a product of two numbers of at most 8 bits
        q[..., 0] = 8.0 if near > 0 else -8.0
        k[..., 0] = synth.round_bf16(np.float32(abs(near) / 8 * (1.0 if prescaled else d ** 0.5 / 1.4426950408889634)))
        v[...] = np.abs(v) * np.float32(2.0 ** exponent)
    got = _attention(hb, dt, lq, lk, 2, 1, d, prescaled=prescaled, edit=edit)
    assert got[4] > 0 if max(lk) == 3000 else dt == "f32" or got[4] == 0
    # (the common part in nats: sums of d products around it are off by up to 60 ln 2 x 2^-24 = 2.5e-6 a rounding, and a probability by as much; the bound has the worst case)
    q, k, v, cu_q, cu_k, causal, factor = got[2]
    bound = P.packed_attention_bound(q, k, v, cu_q, cu_k, dt == "bf16", causal, factor)
    assert got[3] and np.isfinite(got[0]).all() and (np.abs(got[0] - got[1]) <= bound).all(), np.abs(got[0] / got[1] - 1).max()


@pytest.mark.parametrize("prescaled", [False, True])
@pytest.mark.parametrize("factor", [12.0, 40.0])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_scores_far_from_zero_in_some_parts(hb, dt, d, factor, prescaled):
    """Cut keys of which some parts need the running maximum and the others do not: references hundreds apart meet in the merge, in rows that weigh both kinds of parts and rows that weigh one."""
    def edit(q, k, v, cu_q, cu_k):
        k[1000:1500] *= np.float32(factor)
        q[::2] *= np.float32(0.125)                        # these rows weigh all parts
        q[5] = 0.0
        if dt == "bf16":
            for x in (q, k):
                x[...] = synth.round_bf16(x)
    got, want, inputs, same, need = _attention(hb, dt, [100], [3000], 2, 1, d, prescaled=prescaled, edit=edit)
    assert need > 0 and same and np.isfinite(got).all()
    q, k, v, cu_q, cu_k, causal, scale = inputs
    assert (np.abs(got - want) <= P.packed_attention_bound(q, k, v, cu_q, cu_k, dt == "bf16", causal, scale)).all()
    # (as for scores far from zero everywhere)
    assert rel_l2(got, want) < (4e-3 if dt == "bf16" else 1e-3)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_hidden_keys_do_not_reach(hb, dt, d, bad):
    """Infinities and NaN in keys and values of other sequences, behind the last sequence and behind the causal limit; who sees them is not finite."""
    lq, lk = [70, 40, 100, 1], [70, 40, 100, 900]

    def edit(q, k, v, cu_q, cu_k):
        for x in (k, v):
            x[:3] = bad                                    # before the first sequence
            x[cu_k[-1]:] = bad
            x[cu_k[1] + 25, :, 5] = bad                    # in the second sequence, seen by its queries 25 ..
        v[cu_k[2] + 99, 0] = bad                           # the last key of the third, seen by its last query
    got, want, inputs, same, _ = _attention(hb, dt, lq, lk, 2, 1, d, causal=True, spare=3, edit=edit)
    cu_q = inputs[3]
    assert same
    dirty = np.zeros(len(got), dtype=bool)
    dirty[cu_q[1] + 25:cu_q[2]] = True
    dirty[cu_q[3] - 1] = True
    assert np.isfinite(got[~dirty]).all()
    assert not np.isfinite(got[cu_q[1] + 25:cu_q[2], :, 5]).any() and not np.isfinite(got[cu_q[3] - 1]).any()
    q, k, v, cu_q, cu_k, causal, factor = inputs
    k, v = (np.where(np.isfinite(x), x, 0.0) for x in (k, v))
    clean = P.packed_attention(q, k, v, cu_q, cu_k, causal, factor, np.full(got.shape, 7.0))
    bound = P.packed_attention_bound(q, k, v, cu_q, cu_k, dt == "bf16", causal, factor)
    assert (np.abs(got - clean)[~dirty] <= bound[~dirty]).all()


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_hidden_keys_do_not_reach_few_queries(hb, dt, d, bad):
    """The same for a few new tokens per sequence: the first of two does not see the last key."""
    lq, lk = [2, 1, 2, 2], [70, 40, 900, 33]

    def edit(q, k, v, cu_q, cu_k):
        for x in (k, v):
            x[:3] = bad
            x[cu_k[-1]:] = bad
        for s in (0, 2, 3):
            v[cu_k[s + 1] - 1, :, 7] = bad
        k[cu_k[1] - 1] = np.nan
    got, want, inputs, same, _ = _attention(hb, dt, lq, lk, 6, 2, d, causal=True, spare=3, edit=edit)
    q, k, v, cu_q, cu_k, causal, factor = inputs
    assert same
    dirty = np.zeros(len(got), dtype=bool)
    dirty[[cu_q[1] - 1, cu_q[3] - 1, cu_q[4] - 1]] = True
    assert not np.isfinite(got[dirty][:, :, 7]).any() and np.isfinite(got[cu_q[3] - 1][:, :7]).all()
    k, v = (np.where(np.isfinite(x), x, 0.0) for x in (k, v))
    clean = P.packed_attention(q, k, v, cu_q, cu_k, causal, factor, np.full(got.shape, 7.0))
    bound = P.packed_attention_bound(q, k, v, cu_q, cu_k, dt == "bf16", causal, factor)
    assert np.isfinite(got[~dirty]).all() and (np.abs(got - clean)[~dirty] <= bound[~dirty]).all()


@pytest.mark.parametrize("prescaled", [False, True])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_f32_launches_that_fill_the_chip(hb, causal, prescaled):
    """Blocks of 32 rows at head_dim 128."""
    lens = [130, 70, 0, 33, 1, 97]
    _check("f32", *_attention(hb, "f32", lens, lens if causal else [64, 131, 9, 33, 1, 200], 64, 32, 128, causal=causal, prescaled=prescaled, spare=2, layout="kv"))


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_attention_f32_launches_that_fill_the_chip_hidden_keys(hb, bad):
    lens = [130, 70, 0, 33, 1, 97]

    def edit(q, k, v, cu_q, cu_k):
        for x in (k, v):
            x[:2] = bad
            x[cu_k[-1]:] = bad
        v[cu_k[1] - 1, :, 7] = bad                         # the last key of the first sequence, seen by its last query
        v[cu_k[1] + 40, 3] = bad
    got, want, inputs, same, _ = _attention(hb, "f32", lens, lens, 64, 32, 128, causal=True, spare=2, edit=edit, layout="kv")
    q, k, v, cu_q, cu_k, causal, factor = inputs
    dirty = np.zeros(got.shape, dtype=bool)
    dirty[cu_q[1] - 1, :, 7] = True
    dirty[cu_q[1] + 40:cu_q[2], 6:8] = True
    assert same and not np.isfinite(got[dirty]).any() and np.isfinite(got[~dirty]).all()
    k, v = (np.where(np.isfinite(x), x, 0.0) for x in (k, v))
    clean = P.packed_attention(q, k, v, cu_q, cu_k, causal, factor, np.full(got.shape, 7.0))
    assert (np.abs(got - clean)[~dirty] <= P.packed_attention_bound(q, k, v, cu_q, cu_k, False, causal, factor)[~dirty]).all()


@pytest.mark.parametrize("new", [0, 2])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_a_query_that_is_not_finite_is_alone(hb, dt, d, new):
    lq, lk = ([new, 1], [700, 300]) if new else ([150, 40], [150, 40])

    def edit(q, k, v, cu_q, cu_k):
        q[1, 1, 5] = np.nan
    got, want, inputs, same, _ = _attention(hb, dt, lq, lk, 4, 2, d, causal=True, edit=edit)
    assert same and np.isnan(got[1, 1]).all()
    q, k, v, cu_q, cu_k, causal, factor = inputs
    q = np.nan_to_num(q)
    clean = P.packed_attention(q, k, v, cu_q, cu_k, causal, factor)
    ok = np.abs(got - clean) <= P.packed_attention_bound(q, k, v, cu_q, cu_k, dt == "bf16", causal, factor)
    ok[1, 1] = True
    assert ok.all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_values_seen_keep_their_infinity(hb, dt):
    """A value of +inf that a query sees makes that feature +inf, in a tile that not all rows see, and leaves the other features alone."""
    def edit(q, k, v, cu_q, cu_k):
        v[30, 0, 9] = np.inf
    got, _, inputs, _, _ = _attention(hb, dt, [64], [64], 1, 1, 64, causal=True, edit=edit)
    assert (got[30:, 0, 9] == np.inf).all()
    got[30:, 0, 9] = 0.0
    assert np.isfinite(got).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_offsets_outside_the_tensors(hb, dt):
    """Offsets are taken as the nearest row there is: nothing outside is read or written."""
    q, k, v = (synth.normal(s, (50, 2, 64), 1.0, dt) for s in (1, 2, 3))
    dq, dk, dv = (dev(x, tdt(dt)) for x in (q, k, v))
    for cu_q, cu_k in (([-5, 20, 90], [-1, 30, 1000]), ([0, 50, 50], [0, 70, 20]), ([10, 30, 20], [0, 10, 50])):
        o = torch.full((50, 2, 64), 7.0, device="cuda", dtype=tdt(dt))
        tq, tk = (torch.tensor(c, dtype=torch.int32).cuda() for c in (cu_q, cu_k))
        desc = hb.packed_attention_desc(dq, dk, dv, o, tq)
        hb.hyb_packed_attention(desc, dq, dk, dv, o, tq, tk)
        got, want = host(o), P.packed_attention(q, k, v, cu_q, cu_k, o=np.full((50, 2, 64), 7.0))
        if cu_q == sorted(cu_q):
            assert rel_l2(got, want) < TOL_REL[dt]


def _guarded(x, fill, rows=64):
    """(a tensor with x's data, whose neighbours in memory are rows of `fill`; a function that says whether they still are)"""
    whole = torch.full((rows + x.shape[0] + rows, *x.shape[1:]), fill, device="cuda", dtype=x.dtype)
    whole[rows:rows + x.shape[0]] = x
    before = whole.clone()
    bits = {torch.bfloat16: torch.int16, torch.float32: torch.int32, torch.uint8: torch.uint8}[x.dtype]

    def intact():
        return all(torch.equal(whole[part].view(bits), before[part].view(bits)) for part in (slice(0, rows), slice(rows + x.shape[0], None)))
    return whole[rows:rows + x.shape[0]], intact


# (rows of queries, rows of keys, max_q, max_k): uncut row blocks, cut ones, pieces of single tokens, and single tokens whose hints say one piece
GUARDED = [(50, 50, 0, 0), (100, 3000, 100, 3000), (4, 3000, 1, 3000), (4, 3000, 1, 500)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", GUARDED)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_offsets_outside_the_tensors_between_guards(hb, dt, d, case, causal):
    """Offsets beyond the tensors, and offsets that decrease: NaN beside the inputs is not read, rows beside the result and bytes beside the workspace are not written."""
    nq, nk, max_q, max_k = case
    q, k, v = (synth.normal(s, (n, 2, d), 1.0, dt) for s, n in ((1, nq), (2, nk), (3, nk)))
    (dq, q_ok), (dk, k_ok), (dv, v_ok) = (_guarded(dev(x, tdt(dt)), float("nan")) for x in (q, k, v))
    for cu_q, cu_k in (([-3, 1, 2, 3, nq + 40], [-7, nk // 3, nk // 2, nk - 1, nk + 99999]), ([-2 ** 31, -1, nq // 2, 2 ** 31 - 1, 2 ** 31 - 1], [-2 ** 31, 0, nk // 2, 2 ** 31 - 1, 2 ** 31 - 1]),
                       ([0, 1, 2, 3, 4], [nk - 9, nk // 30, nk, 5, nk // 2]), ([3, 1, 4, 0, 2], [0, nk // 4, nk // 2, nk // 2, nk]), ([nq, 3, 1, 1, -4], [nk + 5, nk // 2, 10, 8, -8])):
        ordered = cu_q == sorted(cu_q) and cu_k == sorted(cu_k)
        o, o_ok = _guarded(torch.full((nq, 2, d), 7.0, device="cuda", dtype=tdt(dt)), 9.0)
        tq, tk = (torch.tensor(c, dtype=torch.int32).cuda() for c in (cu_q, cu_k))
        desc = hb.packed_attention_desc(dq, dk, dv, o, tq, max_q, max_k, causal=causal)
        # (numbers that decrease may leave parts of the workspace unwritten that are read)
        ws, ws_ok = _guarded(torch.full((hb.hyb_packed_attention_workspace_bytes(desc),), 255 if ordered else 0, device="cuda", dtype=torch.uint8), 170, 4096)
        hb.hyb_packed_attention(desc, dq, dk, dv, o, tq, tk, ws)
        got = host(o)
        assert q_ok() and k_ok() and v_ok() and o_ok() and ws_ok(), (cu_q, cu_k)
        assert np.isfinite(got).all(), (cu_q, cu_k)
        if ordered:
            clip = [np.clip(c, 0, n) for c, n in ((cu_q, nq), (cu_k, nk))]
            want = P.packed_attention(q, k, v, *clip, causal, None, np.full((nq, 2, d), 7.0))
            assert (np.abs(got - want) <= P.packed_attention_bound(q, k, v, *clip, dt == "bf16", causal)).all(), (cu_q, cu_k)


@pytest.mark.parametrize("sequences", [5, 40])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_caches_with_room_to_grow(hb, dt, d, sequences):
    """Single tokens over caches with spare rows: a sequence without queries owns the rows between two caches, whatever they hold."""
    room, lens = 700, [1 + 173 * i % 700 for i in range(sequences)]

    def edit(q, k, v, cu_q, cu_k):
        for i, n in enumerate(lens):
            k[i * room + n:(i + 1) * room] = np.nan
            v[i * room + n:(i + 1) * room] = np.nan
    lq, lk = [n for _ in lens for n in (1, 0)], [m for n in lens for m in (n, room - n)]
    got, want, inputs, same, _ = _attention(hb, dt, lq, lk, 4, 2, d, causal=True, edit=edit)
    q, k, v, cu_q, cu_k, causal, factor = inputs
    bound = P.packed_attention_bound(q, np.nan_to_num(k), np.nan_to_num(v), cu_q, cu_k, dt == "bf16", causal, factor)
    assert same and np.isfinite(got).all() and (np.abs(got - want) <= bound).all()
    assert rel_l2(got, want) < TOL_REL[dt]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_many_sequences(hb, dt):
    """More sequences than one step of the search looks at, empty ones among them."""
    rng = np.random.default_rng(3)
    lq = rng.integers(0, 4, 5000).tolist()
    lk = [n + int(x) for n, x in zip(lq, rng.integers(0, 9, 5000))]
    _check(dt, *_attention(hb, dt, lq, lk, 2, 1, 64, causal=True))


@pytest.mark.parametrize("prescaled", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hq,hk,d", [(264, 264, 64), (260, 130, 128), (261, 261, 64), (272, 68, 128)])
def test_attention_launches_of_many_rounds(hb, hq, hk, d, causal, prescaled):
    """Thousands of row blocks, in several rounds of workgroups: the same bits as launches of a few heads; with scores far from zero in some heads, and with
    infinities and NaN in keys that causal queries do not see."""
    lq, lk = ([450, 77, 1, 0, 300, 5], [450, 77, 9, 4, 333, 0]) if d == 64 or not causal else ([600, 130, 1, 0, 700, 5], [600, 130, 9, 4, 733, 0])
    g = torch.Generator(device="cuda").manual_seed(11)
    q = torch.randn(sum(lq) + 4, hq, d, generator=g, device="cuda") * (d ** -0.5 * 1.4427 if prescaled else 1.0)
    q[:, 3::16] *= 60.0
    q = q.bfloat16()
    k, v = (torch.randn(sum(lk) + 4, hk, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    k[-4:] = float("nan")
    v[-4:] = float("nan")
    v[lk[0] - 2, :, 7] = float("inf")
    cu_q, cu_k = _offsets(lq), _offsets(lk)
    group = hq // hk

    def run(h0, h1):
        x = q[:, h0 * group:h1 * group], k[:, h0:h1], v[:, h0:h1], torch.full((len(q), (h1 - h0) * group, d), 7.0, device="cuda", dtype=torch.bfloat16)
        desc = hb.packed_attention_desc(*x, cu_q, max(lq), 512, causal=causal, prescaled=prescaled)      # (512: keys are not cut)
        ws = torch.full((hb.hyb_packed_attention_workspace_bytes(desc),), 255, device="cuda", dtype=torch.uint8)
        for _ in range(3):
            hb.hyb_packed_attention(desc, *x, cu_q, cu_k, ws)
        return x[3]
    whole = run(0, hk)
    for h0 in range(0, hk, 10):
        part = run(h0, min(h0 + 10, hk))
        assert torch.equal(part.view(torch.int16), whole[:, h0 * group:min(h0 + 10, hk) * group].contiguous().view(torch.int16)), h0
    assert (whole[sum(lq):] == 7.0).all()
    last = [t for t in range(lq[0]) if not causal or t + lk[0] - lq[0] >= lk[0] - 2]
    assert not torch.isfinite(whole[last[0]:lq[0], :, 7]).any() and torch.isfinite(whole[:last[0]]).all() and torch.isfinite(whole[lq[0]:]).all()
    heads = [0, 3, group, hq - 1]
    sub = lambda x, h: x[:, h].float().cpu().numpy().astype(np.float64)      # noqa: E731
    rows = slice(lq[0], sum(lq))
    for h in heads:
        kk, vv = np.nan_to_num(sub(k, h // group)), np.nan_to_num(sub(v, h // group), posinf=0.0)
        want = P.packed_attention(sub(q, h)[:, None], kk[:, None], vv[:, None], cu_q.tolist(), cu_k.tolist(), causal, 0.6931471805599453 if prescaled else d ** -0.5, np.full((len(q), 1, d), 7.0))
        assert rel_l2(sub(whole, h)[rows], want[rows, 0]) < TOL_REL["bf16"], h


def test_attention_a_request_does_not_depend_on_its_neighbours(hb):
    """The same sequence alone, in front and behind others, with the same sizes of the launch: the same bits."""
    q, k, v = (dev(synth.normal(s, (600, 4, 64), 1.0, "bf16"), torch.bfloat16) for s in (1, 2, 3))
    outs = []
    for order in ((0, 200, 350, 600), (0, 250, 400, 600)):
        lengths = np.diff(order)
        rows = torch.arange(600, device="cuda") if order[1] == 200 else torch.cat([torch.arange(350, 600), torch.arange(200, 350), torch.arange(0, 200)]).cuda()
        x = [t[rows].contiguous() for t in (q, k, v)]
        o, cu = torch.empty_like(x[0]), _offsets(lengths)
        hb.hyb_packed_attention(hb.packed_attention_desc(*x, o, cu, 250, 250), *x, o, cu, cu)
        outs.append(o if order[1] == 200 else torch.empty_like(o).index_copy_(0, rows, o))
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])


def test_attention_full_sequence_agrees_with_joint_attention(hb):
    q, k, v = (dev(synth.normal(s, (1, 8, 333, 64), 1.0, "bf16"), torch.bfloat16) for s in (1, 2, 3))
    o = torch.empty(1, 333, 512, device="cuda", dtype=torch.bfloat16)
    hb.hyb_joint_attention(q, k, v, o)
    t = [x[0].transpose(0, 1) for x in (q, k, v)]           # head-major tensors as they are
    op, cu = torch.empty(333, 8, 64, device="cuda", dtype=torch.bfloat16), _offsets([333])
    hb.hyb_packed_attention(hb.packed_attention_desc(*t, op, cu), *t, op, cu, cu)
    assert rel_l2(host(op).reshape(333, 512), host(o)[0]) < 4e-3


@pytest.mark.parametrize("shape", [(1, 4429, 24, 24, 64, False), (1, 2050, 8, 2, 128, True), (2, 1500, 4, 4, 128, False)])
def test_attention_long_sequences_sampled(hb, shape):
    n, length, hq, hk, d, causal = shape
    g = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.randn(n * length, hq + 2 * hk, d, generator=g, device="cuda").bfloat16()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    o, cu = torch.empty(n * length, hq, d, device="cuda", dtype=torch.bfloat16), _offsets([length] * n)
    desc = hb.packed_attention_desc(q, k, v, o, cu, length, length, causal=causal)
    ws = torch.empty(hb.hyb_packed_attention_workspace_bytes(desc), device="cuda", dtype=torch.uint8)
    hb.hyb_packed_attention(desc, q, k, v, o, cu, cu, ws)
    got = host(o)
    hq_, hk_, hv_ = (host(x) for x in (q, k, v))
    for s in range(n):
        for t in (0, 1, 63, 64, 127, 128, length // 2, length - 2, length - 1):
            at, end = s * length + t, s * length + (t + 1 if causal else length)
            want = P.packed_attention(hq_[at:at + 1], hk_[s * length:end], hv_[s * length:end], [0, 1], [0, end - s * length])
            assert rel_l2(got[at:at + 1], want) < 4e-3, (s, t)


def test_attention_keys_beyond_32_bit_offsets(hb):
    """Keys and values whose last row lies 6 GB behind the first (a row every 256 KB)."""
    rows, d, stride = 24000, 64, 1 << 17
    base = torch.zeros(rows * stride, device="cuda", dtype=torch.bfloat16)
    k, v = (base.as_strided((rows, 1, d), (stride, d, 1), n * d) for n in (0, 1))
    g = torch.Generator(device="cuda").manual_seed(6)
    for t in (k, v):
        t.copy_(torch.randn(rows, 1, d, generator=g, device="cuda").bfloat16())
    q = torch.randn(2, 1, d, generator=g, device="cuda").bfloat16()
    o, tq, tk = torch.empty_like(q), _offsets([1, 1]), torch.tensor([0, 100, rows], dtype=torch.int32).cuda()
    desc = hb.packed_attention_desc(q, k, v, o, tq, 1, rows)
    ws = torch.empty(hb.hyb_packed_attention_workspace_bytes(desc), device="cuda", dtype=torch.uint8)
    hb.hyb_packed_attention(desc, q, k, v, o, tq, tk, ws)
    assert rel_l2(host(o), P.packed_attention(host(q), host(k), host(v), [0, 1, 2], [0, 100, rows])) < 4e-3


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attention_one_row_of_head_major_caches(hb, dt):
    """One token whose heads lie 2 MB apart, queries, keys, values and result: with one key the result is its value."""
    q, k, v, o = (dev(synth.normal(s, (8, 8192, 128), 1.0, dt), tdt(dt))[:, s:s + 1].transpose(0, 1) for s in (1, 2, 3, 4))
    cu = _offsets([1])
    hb.hyb_packed_attention(hb.packed_attention_desc(q, k, v, o, cu, 1, 1), q, k, v, o, cu, cu)
    # (p v / p: none of it rounds in bf16, three times in fp32)
    assert (np.abs(host(o) - host(v)) <= (0.0 if dt == "bf16" else 3 * 2.0 ** -24) * np.abs(host(v))).all()


def test_attention_binding_refusals(hb):
    q, k = (torch.zeros(8, h, 64, device="cuda", dtype=torch.bfloat16) for h in (2, 1))
    o, cu = torch.empty_like(q), _offsets([8])
    desc = hb.packed_attention_desc(q, k, k, o, cu)
    for bad in ((q[:7], k, k, o, cu, cu), (q, k.float(), k, o, cu, cu), (q, k, k, o, cu[:1], cu), (q, k, k, o, cu, cu.long()), (q, k, k, o, cu.cpu(), cu), (q, k.cpu(), k, o, cu, cu), (q, None, k, o, cu, cu),
                (q.transpose(0, 1).contiguous().transpose(0, 1), k, k, o, cu, cu)):
        with pytest.raises((ValueError, TypeError)):
            hb.hyb_packed_attention(desc, *bad)
    with pytest.raises(hb.HybError):
        hb.hyb_packed_attention(hb.packed_attention_desc(q[..., :32], k[..., :32], k[..., :32], o[..., :32], cu), q[..., :32], k[..., :32], k[..., :32], o[..., :32], cu, cu)


# ---- together -----------------------------------------------------------------------------------------------------------------------------

def _packed_block(hb, dt, shapes, text_after, heads, stream=None):
    """Layout -> q, k, v projection -> rotary positions in place -> attention -> output projection, as a denoiser on a packed batch would."""
    hq, hk, d, hidden, dims = heads
    rows = int(P.packed_layout(shapes, 10 ** 9)[0][-1])
    x, w, b = synth.normal(1, (rows, hidden), 1.0, dt), synth.normal(2, ((hq + 2 * hk) * d, hidden), 0.05, dt), synth.normal(3, ((hq + 2 * hk) * d,), 0.1, "f32")
    wo, bo = synth.normal(4, (hidden, hq * d), 0.05, dt), synth.normal(5, (hidden,), 0.1, "f32")
    t = tdt(dt)
    sh = torch.tensor(shapes, dtype=torch.int32).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    dx, dw, db, dwo, dbo = dev(x, t), dev(w, t), dev(b), dev(wo, t), dev(bo)
    offsets, request, positions = torch.empty(len(shapes) + 1, **i32), torch.empty(rows, **i32), torch.empty(rows, 3, **i32)
    qkv, out = torch.empty(rows, (hq + 2 * hk) * d, device="cuda", dtype=t), torch.empty(rows, hidden, device="cuda", dtype=t)
    heads_of = qkv.view(rows, hq + 2 * hk, d)
    q, k, v = heads_of[:, :hq], heads_of[:, hq:hq + hk], heads_of[:, hq + hk:]
    o = torch.empty(rows, hq, d, device="cuda", dtype=t)
    rot = hb.rotary_desc(q, k, dims, q_scale=d ** -0.5 * 1.4426950408889634)
    att = hb.packed_attention_desc(q, k, v, o, offsets, prescaled=True)
    ws = torch.empty(hb.hyb_packed_attention_workspace_bytes(att), device="cuda", dtype=torch.uint8)

    def step():
        hb.hyb_packed_layout(sh, offsets, request, positions, text_after)
        hb.hyb_linear(dx, dw, db, qkv)
        hb.hyb_rotary(rot, positions, q, k)
        hb.hyb_packed_attention(att, q, k, v, o, offsets, offsets, ws)
        hb.hyb_linear(o.view(rows, hq * d), dwo, dbo, out)
        return out

    def oracle(shapes):
        cu, _, pos = P.packed_layout(shapes, rows, text_after)
        y = O.linear(x, w, b).reshape(rows, hq + 2 * hk, d)
        yq, yk = (P.rotary(z, pos, dims) for z in (y[:, :hq], y[:, hq:hq + hk]))
        return O.linear(P.packed_attention(yq, yk, y[:, hq + hk:], cu, cu).reshape(rows, hq * d), wo, bo)
    return step, oracle, out, sh


MIXED = [(1, 8, 8, 13), (1, 5, 9, 0), (3, 4, 4, 7), (0, 0, 0, 21)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 4, 64, 256, (16, 24, 24)), (4, 2, 128, 192, (32, 48, 48))])
def test_packed_block(hb, dt, heads):
    step, oracle, out, _ = _packed_block(hb, dt, MIXED, True, heads)
    step()
    assert err(host(out), oracle(MIXED)) < tol(dt)


def test_packed_block_replays_from_a_graph(hb):
    """Captured on a stream of its own, replayed several times with eager work between, and with other requests of as many rows."""
    step, oracle, out, sh = _packed_block(hb, "bf16", MIXED, False, (4, 2, 64, 256, (16, 24, 24)))
    eager = step().clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    torch.cuda.synchronize()
    other = [MIXED[i] for i in (2, 0, 3, 1)]
    for shapes in (MIXED, other, MIXED):
        sh.copy_(torch.tensor(shapes, dtype=torch.int32))
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        assert torch.equal(replayed, step())
        assert (shapes is other) or torch.equal(replayed, eager)
    assert err(host(replayed), oracle(MIXED)) < tol("bf16")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt,new", [("bf16", 1), ("bf16", 20), ("f32", 1), ("f32", 20)])
def test_cut_keys_replay_from_a_graph(hb, dt, new, d):
    """Both launches of a call whose keys are cut, captured once: replays follow the offsets, whatever the workspace holds, and give the bits of an eager call."""
    n, rows = 5, 6000
    g = torch.Generator(device="cuda").manual_seed(5)
    q = torch.randn(n * new, 4, d, generator=g, device="cuda").to(tdt(dt))
    k, v = (torch.randn(rows, 2, d, generator=g, device="cuda").to(tdt(dt)) for _ in range(2))
    o, cu_q = torch.empty_like(q), _offsets([new] * n)
    cu_k = torch.empty(n + 1, dtype=torch.int32, device="cuda")
    desc = hb.packed_attention_desc(q, k, v, o, cu_q, new, 4000, causal=True)
    need = hb.hyb_packed_attention_workspace_bytes(desc)
    assert need > 0
    ws, own = (torch.empty(need, device="cuda", dtype=torch.uint8) for _ in range(2))
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    cu_k.copy_(_offsets([1200] * n))
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        hb.hyb_packed_attention(desc, q, k, v, o, cu_q, cu_k, ws)
    for lens in ([1200] * 5, [4000, 0, 500, 1, 1499], [30, 40, 3000, 2000, 25], [1200] * 5):
        cu_k.copy_(_offsets(lens))
        ws.fill_(255)
        o.fill_(7.0)
        graph.replay()
        eager = torch.full_like(o, 7.0)
        own.fill_(255)
        hb.hyb_packed_attention(desc, q, k, v, eager, cu_q, cu_k, own)
        torch.cuda.synchronize()
        assert torch.equal(o, eager), lens
        args = host(q), host(k), host(v), cu_q.cpu().numpy(), cu_k.cpu().numpy()
        assert (np.abs(host(o) - P.packed_attention(*args, True)) <= P.packed_attention_bound(*args, dt == "bf16", True)).all(), lens


def test_two_streams_with_a_workspace_each(hb):
    """Calls that overlap in time, on streams of their own."""
    lk = [3000, 1700]
    q, k, v = (dev(synth.normal(s, (n, 4, 64), 1.0, "bf16"), torch.bfloat16) for s, n in ((1, 2), (2, 4700), (3, 4700)))
    cu_q, cu_k = _offsets([1, 1]), _offsets(lk)
    outs = [torch.zeros_like(q) for _ in range(3)]
    desc = hb.packed_attention_desc(q, k, v, outs[0], cu_q, 1, 3000)
    spaces = [torch.empty(hb.hyb_packed_attention_workspace_bytes(desc), device="cuda", dtype=torch.uint8) for _ in range(3)]
    hb.hyb_packed_attention(desc, q, k, v, outs[0], cu_q, cu_k, spaces[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for s, o, ws in zip(streams, outs[1:], spaces[1:]):
            with torch.cuda.stream(s):
                hb.hyb_packed_attention(desc, q, k, v, o, cu_q, cu_k, ws)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
