"""Gated delta rule on the GPU against the fp64 checker: prompts (both kernels), single tokens, and a serving loop of the delta-rule
operators together.

Tolerances are the repository's (tests/util.py, max|x - ref| / max|ref|).  States, whatever the dtype: 1e-4.  With TENSOR each of the three factors
that reach a state (S, the right-hand side, U) is held in two bf16 terms, off by at most 2^-8 * 2^-8 = 2^-16 each, and the product of their
lower terms that is left out is 2^-16 too: 4 * 2^-16 = 6e-5 of the summands' size.  Outputs in bf16: four roundings of 2^-8 each (the state
copy, the right-hand side, the score matrix, the output) of summands that may cancel in part: 2e-2.  Outputs in fp32: 1e-4."""
import numpy as np
import pytest
import torch

from util import Guarded, rel_err

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
TOL_O = {BF: 2e-2, F32: 1e-4}
TOL_S = 1e-4


def _dsla():
    import paper_2506_09316_b200 as dsla
    return dsla


def _draw(T, H, group, d, dtype, seed, gate="mixed", beta="mixed"):
    r = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=r)  # noqa: E731
    q, k = (n(T, H // group, d) for _ in range(2))
    q, k = ((x / x.norm(dim=-1, keepdim=True).clamp_min(1e-6)).to(dtype) for x in (q, k))
    v = n(T, H, d).to(dtype)
    g, b = torch.sigmoid(n(T, H) * 1.5 + 3), torch.sigmoid(n(T, H) + 0.5)
    u = torch.rand(T, H, generator=r)
    if gate == "mixed":
        g = torch.where(u < 0.02, 0.0, torch.where(u > 0.98, 1.0, g))
    elif gate == "tiny":
        g = torch.where(u < 0.3, 1e-30, g)
    else:
        g = torch.full_like(g, gate)
    b = b if beta == "mixed" else torch.full_like(b, beta)
    return [x.cuda() for x in (q, k, v, g, b)]


def _check(lens, H, group, d, dtype, impl, *, seed=0, resume=False, slots=None, dense=False, scale=0.3, gate="mixed", beta="mixed", edit=None, extra_slots=0):
    from oracle import dsla_oracle as orc
    dsla = _dsla()
    T, N = sum(lens), len(lens)
    q, k, v, g, b = _draw(T, H, group, d, dtype, seed, gate, beta)
    if edit:
        edit(q, k, v, g, b)
    nslots = max(N, 1 + max(slots) if slots else 0) + extra_slots
    gs, go = Guarded(nslots * H * d * d, F32), Guarded(v.numel(), dtype)
    st = dsla.dsla_state_alloc_n(nslots, 1, H, d, d, buffer=gs.mid)
    init = torch.randn(nslots, 1, H, d, d, generator=torch.Generator().manual_seed(seed + 1)) * 0.1
    st.tensor.copy_(init)
    want = init.double().numpy().copy()
    if not resume:
        for n in range(N):
            want[slots[n] if slots else n] = 0.0
    o = go.mid.view(v.shape)
    o.fill_(float("nan"))
    cu = None if dense else torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
    sl = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
    dsla.dsla_delta_prefill(q, k, v, g, b, st, o=o, cu_seqlens=cu, slots=sl, max_seqlen=max(lens) if lens else 0, scale=scale, use_initial_state=resume, impl=impl)
    torch.cuda.synchronize()
    assert dsla.dsla_state_last_error(st) == dsla.DSLA_OK
    gs.check("the state store")
    go.check("the output tensor")
    f = [x.double().cpu().numpy() for x in (q, k, v, g, b)]
    cu_np = np.array([0] + list(np.cumsum(lens)))
    wo, ws = orc.delta_prefill(*f, cu_np, scale=scale, state=want, slots=slots)
    eo, es = rel_err(o.double().cpu().numpy(), wo), rel_err(st.tensor.double().cpu().numpy(), ws)
    assert eo <= TOL_O[dtype] and es <= TOL_S, (eo, es)


KERNELS = [("simt", F32, 64), ("simt", F32, 128), ("simt", BF, 64), ("simt", BF, 128)]
CHUNKED = [("tensor", BF, 64), ("tensor", BF, 128)]
KERNELS += CHUNKED
both = pytest.mark.parametrize("impl,dtype,d", KERNELS)


@both
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 513])
def test_one_prompt(impl, dtype, d, T):
    _check([T], 2, 1, d, dtype, impl, seed=T, dense=True)


@both
@pytest.mark.parametrize("resume", [False, True])
def test_packed_prompts(impl, dtype, d, resume):
    _check([5, 0, 64, 130, 1, 77, 0, 63, 256], 3, 1, d, dtype, impl, seed=7, resume=resume, slots=[8, 3, 0, 1, 9, 2, 5, 4, 6], extra_slots=2)


@both
@pytest.mark.parametrize("H,group", [(4, 2), (6, 3), (8, 8)])
def test_grouped_heads(impl, dtype, d, H, group):
    _check([70, 33], H, group, d, dtype, impl, seed=H, resume=True)


@both
@pytest.mark.parametrize("gate,beta", [(1.0, "mixed"), (0.0, "mixed"), ("tiny", "mixed"), (-0.5, "mixed"), ("mixed", 0.0), ("mixed", 1.0), (1.0, 2.0)])
def test_gates_and_betas(impl, dtype, d, gate, beta):
    def clamp(q, k, v, g, b):
        g.clamp_(min=-0.5)
    if gate == -0.5:      # counts as 0
        from oracle import dsla_oracle as orc
        real = orc.delta_prefill
        try:
            orc.delta_prefill = lambda q, k, v, g, b, *a, **kw: real(q, k, v, np.maximum(g, 0), b, *a, **kw)
            _check([150], 2, 1, d, dtype, impl, gate=gate, beta=beta, resume=True, edit=clamp)
        finally:
            orc.delta_prefill = real
    else:
        _check([150], 2, 1, d, dtype, impl, gate=gate, beta=beta, resume=True)


@both
def test_repeated_and_zero_keys(impl, dtype, d):
    """One key over and over (the triangular system is as full as it gets), and tokens without one."""
    def same(q, k, v, g, b):
        k[1:] = k[:1]
        k[40:50] = 0
    _check([140], 2, 1, d, dtype, impl, edit=same, gate=1.0, beta=1.0)


@both
def test_dense_batch(impl, dtype, d):
    _check([100] * 3, 2, 1, d, dtype, impl, dense=True, resume=True)


@both
def test_empty_calls(impl, dtype, d):
    dsla = _dsla()
    st = dsla.dsla_state_alloc_n(2, 1, 2, d, d)
    st.tensor.fill_(3.0)
    q = torch.empty(0, 2, d, dtype=dtype, device="cuda")
    g = torch.empty(0, 2, device="cuda")
    cu = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert dsla.dsla_delta_prefill(q, q, q, g, g, st, cu_seqlens=cu, max_seqlen=0, use_initial_state=True, impl=impl).shape == q.shape
    assert bool((st.tensor == 3).all())
    dsla.dsla_delta_prefill(q, q, q, g, g, st, cu_seqlens=cu, max_seqlen=0, impl=impl)
    assert bool((st.tensor == 0).all())
    dsla.dsla_delta_prefill(q, q, q, g, g, st, impl=impl)      # no sequence at all
    dsla.dsla_delta_decode_step(q, q, q, g, g, st)


@both
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_bad_values_stay_in_their_sequence(impl, dtype, d, bad):
    dsla = _dsla()
    lens = [70, 50, 90]
    q, k, v, g, b = _draw(sum(lens), 2, 1, d, dtype, 3)
    cu = torch.tensor([0, 70, 120, 210], dtype=torch.int32, device="cuda")
    run = lambda st: dsla.dsla_delta_prefill(q, k, v, g, b, st, cu_seqlens=cu, max_seqlen=90, impl=impl)  # noqa: E731
    st, st2 = (dsla.dsla_state_alloc_n(3, 1, 2, d, d) for _ in range(2))
    want = run(st)
    for x in (q, k, v, g, b):
        x[70:120] = bad
    got = run(st2)
    for a, e in ((0, 70), (120, 210)):
        assert torch.equal(want[a:e], got[a:e])
    assert torch.equal(st.tensor[0], st2.tensor[0]) and torch.equal(st.tensor[2], st2.tensor[2])
    assert not bool(torch.isfinite(st2.tensor[1]).any())


@pytest.mark.parametrize("impl,dtype,d", CHUNKED)
def test_bad_values_reach_nothing_before_their_chunk(impl, dtype, d):
    dsla = _dsla()
    q, k, v, g, b = _draw(200, 2, 1, d, dtype, 4)
    st = dsla.dsla_state_alloc_n(1, 1, 2, d, d)
    want = dsla.dsla_delta_prefill(q, k, v, g, b, st, impl=impl)
    v[130] = float("inf")
    got = dsla.dsla_delta_prefill(q, k, v, g, b, st, impl=impl)
    assert torch.equal(want[:128], got[:128]) and not bool(torch.isfinite(got[192:]).all())


@both
def test_prompt_then_tokens(impl, dtype, d):
    """A prompt in two pieces and then token by token is the whole prompt."""
    dsla = _dsla()
    q, k, v, g, b = _draw(150, 4, 2, d, dtype, 5)
    st, whole = (dsla.dsla_state_alloc_n(1, 1, 4, d, d) for _ in range(2))
    want = dsla.dsla_delta_prefill(q, k, v, g, b, whole, impl=impl)
    part = lambda a, e: [x[a:e].contiguous() for x in (q, k, v, g, b)]  # noqa: E731
    got = [dsla.dsla_delta_prefill(*part(0, 70), st, impl=impl), dsla.dsla_delta_prefill(*part(70, 140), st, impl=impl, use_initial_state=True)]
    got += [dsla.dsla_delta_decode_step(*part(t, t + 1), st) for t in range(140, 150)]
    assert rel_err(torch.cat(got).double().cpu(), want.double().cpu()) <= TOL_O[dtype]
    assert rel_err(st.tensor.double().cpu(), whole.tensor.double().cpu()) <= TOL_S


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,group", [(1, 1, 1), (1, 32, 1), (7, 6, 3), (33, 4, 4)])
def test_decode(dtype, d, B, H, group):
    from oracle import dsla_oracle as orc
    dsla = _dsla()
    q, k, v, g, b = _draw(B, H, group, d, dtype, B)
    slots = torch.randperm(B + 2, generator=torch.Generator().manual_seed(B))[:B].to(torch.int32)
    mask = torch.ones(B, dtype=torch.uint8)
    if B > 3:
        slots[2], mask[1] = -1, 0
    gs, go = Guarded((B + 2) * H * d * d, F32), Guarded(v.numel(), dtype)
    st = dsla.dsla_state_alloc_n(B + 2, 1, H, d, d, buffer=gs.mid)
    st.tensor.normal_()
    state = st.tensor.double().cpu().numpy()
    o = go.mid.view(v.shape)
    o.fill_(7.0)
    dsla.dsla_delta_decode_step(q, k, v, g, b, st, o=o, slots=slots.cuda(), scale=0.5, row_mask=mask.cuda())
    live = torch.where(mask > 0, slots, -1).numpy()
    want, ws = orc.delta_prefill(*[x.double().cpu().numpy() for x in (q, k, v, g, b)], np.arange(B + 1), scale=0.5, state=state, slots=live)
    if B > 3:
        want[1] = 7.0
    gs.check("the state store")
    go.check("the output")
    assert rel_err(st.tensor.double().cpu(), ws) <= 1e-5      # fp32 sums of d terms: d * 2^-24 = 8e-6 at most, of terms of both signs
    assert rel_err(o.double().cpu(), want) <= (1e-5 if dtype == F32 else 2 ** -8 + 1e-5)


def test_state_values_that_are_not_finite():
    """A row whose slot holds a NaN spoils its own columns and no other row; a skipped slot is not read."""
    dsla = _dsla()
    q, k, v, g, b = _draw(3, 2, 1, 64, F32, 1)
    st = dsla.dsla_state_alloc_n(3, 1, 2, 64, 64)
    st.tensor.normal_()
    st.tensor[1] = float("nan")
    before = st.tensor.clone()
    o = dsla.dsla_delta_decode_step(q, k, v, g, b, st, slots=torch.tensor([0, -1, 2], dtype=torch.int32, device="cuda"))
    assert bool(torch.isfinite(o).all()) and bool((o[1] == 0).all()) and bool(torch.isfinite(st.tensor[[0, 2]]).all())
    assert torch.equal(torch.isnan(st.tensor), torch.isnan(before))


@both
def test_slots_far_into_a_large_store(impl, dtype, d):
    """Offsets beyond 32 bits: a store of 18 GB, its last slots."""
    dsla = _dsla()
    H = 32
    slots = (18 << 30) // (H * d * d * 4)
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    q, k, v, g, b = _draw(100, H, 1, d, dtype, 2)
    small, big = dsla.dsla_state_alloc_n(1, 1, H, d, d), dsla.dsla_state_alloc_n(slots, 1, H, d, d)
    last = torch.tensor([slots - 1], dtype=torch.int32, device="cuda")
    want = dsla.dsla_delta_prefill(q, k, v, g, b, small, impl=impl)
    got = dsla.dsla_delta_prefill(q, k, v, g, b, big, slots=last, impl=impl)
    assert torch.equal(want, got) and torch.equal(small.tensor[0], big.tensor[-1])
    one = [x[:1].contiguous() for x in (q, k, v, g, b)]
    assert torch.equal(dsla.dsla_delta_decode_step(*one, small), dsla.dsla_delta_decode_step(*one, big, slots=last))
    assert torch.equal(small.tensor[0], big.tensor[-1])
    dsla.dsla_state_copy(big, last, last - 1)
    assert torch.equal(small.tensor[0], big.tensor[-2])


@both
def test_streams_and_graphs(impl, dtype, d):
    """The same results on a side stream, from two streams at once with a workspace each, and from two captured graphs replayed in turn."""
    dsla = _dsla()
    sets = [_draw(150, 4, 1, d, dtype, s) for s in (1, 2)]
    want = []
    for x in sets:
        st = dsla.dsla_state_alloc_n(2, 1, 4, d, d)
        want.append((dsla.dsla_delta_prefill(*x, st, impl=impl).clone(), st.tensor[0].clone()))
    stores = [dsla.dsla_state_alloc_n(2, 1, 4, d, d) for _ in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = []
    for x, st, s in zip(sets, stores, streams):
        got.append(dsla.dsla_delta_prefill(*x, st, impl=impl, stream=s))      # the workspace of the call is recorded on that stream
    torch.cuda.synchronize()
    for (o, S), y, st in zip(want, got, stores):
        assert torch.equal(o, y) and torch.equal(S, st.tensor[0])
    graphs, outs = [], []
    for x, st in zip(sets, stores):
        o = torch.empty_like(x[2])
        need = dsla.dsla_delta_prefill_workspace_bytes(150, 1, 150, 4, d, dtype, impl=impl, dense_T=150)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            dsla.dsla_delta_prefill(*x, st, o=o, impl=impl, workspace=ws)
            dsla.dsla_state_copy(st, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"))
        graphs.append((gr, ws))
        outs.append(o)
    for st in stores:
        st.tensor.fill_(float("nan"))
    for _ in range(2):
        for gr, _ in graphs:
            gr.replay()
    torch.cuda.synchronize()
    for (o, S), y, st in zip(want, outs, stores):
        assert torch.equal(o, y) and torch.equal(S, st.tensor[0]) and torch.equal(S, st.tensor[1])


@both
def test_same_call_twice_is_bitwise_the_same(impl, dtype, d):
    dsla = _dsla()
    x = _draw(333, 3, 1, d, dtype, 9)
    a, b = (dsla.dsla_state_alloc_n(1, 1, 3, d, d) for _ in range(2))
    assert torch.equal(dsla.dsla_delta_prefill(*x, a, impl=impl), dsla.dsla_delta_prefill(*x, b, impl=impl)) and torch.equal(a.tensor, b.tensor)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_serving_loop(dtype):
    """A shared prompt out of a fused projection, forked to three sequences that go on token by token, one of them freed, the store compacted:
    norms, rotation, prompt, copies and single tokens as they are used together, against the checkers run on the same inputs."""
    from oracle import dsla_oracle as orc
    dsla = _dsla()
    T, H, d, steps = 90, 4, 64, 5
    r = torch.Generator().manual_seed(11)
    rows = torch.randn(T + 3 * steps, 3 * H, d, generator=r).to(dtype).cuda()
    gate, beta = (torch.sigmoid(torch.randn(T + 3 * steps, H, generator=r) + m).cuda() for m in (3, 0))
    freq = 10000.0 ** (-torch.arange(0, 32, 2) / 32).cuda()
    pos = torch.cat([torch.arange(T), T + torch.arange(steps).repeat_interleave(3)]).to(torch.int32).cuda()
    st = dsla.dsla_state_alloc_n(4, 1, H, d, d)
    st.tensor.fill_(float("nan"))
    outs = []

    def qkv(a, e):
        q, k = dsla.dsla_qk_norm_rope(rows[a:e, :H], rows[a:e, H:2 * H], positions=pos[a:e], inv_freq=freq, norm="l2")
        return q, k, rows[a:e, 2 * H:].contiguous(), gate[a:e].contiguous(), beta[a:e].contiguous()
    kept = [qkv(0, T)]
    outs.append(dsla.dsla_delta_prefill(*kept[0], st, slots=torch.tensor([3], dtype=torch.int32, device="cuda"), scale=0.2))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    dsla.dsla_state_copy(st, i32(3, 3, 3, -1), i32(0, 1, 2, 3))
    for s in range(steps):
        x = qkv(T + 3 * s, T + 3 * s + 3)
        kept.append(x)
        outs.append(dsla.dsla_delta_decode_step(*x, st, slots=i32(0, 1, 2), scale=0.2))
    final = st.tensor.clone()
    dsla.dsla_state_copy(st, i32(2, -1), i32(1, 2))
    want_state = np.zeros((4, 1, H, d, d))
    wide = [[y.double().cpu().numpy() for y in x] for x in kept]
    for (a, e), x in zip([(0, T)] + [(T + 3 * s, T + 3 * s + 3) for s in range(steps)], wide):      # the norms' own results
        f = rows[a:e].double().cpu().numpy()
        p = pos[a:e].cpu().numpy()
        for y, z in ((x[0], f[:, :H]), (x[1], f[:, H:2 * H])):
            assert rel_err(y, orc.qk_norm_rope(z, None, p, freq.double().cpu().numpy(), norm="l2")) <= (2 ** -8 if dtype == BF else 1e-6) + 1e-6
    o, _ = orc.delta_prefill(*wide[0], scale=0.2, state=want_state, slots=[3])
    assert rel_err(outs[0].double().cpu(), o) <= TOL_O[dtype]
    orc.state_copy(want_state, [3, 3, 3, -1], [0, 1, 2, 3])
    for x, y in zip(wide[1:], outs[1:]):
        o, _ = orc.delta_prefill(*x, np.arange(4), scale=0.2, state=want_state, slots=[0, 1, 2])
        assert rel_err(y.double().cpu(), o) <= TOL_O[dtype]
    assert rel_err(final.double().cpu(), want_state) <= TOL_S
    assert torch.equal(st.tensor[1], final[2]) and torch.equal(st.tensor[0], final[0]) and not bool(st.tensor[2:].any())


@pytest.mark.parametrize("impl,dtype,d", CHUNKED)
@pytest.mark.parametrize("resume", [False, True])
def test_more_heads_than_sms(impl, dtype, d, resume):
    """So many (sequence, head) pairs that a CTA takes 64 columns."""
    _check([70, 200, 1, 0, 129, 64], 40, 2, d, dtype, impl, seed=21, resume=resume, slots=[3, 5, 0, 1, 6, 2], extra_slots=1)


@pytest.mark.parametrize("impl,dtype,d", CHUNKED)
def test_bad_values_stay_in_their_sequence_with_many_heads(impl, dtype, d):
    dsla = _dsla()
    q, k, v, g, b = _draw(150, 96, 1, d, dtype, 3)
    cu = torch.tensor([0, 50, 100, 150], dtype=torch.int32, device="cuda")
    st, st2 = (dsla.dsla_state_alloc_n(3, 1, 96, d, d) for _ in range(2))
    want = dsla.dsla_delta_prefill(q, k, v, g, b, st, cu_seqlens=cu, max_seqlen=50, impl=impl)
    for x in (q, k, v, g, b):
        x[50:100] = float("nan")
    got = dsla.dsla_delta_prefill(q, k, v, g, b, st2, cu_seqlens=cu, max_seqlen=50, impl=impl)
    for a, e, n in ((0, 50, 0), (100, 150, 2)):
        assert torch.equal(want[a:e], got[a:e]) and torch.equal(st.tensor[n], st2.tensor[n])


@both
def test_many_short_sequences(impl, dtype, d):
    """More sequences than are put in order of length, some of them empty."""
    lens = [int(x) for x in torch.randint(0, 40, (140,), generator=torch.Generator().manual_seed(1))]
    _check(lens, 2, 1, d, dtype, impl, seed=22)


@both
def test_rows_behind_the_last_sequence_are_left_alone(impl, dtype, d):
    dsla = _dsla()
    q, k, v, g, b = _draw(200, 2, 1, d, dtype, 6)
    for x in (q, k, v, g, b):
        x[130:] = float("nan")
    cu = torch.tensor([0, 60, 130], dtype=torch.int32, device="cuda")
    o = torch.full_like(v, 5.0)
    st = dsla.dsla_state_alloc_n(2, 1, 2, d, d)
    dsla.dsla_delta_prefill(q, k, v, g, b, st, o=o, cu_seqlens=cu, max_seqlen=70, impl=impl)
    assert bool((o[130:] == 5).all()) and bool(torch.isfinite(o[:130]).all()) and bool(torch.isfinite(st.tensor).all())


@pytest.mark.parametrize("impl", ["tensor", "simt"])
def test_tokens_far_into_a_packed_batch(impl):
    """Element offsets beyond 32 bits: a sequence of 150 tokens behind 540K rows that belong to none (cu_seqlens begins behind them)."""
    dsla = _dsla()
    H, d, far, n = 32, 128, 540_000, 150
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    tail = _draw(n, H, 1, d, BF, 8)
    whole = [torch.zeros((far + n,) + x.shape[1:], dtype=x.dtype, device="cuda") for x in tail]
    for x, y in zip(whole, tail):
        x[far:] = y
    st, small = (dsla.dsla_state_alloc_n(1, 1, H, d, d) for _ in range(2))
    o = torch.zeros_like(whole[2])
    got = dsla.dsla_delta_prefill(*whole, st, o=o, cu_seqlens=torch.tensor([far, far + n], dtype=torch.int32, device="cuda"), max_seqlen=n, impl=impl)
    want = dsla.dsla_delta_prefill(*tail, small, impl=impl)
    assert torch.equal(got[far:], want) and torch.equal(st.tensor, small.tensor) and not bool(got[:far].any())


@pytest.mark.parametrize("impl,dtype,d", CHUNKED)
@pytest.mark.parametrize("resume", [False, True])
def test_many_blocks_a_cta(impl, dtype, d, resume):
    """Several times more (sequence, head, 64 columns) than SMs, of lengths from none to some chunks, in slots out of order."""
    lens = [1, 0, 130, 64, 3, 0, 65, 1, 1, 192, 0, 17, 128, 2, 63, 1]
    _check(lens, 48, 3, d, dtype, impl, seed=23, resume=resume, slots=[(7 * i + 3) % 17 for i in range(16)])


@pytest.mark.parametrize("impl,dtype,d", CHUNKED)
def test_many_blocks_on_two_streams_and_in_graphs(impl, dtype, d):
    """Two such calls at once on two streams, a store and a workspace each, then both from captured graphs: the same bits as one after the other."""
    dsla = _dsla()
    H, lens = 40, [70, 1, 0, 129, 5, 64, 200, 1, 33]
    cu = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
    kw = dict(cu_seqlens=cu, max_seqlen=200, impl=impl, use_initial_state=True)
    sets = [_draw(sum(lens), H, 1, d, dtype, s) for s in (3, 4)]
    stores = [dsla.dsla_state_alloc_n(len(lens), 1, H, d, d) for _ in sets]
    want = []
    for x, st in zip(sets, stores):
        st.tensor.fill_(0.25)
        want.append((dsla.dsla_delta_prefill(*x, st, **kw), st.tensor.clone()))
    need = dsla.dsla_delta_prefill_workspace_bytes(sum(lens), len(lens), 200, H, d, dtype, impl=impl)
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in sets]
    outs = [torch.empty_like(x[2]) for x in sets]
    streams = [torch.cuda.Stream() for _ in sets]

    def check(run):
        for st, o in zip(stores, outs):
            st.tensor.fill_(0.25)
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        for (o, S), y, st in zip(want, outs, stores):
            assert dsla.dsla_state_last_error(st) == dsla.DSLA_OK and torch.equal(o, y) and torch.equal(S, st.tensor)

    def eager():
        for x, st, o, ws, s in zip(sets, stores, outs, spaces, streams):
            dsla.dsla_delta_prefill(*x, st, o=o, workspace=ws, stream=s, **kw)

    graphs = []
    for x, st, o, ws in zip(sets, stores, outs, spaces):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            dsla.dsla_delta_prefill(*x, st, o=o, workspace=ws, **kw)
        graphs.append(gr)

    def replayed():
        for gr, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()

    for run in (eager, replayed, eager, replayed):
        check(run)


@pytest.mark.parametrize("impl,dtype,d", CHUNKED)
def test_far_offsets_with_many_heads(impl, dtype, d):
    """More heads than SMs hold in slabs of 32 columns: tokens and slots whose element offsets pass 32 bits."""
    dsla = _dsla()
    H, n = 40 * 128 // d, 150
    far, slots = 430_000, 3400
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    tail = _draw(n, H, 1, d, dtype, 12)
    whole = [torch.zeros((far + n,) + x.shape[1:], dtype=x.dtype, device="cuda") for x in tail]
    for x, y in zip(whole, tail):
        x[far:] = y
    assert whole[2].numel() > 1 << 31
    st, small = dsla.dsla_state_alloc_n(slots * 128 // d, 1, H, d, d), dsla.dsla_state_alloc_n(1, 1, H, d, d)
    assert st.tensor.numel() > 1 << 31
    st.tensor[-2:] = 0.5
    small.tensor.fill_(0.5)
    got = dsla.dsla_delta_prefill(*whole, st, o=torch.zeros_like(whole[2]), cu_seqlens=torch.tensor([far, far + n], dtype=torch.int32, device="cuda"), max_seqlen=n, impl=impl,
                                  slots=torch.tensor([st.tensor.shape[0] - 1], dtype=torch.int32, device="cuda"), use_initial_state=True)
    want = dsla.dsla_delta_prefill(*tail, small, impl=impl, use_initial_state=True)
    assert torch.equal(got[far:], want) and torch.equal(st.tensor[-1], small.tensor[0]) and not bool(got[:far].any()) and bool((st.tensor[-2] == 0.5).all())


@pytest.mark.parametrize("impl,dtype,d", CHUNKED)
@pytest.mark.parametrize("lens", [[1], [64], [65, 31, 33, 63], [32, 96, 95, 97, 160]])
def test_ends_inside_a_chunk_with_many_heads(impl, dtype, d, lens):
    """Ends on, before and behind the boundaries of 32 tokens, at which outputs leave another way; rows of one sequence border on the next one's."""
    _check(lens, 80, 2, d, dtype, impl, seed=31, resume=True)


@pytest.mark.parametrize("impl,dtype,d", CHUNKED)
@pytest.mark.parametrize("gate,beta", [(0.0, "mixed"), ("tiny", "mixed"), ("mixed", 0.0), (1.0, 2.0), (1.0, 1.0)])
def test_gates_and_repeated_keys_with_many_heads(impl, dtype, d, gate, beta):
    def same(q, k, v, g, b):
        if gate == beta:      # one key over and over, then tokens without one
            k[1:] = k[:1]
            k[40:50] = 0
    _check([140, 10], 80, 1, d, dtype, impl, seed=32, gate=gate, beta=beta, resume=True, edit=same)


@pytest.mark.parametrize("impl,dtype,d", CHUNKED)
def test_rows_that_belong_to_no_sequence_with_many_heads(impl, dtype, d):
    """Rows before the first and behind the last sequence hold NaN and infinities, and stay as they are; so do the slots of no sequence."""
    dsla = _dsla()
    H = 80
    x = _draw(300, H, 1, d, dtype, 33)
    cu = torch.tensor([37, 37, 137, 170, 265], dtype=torch.int32, device="cuda")
    slots = torch.tensor([6, 1, 4, 2], dtype=torch.int32, device="cuda")
    st = dsla.dsla_state_alloc_n(8, 1, H, d, d)
    out = []
    for bad in (0.0, float("nan"), float("inf")):
        y = [z.clone() for z in x]
        for z in y:
            z[:37] = bad
            z[265:] = bad
        st.tensor.fill_(0.25)
        o = torch.full_like(y[2], 5.0)
        dsla.dsla_delta_prefill(*y, st, o=o, cu_seqlens=cu, slots=slots, max_seqlen=100, impl=impl, use_initial_state=True)
        assert bool((o[:37] == 5).all()) and bool((o[265:] == 5).all()) and bool(torch.isfinite(o).all())
        assert all(bool((st.tensor[n] == 0.25).all()) for n in (0, 3, 5, 6, 7)) and dsla.dsla_state_last_error(st) == dsla.DSLA_OK
        out.append((o, st.tensor.clone()))
    assert all(torch.equal(out[0][0], o) and torch.equal(out[0][1], s) for o, s in out[1:])
