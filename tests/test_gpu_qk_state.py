"""Norms and rotation of queries and keys, and copies of state slots, against the fp64 checkers.

A bf16 result is off by its rounding, 2^-8 of the value, and by the fp32 arithmetic before it; an fp32 one by that alone: a sum of d squares
(d * 2^-24 / 2 of the norm at most), a reciprocal root, three products, and the sine and cosine of an angle rounded to fp32 within half a turn
(pi * 2^-24): below 1e-5 of a head's largest value, which both are compared with."""
import numpy as np
import pytest
import torch

from util import SENTINEL, rel_err

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
TOL = {BF: 2 ** -8 + 1e-5, F32: 1e-5}


def _dsla():
    import paper_2506_09316_b200 as dsla
    return dsla


def _freq(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().cuda() if rot else None


def _case(T, H, Hk, d, rot, dtype, norm, inter, weights, seed=0, scale=1.0):
    from oracle import dsla_oracle as orc
    dsla = _dsla()
    r = torch.Generator().manual_seed(seed)
    fused = (torch.randn(T, H + 2 * Hk + 1, d, generator=r) * scale).to(dtype).cuda()
    q, k = fused[:, :H], fused[:, H:H + Hk]
    wq, wk = ((torch.randn(d, generator=r) + 1).cuda() for _ in range(2)) if weights else (None, None)
    pos = torch.randint(-5, 1 << 20, (T,), generator=r, dtype=torch.int32).cuda() if rot else None
    out = torch.full((T, H + Hk + 2, d), SENTINEL, dtype=dtype, device="cuda")
    before = fused.clone()
    qo, ko = dsla.dsla_qk_norm_rope(q, k, wq, wk, positions=pos, inv_freq=_freq(rot), q_out=out[:, 1:1 + H], k_out=out[:, 1 + H:1 + H + Hk], norm=norm, interleaved=inter)
    assert torch.equal(fused, before) and bool((out[:, 0] == out[0, 0, 0]).all()) and bool((out[:, -1] == out[0, 0, 0]).all())
    f = None if not rot else _freq(rot).double().cpu().numpy()
    p = None if not rot else pos.cpu().numpy()
    for x, w, y in ((q, wq, qo), (k, wk, ko)):
        want = orc.qk_norm_rope(x.double().cpu().numpy(), None if w is None else w.double().cpu().numpy(), p, f, norm=norm, interleaved=inter)
        assert rel_err(y.double().cpu(), want) <= TOL[dtype]
    a, b = fused[:, :H], fused[:, H:H + Hk]      # in place
    dsla.dsla_qk_norm_rope(a, b, wq, wk, positions=pos, inv_freq=_freq(rot), q_out=a, k_out=b, norm=norm, interleaved=inter)
    assert torch.equal(a, qo) and torch.equal(b, ko) and torch.equal(fused[:, H + Hk:], before[:, H + Hk:])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,rot", [(64, 0), (64, 16), (64, 48), (64, 64), (128, 0), (128, 32), (128, 112), (128, 128)])
@pytest.mark.parametrize("norm", ["rms", "l2", "none"])
@pytest.mark.parametrize("inter", [False, True])
def test_norms_and_rotations(dtype, d, rot, norm, inter):
    _case(11, 5, 3, d, rot, dtype, norm, inter, weights=rot % 32 == 0)


@pytest.mark.parametrize("T,H,Hk", [(1, 1, 1), (1, 32, 32), (1, 40, 1), (2, 1, 33), (300, 7, 2), (2048, 16, 16)])
@pytest.mark.parametrize("d", [64, 128])
def test_sizes(T, H, Hk, d):
    _case(T, H, Hk, d, 64, BF, "rms", False, True, seed=T)


@pytest.mark.parametrize("scale", [1e-12, 1e12])
def test_range(scale):
    """Squares of 1e12 and of 1e-12 stay within fp32; the norm's eps takes over at the small end."""
    _case(5, 2, 2, 128, 0, F32, "rms", False, False, scale=scale)


def test_no_rows():
    dsla = _dsla()
    q = torch.empty(0, 2, 64, device="cuda")
    a, b = dsla.dsla_qk_norm_rope(q, q)
    assert a.shape == b.shape == q.shape


def test_bad_values_stay_in_their_head():
    dsla = _dsla()
    q = torch.randn(3, 4, 128, device="cuda")
    k = q.clone()
    want = dsla.dsla_qk_norm_rope(q, k)
    q[1, 2, 5] = float("nan")
    k[0, 1, 7] = float("inf")
    got = dsla.dsla_qk_norm_rope(q, k)
    for w, g, at in zip(want, got, ((1, 2), (0, 1))):
        assert not bool(torch.isfinite(g[at]).all())
        g[at] = w[at]
        assert torch.equal(w, g)


def test_far_positions():
    """Angles of positions where an fp32 product has lost its turns."""
    from oracle import dsla_oracle as orc
    dsla = _dsla()
    q = torch.randn(64, 2, 128, device="cuda")
    pos = torch.arange((1 << 31) - 64, 1 << 31).to(torch.int32).cuda()
    a, _ = dsla.dsla_qk_norm_rope(q, q, positions=pos, inv_freq=_freq(128), norm="none")
    want = orc.qk_norm_rope(q.double().cpu().numpy(), None, pos.cpu().numpy(), _freq(128).double().cpu().numpy(), norm="none")
    assert rel_err(a.double().cpu(), want) <= 1e-5


@pytest.mark.parametrize("n_states,H,d", [(1, 3, 64), (2, 2, 128), (4, 1, 64)])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 64, 255, 256, 257, 700])
def test_copies_in_order(n_states, H, d, n):
    """Random lists: forks, chains, cycles, targets named twice, clears, moves of a slot to itself, entries that name no slot."""
    from oracle import dsla_oracle as orc
    dsla = _dsla()
    slots = 13
    r = np.random.default_rng(n)
    src, dst = (r.integers(-2, slots + 2, n).astype(np.int32) for _ in range(2))
    pad = torch.randn(slots + 2, n_states, H, d, d, device="cuda")
    st = dsla.dsla_state_alloc_n(slots, n_states, H, d, d, buffer=pad[1:-1])
    before = pad.clone()
    dsla.dsla_state_copy(st, torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda())
    want = orc.state_copy(before[1:-1].cpu().numpy(), src, dst)
    np.testing.assert_array_equal(st.tensor.cpu().numpy(), want)
    assert torch.equal(pad[0], before[0]) and torch.equal(pad[-1], before[-1])


@pytest.mark.parametrize("n", [3, 40])
def test_fork_compact_and_free(n):
    dsla = _dsla()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    st = dsla.dsla_state_alloc(2 * n, 2, 64, 64)
    st.tensor.normal_()
    b = st.tensor.clone()
    dsla.dsla_state_copy(st, i32([0] * (n - 1)), i32(list(range(1, n))))
    assert all(torch.equal(st.tensor[i], b[0]) for i in range(n)) and torch.equal(st.tensor[n:], b[n:])
    dsla.dsla_state_copy(st, i32(list(range(n, 2 * n)) + [-1] * n), i32(list(range(n)) + list(range(n, 2 * n))))
    assert torch.equal(st.tensor[:n], b[n:]) and not bool(st.tensor[n:].any())
    dsla.dsla_state_copy(st, i32([]), i32([]))
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    dsla.dsla_state_copy(st, i32([-1] * n), i32(list(range(n))), stream=other)
    torch.cuda.synchronize()
    assert not bool(st.tensor.any())


def test_values_are_copied_as_bits():
    dsla = _dsla()
    st = dsla.dsla_state_alloc_n(2, 1, 1, 64, 64)
    bits = torch.randint(-(1 << 31), (1 << 31) - 1, (64, 64), dtype=torch.int64, device="cuda").to(torch.int32)      # NaN payloads among them
    st.tensor[0].view(torch.int32).copy_(bits.view(1, 64, 64))
    dsla.dsla_state_copy(st, torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda"))
    assert torch.equal(st.tensor[1].view(torch.int32).view(64, 64), bits)
