"""How exact the gated delta rule is, each kernel by its own arithmetic, judged for every sequence and head by itself.

An output may be off by its own rounding (2^-8 of its value in bf16, 2^-24 in fp32) and by ARITH[kernel] of the size of what it is summed from, since its summands can
cancel: scale * sum_a |q_a| |S_ab|, the largest of its sequence and head.  A state is compared with the largest value of its sequence and head, before or after the prompt.

TENSOR outputs.  Held in two bf16 terms, off by 2^-8 of what the first leaves, 2^-16: S, R, P, T, P T; left out, 2^-8 * 2^-8: the products of the low terms in P T and in
(P T) R.  7 * 2^-16 = 1.07e-4.  One term in place of any of these two is 2^-8 = 3.9e-3.
TENSOR states.  S, R, Y and the low product of Y R: 4 * 2^-16 = 6.1e-5 if every error had the same sign.  A single token has one of them (Y's); errors of different sign add up by the root of their
number: 2 * 2^-16 where keys differ.
SIMT.  Three products are on the way to a state, and to an output, each of two factors that are off by 2^-21 (the second TF32 term is cut off) and without the product of the low terms, 2^-22: 7.5 * 2^-21 =
3.6e-6 if every error had the same sign, of which half is allowed where keys differ."""
import numpy as np
import pytest
import torch

from test_gpu_delta import BF, CHUNKED, F32, KERNELS, _draw

pytestmark = pytest.mark.gpu
ARITH = {"tensor": 7 * 2.0 ** -16, "simt": 1.8e-6}
STATE = {"tensor": 2 * 2.0 ** -16, "simt": 1.8e-6}
STATE_WORST = {"tensor": 4 * 2.0 ** -16, "simt": 3.6e-6}
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}
both = pytest.mark.parametrize("impl,dtype,d", KERNELS)


def _dsla():
    import paper_2506_09316_b200 as dsla
    return dsla


def _worst(got, want, size, half):
    """The largest error of an element beyond its own rounding, as a share of `size` (of its head); exact where the size is zero."""
    over = np.abs(got - want) - half * np.abs(want)
    if not np.isfinite(over).all():
        return float("inf")
    worst = over.max(initial=0.0)
    return 0.0 if worst <= 0 else float("inf") if size == 0 else worst / (size * (1 + half))


def _definition(x, lens, scale, start):
    """Token by token in fp64: outputs, final states, and the sizes of what the outputs are summed from."""
    q, k, v, g, b = (y.double() for y in x)
    group = v.shape[1] // q.shape[1]
    q, k = q.repeat_interleave(group, 1), k.repeat_interleave(group, 1)
    o, size, state = torch.zeros_like(v), torch.zeros_like(v), start.double().cuda()
    t = 0
    for n, length in enumerate(lens):
        S = state[n, 0]
        for t in range(t, t + length):
            S *= g[t][:, None, None]
            S += k[t][..., None] * (b[t][:, None] * (v[t] - torch.einsum("hk,hkv->hv", k[t], S)))[:, None]
            o[t] = scale * torch.einsum("hk,hkv->hv", q[t], S)
            size[t] = abs(scale) * torch.einsum("hk,hkv->hv", q[t].abs(), S.abs())
        t += length > 0
    return (y.cpu().numpy() for y in (o, state, size))


def _errors(x, lens, impl, *, scale, init=None):
    """Largest errors of outputs and states over all sequences and heads."""
    dsla = _dsla()
    v = x[2]
    (_, H, d), N = v.shape, len(lens)
    cu = [0] + list(np.cumsum(lens))
    st = dsla.dsla_state_alloc_n(N, 1, H, d, d)
    st.tensor.copy_(torch.full((N, 1, H, d, d), float("nan")) if init is None else init)
    o = torch.full_like(v, float("nan"))
    dsla.dsla_delta_prefill(*x, st, o=o, cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"), max_seqlen=max(lens), scale=scale, use_initial_state=init is not None, impl=impl)
    assert dsla.dsla_state_last_error(st) == dsla.DSLA_OK
    start = torch.zeros(N, 1, H, d, d) if init is None else init
    want, state, size = _definition(x, lens, scale, start)
    start, got, got_state = start.numpy(), o.double().cpu().numpy(), st.tensor.double().cpu().numpy()
    eo = es = 0.0
    for n in range(N):
        at = slice(cu[n], cu[n + 1])
        for h in range(H):
            eo = max(eo, _worst(got[at, h], want[at, h], size[at, h].max(initial=0.0), HALF[v.dtype]))
            es = max(es, _worst(got_state[n, 0, h], state[n, 0, h], max(np.abs(start[n, 0, h]).max(), np.abs(state[n, 0, h]).max()), HALF[F32]))
    return eo, es


def _init(N, H, d, seed, size):
    return torch.randn(N, 1, H, d, d, generator=torch.Generator().manual_seed(seed)) * size


@both
@pytest.mark.parametrize("resume", [False, True])
@pytest.mark.parametrize("many", [False, True])
def test_ordinary_inputs(impl, dtype, d, resume, many):
    """Few heads, and so many that other walks serve them."""
    lens, H = [70, 200, 1, 0, 129, 64], 80 if many else 4
    x = _draw(sum(lens), H, 2, d, dtype, 41)
    eo, es = _errors(x, lens, impl, scale=0.3, init=_init(len(lens), H, d, 1, 0.1) if resume else None)
    assert eo <= ARITH[impl] and es <= STATE[impl], (eo, es)


@both
@pytest.mark.parametrize("many", [False, True])
def test_outputs_that_cancel(impl, dtype, d, many):
    """q = k, beta near 1 and a state several times larger than v: what the state answers is taken back by (P T) R, and what is left is of v's size."""
    lens, H = [150, 64, 33], 80 if many else 3
    r = torch.Generator().manual_seed(5)
    q, k, v, _, _ = _draw(sum(lens), H, 1, d, dtype, 42)
    g, b = (1 - s * torch.rand(sum(lens), H, generator=r).cuda() for s in (0.01, 0.05))
    eo, es = _errors([k.clone(), k, v, g, b], lens, impl, scale=0.5, init=_init(len(lens), H, d, 2, 8.0))
    assert eo <= ARITH[impl] and es <= STATE[impl], (eo, es)


@both
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("beta", [1.0, 2.0])
def test_full_triangles(impl, dtype, d, many, beta):
    """One key over and over without forgetting (beta 1), and keys that turn the state over (beta 2): errors of one sign may add up."""
    lens, H = [140, 90], 80 if many else 2
    q, k, v, g, b = _draw(sum(lens), H, 1, d, dtype, 43, gate=1.0, beta=beta)
    if beta == 1.0:
        k[1:] = k[:1]
    eo, es = _errors([q, k, v, g, b], lens, impl, scale=0.3, init=_init(len(lens), H, d, 3, 0.5))
    assert eo <= max(ARITH[impl], STATE_WORST[impl]) and es <= STATE_WORST[impl], (eo, es)


@both
def test_long_prompt_that_forgets_little(impl, dtype, d):
    T, H = 3000, 2
    q, k, v, _, b = _draw(T, H, 1, d, dtype, 44)
    g = 1 - 1e-4 * torch.rand(T, H, generator=torch.Generator().manual_seed(6)).cuda()
    eo, es = _errors([q, k, v, g, b], [T], impl, scale=0.3)
    assert eo <= ARITH[impl] and es <= STATE[impl], (eo, es)


@pytest.mark.parametrize("impl,dtype,d", CHUNKED)
def test_prompt_and_single_tokens_agree(impl, dtype, d):
    """The same tokens as a prompt and one by one: both round the same numbers, so few outputs differ, and by one step."""
    dsla = _dsla()
    T, H = 130, 4
    x = _draw(T, H, 1, d, dtype, 45)
    a, b = (dsla.dsla_state_alloc_n(1, 1, H, d, d) for _ in range(2))
    a.tensor.zero_()
    one = torch.cat([dsla.dsla_delta_decode_step(*[y[t:t + 1].contiguous() for y in x], a) for t in range(T)])
    all_ = dsla.dsla_delta_prefill(*x, b, impl=impl)
    # an error of ARITH of the largest output moves an element of that size over a border between two bf16 numbers, 2^-8 of it apart at least, with a chance of ARITH / 2^-8 = 2.7 %, and of
    # one of a tenth of it with ten times that
    differ = (one != all_).double()
    big = one.double().abs() >= 0.1 * one.double().abs().amax((0, 2), keepdim=True)
    assert differ[big].mean() <= 0.27


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_a_nan_in_a_state_stays_in_its_column(dtype, d):
    """A slot with a NaN in one column of one head: that column of that row's output and state, and nothing else."""
    dsla = _dsla()
    x = _draw(5, 4, 2, d, dtype, 46)
    slots = torch.tensor([3, 1, -1, 0, 2], dtype=torch.int32, device="cuda")
    init = _init(4, 4, d, 4, 1.0).cuda()
    out = []
    for spoilt in (False, True):
        st = dsla.dsla_state_alloc_n(4, 1, 4, d, d)
        st.tensor.copy_(init)
        if spoilt:
            st.tensor[1, 0, 2, 7, 37] = float("nan")
        out.append((dsla.dsla_delta_decode_step(*x, st, slots=slots), st.tensor))
    (o, s), (o2, s2) = out
    assert bool(torch.isfinite(o).all()) and bool(torch.isfinite(s).all())
    bad_o, bad_s = torch.zeros_like(o, dtype=torch.bool), torch.zeros_like(s, dtype=torch.bool)
    bad_o[1, 2, 37] = True          # row 1 has slot 1
    bad_s[1, 0, 2, :, 37] = True
    assert bool(torch.isnan(o2[bad_o]).all()) and bool(torch.isnan(s2[bad_s]).all())
    assert torch.equal(o[~bad_o], o2[~bad_o]) and torch.equal(s[~bad_s], s2[~bad_s])
