"""What the delta-rule, norm and copy entry points refuse, on the host, before anything is launched.  No GPU needed."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2506_09316_b200 import binding
    return binding


def _prefill(b, **kw):
    a = b.dsla_delta_prefill_args()
    a.N, a.T, a.T_total, a.max_seqlen, a.H, a.H_qk, a.d_k, a.d_v, a.dtype, a.scale = 1, 8, 8, 8, 4, 2, 64, 64, b.DSLA_F32, 1.0
    for x, v in kw.items():
        setattr(a, x, v)
    return b._lib.dsla_delta_prefill(ctypes.byref(a), None, None)


def test_delta_prefill(b):
    bad, no = b.DSLA_ERR_INVALID_ARG, b.DSLA_ERR_UNSUPPORTED
    assert b._lib.dsla_delta_prefill(None, None, None) == bad and _prefill(b) == bad      # no store
    for kw in (dict(H=5), dict(H_qk=0), dict(H=0), dict(N=-1), dict(T_total=9), dict(max_seqlen=7), dict(dtype=2), dict(impl=9), dict(d_k=0), dict(T=-8, N=-1)):
        assert _prefill(b, **kw) == bad, kw
    for kw in (dict(d_k=96, d_v=96), dict(d_k=64, d_v=128), dict(impl=b.DSLA_IMPL_TENSOR), dict(impl=b.DSLA_IMPL_TENSOR_PAIR)):
        assert _prefill(b, **kw) == no, kw
    assert b._lib.dsla_delta_prefill_workspace_bytes(None) == 0
    assert b.dsla_delta_prefill_workspace_bytes(512, 1, 512, 4, 64, torch.float32, dense_T=512) == 0
    assert b.dsla_delta_prefill_workspace_bytes(512, 1, 512, 4, 64, torch.bfloat16, impl="simt", dense_T=512) == 0


def test_workspace_is_what_the_kernel_uses(b):
    """A chunk of 64 tokens and a head take Y in two terms [d][64], P T [64][64], all bf16, and two gates per token; packed batches one chunk more per sequence."""
    for d in (64, 128):
        entry = 2 * d * 128 + 64 * 128 + 2 * 64 * 4
        assert b.dsla_delta_prefill_workspace_bytes(4096, 1, 4096, 32, d, dense_T=4096) == 64 * 32 * entry
        assert b.dsla_delta_prefill_workspace_bytes(3 * 65, 3, 65, 8, d, dense_T=65) == 3 * 2 * 8 * entry
        assert b.dsla_delta_prefill_workspace_bytes(1000, 7, 900, 8, d) == (1000 // 64 + 7) * 8 * entry
        assert b.dsla_delta_prefill_workspace_bytes(1000, 7, 900, 8, d, H_qk=2) == (1000 // 64 + 7) * 8 * entry
    assert b.dsla_delta_prefill_workspace_bytes(0, 3, 0, 8, 128) == 0 and b.dsla_delta_prefill_workspace_bytes(1000, 7, 900, 8, 128, H_qk=3) == 0


def test_delta_decode(b):
    a = b.dsla_delta_decode_args()
    a.B, a.H, a.H_qk, a.d_k, a.d_v = 1, 2, 2, 64, 64
    assert b._lib.dsla_delta_decode_step(ctypes.byref(a), None, None) == b.DSLA_ERR_INVALID_ARG
    assert b._lib.dsla_delta_decode_step(None, None, None) == b.DSLA_ERR_INVALID_ARG


def _qk(b, **kw):
    a = b.dsla_qk_norm_rope_args()
    a.q = a.k = a.q_out = a.k_out = a.positions = a.inv_freq = 4096      # never dereferenced: each call is refused
    a.T, a.H, a.H_k, a.d, a.rot, a.norm, a.dtype, a.eps = 2, 4, 2, 64, 32, b.DSLA_NORM_RMS, b.DSLA_BF16, 1e-6
    a.q_stride = a.q_out_stride = 256
    a.k_stride = a.k_out_stride = 128
    for x, v in kw.items():
        setattr(a, x, v)
    return b._lib.dsla_qk_norm_rope(ctypes.byref(a), None)


def test_qk_norm_rope(b):
    assert b._lib.dsla_qk_norm_rope(None, None) == b.DSLA_ERR_INVALID_ARG
    for kw in (dict(H=0), dict(H_k=0), dict(T=-1), dict(rot=80), dict(rot=-16), dict(norm=3), dict(dtype=5), dict(eps=-1.0), dict(eps=float("nan")), dict(q=None),
               dict(k_out=None), dict(positions=None), dict(inv_freq=None), dict(q=4104), dict(k_out=4100), dict(q_stride=255), dict(q_stride=260), dict(k_stride=120),
               dict(k_out_stride=-128), dict(positions=4098)):
        assert _qk(b, **kw) == b.DSLA_ERR_INVALID_ARG, kw
    for kw in (dict(d=96), dict(rot=24)):
        assert _qk(b, **kw) == b.DSLA_ERR_UNSUPPORTED, kw


def test_state_copy(b):
    assert b._lib.dsla_state_copy(None, None, None, 1, None) == b.DSLA_ERR_INVALID_ARG


def test_tensors_that_do_not_fit_together(b):
    """Wrong shapes, types and layouts, and tensors of the host, are errors of the binding: sizes come from q and v alone."""
    from paper_2506_09316_b200 import _native
    q, v, g = torch.zeros(4, 2, 64), torch.zeros(4, 4, 64), torch.zeros(4, 4)
    good = dict(q=q, k=q, v=v, o=v, gate=g, beta=g)
    wrong = [dict(), dict(k=q[:3]), dict(k=q.bfloat16()), dict(o=v.transpose(0, 1)), dict(v=v[..., ::2]), dict(gate=g.double()), dict(beta=g[:, :2]), dict(gate=None),
             dict(q=q.half()), dict(q=q[0])]
    for kw in wrong:
        x = list({**good, **kw}.values())
        with pytest.raises((ValueError, KeyError)):
            _native.delta_decode_step(*x, None, None, None, 1.0, 0)
        with pytest.raises((ValueError, KeyError)):
            _native.delta_prefill(*x, None, None, None, None, 1, 4, 4, 1.0, 0, 0, 0)
    for kw in (dict(), dict(k=q.bfloat16()), dict(q_out=torch.zeros(4, 2, 32)), dict(q=q.transpose(0, 1)), dict(q_weight=torch.zeros(32)), dict(positions=torch.zeros(4))):
        x = {**dict(q=q, k=q, q_out=q, k_out=q, q_weight=None, k_weight=None, positions=torch.zeros(4, dtype=torch.int32), inv_freq=torch.zeros(16)), **kw}
        with pytest.raises(ValueError):
            _native.qk_norm_rope(*x.values(), 1e-6, 1, 0, 0)
    i = torch.zeros(3, dtype=torch.int32)
    for a, c in ((i, i), (i, i[:2]), (i.long(), i.long()), (i, None), (i.view(3, 1), i.view(3, 1))):
        with pytest.raises(ValueError):
            _native.state_copy(a, c, None, 0)
    with pytest.raises(KeyError):
        b.dsla_qk_norm_rope(q, q, norm="layer")
    with pytest.raises(ValueError):
        b.dsla_delta_prefill(q, q, v, g, g, None, cu_seqlens=i)
