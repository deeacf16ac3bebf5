"""Performance cases of the gated delta rule and of what a server needs around it.

The operators: the gated delta rule over prompts (`dsla_delta_prefill`) and over one token per row (`dsla_delta_decode_step`), the norm of
queries and keys for each head with the position rotation (`dsla_qk_norm_rope`), and the copying, forking, compacting and freeing of the
slots of a state store (`dsla_state_copy`).  Each case is one call on inputs that are on the GPU already, at sizes that a server of layers
of 32 heads of 128 (and the small fp32 layer of 4 heads of 64) meets.

`run` computes an operator in its plain form, elementary torch operations in 32 bits, unless `own` is true: then it makes the call that a
user makes.  A caller keeps its output buffers, its workspace and its store between calls, as a serving loop does.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CHUNK = 64          # tokens per chunk of the plain form
THETA = 10000.0     # base of the rotation's frequencies
EPS = 1e-6


# ---- cases ----------------------------------------------------------------------------------------------------------------------------------

def _decode(B, H=32, group=1, d=128, dtype="bf16", masked=False):
    return dict(kind="decode", B=B, H=H, group=group, d=d, dtype=dtype, masked=masked)


def _prefill(lens, H=32, group=1, d=128, dtype="bf16", resume=False):
    """`lens`: lengths as text, or "lo:hi:count:seed" for lengths drawn log-uniformly from [lo, hi].  `group`: value heads for each head of
    queries and keys."""
    return dict(kind="prefill", lens=lens, H=H, group=group, d=d, dtype=dtype, resume=resume)


def _qk(T, H=32, Hk=32, d=128, rot=128, dtype="bf16", norm="rms", interleaved=False):
    """`rot`: channels of a head that are rotated (0: norms alone)."""
    return dict(kind="qk", T=T, H=H, Hk=Hk, d=d, rot=rot, dtype=dtype, norm=norm, interleaved=interleaved)


def _copy(moves, frees, fork, n=1, H=32, d=128):
    """`moves` copies from slot to slot (`fork`: all from one slot), `frees` slots cleared in the same call, stores of n states."""
    return dict(kind="copy", moves=moves, frees=frees, fork=fork, n=n, H=H, d=d)


def listed():
    return [
        # the next token of one chat user in one layer: what a serving loop calls most often
        dict(_decode(1), name="decode_1"),
        # a full decode batch of one layer: 128 sequences, 268 MB of states
        dict(_decode(128), name="decode_128"),
        # a mixed batch of a small fp32 model, some rows of another layer's, some padding, two value heads to a key head
        dict(_decode(45, H=16, group=2, d=64, dtype="f32", masked=True), name="decode_mask_f32"),
        # pieces of 8 prompts of odd lengths that continue from the states in their slots
        dict(_prefill("301,512,77,1000,643,129,850,64", resume=True), name="delta_resume"),
        # the 4K prompt of the benchmark's default workload
        dict(_prefill("4096"), name="delta_4k"),
        # one long document: 64K tokens
        dict(_prefill("65536"), name="delta_64k"),
        # a packed batch of 16 fresh prompts of 1K to 16K tokens, two value heads to a key head
        dict(_prefill("1024:16384:16:1005", group=2), name="delta_ragged"),
        # the small fp32 layer: 4 heads of 64, 512 tokens
        dict(_prefill("512", H=4, d=64, dtype="f32"), name="delta_f32"),
        # queries and keys of one decoded token of 9 rows, unit length, the delta rule's keys without rotation
        dict(_qk(9, H=16, Hk=16, rot=0, norm="l2"), name="qk_rows_9"),
        # queries and keys of a 4K prompt out of a fused projection, normed by rms and rotated
        dict(_qk(4096), name="qk_4k"),
        # a prompt whose state is shared by the 8 sequences that continue it: one dual-state slot forked
        dict(_copy(8, 0, True, n=2), name="state_fork_8"),
        # a store compacted after a batch: 40 slots moved down, 24 freed
        dict(_copy(40, 24, False), name="state_compact_64"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "prompt", "prompt", "packed", "resume", "f32", "qk", "qk", "copy"])
    group = rng.choice([1, 1, 2, 4])
    if kind == "decode":
        return _decode(_log_int(rng, 1, 200), H=rng.choice([8, 16, 24, 32, 40]), group=group, d=rng.choice([64, 128, 128]),
                       dtype=rng.choice(["bf16", "bf16", "f32"]), masked=rng.random() < 0.3)
    if kind == "prompt":
        return _prefill(str(_log_int(rng, 1, 32768)), H=rng.choice([8, 16, 24, 32]), group=group, d=rng.choice([64, 128, 128]))
    if kind == "packed":
        count = rng.randint(2, 24)
        hi = _log_int(rng, 256, 60000 // count)
        return _prefill("%d:%d:%d:%d" % (max(1, hi // 64), hi, count, rng.randrange(1 << 20)), H=rng.choice([8, 16, 24, 32]), group=group,
                        d=rng.choice([64, 128, 128]))
    if kind == "resume":
        return _prefill(",".join(str(_log_int(rng, 1, 2048)) for _ in range(rng.randint(1, 12))), H=rng.choice([8, 16, 24, 32]), group=group,
                        d=rng.choice([64, 128, 128]), resume=True)
    if kind == "f32":
        return _prefill(str(_log_int(rng, 1, 2048)), H=4 * rng.randint(1, 4), group=group, d=rng.choice([64, 128]), dtype="f32",
                        resume=rng.random() < 0.3)
    if kind == "qk":
        d = rng.choice([64, 128, 128])
        return _qk(_log_int(rng, 1, 16384), H=rng.randint(1, 40), Hk=rng.randint(1, 40), d=d, rot=rng.choice([0, 32, 64, d]),
                   dtype=rng.choice(["bf16", "bf16", "f32"]), norm=rng.choice(["rms", "l2"]), interleaved=rng.random() < 0.3)
    return _copy(_log_int(rng, 1, 64), rng.randint(0, 16), rng.random() < 0.5, n=rng.choice([1, 2]), H=rng.choice([4, 8, 16, 32]),
                 d=rng.choice([64, 128]))


def _lengths(case):
    if ":" not in case["lens"]:
        return [int(x) for x in case["lens"].split(",")]
    lo, hi, count, seed = (int(x) for x in case["lens"].split(":"))
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(count, generator=g, dtype=torch.float64)
    return [int(x) for x in torch.exp(math.log(lo) + u * (math.log(hi) - math.log(lo))).round().long()]


# ---- inputs ---------------------------------------------------------------------------------------------------------------------------------

class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, shape, dtype=torch.float32, scale=1.0):
        out = torch.empty(shape, dtype=dtype, device="cuda")
        rows = max(1, (1 << 27) // max(1, math.prod(shape[1:])))
        for r in range(0, shape[0], rows):
            e = min(shape[0], r + rows)
            out[r:e] = torch.randn((e - r,) + tuple(shape[1:]), generator=self.g, device="cuda") * scale
        return out

    def unit(self, shape, dtype):
        """Rows of unit length, as a layer norms its queries and keys."""
        out = torch.empty(shape, dtype=dtype, device="cuda")
        rows = max(1, (1 << 27) // max(1, math.prod(shape[1:])))
        for r in range(0, shape[0], rows):
            e = min(shape[0], r + rows)
            x = torch.randn((e - r,) + tuple(shape[1:]), generator=self.g, device="cuda")
            out[r:e] = x / x.norm(dim=-1, keepdim=True)
        return out

    def gate(self, shape, mean, spread):
        return torch.sigmoid(torch.randn(shape, generator=self.g, device="cuda") * spread + mean)

    def below(self, n, shape):
        return torch.randint(0, n, shape, generator=self.g, device="cuda")

    def permutation(self, n):
        return torch.randperm(n, generator=self.g, device="cuda").to(torch.int32)


def _store(s, slots, n, H, d, r):
    """A store of `slots` slots and its contents; the handle is what a user's program allocates once."""
    data = r.normal((slots, n, H, d, d), scale=0.02)
    if own:
        import paper_2506_09316_b200 as dsla
        s["st"] = dsla.dsla_state_alloc_n(slots, n, H, d, d)
        s["st"].tensor.copy_(data)
        data = s["st"].tensor
    s["state"] = data


def prepare(case, seed):
    r = _Draw(seed)
    s = dict(case)
    if case["kind"] == "qk":
        T, H, Hk, d, rot, dtype = case["T"], case["H"], case["Hk"], case["d"], case["rot"], DTYPES[case["dtype"]]
        fused = r.normal((T, H + 2 * Hk, d), dtype)                    # rows of [q | k | v] as one projection leaves them
        s["q"], s["k"] = fused[:, :H], fused[:, H:H + Hk]
        s["wq"], s["wk"] = (1 + r.normal((d,), scale=0.1) for _ in range(2))
        first = int(r.below(100000, (1,)))                              # a prompt that continues a long context
        s["positions"] = torch.arange(first, first + T, dtype=torch.int32, device="cuda") if rot else None
        s["inv_freq"] = (1.0 / THETA ** (torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)).float() if rot else None
        s["q_out"], s["k_out"] = (torch.empty((T, h, d), dtype=dtype, device="cuda") for h in (H, Hk))
        return s
    if case["kind"] == "copy":
        moves, frees, H, d, n = case["moves"], case["frees"], case["H"], case["d"], case["n"]
        slots = (1 if case["fork"] else moves) + moves + frees
        at = r.permutation(slots)
        lead = 1 if case["fork"] else moves                             # sources, then targets, then what is freed
        s["src"] = torch.cat([at[:lead].expand(moves) if case["fork"] else at[:lead], torch.full((frees,), -1, dtype=torch.int32, device="cuda")])
        s["dst"] = at[lead:].contiguous()
        _store(s, slots, n, H, d, r)
        return s
    H, Hqk, d, dtype = case["H"], case["H"] // case["group"], case["d"], DTYPES[case["dtype"]]
    lens = _lengths(case) if case["kind"] == "prefill" else None
    rows = sum(lens) if lens else case["B"]
    seqs = len(lens) if lens else case["B"]
    s["q"], s["k"], s["v"] = r.unit((rows, Hqk, d), dtype), r.unit((rows, Hqk, d), dtype), r.normal((rows, H, d), dtype)
    s["gate"], s["beta"] = r.gate((rows, H), 4.0, 1.5), r.gate((rows, H), 0.5, 1.0)
    s["scale"] = 1.0 / math.sqrt(d)
    s["o"] = torch.zeros((rows, H, d), dtype=dtype, device="cuda")
    s["slots"] = r.permutation(seqs) if seqs > 1 else None
    _store(s, seqs, 1, H, d, r)
    if case["kind"] == "decode":
        s["mask"] = None
        if case["masked"]:
            s["mask"] = (r.below(4, (seqs,)) > 0).to(torch.uint8)       # rows of this layer's; every eighth slot is padding
            if s["slots"] is not None:
                s["slots"] = torch.where(r.below(8, (seqs,)) == 0, -1, s["slots"])
        return s
    s["longest"], s["lens"] = max(lens), lens
    s["cu"] = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32) if seqs > 1 else None
    s["ws"] = None
    if own:
        import paper_2506_09316_b200 as dsla
        need = dsla.dsla_delta_prefill_workspace_bytes(rows, seqs, s["longest"], H, d, dtype, H_qk=Hqk, dense_T=None if seqs > 1 else s["longest"])
        s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------------------------------

def _rotated(x, cos, sin, rot, interleaved):
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_qk(s):
    rot = s["rot"]
    if rot:
        angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
        cos, sin = angle.cos().float(), angle.sin().float()
    out = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        y = x.float()
        square = (y * y).mean(-1, keepdim=True) if s["norm"] == "rms" else (y * y).sum(-1, keepdim=True)
        y = y * torch.rsqrt(square + EPS) * w
        out.append((_rotated(y, cos, sin, rot, s["interleaved"]) if rot else y).to(x.dtype))
    return tuple(out)


def _plain_copy(s):
    state, src, dst = s["state"], s["src"].long(), s["dst"].long()
    got = state.index_select(0, src.clamp_min(0))
    state.index_copy_(0, dst, torch.where((src < 0)[:, None, None, None, None], 0.0, got))
    return state


def _plain_decode(s):
    H, B, group = s["H"], s["B"], s["group"]
    q, k = (x.float().repeat_interleave(group, 1) for x in (s["q"], s["k"]))
    slots = s["slots"].long() if s["slots"] is not None else torch.arange(B, device="cuda")
    state, at = s["state"], slots.clamp_min(0)
    S = state[at, 0] * s["gate"][:, :, None, None]
    u = s["beta"][:, :, None] * (s["v"].float() - torch.einsum("bhk,bhkv->bhv", k, S))
    S = S + k[..., None] * u[:, :, None]
    o = (s["scale"] * torch.einsum("bhk,bhkv->bhv", q, S)).to(s["o"].dtype)
    live = slots >= 0
    if s["mask"] is not None:
        o = torch.where((s["mask"] == 0)[:, None, None], s["o"], torch.where(live[:, None, None], o, 0.0))
        live = live & (s["mask"] != 0)
        state[slots[live], 0] = S[live]
    else:
        state[at, 0] = S
    s["o"].copy_(o)
    return s["o"], state


def _plain_prefill(s):
    """Chunks of CHUNK tokens.  With D[j, i] the product of the gates i+1..j and G[j] that of the gates up to j (both within the chunk),
    U = (I + tril(beta_j D[j, i] k_j.k_i, -1))^-1 beta (V - G K S),  O = scale (G Q S + tril(Q K^T D) U),  S <- G[end] S + K^T (D[end] U)."""
    H, d, group = s["H"], s["d"], s["group"]
    lens = torch.tensor(s["lens"], device="cuda")
    N, chunks = len(s["lens"]), max(1, -(-s["longest"] // CHUNK))
    first = lens.cumsum(0) - lens
    token = torch.arange(chunks * CHUNK, device="cuda")
    live = token < lens[:, None]                                            # [N, tokens]
    at = torch.where(live, first[:, None] + token, 0)
    to = lambda x: x[at].transpose(1, 2).unflatten(2, (chunks, CHUNK))      # [N, heads, chunks, CHUNK, ...]  # noqa: E731
    here = live.view(N, 1, chunks, CHUNK)
    gate = torch.where(here, to(s["gate"]), 1.0)
    beta = torch.where(here, to(s["beta"]), 0.0)
    K = torch.where(here[..., None], to(s["k"]).float(), 0.0).repeat_interleave(group, 1)
    Q = to(s["q"]).float().repeat_interleave(group, 1)
    V = torch.where(here[..., None], to(s["v"]).float(), 0.0)
    lower = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda").tril()
    L = torch.log(gate.double()).cumsum(-1)
    D = torch.where(lower, torch.exp(L[..., :, None] - L[..., None, :]), 0.0).float()
    G, W = torch.exp(L).float(), torch.exp(L[..., -1:] - L).float()
    A = torch.where(lower.tril(-1), beta[..., None] * D * (K @ K.transpose(-1, -2)), 0.0)
    P = (Q @ K.transpose(-1, -2)) * D
    right = torch.cat([beta[..., None] * V, (beta * G)[..., None] * K], -1)
    right = torch.linalg.solve_triangular(A, right, upper=False, unitriangular=True)
    U0, X = right[..., :d], right[..., d:]
    QG, KW = Q * G[..., None], (K * W[..., None]).transpose(-1, -2)
    slots = s["slots"].long() if s["slots"] is not None else torch.arange(N, device="cuda")
    S = s["state"][slots, 0] if s["resume"] else torch.zeros((N, H, d, d), device="cuda")
    O = torch.empty((N, H, chunks, CHUNK, d), device="cuda")
    for c in range(chunks):
        U = U0[:, :, c] - X[:, :, c] @ S
        O[:, :, c] = QG[:, :, c] @ S + P[:, :, c] @ U
        S = G[:, :, c, -1, None, None] * S + KW[:, :, c] @ U
    s["state"][slots, 0] = S
    s["o"].copy_((s["scale"] * O).flatten(2, 3).transpose(1, 2)[live])
    return s["o"], s["state"]


def run(s):
    kind = s["kind"]
    if not own:
        return {"qk": _plain_qk, "copy": _plain_copy, "decode": _plain_decode, "prefill": _plain_prefill}[kind](s)
    import paper_2506_09316_b200 as dsla
    if kind == "qk":
        return dsla.dsla_qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], positions=s["positions"], inv_freq=s["inv_freq"], q_out=s["q_out"],
                                      k_out=s["k_out"], eps=EPS, norm=s["norm"], interleaved=s["interleaved"])
    if kind == "copy":
        dsla.dsla_state_copy(s["st"], s["src"], s["dst"])
        return s["state"]
    if kind == "decode":
        o = dsla.dsla_delta_decode_step(s["q"], s["k"], s["v"], s["gate"], s["beta"], s["st"], o=s["o"], slots=s["slots"], scale=s["scale"],
                                        row_mask=s["mask"])
    else:
        o = dsla.dsla_delta_prefill(s["q"], s["k"], s["v"], s["gate"], s["beta"], s["st"], o=s["o"], cu_seqlens=s["cu"], slots=s["slots"],
                                    max_seqlen=s["longest"], scale=s["scale"], use_initial_state=s["resume"], workspace=s["ws"])
    return o, s["state"]


# ---- the work and the exact results -----------------------------------------------------------------------------------------------------------

def work(case):
    """Inputs once, outputs once; states read where a call starts from them and written once.  Operations of the recurrence: for each token
    and value head a product with the state, a rank-1 update and a readout."""
    if case["kind"] == "qk":
        values = case["T"] * (case["H"] + case["Hk"]) * case["d"]
        return {"bytes": 2 * values * (2 if case["dtype"] == "bf16" else 4) + 8 * case["d"] + 4 * case["T"], "flops": 10.0 * values}
    if case["kind"] == "copy":
        slot = 4 * case["n"] * case["H"] * case["d"] ** 2
        return {"bytes": slot * ((1 if case["fork"] else case["moves"]) + case["moves"] + case["frees"]), "flops": 0}
    H, d, es = case["H"], case["d"], 2 if case["dtype"] == "bf16" else 4
    token = (2 * (H // case["group"]) + 2 * H) * d * es + 8 * H
    if case["kind"] == "decode":
        rows = case["B"] * (0.66 if case["masked"] else 1.0)
        return {"bytes": rows * (token + 8 * H * d * d), "flops": 6.0 * rows * H * d * d}
    lens = _lengths(case)
    return {"bytes": sum(lens) * token + len(lens) * 4 * H * d * d * (2 if case["resume"] else 1), "flops": 6.0 * sum(lens) * H * d * d}


def exact(case, seed):
    s = prepare(case, seed)
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if case["kind"] == "qk":
        res = []
        for name, w in (("q", "wq"), ("k", "wk")):
            x = wide[name]
            total = torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2
            x = x / torch.sqrt((total / case["d"] if case["norm"] == "rms" else total) + EPS) * wide[w]
            if case["rot"]:
                half = case["rot"] // 2
                turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * wide["inv_freq"])[:, None]
                first = torch.arange(half, device="cuda") * (2 if case["interleaved"] else 1)
                second = first + (1 if case["interleaved"] else half)
                z = torch.complex(x[..., first], x[..., second]) * turn
                x = x.clone()
                x[..., first], x[..., second] = z.real, z.imag
            res.append(x)
        return tuple(res)
    state = wide["state"]
    if case["kind"] == "copy":
        new = state.clone()
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            new[b] = state[a] if a >= 0 else 0.0
        return new
    group, H, d = case["group"], case["H"], case["d"]
    lens = _lengths(case) if case["kind"] == "prefill" else [1] * case["B"]
    if max(lens) * len(lens) * H * d * d > 1 << 37:
        return None
    slots = s["slots"].tolist() if s["slots"] is not None else list(range(len(lens)))
    skip = [m == 0 for m in s["mask"].tolist()] if case["kind"] == "decode" and s["mask"] is not None else [False] * len(lens)
    o = wide["o"]
    begin = [sum(lens[:i]) for i in range(len(lens))]
    order = sorted((i for i in range(len(lens)) if slots[i] >= 0 and not skip[i]), key=lambda i: -lens[i])      # longest first: the live ones lead
    if not order:
        return o, state
    where = torch.tensor([slots[i] for i in order], device="cuda")
    S = state[where, 0]
    if case["kind"] == "prefill" and not case["resume"]:
        S = torch.zeros_like(S)
    starts = torch.tensor([begin[i] for i in order], device="cuda")
    head = torch.arange(H, device="cuda") // group
    ends = [lens[i] for i in order]
    n = len(order)
    for t in range(ends[0]):
        while ends[n - 1] <= t:
            n -= 1
        at = starts[:n] + t
        k, q = s["k"][at][:, head].double(), s["q"][at][:, head].double()
        live = S[:n].mul_(s["gate"][at].double()[..., None, None])
        miss = s["v"][at].double() - torch.matmul(k[..., None, :], live)[..., 0, :]
        live.add_(k[..., :, None] * (s["beta"][at].double()[..., None] * miss)[..., None, :])
        o[at] = s["scale"] * torch.matmul(q[..., None, :], live)[..., 0, :]
    state[where, 0] = S
    return o, state
