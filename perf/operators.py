"""Measured cases of attention's neighbours: norm and rotation of queries and keys, and attention over a paged cache.

A case is a dict of plain values; ``listed()`` gives the fixed ones, ``draw(rng)`` one more of the same ranges.
``prepare(case, seed)`` makes on the GPU what a program has in hand before the call, ``run(state)`` is one pass through an
operator, ``work(case)`` the bytes and operations a pass cannot do without and ``exact(case, seed)`` the outputs in 64 bits.

Kinds of passes:
  rotate       queries and keys of a fused activation: norm of each head, then the rotation by position (training, forward)
  rotate_grad  the gradients of that, those of the two norm weights among them
  append       new tokens' keys, normed and rotated, and values into a paged cache; their queries normed and rotated
  attend       attention of the new tokens over the paged cache, with the strided set of the training-time attention

``own`` is set from outside: false, ``run`` computes the plain forms; true, it calls the library.
"""
import math

import torch

own = False

EPS = 1e-6
BASE = 10000.0


# ------------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one sequence of 1024 tokens of GPT-2 small (12 heads of 64): the smallest training call
        _rotate("rotate", "rotate_one", tokens=1024, seq=1024),
        # 16 such sequences, the benchmark's batch
        _rotate("rotate", "rotate_batch", tokens=16384, seq=1024),
        # single precision, wide heads of which a part turns in neighbouring pairs, few key heads, positions far out, ragged rows
        _rotate("rotate", "rotate_fp32_far", dtype="fp32", tokens=2999, seq=997, heads=10, kv_heads=2, head_dim=80, rot_dim=48,
                interleaved=True, first=200000),
        # the gradients for one sequence and for 16 sequences of GPT-2 large (20 heads)
        _rotate("rotate_grad", "rotate_grad_one", tokens=1024, seq=1024),
        _rotate("rotate_grad", "rotate_grad_batch", tokens=16384, seq=1024, heads=20, kv_heads=20),
        # one token for each of 32 sequences: the append of a generation step
        _append("append_tokens", batch=32, new=(1, 1), length=(200, 4000)),
        # prompts of ragged length in pages of an odd size, more queries than keys, some rows of the buffer unused
        _append("append_prompts", batch=11, new=(37, 2000), length=(37, 4000), heads=20, kv_heads=4, page=24, spare=61),
        # one token for each of 8 sequences under the strided set: the smallest call
        _attend("attend_tokens_strided", batch=8, new=(1, 1), length=(300, 4000), stride=256),
        # generation over long ragged contexts, every earlier position attended, four key heads for twenty queries
        _attend("attend_tokens_long", batch=16, new=(1, 1), length=(1500, 32768), heads=20, kv_heads=4),
        # five draft tokens a sequence in pages of an odd size
        _attend("attend_drafts", batch=24, new=(3, 5), length=(100, 5000), heads=12, kv_heads=6, page=24),
        # chunks of prompts under the strided set
        _attend("attend_chunks_strided", batch=4, new=(512, 512), length=(2048, 8192), stride=256, page=64),
        # chunks of long prompts, every earlier position attended: the largest call
        _attend("attend_chunks_long", batch=3, new=(1000, 2048), length=(4000, 12000), page=64),
    ]


def _rotate(kind, name, tokens, seq, dtype="bf16", heads=12, kv_heads=12, head_dim=64, rot_dim=64, interleaved=False, norm=True,
            first=0):
    return dict(name=name, kind=kind, dtype=dtype, tokens=tokens, seq=seq, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                rot_dim=rot_dim, interleaved=interleaved, norm=norm, first=first)


def _append(name, batch, new, length, heads=12, kv_heads=12, head_dim=64, rot_dim=64, interleaved=False, norm=True, page=16,
            spare=0):
    return dict(name=name, kind="append", batch=batch, new_lo=new[0], new_hi=new[1], len_lo=length[0], len_hi=length[1],
                heads=heads, kv_heads=kv_heads, head_dim=head_dim, rot_dim=rot_dim, interleaved=interleaved, norm=norm,
                page=page, spare=spare)


def _attend(name, batch, new, length, heads=12, kv_heads=12, head_dim=64, stride=0, page=16, spare=0):
    """stride 0: every earlier position."""
    return dict(name=name, kind="attend", batch=batch, new_lo=new[0], new_hi=new[1], len_lo=length[0], len_hi=length[1],
                heads=heads, kv_heads=kv_heads, head_dim=head_dim, stride=stride, page=page, spare=spare)


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    """Query heads and key heads: as many of both, or several queries to a key."""
    kv = rng.randint(1, 20)
    return (kv, kv) if rng.random() < 0.5 else (min(40, kv * rng.randint(2, 8)) // kv * kv, kv)


def draw(rng):
    most = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("rotate", "rotate_grad", "append", "attend")}
    while True:
        case = _draw_one(rng)
        if _cost(case) <= most[case["kind"]]:
            del case["name"]
            return case


def _draw_one(rng):
    kind = rng.choice(["rotate", "rotate_grad", "append", "attend", "attend", "attend"])
    heads, kv = _heads(rng)
    page = rng.choice([16, 16, 32, 64, 64, 128, _log(rng, 3, 100)])
    if kind in ("rotate", "rotate_grad"):
        D = rng.choice([64, 64, 128, 8 * rng.randint(2, 32)])
        seq = _log(rng, 1, 4096)
        return _rotate(kind, "", tokens=_log(rng, 1, 20000), seq=seq, dtype=rng.choice(["bf16", "bf16", "fp32"]), heads=heads,
                       kv_heads=kv, head_dim=D, rot_dim=rng.choice([D // 16 * 16, 16 * rng.randint(0, D // 16)]),
                       interleaved=rng.random() < 0.5, norm=rng.random() < 0.8, first=rng.choice([0, 0, _log(rng, 1, 500000)]))
    one = rng.random() < 0.5
    batch = _log(rng, 1, 64)
    new_hi = 1 if one else _log(rng, 2, 2048)
    new_lo = rng.randint(max(1, new_hi // 4), new_hi)
    len_hi = _log(rng, max(new_hi, 16), 32768)
    len_lo = rng.randint(min(new_hi, len_hi), len_hi)
    spare = rng.choice([0, 0, rng.randint(1, 70)])
    D = rng.choice([64, 64, 64, 128])
    if kind == "append":
        return _append("", batch, (new_lo, new_hi), (len_lo, len_hi), heads, kv, D, rng.choice([D, D // 2]), rng.random() < 0.5,
                       rng.random() < 0.5, page, spare)
    return _attend("", batch, (new_lo, new_hi), (len_lo, len_hi), heads, kv, D,
                   rng.choice([0, 0, 64, 128, 128, 256, 256, 512, 1024]), page, spare)


def _cost(case):
    """Seconds at 6 TB/s and 1 PFLOP/s: only for keeping drawn cases in bounds."""
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / 1e15


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly apart in their logarithm, in a mixed order."""
    if n == 1:
        return [hi]
    step = next(k for k in (7, 5, 3, 2, 1) if math.gcd(k, n) == 1)
    v = [int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]
    return [v[(step * i + n // 2) % n] for i in range(n)]


def _lengths(case):
    """New tokens and length (new tokens included) of every sequence."""
    new = _spread(case["new_lo"], case["new_hi"], case["batch"])
    length = _spread(case["len_lo"], case["len_hi"], case["batch"])
    return new, [max(a, b) for a, b in zip(new, length)]


# ------------------------------------------------------------------------------------------------------------ the inputs
class _State:
    pass


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(0x51524F54 + 7919 * seed)


def _normal(shape, dtype, g, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _unit(shape, g):
    """Rows as they leave the norm: mean square one, times a weight a column."""
    x = _normal(shape, torch.float32, g)
    x *= torch.rsqrt((x * x).mean(-1, keepdim=True)) * (0.7 + 0.8 * torch.rand(shape[-1], generator=g, device="cuda"))
    return x.to(torch.bfloat16)


def _rotation(s, case, g):
    D, half = case["head_dim"], case["rot_dim"] // 2
    s.inv_freq = (BASE ** (-torch.arange(half, dtype=torch.float64, device="cuda") / max(half, 1))).float()
    s.gamma_q = s.gamma_k = None
    if case["norm"]:
        s.gamma_q = 0.7 + 0.8 * torch.rand(D, generator=g, device="cuda")
        s.gamma_k = 0.7 + 0.8 * torch.rand(D, generator=g, device="cuda")
    if own:
        import paper_2408_11746_b200 as mst
        s.rot = mst.Rotation(D, case["rot_dim"], s.inv_freq, s.gamma_q, s.gamma_k, EPS, case["interleaved"])


def prepare(case, seed):
    g = _generator(seed)
    s = _State()
    s.case, s.kind = case, case["kind"]
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    if s.kind in ("rotate", "rotate_grad"):
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        T = case["tokens"]
        s.qkv = _normal((T, (H + 2 * G) * D), dtype, g, 1.5)      # the fused activation: queries, keys, values
        s.positions = None
        if case["first"]:
            s.positions = (case["first"] + torch.arange(T, device="cuda") % case["seq"]).to(torch.int32)
        _rotation(s, case, g)
        s.qk = torch.zeros((T, (H + G) * D), dtype=dtype, device="cuda")
        if s.kind == "rotate_grad":
            s.dqk = _normal((T, (H + G) * D), dtype, g)
            s.dgamma_q = torch.zeros(D, device="cuda") if case["norm"] else None
            s.dgamma_k = torch.zeros(D, device="cuda") if case["norm"] else None
            if own:
                import paper_2408_11746_b200 as mst
                s.ws = torch.empty(max(1, mst.mst_qk_norm_rotate_bwd_workspace(s.rot, T)), dtype=torch.uint8, device="cuda")
        return s
    new, length = _lengths(case)
    B, page = case["batch"], case["page"]
    s.new, s.length = new, length
    s.tokens = sum(new) + case["spare"]
    first = [0]
    for n in new:
        first.append(first[-1] + n)
    s.host_first = first
    s.first = torch.tensor(first, dtype=torch.int32, device="cuda")
    s.len = torch.tensor(length, dtype=torch.int32, device="cuda")
    pages = [(n + page - 1) // page for n in length]
    s.pages = pages
    total = sum(pages)
    order = torch.randperm(total + 3, generator=g, device="cuda").to(torch.int32)
    s.table = torch.full((B, max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        s.table[b, :n] = order[at:at + n]
        at += n
    s.K = _unit((total + 3, page, G, D), g)
    s.V = _normal((total + 3, page, G, D), torch.bfloat16, g)
    if own:
        import paper_2408_11746_b200 as mst
        s.cache = mst.PagedCache(s.K, s.V)
        s.batch = mst.PagedBatch(s.first, s.len, s.table, s.tokens, max(new), max(length))
    if s.kind == "append":
        s.qkv = _normal((s.tokens, (H + 2 * G) * D), torch.bfloat16, g, 1.5)
        _rotation(s, case, g)
        s.q = torch.zeros((s.tokens, H * D), dtype=torch.bfloat16, device="cuda")
        return s
    s.q = _unit((s.tokens, H, D), g).view(s.tokens, H * D)
    s.stride = case["stride"] or 1 << 30
    s.out = torch.zeros((s.tokens, H * D), dtype=torch.bfloat16, device="cuda")
    s.lse = torch.zeros((H, s.tokens), device="cuda")
    if own:
        import paper_2408_11746_b200 as mst
        s.ws = torch.empty(max(1, mst.mst_paged_attention_workspace(s.cache, s.batch, H, s.stride)), dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------------------------------------------------- the plain forms
def _cos_sin(positions, inv_freq):
    a = positions.double()[:, None] * inv_freq.double()[None, :]
    return torch.cos(a).float()[:, None, :], torch.sin(a).float()[:, None, :]


def _turn(x, cos, sin, rot, interleaved):
    """x [tokens, heads, D] fp32: its first `rot` columns turned by the angles, pair by pair."""
    if rot == 0:
        return x
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2] = a * cos - b * sin
        y[..., 1:rot:2] = a * sin + b * cos
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2] = a * cos - b * sin
        y[..., rot // 2:rot] = a * sin + b * cos
    return y


def _norm_turn(x, gamma, cos, sin, case):
    x = x.float()
    if gamma is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma
    return _turn(x, cos, sin, case["rot_dim"], case["interleaved"])


def _norm_turn_grad(x, dy, gamma, cos, sin, case):
    x, dz = x.float(), _turn(dy.float(), cos, -sin, case["rot_dim"], case["interleaved"])
    if gamma is None:
        return dz, None
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dgamma = (dz * n).sum((0, 1), dtype=torch.float64).float()
    dn = dz * gamma
    return r * (dn - n * (dn * n).mean(-1, keepdim=True)), dgamma


def _plain_rotate(s):
    c = s.case
    T, H, G, D = c["tokens"], c["heads"], c["kv_heads"], c["head_dim"]
    positions = s.positions if s.positions is not None else torch.arange(T, device="cuda") % c["seq"]
    cos, sin = _cos_sin(positions, s.inv_freq)
    x = s.qkv[:, :(H + G) * D].reshape(T, H + G, D)
    if s.kind == "rotate":
        y = s.qk.view(T, H + G, D)
        y[:, :H] = _norm_turn(x[:, :H], s.gamma_q, cos, sin, c).to(y.dtype)
        y[:, H:] = _norm_turn(x[:, H:], s.gamma_k, cos, sin, c).to(y.dtype)
        return [s.qk]
    dy = s.dqk.view(T, H + G, D)
    dx = s.qk.view(T, H + G, D)
    dq, s.dgamma_q = _norm_turn_grad(x[:, :H], dy[:, :H], s.gamma_q, cos, sin, c)
    dk, s.dgamma_k = _norm_turn_grad(x[:, H:], dy[:, H:], s.gamma_k, cos, sin, c)
    dx[:, :H] = dq.to(dx.dtype)
    dx[:, H:] = dk.to(dx.dtype)
    return [s.qk, s.dgamma_q, s.dgamma_k]


def _plain_append(s):
    c = s.case
    H, G, D, page = c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    n = s.host_first[-1]
    token = torch.arange(n, device="cuda")
    b = torch.bucketize(token, s.first[1:].long(), right=True)
    positions = s.len.long()[b] - s.first.long()[b + 1] + token
    cos, sin = _cos_sin(positions, s.inv_freq)
    x = s.qkv[:n].view(n, H + 2 * G, D)
    s.q.view(-1, H, D)[:n] = _norm_turn(x[:, :H], s.gamma_q, cos, sin, c).to(torch.bfloat16)
    where = s.table[b, positions // page].long()
    s.K[where, positions % page] = _norm_turn(x[:, H:H + G], s.gamma_k, cos, sin, c).to(torch.bfloat16)
    s.V[where, positions % page] = x[:, H + G:]
    return [s.q, s.K, s.V]


def _plain_attend(s):
    c = s.case
    H, G, D = c["heads"], c["kv_heads"], c["head_dim"]
    for b, (n, length) in enumerate(zip(s.new, s.length)):
        t0 = s.host_first[b]
        which = s.table[b, :s.pages[b]].long()
        k = s.K[which].view(-1, G, D)[:length].float().permute(1, 2, 0)          # [G, D, length]
        v = s.V[which].view(-1, G, D)[:length].float().transpose(0, 1)           # [G, length, D]
        q = s.q[t0:t0 + n].view(n, G, H // G, D).float().permute(1, 2, 0, 3)     # [G, H / G, n, D]
        back = torch.arange(length - n, length, device="cuda")[:, None] - torch.arange(length, device="cuda")[None, :]
        keep = (back >= 0) & ((back < s.stride) | (back % s.stride == 0))
        x = torch.matmul(q.reshape(G, H // G * n, D), k).view(G, H // G, n, length) / math.sqrt(D)
        x = x.masked_fill_(~keep, -math.inf)
        top = x.amax(-1, keepdim=True)
        p = torch.exp(x.sub_(top))
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(G, H // G * n, length), v).view(G, H // G, n, D) / total
        s.out[t0:t0 + n] = o.permute(2, 0, 1, 3).reshape(n, H * D).to(torch.bfloat16)
        s.lse[:, t0:t0 + n] = (top + torch.log(total)).view(H, n)
    return [s.out, s.lse]


# -------------------------------------------------------------------------------------------------------------- one pass
def run(s):
    c = s.case
    if not own:
        return {"rotate": _plain_rotate, "rotate_grad": _plain_rotate, "append": _plain_append, "attend": _plain_attend}[s.kind](s)
    import paper_2408_11746_b200 as mst
    H, G, D = c["heads"], c["kv_heads"], c["head_dim"]
    if s.kind == "attend":
        mst.mst_paged_attention(s.cache, s.batch, H, s.stride, s.q, H * D, s.out, H * D, s.lse, s.ws)
        return [s.out, s.lse]
    x, e = s.qkv.data_ptr(), s.qkv.element_size()
    ld = s.qkv.stride(0)
    if s.kind == "append":
        mst.mst_paged_append(s.cache, s.batch, s.rot, H, x, x + H * D * e, x + (H + G) * D * e, ld, s.q, H * D)
        return [s.q, s.K, s.V]
    dtype = mst.MST_BF16 if c["dtype"] == "bf16" else mst.MST_F32
    y, ldo = s.qk.data_ptr(), s.qk.stride(0)
    if s.kind == "rotate":
        mst.mst_qk_norm_rotate_fwd(s.rot, dtype, c["tokens"], c["seq"], s.positions, H, G, x, x + H * D * e, ld, y, y + H * D * e,
                                   ldo)
        return [s.qk]
    d = s.dqk.data_ptr()
    mst.mst_qk_norm_rotate_bwd(s.rot, dtype, c["tokens"], c["seq"], s.positions, H, G, x, x + H * D * e, ld, d, d + H * D * e,
                               s.dqk.stride(0), y, y + H * D * e, ldo, s.dgamma_q, s.dgamma_k, s.ws)
    return [s.qk, s.dgamma_q, s.dgamma_k]


# --------------------------------------------------------------------------------------------------------- necessary work
def _seen(n, length, stride):
    """Positions that some of the last n of `length` attend to."""
    if stride == 0 or n >= stride:
        return length
    window = min(length, stride + n - 1)
    before = length - window                     # positions 0 .. before - 1; of each `stride` of them n are seen
    return window + sum(1 for j in range(before) if (length - 1 - j) % stride < n)


def _pairs(n, length, stride):
    if stride == 0:
        return n * (2 * length - n + 1) // 2
    return sum(min(i + 1, stride) + i // stride for i in range(length - n, length))


def work(case):
    kind, H, G, D = case["kind"], case["heads"], case["kv_heads"], case["head_dim"]
    if kind in ("rotate", "rotate_grad"):
        e = 2 if case["dtype"] == "bf16" else 4
        values = case["tokens"] * (H + G) * D
        positions = 4 * case["tokens"] if case["first"] else 0
        grad = kind == "rotate_grad"
        arrays = 2 if not grad else 3 if case["norm"] else 2
        return {"bytes": float(arrays * e * values + positions + 2 * case["rot_dim"] + (8 * D * (2 if grad else 1) if case["norm"] else 0)),
                "flops": float(values * ((16 if grad else 7) if case["norm"] else 3))}
    new, length = _lengths(case)
    n = sum(new)
    tables = 4 * sum((a + case["page"] - 1) // case["page"] for a in length) + 8 * case["batch"]
    if kind == "append":
        return {"bytes": float(2 * 2 * n * (H + 2 * G) * D + 8 * case["batch"] + 4 * n + 2 * case["rot_dim"]),
                "flops": float(n * (H + G) * D * (7 if case["norm"] else 3))}
    seen = sum(_seen(a, b, case["stride"]) for a, b in zip(new, length))
    pairs = sum(_pairs(a, b, case["stride"]) for a, b in zip(new, length))
    return {"bytes": float(2 * 2 * n * H * D + 4 * n * H + 2 * 2 * seen * G * D + tables), "flops": float(4 * D * H * pairs)}


# ------------------------------------------------------------------------------------------------------------- in 64 bits
def _exact_turn(x, gamma, positions, inv_freq, case):
    """x [tokens, heads, D] float64: as complex numbers, one a pair, times exp(i angle)."""
    if gamma is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS) * gamma.double()
    rot = case["rot_dim"]
    if rot == 0:
        return x
    angle = torch.outer(positions.double(), inv_freq.double())[:, None, :]
    spin = torch.polar(torch.ones_like(angle), angle)
    if case["interleaved"]:
        z = torch.view_as_complex(x[..., :rot].unflatten(-1, (rot // 2, 2)).contiguous()) * spin
        return torch.cat([torch.view_as_real(z).flatten(-2), x[..., rot:]], -1)
    z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * spin
    return torch.cat([z.real, z.imag, x[..., rot:]], -1)


def _exact_rotate(s):
    """The gradients come out of the forward definition by differentiation."""
    c = s.case
    T, H, G, D = c["tokens"], c["heads"], c["kv_heads"], c["head_dim"]
    at = torch.arange(T, device="cuda") % c["seq"] if s.positions is None else s.positions
    grad = s.kind == "rotate_grad"
    out, weights = [], []
    for lo, n, gamma in ((0, H, s.gamma_q), (H, G, s.gamma_k)):
        x = s.qkv[:, lo * D:(lo + n) * D].double().view(T, n, D).requires_grad_(grad)
        w = gamma.double().requires_grad_(grad) if gamma is not None else None
        y = _exact_turn(x, w, at, s.inv_freq, c)
        if grad:
            y.backward(s.dqk[:, lo * D:(lo + n) * D].double().view(T, n, D))
            y = x.grad
            weights.append(w.grad if w is not None else None)
        out.append(y.detach().reshape(T, n * D))
    return [torch.cat(out, 1)] + weights


def _exact_append(s):
    c = s.case
    H, G, D, page = c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    q, K, V = s.q.double(), s.K.double(), s.V.double()
    table = s.table.tolist()
    for b, (n, length) in enumerate(zip(s.new, s.length)):
        t0 = s.host_first[b]
        at = torch.arange(length - n, length, device="cuda")
        x = s.qkv[t0:t0 + n].double().view(n, H + 2 * G, D)
        q[t0:t0 + n] = _exact_turn(x[:, :H], s.gamma_q, at, s.inv_freq, c).reshape(n, H * D)
        k = _exact_turn(x[:, H:H + G], s.gamma_k, at, s.inv_freq, c)
        for p in range((length - n) // page, (length - 1) // page + 1):
            lo, hi = max(p * page, length - n), min((p + 1) * page, length)
            K[table[b][p], lo - p * page:hi - p * page] = k[lo - (length - n):hi - (length - n)]
            V[table[b][p], lo - p * page:hi - p * page] = x[lo - (length - n):hi - (length - n), H + G:]
    return [q, K, V]


def _exact_attend(s):
    c = s.case
    H, G, D = c["heads"], c["kv_heads"], c["head_dim"]
    out, lse = s.out.double(), s.lse.double()
    for b, (n, length) in enumerate(zip(s.new, s.length)):
        t0 = s.host_first[b]
        j = torch.arange(length, device="cuda")
        where, inside = s.table[b].long()[j // c["page"]], j % c["page"]
        i = torch.arange(length - n, length, device="cuda")[:, None]
        out_of_set = (j > i) | ((i - j >= s.stride) & ((i - j).remainder(s.stride) != 0))
        for h in range(H):
            k, v = s.K[where, inside, h * G // H].double(), s.V[where, inside, h * G // H].double()
            x = s.q[t0:t0 + n, h * D:(h + 1) * D].double() @ k.T * D ** -0.5
            x = torch.where(out_of_set, -math.inf, x)
            z = torch.logsumexp(x, 1)
            lse[h, t0:t0 + n] = z
            out[t0:t0 + n, h * D:(h + 1) * D] = torch.exp(x - z[:, None]) @ v
    return [out, lse]


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "rotate_grad": _exact_rotate, "append": _exact_append, "attend": _exact_attend}[s.kind](s)
