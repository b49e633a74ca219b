"""Norm and rotation of queries and keys through the C ABI, forward and gradients, against the plain definition in 64 bits.

Tolerances.  A result of b bits is rounded once (half a step, eps / 2 of its value: 2^-8 bf16, 2^-24 fp32).  Before that everything is fp32: a
sum of D <= 256 squares in a chain of 8 + 5 additions, one reciprocal root (2 ulp), three products and one sum a value, sine and cosine of an
angle that is off by at most 2^-23 (reduced in fp64, then rounded) with 2 ulp: less than 24 roundings of 2^-24 = 1.5e-6 of the pair's
length; 2e-6 is allowed.  The gradients have two such chains one behind the other and a difference: 4e-6 of the sum of their terms' sizes.  A weight's gradient adds
up one term a token and head: at most 256 additions one after the other for the sizes here, 256 * 2^-24 = 1.5e-5 of the sum of sizes, and 4e-6 a term.
"""
import numpy as np
import pytest

from oracle import rotation

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    import paper_2408_11746_b200 as mst
    from gpu_util import dev, host

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
EPS = 1e-5


class Case:
    """A fused activation [tokens, ld] with heads_q + heads_k heads, and all that belongs to it; on the host in float64, bf16-exact where bf16."""

    def __init__(self, tokens, hq, hk, D, rot, interleaved=False, dtype="bf16", norm="qk", seq=7, first=None, pad=0, seed=0):
        g = torch.Generator().manual_seed(1000 + seed)
        self.tokens, self.hq, self.hk, self.D, self.rot, self.inter, self.dtype, self.seq, self.pad = tokens, hq, hk, D, rot, interleaved, dtype, seq, pad
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.code = 1 if dtype == "bf16" else 0
        self.width = (hq + hk) * D
        rnd = lambda *s: torch.randn(*s, generator=g).to(self.tdt)
        self.x, self.dy = rnd(tokens, self.width), rnd(tokens, self.width)
        self.inv_freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))
        self.inv_freq = self.inv_freq.float()
        w = 0.5 + torch.rand(2, D, generator=g)
        self.gamma = [w[0] if "q" in norm else None, w[1] if "k" in norm else None]
        self.pos = torch.arange(tokens) % seq if first is None else first + torch.randint(0, 1000, (tokens,), generator=g)
        self.positions = None if first is None else self.pos.to(torch.int32).to(dev())
        up = lambda t: None if t is None else t.to(dev())
        self.dev_freq, self.dev_gamma = up(self.inv_freq), [up(t) for t in self.gamma]
        self.rotation = mst.Rotation(D, rot, self.dev_freq, *self.dev_gamma, EPS, interleaved)

    def padded(self, t=None):
        b = torch.full((self.tokens, self.width + self.pad), float("nan"), dtype=self.tdt, device=dev())
        if t is not None:
            b[:, : self.width] = t.to(dev())
        return b

    def at(self, t):
        """addresses of the queries and the keys"""
        return t.data_ptr(), t.data_ptr() + self.hq * self.D * t.element_size()

    def forward(self, src, dst, stream=None):
        mst.mst_qk_norm_rotate_fwd(self.rotation, self.code, self.tokens, self.seq, self.positions, self.hq, self.hk, *self.at(src), src.stride(0),
                                   *self.at(dst), dst.stride(0), stream=stream)

    def backward(self, x, dy, dx, weights=True, stream=None, out=None):
        dg = out if out is not None else [torch.full((self.D,), float("nan"), device=dev()) if weights and w is not None else None for w in self.gamma]
        n = mst.mst_qk_norm_rotate_bwd_workspace(self.rotation, self.tokens)
        ws = torch.full((max(n, 1),), 0xFF, dtype=torch.uint8, device=dev())
        mst.mst_qk_norm_rotate_bwd(self.rotation, self.code, self.tokens, self.seq, self.positions, self.hq, self.hk, *self.at(x), x.stride(0),
                                   *self.at(dy), dy.stride(0), *self.at(dx), dx.stride(0), *dg, ws, stream=stream)
        return dg

    def sides(self, a):
        """(rows [tokens, heads, D], weight) of the queries and the keys"""
        a = host(a[:, : self.width]).astype(np.float64) if isinstance(a, torch.Tensor) else a
        a = a.reshape(self.tokens, self.hq + self.hk, self.D)
        return [(a[:, : self.hq], self.gamma[0]), (a[:, self.hq:], self.gamma[1])]

    def check_forward(self, got):
        for (y, w), (x, _) in zip(self.sides(got), self.sides(self.x)):
            w = None if w is None else w.numpy()
            ref = rotation.norm_rotate(x, w, self.pos.numpy(), self.inv_freq.numpy(), self.rot, self.inter, EPS)
            size = rotation.pair_sizes(rotation.norm_rotate(x, w, self.pos.numpy(), self.inv_freq.numpy(), 0, False, EPS), self.rot, self.inter)
            assert (np.abs(y - ref) <= HALF[self.dtype] * np.abs(ref) + 2e-6 * size + 1e-30).all()

    def check_backward(self, dx, dg):
        f = self.inv_freq.numpy()
        for (d, w), (x, _), (dy, _), g in zip(self.sides(dx), self.sides(self.x), self.sides(self.dy), dg):
            w = None if w is None else w.numpy().astype(np.float64)
            ref, ref_g = rotation.norm_rotate_bwd(x, w, self.pos.numpy(), f, self.rot, self.inter, EPS, dy)
            z = rotation.pair_sizes(dy, self.rot, self.inter)
            size = z
            if w is not None:
                r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
                size = r * (z * w + np.abs(x) * r * r * (z * w * np.abs(x)).mean(-1, keepdims=True))
            assert (np.abs(d - ref) <= HALF[self.dtype] * np.abs(ref) + 4e-6 * size + 1e-30).all()
            if g is not None:
                terms = (z * np.abs(x) * r).sum((0, 1))
                assert (np.abs(host(g) - ref_g) <= 2e-5 * terms + 1e-30).all()


SHAPES = [
    dict(tokens=64, hq=12, hk=12, D=64, rot=64),                                        # GPT-2 small
    dict(tokens=1, hq=1, hk=1, D=64, rot=64, seq=1),                                    # the least
    dict(tokens=37, hq=20, hk=4, D=64, rot=32, pad=8),                                  # groups, half of the values turn, rows apart
    dict(tokens=33, hq=5, hk=3, D=128, rot=128, first=500000),                          # odd counts, far positions
    dict(tokens=19, hq=3, hk=1, D=80, rot=48, first=0),                                 # ten lanes of sixteen
    dict(tokens=300, hq=2, hk=2, D=8, rot=0, seq=300),                                  # one lane a row, no rotation
    dict(tokens=50, hq=7, hk=7, D=16, rot=16),
    dict(tokens=21, hq=3, hk=2, D=40, rot=16),
    dict(tokens=9, hq=6, hk=2, D=256, rot=256, first=123456),
    dict(tokens=13, hq=4, hk=0, D=64, rot=64),                                          # one side only
    dict(tokens=13, hq=0, hk=4, D=96, rot=96),
    dict(tokens=3001, hq=3, hk=3, D=64, rot=64, seq=1024),                              # more tokens than warps run at once take in one go
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward_and_gradients(i, interleaved, dtype):
    c = Case(interleaved=interleaved, dtype=dtype, seed=i, **SHAPES[i])
    y = c.padded()
    c.forward(c.padded(c.x), y)
    dx = c.padded()
    dg = c.backward(c.padded(c.x), c.padded(c.dy), dx)
    torch.cuda.synchronize()
    c.check_forward(y)
    c.check_backward(dx, dg)
    if c.pad:
        assert torch.isnan(y[:, c.width:]).all() and torch.isnan(dx[:, c.width:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", ["", "q", "k"])
def test_sides_without_a_norm(norm, dtype):
    c = Case(41, 4, 2, 64, 64, dtype=dtype, norm=norm)
    y, dx = c.padded(), c.padded()
    c.forward(c.padded(c.x), y)
    dg = c.backward(c.padded(c.x), c.padded(c.dy), dx)
    torch.cuda.synchronize()
    c.check_forward(y)
    c.check_backward(dx, dg)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_and_without_weight_gradients(dtype):
    c = Case(130, 9, 3, 64, 64, dtype=dtype)
    y = c.padded(c.x)
    c.forward(y, y)
    a, b = c.padded(c.dy), c.padded(c.x)
    c.backward(c.padded(c.x), a, a, weights=False)       # over the upstream gradient
    c.backward(b, c.padded(c.dy), b, weights=False)      # over the input
    torch.cuda.synchronize()
    c.check_forward(y)
    c.check_backward(a, [None, None])
    assert torch.equal(a, b)


def test_results_repeat_and_do_not_depend_on_the_workspace():
    c = Case(1000, 12, 12, 64, 64)
    x, dy = c.padded(c.x), c.padded(c.dy)
    got = []
    for _ in range(3):
        dx = c.padded()
        got.append([dx] + c.backward(x, dy, dx))
    torch.cuda.synchronize()
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_far_positions_keep_their_angles():
    # 2^24 + 1 is no fp32 number; neighbouring positions differ by one radian in the fastest pair
    c = Case(4, 1, 1, 64, 64, dtype="f32", norm="", first=0)
    c.pos = torch.tensor([(1 << 24) + 1, (1 << 24) + 2, (1 << 30) + 3, -5])
    c.positions = c.pos.to(torch.int32).to(dev())
    y = c.padded()
    c.forward(c.padded(c.x), y)
    torch.cuda.synchronize()
    c.check_forward(y)


def test_extreme_rows():
    # zeros, the largest finite values whose squares still add up, infinities and NaN: a row stays on its own
    c = Case(6, 2, 2, 64, 64, seq=6)
    c.x[1] = 0
    c.x[2] = 1e17
    x = c.x.clone()
    x[3, 5], x[4, 70] = float("inf"), float("nan")
    y = c.padded()
    c.forward(c.padded(x), y)
    torch.cuda.synchronize()
    y = host(y).reshape(6, 4, 64)
    ok = np.ones((6, 4), bool)
    ok[3, 0] = ok[4, 1] = False
    assert np.isfinite(y[ok]).all() and np.isnan(y[3, 0]).any() and np.isnan(y[4, 1]).all()
    assert (y[1] == 0).all()
    ref = rotation.norm_rotate(c.x[2].double().numpy().reshape(1, 4, 64)[:, :2], c.gamma[0].numpy(), [2], c.inv_freq.numpy(), 64, False, EPS)
    np.testing.assert_allclose(y[2, :2], ref[0], rtol=0.01, atol=0.01)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 32])
def test_values_that_do_not_turn_stay_on_their_own(rot, interleaved):
    c = Case(5, 2, 1, 64, rot, interleaved, norm="")
    x, dy = c.x.clone(), c.dy.clone()
    x[1, 40], x[2, 64 + 63], dy[3, 50] = float("inf"), float("nan"), float("-inf")
    y, dx = c.padded(), c.padded()
    c.forward(c.padded(x), y)
    c.backward(c.padded(x), c.padded(dy), dx)
    torch.cuda.synchronize()
    y, dx = host(y), host(dx)
    assert np.isinf(y[1, 40]) and np.isnan(y[2, 127]) and np.isinf(dx[3, 50])
    assert np.isfinite(y).sum() == y.size - 2 and np.isfinite(dx).sum() == dx.size - 1


def test_streams_and_a_captured_graph():
    c = Case(200, 12, 12, 64, 64)
    x, dy = c.padded(c.x), c.padded(c.dy)
    want_y, want_dx = c.padded(), c.padded()
    c.forward(x, want_y)
    want_dg = c.backward(x, dy, want_dx)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y, dx = c.padded(), c.padded()
    dg = [torch.zeros(64, device=dev()) for _ in range(2)]
    torch.cuda.synchronize()
    c.forward(x, y, stream=side)
    c.backward(x, dy, dx, stream=side, out=dg)
    side.synchronize()
    assert torch.equal(y, want_y) and torch.equal(dx, want_dx) and all(torch.equal(a, b) for a, b in zip(dg, want_dg))
    graph = torch.cuda.CUDAGraph()
    n = mst.mst_qk_norm_rotate_bwd_workspace(c.rotation, c.tokens)
    ws = torch.empty(n, dtype=torch.uint8, device=dev())
    with torch.cuda.graph(graph):
        c.forward(x, y)
        mst.mst_qk_norm_rotate_bwd(c.rotation, c.code, c.tokens, c.seq, None, c.hq, c.hk, *c.at(x), x.stride(0), *c.at(dy), dy.stride(0),
                                   *c.at(dx), dx.stride(0), *dg, ws)
    for t in (y, dx, *dg):
        t.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want_y) and torch.equal(dx, want_dx) and all(torch.equal(a, b) for a, b in zip(dg, want_dg))


def test_pointers_of_the_host_are_refused():
    c = Case(4, 2, 2, 64, 64)
    x, y = c.padded(c.x), c.padded()
    for src, dst in ((c.x, y), (x, c.x), (c.x.pin_memory(), y)):
        with pytest.raises(mst.MstError) as e:
            c.forward(src, dst)
        assert e.value.status == 1
    bad = mst.Rotation(64, 64, c.inv_freq, *c.dev_gamma, EPS)
    with pytest.raises(mst.MstError) as e:
        mst.mst_qk_norm_rotate_fwd(bad, 1, 4, 4, None, 2, 2, *c.at(x), 256, *c.at(y), 256)
    assert e.value.status == 1


def test_no_tokens_gives_zero_weight_gradients():
    c = Case(0, 2, 2, 64, 64)
    dg = [torch.ones(64, device=dev()), torch.ones(64, device=dev())]
    ws = torch.empty(mst.mst_qk_norm_rotate_bwd_workspace(c.rotation, 0), dtype=torch.uint8, device=dev())
    t = torch.zeros(256, dtype=torch.bfloat16, device=dev())
    mst.mst_qk_norm_rotate_bwd(c.rotation, 1, 0, 1, None, 2, 2, t, t, 256, t, t, 256, t, t, 256, *dg, ws)
    torch.cuda.synchronize()
    assert not dg[0].any() and not dg[1].any()


def test_no_tokens_and_empty_tensors():
    c = Case(0, 2, 2, 64, 64)
    e = torch.empty((0, 256), dtype=torch.bfloat16, device=dev())
    dg = [torch.ones(64, device=dev()), torch.ones(64, device=dev())]
    ws = torch.empty(mst.mst_qk_norm_rotate_bwd_workspace(c.rotation, 0), dtype=torch.uint8, device=dev())
    mst.mst_qk_norm_rotate_fwd(c.rotation, 1, 0, 1, None, 2, 2, e, e, 256, e, e, 256)
    mst.mst_qk_norm_rotate_bwd(c.rotation, 1, 0, 1, None, 2, 2, e, e, 256, e, e, 256, e, e, 256, *dg, ws)
    torch.cuda.synchronize()
    assert not dg[0].any() and not dg[1].any()


@pytest.mark.parametrize("top", [1.0, 1000.0])
@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_at_every_position(interleaved, top):
    """Pairs (1, 0): the results are cosines and sines themselves, nothing else is rounded.  The angle is rounded to fp32 as a number of half turns of
    at most 1 (2^-25 of half a turn, 9.4e-8), sincospi's results by up to 2 units of 2^-24 (1.2e-7): 2.2e-7."""
    from test_angle import INV_TWO_PI, BITS
    from fractions import Fraction
    T, D = 400, 256
    c = Case(T, 1, 1, D, D, interleaved, dtype="f32", norm="", first=0)
    g = torch.Generator().manual_seed(5)
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (T,), generator=g)
    pos[::3] = (1 << 31) - 1 - torch.randint(0, 1 << 20, pos[::3].shape, generator=g)
    pos[:4] = torch.tensor([0, 1, (1 << 31) - 1, -(1 << 31)])
    c.positions = pos.to(torch.int32).to(dev())
    f = (top * 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2) * torch.rand(1, generator=g).item())).float()
    c.dev_freq.copy_(f)
    x = torch.zeros(T, 2, D)
    x[..., slice(0, D, 2) if interleaved else slice(0, D // 2)] = 1.0
    x = x.view(T, 2 * D)
    y, dx = c.padded(), c.padded()
    c.forward(c.padded(x), y)
    c.backward(c.padded(x), c.padded(x), dx)
    torch.cuda.synchronize()
    # pos * f / 2 pi in whole numbers: f is a 24-bit number times a power of two
    angle = np.empty((T, D // 2))
    for i, fi in enumerate(f.tolist()):
        n, d = Fraction(fi).as_integer_ratio()
        for t, p in enumerate(pos.tolist()):
            angle[t, i] = 2 * np.pi * ((((p * n * INV_TWO_PI) // d) >> (BITS - 80)) % (1 << 80)) * 2.0 ** -80
    for got, sign in ((y, 1.0), (dx, -1.0)):
        h = host(got).astype(np.float64).reshape(T, 2, D)
        a, b = (h[..., 0::2], h[..., 1::2]) if interleaved else (h[..., : D // 2], h[..., D // 2:])
        assert np.abs(a - np.cos(angle)[:, None]).max() <= 2.2e-7
        assert np.abs(b - sign * np.sin(angle)[:, None]).max() <= 2.2e-7


def test_frequencies_that_are_no_numbers():
    c = Case(5, 2, 1, 64, 64, norm="", dtype="f32", first=0)
    c.dev_freq[3], c.dev_freq[30] = float("inf"), float("nan")
    y, dx = c.padded(), c.padded()
    c.forward(c.padded(c.x), y)
    c.backward(c.padded(c.x), c.padded(c.dy), dx)
    torch.cuda.synchronize()
    for t in (y, dx):
        h = host(t).reshape(5, 3, 2, 32)
        assert np.isnan(h[..., [3, 30]]).all() and np.isfinite(np.delete(h, [3, 30], -1)).all()
