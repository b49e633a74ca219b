"""Paged cache: append (keys normed and rotated on the way) and attention of new tokens, through the C ABI, against the plain definition in 64 bits.

Tolerances of the attention.  A result is rounded once (2^-8 of its value).  The softmax weights are rounded to bf16 before they multiply the values: 2^-8 of each
term, so 2^-8 of sum_j P_j |v_j|.  Scores are fp32 sums of d <= 128 exact products: d 2^-24 sum |q k| / sqrt(d) <= 5e-5 for the values here
(|q|, |k| up to about 5), the exponent is rounded at up to 2^5 (2^-19 ln 2), 2^x and the sums add 1e-6 a step of at most some hundred: 2e-4 in all, for the
terms and for the sum of weights, 4e-4 of the same sum; 2e-4 for lse.
"""
import numpy as np
import pytest

from oracle import paged, rotation

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    import paper_2408_11746_b200 as mst
    from gpu_util import dev, host

EPS = 1e-5
FAR = 1 << 30
BAD_PAGE = 16
ROWS_OUTSIDE = 64


class Case:
    def __init__(self, new, length, heads=4, kv=4, D=64, page=16, seed=0, spare=0, heads_first=False, max_new=None, max_len=None, std=1.0,
                 table_extra=0):
        g = torch.Generator().manual_seed(2000 + seed)
        self.new, self.length, self.heads, self.kv, self.D, self.page = list(new), list(length), heads, kv, D, page
        self.first = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.rows = int(self.first[-1])
        self.tokens = self.rows + spare
        pages = [max(0, (n + page - 1) // page) for n in length]
        total = sum(pages) + 3
        order = torch.randperm(total, generator=g).to(torch.int32)
        self.table = torch.full((len(new), max(pages + [1]) + table_extra), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(pages):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (total, kv, page, D) if heads_first else (total, page, kv, D)
        rnd = lambda s, std=1.0: (torch.randn(*s, generator=g) * std).to(torch.bfloat16)
        self.K, self.V = rnd(shape, std), rnd(shape)
        if heads_first:
            self.K, self.V = self.K.transpose(1, 2), self.V.transpose(1, 2)
        self.Q = rnd((self.tokens, heads * D), std)
        self.max_new = max(list(new) + [0]) if max_new is None else max_new
        self.max_len = max(max(length), 0) if max_len is None else max_len

    def upload(self):
        layout = lambda t: t.transpose(1, 2).to(dev()).transpose(1, 2) if not t.is_contiguous() else t.to(dev())
        self.dK, self.dV = layout(self.K), layout(self.V)
        self.cache = mst.PagedCache(self.dK, self.dV)
        self.dev_first = torch.from_numpy(self.first).to(dev())
        self.dev_len = torch.tensor(self.length, dtype=torch.int32, device=dev())
        self.dev_table = self.table.to(dev())
        self.batch = mst.PagedBatch(self.dev_first, self.dev_len, self.dev_table, self.tokens, self.max_new, self.max_len)
        return self

    def workspace(self, stride):
        n = mst.mst_paged_attention_workspace(self.cache, self.batch, self.heads, stride)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device=dev()) if n else None

    def buffers(self, pad=0):
        q = torch.full((self.tokens, self.heads * self.D + pad), float("nan"), dtype=torch.bfloat16, device=dev())
        q[:, : self.heads * self.D] = self.Q.to(dev())
        return q, torch.full_like(q, 7.0), torch.full((self.heads, self.tokens), 7.0, device=dev())

    def attend(self, stride, pad=0, lse=True):
        q, out, z = self.buffers(pad)
        mst.mst_paged_attention(self.cache, self.batch, self.heads, stride, q, q.stride(0), out, out.stride(0), z if lse else None, self.workspace(stride))
        torch.cuda.synchronize()
        return out, z

    def check(self, stride, out, z, flags=0, pad=0):
        assert mst.mst_device_error_flags() == flags
        C = self.heads * self.D
        ref, ref_z, weight = paged.paged_attention(self.Q.float().numpy().reshape(self.tokens, self.heads, self.D), self.K.float().numpy(),
                                                   self.V.float().numpy(), self.first, self.length, self.table.numpy(), stride)
        o, n = host(out[:, :C]).reshape(ref.shape).astype(np.float64), self.rows
        assert (np.abs(o[:n] - ref[:n]) <= 2.0 ** -8 * np.abs(ref[:n]) + (2.0 ** -8 + 4e-4) * weight[:n] + 1e-30).all()
        assert (o[n:] == 7.0).all() and (out[:, C:] == 7.0).all()
        if z is not None:
            zz = host(z).astype(np.float64)
            empty = np.isneginf(ref_z[:, :n])
            assert (np.isneginf(zz[:, :n]) == empty).all()
            assert (np.abs(zz[:, :n][~empty] - ref_z[:, :n][~empty]) <= 2e-4).all()
            assert (zz[:, n:] == 7.0).all()

    def said(self, form):
        """What the call is told of its sizes, which decides the kernel and how the work is cut up and nothing else: "few" rows, 128-row "tiles",
        "ranges" of tiles (two or three from 1024 positions, or from 48 tiles and strided keys on), tiles of which a block sees to one after "again"
        another, or as things are."""
        self.batch.max_new, self.batch.max_len = {"few": (1, self.max_len), "tiles": (4096, 1 << 20), "ranges": (700, 3000), "far": (4000, 6000), "again": (40, 1 << 20),
                                                  "true": (self.max_new, self.max_len)}[form]
        return self

    def run(self, stride, pad=0):
        self.upload()
        for form in ("true", "few", "tiles", "ranges", "far", "again"):
            out, z = self.said(form).attend(stride, pad)
            self.check(stride, out, z)


# new tokens and lengths: one token each; drafts; chunks; nothing new; nothing at all; a length that is its new tokens
ONE = ([1] * 5, [1, 17, 300, 64, 1025])
DRAFTS = ([5, 3, 0, 1, 4], [5, 700, 33, 2, 129])
CHUNK = ([130, 1, 67], [130, 400, 321])


@pytest.mark.parametrize("stride", [FAR, 64, 128, 100])
@pytest.mark.parametrize("shape", [ONE, DRAFTS, CHUNK])
@pytest.mark.parametrize("heads,kv,D,page,heads_first", [(4, 4, 64, 16, False), (6, 2, 64, 64, True), (2, 1, 128, 24, False), (7, 1, 64, 7, False),
                                                         (3, 3, 128, 1, True)])
def test_attention(heads, kv, D, page, heads_first, shape, stride):
    Case(*shape, heads, kv, D, page, heads_first=heads_first, spare=3, seed=stride % 97 + D).run(stride, pad=8)


@pytest.mark.parametrize("page", [16, 12])
@pytest.mark.parametrize("stride", [FAR, 64])
@pytest.mark.parametrize("layout", ["slots of all pages side by side", "keys and values of a page side by side", "padded heads", "heads, then slots, then pages"])
def test_orders_of_the_cache(layout, stride, page):
    c = Case(*CHUNK, 4, 2, page=page, seed=3).upload()
    n = c.dK.shape[0]
    if layout == "slots of all pages side by side":
        c.dK, c.dV = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (c.dK, c.dV))
    elif layout == "keys and values of a page side by side":
        both = torch.stack([c.dK, c.dV], dim=1)
        c.dK, c.dV = both[:, 0], both[:, 1]
    elif layout == "padded heads":
        pad = torch.full((2, n, page, 3, 72), float("nan"), dtype=torch.bfloat16, device=dev())
        pad[:, :, :, :2, :64] = torch.stack([c.dK, c.dV])
        c.dK, c.dV = pad[0][:, :, :2, :64], pad[1][:, :, :2, :64]
    else:
        c.dK, c.dV = (t.permute(2, 1, 0, 3).contiguous().permute(2, 1, 0, 3) for t in (c.dK, c.dV))
    c.cache = mst.PagedCache(c.dK, c.dV)
    for form in ("few", "tiles", "ranges"):
        c.check(stride, *c.said(form).attend(stride))


@pytest.mark.parametrize("stride", [FAR, 200])
@pytest.mark.parametrize("heads,kv", [(2, 2), (5, 1), (40, 1)])
def test_tiles_of_many_sequences(heads, kv, stride):
    # long and short sequences that end far apart or alike, none, 32 and more of them
    Case([300, 1, 0, 520, 129, 260], [900, 1500, 10, 520, 2600, 2500], heads, kv, seed=1, spare=2).run(stride)
    Case([300, 290, 310], [700, 690, 705], heads, kv, seed=2).run(stride)
    Case([(7 * i) % 50 for i in range(32)], [60 + (37 * i) % 500 for i in range(32)], heads, kv, seed=3).run(stride)
    Case([(7 * i) % 50 for i in range(33)], [60 + (37 * i) % 500 for i in range(33)], heads, kv, seed=4).run(stride)


@pytest.mark.parametrize("stride", [1, 2, 3, 17, 31])
def test_short_strides(stride):
    Case([1, 40, 6], [333, 90, 6], 4, 2).run(stride)


@pytest.mark.parametrize("heads,kv", [(40, 1), (33, 1), (16, 1), (20, 4)])
def test_many_heads_to_a_key_head(heads, kv):
    Case([1, 3, 20], [70, 260, 41], heads, kv).run(FAR)
    Case([1, 3, 20], [270, 460, 41], heads, kv).run(64)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("stride", [FAR, 64, 256])
def test_long_lists_in_ranges(stride, D):
    # few rows over long lists: ranges of one list in several blocks, joined by the second launch
    Case([1, 1, 3], [6000, 257, 4097], 4, 2, D, 16).run(stride)
    Case([70, 1, 3], [3000, 257, 2049], 2, 2, D, 64).run(stride)


@pytest.mark.parametrize("max_new,max_len", [(0, 0), (1, 1), (1, 100000), (1000, 1), (3, 700)])
@pytest.mark.parametrize("stride", [FAR, 128])
def test_what_is_said_of_sizes_does_not_change_results(stride, max_new, max_len):
    Case([1, 50, 7], [2000, 333, 7], 4, 2, max_new=max_new, max_len=max_len).run(stride)


def test_lengths_below_the_new_tokens():
    Case([4, 3, 2], [2, 0, -5], 2, 2).run(FAR)
    Case([40, 3, 200], [2, 0, 150], 2, 2).run(64)


@pytest.mark.parametrize("stride", [FAR, 64])
@pytest.mark.parametrize("new", [1, 90])
def test_pages_that_do_not_exist(new, stride):
    c = Case([new, new], [500, 420], 2, 2, page=16)
    c.table[0, 3], c.table[0, 31], c.table[1, 10], c.table[1, 0] = -1, 10 ** 6, -(1 << 31), c.K.shape[0]
    c.upload()
    for form in ("few", "tiles"):
        out, z = c.said(form).attend(stride)
        c.check(stride, out, z, flags=BAD_PAGE)
        assert mst.mst_device_error_flags() == 0


@pytest.mark.parametrize("stride", [FAR, 64, 170])
@pytest.mark.parametrize("new", [2, 90])
def test_a_table_shorter_than_the_length(new, stride):
    c = Case([new], [400], 2, 2, page=16)
    c.table = c.table[:, :20].contiguous()
    c.upload()
    for form in ("few", "tiles"):
        out, z = c.said(form).attend(stride)
        c.check(stride, out, z, flags=BAD_PAGE)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("stride", [FAR, 64])
@pytest.mark.parametrize("form", ["few", "tiles"])
@pytest.mark.parametrize("new,page", [([1, 6], 16), ([96, 200], 64), ([33, 70], 7)])
def test_what_is_not_attended_does_not_reach_a_result(new, page, stride, value, form):
    # the last token's key and value are no numbers, nor is what the pages hold behind the lengths, nor a page of nobody; rows before it do not see them
    c = Case(new, [300, 420], 4, 2, page=page)
    K, V = c.K.clone(), c.V.clone()
    used = torch.zeros(K.shape[:2], dtype=torch.bool)
    for b in range(2):
        for p in range(c.length[b]):
            used[c.table[b, p // page], p % page] = True
    K[~used], V[~used] = value, value
    last = c.length[1] - 1
    at = (int(c.table[1, last // page]), last % page)
    c.K, c.V = K, V
    c.K[at] = value
    c.V[at] = value
    c.upload()
    out, z = c.said(form).attend(stride)
    assert mst.mst_device_error_flags() == 0
    keep = host(out)[: c.rows - 1]
    assert np.isfinite(keep).all()
    c.K[at] = 0.0
    c.V[at] = 0.0
    n = c.rows - 1
    ref, ref_z, weight = paged.paged_attention(c.Q.float().numpy().reshape(c.tokens, 4, 64), c.K.float().numpy(), c.V.float().numpy(), c.first, c.length,
                                               c.table.numpy(), stride)
    o = keep.reshape(n, 4, 64)
    assert (np.abs(o - ref[:n]) <= 2.0 ** -8 * np.abs(ref[:n]) + (2.0 ** -8 + 4e-4) * weight[:n]).all()
    assert (np.abs(host(z)[:, :n] - ref_z[:, :n]) <= 2e-4).all()
    if value == value and value < 0:
        return                                        # a key of -inf: scores of either sign of infinity or NaN, by the query's signs
    assert np.isnan(host(out)[c.rows - 1]).any()       # the row that does see them


@pytest.mark.parametrize("new", [1, 5, 100])
def test_peaked_rows(new):
    c = Case([new, new], [900, 300], 2, 2, std=4.0)       # scores of variance 256: a few keys have all the weight
    c.upload()
    out, z = c.said("tiles" if new == 100 else "few").attend(FAR)
    # scores up to about 100: their rounding (2^-24 of sum |q k| / 8, some 300) and that of the exponents at 2^7 are below 4e-5 each
    c.check(FAR, out, z)


def test_lengths_and_rows_that_make_no_sense():
    # far beyond the table, below zero, rows that overlap, go backwards or lie outside: the sequence in between is served, nothing outside is written
    c = Case([1, 3, 40], [50, 60, 300], 2, 2)
    for form in ("few", "tiles"):
        for stride in (FAR, 64, 7):
            c.upload().said(form)
            c.dev_len.copy_(torch.tensor([(1 << 31) - 1, -(1 << 31), 300], dtype=torch.int32))
            out, z = c.attend(stride)
            assert mst.mst_device_error_flags() == BAD_PAGE
            ref, ref_z, weight = paged.paged_attention(c.Q.float().numpy().reshape(c.tokens, 2, 64), c.K.float().numpy(), c.V.float().numpy(), [0, 0, 4, 44],
                                                       [0, 0, 300], c.table.numpy(), stride)
            o = host(out).reshape(ref.shape)
            assert (np.abs(o[4:] - ref[4:]) <= 2.0 ** -8 * np.abs(ref[4:]) + (2.0 ** -8 + 4e-4) * weight[4:]).all()
            assert (o[1:4] == 0).all() and np.isneginf(host(z)[:, 1:4]).all()
            c.dev_first.copy_(torch.tensor([-7, 1 << 30, 4, 3], dtype=torch.int32))
            out, z = c.attend(stride)
            assert (host(out) == 7.0).all() and (host(z) == 7.0).all()
            mst.mst_device_error_flags()


def _cut(c, tokens):
    """What the oracle is told of a step whose rows go beyond `tokens`: those below it, where they are."""
    beyond = np.maximum(c.first[1:].astype(np.int64) - np.maximum(c.first[:-1], tokens), 0)
    c.length = (np.array(c.length) - beyond).tolist()
    c.first = np.minimum(c.first, tokens)
    c.rows = tokens


@pytest.mark.parametrize("ahead", [0, 32])
@pytest.mark.parametrize("stride", [FAR, 64, 7])
def test_rows_beyond_the_activations(stride, ahead):
    # one sequence is cut short by the number of rows, one lies behind it: what rows there are is served, and the call says so
    c = Case([1] * ahead + [3, 40, 60, 5], [9] * ahead + [50, 300, 400, 70], 4, 2)
    c.tokens = 70 + ahead
    c.Q = c.Q[: c.tokens].contiguous()
    c.upload()
    _cut(c, c.tokens)
    for form in ("true", "few", "tiles", "ranges", "far", "again"):
        out, z = c.said(form).attend(stride)
        c.check(stride, out, z, flags=ROWS_OUTSIDE)
    assert mst.mst_device_error_flags() == 0


def test_no_lse_and_repeats():
    for new, length, form in (([1, 1], [5000, 300], "true"), ([100, 300], [2000, 300], "true"), ([100, 300], [2000, 300], "tiles"), ([100, 300], [6000, 300], "far")):
        c = Case(new, length, 4, 2).upload().said(form)
        a, z = c.attend(128)
        for _ in range(3):
            b, y = c.attend(128)
            assert torch.equal(a, b) and torch.equal(z, y)
        b, y = c.attend(128, lse=False)
        assert torch.equal(a, b) and (y == 7.0).all()


def test_random_shapes():
    rng = np.random.default_rng(77)
    for case in range(24):
        B = int(rng.integers(1, 5))
        most = int(rng.choice([1, 6, 200]))
        new = rng.integers(0, most + 1, B)
        length = [int(n + rng.integers(0, 900)) for n in new]
        kv = int(rng.integers(1, 4))
        heads = kv * int(rng.integers(1, 6))
        stride = int(rng.choice([FAR, 64, 128, 192, 320, int(rng.integers(1, 700))]))
        Case(new.tolist(), length, heads, kv, int(rng.choice([64, 64, 128])), int(rng.choice([8, 16, 32, 64, 128, int(rng.integers(1, 90))])), seed=case,
             spare=int(rng.integers(0, 5)), heads_first=bool(rng.integers(0, 2)), table_extra=int(rng.integers(0, 3))).run(stride)


def test_offsets_beyond_32_bits():
    # a pool of which the last pages lie more than 2^32 elements behind the first; pages in between are never touched
    page, pages = 64, (1 << 32) // (64 * 2 * 64) + 40
    K = torch.empty((pages, page, 2, 64), dtype=torch.bfloat16, device=dev())
    V = torch.empty_like(K)
    for new in (1, 80):
        c = Case([new, 1], [500, 200], 4, 2, page=page).upload()
        used = c.table[c.table >= 0]
        far = torch.arange(pages - len(used), pages, dtype=torch.int32)
        K[far.long()], V[far.long()] = c.dK[used.long().to(dev())], c.dV[used.long().to(dev())]
        c.dev_table = c.dev_table.clone()
        c.dev_table[c.dev_table >= 0] = far.to(dev())
        c.cache = mst.PagedCache(K, V)
        c.batch = mst.PagedBatch(c.dev_first, c.dev_len, c.dev_table, c.tokens, c.max_new, c.max_len)
        for stride in (FAR, 64):
            for form in ("few", "tiles"):
                c.check(stride, *c.said(form).attend(stride))


def test_streams_and_captured_graphs_side_by_side():
    a, b = Case([1, 1], [5000, 700], 4, 2, seed=1).upload(), Case([90, 40], [1500, 800], 4, 2, seed=2).upload().said("tiles")
    want = [a.attend(128), b.attend(128)]
    graphs, outs, keep = [], [], []
    for c in (a, b):
        q, out, z = c.buffers()
        ws = c.workspace(128)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mst.mst_paged_attention(c.cache, c.batch, 4, 128, q, 256, out, 256, z, ws)
        graphs.append(g)
        outs.append((out, z))
        keep.append((q, ws))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for (o, z), (ro, rz) in zip(outs, want):
        assert torch.equal(o, ro) and torch.equal(z, rz)
    # a replayed graph sees the lengths and tables of its day
    a.dev_len.copy_(torch.tensor([4000, 650], dtype=torch.int32))
    graphs[0].replay()
    torch.cuda.synchronize()
    a.length = [4000, 650]
    a.check(128, *outs[0])


def test_pointers_of_the_host_are_refused():
    c = Case([1], [40], 2, 2).upload()
    q, out, z = c.buffers()
    h = torch.zeros(1, 128, dtype=torch.bfloat16)
    for args in ((h, out, z), (q, h, z), (q, out, torch.zeros(2, 1))):
        with pytest.raises(mst.MstError) as e:
            mst.mst_paged_attention(c.cache, c.batch, 2, 64, args[0], 128, args[1], 128, args[2])
        assert e.value.status == 1
    c.batch = mst.PagedBatch(c.dev_first, c.dev_len, c.table, 1, 1, 40)
    with pytest.raises(mst.MstError) as e:
        c.attend(64)
    assert e.value.status == 1


# ---------------------------------------------------------------------------------------------- append
def _rotation(D, rot, interleaved, norm, seed=0):
    g = torch.Generator().manual_seed(seed)
    f = (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))).float()
    w = 0.5 + torch.rand(2, D, generator=g)
    gq, gk = (w[0], w[1]) if norm else (None, None)
    up = lambda t: None if t is None else t.to(dev())
    return mst.Rotation(D, rot, up(f), up(gq), up(gk), EPS, interleaved), f.numpy(), [None if t is None else t.numpy() for t in (gq, gk)]


def _append_ref(c, x, f, gamma, rot, inter):
    """(q, K, V) in 64 bits and what their rounding is measured by; x [tokens, heads + 2 kv, D]"""
    seq, pos = paged.positions(c.first, c.length)
    n, H, G = c.rows, c.heads, c.kv
    ref_q = rotation.norm_rotate(x[:n, :H], gamma[0], pos, f, rot, inter, EPS)
    ref_k = rotation.norm_rotate(x[:n, H:H + G], gamma[1], pos, f, rot, inter, EPS)
    K, V = c.K.double().numpy().copy(), c.V.double().numpy().copy()
    for t in range(n):
        if pos[t] < 0:
            continue
        page, slot = paged.slots(c.table[seq[t]].numpy(), c.page, K.shape[0], pos[t:t + 1])
        if page[0] >= 0:
            K[page[0], slot[0]], V[page[0], slot[0]] = ref_k[t], x[t, H + G:]
    return ref_q, K, V, pos


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("new,length,heads,kv,D,rot,page,heads_first", [
    ([1] * 40, list(range(1, 801, 20)), 12, 12, 64, 64, 16, False), ([5, 0, 130, 1], [5, 9, 400, 1000], 20, 4, 64, 32, 24, True),
    ([3, 2], [2, 0], 2, 1, 128, 128, 7, False), ([17], [70000], 3, 3, 80, 48, 128, False), ([300, 31], [300, 77], 2, 2, 8, 0, 64, False)])
def test_append(new, length, heads, kv, D, rot, page, heads_first, interleaved, norm):
    c = Case(new, length, heads, kv, D, page, spare=2, heads_first=heads_first).upload()
    r, f, gamma = _rotation(D, rot, interleaved, norm)
    x = torch.randn(c.tokens, heads + 2 * kv, D).to(torch.bfloat16)
    d = x.view(c.tokens, -1).to(dev())
    q = torch.full((c.tokens, heads * D + 8), 7.0, dtype=torch.bfloat16, device=dev())
    at = lambda h: d.data_ptr() + 2 * h * D
    mst.mst_paged_append(c.cache, c.batch, r, heads, at(0), at(heads), at(heads + kv), d.stride(0), q, q.stride(0))
    torch.cuda.synchronize()
    assert mst.mst_device_error_flags() == 0
    xd = x.double().numpy()
    ref_q, K, V, pos = _append_ref(c, xd, f, gamma, rot, interleaved)
    got = host(q).astype(np.float64)
    here = got[: c.rows, : heads * D].reshape(c.rows, heads, D)
    size = rotation.pair_sizes(ref_q, rot, interleaved)
    ok = np.abs(here - ref_q) <= 2.0 ** -8 * np.abs(ref_q) + 2e-6 * size + 1e-30
    assert ok[pos >= 0].all() and (here[pos < 0] == 7.0).all()
    assert (got[c.rows:] == 7.0).all() and (got[:, heads * D:] == 7.0).all()
    np.testing.assert_array_equal(host(c.dV), V)
    assert (np.abs(host(c.dK) - K) <= 2.0 ** -8 * np.abs(K) + 2e-6 * rotation.pair_sizes(K, rot, interleaved) + 1e-30).all()


def test_append_without_rotation_or_queries_and_with_bad_pages():
    c = Case([40, 3], [100, 3], 2, 2, 64, 16)
    c.table[0, 5] = 10 ** 6
    c.upload()
    x = torch.randn(c.tokens, 6, 64).to(torch.bfloat16)
    d = x.view(c.tokens, -1).to(dev())
    mst.mst_paged_append(c.cache, c.batch, None, 0, None, d.data_ptr() + 256, d.data_ptr() + 512, 384)
    torch.cuda.synchronize()
    assert mst.mst_device_error_flags() == BAD_PAGE and mst.mst_device_error_flags() == 0
    _, K, V, _ = _append_ref(c, x.double().numpy(), np.zeros(0), [None, None], 0, False)
    np.testing.assert_array_equal(host(c.dK), K)
    np.testing.assert_array_equal(host(c.dV), V)


@pytest.mark.parametrize("first", [[0, 3, 43, 103], [0, 3, 43, 70, 103], [-2, 3, 43]])
@pytest.mark.parametrize("form", ["few", "tiles"])
def test_append_and_attention_of_rows_that_are_not_there(first, form):
    # a step with rows beyond the activations (70 of them), or below: both calls serve the same rows, and both say so
    new = np.diff(first).tolist()
    c = Case(new, [n + 200 for n in new], 4, 2)
    c.tokens = min(70, first[-1])
    c.Q = c.Q[: c.tokens].contiguous()
    c.first = np.array(first, np.int32)
    c.upload().said(form)
    r, f, gamma = _rotation(64, 64, False, True)
    x = torch.randn(c.tokens, 8, 64).to(torch.bfloat16)
    d = x.view(c.tokens, -1).to(dev())
    q = torch.full((c.tokens, 256), 7.0, dtype=torch.bfloat16, device=dev())
    at = lambda h: d.data_ptr() + 128 * h
    mst.mst_paged_append(c.cache, c.batch, r, 4, at(0), at(4), at(6), 512, q, 256)
    torch.cuda.synchronize()
    assert mst.mst_device_error_flags() == ROWS_OUTSIDE and mst.mst_device_error_flags() == 0
    _cut(c, c.tokens)
    lo = 0
    if c.first[0] < 0:           # the oracle has no such rows: the sequence goes, its row of the table too
        lo = int(c.first[1])
        c.first, c.length, c.table = c.first[1:] - lo, c.length[1:], c.table[1:]
        c.rows -= lo
    ref_q, K, V, _ = _append_ref(c, x.double().numpy()[lo:], f, gamma, 64, False)
    got = host(q)
    assert (got[:lo] == 7.0).all()
    here = got[lo:].reshape(c.rows, 4, 64)
    assert (np.abs(here - ref_q) <= 2.0 ** -8 * np.abs(ref_q) + 2e-6 * rotation.pair_sizes(ref_q, 64, False) + 1e-30).all()
    np.testing.assert_array_equal(host(c.dV), V)
    assert (np.abs(host(c.dK) - K) <= 2.0 ** -8 * np.abs(K) + 2e-6 * rotation.pair_sizes(K, 64, False) + 1e-30).all()
    c.Q, c.K, c.V = q.cpu(), c.dK.cpu(), c.dV.cpu()
    out, z = c.attend(128)
    assert (out[:lo] == 7.0).all() and (z[:, :lo] == 7.0).all()
    c.Q, c.tokens = c.Q[lo:], c.tokens - lo
    c.check(128, out[lo:], z[:, lo:], flags=ROWS_OUTSIDE)


def test_append_in_place_queries():
    c = Case([40, 3], [100, 3], 4, 2).upload()
    r, _, _ = _rotation(64, 64, False, True)
    d = torch.randn(c.tokens, 8 * 64).to(torch.bfloat16).to(dev())
    q, e = torch.empty(c.tokens, 256, dtype=torch.bfloat16, device=dev()), d.clone()
    at = lambda t, h: t.data_ptr() + 128 * h
    mst.mst_paged_append(c.cache, c.batch, r, 4, d, at(d, 4), at(d, 6), 512, q, 256)
    mst.mst_paged_append(c.cache, c.batch, r, 4, e, at(e, 4), at(e, 6), 512, e, 512)
    torch.cuda.synchronize()
    assert torch.equal(e[:, :256], q) and torch.equal(e[:, 256:], d[:, 256:])


# ---------------------------------------------------------------------------------------------- as they are used
@pytest.mark.parametrize("stride", [128, 256, 512])
def test_generation_agrees_with_the_training_time_attention(stride):
    """A fused activation through norm, rotation and the strided attention, as in training; and the same sequences piece by piece - a prompt
    in chunks, then token by token - through append and paged attention.  Both round q and k to bf16 once, at the same place, and results are bf16 of
    sums whose weights are bf16: 2^-8 of each result and of sum P |v| for either side."""
    B, n, H, D = 2, 512, 3, 64
    C = H * D
    qkv = torch.randn(B * n, 3 * C).to(torch.bfloat16).to(dev())
    r, _, _ = _rotation(D, D, False, True)
    qk = torch.empty(B * n, 2 * C, dtype=torch.bfloat16, device=dev())
    x, y = qkv.data_ptr(), qk.data_ptr()
    mst.mst_qk_norm_rotate_fwd(r, mst.MST_BF16, B * n, n, None, H, H, x, x + 2 * C, 3 * C, y, y + 2 * C, 2 * C)
    both = torch.cat([qk, qkv[:, 2 * C:]], 1)
    out = torch.empty(B * n, C, dtype=torch.bfloat16, device=dev())
    lse = torch.empty(B, H, n, device=dev())
    z = both.data_ptr()
    mst.mst_strided_attention_fwd(z, z + 2 * C, z + 4 * C, 3 * C, B, n, H, D, stride, out, C, lse)
    page = 32
    per = n // page
    table = torch.randperm(B * per).to(torch.int32).view(B, per).to(dev())
    K, V = (torch.full((B * per, page, H, D), float("nan"), dtype=torch.bfloat16, device=dev()) for _ in range(2))
    cache = mst.PagedCache(K, V)
    rows = qkv.view(B, n, 3 * C)
    got, got_z = torch.empty(B, n, C, dtype=torch.bfloat16, device=dev()), torch.empty(B, H, n, device=dev())
    at = [0, 0]
    steps = [(200, 131), (250, 1), (1, 300), (1, 40)] + [(1, 1)] * 40
    for step in steps + [(n, n)]:
        step = [min(s, n - a) for s, a in zip(step, at)]
        new = torch.cat([rows[b, at[b]:at[b] + step[b]] for b in range(B)]).contiguous()
        at = [a + s for a, s in zip(at, step)]
        first = torch.tensor([0, step[0], sum(step)], dtype=torch.int32, device=dev())
        length = torch.tensor(at, dtype=torch.int32, device=dev())
        many = max(step) > 100                       # the prompts' chunks in tiles
        batch = mst.PagedBatch(first, length, table, sum(step), 4096 if many else max(step), 1 << 20 if many else max(at))
        q = torch.empty(max(sum(step), 1), C, dtype=torch.bfloat16, device=dev())
        o, zz = torch.empty_like(q), torch.empty(H, max(sum(step), 1), device=dev())
        p = new.data_ptr()
        mst.mst_paged_append(cache, batch, r, H, p, p + 2 * C, p + 4 * C, 3 * C, q, C)
        need = mst.mst_paged_attention_workspace(cache, batch, H, stride)
        ws = torch.empty(need, dtype=torch.uint8, device=dev()) if need else None
        mst.mst_paged_attention(cache, batch, H, stride, q, C, o, C, zz, ws)
        t = 0
        for b in range(B):
            got[b, at[b] - step[b]:at[b]] = o[t:t + step[b]]
            got_z[b, :, at[b] - step[b]:at[b]] = zz[:, t:t + step[b]]
            t += step[b]
    torch.cuda.synchronize()
    assert at == [n, n] and mst.mst_device_error_flags() == 0
    want, v = host(out).reshape(B, n, H, D), host(qkv[:, 2 * C:]).reshape(B, n, H, D)
    from oracle import attention as att
    q64, k64 = (host(qk[:, i * C:(i + 1) * C]).reshape(B, n, H, D).transpose(0, 2, 1, 3) for i in range(2))
    weight, _ = att.strided_attention(q64, k64, np.abs(v).transpose(0, 2, 1, 3), stride)
    weight = weight.transpose(0, 2, 1, 3)
    g = host(got).reshape(B, n, H, D)
    assert (np.abs(g - want) <= 2 * (2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 4e-4) * weight)).all()
    assert (np.abs(host(got_z) - host(lse)) <= 4e-4).all()


def test_training_step_around_the_attention():
    """qkv -> norm and rotation -> strided attention and back again; the gradient of the fused activation against the plain definition's, in 64 bits."""
    from oracle import attention as att
    B, n, H, D, stride = 2, 256, 2, 64, 128
    C = H * D
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn(B * n, 3 * C, generator=g).to(torch.bfloat16)
    dout = torch.randn(B * n, C, generator=g).to(torch.bfloat16)
    r, f, gamma = _rotation(D, D, False, True)
    d, do = qkv.to(dev()), dout.to(dev())
    qk, dqkv, dqk = torch.empty(B * n, 2 * C, dtype=torch.bfloat16, device=dev()), torch.empty_like(d), torch.empty(B * n, 3 * C, dtype=torch.bfloat16, device=dev())
    x, y = d.data_ptr(), qk.data_ptr()
    mst.mst_qk_norm_rotate_fwd(r, mst.MST_BF16, B * n, n, None, H, H, x, x + 2 * C, 3 * C, y, y + 2 * C, 2 * C)
    full = torch.cat([qk, d[:, 2 * C:]], 1)
    out, lse = torch.empty(B * n, C, dtype=torch.bfloat16, device=dev()), torch.empty(B, H, n, device=dev())
    z, w = full.data_ptr(), dqk.data_ptr()
    mst.mst_strided_attention_fwd(z, z + 2 * C, z + 4 * C, 3 * C, B, n, H, D, stride, out, C, lse)
    mst.mst_strided_attention_bwd(z, z + 2 * C, z + 4 * C, 3 * C, out, C, do, C, lse, B, n, H, D, stride, w, w + 2 * C, w + 4 * C, 3 * C)
    dg = [torch.empty(D, device=dev()) for _ in range(2)]
    ws = torch.empty(mst.mst_qk_norm_rotate_bwd_workspace(r, B * n), dtype=torch.uint8, device=dev())
    t = dqkv.data_ptr()
    mst.mst_qk_norm_rotate_bwd(r, mst.MST_BF16, B * n, n, None, H, H, x, x + 2 * C, 3 * C, w, w + 2 * C, 3 * C, t, t + 2 * C, 3 * C, *dg, ws)
    torch.cuda.synchronize()
    a = qkv.double().numpy().reshape(B * n, 3 * H, D)
    pos = np.tile(np.arange(n), B)
    heads = lambda m: m.reshape(B, n, H, D).transpose(0, 2, 1, 3)
    rows = lambda m: m.transpose(0, 2, 1, 3).reshape(B * n, H, D)
    q, k = (rotation.norm_rotate(a[:, i * H:(i + 1) * H], gamma[i], pos, f, D, False, EPS) for i in range(2))
    dq, dk, _ = att.strided_attention_bwd(heads(q), heads(k), heads(a[:, 2 * H:]), heads(dout.double().numpy()), stride)
    got = host(dqkv).reshape(B * n, 3 * H, D)
    for i, up in enumerate((dq, dk)):
        ref, ref_g = rotation.norm_rotate_bwd(a[:, i * H:(i + 1) * H], gamma[i], pos, f, D, False, EPS, rows(up))
        # the attention's gradients come with 2e-2 of their largest (its own tolerance); the turn and the norm hand that on
        assert np.abs(got[:, i * H:(i + 1) * H] - ref).max() <= 3e-2 * np.abs(ref).max()
        assert np.abs(host(dg[i]) - ref_g).max() <= 3e-2 * np.abs(ref_g).max()
