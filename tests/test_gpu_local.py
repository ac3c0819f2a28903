"""A party's local operators on the GPU, through the binding, against the definitions in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import local_cases as cases  # noqa: E402


def dev(t):
    """On the GPU with the host tensor's strides and its distance from an aligned address."""
    if t is None:
        return None
    whole = torch.as_strided(t, (t.untyped_storage().nbytes() // t.element_size(),), (1,), 0).cuda()
    return torch.as_strided(whole, t.shape, t.stride(), t.storage_offset())


def back(*ts):
    return tuple(t if t is None else t.cpu() for t in ts)


class Gpu:
    """The binding's functions on host tensors."""

    def __init__(self, api):
        self.api = api

    def status(self):
        return torch.zeros(1, dtype=torch.int32, device="cuda")

    def dropout(self, x, p, seed, offset, residual=None):
        return self.api.haflo_dropout(dev(x), p, seed, offset, residual=dev(residual)).cpu()

    def adapter_forward(self, x, w, a, b, scale, index, p, seed, offset):
        st = self.status()
        return back(*self.api.haflo_adapter_forward(*map(dev, (x, w, a, b, scale, index)), p, seed, offset, status=st)) + (int(st),)

    def adapter_backward(self, dy, x, w, a, b, scale, index, h, p, seed, offset):
        st = self.status()
        return back(*self.api.haflo_adapter_backward(*map(dev, (dy, x, w, a, b, scale, index, h)), p, seed, offset, status=st)) + (int(st),)

    def label_logprobs(self, x, label, top):
        st = self.status()
        return back(*self.api.haflo_label_logprobs(dev(x), dev(label), top, status=st)) + (int(st),)

    def label_logprobs_backward(self, x, label, lse, entropy, dlogp, dentropy, top_index, dtop):
        return self.api.haflo_label_logprobs_backward(*map(dev, (x, label, lse, entropy, dlogp, dentropy, top_index, dtop))).cpu()


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2107_13797_amd import api
    api.lib()
    return api


@pytest.fixture(scope="module")
def run(api):
    return Gpu(api)


@pytest.mark.parametrize("case", cases.DROPOUT, ids=str)
def test_dropout(run, case):
    cases.check_dropout(run, *case)


def test_dropout_special(run):
    cases.check_dropout_special(run)


@pytest.mark.parametrize("case", cases.ADAPTERS + cases.ADAPTERS_LARGE, ids=str)
def test_adapters(run, case):
    cases.check_adapters(run, *case)


def test_adapters_other_parties_infinities(run):
    cases.check_adapters_other_parties_infinities(run)


@pytest.mark.parametrize("case", cases.LABELS + cases.LABELS_LARGE, ids=str)
def test_labels(run, case):
    cases.check_labels(run, *case)


def test_labels_nan(run):
    cases.check_labels_nan(run)


def test_in_place_and_vectors(api):
    x = torch.randn(1000, device="cuda").to(torch.bfloat16)
    want = api.haflo_dropout(x, 0.5, 3)
    again = x.clone()
    assert api.haflo_dropout(again, 0.5, 3, out=again) is again and torch.equal(again, want) and want.shape == x.shape
    res = torch.randn(40, 24, device="cuda")
    m = torch.randn(40, 24, device="cuda")
    want = api.haflo_dropout(m, 0.1, 4, residual=res)
    assert torch.equal(api.haflo_dropout(m, 0.1, 4, residual=res, out=res), want)
    logits, label = torch.randn(9, 3001, device="cuda").half(), torch.arange(9, dtype=torch.int32, device="cuda")
    logp, entropy, lse, _, _ = api.haflo_label_logprobs(logits, label)
    ones = torch.ones(9, device="cuda")
    want = api.haflo_label_logprobs_backward(logits, label, lse, entropy, ones)
    assert torch.equal(api.haflo_label_logprobs_backward(logits, label, lse, entropy, ones, out=logits), want)


def test_gradients_against_differences(api):
    """Backward calls against differences of forward calls along random directions, in float32. With step t the quotient is off by
    the third derivative's t^2 and the forward results' roundings over t; both directions' terms are bounded by `room`."""
    gen = torch.Generator().manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
    rows, cols, t = 6, 40, 2.0 ** -7
    x, label = rnd(rows, cols), torch.tensor([0, 3, -1, 39, 7, 7], dtype=torch.int32, device="cuda")
    cl, ch, ct, dirn = rnd(rows), rnd(rows), rnd(rows, 3), rnd(rows, cols)

    def value(v):
        logp, entropy, _, top, _ = api.haflo_label_logprobs(v, label, 3)
        return float((cl * logp).double().sum() + (ch * entropy).double().sum() + (ct * top).double().sum())

    _, entropy, lse, _, index = api.haflo_label_logprobs(x, label, 3)
    dx = api.haflo_label_logprobs_backward(x, label, lse, entropy, cl, ch, index, ct)
    got, want = float((dx * dirn).double().sum()), (value(x + t * dirn) - value(x - t * dirn)) / (2 * t)
    # third derivatives of these are below 8 |direction|^3 in each row, values below 64
    room = t * t * 8 * float(dirn.abs().amax(1).pow(3).sum()) * float(cl.abs().max() + ch.abs().max() + ct.abs().sum(1).max()) + 64 * rows * 2.0 ** -22 / t
    assert abs(got - want) <= room

    # the adapters' result is linear in each of x, a and b: the quotient is exact but for roundings
    n, r, inner, outer = 3, 4, 24, 20
    x, w, a, b, scale = rnd(rows, inner), rnd(outer, inner), rnd(n, r, inner), rnd(n, outer, r), rnd(n).abs() + 0.5
    ids, dy = torch.tensor([0, 2, -1, 0, 1, 2], dtype=torch.int32, device="cuda"), rnd(rows, outer)
    fwd = lambda x, a, b: api.haflo_adapter_forward(x, w, a, b, scale, ids, 0.25, 11, 3)  # noqa: E731
    y, h = fwd(x, a, b)
    grads = api.haflo_adapter_backward(dy, x, w, a, b, scale, ids, h, 0.25, 11, 3)
    for i, arg in enumerate((x, a, b)):
        d = rnd(*arg.shape)
        plus, minus = ([v + s * d if j == i else v for j, v in enumerate((x, a, b))] for s in (1.0, -1.0))
        want = float(((fwd(*plus)[0].double() - fwd(*minus)[0].double()) * dy).sum()) / 2
        size = float((y.abs().max() + fwd(*plus)[0].abs().max()) * dy.abs().sum())
        assert abs(float((grads[i].double() * d).sum()) - want) <= size * (inner + r + 8) * 2.0 ** -20


def test_same_bits_again(api):
    """No result depends on timing."""
    gen = torch.Generator().manual_seed(6)
    x, w, a, b, scale, index, dy = map(dev, cases.adapter_inputs("bf16", 700, 520, 264, 16, 5, "mixed", 0))
    y, h = api.haflo_adapter_forward(x, w, a, b, scale, index, 0.1, 1)
    first = [y, h, *api.haflo_adapter_backward(dy, x, w, a, b, scale, index, h, 0.1, 1)]
    logits, label = torch.randn(3, 70001, generator=gen).bfloat16().cuda(), torch.tensor([5, -1, 70000], dtype=torch.int32, device="cuda")
    seen = api.haflo_label_logprobs(logits, label, 20)
    for _ in range(3):
        y, h = api.haflo_adapter_forward(x, w, a, b, scale, index, 0.1, 1)
        assert all(torch.equal(p, q) for p, q in zip(first, [y, h, *api.haflo_adapter_backward(dy, x, w, a, b, scale, index, h, 0.1, 1)]))
        assert all(torch.equal(p, q) for p, q in zip(seen, api.haflo_label_logprobs(logits, label, 20)))


def test_side_stream_and_graph(api):
    """A step captured on a side stream and replayed on new contents of the same buffers gives what the eager calls give."""
    x, w, a, b, scale, index, dy = map(dev, cases.adapter_inputs("bf16", 200, 136, 136, 8, 3, "mixed", 0))
    label = torch.arange(200, dtype=torch.int32, device="cuda") % 136
    minus = torch.full((200,), -1.0 / 200, device="cuda")

    def step():
        y, h = api.haflo_adapter_forward(x, w, a, b, scale, index, 0.2, 9, 1)
        logp, entropy, lse, top, at = api.haflo_label_logprobs(y, label, 2)
        dlogits = api.haflo_label_logprobs_backward(y, label, lse, entropy, minus)
        dx, da, db = api.haflo_adapter_backward(dlogits, x, w, a, b, scale, index, h, 0.2, 9, 1)
        return y, logp, entropy, top, at, api.haflo_dropout(dx, 0.5, 2, residual=x), da, db

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for k in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(k)).to(x.dtype))
        torch.cuda.synchronize()
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))


def test_long_rows_and_far_offsets(api):
    """Elements past 2^31 in one array: dropout of the last rows of a wide matrix, labels in the last of many rows."""
    rows, cols = 70001, 32768
    x = torch.empty((rows, cols), dtype=torch.float16, device="cuda").fill_(1.0)
    y = api.haflo_dropout(x, 0.5, 123, 7)
    last = y[-2:].double().cpu()
    f = torch.zeros(2, cols, dtype=torch.float64)
    for r in range(2):
        for g in range(0, cols // 8, 97):
            words = cases.philox(g, rows - 2 + r, 123, 7)
            for j in range(8):
                f[r, 8 * g + j] = 2.0 * ((words[j // 2] >> (16 * (j % 2)) & 0xFFFF) >= 32768)
                assert last[r, 8 * g + j] == f[r, 8 * g + j]
    x[-1, 77] = 12.0
    label = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    label[-1] = 77
    logp, entropy, lse, top, at = api.haflo_label_logprobs(x, label, 1)
    s = math.exp(1.0 - 12.0) * (cols - 1) + 1.0
    assert int(at[-1, 0]) == 77 and abs(float(logp[-1]) + math.log(s)) < 1e-5 and float(logp[:-1].abs().max()) == 0.0
    dx = api.haflo_label_logprobs_backward(x, label, lse, entropy, torch.ones(rows, device="cuda"), out=x)
    assert abs(float(dx[-1, 77]) - (1.0 - 1.0 / s)) < 1e-3 and not bool(dx[:-1].any())


def test_refusals(api):
    f32, i32 = torch.float32, torch.int32
    x = torch.zeros(4, 8, device="cuda")
    bad = [
        lambda: api.haflo_dropout(x.double(), 0.5, 1), lambda: api.haflo_dropout(x, 1.5, 1), lambda: api.haflo_dropout(x, -0.1, 1),
        lambda: api.haflo_dropout(x, math.nan, 1), lambda: api.haflo_dropout(x.cpu(), 0.5, 1), lambda: api.haflo_dropout(x.t(), 0.5, 1),
        lambda: api.haflo_dropout(x, 0.5, 1, residual=x[:3]), lambda: api.haflo_dropout(x, 0.5, 1, out=x.half()),
        lambda: api.haflo_dropout(x[:1].expand(4, 8), 0.5, 1),
    ]
    w, a, b = torch.zeros(6, 8, device="cuda"), torch.zeros(2, 3, 8, device="cuda"), torch.zeros(2, 6, 3, device="cuda")
    s, i = torch.zeros(2, device="cuda"), torch.zeros(4, dtype=i32, device="cuda")
    big = torch.zeros(2, 129, 8, device="cuda")
    fwd = api.haflo_adapter_forward
    bad += [
        lambda: fwd(x, w[:, :7], a, b, s, i), lambda: fwd(x, w, a.half(), b, s, i), lambda: fwd(x, w, a, b[:, :5], s, i),
        lambda: fwd(x, w, a, b, s[:1], i), lambda: fwd(x, w, a, b, s, i.long()), lambda: fwd(x, w, a, b, s, i[:3]), lambda: fwd(x, w, a[0], b, s, i),
        lambda: fwd(x, w, big, torch.zeros(2, 6, 129, device="cuda"), s, i), lambda: fwd(x, w, a, b, s, i, 2.0), lambda: fwd(x[0], w, a, b, s, i),
        lambda: fwd(x, w, a[:0], b[:0], s[:0], i), lambda: fwd(x, w, a.transpose(1, 2).contiguous().transpose(1, 2), b, s, i),
    ]
    y, h = fwd(x, w, a, b, s, i)
    bad += [lambda: api.haflo_adapter_backward(y[:3], x, w, a, b, s, i, h), lambda: api.haflo_adapter_backward(y, x, w, a, b, s, i, h[:, :2]),
            lambda: api.haflo_adapter_backward(y.half(), x, w, a, b, s, i, h), lambda: api.haflo_adapter_backward(y, x, w, a, b, s, i, h, 1.1)]
    one = torch.zeros(4, device="cuda")
    lab = api.haflo_label_logprobs
    bad += [
        lambda: lab(x, i.long()), lambda: lab(x, i[:2]), lambda: lab(x, i, 9), lambda: lab(torch.zeros(4, 100, device="cuda"), i, 65),
        lambda: lab(x[:, :0], i), lambda: lab(x.to(i32), i), lambda: lab(x, i, -1),
        lambda: api.haflo_label_logprobs_backward(x, i, one, one, one[:3]), lambda: api.haflo_label_logprobs_backward(x, i, one, one, one.half()),
        lambda: api.haflo_label_logprobs_backward(x, i, one, one, one, None, None, torch.zeros(4, 2, device="cuda")),
    ]
    for n, call in enumerate(bad):
        with pytest.raises(api.HafloError):
            call()
            pytest.fail("call %d was not refused" % n)
    # nothing to do is no error
    assert api.haflo_dropout(x[:0], 0.5, 1).shape == (0, 8)
    assert lab(x[:0], i[:0], 2)[4].shape == (0, 2)
    y, h = fwd(x[:0], w, a, b, s, i[:0])
    dx, da, db = api.haflo_adapter_backward(y, x[:0], w, a, b, s, i[:0], h)
    assert y.shape == (0, 6) and dx.shape == (0, 8) and da.dtype == f32 and not da.any() and not db.any()


def test_adapters_without_dx(api):
    g = torch.Generator(device="cuda").manual_seed(5)
    for rows in (7, 300):
        x, w = torch.randn(rows, 40, generator=g, device="cuda"), torch.randn(24, 40, generator=g, device="cuda")
        a, b = torch.randn(3, 5, 40, generator=g, device="cuda"), torch.randn(3, 24, 5, generator=g, device="cuda")
        scale, index = torch.ones(3, device="cuda"), (torch.arange(rows, device="cuda") % 4 - 1).to(torch.int32)
        y, h = api.haflo_adapter_forward(x, w, a, b, scale, index, 0.25, 9, 1)
        _, da, db = api.haflo_adapter_backward(y, x, w, a, b, scale, index, h, 0.25, 9, 1)
        none, da2, db2 = api.haflo_adapter_backward(y, x, w, a, b, scale, index, h, 0.25, 9, 1, need_dx=False)
        assert none is None and torch.equal(da, da2) and torch.equal(db, db2)


def test_adapters_past_32_bits(api):
    """x and dx of more than 4 GiB. Small integers: every sum is exact in 32 bits, so is each result before its rounding."""
    g = torch.Generator(device="cuda").manual_seed(6)
    rows, inner, outer, rank = 70000, 32768, 16, 2
    bf16 = torch.bfloat16

    def ints(*shape):
        return torch.randint(-1, 2, shape, generator=g, device="cuda", dtype=torch.int8).to(bf16)

    x, w, a, b = ints(rows, inner), ints(outer, inner), ints(2, rank, inner), ints(2, outer, rank)
    scale, index = torch.tensor([1.0, 2.0], device="cuda"), torch.randint(-1, 2, (rows,), generator=g, device="cuda").to(torch.int32)
    dy = ints(rows, outer)
    y, h = api.haflo_adapter_forward(x, w, a, b, scale, index)
    dx, da, db = api.haflo_adapter_backward(dy, x, w, a, b, scale, index, h)
    some = torch.cat([torch.arange(40), torch.arange(rows - 40, rows)]).cuda()
    xs, dys, of = x[some].double(), dy[some].double(), index[some].long()
    by = torch.where(of < 0, 0.0, scale.double()[of])
    hs = by[:, None] * (a.double()[of] @ xs[:, :, None])[..., 0]
    assert torch.equal(h[some].double(), hs)
    assert torch.equal(y[some], (xs @ w.double().t() + (b.double()[of] @ hs[:, :, None])[..., 0]).to(bf16))
    gs = by[:, None] * (dys[:, None, :] @ b.double()[of])[:, 0]
    assert torch.equal(dx[some], (dys @ w.double() + (gs[:, None, :] @ a.double()[of])[:, 0]).to(bf16))
    cols = torch.cat([torch.arange(9), torch.arange(inner - 9, inner)]).cuda()
    for p in range(2):
        mine = (index == p).nonzero()[:, 0]
        gp = scale[p].double() * (dy[mine].double() @ b[p].double())
        assert torch.equal(da[p][:, cols].double(), gp.t() @ x[mine][:, cols].double())
        assert torch.equal(db[p].double(), dy[mine].double().t() @ h[mine].double())


def test_homo_adapters_round_end_to_end(api):
    """Local steps of several parties, the encrypted average of their adapters, an answer under it: the decoded sum is the exact
    integer sum of the quantised weights, the parties' losses have fallen, and the answer's labels stand in order."""
    from paper_2107_13797_amd.examples import homo_adapters
    p, q = api.haflo_keygen(1024, 11)
    own, pub = api.haflo_ctx_create_private(p, q, 1024), api.haflo_ctx_create_public(p * q, 1024)
    res = homo_adapters.run_round(api, pub, own, parties=3, rows=150, width=72, labels=10, rank=4, steps=6, seed=3)
    own.close()
    pub.close()
    assert res["weights"] == 4 * (72 + 72 + 72 + 10)
    assert res["sum_q"] == res["want_sum_q"]
    assert res["loss"]["local"] < res["loss"]["before"]
    logps = [v for _, v in res["answer"]]
    assert len(set(i for i, _ in res["answer"])) == 5 and logps == sorted(logps, reverse=True) and max(logps) < 0


@pytest.mark.parametrize("case", [
    ("bf16", 65, 1033, 130, 16, 5, 0.1, "mixed", 1), ("f16", 130, 7, 65, 5, 3, 0.2, "mixed", 0), ("f32", 193, 300, 41, 33, 9, 0.0, "sorted", 3),
    ("bf16", 256, 520, 1001, 70, 2, 0.05, "mixed", 0), ("f32", 257, 65, 520, 4, 4, 0.1, "mixed", 0)], ids=str)
def test_adapters_some_rows(run, case):
    """Between one and four groups of 64 rows, and one row more."""
    cases.check_adapters(run, *case)


@pytest.mark.parametrize("case", [("bf16", 8200, 2051, 1, 0, 3, "ties"), ("f32", 8195, 2049, 0, 0, 0, "ties")], ids=str)
def test_labels_many_rows(run, case):
    """Rows that a wavefront takes for their number, longer than it takes otherwise."""
    cases.check_labels(run, *case)


@pytest.mark.parametrize("case", cases.ADAPTERS_SHORT_SUMS, ids=str)
def test_adapters_short_sums(run, case):
    cases.check_adapters(run, *case)


@pytest.mark.parametrize("rows", [200, 300])
@pytest.mark.parametrize("kind", cases.TYPES)
def test_adapters_cancelling(run, kind, rows):
    cases.check_adapters_cancelling(run, kind, rows)


@pytest.mark.parametrize("kind", cases.TYPES)
def test_adapters_own_infinities(run, kind):
    cases.check_adapters_own_infinities(run, kind)


@pytest.mark.parametrize("case", cases.LABELS_FAR, ids=str)
def test_labels_far(run, case):
    cases.check_labels_far(run, *case)


@pytest.mark.parametrize("cols", [2, 33, 700, 1500, 4000, 9000, 33001, 50000])
@pytest.mark.parametrize("kind", cases.TYPES)
def test_labels_gradient_in_place(api, kind, cols):
    """Every form of the gradient reads a row before it writes it."""
    g = torch.Generator(device="cuda").manual_seed(cols)
    logits = torch.randn(37, cols, generator=g, device="cuda").to(cases.TYPES[kind])
    label = torch.randint(-1, cols, (37,), generator=g, device="cuda").to(torch.int32)
    _, entropy, lse, _, index = api.haflo_label_logprobs(logits, label, 2)
    dlogp, dh, dtop = (torch.randn(37, *s, generator=g, device="cuda") for s in ((), (), (2,)))
    want = api.haflo_label_logprobs_backward(logits, label, lse, entropy, dlogp, dh, index, dtop)
    got = api.haflo_label_logprobs_backward(logits, label, lse, entropy, dlogp, dh, index, dtop, out=logits)
    assert got is logits and torch.equal(got, want)


def test_labels_far_columns(run):
    cases.check_labels_far_columns(run)


def test_in_place_refusals(api):
    wide = torch.zeros(4, 16, device="cuda")
    dense = torch.as_strided(wide, (4, 8), (8, 1))
    zero, label = torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for x, out in ((wide[:, :8], dense), (dense, wide[:, :8])):
        for call in (lambda: api.haflo_dropout(x, 0.5, 1, out=out), lambda: api.haflo_dropout(x.clone(), 0.5, 1, residual=x, out=out),
                     lambda: api.haflo_label_logprobs_backward(x, label, zero, zero, zero, out=out)):
            with pytest.raises(api.HafloError):
                call()
    assert api.haflo_dropout(wide[:, :8], 0.5, 1, out=wide[:, :8]).shape == (4, 8)


def test_labels_of_very_many_rows(api):
    """More rows than wavefronts fit one launch, whose lanes are counted in 32 bits."""
    rows, cols = 2 ** 26 + 5, 33
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    label = torch.zeros(rows, dtype=torch.int32, device="cuda")
    some = torch.tensor([0, 1, 2 ** 26 - 1, 2 ** 26, rows - 1], device="cuda")
    x[some, 5] = torch.arange(1, 6, device="cuda").bfloat16()
    label[some] = 5
    logp, entropy, lse, _, _ = api.haflo_label_logprobs(x, label)
    want = torch.full((rows,), math.log(cols), device="cuda")
    want[some] = torch.log(cols - 1 + torch.exp(torch.arange(1, 6, device="cuda").double())).float()
    assert float((lse - want).abs().max()) < 1e-5
    assert float((logp[some] - (torch.arange(1, 6, device="cuda") - want[some])).abs().max()) < 1e-5 and float((logp - x[:, 5].float() + want).abs().max()) < 1e-5


@pytest.mark.parametrize("case", cases.ADAPTERS_MANY + cases.ADAPTERS_TILES, ids=str)
def test_adapters_many(run, case):
    cases.check_adapters_of_many(run, *case)


@pytest.mark.parametrize("rows", [40, 300])
@pytest.mark.parametrize("kind", cases.TYPES)
def test_adapters_isolation(run, kind, rows):
    cases.check_adapters_isolation(run, kind, rows)


def test_graph_of_many_rows(api):
    """As test_side_stream_and_graph, with the kernels for more than 256 rows: their lists of rows, layouts and joined sums."""
    x, w, a, b, scale, index, dy = map(dev, cases.adapter_inputs("f16", 700, 1033, 130, 8, 5, "mixed", 0))

    def step():
        y, h = api.haflo_adapter_forward(x, w, a, b, scale, index, 0.2, 9, 1)
        return (y, h, *api.haflo_adapter_backward(dy, x, w, a, b, scale, index, h, 0.2, 9, 1))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for k in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(k)).to(x.dtype))
        index.copy_(torch.randint(-1, 5, index.shape, generator=torch.Generator().manual_seed(k)).to(torch.int32))
        torch.cuda.synchronize()
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))


FAR_GRADIENT = [("bf16", 70000), ("f16", 70000), ("f32", 36000)]


@pytest.mark.parametrize("kind,rows", FAR_GRADIENT)
def test_adapters_gradient_past_32_bits(api, kind, rows):
    """dy of more than 4 GiB, with dropout. Small integers and a factor of two: every sum is exact in 32 bits."""
    g = torch.Generator(device="cuda").manual_seed(8)
    inner, outer, rank, dtype = 16, 32768, 2, cases.TYPES[kind]

    def ints(*shape):
        return torch.randint(-1, 2, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)

    x, w, a, b, dy = ints(rows, inner), ints(outer, inner), ints(2, rank, inner), ints(2, outer, rank), ints(rows, outer)
    scale, index = torch.tensor([1.0, 2.0], device="cuda"), torch.randint(-1, 2, (rows,), generator=g, device="cuda").to(torch.int32)
    y, h = api.haflo_adapter_forward(x, w, a, b, scale, index, 0.5, 77)
    dx, da, db = api.haflo_adapter_backward(dy, x, w, a, b, scale, index, h, 0.5, 77)
    kept = api.haflo_dropout(torch.ones_like(x), 0.5, 77).double()
    some = torch.cat([torch.arange(40), torch.arange(rows - 40, rows)]).cuda()
    dys, of = dy[some].double(), index[some].long()
    by = torch.where(of < 0, 0.0, scale.double()[of])
    gs = by[:, None] * (dys[:, None, :] @ b.double()[of])[:, 0]
    assert torch.equal(dx[some], (dys @ w.double() + kept[some] * (gs[:, None, :] @ a.double()[of])[:, 0]).to(dtype))
    cols = torch.cat([torch.arange(9), torch.arange(outer - 9, outer)]).cuda()
    for p in range(2):
        mine = (index == p).nonzero()[:, 0]
        assert torch.equal(db[p][cols].double(), dy[mine][:, cols].double().t() @ h[mine].double())


FAR_FORWARD = [("f16", 70000), ("f32", 36000), ("bf16", 70000)]  # the last by test_adapters_past_32_bits


@pytest.mark.parametrize("kind,rows", FAR_FORWARD[:2])
def test_adapters_past_32_bits_of_other_types(api, kind, rows):
    """x of more than 4 GiB in the other types, as test_adapters_past_32_bits."""
    g = torch.Generator(device="cuda").manual_seed(9)
    inner, outer, rank, dtype = 32768, 16, 2, cases.TYPES[kind]

    def ints(*shape):
        return torch.randint(-1, 2, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)

    x, w, a, b = ints(rows, inner), ints(outer, inner), ints(2, rank, inner), ints(2, outer, rank)
    scale, index = torch.tensor([1.0, 2.0], device="cuda"), torch.randint(-1, 2, (rows,), generator=g, device="cuda").to(torch.int32)
    y, h = api.haflo_adapter_forward(x, w, a, b, scale, index)
    some = torch.cat([torch.arange(40), torch.arange(rows - 40, rows)]).cuda()
    xs, of = x[some].double(), index[some].long()
    by = torch.where(of < 0, 0.0, scale.double()[of])
    hs = by[:, None] * (a.double()[of] @ xs[:, :, None])[..., 0]
    assert torch.equal(h[some].double(), hs)
    assert torch.equal(y[some], (xs @ w.double().t() + (b.double()[of] @ hs[:, :, None])[..., 0]).to(dtype))


@pytest.mark.parametrize("case", cases.ADAPTERS_FORMS, ids=str)
def test_adapters_forms(run, case):
    cases.check_adapters_of_many(run, *case)


@pytest.mark.parametrize("case", cases.LABELS_FORMS, ids=str)
def test_labels_forms(run, case):
    cases.check_labels_far(run, *case)
