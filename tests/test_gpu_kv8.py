"""The paged 8-bit key/value cache through the C ABI, against oracle/kv8_oracle.py: plan, rotary rows, append and attention, each at
the sizes and contents where it can go wrong, and a run of them together.

Tolerances, derived before the first run.
  plan, append: none.  Whole numbers, and binary32 steps that are each one correctly rounded operation.
  rotary rows: the angle is off by 2^-25 turns + sincospif's 2 ulp (together under 2^-21.8 of the pair's size), products and
      sum in binary32: (2^-21 |a| + 2^-21 |b|) m, then the output's rounding, half of eps.
  attention, against 64 bits on the cached values, with w the exact weights, T = sum w |V|, A = sum w 128 vs, B = scale max_p sum_d |q_d| |K_d|,
      C = scale max|q| max_p sum_d |K_d|:
      a score is off by ds <= 2^-16 C (q in 16 bits against its row's largest magnitude, the product with the codes exact) + 2^-20 (1 + B)
      (products with the scales, differences, ex2); a weight by a factor within e^ds, in numerator and denominator: 3 ds T;
      weights in 16 bits against their tile's largest: each off by 2^-17 of it, 32 in a tile, so at most 2^-12 A in the numerator and 2^-12 T
      through the denominator (the sum is of the rounded weights); sums over tiles in binary32: 2^-18 (T + A); then the output's rounding.
"""
import numpy as np
import pytest

from oracle import kv8_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TD = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def aq():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2605_24011_b200 import aq as mod
    return mod


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


# ---- plan ----------------------------------------------------------------------------------------------------------
class Planner:
    def __init__(self, aq, n, width, page, cap, n_rows, n_free):
        self.aq, self.page, self.n_rows, self.cap = aq, page, n_rows, cap
        self.lens, self.table = [0] * n, [[-1] * width for _ in range(n)]
        self.free = list(np.random.default_rng(n * 31 + width).permutation(n_free) + 7)
        self.d = dict(lens=_i32(self.lens), table=_i32(self.table), free=_i32(self.free + [-5] * (cap - n_free)), n_free=_i32([n_free]),
                      row_start=_i32([9] * (n + 1)), pos=_i32([9] * n_rows), new=_i32([0] * n))

    def call(self, stream=None):
        d = self.d
        self.aq.aq_kv8_plan(d["lens"], d["new"], d["table"], d["free"], d["n_free"], self.page, d["lens"], d["n_free"], d["row_start"], d["pos"], stream)

    def expect(self, new):
        """The oracle's step; False where it does not fit."""
        got = O.plan(self.lens, new, self.table, self.free, self.page, self.n_rows, self.cap)
        if got is None:
            row_start, pos = [0] * (len(self.lens) + 1), [-1] * self.n_rows
        else:
            self.lens, self.table, self.free, row_start, pos = got
        d = self.d
        assert d["lens"].tolist() == self.lens and d["row_start"].tolist() == row_start and d["pos"].tolist() == pos
        assert d["table"].tolist() == self.table and d["n_free"].tolist() == [len(self.free)]
        assert d["free"].tolist()[: len(self.free)] == self.free
        return got is not None

    def step(self, new):
        self.d["new"].copy_(_i32(new))
        self.call()
        return self.expect(new)


@pytest.mark.parametrize("n,width,page,n_rows", ((1, 1, 32, 1), (3, 5, 32, 64), (33, 4, 64, 500), (200, 9, 128, 4096), (1024, 3, 1024, 6000)))
def test_plan_over_many_steps(aq, n, width, page, n_rows):
    g = np.random.default_rng(n)
    p = Planner(aq, n, width, page, n * width + 3, n_rows, n * width)
    fits = 0
    for step in range(30):
        new = []
        room, loose = n_rows, step % 5 == 4   # now and then a step that may not fit
        for b in range(n):
            kind = g.integers(0, 10)
            add = -1 if kind == 0 else 0 if kind < 3 else 1 if kind < 7 else int(g.integers(0, 2 * page))
            if not loose:
                add = min(add, width * page - p.lens[b], room)
            new.append(add)
            room -= max(add, 0)
        ok = p.step(new)
        fits += ok
        if ok:
            aq.aq_check()
        else:
            with pytest.raises(aq.AqError) as e:
                aq.aq_check()
            assert e.value.status == aq.AQ_ERR_RANGE
            aq.aq_check()   # reported once
    assert fits > 0


def test_plan_all_or_nothing(aq):
    for new, lens, n_free, cap in (([3, 200], [0, 0], 9, 16), ([65, 65], [0, 0], 3, 16), ([-1, 1], [64, 0], 5, 6), ([-2, 1], [0, 0], 5, 16),
                                   ([2 ** 31 - 1, 1], [0, 0], 5, 16), ([1, 1], [-1, 0], 5, 16), ([0, 0], [129, 0], 5, 16)):
        p = Planner(aq, 2, 2, 64, cap, 150, n_free)
        p.lens = list(lens)
        p.d["lens"].copy_(_i32(lens))
        if lens[0] == 64:
            p.table[0][0] = 40
            p.d["table"].copy_(_i32(p.table))
            p.free += [1]                    # six of six places taken: nothing can be given back
            p.d["free"][:6].copy_(_i32(p.free))
            p.d["n_free"].fill_(6)
        assert not p.step(new), (new, lens)
        with pytest.raises(aq.AqError):
            aq.aq_check()


def test_plan_replayed(aq):
    """A captured step follows the arrays that it is replayed on."""
    p = Planner(aq, 4, 6, 32, 30, 40, 24)
    assert p.step([5, 0, 1, 2])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            p.call()
    for new in ([1, 1, 1, 1], [-1, 30, 0, 1], [7, -1, 3, 3]):
        p.d["new"].copy_(_i32(new))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert p.expect(new)
    aq.aq_check()


# ---- rotary rows ---------------------------------------------------------------------------------------------------
ROPE = [  # rows, heads, extra heads between rows, head dim, rot, layout, scaling, factor, far, src, dst
    (1, 64, 0, 128, 128, "half", "none", 1.0, 4096, "f16", "f16"),
    (37, 40, 8, 128, 64, "pairs", "linear", 4.0, 8000, "f32", "f16"),
    (50, 9, 1, 256, 256, "half", "parts", 16.0, 1000000, "bf16", "bf16"),
    (1000, 2, 0, 64, 30, "half", "base", 2.5, 100000, "f16", "f16"),
    (13, 3, 1, 80, 38, "pairs", "none", 1.0, 2 ** 31 - 1, "f32", "f32"),
    (65, 5, 2, 33, 2, "half", "none", 1.0, 70, "bf16", "bf16"),
    (3, 1, 0, 2, 2, "pairs", "parts", 8.0, 9000, "f32", "bf16"),
    (700, 17, 0, 96, 96, "pairs", "linear", 1.5, 30000, "f16", "f16"),
    (4096, 4, 0, 128, 112, "half", "none", 1.0, 50000, "bf16", "bf16"),
]


@pytest.mark.parametrize("case", ROPE, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("how", ("out", "in place", "one element off"))
def test_rope_rows(aq, case, how):
    T, H, extra, D, rot, layout, scaling, factor, far, src, dst = case
    if how == "in place" and src != dst:
        pytest.skip("in place has one type")
    g = np.random.default_rng(T * 7 + D)
    off = 1 if how == "one element off" else 0      # rows that are not 16-byte aligned
    flat = torch.from_numpy(g.standard_normal(T * (H + extra) * D + 8).astype(np.float32)).to(TD[src]).cuda()
    buf = flat[off: off + T * (H + extra) * D].view(T, H + extra, D)
    x = buf[:, :H]
    before = buf.clone()
    pos = g.integers(0, far + 1, T) if far < 2 ** 31 - 1 else g.integers(2 ** 31 - 5000, 2 ** 31, T)
    pos[0], pos[-1] = min(far, pos.max()), 0
    if T > 4:
        pos[2], pos[T // 2] = -1, -(2 ** 31)
    rope = aq.aq_rope_setup(rot, layout=layout, scaling=scaling, factor=factor, trained=4096)
    out = x if how == "in place" else torch.full((T, H, D), 7.0, dtype=TD[dst], device="cuda")
    left = out.clone()
    got = aq.aq_rope_rows(rope, x, _i32(pos), None if how == "in place" else out)
    assert got is out
    xn = before[:, :H].double().cpu().numpy()
    m = 0.1 * np.log(factor) + 1 if scaling == "parts" else 1.0
    want = O.rope_rows(xn, pos, O.rope_frequencies(rot, 10000.0, scaling, factor, 4096), layout, m)
    a, b = (np.arange(rot // 2), np.arange(rot // 2) + rot // 2) if layout == "half" else (np.arange(0, rot, 2), np.arange(1, rot, 2))
    size = np.zeros_like(xn)
    size[..., a] = size[..., b] = (np.abs(xn[..., a]) + np.abs(xn[..., b])) * m
    # (a binary64 angle of 2^31 radians is itself off by 2^-22 radians in the oracle and by the frequency's 2^-52 in the call)
    lim = (2.0 ** -21 + (2.0 ** -19 if far == 2 ** 31 - 1 else 0)) * size + HALF_STEP[dst] * np.abs(want) * 1.001 + 1e-12 + (2.0 ** -25 if dst == "f16" else 0)
    real = pos >= 0
    gn = got.double().cpu().numpy()
    assert np.all(np.abs(gn - want)[real] <= lim[real]), np.max((np.abs(gn - want) / np.maximum(lim, 1e-30))[real])
    assert torch.equal(got[~torch.from_numpy(real).cuda()], left[~torch.from_numpy(real).cuda()])
    assert torch.equal(buf[:, H:], before[:, H:])    # what lies between the rows is not touched
    if how == "in place":
        return
    assert torch.equal(x, before[:, :H])


@pytest.mark.parametrize("how,case", (("in place", (4000, 40, 8, 128, 128, "half", "parts", 8.0, 120000, "bf16", "bf16")),
                                      ("out", (2500, 40, 0, 128, 64, "pairs", "none", 1.0, 4096, "f32", "f16")),
                                      ("one element off", (1500, 9, 1, 81, 38, "pairs", "none", 1.0, 4096, "f16", "f16"))), ids=str)
def test_rope_rows_with_several_turns_per_thread(aq, how, case):
    test_rope_rows(aq, case, how)


# ---- a cache in use ------------------------------------------------------------------------------------------------
def _up11(x):
    return ((x.contiguous().view(torch.int32) + 0x1FFF) & ~0x1FFF).view(torch.float32)


class Served:
    """Requests with cached positions in pages of no order; pages that nobody holds are full of what must not be used."""

    def __init__(self, aq, lens, Hkv, D, page, seed, spare=3, outliers=True):
        g = torch.Generator().manual_seed(seed)
        held = [-(-L // page) for L in lens]
        n = sum(held) + spare
        x = torch.randn(n, Hkv, page // 32, 32, D, generator=g) * (0.2 + 2 * torch.rand(1, Hkv, 1, 1, D, generator=g))
        y = torch.randn(n, Hkv, page // 32, 32, D, generator=g) * (0.1 + 3 * torch.rand(n, Hkv, page // 32, 1, 1, generator=g))
        if outliers:
            y[torch.rand(y.shape, generator=g) < 0.001] *= 20
        self.ks, self.vs = _up11(x.abs().amax((3, 4)) / 127), _up11(y.abs().amax((3, 4)) / 127)
        self.k = torch.round(x / self.ks[..., None, None]).to(torch.int8).view(n, Hkv, page, D)
        self.v = torch.round(y / self.vs[..., None, None]).to(torch.int8).view(n, Hkv, page, D)
        order = torch.randperm(n, generator=g).tolist()
        self.table = [[order.pop() for _ in range(h)] + [-7] * (max(held + [1]) - h) for h in held]
        for p in order:                       # pages of nobody
            self.ks[p] = float("nan")
            self.vs[p] = float("inf")
        for b, L in enumerate(lens):          # blocks behind a request's last position
            if held[b]:
                first = -(-(L % page) // 32) if L % page else page // 32
                self.ks[self.table[b][held[b] - 1], :, first:] = float("nan")
                self.vs[self.table[b][held[b] - 1], :, first:] = float("nan")
        self.lens, self.page, self.Hkv, self.D = list(lens), page, Hkv, D
        self.cache = aq.Kv8Cache(self.k.cuda(), self.v.cuda(), self.ks.cuda(), self.vs.cuda())

    def batch(self, aq, rows=None):
        """rows: new tokens per request, or None (the same for all)."""
        self.rows = rows
        rs = None if rows is None else _i32([0] + list(np.cumsum(rows)))
        return aq.Kv8Batch(_i32(self.lens), _i32(self.table), rs)


def _attn_reference(s, q, rows, scale):
    """want and the tolerance without the output's rounding, for real rows; q float64 [T][H][D]."""
    T, H, D = q.shape
    G = H // s.Hkv
    scale = scale if scale > 0 else 1 / np.sqrt(D)
    want, tol = np.zeros((T, H, D)), np.zeros((T, H, D))
    t = 0
    for b, n in enumerate(rows):
        if n == 0:
            continue
        L = s.lens[b]
        K, V = O.gather(s.k.numpy(), s.ks.numpy(), s.table[b], L), O.gather(s.v.numpy(), s.vs.numpy(), s.table[b], L)
        Vo = O.gather(np.full(s.k.shape, 128, np.int16), s.vs.numpy(), s.table[b], L)
        for i in range(n):
            see = max(0, L - n + i + 1)
            for h in range(H):
                kv, qh = h // G, q[t + i, h]
                want[t + i, h], T_, w = O.attn(qh, K[kv, :see], V[kv, :see], scale)
                if see == 0:
                    continue
                A = w @ Vo[kv, :see]
                B = scale * np.max(np.abs(K[kv, :see]) @ np.abs(qh))
                C = scale * np.max(np.abs(qh)) * np.max(np.abs(K[kv, :see]).sum(1))
                ds = 2.0 ** -16 * C + 2.0 ** -20 * (1 + B)
                tol[t + i, h] = (2.0 ** -12 + 3 * ds + 2.0 ** -18) * T_ + (2.0 ** -12 + 2.0 ** -18) * A + 1e-30
        t += n
    return want, tol


def _check_attn(aq, lens, Hkv, G, D, page, rows=None, name="f16", seed=0, scale=0.0, outs=None, tail=2, qscale=1.0, strided=False, scratch=None):
    s = Served(aq, lens, Hkv, D, page, seed)
    batch = s.batch(aq, rows)
    each = rows if rows is not None else [1] * len(lens)
    T, H = sum(each) + (tail if rows is not None else 0), Hkv * G
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn(T, H, D, generator=g) * qscale).to(TD[name])
    want, tol = _attn_reference(s, q.double().numpy(), each, scale)
    scratch = aq.aq_kv8_scratch() if scratch is None else scratch
    real = sum(each)
    for out_name in outs or ("f32", name):
        if strided:
            qd = torch.zeros(T, H + 2, D, dtype=TD[name], device="cuda")
            qd[:, 1: H + 1] = q.cuda()
            qd = qd[:, 1: H + 1]
            out = torch.full((T, H + 1, D), float("nan"), dtype=TD[out_name], device="cuda")[:, :H]
        else:
            qd, out = q.cuda(), torch.full((T, H, D), float("nan"), dtype=TD[out_name], device="cuda")
        for again in range(2):
            aq.aq_kv8_attn(s.cache, batch, qd, out, scratch, scale)
            first = out.clone() if again == 0 else first
        aq.aq_check()
        assert torch.equal(first.nan_to_num(9.0), out.nan_to_num(9.0))        # sums in a fixed order
        got = out.double().cpu().numpy()
        assert np.all(np.isnan(got[real:])), "rows behind the last request's were written"
        err = np.abs(got[:real] - want[:real])
        lim = tol[:real] + HALF_STEP[out_name] * (np.abs(want[:real]) + tol[:real]) + (2.0 ** -25 if out_name == "f16" else 0)
        assert np.all(np.isfinite(got[:real])) and np.all(err <= lim), f"{out_name}: worst {np.max(err / np.maximum(lim, 1e-300)):.3g} tolerances"
    return scratch


@pytest.mark.parametrize("name", ("f16", "bf16"))
@pytest.mark.parametrize("D", (64, 128, 256))
def test_attention_lengths(aq, D, name):
    # one position; a tile less one, whole, and one more; pages' edges; nothing
    _check_attn(aq, [1, 31, 32, 33, 0, 63, 64, 65, 128, 129, 200], 2, 4, D, 64, name=name, seed=D)


@pytest.mark.parametrize("D", (64, 128, 256))
@pytest.mark.parametrize("Hkv,G", ((1, 1), (1, 8), (1, 16), (3, 3), (8, 4), (5, 7), (2, 20)))
def test_attention_heads(aq, Hkv, G, D):
    _check_attn(aq, [100, 7, 300], Hkv, G, D, 32, name="bf16" if G % 2 else "f16", seed=G + D, outs=("f32",))


@pytest.mark.parametrize("page", (32, 64, 256, 1024))
def test_attention_pages(aq, page):
    _check_attn(aq, [1500, 1024, 33, page, page + 1, page - 1], 2, 2, 128, page, seed=page)


@pytest.mark.parametrize("D", (64, 128, 256))
def test_attention_ragged_rows(aq, D):
    # requests without rows, without positions, with more rows than positions; rows that fill several blocks of query rows
    _check_attn(aq, [40, 0, 5, 300, 90, 17, 0, 64], 2, 3, D, 32, rows=[3, 0, 5, 8, 0, 17, 2, 1], seed=D, strided=True)
    _check_attn(aq, [40, 3, 5], 2, 3, D, 32, rows=[5, 8, 0], name="bf16", seed=D + 1, tail=0)


@pytest.mark.parametrize("lens", ([5000], [20011], [3, 9000, 1, 0, 700]), ids=str)
@pytest.mark.parametrize("Hkv,G,D", ((1, 1, 64), (1, 8, 256), (1, 12, 128), (4, 2, 128)))
def test_attention_long(aq, lens, Hkv, G, D):
    # items that many CTAs share: merged in groups, then the groups
    _check_attn(aq, lens, Hkv, G, D, 128, seed=Hkv, outs=("f32",))


def test_attention_many_requests(aq):
    g = np.random.default_rng(5)
    lens = [int(v) for v in g.integers(0, 70, 1024)]
    _check_attn(aq, lens, 1, 2, 64, 32, seed=5, outs=("f32",))
    _check_attn(aq, lens[:300], 1, 2, 128, 32, rows=[int(v) for v in g.integers(0, 4, 300)], seed=6, outs=("f16",))


@pytest.mark.parametrize("Hkv,G,D,rows", ((8, 4, 128, 1), (8, 4, 128, 2), (8, 4, 128, 3), (8, 4, 128, 4), (6, 3, 64, 5), (5, 8, 256, 1), (5, 2, 256, 1), (9, 5, 64, 2)))
def test_attention_runs_over_several_items(aq, Hkv, G, D, rows):
    # items shared by CTAs and warps, runs that end one and begin the next, for every number of query rows per pass
    lens = [2100, 1999, 2500, 31, 1900, 2222]
    _check_attn(aq, lens, Hkv, G, D, 128, rows=[rows] * len(lens), seed=rows + D, outs=("f32",), tail=1)


def test_attention_many_requests_with_long_ones_among_them(aq):
    g = np.random.default_rng(15)
    lens = [int(v) for v in g.integers(0, 300, 60)]
    lens[7], lens[41], lens[59] = 7000, 5003, 4097
    _check_attn(aq, lens, 2, 2, 64, 64, seed=15, outs=("f32",))
    _check_attn(aq, lens, 2, 2, 128, 64, rows=[min(L, int(v)) for L, v in zip(lens, g.integers(0, 9, 60))], seed=16, outs=("f32",))


@pytest.mark.parametrize("n,Hkv,L", ((25, 4, 1700), (38, 4, 1700), (19, 8, 1601), (75, 2, 1300), (100, 3, 1300)))
def test_attention_items_that_are_alike(aq, n, Hkv, L):
    """100, 152, 152, 150 and 300 items of one length: whole ones for every CTA where that keeps most of them busy, parts otherwise."""
    _check_attn(aq, [L] * n, Hkv, 2, 64, 64, seed=n)


def test_attention_more_rows_than_a_pass_takes(aq):
    _check_attn(aq, [5000, 40, 2200], 1, 4, 128, 128, rows=[40, 2, 1], seed=17, outs=("f32",))
    _check_attn(aq, [3000, 40], 2, 8, 256, 64, rows=[5, 3], seed=18, outs=("f32",))


def test_attention_a_prompt(aq):
    _check_attn(aq, [150, 70], 2, 2, 128, 64, rows=[150, 33], seed=8, outs=("f32",))


def test_attention_peaked_flat_and_scaled(aq):
    _check_attn(aq, [700, 900], 2, 4, 128, 64, seed=1, qscale=8.0)     # a few positions have all the weight
    _check_attn(aq, [700, 900], 2, 4, 128, 64, seed=2, qscale=0.0)     # the mean of the values
    _check_attn(aq, [700, 900], 2, 4, 64, 64, seed=3, scale=0.7)
    _check_attn(aq, [700], 2, 4, 128, 64, name="bf16", seed=4, qscale=1e30, scale=1e-30)   # beyond binary16 on the way
    _check_attn(aq, [700], 2, 4, 128, 64, name="bf16", seed=4, qscale=1e-30, scale=1e30)


def test_attention_many_light_positions(aq):
    """One position with nearly all weight and 40000 that share the rest, each 2^-27 of it: what they add is not lost."""
    L, D, page = 40001, 64, 1024
    s = Served(aq, [L], 1, D, page, 3)
    q = torch.zeros(1, 1, D, dtype=torch.float16)
    q[0, 0, 0] = 1.0
    s.k.zero_()
    s.ks.fill_(2.0 ** -6)
    s.k[s.table[0][20], 0, 17, 0] = 64            # score 1 * 64 / 64 * scale
    s.v.fill_(64)
    s.vs.fill_(2.0 ** -6)
    s.v[s.table[0][20], 0, 17] = 0                # all of the output comes from the light ones
    scale = 27 * float(np.log(2))
    s.cache = aq.Kv8Cache(s.k.cuda(), s.v.cuda(), s.ks.cuda(), s.vs.cuda())
    out = torch.empty(1, 1, D, dtype=torch.float32, device="cuda")
    aq.aq_kv8_attn(s.cache, s.batch(aq), q.cuda(), out, aq.aq_kv8_scratch(), scale)
    w = 40000 * 2.0 ** -27
    # The weights are powers of two; ex2 is within 2^-22, the scores' 27 within 2^-18 of themselves: 2^-12 w.  In the heavy position's tile
    # 31 light ones lie under 2^-17 of it and are lost, in every other tile they are the largest: 31 * 2^-27 = 2.31e-7 < 2^-22 * 2.
    assert np.all(np.abs(out.double().cpu().numpy() - w / (1 + w)) <= 2.0 ** -12 * w + 2.0 ** -22 * 2)


def test_attention_masked_blocks_may_hold_anything(aq):
    """A block that only later tokens see, with NaN for a scale, leaves earlier tokens as they are; a NaN in a query row stays in its row."""
    s = Served(aq, [66], 1, 128, 64, 9)
    q = torch.randn(3, 2, 128).half()
    want, tol = _attn_reference(s, q.double().numpy(), [3], 0.0)
    page = s.table[0][1]                          # positions 64, 65: seen by the last two tokens
    for which in (s.ks, s.vs):
        kept = which[page, 0, 0].item()
        which[page, 0, 0] = float("nan")
        s.cache = aq.Kv8Cache(s.k.cuda(), s.v.cuda(), s.ks.cuda(), s.vs.cuda())
        out = torch.empty(3, 2, 128, dtype=torch.float32, device="cuda")
        aq.aq_kv8_attn(s.cache, s.batch(aq, [3]), q.cuda(), out, aq.aq_kv8_scratch())
        got = out.double().cpu().numpy()
        assert np.all(np.abs(got[0] - want[0]) <= tol[0] * 1.01) and np.all(np.isnan(got[1:]))
        which[page, 0, 0] = kept
    s.cache = aq.Kv8Cache(s.k.cuda(), s.v.cuda(), s.ks.cuda(), s.vs.cuda())
    q[1, 0, 5] = float("nan")
    q[2, 1, 7] = float("inf")
    aq.aq_kv8_attn(s.cache, s.batch(aq, [3]), q.cuda(), out, aq.aq_kv8_scratch())
    got = out.double().cpu().numpy()
    bad = np.zeros((3, 2), bool)
    bad[1, 0] = bad[2, 1] = True
    assert np.all(np.isnan(got[bad])) and np.all(np.abs(got - want)[~bad] <= tol[~bad] * 1.01)
    aq.aq_check()


def test_attention_pages_outside_the_pool_are_not_followed(aq):
    s = Served(aq, [200, 100], 2, 128, 32, 11)
    q = torch.randn(2, 4, 128).half().cuda()
    out = torch.full((2, 4, 128), float("nan"), dtype=torch.float32, device="cuda")
    scratch = aq.aq_kv8_scratch()
    for bad in (-1, s.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        table = [list(r) for r in s.table]
        table[0][3] = bad
        aq.aq_kv8_attn(s.cache, aq.Kv8Batch(_i32(s.lens), _i32(table)), q, out, scratch)
        with pytest.raises(aq.AqError) as e:
            aq.aq_check()
        assert e.value.status == aq.AQ_ERR_RANGE
        # those 32 positions count as masked
        K, V = (O.gather(c.numpy(), sc.numpy(), s.table[0], 200) for c, sc in ((s.k, s.ks), (s.v, s.vs)))
        keep = np.r_[0:96, 128:200]
        for h in range(4):
            want, T, _ = O.attn(q[0, h].double().cpu().numpy(), K[h // 2][keep], V[h // 2][keep], 1 / np.sqrt(128))
            assert np.all(np.abs(out[0, h].double().cpu().numpy() - want) <= 2.0 ** -9 * (T + 1))
    # lengths that do not fit the table are held inside it, row marks inside the step
    aq.aq_kv8_attn(s.cache, aq.Kv8Batch(_i32([10 ** 9, -5]), _i32(s.table)), q, out, scratch)
    with pytest.raises(aq.AqError):
        aq.aq_check()
    assert torch.equal(out[1], torch.zeros_like(out[1]))
    aq.aq_kv8_attn(s.cache, aq.Kv8Batch(_i32(s.lens), _i32(s.table), _i32([-9, 1, 50])), q, out, scratch)
    aq.aq_check()
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("n", (3, 41))
def test_attention_row_marks_that_name_too_many_rows(aq, n):
    """Marks that descend: requests that have more rows between them than the step has.  Nothing is written."""
    s = Served(aq, [100] * n, 2, 128, 32, 17)
    q = torch.randn(2, 4, 128).half().cuda()
    out = torch.full((2, 4, 128), float("nan"), dtype=torch.float32, device="cuda")
    scratch = aq.aq_kv8_scratch()
    aq.aq_kv8_attn(s.cache, aq.Kv8Batch(_i32(s.lens), _i32(s.table), _i32([0, 2] * ((n + 1) // 2))), q, out, scratch)
    with pytest.raises(aq.AqError) as e:
        aq.aq_check()
    assert e.value.status == aq.AQ_ERR_RANGE and bool(torch.isnan(out).all())
    marks = [0] * (n - 1) + [1, 2]
    aq.aq_kv8_attn(s.cache, aq.Kv8Batch(_i32(s.lens), _i32(s.table), _i32(marks)), q, out, scratch)
    aq.aq_check()
    want, tol = _attn_reference(s, q.double().cpu().numpy(), [0] * (n - 2) + [1, 1], 0.0)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol * (1 + 2.0 ** -24) + 2.0 ** -24 * np.abs(want))


@pytest.mark.parametrize("D", (64, 256))
def test_attention_tiny_queries_and_huge_keys(aq, D):
    """bfloat16 rows under 2^-113 are in steps of 1 / 3e38.  Beside the module's tolerance: a score is off by half of that per element, under
    2^-128 scale sum_d |K_d|, and by 2^-19 of itself more, as the step's product with the scale is a subnormal of 20 bits."""
    s = Served(aq, [90], 1, D, 64, 18, spare=0)
    up = 2.0 ** 114
    s.ks = s.ks * up
    s.cache = aq.Kv8Cache(s.k.cuda(), s.v.cuda(), s.ks.cuda(), s.vs.cuda())
    q = (torch.randn(1, 6, D, generator=torch.Generator().manual_seed(18)) * 2.0 ** -116).to(torch.bfloat16)
    out = torch.empty(1, 6, D, dtype=torch.float32, device="cuda")
    aq.aq_kv8_attn(s.cache, s.batch(aq), q.cuda(), out, aq.aq_kv8_scratch())
    aq.aq_check()
    qh = q.double().numpy()
    want, tol = _attn_reference(s, qh, [1], 0.0)
    K, V = (O.gather(c.numpy(), sc.numpy(), s.table[0], 90) for c, sc in ((s.k, s.ks), (s.v, s.vs)))
    for h in range(6):
        _, T, _ = O.attn(qh[0, h], K[0], V[0], 1 / np.sqrt(D))
        B = np.max(np.abs(K[0]) @ np.abs(qh[0, h])) / np.sqrt(D)
        ds = 2.0 ** -128 * np.max(np.abs(K[0]).sum(1)) / np.sqrt(D) + 2.0 ** -19 * B
        tol[0, h] += 3 * ds * T
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol * (1 + 2.0 ** -24) + 2.0 ** -24 * np.abs(want))


def test_attention_far_into_a_large_pool(aq):
    """Offsets past 2^32 bytes: pages at both ends of a pool of 4.6 GB of keys."""
    page, Hkv, D = 1024, 8, 256
    n = 2 ** 32 // (page * Hkv * D) + 40
    k, v = (torch.empty(n, Hkv, page, D, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((n, Hkv, page // 32), float("nan"), device="cuda") for _ in range(2))
    s = Served(aq, [1500], Hkv, D, page, 21)
    there = [n - 1, 3]
    for i, p in enumerate(there):
        k[p], v[p], ks[p], vs[p] = (x[s.table[0][i]].cuda() for x in (s.k, s.v, s.ks, s.vs))
    q = torch.randn(1, Hkv, D).half()
    want, tol = _attn_reference(s, q.double().numpy(), [1], 0.0)
    out = torch.empty(1, Hkv, D, dtype=torch.float32, device="cuda")
    cache = aq.Kv8Cache(k, v, ks, vs)
    aq.aq_kv8_attn(cache, aq.Kv8Batch(_i32([1500]), _i32([there])), q.cuda(), out, aq.aq_kv8_scratch())
    aq.aq_check()
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol * 1.01)
    # and what an append writes there
    x = torch.randn(2, 2, Hkv, D, device="cuda").half()
    aq.aq_kv8_append(cache, aq.Kv8Batch(_i32([1026]), _i32([[7, n - 1]])), x[0], x[1])
    aq.aq_check()
    kk, kks = O.append_block(np.zeros((32, D), np.int8), 0, 0, x[0, :, 3].float().cpu().numpy())
    assert np.array_equal(k[n - 1, 3, :2].cpu().numpy(), kk[:2]) and float(ks[n - 1, 3, 0]) == float(kks)


def test_attention_streams_and_graphs(aq):
    """Two captured graphs with scratch of their own, replayed at the same time on two streams, on lengths that change."""
    one, two = Served(aq, [3000, 800], 4, 128, 64, 31), Served(aq, [2500, 1300], 4, 128, 64, 32)
    jobs = []
    for s in (one, two):
        q = torch.randn(2, 16, 128).half().cuda()
        b = s.batch(aq)
        j = dict(s=s, q=q, b=b, out=torch.zeros(2, 16, 128, dtype=torch.float16, device="cuda"), scratch=aq.aq_kv8_scratch(), stream=torch.cuda.Stream())
        aq.aq_kv8_attn(s.cache, b, q, j["out"], j["scratch"])
        torch.cuda.synchronize()
        j["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(j["graph"], stream=j["stream"]):
            for _ in range(3):
                aq.aq_kv8_attn(s.cache, b, q, j["out"], j["scratch"])
        jobs.append(j)
    for lens in ([3000, 800], [1, 500], [2999, 0], [64, 65]):
        for j in jobs:
            j["s"].lens = [min(a, m) for a, m in zip(lens, j["s"].lens)] if lens[0] > 64 else lens
            j["b"].lens.copy_(_i32(j["s"].lens))
            j["s"].now = list(j["s"].lens)
        torch.cuda.synchronize()
        for _ in range(5):
            for j in jobs:
                with torch.cuda.stream(j["stream"]):
                    j["graph"].replay()
        torch.cuda.synchronize()
        for j in jobs:
            s = j["s"]
            # (what lay behind the old lengths is cached values all the same: only the last block's scale was a NaN)
            want, tol = _attn_reference(s, j["q"].double().cpu().numpy(), [1, 1], 0.0)
            got = j["out"].double().cpu().numpy()
            assert np.all(np.abs(got - want) <= tol * 1.01 + HALF_STEP["f16"] * np.abs(want) + 2.0 ** -25)
    aq.aq_check()


# ---- append --------------------------------------------------------------------------------------------------------
def _check_append(aq, lens, rows, Hkv, D, page, name, seed, extra=0, values=None):
    """lens: with the new tokens."""
    s = Served(aq, lens, Hkv, D, page, seed)
    s.ks.nan_to_num_(0.25, 0.25)
    s.vs.nan_to_num_(0.25, 0.25)
    s.cache = aq.Kv8Cache(s.k.cuda(), s.v.cuda(), s.ks.cuda(), s.vs.cuda())
    batch = s.batch(aq, rows)
    each = rows if rows is not None else [1] * len(lens)
    T = sum(each) + extra
    g = torch.Generator().manual_seed(seed + 5)
    x = (torch.randn(T, 2, Hkv, D, generator=g) * (10 ** (2 * torch.rand(T, 2, Hkv, 1, generator=g) - 1))).to(TD[name])
    if values is not None:
        values(x)
    xd = x.cuda()
    before = xd.clone()
    aq.aq_kv8_append(s.cache, batch, xd[:, 0], xd[:, 1])
    aq.aq_check()
    row_start = [0] + list(np.cumsum(each))
    want = O.append(s.k.numpy(), s.ks.numpy(), s.v.numpy(), s.vs.numpy(), lens, row_start, s.table, x[:, 0].float().numpy(), x[:, 1].float().numpy())
    for got, w, what in zip((s.cache.k, s.cache.k_scale, s.cache.v, s.cache.v_scale), want, ("k", "k_scale", "v", "v_scale")):
        assert np.array_equal(got.cpu().numpy(), w, equal_nan=w.dtype.kind == "f"), what
    assert torch.equal(xd, before) or bool(torch.isnan(before).any())
    return s


@pytest.mark.parametrize("name", ("f16", "bf16"))
@pytest.mark.parametrize("D", (64, 128, 256))
def test_append_is_exact(aq, D, name):
    # one row each, at every kind of place in a block and a page
    _check_append(aq, [1, 2, 31, 32, 33, 64, 65, 96, 97, 128, 129], None, 3, D, 64, name, D)
    # ragged rows: blocks begun, gone on with, whole, several pages; requests that bring nothing, rows of nobody
    _check_append(aq, [5, 40, 200, 64, 0, 300, 33], [5, 0, 130, 1, 0, 300, 31], 2, D, 32, name, D + 1, extra=3)


@pytest.mark.parametrize("Hkv", (1, 2, 7, 32))
def test_append_heads(aq, Hkv):
    _check_append(aq, [50, 70, 9], [1, 40, 9], Hkv, 128, 128, "f16", Hkv)


def test_append_many_rows_and_requests(aq):
    _check_append(aq, [4000, 96], [4000, 96], 2, 128, 64, "bf16", 1)                                # CTAs of many rows
    g = np.random.default_rng(7)
    lens = [int(v) for v in g.integers(0, 90, 1024)]
    _check_append(aq, lens, [min(L, int(v)) for L, v in zip(lens, g.integers(0, 5, 1024))], 1, 64, 32, "f16", 2)
    _check_append(aq, [1 + int(v) for v in g.integers(0, 90, 700)], None, 3, 64, 32, "f16", 3)


def test_append_values(aq):
    def zeros(x):
        x.zero_()
    def ties(x):   # quotients at halves: scale 2^-6 exactly, values (k + 1/2) 2^-6
        x.copy_(((torch.arange(x.numel()).view(x.shape) % 253) - 126.0 + 0.5).to(x.dtype) / 64)
        x[..., 0] = 127 / 64
    def tiny(x):
        x.mul_(2.0 ** -14 if x.dtype == torch.float16 else 2.0 ** -120)
    def huge(x):
        x.mul_(100 if x.dtype == torch.float16 else 2.0 ** 110)
    def broken(x):
        x[1, 0, 0, 3], x[2, 1, 1, 5], x[9, 0, 1, 0] = float("nan"), float("inf"), -float("inf")
    for name in ("f16", "bf16"):
        for i, values in enumerate((zeros, ties, tiny, huge, broken)):
            _check_append(aq, [40, 77, 5], [1, 60, 5], 2, 64, 64, name, 40 + i, values=values)


def test_append_position_by_position(aq):
    """A request that grows by one token at a time: scales that grow, older codes put on them."""
    s = Served(aq, [100], 2, 128, 64, 50)
    k, ks, v, vs = s.k.numpy(), s.ks.numpy(), s.v.numpy(), s.vs.numpy()
    g = np.random.default_rng(51)
    for L in range(1, 101):
        x = torch.from_numpy(g.standard_normal((1, 2, 2, 128)) * 1.1 ** (L % 32)).to(torch.bfloat16)
        aq.aq_kv8_append(s.cache, aq.Kv8Batch(_i32([L]), _i32(s.table)), x[:, 0].cuda(), x[:, 1].cuda())
        k, ks, v, vs = O.append(k, ks, v, vs, [L], [0, 1], s.table, x[:, 0].float().numpy(), x[:, 1].float().numpy())
    aq.aq_check()
    for got, w in zip((s.cache.k, s.cache.k_scale, s.cache.v, s.cache.v_scale), (k, ks, v, vs)):
        assert np.array_equal(got.cpu().numpy(), w, equal_nan=w.dtype.kind == "f")


def test_append_pages_outside_the_pool_are_not_written(aq):
    s = Served(aq, [100, 40], 2, 128, 32, 60)
    x = torch.randn(101, 2, 2, 128).half().cuda()
    kept = [t.clone() for t in (s.cache.k, s.cache.v)]
    for lens, rows, table in (([100, 40], [100, 1], [[-1] * 4, [s.k.shape[0]] * 4]), ([5, 10 ** 6], [100, 1], None), ([-3, 2 ** 31 - 1], [100, 1], None)):
        b = aq.Kv8Batch(_i32(lens), _i32(table or [[-1] * 4] * 2), _i32([0] + list(np.cumsum(rows))))
        aq.aq_kv8_append(s.cache, b, x[:, 0], x[:, 1])
        with pytest.raises(aq.AqError) as e:
            aq.aq_check()
        assert e.value.status == aq.AQ_ERR_RANGE
        assert torch.equal(s.cache.k, kept[0]) and torch.equal(s.cache.v, kept[1])


# ---- the binding ---------------------------------------------------------------------------------------------------
def test_calls_on_a_stream_of_the_callers(aq):
    """stream=: behind what that stream has before, whatever torch's current stream is."""
    side = torch.cuda.Stream()
    s = Served(aq, [900, 40], 2, 128, 64, 80)
    b, q = s.batch(aq), torch.randn(2, 8, 128).half()
    want, tol = _attn_reference(s, q.double().numpy(), [1, 1], 0.0)
    qd, late = q.cuda(), torch.zeros(2, 8, 128, dtype=torch.float16, device="cuda")
    out, scratch = torch.zeros(2, 8, 128, device="cuda"), aq.aq_kv8_scratch()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late.copy_(qd)
    aq.aq_kv8_attn(s.cache, b, late, out, scratch, stream=side)
    side.synchronize()
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol * 1.01)
    # the other calls
    k = torch.randn(2, 2, 128).half()
    later = torch.zeros_like(k, device="cuda")
    kd = k.cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        later.copy_(kd)
    aq.aq_rope_rows(aq.aq_rope_setup(128), later, _i32([3, 0]), stream=side.cuda_stream)
    aq.aq_kv8_append(s.cache, b, later, later, stream=side.cuda_stream)
    aq.aq_check(side)
    turned = O.rope_rows(k.double().numpy(), [3, 0], O.rope_frequencies(128), "half")
    assert np.all(np.abs(later.double().cpu().numpy() - turned) <= 2.0 ** -20 * 8 + 2.0 ** -11 * np.abs(turned))
    now = O.append(s.k.numpy(), s.ks.numpy(), s.v.numpy(), s.vs.numpy(), [900, 40], [0, 1, 2], s.table, later.float().cpu().numpy(), later.float().cpu().numpy())
    for got, w in zip((s.cache.k, s.cache.k_scale, s.cache.v, s.cache.v_scale), now):
        assert np.array_equal(got.cpu().numpy(), w, equal_nan=w.dtype.kind == "f")


def test_binding_refuses(aq):
    s = Served(aq, [90, 40], 2, 128, 64, 81)
    b, q = s.batch(aq), torch.zeros(2, 8, 128, dtype=torch.float16, device="cuda")
    out, scratch = torch.zeros_like(q), aq.aq_kv8_scratch()
    k = torch.zeros(2, 2, 128, dtype=torch.float16, device="cuda")
    i, pos, rope = _i32([1, 2]), _i32([5, 6]), aq.aq_rope_setup(128)
    attn = lambda **kw: aq.aq_kv8_attn(**{**dict(cache=s.cache, batch=b, q=q, out=out, scratch=scratch), **kw})
    append = lambda **kw: aq.aq_kv8_append(**{**dict(cache=s.cache, batch=b, k=k, v=k), **kw})
    turn = lambda **kw: aq.aq_rope_rows(**{**dict(rope=rope, x=q, pos=pos, out=out), **kw})
    plan = lambda **kw: aq.aq_kv8_plan(**{**dict(lens=i, new=i, table=_i32([[0, 1], [2, 3]]), free=i, n_free=_i32([2]), page=64, lens_out=i, n_free_out=_i32([2]),
                                                 row_start=_i32([0, 1, 2]), pos=pos), **kw})
    bad = [lambda: attn(q=q.cpu()), lambda: attn(q=q.float()[:, :, :64].half()), lambda: attn(q=q[:, ::2]), lambda: attn(q=q[0]), lambda: attn(out=out[:1]),
           lambda: attn(scratch=scratch.cpu()), lambda: attn(q=q.int()), lambda: append(k=k[:, :1]), lambda: append(v=k.bfloat16()), lambda: append(k=k.transpose(0, 1)),
           lambda: append(v=torch.zeros(2, 3, 128, dtype=torch.float16, device="cuda")[:, :2]), lambda: turn(pos=pos.long()), lambda: turn(pos=pos[:1]),
           lambda: turn(out=out[:, :4]), lambda: turn(x=[1]), lambda: plan(lens=i.long()), lambda: plan(new=_i32([1])), lambda: plan(pos=_i32([1, 2, 3, 4])[::2]),
           lambda: plan(table=i), lambda: plan(n_free=i), lambda: plan(row_start=i), lambda: aq.Kv8Cache(s.cache.k[:, :, ::2], s.cache.v, s.cache.k_scale, s.cache.v_scale),
           lambda: aq.Kv8Cache(s.cache.k.float(), s.cache.v, s.cache.k_scale, s.cache.v_scale), lambda: aq.Kv8Batch(b.lens.long(), b.table),
           lambda: aq.Kv8Batch(b.lens, b.table.t()[:1].t())]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(n)
    for n, (call, status) in enumerate(((lambda: attn(scratch=scratch[:100]), aq.AQ_ERR_INVALID_ARG), (lambda: attn(q=q[:, :7], out=out[:, :7]), aq.AQ_ERR_INVALID_ARG),
                                        (lambda: attn(q=q.float(), out=out.float()), aq.AQ_ERR_UNSUPPORTED), (lambda: plan(page=48), aq.AQ_ERR_INVALID_ARG),
                                        (lambda: turn(out=out.float()), aq.AQ_ERR_UNSUPPORTED), (lambda: turn(rope=aq.aq_rope_setup(256)), aq.AQ_ERR_INVALID_ARG),
                                        (lambda: append(k=k.float(), v=k.float()), aq.AQ_ERR_UNSUPPORTED))):
        with pytest.raises(aq.AqError) as e:
            call()
        assert e.value.status == status, n
    aq.aq_check()


# ---- together ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("name,Hkv,G,D,page", (("f16", 2, 4, 128, 32), ("bf16", 1, 8, 256, 64), ("f16", 4, 1, 64, 32)))
def test_serving_steps(aq, name, Hkv, G, D, page):
    """plan, rotary rows, append, attention, step after step: prompts, decode steps, requests that end and slots that are used again,
    in arrays of one size, as a captured step has them."""
    g = np.random.default_rng(70)
    n, width, n_rows, H = 5, 12, 96, Hkv * G
    pool = 40
    cache = aq.Kv8Cache(*(torch.zeros(pool, Hkv, page, D, dtype=torch.int8, device="cuda") for _ in range(2)),
                        *(torch.full((pool, Hkv, page // 32), float("nan"), device="cuda") for _ in range(2)))
    p = Planner(aq, n, width, page, pool, n_rows, pool - 7)
    p.free = list(range(pool - 7))
    p.d["free"][: pool - 7].copy_(_i32(p.free))
    batch = aq.Kv8Batch(p.d["lens"], p.d["table"], p.d["row_start"])
    rope = aq.aq_rope_setup(D // 2, layout="pairs", scaling="parts", factor=4.0, trained=2048)
    f = O.rope_frequencies(D // 2, 10000.0, "parts", 4.0, 2048)
    m = 0.1 * np.log(4.0) + 1
    scratch, W = aq.aq_kv8_scratch(), (H + 2 * Hkv)
    qkv = torch.zeros(n_rows, W, D, dtype=TD[name], device="cuda")
    out = torch.zeros(n_rows, H, D, dtype=TD[name], device="cuda")

    def calls():
        p.call()
        aq.aq_rope_rows(rope, qkv[:, : H + Hkv], p.d["pos"])
        aq.aq_kv8_append(cache, batch, qkv[:, H: H + Hkv], qkv[:, H + Hkv:])
        aq.aq_kv8_attn(cache, batch, qkv[:, :H], out, scratch)
    graph = None
    for step, new in enumerate(([50, 3, 0, 1, 20], [1, 1, 1, 1, 1], [1, 40, -1, 1, 1], [-1, 1, 33, 1, 0], [64, 1, 1, 1, -1], [1, 1, 1, 1, 17], [1, 1, 1, 1, 1])):
        x = torch.from_numpy(g.standard_normal((n_rows, W, D))).to(TD[name])
        qkv.copy_(x)
        out.fill_(-5.0)
        p.d["new"].copy_(_i32(new))
        before = [t.cpu().numpy().copy() for t in (cache.k, cache.k_scale, cache.v, cache.v_scale)]
        if step == 3:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                calls()
        if graph is None:
            calls()
        else:
            graph.replay()
        aq.aq_check()
        assert p.expect(new)
        row_start, pos = p.d["row_start"].tolist(), p.d["pos"].tolist()
        turned = qkv.double().cpu().numpy()
        want = O.rope_rows(x[:, : H + Hkv].double().numpy(), pos, f, "pairs", m)
        err = np.abs(turned[:, : H + Hkv] - want)
        assert np.all(err <= 2.0 ** -20 * 8 * m + HALF_STEP[name] * np.abs(want) * 1.001 + 2.0 ** -25)
        assert np.array_equal(turned[:, H + Hkv:], x[:, H + Hkv:].double().numpy())
        # the cache: what the append's definition makes of the rows that the GPU rotated
        now = O.append(*before, p.lens, row_start, p.table, turned[:, H: H + Hkv].astype(np.float32), turned[:, H + Hkv:].astype(np.float32))
        for got, w in zip((cache.k, cache.k_scale, cache.v, cache.v_scale), now):
            assert np.array_equal(got.cpu().numpy(), w, equal_nan=w.dtype.kind == "f")
        s = Served.__new__(Served)
        s.k, s.ks, s.v, s.vs = (torch.from_numpy(w) for w in now)
        s.table, s.lens, s.Hkv = p.table, p.lens, Hkv
        rows = [max(v, 0) for v in new]
        ref, tol = _attn_reference(s, turned[:, :H], rows, 0.0)
        got = out.double().cpu().numpy()
        T = row_start[-1]
        assert np.all(np.abs(got[:T] - ref[:T]) <= tol[:T] * 1.01 + HALF_STEP[name] * np.abs(ref[:T]) + 2.0 ** -25)
        assert np.all(got[T:] == -5.0)
