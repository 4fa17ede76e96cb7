"""The paged 8-bit cache at the edges of what its calls document: subnormal blocks, lengths past the table, values near the end of the
type's range, steps whose row marks descend, ragged batches of few items.  Oracle and tolerances as in test_gpu_kv8.py."""
import numpy as np
import pytest

from oracle import kv8_oracle as O
from test_gpu_kv8 import Served, _attn_reference, _check_append, _check_attn, _i32, aq  # noqa: F401  (aq: the module's fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _bf16_patterns(below, seed):
    """bfloat16 values of either sign whose magnitudes have patterns under `below`: 0x80 is 2^-126, 1 is 2^-133."""
    def fill(x):
        g = torch.Generator().manual_seed(seed)
        m = torch.randint(0, below, x.shape, generator=g) + 0x8000 * torch.randint(0, 2, x.shape, generator=g)
        x.copy_(torch.where(m >= 0x8000, m - 0x10000, m).to(torch.int16).view(torch.bfloat16))
    return fill


@pytest.mark.parametrize("below", (2, 3, 0x10, 0x80, 0x100, 0x180, 0x400))
@pytest.mark.parametrize("D", (64, 128, 256))
def test_append_of_subnormal_blocks_is_exact(aq, D, below):
    """Blocks whose scale is a subnormal binary32: the definition's 11 significant bits, not a multiple of 2^-136."""
    _check_append(aq, [40, 77, 5], [1, 60, 5], 2, D, 64, "bf16", 90 + D, values=_bf16_patterns(below, below))
    _check_append(aq, [1, 33, 64], None, 3, D, 64, "bf16", 91 + D, values=_bf16_patterns(below, below + 1))


@pytest.mark.parametrize("start", (2.0 ** -133, 2.0 ** -128, 2.0 ** -124))
def test_append_position_by_position_in_subnormals(aq, start):
    """Scales that grow by a quarter through the subnormal range, older codes put on them."""
    s = Served(aq, [64], 1, 64, 64, 92)
    k, ks, v, vs = s.k.numpy(), s.ks.numpy(), s.v.numpy(), s.vs.numpy()
    g = np.random.default_rng(93)
    for L in range(1, 65):
        x = torch.from_numpy(g.standard_normal((1, 2, 1, 64)) * start * 1.15 ** (L % 32)).to(torch.bfloat16)
        aq.aq_kv8_append(s.cache, aq.Kv8Batch(_i32([L]), _i32(s.table)), x[:, 0].cuda(), x[:, 1].cuda())
        k, ks, v, vs = O.append(k, ks, v, vs, [L], [0, 1], s.table, x[:, 0].float().numpy(), x[:, 1].float().numpy())
    aq.aq_check()
    for got, w in zip((s.cache.k, s.cache.k_scale, s.cache.v, s.cache.v_scale), (k, ks, v, vs)):
        assert np.array_equal(got.cpu().numpy(), w, equal_nan=w.dtype.kind == "f")


def test_append_to_a_block_whose_scale_is_infinite(aq):
    """need <= s' then: the scale stays, code = rint(x / inf) = 0, the older codes stay."""
    s = Served(aq, [50, 20], 2, 128, 64, 94)
    s.ks.nan_to_num_(0.25, 0.25)
    s.vs.nan_to_num_(0.25, 0.25)
    s.ks[s.table[0][0]], s.vs[s.table[1][0]] = float("inf"), float("inf")
    s.cache = aq.Kv8Cache(s.k.cuda(), s.v.cuda(), s.ks.cuda(), s.vs.cuda())
    x = torch.randn(5, 2, 2, 128, generator=torch.Generator().manual_seed(94)).half()
    xd = x.cuda()
    for rows in ([3, 2], [1, 4]):
        aq.aq_kv8_append(s.cache, s.batch(aq, rows), xd[:, 0], xd[:, 1])
    aq.aq_check()
    want = (s.k.numpy(), s.ks.numpy(), s.v.numpy(), s.vs.numpy())
    for rows in ([0, 3, 5], [0, 1, 5]):
        want = O.append(*want, [50, 20], rows, s.table, x[:, 0].float().numpy(), x[:, 1].float().numpy())
    for got, w in zip((s.cache.k, s.cache.k_scale, s.cache.v, s.cache.v_scale), want):
        assert np.array_equal(got.cpu().numpy(), w, equal_nan=w.dtype.kind == "f")


@pytest.mark.parametrize("others", (1, 40))
@pytest.mark.parametrize("D,rows", ((128, 8), (64, 3), (256, 17)))
def test_attention_of_a_length_past_the_table(aq, D, rows, others):
    """Only the positions that do not fit count as masked: a row's own position is where the caller's length puts it, as the append has it."""
    page, width = 32, 3
    s = Served(aq, [page * width] + [20] * others, 2, D, page, 95)
    T = rows + others
    q = torch.randn(T, 4, D, generator=torch.Generator().manual_seed(95)).half()
    for past in (1, 5, 40, 2 ** 31 - 1 - page * width):
        out = torch.full((T, 4, D), float("nan"), device="cuda")
        batch = aq.Kv8Batch(_i32([page * width + past] + [20] * others), _i32(s.table), _i32([0] + list(range(rows, T + 1))))
        aq.aq_kv8_attn(s.cache, batch, q.cuda(), out, aq.aq_kv8_scratch())
        with pytest.raises(aq.AqError) as e:
            aq.aq_check()
        assert e.value.status == aq.AQ_ERR_RANGE
        got = out.double().cpu().numpy()
        for i in range(rows):
            # the row as the only new token of a request of the length that it sees
            one = Served.__new__(Served)
            one.k, one.ks, one.v, one.vs, one.table, one.Hkv = s.k, s.ks, s.v, s.vs, s.table, 2
            one.lens = [min(page * width, page * width + past - rows + i + 1)]
            want, tol = _attn_reference(one, q[i: i + 1].double().numpy(), [1], 0.0)
            assert np.all(np.abs(got[i] - want[0]) <= tol[0] * (1 + 2.0 ** -24) + 2.0 ** -24 * np.abs(want[0])), (past, i)
        s.lens = [0] + [20] * others
        want, tol = _attn_reference(s, q.double().numpy()[rows:], [0] + [1] * others, 0.0)
        assert np.all(np.abs(got[rows:] - want) <= tol * (1 + 2.0 ** -24) + 2.0 ** -24 * np.abs(want))


@pytest.mark.parametrize("up,lens,D", ((2.0 ** 109, [700, 33], 128), (2.0 ** 112, [60, 1], 64), (2.0 ** 106, [9000], 256)))
def test_attention_of_values_near_the_end_of_the_range(aq, up, lens, D):
    """bfloat16 reaches 3.4e38: the weighted sum of the values stays in binary32 as long as the sum of the values does."""
    s = Served(aq, lens, 2, D, 64, 96)
    s.vs = s.vs * up
    s.cache = aq.Kv8Cache(s.k.cuda(), s.v.cuda(), s.ks.cuda(), s.vs.cuda())
    q = torch.randn(len(lens), 8, D, generator=torch.Generator().manual_seed(96)).to(torch.bfloat16)
    want, tol = _attn_reference(s, q.double().numpy(), [1] * len(lens), 0.0)
    assert np.max(np.abs(want)) * max(lens) < 2.0 ** 127
    for name, half in ((torch.float32, 2.0 ** -24), (torch.bfloat16, 2.0 ** -8)):
        out = torch.empty(len(lens), 8, D, dtype=name, device="cuda")
        aq.aq_kv8_attn(s.cache, s.batch(aq), q.cuda(), out, aq.aq_kv8_scratch())
        aq.aq_check()
        got = out.double().cpu().numpy()
        assert np.all(np.abs(got - want) <= tol + half * (np.abs(want) + tol))


@pytest.mark.parametrize("down", (2.0 ** -90, 2.0 ** -110, 2.0 ** -140))
def test_attention_of_tiny_values(aq, down):
    """Beside the module's tolerance 2^-122 per tile of 32 positions: a tile's scale enters as vs 2^-16 times its weight, off by 2^-150 at most where
    that is subnormal, and is multiplied by 128 (65535 w) at most for each position, over the normaliser, 65535 2^-16 at least; the binary32
    sums and the quotient are off by 2^-150 each there."""
    s = Served(aq, [100, 1], 2, 128, 64, 97)
    s.vs = (s.vs.double() * down).float()
    s.cache = aq.Kv8Cache(s.k.cuda(), s.v.cuda(), s.ks.cuda(), s.vs.cuda())
    q = torch.randn(2, 8, 128, generator=torch.Generator().manual_seed(97)).to(torch.bfloat16)
    want, tol = _attn_reference(s, q.double().numpy(), [1, 1], 0.0)
    out = torch.empty(2, 8, 128, device="cuda")
    aq.aq_kv8_attn(s.cache, s.batch(aq), q.cuda(), out, aq.aq_kv8_scratch())
    aq.aq_check()
    # (the reference's tolerance has 1e-30 of its own, far more than these values: it goes)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= (tol - 1e-30) * (1 + 2.0 ** -24) + 2.0 ** -24 * np.abs(want) + 4 * 2.0 ** -122)


def test_attention_row_marks_whose_line_wraps(aq):
    """Descending marks of 1024 requests that name 2^21 rows: a line of 2^32 places, 0 in 32 bits, is reported like any other."""
    n, L = 1024, 8190 * 32
    cache = aq.Kv8Cache(*(torch.zeros(2, 1, 1024, 64, dtype=torch.int8, device="cuda") for _ in range(2)), *(torch.ones(2, 1, 32, device="cuda") for _ in range(2)))
    batch = aq.Kv8Batch(_i32([L] * n), _i32(np.zeros((n, 256))), _i32([0, 4096] * (n // 2) + [0]))
    q = torch.zeros(4096, 4, 64, dtype=torch.float16, device="cuda")
    out = torch.full((4096, 4, 64), float("nan"), dtype=torch.float16, device="cuda")
    aq.aq_kv8_attn(cache, batch, q, out, aq.aq_kv8_scratch())
    with pytest.raises(aq.AqError) as e:
        aq.aq_check()
    assert e.value.status == aq.AQ_ERR_RANGE and bool(torch.isnan(out).all())


@pytest.mark.parametrize("D,G", ((64, 1), (128, 4), (256, 8)))
def test_attention_few_items_and_one_long_one(aq, D, G):
    """Fewer items than CTAs, one far longer than the average: shared by CTAs while the others stay short."""
    _check_attn(aq, [600 * 32] + [29 * 32] * 39, 1, G, D, 128, seed=98, outs=("f32",))
    _check_attn(aq, [9, 60 * 32, 40, 64], 2, G, D, 32, rows=[1, 2, 1, 0], seed=99, outs=("f32",))


@pytest.mark.parametrize("name,big", (("f16", 100.0), ("f16", 3000.0), ("bf16", 100.0), ("bf16", 30000.0)))
@pytest.mark.parametrize("D,G", ((64, 1), (128, 4), (256, 8)))
def test_attention_of_queries_with_outliers(aq, D, G, name, big):
    """A few elements far larger than the rest, on channels where the keys are small: the module's tolerance, 1.03 times
    it as a query's element is off by 1/65278 of its row's largest, 1.004 2^-16, where it counts 2^-16."""
    s = Served(aq, [700, 90], 2, D, 64, 100)
    for channel in (3, D - 5):
        s.k[..., channel] = torch.sign(s.k[..., channel]).to(torch.int8)
    s.cache = aq.Kv8Cache(s.k.cuda(), s.v.cuda(), s.ks.cuda(), s.vs.cuda())
    q = torch.randn(2, 2 * G, D, generator=torch.Generator().manual_seed(100))
    q[..., 3], q[..., D - 5] = big, -0.8 * big
    q = q.to({"f16": torch.float16, "bf16": torch.bfloat16}[name])
    want, tol = _attn_reference(s, q.double().numpy(), [1, 1], 0.0)
    for out_type, half in ((torch.float32, 2.0 ** -24), (q.dtype, 2.0 ** -11 if name == "f16" else 2.0 ** -8)):
        out = torch.empty(2, 2 * G, D, dtype=out_type, device="cuda")
        aq.aq_kv8_attn(s.cache, s.batch(aq), q.cuda(), out, aq.aq_kv8_scratch())
        aq.aq_check()
        assert np.all(np.abs(out.double().cpu().numpy() - want) <= 1.03 * tol + half * (np.abs(want) + tol) + (2.0 ** -25 if name == "f16" else 0))


@pytest.mark.parametrize("layout", ("half", "pairs"))
def test_rope_rows_of_frequencies_set_by_the_caller(aq, layout):
    rope = aq.aq_rope_setup(64, layout=layout)
    f = np.random.default_rng(101).random(32) * 0.7
    for i, w in enumerate(f):
        rope.turns[i] = w / (2 * np.pi)
    x = torch.randn(9, 3, 80, generator=torch.Generator().manual_seed(101))
    pos = [0, 1, 17, 5000, -1, 99, 3, 2, 700]
    got = aq.aq_rope_rows(rope, x.cuda(), _i32(pos)).double().cpu().numpy()
    want = O.rope_rows(x.double().numpy(), pos, f, layout)
    # as in test_gpu_kv8.py; the angle's two roundings in binary64 are under 2^-38 radians at 5000
    assert np.all(np.abs(got - want) <= 2.0 ** -21 * 2 * np.abs(x.numpy()).max() + 2.0 ** -24 * np.abs(want))
