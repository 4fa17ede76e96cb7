"""The paged 8-bit cache and rotary rows without a GPU: what the host refuses, the index arithmetic of the attention's line of
tiles, rotary frequencies, and the oracle against hand-made cases."""
import ctypes as C
import os
import shutil
import subprocess
import textwrap

import numpy as np
import pytest

from oracle import kv8_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HDR = os.path.join(ROOT, "paper_2605_24011_b200", "csrc")
FAKE = 0x10000   # never followed: these calls fail in their checks


@pytest.fixture(scope="module")
def aq():
    from paper_2605_24011_b200 import aq as mod
    return mod


# ---- refusals ----------------------------------------------------------------------------------------------------
def _cache(aq, **kw):
    d = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, n_pages=8, page=64, n_kv_heads=8, head_dim=128)
    d.update(kw)
    return aq._Kv8CacheC(d["k"], d["v"], d["k_scale"], d["v_scale"], d["n_pages"], d["page"], d["n_kv_heads"], d["head_dim"], 0)


def _batch(aq, **kw):
    d = dict(lens=FAKE, row_start=FAKE, table=FAKE, width=4, n=2)
    d.update(kw)
    return aq._Kv8BatchC(d["lens"], d["row_start"], d["table"], d["width"], d["n"], 0)


BAD_CACHE = [dict(k=0), dict(v=0), dict(k_scale=0), dict(v_scale=0), dict(k=FAKE + 8), dict(v=FAKE + 1), dict(k_scale=FAKE + 2), dict(n_pages=0),
             dict(n_pages=1 << 31), dict(page=16), dict(page=48), dict(page=2048), dict(page=0), dict(page=-64), dict(n_kv_heads=0)]
BAD_BATCH = [dict(lens=0), dict(table=0), dict(lens=FAKE + 2), dict(row_start=FAKE + 1), dict(width=0), dict(width=(1 << 20) + 1), dict(n=0), dict(n=-1),
             dict(row_start=0, n=3)]   # 8 rows are not three times anything
UNSUPPORTED = [(dict(head_dim=96), {}), (dict(n_kv_heads=257), {}), ({}, dict(n=1025))]


def test_append_refuses(aq):
    lib = aq.raw_lib()

    def call(c=None, b=None, k=FAKE, v=FAKE, stride=1024, rows=8, dt=aq.AQ_F16):
        c, b = _cache(aq, **(c or {})), _batch(aq, **(b or {}))
        return lib.aq_kv8_append(C.byref(c), C.byref(b), k, v, stride, rows, dt, None)
    for c in BAD_CACHE:
        assert call(c=c) == aq.AQ_ERR_INVALID_ARG, c
    for b in BAD_BATCH:
        assert call(b=b) == aq.AQ_ERR_INVALID_ARG, b
    for c, b in UNSUPPORTED:
        assert call(c=c, b=b, stride=1 << 20) == aq.AQ_ERR_UNSUPPORTED, (c, b)
    for kw in (dict(k=0), dict(v=0), dict(k=FAKE + 2), dict(stride=1023), dict(stride=1016), dict(stride=1028), dict(rows=0), dict(rows=4097), dict(dt=7)):
        assert call(**kw) == aq.AQ_ERR_INVALID_ARG, kw
    assert call(dt=aq.AQ_F32) == aq.AQ_ERR_UNSUPPORTED
    assert lib.aq_kv8_append(None, C.byref(_batch(aq)), FAKE, FAKE, 1024, 8, 0, None) == aq.AQ_ERR_INVALID_ARG
    assert lib.aq_kv8_append(C.byref(_cache(aq)), None, FAKE, FAKE, 1024, 8, 0, None) == aq.AQ_ERR_INVALID_ARG


def test_attention_refuses(aq):
    lib = aq.raw_lib()
    big = aq.AQ_KV8_SCRATCH_BYTES

    def call(c=None, b=None, q=FAKE, qs=4096, out=2 * FAKE, os_=4096, rows=8, heads=32, scale=0.0, dt=aq.AQ_F16, odt=aq.AQ_F32, sc=FAKE, n=big):
        c, b = _cache(aq, **(c or {})), _batch(aq, **(b or {}))
        return lib.aq_kv8_attn(C.byref(c), C.byref(b), q, qs, out, os_, rows, heads, scale, dt, odt, sc, n, None)
    for c in BAD_CACHE:
        assert call(c=c) == aq.AQ_ERR_INVALID_ARG, c
    for b in BAD_BATCH:
        assert call(b=b) == aq.AQ_ERR_INVALID_ARG, b
    for c, b in UNSUPPORTED:
        assert call(c=c, b=b, heads=257, qs=1 << 20, os_=1 << 20) == aq.AQ_ERR_UNSUPPORTED, (c, b)
    for kw in (dict(q=0), dict(out=0), dict(out=FAKE), dict(sc=0), dict(q=FAKE + 4), dict(out=FAKE + 8), dict(sc=FAKE + 128), dict(n=big - 1), dict(heads=33), dict(heads=0),
               dict(qs=4092), dict(qs=4088), dict(os_=4094), dict(os_=4088), dict(rows=0), dict(rows=4097), dict(dt=5), dict(odt=5),
               dict(scale=float("inf")), dict(scale=float("nan"))):
        assert call(**kw) == aq.AQ_ERR_INVALID_ARG, kw
    assert call(dt=aq.AQ_F32) == aq.AQ_ERR_UNSUPPORTED
    # more tiles than the line can count
    assert call(c=dict(page=1024, n_kv_heads=256), b=dict(width=1 << 20, row_start=FAKE), heads=256 * 16, qs=1 << 20, os_=1 << 20, rows=4096) == aq.AQ_ERR_UNSUPPORTED


def test_plan_refuses(aq):
    lib = aq.raw_lib()

    def call(ptr=None, n=4, page=64, width=8, cap=16, rows=32):
        p = [FAKE] * 9
        if ptr is not None:
            p[ptr[0]] = ptr[1]
        return lib.aq_kv8_plan(p[0], p[1], n, page, p[2], width, p[3], cap, p[4], p[5], p[6], p[7], p[8], rows, None)
    for i in range(9):
        assert call(ptr=(i, None)) == aq.AQ_ERR_INVALID_ARG and call(ptr=(i, FAKE + 2)) == aq.AQ_ERR_INVALID_ARG
    for kw in (dict(n=0), dict(page=16), dict(page=100), dict(width=0), dict(width=(1 << 20) + 1), dict(width=1 << 20, page=2048), dict(cap=-1), dict(cap=1 << 31),
               dict(rows=0), dict(rows=(1 << 20) + 1)):
        assert call(**kw) == aq.AQ_ERR_INVALID_ARG, kw
    assert call(n=1025) == aq.AQ_ERR_UNSUPPORTED


def test_rope_refuses(aq):
    lib = aq.raw_lib()
    out = aq.Rope()

    def setup(rot=128, layout=0, theta=1e4, scaling=0, factor=1.0, trained=4096.0, low=0.0, high=0.0, mag=0.0, o=out):
        return lib.aq_rope_setup(rot, layout, theta, scaling, factor, trained, low, high, mag, C.byref(o) if o is not None else None)
    nan, inf = float("nan"), float("inf")
    assert setup() == aq.AQ_OK
    for kw in (dict(rot=0), dict(rot=3), dict(rot=258), dict(layout=2), dict(theta=1.0), dict(theta=nan), dict(theta=inf), dict(scaling=4), dict(scaling=-1),
               dict(factor=0.5), dict(factor=nan), dict(mag=-1.0), dict(mag=inf), dict(scaling=3, trained=0.0), dict(scaling=3, low=4.0, high=4.0),
               dict(scaling=3, low=-1.0, high=4.0), dict(scaling=3, high=inf, low=1.0), dict(o=None)):
        assert setup(**kw) == aq.AQ_ERR_INVALID_ARG, kw
    r = aq.aq_rope_setup(64)

    def rows(rope=r, x=FAKE, dt=0, xs=1024, o=2 * FAKE, odt=0, os_=1024, T=8, H=8, D=128, pos=FAKE):
        return lib.aq_rope_rows(C.byref(rope) if rope is not None else None, x, dt, xs, o, odt, os_, T, H, D, pos, None)
    for kw in (dict(rope=None), dict(x=None), dict(o=None), dict(pos=None), dict(pos=FAKE + 2), dict(x=FAKE + 1), dict(o=FAKE + 1), dict(dt=2, odt=2, x=FAKE + 2),
               dict(dt=3), dict(odt=3), dict(T=0), dict(H=0), dict(D=32), dict(xs=1023), dict(os_=1000), dict(T=1 << 28), dict(rope=aq.Rope()),
               dict(o=FAKE, os_=2048), dict(dt=2, odt=0, o=FAKE)):
        assert rows(**kw) == aq.AQ_ERR_INVALID_ARG, kw
    assert rows(D=1026, xs=1 << 20, os_=1 << 20) == aq.AQ_ERR_UNSUPPORTED and rows(H=4097, xs=1 << 20, os_=1 << 20) == aq.AQ_ERR_UNSUPPORTED
    assert rows(dt=0, odt=1) == aq.AQ_ERR_UNSUPPORTED and rows(dt=0, odt=2) == aq.AQ_ERR_UNSUPPORTED


def test_binding_refuses_tensors_that_the_library_would_misread(aq):
    torch = pytest.importorskip("torch")
    k = torch.zeros(4, 2, 64, 128, dtype=torch.int8)
    s = torch.zeros(4, 2, 2)
    with pytest.raises(ValueError):
        aq.Kv8Cache(k, k, s, s)                    # not on a GPU
    with pytest.raises(ValueError):
        aq.Kv8Cache(k, k, s[:, :, :1], s)          # a scale for every 64
    with pytest.raises(ValueError):
        aq.Kv8Cache(k, k[:, :, :, :64], s, s)
    with pytest.raises(ValueError):
        aq.Kv8Batch(torch.zeros(3, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32))
    with pytest.raises(ValueError):
        aq.Kv8Batch(torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32))
    i = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros(4, 8, 64)
    class D:                                       # a descriptor's place
        addr, device = FAKE, 0
    for call in (lambda: aq.aq_kv8_plan(i, i, i.view(2, 2), i, i, 64, i, i, i, i), lambda: aq.aq_rope_rows(aq.aq_rope_setup(64), x, i),
                 lambda: aq.aq_kv8_append(D, D, x, x), lambda: aq.aq_kv8_attn(D, D, x, x, i)):
        with pytest.raises((ValueError, RuntimeError)):   # (RuntimeError: no device at all)
            call()


# ---- the line of tiles -------------------------------------------------------------------------------------------
SRC = textwrap.dedent(r"""
    #include <cstdio>
    #include <initializer_list>
    #include "aq_kv8_runs.h"
    using namespace aq;
    #define CHECK(c) do { if (!(c)) { std::printf("FAIL line %d: %s\n", __LINE__, #c); return 1; } } while (0)
    int main() {
        // every place belongs to the share that cta_of says, shares differ by one place at most, warps' runs too
        for (uint32_t total : {1u, 2u, 7u, 8u, 9u, 63u, 64u, 511u, 1183u, 1184u, 1185u, 5000u})
            for (uint32_t n : {1u, 2u, 8u, 16u, 24u, 147u, 148u}) {
                if (n > total) continue;
                const Kv8Cut cut = kv8_cut(total, n);
                CHECK(kv8_begin(cut, 0) == 0 && kv8_begin(cut, n) == total);
                for (uint32_t i = 0; i < n; ++i) {
                    const uint32_t a = kv8_begin(cut, i), e = kv8_begin(cut, i + 1);
                    CHECK(e - a == total / n || e - a == (total + n - 1) / n);
                    CHECK(e > a);
                    for (uint32_t x = a; x < e; ++x) CHECK(kv8_cta_of(cut, x) == i);
                    for (uint32_t W : {4u, 8u, 16u}) {
                        CHECK(kv8_warp_begin(a, e, 0, W) == a && kv8_warp_begin(a, e, W, W) == e);
                        for (uint32_t w = 0; w < W; ++w) {
                            const uint32_t len = kv8_warp_begin(a, e, w + 1, W) - kv8_warp_begin(a, e, w, W);
                            CHECK(len == (e - a) / W || len == (e - a + W - 1) / W);
                        }
                    }
                }
            }
        // counts near 2^31
        const uint32_t big = 0x7ffffff0u;
        const Kv8Cut cut = kv8_cut(big, 148);
        CHECK(kv8_begin(cut, 148) == big);
        for (uint32_t i : {0u, 1u, 70u, 147u}) {
            const uint32_t a = kv8_begin(cut, i), e = kv8_begin(cut, i + 1);
            CHECK(a < e && kv8_cta_of(cut, a) == i && kv8_cta_of(cut, e - 1) == i && kv8_warp_begin(a, e, 15, 16) < e);
        }
        // a launch has no CTA without a place: at least two places per item
        for (uint32_t W : {4u, 8u, 16u})
            for (uint32_t total = 2; total < 3000; ++total)
                for (uint32_t items : {1u, (total + 5) / 7, total / 2}) {
                    const uint32_t ctas = kv8_ctas(total, items, W, 148);
                    CHECK(ctas >= 1 && ctas <= 148 && ctas <= total);
                }
        for (uint32_t d = 1; d <= 256; ++d)
            for (uint32_t x : {0u, 1u, d - 1, d, d + 1, 7 * d - 1, 7 * d, 4095 * d, 4096 * d - 1, 4096 * d})
                CHECK(kv8_div(x, kv8_magic(d)) == x / d);
        CHECK(kv8_snap(10, 10, 7) == 10 && kv8_snap(11, 10, 7) == 17 && kv8_snap(17, 10, 7) == 17 && kv8_snap(18, 10, 7) == 24);
        CHECK(kv8_whole_items(kv8_cut(1000, 10), 8) == 32 && kv8_whole_items(kv8_cut(100000, 10), 8) == 625);
        // rows of a step whatever the caller's array says
        CHECK(kv8_rows(3, 7, 10).first == 3 && kv8_rows(3, 7, 10).n == 4);
        CHECK(kv8_rows(7, 3, 10).n == 0 && kv8_rows(-5, 3, 10).first == 0 && kv8_rows(-5, 3, 10).n == 3);
        CHECK(kv8_rows(4, 99, 10).n == 6 && kv8_rows(99, 100, 10).first == 10 && kv8_rows(99, 100, 10).n == 0);
        CHECK(kv8_rows(-2147483647 - 1, 2147483647, 10).n == 10);
        const int marks[6] = {0, 0, 4, 4, 4, 9};
        CHECK(kv8_find(marks, 5, 0) == 1 && kv8_find(marks, 5, 3) == 1 && kv8_find(marks, 5, 4) == 4 && kv8_find(marks, 5, 8) == 4 && kv8_find(marks, 5, 99) == 4);
        CHECK(kv8_find(marks, 1, 5) == 0 && kv8_find(marks, 5, -3) == 0);
        // merge groups cover all entries with few reads
        for (int n = 1; n <= 192; ++n) {
            const int g = kv8_merge_group(n), groups = (n + g - 1) / g;
            CHECK(g >= 1 && g <= 14 && groups <= 14 && (n <= 14) == (groups == 1));
        }
        std::printf("ok\n");
        return 0;
    }
""")


def test_line_of_tiles(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(SRC)
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", HDR, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr


# ---- rotary frequencies --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rot", (2, 4, 38, 64, 128, 256))
@pytest.mark.parametrize("scaling,factor", (("none", 1.0), ("linear", 4.0), ("base", 3.7), ("parts", 8.0), ("parts", 1.0)))
def test_rope_setup(aq, rot, scaling, factor):
    r = aq.aq_rope_setup(rot, layout="pairs", theta=500000.0, scaling=scaling, factor=factor, trained=8192)
    f = O.rope_frequencies(rot, 500000.0, scaling, factor, 8192)
    got = np.array(r.turns[: rot // 2]) * (2 * np.pi)
    # a frequency comes from exp2 and log2 in binary64: a few units in the last place of exponents up to 19 + 17
    assert np.all(np.abs(got - f) <= 2.0 ** -46 * f)
    assert all(v == 0 for v in r.turns[rot // 2:]) and r.rot_dim == rot and r.layout == 1
    want = 0.1 * np.log(factor) + 1 if scaling == "parts" else 1.0
    assert abs(r.magnitude - want) <= 2.0 ** -24 * want
    assert aq.aq_rope_setup(rot, scaling=scaling, factor=factor, trained=8192, magnitude=0.5).magnitude == 0.5


# ---- the oracle ------------------------------------------------------------------------------------------------------
def test_oracle_up11():
    assert O.up11(np.float32(0)) == 0 and O.up11(np.float32(1)) == 1 and O.up11(np.float32(2047)) == 2047 and O.up11(np.float32(2049)) == 2050
    assert O.up11(np.nextafter(np.float32(1), np.float32(2))) == np.float32(1 + 2.0 ** -10)
    g = np.random.default_rng(1)
    for y in np.abs(g.standard_normal(200)).astype(np.float32):
        u = O.up11(y)
        assert u >= y and u <= y * (1 + 2.0 ** -10) and (int(u.view(np.uint32)) & 0x1FFF) == 0


def test_oracle_append_block_bounds():
    """A value is off by half a step when written, and by less than 2.5 of the block's steps after any growth."""
    g = np.random.default_rng(2)
    for trial in range(20):
        codes, scale = np.full((32, 8), 99, np.int8), np.float32(7)
        truth = []
        for p in range(32):
            x = (g.standard_normal(8) * 1.2 ** (p if trial % 2 else 0)).astype(np.float16).astype(np.float32)
            codes, scale = O.append_block(codes, scale, p, x[None])
            truth.append(x)
            got = codes[: p + 1].astype(np.float64) * float(scale)
            assert np.all(np.abs(got[p] - x) <= 0.5 * scale * (1 + 2.0 ** -20))
            assert np.all(np.abs(got - np.array(truth)) < 2.5 * scale)
            assert np.all(codes[p + 1:] == 99)
    codes, scale = O.append_block(np.zeros((32, 4), np.int8), np.float32(0), 0, np.zeros((3, 4), np.float32))
    assert scale == 0 and not codes.any()
    codes, scale = O.append_block(codes, scale, 3, np.array([[1, np.inf, 0, 0]], np.float32))
    assert np.isnan(scale)
    codes, scale = O.append_block(codes, scale, 4, np.ones((1, 4), np.float32))
    assert np.isnan(scale)
    codes, scale = O.append_block(codes, scale, 0, np.ones((1, 4), np.float32))
    assert scale == O.up11(np.float32(1) / np.float32(127)) and codes[0, 0] == 127


def test_oracle_plan():
    table = [[5, 6, -1], [7, -1, -1], [-1, -1, -1]]
    lens, t, free, rs, pos = O.plan([64, 10, 0], [1, -1, 33], table, [1, 2, 3], 32, 40, 8)
    assert lens == [65, 0, 33] and t == [[5, 6, 7], [7, -1, -1], [3, 2, -1]] and free == [1]
    assert rs == [0, 1, 1, 34] and pos == [64] + list(range(33)) + [-1] * 6
    assert O.plan([64], [33], [[5, 6, -1]], [1], 32, 64, 8) is None       # past the table
    assert O.plan([64], [1], [[5, 6, -1]], [], 32, 64, 8) is None         # no page left
    assert O.plan([64], [9], [[5, 6, -1]], [1], 32, 8, 8) is None         # too few rows
    assert O.plan([64], [-1], [[5, 6, -1]], [1], 32, 8, 2) is None        # the stack is full
    assert O.plan([64], [0], [[5, 6, -1]], [], 32, 8, 0) == ([64], [[5, 6, -1]], [], [0, 0], [-1] * 8)


def test_oracle_attention_and_gather():
    g = np.random.default_rng(3)
    codes, scales = g.integers(-127, 128, (5, 2, 64, 8)).astype(np.int8), g.random((5, 2, 2)).astype(np.float32)
    K = O.gather(codes, scales, [3, 1], 70)
    assert K.shape == (2, 70, 8)
    assert np.array_equal(K[1, 69], codes[1, 1, 5].astype(float) * float(scales[1, 1, 0])) and np.array_equal(K[0, 40], codes[3, 0, 40].astype(float) * float(scales[3, 0, 1]))
    o, T, w = O.attn(np.zeros(8), K[0], K[1], 1.0)
    assert np.allclose(o, K[1].mean(0)) and np.allclose(T, np.abs(K[1]).mean(0)) and abs(w.sum() - 1) < 1e-12
    o, T, w = O.attn(np.zeros(8), K[0][:0], K[1][:0], 1.0)
    assert not o.any()
    x = g.standard_normal((2, 3, 8))
    f = O.rope_frequencies(6)
    y = O.rope_rows(x, [0, -1], f, "half")
    assert np.array_equal(x, y)
    y = O.rope_rows(x, [5, 7], f, "pairs", 2.0)
    assert np.allclose((y[..., :6] ** 2).sum(-1), 4 * (x[..., :6] ** 2).sum(-1)) and np.array_equal(y[..., 6:], x[..., 6:])


ALIKE = textwrap.dedent(r"""
    #include <cstdio>
    #include <initializer_list>
    #include "aq_kv8_runs.h"
    using namespace aq;
    #define CHECK(c) do { if (!(c)) { std::printf("FAIL line %d: %s\n", __LINE__, #c); return 1; } } while (0)
    int main() {
        for (uint32_t most : {1u, 3u, 132u, 148u})
            for (uint32_t items = 1; items < 1200; ++items)
                for (uint32_t longest : {1u, 16u, 128u, 5000u, 0x7fffffffu / items - 2u}) {
                    const uint32_t len = longest + KV8_ITEM_COST;
                    const uint64_t all = (uint64_t)len * items;
                    if (all >= 0x80000000u) continue;
                    const uint32_t total = (uint32_t)all, each = kv8_alike(total, items, longest, most);
                    // not where items differ
                    CHECK(kv8_alike(total - 1u, items, longest, most) == 0u && kv8_alike(total + 1u, items, longest, most) == 0u);
                    const uint32_t least = (items + most - 1u) / most, ctas = (items + least - 1u) / least;
                    CHECK(each == 0u || each == least);
                    CHECK((each == 0u) == ((uint64_t)items * 3u < (uint64_t)least * most * 2u));
                    if (each == 0u) continue;
                    CHECK(ctas * 3u >= most * 2u);
                    // shares begin and end with items, in 32 bits, and cover the line; whose share a place is in
                    const Kv8Cut cut{each * len, 0u};
                    CHECK((uint64_t)each * len * most <= 0xffffffffu && (uint64_t)ctas * each * len >= total);
                    uint32_t end = 0;
                    for (uint32_t i = 0; i < most; ++i) {
                        uint32_t a = kv8_begin(cut, i), e = kv8_begin(cut, i + 1);
                        a = a < total ? a : total; e = e < total ? e : total;
                        CHECK(a == end && a % len == 0u && e % len == 0u && (a < e) == (i < ctas));
                        if (a < e) CHECK(kv8_cta_of(cut, a) == i && kv8_cta_of(cut, e - 1u) == i);
                        end = e;
                    }
                    CHECK(end == total);
                }
        std::printf("ok\n");
        return 0;
    }
""")


def test_items_that_are_alike(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(ALIKE)
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", HDR, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr
