"""The paged 8-bit cache's host arithmetic and build at the edges, without a GPU."""
import ctypes as C
import os
import shutil
import subprocess
import sys
import textwrap

import numpy as np
import pytest

from oracle import kv8_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HDR = os.path.join(ROOT, "paper_2605_24011_b200", "csrc")


def _compiled(tmp_path, name, text, *more):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    src, out = tmp_path / (name + ".cpp"), tmp_path / name
    src.write_text(textwrap.dedent(text))
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", *more, "-I", HDR, str(src), "-o", str(out)], check=True)
    return str(out)


def test_up11_of_all_magnitudes(tmp_path):
    """The scale's rounding against the definition, subnormals among them."""
    lib = C.CDLL(_compiled(tmp_path, "up11.so", r"""
        #include "aq_kv8_runs.h"
        extern "C" uint32_t up11(uint32_t x) { return aq::kv8_up11(x); }
    """, "-shared", "-fPIC"))
    lib.up11.argtypes, lib.up11.restype = [C.c_uint32], C.c_uint32
    g = np.random.default_rng(1)
    edges = [x for e in range(0, 31) for x in (2 ** e - 1, 2 ** e, 2 ** e + 1) if x < 0x7F000000]
    # a block's need where its largest magnitude is 1.5 * 2^-125 and smaller
    halves = [int((np.float32(m) / np.float32(127)).view(np.uint32)) for m in (1.5 * 2.0 ** -125, 2.0 ** -133, 2.0 ** -126, 2.0 ** -119)]
    for x in edges + halves + [0, 0x7FFFFF, 0x800000, 0x7F000000] + [int(v) for v in g.integers(0, 0x7F000000, 3000)] + [int(v) for v in g.integers(0, 0x800000, 3000)]:
        got, want = lib.up11(x), O.up11(np.uint32(x).view(np.float32))
        assert got == int(want.view(np.uint32)), hex(x)
    assert lib.up11(0x7F800000) == 0x7F800000


def test_ctas_of_ragged_items(tmp_path):
    """A CTA per item only where no item is then shared by CTAs; else a CTA for every so many places."""
    exe = _compiled(tmp_path, "ctas", r"""
        #include <cstdio>
        #include <initializer_list>
        #include "aq_kv8_runs.h"
        using namespace aq;
        #define CHECK(c) do { if (!(c)) { std::printf("FAIL line %d: %s\n", __LINE__, #c); return 1; } } while (0)
        int main() {
            for (uint32_t W : {8u, 12u, 16u})
                for (uint32_t most : {1u, 20u, 148u})
                    for (uint32_t items = 1; items <= 200; ++items)
                        for (uint32_t rest : {1u, 2u, 10u, 29u, 50u, 70u})
                            for (uint32_t longest : {1u, 2u, 29u, 4u * W, 4u * W + 1u, 60u, 100u, 600u, 100000u}) {
                                if (longest < rest) continue;
                                const uint32_t total = longest + KV8_ITEM_COST + (items - 1u) * (rest + KV8_ITEM_COST);
                                const uint32_t n = kv8_launch(total, items, longest, W, most), even = kv8_even_ctas(total, W, most);
                                CHECK(n >= 1u && n <= most && n <= total);
                                const Kv8Cut cut = kv8_cut(total, n);
                                const bool alike = cut.more == 0u && cut.each == longest + KV8_ITEM_COST;
                                // fewer CTAs than the places ask for, or more: a CTA per item, and none of them shared
                                if (n != even) CHECK(n == items && (longest <= kv8_whole_items(cut, W) || alike));
                                // and as before where all are short or alike
                                if (longest <= 4u * W || rest == longest) CHECK(n == kv8_ctas(total, items, W, most));
                            }
            CHECK(kv8_launch(602u + 39u * 31u, 40u, 600u, 12u, 148u) == 148u && kv8_launch(32u * 18u, 32u, 16u, 12u, 148u) == 32u);
            std::printf("ok\n");
            return 0;
        }
    """, "-fsanitize=undefined", "-fno-sanitize-recover")
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr


def test_scratch_is_on_the_device_that_was_named(monkeypatch):
    """Device 0 by its number is not the current device."""
    torch = pytest.importorskip("torch")
    from paper_2605_24011_b200 import aq
    asked = []
    monkeypatch.setattr(torch, "zeros", lambda n, dtype, device: asked.append((n, dtype, device)))
    for device in (0, 1, "cuda:0", torch.device("cuda", 0), None):
        aq.aq_kv8_scratch() if device is None else aq.aq_kv8_scratch(device)
    assert asked == [(aq.AQ_KV8_SCRATCH_BYTES, torch.uint8, d) for d in (0, 1, "cuda:0", torch.device("cuda", 0), "cuda")]


@pytest.fixture
def builder(tmp_path, monkeypatch):
    """The build with compilers that only write their outputs: (module, list of programs run, set of those that fail)."""
    from paper_2605_24011_b200 import build as B
    ran, failing = [], set()

    def run(cmd, **kw):
        ran.append(os.path.basename(cmd[0]))
        bad = ran[-1] in failing
        if not bad:
            with open(cmd[cmd.index("-o") + 1], "w") as f:
                f.write("x")
        return subprocess.CompletedProcess(cmd, int(bad), "", "it failed" if bad else "")
    monkeypatch.setattr(B, "subprocess", type("Fake", (), {"run": staticmethod(run)}))
    monkeypatch.setattr(B, "OUT", str(tmp_path / "libaq.so"))
    monkeypatch.setattr(B, "TORCH_OUT", str(tmp_path / "_aq_torch.so"))
    monkeypatch.setattr(B, "OBJ", str(tmp_path / "_build"))
    return B, ran, failing


def test_library_is_built_without_torch(builder, monkeypatch, capsys):
    B, ran, _ = builder
    monkeypatch.setitem(sys.modules, "torch", None)   # an import fails
    assert B.build() == B.OUT and os.path.exists(B.OUT) and not os.path.exists(B.TORCH_OUT)
    assert "torch" in capsys.readouterr().err and "g++" not in ran
    n = len(ran)
    B.build()
    assert len(ran) == n   # the library is not linked again for the sake of what cannot be built


def test_library_is_there_when_the_calls_on_tensors_do_not_compile(builder):
    pytest.importorskip("torch")
    B, ran, failing = builder
    failing.add("g++")
    with pytest.raises(RuntimeError, match="aq_torch"):
        B.build()
    assert os.path.exists(B.OUT) and not os.path.exists(B.TORCH_OUT)
    failing.clear()
    ran.clear()
    B.build()
    assert ran == ["g++"] and os.path.exists(B.TORCH_OUT)


def test_calls_on_tensors_are_compiled_again_for_another_torch(builder, monkeypatch):
    torch = pytest.importorskip("torch")
    B, ran, _ = builder
    B.build()
    assert "g++" in ran
    ran.clear()
    B.build()
    assert ran == []
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    B.build()
    assert ran == ["g++"]


def test_calls_on_tensors_for_another_torch_are_not_loaded(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2605_24011_b200 import aq
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    monkeypatch.setattr(aq, "_calls", aq._Calls())
    with pytest.raises(ImportError, match="0.0.1"):
        aq.aq_rope_rows(aq.aq_rope_setup(64), torch.zeros(1, 1, 64), torch.zeros(1, dtype=torch.int32))
