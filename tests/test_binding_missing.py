"""Where the compiled binding is not there, or is of another torch, calls go the long way; the library is built without it."""

import os
import shutil
import sys
import types
import warnings

import pytest
import torch

import paper_2606_22327_amd as package
from paper_2606_22327_amd import build as B
from paper_2606_22327_amd import kvcache as C
from paper_2606_22327_amd import logprobs as L
from test_kvcache import BF, batch_of, make

NAME = "paper_2606_22327_amd._svfbinding"


def replace(monkeypatch, module):
    monkeypatch.setattr(C, "_bound", None)
    monkeypatch.setitem(sys.modules, NAME, module)
    monkeypatch.delattr(package, "_svfbinding", raising=False)


@pytest.mark.parametrize("module", [None, types.SimpleNamespace(torch_version="1.0.0"), types.SimpleNamespace()],
                         ids=["missing", "of another torch", "of no torch"])
def test_calls_go_the_long_way(module, monkeypatch):
    replace(monkeypatch, module)
    with pytest.warns(RuntimeWarning, match="__graft_entry__"):
        b = C._binding()
    for f, n in ((b.append, 13), (b.attend, 10), (b.score, 6)):
        assert f(*([None] * n)) is None
    with warnings.catch_warnings():
        warnings.simplefilter("error")          # once is enough
        assert C._binding() is b


def test_the_one_that_is_built_is_of_this_torch():
    from paper_2606_22327_amd import _svfbinding
    assert _svfbinding.torch_version == str(torch.__version__)


def test_the_library_is_built_without_a_compiler_for_the_binding(monkeypatch, tmp_path):
    old = tmp_path / "_svfbinding.so"
    old.write_bytes(b"of an earlier library")
    monkeypatch.setattr(B, "BINDING", str(old))
    monkeypatch.setattr(shutil, "which", lambda name, *a, **k: None)
    with pytest.warns(RuntimeWarning, match="binding"):
        assert B.build_binding() is None
    assert not os.path.exists(old)              # it would call a library that it does not know


def test_a_binding_that_does_not_compile_is_an_error(monkeypatch, tmp_path):
    monkeypatch.setattr(B, "BINDING", str(tmp_path / "_svfbinding.so"))
    monkeypatch.setattr(B, "CSRC", str(tmp_path))           # no source there
    with pytest.raises(Exception, match="g\\+\\+"):
        B.build_binding()


@pytest.mark.gpu
def test_results_without_the_binding(monkeypatch):
    s = make(1, [300, 50, 1], [3, 40, 1], 8, 2, 128, 16, BF, garbage=0.0, stats=True)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((44, 2, 128), generator=g).to(BF).cuda() for _ in range(2))
    pos, x = torch.randint(0, 99, (44, 2), generator=g).int().cuda(), torch.randn((7, 3001), generator=g).cuda()

    def run():
        c, b, q = C.Cache(*(s[n].cuda() for n in ("k", "v", "weight", "position"))), batch_of(s), s["q"].cuda()
        q = C.append(q, k, v, pos, C.rope_table(100, 128), b, c, axes=C.pair_axes((32, 32)))
        return [q, *C.attend(q, b, c, window=20, first=5, add_weight=True), *c, *L.score(x, torch.arange(7).cuda(), top=4)]

    want = run()
    replace(monkeypatch, None)
    with pytest.warns(RuntimeWarning, match="__graft_entry__"):
        got = run()
    assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(want, got))
