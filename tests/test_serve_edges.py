"""What the serving side refuses or does without on the host, without a GPU."""
import os
import subprocess

import pytest
import torch

from paper_1603_06809_b200 import build as BU
from paper_1603_06809_b200 import replica as P


def host_replica(requests, cap, page):
    s = P.Shape(hidden=64, q_heads=2, kv_heads=1, dim=8, vocab=20, adapters=2, rank=8, prompt=16, page=page)
    layout = P.Layout(s)
    return P.Replica(s, layout, torch.zeros(layout.nbytes, dtype=torch.uint8), requests, cap)


@pytest.mark.parametrize("cap,page,n", [(24, 8, 25), (20, 8, 25), (1, 1, 2), (16, 16, 17)])
def test_replica_refuses_more_tokens_than_a_cache_holds(cap, page, n):
    rep = host_replica(3, cap, page)
    step = dict(adapter=torch.zeros(3, dtype=torch.int32), draft_probs=None, draft_tokens=None, uniforms=None, noise=None, temperature=None)
    with pytest.raises(ValueError):
        rep.step(torch.zeros(3, n, 64, dtype=torch.bfloat16), **step)
    rep.length[1] = rep.cap
    rep.at_most = rep.cap
    with pytest.raises(ValueError):
        rep.step(torch.zeros(3, 1, 64, dtype=torch.bfloat16), **step)
    assert rep.length.tolist() == [0, rep.cap, 0]


def test_replica_reads_the_lengths_when_all_drafts_would_fill_the_cache():
    rep = host_replica(2, 12, 4)
    for done in range(6):                                     # four new tokens a step, of which one stays
        rep._make_room(4)
        rep.length += 1
        assert int(rep.length.max()) <= rep.at_most <= rep.cap
    rep._make_room(4)
    rep.length[1] += 4                                        # 10 of 12
    with pytest.raises(ValueError):
        rep._make_room(3)
    rep._make_room(2)


# ---- what has to be built for whom
def refuse(error):
    def run(*_, **__):
        raise error
    return run


@pytest.mark.parametrize("error", [OSError("no compiler"), subprocess.CalledProcessError(1, "c++"), ImportError("no torch")])
@pytest.mark.parametrize("there", [False, True])
def test_the_library_alone_does_without_the_extension_module(error, there, tmp_path, monkeypatch):
    lib, bind = tmp_path / "lib.so", tmp_path / "bind.so"
    lib.touch()
    if there:                                                 # but older than its source
        bind.touch()
        (tmp_path / "bind.cpp").touch()
        os.utime(bind, (1, 1))
        monkeypatch.setattr(BU, "BIND_SOURCES", [str(tmp_path / "bind.cpp")])
    monkeypatch.setattr(BU, "LIB_PATH", str(lib))
    monkeypatch.setattr(BU, "BIND_PATH", str(bind))
    monkeypatch.setattr(BU, "_build_bind", refuse(error))
    assert BU.ensure_built() == str(lib)
    with pytest.raises(type(error)):                          # asked for by name, it is an error
        BU.build()


@pytest.mark.parametrize("error", [OSError("no compiler"), subprocess.CalledProcessError(1, "nvcc")])
def test_without_the_library_there_is_nothing_to_go_on_with(error, tmp_path, monkeypatch):
    lib, bind = tmp_path / "lib.so", tmp_path / "bind.so"
    bind.touch()
    monkeypatch.setattr(BU, "LIB_PATH", str(lib))
    monkeypatch.setattr(BU, "BIND_PATH", str(bind))
    monkeypatch.setattr(BU, "_run", refuse(error))
    with pytest.raises(type(error)):
        BU.ensure_built()
    lib.touch()
    os.utime(lib, (1, 1))                                     # older than its sources: kept
    assert BU.ensure_built() == str(lib)
