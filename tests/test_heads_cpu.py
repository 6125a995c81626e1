"""Host-side checks of head norms and rotations that need no GPU: exports, argument errors (found before any HIP
call, so nothing is enqueued), workspace sizes, and the torch wrappers' checks."""
import os
import re

import numpy as np
import pytest

import paper_2502_06155_amd as ta
from paper_2502_06155_amd._lib import lib
from paper_2502_06155_amd.rope import _ref
from tests.conftest import ROOT

NULL, SHAPE, DIM, ALIGN, SCALE, OVERLAP = 1, 2, 3, 5, 6, 7
M = 1 << 20  # addresses a MiB apart: every tensor below is smaller
B, S, H, HKV, D = 2, 30, 4, 2, 64


def test_every_declared_symbol_is_exported_and_bound():
    src = open(os.path.join(ROOT, "include", "head_rope.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"^\s*int\s+(head_rope\w+)\s*\(", src, flags=re.M)))
    assert len(names) == 3
    for name in names:
        assert hasattr(lib, name) and hasattr(ta, name), name
    assert f"#define TA_ROPE_AXES {ta.ROPE_AXES}" in src


def spec(**kw):
    a = dict(B=B, S=S, H=H, Hkv=HKV, d=D, norm=2, eps=1e-6, q_weight=16 * M, k_weight=17 * M, q_bias=18 * M,
             k_bias=19 * M, layout=2, axes=2, dims=(32, 16), freqs=20 * M, positions=21 * M, positions_batch=60,
             lens=22 * M)
    a.update(kw)
    a["dims"] = tuple(a["dims"]) + (0,) * (4 - len(a["dims"]))
    return ta.HeadRopeSpec(**a)


def rows(at, heads, total=None, **kw):
    total = total or heads
    a = dict(data=at, batch=S * total * D, token=total * D, head=D)
    a.update(kw)
    return ta.Rows(**a)


def fwd(s=None, **kw):
    a = dict(q=rows(M, H), k=rows(2 * M, HKV), v=rows(3 * M, HKV), qo=4 * M, ko=5 * M, vo=6 * M)
    a.update(kw)
    s = spec() if s is None else s
    return lib.head_rope_fwd(_ref(s), _ref(a["q"]), _ref(a["k"]), _ref(a["v"]), a["qo"], a["ko"], a["vo"], None)


def bwd(s=None, **kw):
    a = dict(q=rows(M, H), k=rows(2 * M, HKV), gq=3 * M, gk=4 * M, gv=5 * M, dq=rows(6 * M, H), dk=rows(7 * M, HKV),
             dv=rows(8 * M, HKV), qw=9 * M, kw=10 * M, qb=11 * M, kb=12 * M, ws=24 * M, n=1 << 24)
    a.update(kw)
    s = spec() if s is None else s
    refs = [_ref(a[x]) for x in ("q", "k")], [_ref(a[x]) for x in ("dq", "dk", "dv")]
    return lib.head_rope_bwd(_ref(s), *refs[0], a["gq"], a["gk"], a["gv"], *refs[1], a["qw"], a["kw"], a["qb"], a["kb"],
                             a["ws"], a["n"], None)


@pytest.mark.parametrize("call", [fwd, bwd])
@pytest.mark.parametrize("status,kw", [
    (SHAPE, dict(B=0)), (SHAPE, dict(S=0)), (SHAPE, dict(H=0)), (SHAPE, dict(Hkv=-1)), (DIM, dict(d=80)),
    (SHAPE, dict(B=1 << 16, S=1 << 15)), (SHAPE, dict(S=1 << 25, B=1)), (SHAPE, dict(H=65535)),
    (SHAPE, dict(norm=3)), (SHAPE, dict(norm=-1)), (SHAPE, dict(layout=4)), (SHAPE, dict(norm=0)),
    (SHAPE, dict(norm=1)), (SCALE, dict(eps=0.0)), (SCALE, dict(eps=-1.0)), (SCALE, dict(eps=float("nan"))),
    (SCALE, dict(eps=float("inf"))), (SCALE, dict(eps=1e-40)), (SHAPE, dict(axes=0)), (SHAPE, dict(axes=5)),
    (SHAPE, dict(dims=(31, 16))), (SHAPE, dict(dims=(0, 16))), (SHAPE, dict(dims=(-2, 16))), (SHAPE, dict(dims=(48, 32))),
    (SHAPE, dict(dims=(1 << 30, 1 << 30))), (NULL, dict(freqs=None)), (NULL, dict(positions=None)),
    (SHAPE, dict(positions_batch=-1)), (ALIGN, dict(freqs=20 * M + 4)), (ALIGN, dict(positions=21 * M + 2)),
    (ALIGN, dict(q_weight=16 * M + 8)), (ALIGN, dict(k_bias=19 * M + 4)), (ALIGN, dict(lens=22 * M + 1))])
def test_specs_that_are_refused(call, status, kw):
    assert call(spec(**kw)) == status


def test_a_spec_must_be_there():
    assert lib.head_rope_fwd(None, None, None, None, None, None, None, None) == NULL
    assert lib.head_rope_bwd_workspace(None, None) == NULL
    assert lib.head_rope_bwd_workspace(_ref(spec()), None) == NULL


@pytest.mark.parametrize("status,kw", [
    (NULL, dict(qo=None)), (NULL, dict(k=None)), (NULL, dict(v=rows(None, HKV))),
    (NULL, dict(q=None, k=None, v=None, qo=None, ko=None, vo=None)),
    (ALIGN, dict(q=rows(M + 8, H))), (ALIGN, dict(ko=5 * M + 4)), (ALIGN, dict(q=rows(M, H, head=D + 4))),
    (ALIGN, dict(k=rows(2 * M, HKV, token=-128))), (ALIGN, dict(v=rows(2 * M, HKV, batch=3))),
    (SHAPE, dict(q=rows(M, H, batch=1 << 62))),
    (OVERLAP, dict(qo=M + 64)), (OVERLAP, dict(ko=3 * M)), (OVERLAP, dict(ko=4 * M)), (OVERLAP, dict(vo=16 * M)),
    (OVERLAP, dict(vo=20 * M)), (OVERLAP, dict(vo=21 * M)), (OVERLAP, dict(vo=22 * M)),
    (OVERLAP, dict(k=rows(2 * M, HKV, token=1 << 16), ko=3 * M))])
def test_forward_refuses(status, kw):
    assert fwd(**kw) == status, lib.tile_attn_last_error()


@pytest.mark.parametrize("status,kw", [
    (NULL, dict(q=None)), (NULL, dict(gq=None)), (NULL, dict(dv=None)), (NULL, dict(dk=rows(None, HKV))),
    (ALIGN, dict(gk=4 * M + 8)), (ALIGN, dict(dq=rows(6 * M + 2, H))), (ALIGN, dict(qw=9 * M + 4)),
    (ALIGN, dict(ws=24 * M + 8)), (SHAPE, dict(n=16)), (SHAPE, dict(ws=None)),
    (OVERLAP, dict(dq=rows(6 * M, H, head=0))), (OVERLAP, dict(dq=rows(6 * M, H, head=32))),
    (OVERLAP, dict(dv=rows(8 * M, HKV, token=D))), (OVERLAP, dict(dv=rows(8 * M, HKV, batch=0))),
    (OVERLAP, dict(dk=rows(6 * M + 64, HKV))), (OVERLAP, dict(dq=rows(M, H))), (OVERLAP, dict(dq=rows(4 * M, H))),
    (OVERLAP, dict(qw=10 * M)), (OVERLAP, dict(kb=3 * M)), (OVERLAP, dict(ws=2 * M)), (OVERLAP, dict(ws=6 * M)),
    (OVERLAP, dict(qb=16 * M)), (OVERLAP, dict(dv=rows(22 * M, HKV))),
    # rows of one tensor that do not stand heads behind heads
    (OVERLAP, dict(dk=rows(6 * M + 2 * D * 3, HKV, H + HKV), dq=rows(6 * M, H, H + HKV))),
    (OVERLAP, dict(dk=rows(6 * M + 2 * D * H, HKV, H + HKV), dq=rows(6 * M, H, H + HKV - 1))),
    (OVERLAP, dict(dk=rows(6 * M + 2 * D * H, HKV, H + 1), dq=rows(6 * M, H, H + 1)))])
def test_gradients_refuse(status, kw):
    assert bwd(**kw) == status, lib.tile_attn_last_error()


def test_sums_need_what_they_are_of():
    plain = spec(norm=0, q_weight=None, k_weight=None, q_bias=None, k_bias=None)
    rms = spec(norm=1, q_bias=None, k_bias=None)
    none = dict(qw=None, kw=None, qb=None, kb=None)
    assert bwd(plain, **{**none, "qw": 9 * M}) == SHAPE
    assert bwd(rms, **{**none, "kb": 9 * M}) == SHAPE
    assert bwd(**{**none, "kw": 9 * M}, k=None, gk=None, dk=None) == SHAPE


def test_packed_structs_are_the_structures():
    from paper_2502_06155_amd import rope

    v = spec(dims=(2, 4, 6, 8), axes=4, positions_batch=5)
    at = [getattr(v, n) for n, _ in v._fields_]
    flat = [y for x in at for y in (list(x) if hasattr(x, "__len__") else [x])]
    assert rope._PACKED_SPEC.pack(*flat) == bytes(v)
    assert rope._PACKED_ROWS.pack(1, 2, 3, 4) == bytes(ta.Rows(1, 2, 3, 4))


def test_workspaces():
    size = lambda **kw: ta.head_rope_bwd_workspace(spec(**kw))  # noqa: E731
    assert size(norm=0, q_weight=None, k_weight=None, q_bias=None, k_bias=None) == 0
    assert 0 < size(S=1, B=1) < size() <= size(S=100000) <= 1024 * 4 * 64 * 4


def test_wrappers_refuse():
    torch = pytest.importorskip("torch")
    x = torch.zeros(1, 3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        ta.head_rope(x, x, x)
    with pytest.raises(ValueError, match="one of"):
        ta.head_rope(None, None, None)
    with pytest.raises(ValueError, match=r"\[B, S, heads, d\]"):
        ta.head_rope(x[0], None, None)


def test_frequencies_and_grids():
    pytest.importorskip("torch")
    f = ta.rope_freqs((4, 6), theta=100.0, device="cpu").numpy()
    assert np.allclose(f, [1, 0.1, 1, 100 ** (-1 / 3), 100 ** (-2 / 3)], rtol=1e-15)
    p = ta.grid_positions(2, 2, 3, text=2, device="cpu").numpy()
    assert p.shape == (14, 3) and not p[:2].any()
    assert [tuple(x) for x in p[2:6]] == [(0, 0, 0), (0, 0, 1), (0, 0, 2), (0, 1, 0)] and tuple(p[-1]) == (1, 1, 2)
