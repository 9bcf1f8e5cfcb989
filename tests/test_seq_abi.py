"""C ABI checks of linear attention and group norm that need no GPU: sizes of
workspaces, and refusals before anything is launched."""
import pytest

L = pytest.importorskip("paper_2501_12381_amd.lib")
F32, BF16 = L.GSPN_F32, L.GSPN_BF16
FAKE = 1 << 40  # never dereferenced: every call below is refused by the host's checks


@pytest.fixture(autouse=True)
def no_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("host checks with made-up pointers run only without a GPU")


def at(i):
    return FAKE + (i << 32)


def lin(fn="fwd", **kw):
    a = dict(q=at(0), k=at(1), v=at(2), a=at(3), s0=None, cu=None, o=at(4), sf=None, n=2, B=2, T=100, H=4, Hk=2,
             Dk=32, Dv=32, strides=None, dtype=F32, flags=0, ws=at(20), bytes=1 << 31, dout=at(5), dsf=None, dq=at(6),
             dk=at(7), dv=at(8), da=at(9), ds0=None, fws=None)
    a.update(kw)
    sizes = [a[x] for x in ("n", "B", "T", "H", "Hk", "Dk", "Dv")]
    if fn == "fwd":
        return L.gspn_linattn_fwd(a["q"], a["k"], a["v"], a["a"], a["s0"], a["cu"], a["o"], a["sf"], *sizes,
                                  a["strides"], a["dtype"], a["flags"], 1.0, a["ws"], a["bytes"], None)
    return L.gspn_linattn_bwd(a["dout"], a["q"], a["k"], a["v"], a["a"], a["s0"], a["dsf"], a["cu"], a["dq"], a["dk"],
                              a["dv"], a["da"], a["ds0"], *sizes, a["strides"], a["dtype"], a["flags"], 1.0, a["fws"],
                              a["ws"], a["bytes"], None)


@pytest.mark.parametrize("fn", ["fwd", "bwd"])
def test_linattn_refusals(fn):
    assert lin(fn, dtype=7) == 4
    assert lin(fn, flags=2) == 7
    assert lin(fn, H=0) == 2 and lin(fn, T=-1) == 2 and lin(fn, Dk=0) == 2 and lin(fn, B=-1, n=-1) == 2
    assert lin(fn, Hk=3) == 2  # 4 value heads
    assert lin(fn, n=3) == 2  # batched: one sequence a row
    assert lin(fn, cu=at(10)) == 2  # packed: one row
    assert lin(fn, Dk=129) == 7 and lin(fn, Dv=200) == 7
    assert lin(fn, T=1 << 40) == 7
    assert lin(fn, B=1 << 30, n=1 << 30, T=1 << 30) in (2, 7)
    for x in ("q", "k", "v", "a"):
        assert lin(fn, **{x: None}) == 1
        assert lin(fn, **{x: at(11) + 2}) == 5
    assert lin(fn, s0=at(12) + 2) == 5
    import ctypes
    assert lin(fn, strides=(ctypes.c_int64 * 9)(*([-1] * 9))) == 2
    assert lin(fn, strides=(ctypes.c_int64 * 9)(*([1 << 62] * 9))) == 2


def test_linattn_outputs_and_workspace():
    assert lin(o=None) == 1 and lin(o=at(4) + 2) == 5 and lin(o=at(2)) == 6
    assert lin(o=at(4), sf=at(4) + 64) == 6
    long = dict(B=1, n=1, T=10000)
    assert lin(**long, ws=None) == 8 and lin(**long, bytes=1000) == 8 and lin(**long, ws=at(20) + 8) == 5
    assert lin(**long, ws=at(2)) == 6
    for x in ("dq", "dk", "dv", "da", "dout"):
        assert lin("bwd", **{x: None}) == 1
        assert lin("bwd", **{x: at(11) + 1}) == 5
    assert lin("bwd", dq=at(0)) == 6 and lin("bwd", dk=at(6)) == 6
    assert lin("bwd", ws=None) == 8 and lin("bwd", bytes=64) == 8
    assert lin("bwd", **long, fws=at(30) + 8) == 5


def test_linattn_workspace_sizes():
    fwd, bwd = L.gspn_linattn_fwd_workspace_bytes, L.gspn_linattn_bwd_workspace_bytes
    assert fwd(64, 64, 100, 8, 8, 64, 64, 0, BF16) == 0  # whole sequences fill the card
    assert fwd(1, 1, 100000, 8, 8, 64, 64, 0, BF16) > 0  # one is cut
    assert fwd(1, 1, 0, 8, 8, 64, 64, 0, BF16) == 0
    assert bwd(2, 2, 100, 4, 2, 128, 128, 0, BF16) % 256 == 0
    # the backward holds a state for each chunk of 64 tokens, in the element type
    assert bwd(256, 256, 640, 2, 2, 128, 128, 0, BF16, 1) >= 512 * 10 * 128 * 128 * 2
    assert fwd(3, 3, 100, 4, 3, 64, 64, 0, BF16) == 0 and bwd(1, 1, 10, 1, 1, 129, 1, 0, F32) == 0  # refused sizes
    assert fwd(5, 1, 5000, 8, 8, 64, 64, 1, F32) > 0


def step(**kw):
    a = dict(q=at(0), k=at(1), v=at(2), a=at(3), state=at(4), slots=None, o=at(5), n=8, B=4, H=4, Hk=2, Dk=32, Dv=32,
             strides=None, dtype=BF16, flags=0)
    a.update(kw)
    return L.gspn_linattn_step(*(a[x] for x in ("q", "k", "v", "a", "state", "slots", "o", "n", "B", "H", "Hk", "Dk",
                                                "Dv", "strides", "dtype", "flags")), 1.0, None)


def test_step_refusals():
    assert step(dtype=9) == 4 and step(flags=8) == 7 and step(Hk=3) == 2 and step(Dk=200) == 7 and step(B=-1) == 2
    assert step(n=3) == 2  # four rows without slots
    assert step(n=-1, slots=at(6)) == 2
    assert step(state=None) == 1 and step(o=None) == 1 and step(q=None) == 1
    assert step(state=at(4) + 4) == 5 and step(slots=at(6) + 2) == 5 and step(o=at(5) + 1) == 5
    assert step(o=at(4)) == 6 and step(state=at(0)) == 6
    assert step(B=0) == 0


def norm(fn="fwd", **kw):
    a = dict(x=at(0), w=at(1), b=at(2), y=at(3), mean=at(4), rstd=at(5), dy=at(6), dw=at(7), db=at(8), B=2, L=5000,
             C=64, G=4, eps=1e-5, act=0, dtype=BF16, ws=at(9), bytes=1 << 30)
    a.update(kw)
    sizes = [a[x] for x in ("B", "L", "C", "G")]
    if fn == "fwd":
        return L.gspn_group_norm_fwd(a["x"], a["w"], a["b"], a["y"], a["mean"], a["rstd"], *sizes, a["eps"], a["act"],
                                     a["dtype"], a["ws"], a["bytes"], None)
    return L.gspn_group_norm_bwd(a["dy"], a["x"], a["w"], a["b"], a["mean"], a["rstd"], a["y"], a["dw"], a["db"], *sizes,
                                 a["act"], a["dtype"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("fn", ["fwd", "bwd"])
def test_group_norm_refusals(fn):
    assert norm(fn, dtype=3) == 4 and norm(fn, act=3) == 7 and norm(fn, act=-1) == 7
    assert norm(fn, G=5) == 2 and norm(fn, G=0) == 2 and norm(fn, C=0) == 2 and norm(fn, B=-1) == 2
    assert norm(fn, C=8200, G=8) == 7
    assert norm(fn, B=1 << 50) in (2, 7)
    for x in ("x", "y", "mean", "rstd"):
        assert norm(fn, **{x: None}) == 1
        assert norm(fn, **{x: at(11) + 1}) == 5
    assert norm(fn, w=at(11) + 1) == 5
    assert norm(fn, y=at(0)) == 6
    assert norm(fn, ws=None) == 8 and norm(fn, bytes=8) == 8 and norm(fn, ws=at(9) + 16) == 5
    assert norm(fn, B=0) == 0 and norm(fn, L=0) == 0


def test_group_norm_options():
    assert norm(eps=-1.0) == 7 and norm(eps=float("inf")) == 7 and norm(eps=float("nan")) == 7
    assert norm("bwd", dy=None) == 1 and norm("bwd", dw=at(0)) == 6
    size = L.gspn_group_norm_fwd_workspace_bytes
    assert size(2, 16, 64, 4, BF16) == 0 and size(2, 5000, 64, 4, BF16) > 0  # one launch, two launches
    assert size(2, 5000, 64, 5, BF16) == 0 and L.gspn_group_norm_bwd_workspace_bytes(0, 5, 64, 4, F32) == 0
