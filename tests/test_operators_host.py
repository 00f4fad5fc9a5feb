"""CPU-only checks of the operators' boundary: arguments are checked on the host (no kernel is launched by any of these calls), workspaces are sized sensibly, and
the Python entry points refuse what has no GPU path."""
import ctypes

import pytest

from paper_2501_14336_amd import binding as B

GOOD = dict(x=0x10000, batch=3, n=1000, stride=1000, dt=0, inv_t=1.0)


def _call(name, order, **kw):
    args = [kw[a] for a in order]
    return getattr(B.load(), name)(*args)


def _size(name, *args):
    out = ctypes.c_size_t(0)
    st = getattr(B.load(), name)(*args, ctypes.byref(out))
    return st, out.value


LOGPROBS = "x batch n stride dt inv_t tokens m k lp h stats top at ws ws_bytes stream".split()
LOGPROBS_GOOD = dict(GOOD, tokens=0x20000, m=2, k=4, lp=0x30000, h=0x40000, stats=0x50000, top=0x60000, at=0x70000, ws=0x80000, ws_bytes=1 << 40, stream=None)
LOGPROBS_BACK = "x batch n stride dt inv_t tokens m stats g h gh out out_stride stream".split()
LOGPROBS_BACK_GOOD = dict(GOOD, tokens=0x20000, m=2, stats=0x30000, g=0x40000, h=0x50000, gh=0x60000, out=0x100000, out_stride=1000, stream=None)
LISTS = "x batch n stride dt inv_t values values_dt columns k lse".split()
LISTS_GOOD = dict(GOOD, values=0x20000, values_dt=2, columns=0x30000, k=7, lse=0x40000)
DISTILL = LISTS + "loss stats ws ws_bytes stream".split()
DISTILL_GOOD = dict(LISTS_GOOD, loss=0x50000, stats=0x60000, ws=0x80000, ws_bytes=1 << 40, stream=None)
DISTILL_BACK = LISTS + "stats g out out_stride stream".split()
DISTILL_BACK_GOOD = dict(LISTS_GOOD, stats=0x50000, g=0x60000, out=0x100000, out_stride=1000, stream=None)
STEP = LISTS + "weights loss out out_stride ws ws_bytes stream".split()
STEP_GOOD = dict(LISTS_GOOD, weights=0x50000, loss=0x60000, out=0x100000, out_stride=1000, ws=0x80000, ws_bytes=1 << 40, stream=None)
ROUTE = "x batch n stride dt bias groups topk_groups k flags scale weights experts counts stream".split()
ROUTE_GOOD = dict(GOOD, bias=0x20000, groups=10, topk_groups=3, k=6, flags=7, scale=1.0, weights=0x30000, experts=0x40000, counts=0x50000, stream=None)
ROUTE_BACK = "x batch n stride dt experts k flags scale g out out_stride stream".split()
ROUTE_BACK_GOOD = dict(GOOD, experts=0x20000, k=6, flags=3, scale=1.0, g=0x30000, out=0x100000, out_stride=1000, stream=None)

ROWS_BAD = [dict(x=None), dict(batch=0), dict(batch=-1), dict(batch=1 << 31), dict(n=0), dict(n=(1 << 31) + 1), dict(stride=999), dict(dt=3), dict(dt=-1)]
TEMPERATURES_BAD = [dict(inv_t=v) for v in (0.0, -1.0, float("inf"), float("nan"), 1e-38, 3e38)]


@pytest.mark.parametrize("name,order,good,invalid,misaligned", [
    ("rtopk_logprobs", LOGPROBS, LOGPROBS_GOOD,
     ROWS_BAD + TEMPERATURES_BAD + [dict(m=-1), dict(k=-1), dict(k=1001), dict(tokens=None), dict(lp=None), dict(top=None), dict(at=None), dict(ws=None)],
     [dict(x=0x10002), dict(tokens=0x20004), dict(lp=0x30002), dict(h=0x40001), dict(stats=0x50002), dict(top=0x60001), dict(at=0x70004), dict(ws=0x80080)]),
    ("rtopk_logprobs_backward", LOGPROBS_BACK, LOGPROBS_BACK_GOOD,
     ROWS_BAD + TEMPERATURES_BAD + [dict(m=-1), dict(tokens=None), dict(stats=None), dict(g=None), dict(h=None), dict(out=None), dict(out_stride=999),
                                    dict(out=0x10000), dict(out=0x10000 + 11996), dict(out=0x10000 - 11996)],
     [dict(x=0x10001), dict(out=0x100002), dict(tokens=0x20004), dict(stats=0x30001), dict(g=0x40002), dict(h=0x50002), dict(gh=0x60003)]),
    ("rtopk_distill", DISTILL, DISTILL_GOOD,
     ROWS_BAD + TEMPERATURES_BAD + [dict(values=None), dict(values_dt=5), dict(columns=None), dict(k=0), dict(loss=None), dict(ws=None)],
     [dict(x=0x10001), dict(values=0x20001), dict(columns=0x30004), dict(lse=0x40001), dict(loss=0x50002), dict(stats=0x60001), dict(ws=0x80010)]),
    ("rtopk_distill_backward", DISTILL_BACK, DISTILL_BACK_GOOD,
     ROWS_BAD + TEMPERATURES_BAD + [dict(values=None), dict(columns=None), dict(k=0), dict(stats=None), dict(g=None), dict(out=None), dict(out_stride=10), dict(out=0x10400)],
     [dict(out=0x100001), dict(values=0x20001), dict(columns=0x30001), dict(stats=0x50001), dict(g=0x60002)]),
    ("rtopk_distill_step", STEP, STEP_GOOD,
     ROWS_BAD + TEMPERATURES_BAD + [dict(values=None), dict(columns=None), dict(k=0), dict(weights=None), dict(loss=None), dict(out=None), dict(out_stride=10), dict(out=0x10400),
                                    dict(ws=None)],
     [dict(out=0x100001), dict(values=0x20001), dict(columns=0x30001), dict(weights=0x50001), dict(loss=0x60002), dict(ws=0x80010)]),
    ("rtopk_route", ROUTE, ROUTE_GOOD,
     ROWS_BAD + [dict(n=1025, stride=1025), dict(groups=0), dict(groups=3), dict(groups=100), dict(topk_groups=0), dict(topk_groups=11), dict(k=0), dict(k=65),
                 dict(groups=50, topk_groups=1, k=21), dict(flags=8), dict(scale=float("nan")), dict(weights=None), dict(experts=None)],
     [dict(x=0x10001), dict(bias=0x20001), dict(weights=0x30002), dict(experts=0x40004), dict(counts=0x50004)]),
    ("rtopk_route_backward", ROUTE_BACK, ROUTE_BACK_GOOD,
     ROWS_BAD + [dict(n=1025, stride=1025), dict(k=0), dict(k=65), dict(flags=8), dict(scale=float("nan")), dict(experts=None), dict(g=None), dict(out=None), dict(out_stride=1),
                 dict(out=0x10000)],
     [dict(x=0x10001), dict(out=0x100002), dict(experts=0x20004), dict(g=0x30001)]),
])
def test_arguments_are_checked_before_anything_is_launched(name, order, good, invalid, misaligned):
    # (every address is made up: a call that got as far as a launch would not come back with these)
    for bad in invalid:
        assert _call(name, order, **dict(good, **bad)) == 1, (name, bad)
    for bad in misaligned:
        assert _call(name, order, **dict(good, **bad)) == 3, (name, bad)
    if "ws_bytes" in good:
        assert _call(name, order, **dict(good, ws_bytes=0)) == 2


def test_workspaces():
    for args in ((0, 10, 1, 1, 0), (1, 0, 1, 0, 0), (1, 10, -1, 0, 0), (1, 10, 1, 11, 0), (1, 10, 1, 1, 3), (1, (1 << 31) + 1, 1, 0, 0)):
        assert _size("rtopk_logprobs_workspace_bytes", *args)[0] == 1, args
    for args in ((0, 10, 1, 0), (1, 0, 1, 0), (1, 10, 0, 0), (1, 10, 1, 3)):
        assert _size("rtopk_distill_workspace_bytes", *args)[0] == 1, args
    assert B.load().rtopk_logprobs_workspace_bytes(1, 10, 1, 1, 0, None) == 1
    for batch, n in ((1, 1), (1, 131072), (1024, 131072), (70000, 50), (2, 1 << 31)):
        st, need = _size("rtopk_logprobs_workspace_bytes", batch, n, 1, 0, 2)
        assert st == 0 and 256 <= need <= (1 << 20) + 64 * batch
        st, need = _size("rtopk_distill_workspace_bytes", batch, n, 10, 2)
        assert st == 0 and 32 * batch <= need <= (4 << 20) + 256 * batch


def test_python_entry_points_refuse_cpu_tensors():
    torch = pytest.importorskip("torch")
    import paper_2501_14336_amd as package
    x, at = torch.zeros((2, 10)), torch.zeros((2, 1), dtype=torch.int64)
    for call in (lambda: package.logprobs(x, at), lambda: package.distill(x, x[:, :1], at), lambda: package.distill_step(x, x[:, :1], at, x[:, 0]),
                 lambda: package.route(x, 2), lambda: package.logprobs_backward(x, at, x, x), lambda: package.route_backward(x, at, x)):
        with pytest.raises(B.RtopkError):
            call()
