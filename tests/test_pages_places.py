"""Page calls refuse what does not lie where the tables lie, and tables that no GPU can read."""
import pytest
import torch

from paper_2407_07304_b200 import binding as slim

PAGES, ROWS, STRIDE = 6, 2, 3


def i32(n):
    return torch.zeros(n, dtype=torch.int32)


def setup(device, on_host=()):
    put = lambda name, t: t if name in on_host else t.to(device)  # noqa: E731
    place = lambda name: "cpu" if name in on_host else device  # noqa: E731
    return dict(layers=slim.PageLayers([slim.SlimCache4(1, 1, 1, device=place("layers"), num_pages=PAGES)]),
                src=slim.SlimPages.empty(PAGES, ROWS, STRIDE, place("src")), dst=slim.SlimPages.empty(PAGES, ROWS, STRIDE, place("dst")),
                parent=put("parent", i32(ROWS)), kv=put("kv", i32(ROWS)), len=put("len", i32(ROWS)), result=put("result", i32(2)),
                ws=put("ws", slim.pages_workspace(PAGES, ROWS, "cpu")))


CALLS = {
    "fork": (("layers", "src", "dst", "parent", "kv", "len", "result", "ws"),
             lambda f: slim.slim_pages_fork(f["layers"], f["src"], f["dst"], f["parent"], f["kv"], f["len"], f["result"], f["ws"])),
    "grow": (("src", "kv", "result", "ws"), lambda f: slim.slim_pages_grow(f["src"], f["kv"], 1, f["result"], f["ws"])),
    "compact": (("layers", "src", "dst", "result", "ws"), lambda f: slim.slim_pages_compact(f["layers"], f["src"], f["dst"], f["result"], f["ws"])),
}


@pytest.mark.parametrize("call", CALLS)
def test_host_memory(call):
    """Everything fits: what is left to refuse is that no GPU can read any of it."""
    with pytest.raises(slim.SlimError, match="not a GPU's") as e:
        CALLS[call][1](setup("cpu"))
    assert e.value.code == slim.SLIM_ERR_INVALID_ARG


def test_tables_of_two_places():
    with pytest.raises(TypeError):
        slim.SlimPages(i32(PAGES), torch.zeros((ROWS, STRIDE), dtype=torch.int32, device="meta"), i32(ROWS))


@pytest.mark.gpu
@pytest.mark.parametrize("call,name", [(c, n) for c, (names, _) in CALLS.items() for n in names])
def test_one_of_them_on_the_host(call, name):
    with pytest.raises(slim.SlimError, match="device|lie|not a GPU's"):
        CALLS[call][1](setup("cuda", (name,)))


@pytest.mark.gpu
@pytest.mark.parametrize("call", CALLS)
def test_all_on_the_gpu(call):
    f = setup("cuda")
    CALLS[call][1](f)
    assert f["src"].refs.sum() == (ROWS if call == "grow" else 0)


@pytest.mark.gpu
def test_layers_of_two_places():
    with pytest.raises(ValueError):
        slim.PageLayers([slim.SlimCache4(1, 1, 1, device=d, num_pages=PAGES) for d in ("cpu", "cuda")])
