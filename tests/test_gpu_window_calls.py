"""Windowed attention and the cache through the marshalling extension and through ctypes: the same bits for calls that it takes, and for
every call that one of the two refuses the same error from both."""
import pytest
import torch

from paper_2512_05754_amd import binding
from test_gpu_calls import both

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def normal(shape, seed, dtype=torch.bfloat16):
    return torch.randn(shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).to(dtype)


def state(dtype, L=40, n=300, B=2, Hq=4, Hkv=2, d=64, page=32, bits=4):
    q, do = (normal((B, Hq, L, d), i, dtype) for i in (1, 2))
    k, v = (normal((B, n, Hkv, d), i, dtype).transpose(1, 2) for i in (3, 4))  # not contiguous
    pages = -(-n // page)
    table = torch.randperm(B * pages, generator=torch.Generator().manual_seed(5)).view(B, pages).to(torch.int32).to(DEV)
    lens = torch.tensor([n, n - 100], dtype=torch.int32, device=DEV)
    cache = binding.cache_empty(B * pages, Hkv, page, d, bits, DEV).zero_()
    starts = torch.zeros(B, dtype=torch.int32, device=DEV)
    return dict(q=q, k=k, v=v, do=do, table=table, lens=lens, cache=cache, starts=starts, bits=bits, page=page, counts=lens)


def same(a, b):
    return a.shape == b.shape and a.dtype == b.dtype and a.stride() == b.stride() and torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


WINDOW = dict(left=100, right=0, sinks=3, chunk=1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("given", [False, True])
def test_the_same_bits(usv, monkeypatch, dtype, given):
    s = state(dtype)
    q, k, v, do = (s[n] for n in ("q", "k", "v", "do"))

    def run():
        more = [{}, {}]
        if given:
            ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
            more = [dict(out=torch.empty_like(q), lse=torch.empty(q.shape[:3], device=DEV), workspace=ws),
                    dict(dq=torch.empty_like(q), dk=torch.empty(k.shape, dtype=dtype, device=DEV), dv=torch.empty_like(v), workspace=ws)]
        out, lse = binding.window_attn(q, k, v, **WINDOW, seq_lens=s["lens"], return_lse=True, **more[0])
        alone = binding.window_attn(q, k, v, 100, sinks=3, seq_lens=s["lens"], scale=0.2, q_start=None)
        grads = binding.window_attn_backward(q, k, v, out, lse, do, **WINDOW, seq_lens=s["lens"], **more[1])
        if given:
            assert out is more[0]["out"] and lse is more[0]["lse"] and all(g is more[1][n] for g, n in zip(grads, ("dq", "dk", "dv")))
        got = [out, lse, alone, *grads]
        assert binding.cache_write(s["cache"], k, v, s["table"], s["starts"], bits=s["bits"], counts=s["counts"]) is s["cache"]
        got.append(s["cache"].clone())
        kv = dict(k=torch.zeros(k.shape, dtype=dtype, device=DEV), v=torch.zeros(k.shape, dtype=dtype, device=DEV)) if given else {}
        counts = s["counts"] if given else None
        got += binding.cache_read(s["cache"], s["table"], s["starts"], k.shape[2], head_dim=64, bits=s["bits"], counts=counts, dtype=dtype, **kv)
        if dtype == torch.bfloat16:
            got += binding.cache_attn(q, s["cache"], s["table"], s["lens"], **WINDOW, bits=s["bits"], return_lse=True, **more[0])
        return [t.clone() for t in got]

    a, b, returned = both(monkeypatch, run)
    assert isinstance(a, list) and isinstance(b, list), (a, b)
    names = ["window_attn", "window_attn_backward", "cache_write", "cache_read"] + (["cache_attn"] if dtype == torch.bfloat16 else [])
    assert sorted(returned) == sorted(names) and all(type(returned[n]) in (torch.Tensor, tuple) for n in names)  # the extension did it all
    for i, (x, y) in enumerate(zip(a, b)):
        assert same(x, y), i


def test_few_rows_and_nothing(usv, monkeypatch):
    """Calls that make scratch of their own (keys shared out), and empty ones."""
    s = state(torch.bfloat16, L=1, n=9000)
    q, k, v = s["q"], s["k"], s["v"]
    binding.cache_write(s["cache"], k, v, s["table"], s["starts"])
    assert binding.window_workspace_bytes(q, k, -1) > 0 and binding.cache_attn_workspace_bytes(q, s["cache"], s["table"]) > 0

    def run():
        got = [*binding.window_attn(q, k, v, -1, return_lse=True), *binding.cache_attn(q, s["cache"], s["table"], s["lens"], return_lse=True)]
        got += binding.window_attn(q[:, :, :0], k, v, -1, return_lse=True)
        got += binding.window_attn(q, k[:, :, :0], v[:, :, :0], -1, return_lse=True)
        got += binding.cache_read(s["cache"], s["table"], s["starts"], 0, head_dim=64)
        got += binding.cache_attn(q[:, :, :0], s["cache"], s["table"], s["lens"], return_lse=True)
        return [t.clone() for t in got]

    a, b, returned = both(monkeypatch, run)
    assert isinstance(a, list) and isinstance(b, list), (a, b)
    assert all(type(x) is tuple for x in returned.values())
    for i, (x, y) in enumerate(zip(a, b)):
        assert same(x, y), i


CHANGES = {
    "cpu q": lambda s: dict(q=s["q"].cpu()), "half": lambda s: dict(q=s["q"].half(), k=s["k"].half(), v=s["v"].half()), "k of another type": lambda s: dict(k=s["k"].float()),
    "three dimensions": lambda s: dict(q=s["q"][0]), "v shorter": lambda s: dict(v=s["v"][:, :, :5]), "batch differs": lambda s: dict(q=s["q"][:1]),
    "one key row for all": lambda s: dict(k=s["k"][:, :, :1].expand(s["k"].shape)), "channels apart": lambda s: dict(q=s["q"].repeat(1, 1, 1, 2)[..., ::2]),
    "not a tensor": lambda s: dict(q=[1.0]), "k not a tensor": lambda s: dict(k=None), "head dimension": lambda s: dict(q=s["q"][..., :32], k=s["k"][..., :32], v=s["v"][..., :32]),
    "key heads": lambda s: dict(k=s["k"].repeat(1, 2, 1, 1)[:, :3], v=s["v"].repeat(1, 2, 1, 1)[:, :3]), "lens int64": lambda s: dict(lens=s["lens"].long()),
    "lens too many": lambda s: dict(lens=s["lens"].repeat(2)), "lens on the CPU": lambda s: dict(lens=s["lens"].cpu()), "chunk 0": lambda s: dict(chunk=0), "chunk a string": lambda s: dict(chunk="a"),
    "left far": lambda s: dict(left=1 << 31), "sinks negative": lambda s: dict(sinks=-1), "scale nan": lambda s: dict(scale=float("nan")), "scale a string": lambda s: dict(scale="x"),
    "out short": lambda s: dict(out=s["q"][:, :, :3]), "out fp32": lambda s: dict(out=s["q"].float()), "out overlaps": lambda s: dict(out=s["q"][:, :1].expand(s["q"].shape)),
    "lse fp16": lambda s: dict(lse=torch.zeros(s["q"].shape[:3], device=DEV).half()), "lse short": lambda s: dict(lse=torch.zeros(3, device=DEV)),
    "workspace not contiguous": lambda s: dict(workspace=torch.zeros(64, device=DEV)[::2]), "workspace a number": lambda s: dict(workspace=5),
    "bits 3": lambda s: dict(bits=3), "bits 16": lambda s: dict(bits=16), "bits 8": lambda s: dict(bits=8), "cache of another type": lambda s: dict(cache=s["cache"].view(torch.int8)),
    "cache of two dimensions": lambda s: dict(cache=s["cache"].flatten(1)), "table int64": lambda s: dict(table=s["table"].long()), "table of one dimension": lambda s: dict(table=s["table"][0]),
    "table of another batch": lambda s: dict(table=s["table"][:1]), "starts int64": lambda s: dict(starts=s["starts"].long()), "starts short": lambda s: dict(starts=s["starts"][:1]),
    "counts short": lambda s: dict(counts=s["counts"][:1]), "rows negative": lambda s: dict(rows=-1), "rows too many": lambda s: dict(rows=(1 << 26) + 1),
    "read into another type": lambda s: dict(into=torch.zeros(s["k"].shape, dtype=torch.float16, device=DEV)), "read into another shape": lambda s: dict(into=s["q"]),
    "dtype": lambda s: dict(dtype=torch.float16), "no lens": lambda s: dict(lens=None),
}


@pytest.mark.parametrize("what", CHANGES)
def test_the_same_errors(usv, monkeypatch, what):
    """A call with one thing wrong: whichever functions take that thing refuse it alike, the others answer alike."""
    s = state(torch.bfloat16)
    lse0 = torch.zeros(s["q"].shape[:3], device=DEV)
    t = dict(s, left=10, sinks=1, chunk=1, scale=0.0, rows=5, dtype=torch.bfloat16, out=None, lse=None, workspace=None, into=None)
    t.update(CHANGES[what](s))
    window = dict(left=t["left"], sinks=t["sinks"], chunk=t["chunk"], scale=t["scale"])
    calls = {
        "window_attn": lambda: binding.window_attn(t["q"], t["k"], t["v"], **window, seq_lens=t["lens"], out=t["out"], lse=t["lse"], workspace=t["workspace"]),
        "window_attn_backward": lambda: binding.window_attn_backward(t["q"], t["k"], t["v"], s["q"], lse0 if t["lse"] is None else t["lse"], s["do"], **window, seq_lens=t["lens"],
                                                                     dq=t["out"], workspace=t["workspace"]),
        "cache_write": lambda: binding.cache_write(t["cache"], t["k"], t["v"], t["table"], t["starts"], bits=t["bits"], counts=t["counts"]),
        "cache_read": lambda: binding.cache_read(t["cache"], t["table"], t["starts"], t["rows"], head_dim=64, bits=t["bits"], counts=t["counts"], dtype=t["dtype"], k=t["into"]),
        "cache_attn": lambda: binding.cache_attn(t["q"], t["cache"], t["table"], t["lens"], **window, bits=t["bits"], out=t["out"], lse=t["lse"], workspace=t["workspace"]),
    }
    refused = 0
    for name, f in calls.items():
        if what == "rows too many" and name != "cache_read":
            continue
        a, b, _ = both(monkeypatch, f)
        error = isinstance(a, tuple) and isinstance(a[0], type)
        assert error == (isinstance(b, tuple) and isinstance(b[0], type)), (name, a, b)
        if error:
            refused += 1
            assert a == b, name
    assert refused
