"""The native argument checks of the paged cache's and the sampling's calls
against the general path in Python: the same outputs, or the same error."""
import numpy as np
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import device, say

pytestmark = pytest.mark.gpu

R, HQ, HKV, D, PAGE, P, COLS, V = 3, 4, 2, 64, 16, 12, 4, 101


class General:
    """Stands in for the native module: declines every call."""

    def __getattr__(self, name):
        return lambda *a: None


class Spy:
    """The native module, with what each call returned."""

    def __init__(self, native):
        self.native, self.seen = native, []

    def __getattr__(self, name):
        def call(*a):
            r = getattr(self.native, name)(*a)
            self.seen.append(r)
            return r
        return call


def inputs():
    dev = device()
    g = torch.Generator(device=dev).manual_seed(7)
    r = lambda *s, dt=torch.bfloat16: torch.randn(*s, device=dev, dtype=dt, generator=g)
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev)
    f = lambda a: torch.full((R,), a, device=dev)
    return dict(
        q=r(R, HQ, D), K=r(P, HKV, PAGE, D), V=r(P, HKV, PAGE, D), k=r(R, HKV, D), v=r(R, HKV, D),
        table=torch.randperm(P, device=dev, generator=g).view(R, COLS).int(), n=i(5, 33, 64), start=i(4, 0, 17),
        off=i(0, 1, 1, 3), out=r(R, HQ, D), ws=api.new_workspace(api.paged_attn_workspace_bytes(R, HQ, HKV, PAGE, COLS, D), dev),
        x=r(R, V, dt=torch.float32), u=torch.rand(R, device=dev, generator=g), T=f(0.8), tk=i(10, 0, 3), tp=f(0.9), mp=f(0.01),
        so=(i(1, 2, 3), f(0.0)), ws2=api.new_workspace(api.token_sample_workspace_bytes(R, V), dev))


def sealed(x):
    """A tensor whose data pointer torch refuses to give (it throws)."""
    x = x.clone()
    torch._C._set_throw_on_mutable_data_ptr(x)
    return x


def wide(x):
    return torch.cat([x, x], dim=1)[:, :x.shape[1]]


CALLS = {
    "append": lambda x: api.paged_append(x["K"], x["V"], x["k"], x["v"], x["table"], x["start"], x["off"]),
    "append one": lambda x: api.paged_append(x["K"], x["V"], x["k"], x["v"], x["table"], x["start"]),
    "attn": lambda x: api.paged_attn(x["q"], x["K"], x["V"], x["table"], x["n"], out=x["out"], workspace=x["ws"],
                                     scale=x.get("scale")),
    "attn new": lambda x: api.paged_attn(x["q"], x["K"], x["V"], x["table"], x["n"], out=x["out"], workspace=x["ws"],
                                         k=x["k"], v=x["v"], scale=x.get("scale")),
    "sample": lambda x: api.token_sample(x["x"], x["u"], x["T"], x["tk"], x["tp"], x["mp"], out=x["so"], workspace=x["ws2"]),
    "sample plain": lambda x: api.token_sample(x["x"], x["u"], out=x["so"], workspace=x["ws2"]),
}
CHANGES = {
    "plain": {}, "scale": dict(scale=0.5), "scale int": dict(scale=1), "scale numpy": dict(scale=np.float32(0.5)),
    "scale inf": dict(scale=float("inf")), "scale text": dict(scale="x"),
    "token major": lambda x: {n: x[n].transpose(1, 2).contiguous().transpose(1, 2) for n in "KV"},
    "K alone token major": lambda x: dict(K=x["K"].transpose(1, 2).contiguous().transpose(1, 2)),
    "rows strided": lambda x: {n: x[n].transpose(2, 3).contiguous().transpose(2, 3) for n in "KV"},
    "cut": lambda x: dict(zip("qkv", torch.cat([x["q"], x["k"], x["v"]], 1).split([HQ, HKV, HKV], 1))),
    "odd stride": lambda x: {n: torch.cat([x[n], x[n][..., :1]], -1)[..., :D] for n in "qkv"},
    "q f32": lambda x: dict(q=x["q"].float()), "k f32": lambda x: dict(k=x["k"].float()),
    "all f32": lambda x: {n: x[n].float() for n in ("q", "K", "V", "k", "v", "out")},
    "f16": lambda x: {n: x[n].half() for n in ("q", "K", "V", "k", "v", "out", "x")},
    "q 2d": lambda x: dict(q=x["q"][0]), "k rows": lambda x: dict(k=x["k"][:2], v=x["v"][:2]), "V none": dict(V=None),
    "k none": dict(k=None), "table long": lambda x: dict(table=x["table"].long()), "table ld": lambda x: dict(table=wide(x["table"])),
    "table columns": lambda x: dict(table=x["table"].t().contiguous().t()), "table rows": lambda x: dict(table=x["table"][:2]),
    "table cpu": lambda x: dict(table=x["table"].cpu()), "table empty": lambda x: dict(table=x["table"][:, :0]),
    "n long": lambda x: dict(n=x["n"].long(), start=x["start"].long()), "off short": lambda x: dict(off=x["off"][:3]),
    "out none": dict(out=None), "out q": lambda x: dict(out=x["q"]), "out f32": lambda x: dict(out=x["out"].float()),
    "so one": lambda x: dict(so=x["so"][:1]), "so swapped": lambda x: dict(so=x["so"][::-1]),
    "small workspace": lambda x: dict(ws=x["ws"][:8], ws2=x["ws2"][:8]), "workspace none": dict(ws=None, ws2=None),
    "x bf16": lambda x: dict(x=x["x"].bfloat16()), "x wide": lambda x: dict(x=wide(x["x"])), "x columns": lambda x: dict(x=x["x"].t().contiguous().t()),
    "u double": lambda x: dict(u=x["u"].double()), "T float": dict(T=0.8), "tk long": lambda x: dict(tk=x["tk"].long()),
    "tp none": dict(tp=None), "mp two": lambda x: dict(mp=x["mp"][:2]), "q parameter": lambda x: dict(q=torch.nn.Parameter(x["q"]), x=torch.nn.Parameter(x["x"])),
    "sealed": lambda x: dict(K=sealed(x["K"]), x=sealed(x["x"])),
    "no rows": lambda x: {**{n: x[n][:0] for n in ("q", "k", "v", "table", "n", "start", "out", "x", "u", "T", "tk", "tp", "mp")},
                          "so": tuple(o[:0] for o in x["so"]), "off": x["off"][:1]},
}


def raw(t):
    c = t.detach().cpu().contiguous()
    return str(t.dtype), tuple(t.shape), c.view(torch.uint8).numpy().tobytes() if c.numel() else b""


def outcome(call, change):
    x = inputs()
    x.update(change(x) if callable(change) else change)
    try:
        r = CALLS[call](x)
        torch.cuda.synchronize()
    except Exception as e:  # noqa: BLE001 - both paths have to raise the same
        return type(e).__name__, str(e).split("0x")[0]
    seen = [r] if isinstance(r, torch.Tensor) else list(r) if r is not None else []
    seen += [x[n] for n in ("K", "V")]
    return [raw(t) if t is not None else None for t in seen]


@pytest.mark.parametrize("call", CALLS)
def test_native_checks_take_and_refuse_what_the_general_path_does(call, monkeypatch):
    for name, change in CHANGES.items():
        say(f"[front] {call}: {name}")
        monkeypatch.setattr(api, "_fast", None)
        a = outcome(call, change)
        monkeypatch.setattr(api, "_fast", General())
        b = outcome(call, change)
        assert a == b, (call, name, a if isinstance(a, tuple) else "", b if isinstance(b, tuple) else "")


@pytest.mark.parametrize("call", CALLS)
def test_the_native_module_takes_the_plain_call(call, monkeypatch):
    for name in ("plain", "token major", "cut", "table ld"):
        spy = Spy(api._load_fast())
        monkeypatch.setattr(api, "_fast", spy)
        outcome(call, CHANGES[name])
        assert spy.seen == [0], name
