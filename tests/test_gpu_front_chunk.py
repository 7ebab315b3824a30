"""The native argument checks of growing rows, rotary positions and the attention of several new
tokens against the general path in Python: the same outputs, or the same error."""
import numpy as np
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import device, say
from test_gpu_front_paged import General, Spy, raw, sealed, wide

pytestmark = pytest.mark.gpu

R, N, HQ, HKV, D, PAGE, P, COLS = 3, 12, 4, 2, 64, 16, 15, 5


def inputs():
    dev = device()
    g = torch.Generator(device=dev).manual_seed(8)
    r = lambda *s, dt=torch.bfloat16: torch.randn(*s, device=dev, dtype=dt, generator=g)
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev)
    ids = torch.randperm(P, device=dev, generator=g).int()
    table = torch.full((R, COLS), -1, dtype=torch.int32, device=dev)
    table[0, :2], table[1, :3], table[2, :1] = ids[:2], ids[2:5], ids[5:6]
    return dict(q=r(N, HQ, D), K=r(P, HKV, PAGE, D), V=r(P, HKV, PAGE, D), table=table, n=i(20, 40, 7), off=i(0, 5, 6, 11), out=r(N, HQ, D),
                ws=api.new_workspace(api.paged_chunk_attn_workspace_bytes(N, R, HQ, HKV, PAGE, COLS, D), dev),
                want=i(60, 20, 30), free=torch.cat([ids[6:], ids[:6] * 0]), count=i(9), page=PAGE, start=i(1, 2, 3), offs=i(9, 9, 9, 9),
                pos=torch.zeros(70, dtype=torch.int32, device=dev), slots=torch.zeros(70, dtype=torch.int64, device=dev),
                ws2=api.new_workspace(api.paged_resize_workspace_bytes(R, 70), dev), k=r(N, HKV, D), ko=r(N, HKV, D),
                at=torch.arange(N, device=dev).int(), freq=api.rotary_frequencies(D, device=dev), inter=False, mag=1.0)


CALLS = {
    "chunk": lambda x: api.paged_chunk_attn(x["q"], x["K"], x["V"], x["table"], x["n"], x["off"], out=x["out"], workspace=x["ws"],
                                            scale=x.get("scale")),
    "resize": lambda x: api.paged_resize(x["table"], x["n"], x["want"], x["free"], x["count"], x["page"], x["start"], x["offs"], x["pos"],
                                         x["slots"], workspace=x["ws2"]),
    "resize plain": lambda x: api.paged_resize(x["table"], x["n"], x["want"], x["free"], x["count"], x["page"], workspace=x["ws2"]),
    "rotary": lambda x: api.rotary(x["q"], x["at"], x["freq"], k=x["k"], out=x["out"], k_out=x["ko"], interleaved=x["inter"], magnitude=x["mag"]),
    "rotary in place": lambda x: api.rotary(x["q"], x["at"], x["freq"], k=x["k"], out=x["q"], k_out=x["k"], interleaved=x["inter"]),
    "rotary alone": lambda x: api.rotary(x["q"], x["at"], x["freq"], out=x["out"], magnitude=x["mag"]),
}
CHANGES = {
    "plain": {}, "scale": dict(scale=0.5), "scale int": dict(scale=1), "scale numpy": dict(scale=np.float32(0.5)),
    "scale inf": dict(scale=float("inf")), "scale text": dict(scale="x"), "page numpy": dict(page=np.int64(16)), "page 0": dict(page=0),
    "page text": dict(page="x"), "page large": dict(page=2**40), "interleaved": dict(inter=True), "interleaved 1": dict(inter=1),
    "magnitude int": dict(mag=2), "magnitude text": dict(mag="x"), "magnitude numpy": dict(mag=np.float64(1.5)),
    "token major": lambda x: {n: x[n].transpose(1, 2).contiguous().transpose(1, 2) for n in "KV"},
    "K alone token major": lambda x: dict(K=x["K"].transpose(1, 2).contiguous().transpose(1, 2)),
    "rows strided": lambda x: {n: x[n].transpose(2, 3).contiguous().transpose(2, 3) for n in "KV"},
    "cut": lambda x: dict(zip("qk", torch.cat([x["q"], x["k"], x["ko"]], 1).split([HQ, HKV, HKV], 1))),
    "odd stride": lambda x: {n: torch.cat([x[n], x[n][..., :1]], -1)[..., :D] for n in "qk"},
    "q f32": lambda x: dict(q=x["q"].float()), "k f32": lambda x: dict(k=x["k"].float()), "ko f32": lambda x: dict(ko=x["ko"].float()),
    "all f32": lambda x: {n: x[n].float() for n in ("q", "K", "V", "k", "ko", "out")},
    "f16": lambda x: {n: x[n].half() for n in ("q", "K", "V", "k", "ko", "out")},
    "q 2d": lambda x: dict(q=x["q"][0]), "k rows": lambda x: dict(k=x["k"][:2]), "k narrow": lambda x: dict(k=x["k"][..., :32], ko=x["ko"][..., :32]),
    "k none": dict(k=None), "ko none": dict(ko=None), "no k": dict(k=None, ko=None), "V none": dict(V=None),
    "table long": lambda x: dict(table=x["table"].long()), "table ld": lambda x: dict(table=wide(x["table"])),
    "table columns": lambda x: dict(table=x["table"].t().contiguous().t()), "table rows": lambda x: dict(table=x["table"][:2]),
    "table cpu": lambda x: dict(table=x["table"].cpu()), "table empty": lambda x: dict(table=x["table"][:, :0]),
    "n long": lambda x: dict(n=x["n"].long()), "off short": lambda x: dict(off=x["off"][:3], offs=x["offs"][:3]),
    "out none": dict(out=None), "out q": lambda x: dict(out=x["q"]), "out f32": lambda x: dict(out=x["out"].float()),
    "out strided": lambda x: dict(out=x["out"].transpose(0, 1).contiguous().transpose(0, 1)),
    "want short": lambda x: dict(want=x["want"][:2]), "want n": lambda x: dict(want=x["n"]), "free 2d": lambda x: dict(free=x["free"][None]),
    "free long": lambda x: dict(free=x["free"].long()), "count two": lambda x: dict(count=x["want"][:2]), "start none": dict(start=None),
    "pos none": dict(pos=None), "slots none": dict(slots=None), "slots int": lambda x: dict(slots=x["slots"].int()),
    "slots short": lambda x: dict(slots=x["slots"][:9]), "pos long": lambda x: dict(pos=x["pos"].long()), "start q": lambda x: dict(start=x["q"]),
    "at long": lambda x: dict(at=x["at"].long()), "at short": lambda x: dict(at=x["at"][:3]), "freq f32": lambda x: dict(freq=x["freq"].float()),
    "freq long": lambda x: dict(freq=torch.cat([x["freq"]] * 2)), "freq part": lambda x: dict(freq=x["freq"][:5]),
    "freq none": lambda x: dict(freq=x["freq"][:0]), "freq strided": lambda x: dict(freq=x["freq"][::2]),
    "small workspace": lambda x: dict(ws=x["ws"][:8], ws2=x["ws2"][:8]), "workspace none": dict(ws=None, ws2=None),
    "q parameter": lambda x: dict(q=torch.nn.Parameter(x["q"])), "sealed": lambda x: dict(K=sealed(x["K"]), k=sealed(x["k"]), free=sealed(x["free"])),
    "no rows": lambda x: {**{n: x[n][:0] for n in ("q", "k", "ko", "table", "n", "want", "start", "out", "at")}, "off": x["off"][:1], "offs": x["offs"][:1]},
}


def outcome(call, change):
    x = inputs()
    x.update(change(x) if callable(change) else change)
    with torch.no_grad():
        try:
            r = CALLS[call](x)
            torch.cuda.synchronize()
        except Exception as e:  # noqa: BLE001 - both paths have to raise the same
            return type(e).__name__, str(e).split("0x")[0]
    # tokens of no row are uninitialised in an output made by the call
    seen = [t[:11] for t in ([r] if isinstance(r, torch.Tensor) else list(r) if r is not None else [])]
    made = [x[n] for n in ("table", "n", "count", "start", "offs", "pos", "slots", "q", "k") if isinstance(x[n], torch.Tensor)]
    kept = x["free"][:int(x["count"][0])] if "resize" in call else x["free"]
    return [raw(t) for t in seen + made + [kept]]


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
        assert spy.seen[-1] == 0 and None not in spy.seen, name
