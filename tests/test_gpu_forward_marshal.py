"""The native argument marshalling of the calls around the forward against the
Python marshalling of the same wrappers: the same outputs, and the same
exceptions for arguments that either refuses."""
import pytest
import torch

from tests import forward_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2510_22876_amd import specdec
    assert specdec._native is not None, "the native marshalling is not built"
    return specdec


def _calls(sd, page):
    """{name: (function, keyword arguments, names of the written tensors)} on buffers of their own."""
    c = ref.Cache([9, 0, 33], 3, 2, 32, page)
    c.fill(3, torch.Generator().manual_seed(1))
    g = torch.Generator(device="cuda").manual_seed(2)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    B, T, Hq, D, V = 3, 3, 4, 32, 501
    i32 = dict(dtype=torch.int32, device="cuda")
    half = torch.rand(16, generator=g, device="cuda")
    where = dict(table=c.table, lens=c.lens) if page else dict(W_in=c.W_in, pad_in=c.pad)
    cache = "pool" if page else "kv"
    append = dict(qkv=n(B, T, Hq + 4, D), layer=1, q_out=torch.zeros((B, T, Hq, D), dtype=torch.bfloat16, device="cuda"),
                  inv_freq=half, q_norm=n(D), k_norm=n(D), eps=1e-5, adjacent=True, dev_status=torch.zeros(1, **i32),
                  **{cache: c.kv.cuda()}, **where)
    attend = dict(q=n(B, T, Hq, D).bfloat16(), layer=1, out=torch.zeros((B, T, Hq, D), dtype=torch.bfloat16, device="cuda"),
                  workspace=sd.alloc_attend_workspace(B, T, Hq, 2, D, c.max_len if page else c.W_in), scale=0.3,
                  dev_status=torch.zeros(1, **i32), **{cache: c.kv.cuda()}, **where)
    if page:
        attend["max_len"] = c.max_len
    x = n(B, T, V)
    logits = dict(logits=x, out=torch.zeros_like(x), s=torch.randint(0, V, (B, 40), generator=g, **i32), width=37,
                  draft=torch.randint(0, V, (B, T - 1), generator=g, **i32), begin=torch.tensor([3, 0, 37], **i32), lens=None,
                  prompt=torch.tensor([2, 50, 0], **i32), repetition=1 + n(B).abs(), presence=n(B), frequency=n(B),
                  bias_ids=torch.randint(0, V, (B, 6), generator=g, **i32), bias=n(B, 6),
                  mask=torch.randint(-2 ** 31, 2 ** 31 - 1, (B, T, 17), generator=g, **i32), dev_status=torch.zeros(1, **i32))
    end = "paged" if page else "window"
    return {"append": (getattr(sd, f"specdec_append_{end}"), append, (cache, "q_out", "dev_status")),
            "attend": (getattr(sd, f"specdec_attend_{end}"), attend, ("out", "dev_status")),
            "logits": (sd.specdec_process_logits, logits, ("out", "dev_status"))}


VARIANTS = {"append": [{}, dict(inv_freq=None), dict(q_norm=None), dict(k_norm=None, dev_status=None), dict(eps=0)],
            "attend": [{}, dict(scale=None), dict(scale=1), dict(dev_status=None)],
            "logits": [{}, dict(mask=None), dict(bias_ids=None, bias=None), dict(begin=None, lens=torch.tensor([5, 39, 0], dtype=torch.int32)),
                       dict(repetition=None, presence=None, frequency=None, s=None, draft=None, begin=None)]}


@pytest.mark.parametrize("page", [0, 8])
def test_native_and_python_marshalling_agree(sd, monkeypatch, page):
    native = sd._native
    for name, variants in VARIANTS.items():
        for change in variants:
            got = []
            for route in (native, None):
                monkeypatch.setattr(sd, "_native", route)
                f, args, written = _calls(sd, page)[name]
                args = {**args, **{k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in change.items()}}
                f(**args)
                torch.cuda.synchronize()
                got.append([args[w] for w in written if args[w] is not None])
            for a, b in zip(*got):
                a, b = (t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32) for t in (a, b))
                assert torch.equal(a, b), (name, change)


@pytest.mark.parametrize("page", [0, 8])
def test_refused_arguments_raise_alike(sd, monkeypatch, page):
    native = sd._native
    calls = _calls(sd, page)
    index = "lens" if page else "pad_in"
    wrong = {"append": [dict(qkv=calls["append"][1]["qkv"].double()), dict(qkv=calls["append"][1]["qkv"][..., ::2]), dict(layer=7),
                        dict(layer=1.5), dict(q_out=None), dict(q_norm=torch.ones(4, device="cuda")), dict(eps=-1.0),
                        dict(inv_freq=torch.ones(40, device="cuda")), {index: calls["append"][1][index][:2]},
                        {index: calls["append"][1][index].long()}, dict(dev_status=torch.zeros(1))],
             "attend": [dict(q=calls["attend"][1]["q"].float()), dict(out=calls["attend"][1]["out"][:2]), dict(scale=float("inf")),
                        dict(workspace=torch.empty(1, dtype=torch.int64, device="cuda")), {index: None}, dict(layer=-1),
                        dict(out=calls["attend"][1]["q"])],
             "logits": [dict(out=calls["logits"][1]["out"][:, :2]), dict(width=40), dict(width=-1), dict(bias=None), dict(s=None),
                        dict(mask=calls["logits"][1]["mask"][..., :15].contiguous()), dict(draft=None), dict(prompt=calls["logits"][1]["prompt"].cpu()),
                        dict(repetition=calls["logits"][1]["repetition"].double()), dict(lens=3)]}
    for name, changes in wrong.items():
        f, args, _ = calls[name]
        for change in changes:
            said = []
            for route in (native, None):
                monkeypatch.setattr(sd, "_native", route)
                with pytest.raises(Exception) as e:
                    f(**{**args, **change})
                said.append((e.type, str(e.value)))
            assert said[0] == said[1], (name, change)
    torch.cuda.synchronize()


@pytest.mark.parametrize("page", [0, 8])
def test_workspace_views_with_gaps_or_repeats_are_refused(sd, monkeypatch, page):
    """Their elements count more or other bytes than are theirs to write."""
    native = sd._native
    f, args, _ = _calls(sd, page)["attend"]
    ws = args["workspace"]
    for view in (ws[:1].expand(ws.numel()), torch.empty((ws.numel(), 2), dtype=ws.dtype, device="cuda")[:, 0]):
        for route in (native, None):
            monkeypatch.setattr(sd, "_native", route)
            with pytest.raises(ValueError, match="contiguous"):
                f(**{**args, "workspace": view})
    torch.cuda.synchronize()
