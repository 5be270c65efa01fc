"""specdec_process_logits against a 64-bit implementation: types, vocabularies
of any size, histories with repeats, drafts, prompts, repeated biases, masks
that leave a row empty, in place and out of place."""
import numpy as np
import pytest
import torch

from tests import forward_ref as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def sd():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2510_22876_amd import specdec
    yield specdec
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _case(B, k, V, dtype, n, seed, penalties=True, n_bias=0, allow=0.0, unpadded=False):
    """Inputs on the host; tokens cluster on a few values, some lie outside the vocabulary."""
    r = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    width = max(n)
    c = dict(B=B, k=k, V=V, n=n, logits=(3 * torch.randn((B, k + 1, V), generator=g)).to(DT[dtype]), width=width)
    s = (V * r.random((B, width + 4)) ** 4).astype(np.int32)
    s[r.random(s.shape) < 0.05] = -1
    s[r.random(s.shape) < 0.02] = V
    c["s"], c["draft"] = s, (V * r.random((B, k)) ** 4).astype(np.int32)
    c["begin"] = None if unpadded else np.asarray([width - x for x in n], np.int32)
    c["lens"] = np.asarray(n, np.int32) if unpadded else None
    c["prompt"] = np.asarray([x // 2 for x in n], np.int32)
    c["pen"] = [a.astype(np.float32) for a in (1 + r.random(B), r.normal(size=B), r.random(B))] if penalties else [None] * 3
    c["bias_ids"] = c["bias"] = c["mask"] = None
    if n_bias:
        c["bias_ids"] = r.integers(-1, min(V, 3 * n_bias) + 1, size=(B, n_bias)).astype(np.int32)   # repeats, and ids outside
        c["bias"] = r.normal(size=(B, n_bias)).astype(np.float32)
    if allow:
        c["mask"] = r.random((B, k + 1, V)) < allow
    return c


def _words(mask, more=0):
    """bool [..][V] -> int32 words, the unused bits set."""
    V = mask.shape[-1]
    pad = np.ones(mask.shape[:-1] + (-V % 32 + 32 * more,), bool)
    bits = np.concatenate([mask, pad], -1)
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int32)


def _run(sd, c, in_place=False, native=True, **over):
    dev = lambda a: None if a is None else torch.as_tensor(a, device="cuda")   # noqa: E731
    x = c["logits"].cuda()
    out = x if in_place else torch.full_like(x, 77.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    a = dict(s=dev(c["s"]), width=c["width"], draft=dev(c["draft"]), begin=dev(c["begin"]), lens=dev(c["lens"]),
             prompt=dev(c["prompt"]), repetition=dev(c["pen"][0]), presence=dev(c["pen"][1]), frequency=dev(c["pen"][2]),
             bias_ids=dev(c["bias_ids"]), bias=dev(c["bias"]), mask=None if c["mask"] is None else dev(_words(c["mask"])),
             dev_status=status)
    a.update(over)
    sd.specdec_process_logits(x, out, **a)
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(x.cpu().view(torch.int8), c["logits"].view(torch.int8)), "the input was written"
    return out.cpu(), int(status.cpu()[0])


def _check(c, out, skip=(), pen=None, prompt=True):
    for i in range(c["B"]):
        if i in skip:
            continue
        b = 0 if c["begin"] is None else int(c["begin"][i])
        e = c["width"] if c["lens"] is None else int(c["lens"][i])
        p = [None if a is None else float(a[i]) for a in (pen or c["pen"])]
        hist = c["s"][i, b:e + 1].tolist() if any(a is not None for a in p) else []
        drafts = c["draft"][i].tolist() if hist else []
        bias = [] if c["bias"] is None else [(int(t), float(v)) for t, v in zip(c["bias_ids"][i], c["bias"][i])]
        mask = None if c["mask"] is None else torch.as_tensor(c["mask"][i])
        want, bound = ref.logits(c["logits"][i], hist, drafts, int(c["prompt"][i]) if prompt else 0, *p, bias, mask,
                                 c["logits"].dtype)
        ref.check(out[i], want, bound, f"row {i}")


CASES = {   # (B, k, V, dtype, entries, biases, allowed share)
    "tiny": (2, 4, 1000, "f32", [8, 40], 5, 0.3),
    "one_token_vocabulary": (2, 2, 1, "f32", [3, 1], 1, 0.5),
    "v31": (3, 1, 31, "bf16", [0, 5, 9], 3, 0.5),
    "v33": (1, 3, 33, "f16", [20], 0, 0.9),
    "v4097": (2, 5, 4097, "bf16", [100, 700], 40, 0.5),
    "no_draft": (3, 0, 5003, "f16", [50, 0, 2000], 10, 0.0),
    "odd_rows": (2, 2, 20011, "f32", [33, 900], 0, 0.7),
    "wide": (1, 7, 50257, "bf16", [3000], 300, 0.05),
    "long_window": (1, 64, 3001, "f16", [100], 7, 0.5),
    "many_biases": (2, 1, 9000, "f32", [64, 64], 1024, 0.0),
    "aligned": (4, 4, 32768, "bf16", [10, 100, 1000, 4000], 64, 0.9),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("unpadded", [False, True])
def test_matches_64_bits(sd, name, unpadded):
    B, k, V, dtype, n, n_bias, allow = CASES[name]
    c = _case(B, k, V, dtype, n, 1, True, n_bias, allow, unpadded)
    out, status = _run(sd, c)
    assert status in (0, sd.DEV_EMPTY_MASK) and (status == 0 or not c["mask"].any(-1).all())
    _check(c, out)
    again, _ = _run(sd, c, in_place=True)
    assert torch.equal(out.float().nan_to_num(7.0), again.float().nan_to_num(7.0)), "in place differs"


@pytest.mark.parametrize("V", [5, 8, 21, 2051])
def test_many_drafts_a_unit(sd, V):
    """Drafts of a small vocabulary: several and repeated ones among eight neighbouring logits and among the last few, with
    prompts that end before, among and behind them."""
    c = _case(4, 64, V, "bf16", [7, 30, 1, 12], 6, n_bias=4)
    r = np.random.default_rng(8)
    c["draft"] = (V - 1 - r.integers(0, min(V, 20), size=(4, 64))).astype(np.int32)
    c["prompt"] = np.asarray([3, 40, 70, 200], np.int32)
    out, status = _run(sd, c)
    assert status == 0
    _check(c, out)
    again, _ = _run(sd, c, in_place=True)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)), "in place differs"


@pytest.mark.parametrize("which", range(3))
def test_each_penalty_alone(sd, which):
    c = _case(2, 3, 3000, "f32", [30, 400], 2)
    names = ("repetition", "presence", "frequency")
    out, _ = _run(sd, c, prompt=None, **{x: None for j, x in enumerate(names) if j != which})
    _check(c, out, pen=[a if j == which else None for j, a in enumerate(c["pen"])], prompt=False)


def test_mask_alone_and_nothing_at_all(sd):
    c = _case(3, 2, 7001, "bf16", [5, 6, 7], 3, penalties=False, allow=0.1)
    for in_place in (False, True):
        out, status = _run(sd, c, in_place, s=None, draft=None, begin=None, prompt=None)
        assert status == 0
        _check(c, out)
    c["mask"] = None
    out, _ = _run(sd, c, s=None, draft=None, begin=None, prompt=None)
    assert torch.equal(out.view(torch.int16), c["logits"].view(torch.int16))


def test_masks_that_allow_nothing(sd):
    """Flagged; bits of the last word beyond the vocabulary allow nothing either.  Words beyond the row's are not read."""
    c = _case(2, 2, 45, "f32", [5, 6], 4, allow=0.5)
    c["mask"][1, 1] = False
    c["mask"][..., 44] = True
    c["mask"][1, 1, 44] = False
    out, status = _run(sd, c)
    assert status == sd.DEV_EMPTY_MASK and bool(torch.isneginf(out[1, 1]).all())
    _check(c, out)
    out, status = _run(sd, c, mask=torch.as_tensor(_words(c["mask"], 3), device="cuda"))
    assert status == sd.DEV_EMPTY_MASK
    _check(c, out)
    c["mask"][1, 1, 44] = True
    assert _run(sd, c)[1] == 0


def test_special_values(sd):
    """Infinities, NaN and the types' largest values among the logits."""
    for dtype in DT:
        c = _case(1, 1, 600, dtype, [200], 5, n_bias=20, allow=0.9)
        x = c["logits"]
        top = torch.finfo(x.dtype).max
        for j, v in enumerate((float("inf"), float("-inf"), float("nan"), top, -top, 0.0, -0.0)):
            x[0, :, j * 3] = v
        c["pen"] = [np.asarray([a], np.float32) for a in (1.0, 0.5, 0.25)]   # no overflow past the largest value
        c["bias"] = -np.abs(c["bias"])
        x[0, :, 12] = -1.0                                                    # the lowest value less something
        out, _ = _run(sd, c)
        _check(c, out)


def test_rows_out_of_range_are_left_alone(sd):
    c = _case(5, 2, 2000, "f32", [40, 30, 20, 10, 5], 6)
    begin = c["begin"].copy()
    begin[1], begin[3] = -1, c["width"] + 1
    out, status = _run(sd, c, begin=torch.as_tensor(begin, device="cuda"))
    assert status == sd.DEV_BAD_PAD_IN and bool((out[[1, 3]] == 77).all())
    _check(c, out, skip=(1, 3))
    c = _case(4, 2, 2000, "f32", [40, 30, 20, 10], 6, unpadded=True)
    lens = c["lens"].copy()
    lens[0], lens[2] = c["s"].shape[1], -1
    out, status = _run(sd, c, lens=torch.as_tensor(lens, device="cuda"))
    assert status == sd.DEV_BAD_PAD_IN and bool((out[[0, 2]] == 77).all())
    _check(c, out, skip=(0, 2))


@pytest.mark.parametrize("prompt", [-5, 0, 31, 32, 33, 1 << 30])
def test_prompt_lengths(sd, prompt):
    """A prompt longer than the history reaches into the drafts; a negative one is none."""
    c = _case(1, 3, 100, "f32", [30], 7)
    c["prompt"] = np.asarray([prompt], np.int32)
    out, _ = _run(sd, c)
    _check(c, out)


def test_split_over_launches(sd, monkeypatch):
    c = _case(5, 2, 30000, "bf16", [40, 30, 20, 10, 5], 8, n_bias=9, allow=0.5)
    whole, _ = _run(sd, c)
    monkeypatch.setenv("SPECDEC_MAX_LAUNCH_ITEMS", str(256 * 3))
    parts, _ = _run(sd, c)
    assert torch.equal(whole.view(torch.int16), parts.view(torch.int16))


def test_offsets_past_32_bits(sd):
    """The last of 17 rows of 2^27 + 3 logits lies beyond 2^32 bytes, and 2^31 elements into the buffer."""
    V, B = (1 << 27) + 3, 17
    x = torch.zeros((B, 1, V), dtype=torch.bfloat16, device="cuda")
    s = torch.full((B, 3), V - 1, dtype=torch.int32, device="cuda")
    f = torch.full((B,), 2.0, device="cuda")
    sd.specdec_process_logits(x, x, s, 2, draft=torch.empty((B, 0), dtype=torch.int32, device="cuda"), frequency=f)
    torch.cuda.synchronize()
    assert bool((x[:, 0, V - 1] == -6).all()) and int((x != 0).sum()) == B


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("V", [21, 4096, 5001])
def test_untouched_logits_keep_their_bits(sd, dtype, V):
    """-0.0 among them: a drafted token's logit ahead of its draft, a prompt's under a penalty of answered tokens alone, and
    logits that only share a unit of eight with changed ones."""
    c = _case(1, 3, V, dtype, [40], 9, n_bias=2)
    c["s"][:] = 1
    c["s"][0, 5] = V - 2
    c["draft"] = np.asarray([[3, V - 1, 3]], np.int32)
    c["prompt"] = np.asarray([30], np.int32)
    c["bias_ids"] = np.asarray([[6, 6]], np.int32)
    c["pen"] = [None, c["pen"][1], c["pen"][2]]
    x = c["logits"]
    x[0, :, :10] = -0.0
    x[0, :, -4:] = -0.0
    changed = torch.zeros_like(x, dtype=torch.bool)
    changed[0, :, [1, 6]] = True                          # the history and the bias
    changed[0, 1:, 3] = True
    changed[0, 2:, V - 1] = True
    out, status = _run(sd, c)
    assert status == 0
    _check(c, out)
    whole = torch.int32 if dtype == "f32" else torch.int16
    assert torch.equal(out.view(whole)[~changed], x.view(whole)[~changed])
    assert not bool((out.view(whole)[changed] == x.view(whole)[changed]).any())
    again, _ = _run(sd, c, in_place=True)
    assert torch.equal(out.view(whole), again.view(whole)), "in place differs"
