"""specdec_append_window / specdec_append_paged against a 64-bit implementation:
types, head sizes, partial and adjacent rotation, pages that the window ends
inside, far positions, sequences that have to be left untouched."""
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


def _inputs(c, Hq, dtype, half, norm, seed):
    g = torch.Generator().manual_seed(seed)
    B, D = len(c.n), c.D
    x = torch.randn((B, c.T, Hq + 2 * c.H, D), generator=g).to(dtype)
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(dtype) if norm else None for _ in range(2)]
    f = (10000.0 ** (-torch.arange(half).double() / max(half, 1))).float() if half else None
    return x, w, f


def _run(sd, c, x, w, f, adjacent, eps=1e-5, **over):
    """The call on device copies; (q_out, cache) on the host."""
    dev = lambda t: None if t is None else t.cuda()   # noqa: E731
    Hq = x.shape[2] - 2 * c.H
    q = torch.full((x.shape[0], c.T, Hq, c.D), float("nan"), dtype=torch.bfloat16, device="cuda")
    kv, status = c.kv.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    rest = dict(inv_freq=dev(f), q_norm=dev(w[0]), k_norm=dev(w[1]), eps=eps, adjacent=adjacent, dev_status=status)
    if c.page:
        sd.specdec_append_paged(dev(x), kv, c.layer, over.get("table", c.table), over.get("lens", c.lens), q, **rest)
    else:
        sd.specdec_append_window(dev(x), kv, c.layer, c.W_in, over.get("pad", c.pad), q, **rest)
    torch.cuda.synchronize()
    return q.cpu(), kv.cpu(), int(status.cpu()[0])


def _check(c, x, w, f, adjacent, q, kv, eps=1e-5, skip=()):
    Hq = x.shape[2] - 2 * c.H
    want = c.kv.clone()
    for i, n in enumerate(c.n):
        if i in skip:
            assert bool(torch.isnan(q[i]).all()), f"row {i} was to be left untouched"
            continue
        y, v, b = ref.append(x[i], Hq, c.H, n, c.T, w[0], w[1], eps, f, adjacent)
        b = b + 2.0 ** -8 * y.abs() + 2.0 ** -133
        ref.check(q[i], y[:, :Hq], b[:, :Hq], f"queries of row {i}")
        for r in range(c.T):
            row, col = c.where(i, n + r)
            ref.check(kv[c.layer, 0, row, :, col], y[r, Hq:], b[r, Hq:], f"key {r} of row {i}")
            assert torch.equal(kv[c.layer, 1, row, :, col], v[r].to(torch.float32).to(torch.bfloat16)), f"value {r} of row {i}"
            want[c.layer, :, row, :, col] = kv[c.layer, :, row, :, col]
    assert torch.equal(kv.view(torch.int16), want.view(torch.int16)), "something else in the cache was written"


CASES = {   # (dtype, Hq, H, D, T, entries, page, rotated pairs, norm, adjacent)
    "one": ("bf16", 32, 8, 128, 1, [1000], 16, 64, True, False),
    "mha_f16": ("f16", 6, 6, 128, 6, [3, 0, 17], 0, 64, False, False),
    "tiny_f32": ("f32", 4, 2, 16, 5, [8, 40], 0, 8, True, False),
    "smallest_head": ("bf16", 3, 1, 8, 2, [0, 5], 0, 4, True, True),
    "d24_odd_pairs": ("f32", 5, 5, 24, 3, [2, 9], 1, 5, True, False),
    "d64_adjacent": ("f16", 24, 4, 64, 4, [30, 31, 32, 33], 32, 32, True, True),
    "d80_partial": ("bf16", 12, 12, 80, 7, [11, 64], 3, 20, False, False),
    "d96_no_turn": ("f32", 16, 2, 96, 2, [1, 2, 3], 100, 0, True, False),
    "d256": ("bf16", 8, 2, 256, 3, [250, 0], 24, 128, True, False),
    "d256_adjacent": ("f32", 2, 2, 256, 2, [7], 0, 128, True, True),
    "long_window": ("bf16", 28, 4, 128, 65, [0, 63, 64], 16, 32, True, True),
    "many_rows": ("f16", 4, 1, 128, 2, list(range(37)), 7, 64, True, False),
    "pool_slots": ("bf16", 4, 4, 64, 3, [5, 5], 40, 32, False, False),
}


@pytest.mark.parametrize("name", CASES)
def test_matches_64_bits(sd, name):
    dtype, Hq, H, D, T, n, page, half, norm, adjacent = CASES[name]
    c = ref.Cache(n, T, H, D, page, slots=name == "pool_slots")
    c.fill(0, torch.Generator().manual_seed(1))
    x, w, f = _inputs(c, Hq, DT[dtype], half, norm, 2)
    q, kv, status = _run(sd, c, x, w, f, adjacent)
    assert status == 0
    _check(c, x, w, f, adjacent, q, kv)


def test_far_positions(sd):
    """Positions up to 2^24 - 1 in the last page of a long sequence; the pages before it are never needed."""
    T, H, D, P = 4, 1, 16, 1 << 20
    c = ref.Cache([0], T, H, D, P, layers=1, layer=0, room=0)
    n = 16 * P - T
    c.n, c.table_np = [n], np.full((1, 16), -1, np.int32)
    c.table_np[0, 15] = 0
    c.table, c.lens = torch.as_tensor(c.table_np, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    x, w, f = _inputs(c, 2, torch.float32, 8, False, 3)
    q, kv, status = _run(sd, c, x, w, f, False)
    assert status == 0
    _check(c, x, w, f, False, q, kv)


def test_zero_rows_and_eps(sd):
    """A head of zeros stays zero with eps > 0, and is 0 / 0 with eps = 0."""
    c = ref.Cache([4], 1, 1, 16)
    c.fill(0, torch.Generator().manual_seed(1))
    x, w, f = _inputs(c, 2, torch.float32, 8, True, 4)
    x[0, 0, 0] = 0
    q, _, _ = _run(sd, c, x, w, f, False, eps=1e-6)
    assert bool((q[0, 0, 0] == 0).all()) and bool(torch.isfinite(q).all())
    q, _, _ = _run(sd, c, x, w, f, False, eps=0.0)
    assert bool(torch.isnan(q[0, 0, 0]).all()) and bool(torch.isfinite(q[0, 0, 1]).all())


@pytest.mark.parametrize("page", [0, 4])
def test_sequences_out_of_range_are_left_alone(sd, page):
    n, T = [5, 3, 0, 6, 2], 3
    c = ref.Cache(n, T, 2, 16, page, room=2)
    c.fill(0, torch.Generator().manual_seed(1))
    x, w, f = _inputs(c, 4, torch.bfloat16, 8, True, 5)
    if page:
        table, lens = c.table_np.copy(), np.asarray(n, np.int32)
        lens[0] = -1
        lens[1] = table.shape[1] * page - T + 1           # one entry beyond the table
        table[3, 2] = c.shape[2]                          # the window's last page: entry 8
        table[4, 0] = -7                                  # the page of entries 2 and 3
        q, kv, status = _run(sd, c, x, w, f, False, table=torch.as_tensor(table, device="cuda"),
                             lens=torch.as_tensor(lens, device="cuda"))
        assert status == sd.DEV_BAD_SLOT
        _check(c, x, w, f, False, q, kv, skip=(0, 1, 3, 4))
    else:
        pad = c.pad_np.copy()
        pad[0], pad[3] = -1, c.W_in - T + 1
        q, kv, status = _run(sd, c, x, w, f, False, pad=torch.as_tensor(pad, device="cuda"))
        assert status == sd.DEV_BAD_PAD_IN
        _check(c, x, w, f, False, q, kv, skip=(0, 3))


def test_split_over_launches(sd, monkeypatch):
    c = ref.Cache(list(range(9)), 3, 2, 32, 8)
    c.fill(0, torch.Generator().manual_seed(1))
    x, w, f = _inputs(c, 6, torch.bfloat16, 16, True, 6)
    whole = _run(sd, c, x, w, f, False)
    monkeypatch.setenv("SPECDEC_MAX_LAUNCH_ITEMS", str(256 * 5))
    parts = _run(sd, c, x, w, f, False)
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(whole[:2], parts[:2]))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("D, half, adjacent", [(16, 4, True), (16, 5, True), (16, 0, True), (16, 5, False), (16, 4, False), (24, 7, False),
                                               (128, 33, False), (256, 66, True)])
def test_unrotated_elements_stay_as_they_are(sd, dtype, D, half, adjacent):
    """Infinities, NaN and -0.0 beyond the rotated elements, of which a lane may hold both kinds, are copied and reach no
    other element."""
    c = ref.Cache([3, 70], 2, 2, D)
    c.fill(0, torch.Generator().manual_seed(1))
    x, w, f = _inputs(c, 4, DT[dtype], half, False, 7)
    odd = torch.tensor([float("inf"), float("-inf"), float("nan"), -0.0], dtype=DT[dtype])
    for h in range(6):                                    # queries and keys
        for j, d in enumerate(range(2 * half + h % 2, D, 2 if adjacent else 3)):
            x[:, :, h, d] = odd[(j + h) % 4]
    q, kv, status = _run(sd, c, x, w, f, adjacent)
    assert status == 0
    _check(c, x, w, f, adjacent, q, kv)
    plain = x.to(torch.float32).to(torch.bfloat16)
    same = lambda a, b: torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(   # noqa: E731
        a[~torch.isnan(a)].view(torch.int16), b[~torch.isnan(b)].view(torch.int16))
    assert same(q[..., 2 * half:], plain[:, :, :4, 2 * half:])
    for i, n in enumerate(c.n):
        for r in range(c.T):
            row, col = c.where(i, n + r)
            assert same(kv[c.layer, 0, row, :, col, 2 * half:], plain[i, r, 4:6, 2 * half:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-5])
def test_norms_of_tiny_and_huge_heads(sd, dtype, eps):
    """Squares that fp32 does not hold: their mean below its normal numbers, or beyond its largest."""
    c = ref.Cache([4, 9], 2, 2, 96)
    c.fill(0, torch.Generator().manual_seed(1))
    x, w, f = _inputs(c, 4, torch.float32, 16, True, 11)
    size = 2.0 ** torch.tensor([-120.0, -70.0, -64.0, 62.0, 100.0, 0.0])   # queries and keys; the last is ordinary
    x[:, :, :6] *= size[:, None]
    x, w = x.to(DT[dtype]), [t.to(DT[dtype]) for t in w]
    q, kv, status = _run(sd, c, x, w, f, False, eps=eps)
    assert status == 0
    _check(c, x, w, f, False, q, kv, eps=eps)
