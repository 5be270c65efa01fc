"""The forward-side calls in every compiled form: head sizes, tiles of queries,
layouts and units that serving sizes run, and which entries an attention takes,
counted exactly."""
import numpy as np
import pytest
import torch

from tests import forward_ref as ref
from tests import test_gpu_append as append
from tests import test_gpu_attend as attend
from tests import test_gpu_logits as logits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2510_22876_amd import specdec
    yield specdec
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


# ---- attention: head sizes by tiles of 16 queries by layouts, whole and cut ------------------------------------------

@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("queries", [(5, 3), (6, 4), (6, 7)])   # window, query heads a KV head: 15, 24 and 42 rows
@pytest.mark.parametrize("D", [16, 56, 64, 80, 96, 128, 136, 200, 256])
def test_attention_forms(sd, D, queries, page, cut):
    T, G = queries
    n = [1500, 0, 700] if cut else [300, 0, 33, 95]
    c = ref.Cache(n, T, 2, D, page)
    c.fill(T, torch.Generator().manual_seed(1))
    q = attend._queries(c, 2 * G, 2, 2.0)
    out, status = attend._run(sd, c, q)
    assert status == 0
    attend._check(c, q, out)


# ---- which entries are taken --------------------------------------------------------------------------------------

def _marked(c):
    """Values that mark their entry's tile of 32: element (j / 32) % D is 1, the others 0; keys are random."""
    c.fill(c.T, torch.Generator().manual_seed(1))
    for i, n in enumerate(c.n):
        j = np.arange(n + c.T)
        rows, cols = zip(*(c.where(i, int(x)) for x in j))
        v = torch.zeros((n + c.T, c.H, c.D), dtype=torch.bfloat16)
        v[torch.as_tensor(j), :, torch.as_tensor(j // 32 % c.D)] = 1.0
        c.kv[c.layer, 1][torch.tensor(rows), :, torch.tensor(cols)] = v
    return c


def _shares(c, i):
    """[T][D]: what share of a query's entries each element marks."""
    n, out = c.n[i], torch.zeros((c.T, c.D), dtype=torch.float64)
    for r in range(c.T):
        m = n + r + 1
        out[r] = torch.as_tensor(np.bincount(np.arange(m) // 32 % c.D, minlength=c.D)).double() / m
    return out


@pytest.mark.parametrize("page", [0, 16, 24])
@pytest.mark.parametrize("name", ["long_one", "equal", "unequal", "unequal_groups", "few_unequal", "boundaries", "wide_heads"])
def test_every_entry_is_taken_once(sd, name, page):
    """With a scale of 0 every weight is exactly 1 and the sums are whole numbers, so that an entry left out or taken twice
    at the edge of a tile, a wave or a piece changes an element by more than its bound.  An element counts at most 64
    entries, so that one more or less is 1/64 of it; the result's reciprocal and product round by 2^-23 together, its
    rounding to bf16 by at most 2^-8."""
    n, T, H, G, D = {
        "long_one": ([4000], 1, 2, 1, 64), "equal": ([3000 - 31 * i for i in range(6)], 5, 2, 7, 64),
        "unequal": ([4000, 3, 1000, 0, 2049, 511, 65], 8, 2, 4, 64), "unequal_groups": ([2500, 100, 1200], 33, 1, 4, 64),
        "few_unequal": ([200, 4060, 1521], 1, 1, 4, 64), "boundaries": ([128 * a + b for a in (5, 8) for b in range(-2, 2)], 2, 1, 1, 64),
        "wide_heads": ([3500, 900, 1], 6, 1, 6, 256)}[name]
    c = _marked(ref.Cache(n, T, H, D, page))
    q = attend._queries(c, H * G, 2, 2.0)
    out, status = attend._run(sd, c, q, scale=0.0)
    assert status == 0
    for i in range(len(n)):
        want = _shares(c, i)
        assert float((want * torch.arange(n[i] + 1, n[i] + T + 1)[:, None]).max()) <= 64.001
        bound = want * (2.0 ** -8 + 2.0 ** -22)
        ref.check(out[i], want[:, None].expand(-1, H * G, -1), bound[:, None].expand(-1, H * G, -1), f"row {i} of {n[i]} entries")


# ---- logits: two units of 8 a lane, taken where the batch and the vocabulary are large ------------------------------

@pytest.mark.parametrize("dtype", logits.DT)
@pytest.mark.parametrize("what", ["everything", "penalties", "mask", "bias"])
def test_logits_of_large_batches(sd, dtype, what):
    B, V = 66, 32771                                      # 66 times 9 chunks of 4096
    r = np.random.default_rng(1)
    n = [int(x) for x in r.integers(0, 90, B)]
    n[3] = 2600                                           # beyond the tokens that are read ahead
    k = 2 if what == "everything" else 1
    c = logits._case(B, k, V, dtype, n, 2, penalties=what in ("everything", "penalties"), n_bias=30 if what in ("everything", "bias") else 0,
                     allow=0.9 if what in ("everything", "mask") else 0.0)
    c["draft"][:, 0] = c["s"][:, -5] % V                  # drafts in the history, and some among the last logits
    c["draft"][::2, -1] = V - 1 - r.integers(0, 12, len(c["draft"][::2]))
    off = {} if what in ("everything", "penalties") else dict(s=None, draft=None, begin=None, prompt=None)
    out, status = logits._run(sd, c, **off)
    assert status == 0
    logits._check(c, out)
    again, _ = logits._run(sd, c, in_place=True, **off)
    assert torch.equal(out.float().nan_to_num(7.0), again.float().nan_to_num(7.0)), "in place differs"


# ---- append: several heads a group of lanes, taken where there are many tokens --------------------------------------

@pytest.mark.parametrize("dtype", append.DT)
@pytest.mark.parametrize("form", [(24, 8, 128, 9, 64, True, False, 0), (24, 8, 128, 20, 32, True, True, 16), (12, 4, 256, 9, 128, False, False, 0),
                                  (21, 3, 256, 7, 96, True, False, 64), (40, 20, 96, 18, 48, True, True, 0), (120, 30, 24, 40, 5, False, False, 7)])
def test_append_of_many_tokens(sd, dtype, form):
    Hq, H, D, T, half, norm, adjacent, page = form
    B = 60
    tokens, groups = B * T, 256 // {24: 4, 96: 16, 128: 16, 256: 32}[D]
    assert -(-1024 // tokens) < -(-(Hq + 2 * H) // groups), "the heads are to outnumber the groups of lanes"
    c = ref.Cache([int(x) for x in np.random.default_rng(2).integers(0, 50, B)], T, H, D, page)
    c.fill(0, torch.Generator().manual_seed(1))
    x, w, f = append._inputs(c, Hq, append.DT[dtype], half, norm, 3)
    q, kv, status = append._run(sd, c, x, w, f, adjacent)
    assert status == 0
    append._check(c, x, w, f, adjacent, q, kv)
