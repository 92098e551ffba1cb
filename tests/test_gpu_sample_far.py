"""Drawing where |logit| / temperature is large: a weight depends on a logit's distance to the largest one alone, whatever both have in common.

Rows of two tokens with u, top_p or min_p 2^-34.5 to 2^-33.5 from the border between them. Weights are at most 2^-34 of themselves off, so a share
s = a / (a + b) at most s (1 - s) 2 x 2^-34 <= 2^-35, and every row has one right answer."""
import numpy as np
import pytest
import torch

from sample_util import draw
from test_gpu_sample import check

pytestmark = pytest.mark.gpu
# (largest logit, around which temperature; the other token is some steps of fp32 below)
PLACES = {"none in common": (3.0, 0.7), "100000 at 0.02": (1e5, 0.02), "1000000 at 0.1": (1e6, 0.1), "-1000000 at 0.3": (-1e6, 0.3), "30 at 1e-5": (30.0, 1e-5),
          "0.75 at 1e-7": (0.75, 1e-7), "3e30 at 1e24": (3e30, 1e24), "100 at 1e-5": (100.0, 1e-5), "-7000 at 0.002": (-7000.0, 0.002)}


def near_borders(top, around, of, n=48, seed=0):
    """n of (larger logit, smaller one, temperature, number): numbers that fp32 holds, near of(their difference / temperature), a number of [1/2, 1)."""
    rng = np.random.default_rng(seed)
    rows = []
    for _ in range(200):
        if len(rows) >= n:
            break
        t = (around * rng.uniform(0.7, 1.4, 20000)).astype(np.float32)
        a = np.float32(top) * (1 + rng.uniform(0, 1e-3, 20000)).astype(np.float32)
        b = (a.astype(np.float64) - t.astype(np.float64) * rng.uniform(0.05, 0.65, 20000)).astype(np.float32)
        d = (a.astype(np.float64) - b.astype(np.float64)) / t.astype(np.float64)
        border = of(d)
        off = np.abs(border * 2.0**24 - np.rint(border * 2.0**24))
        ok = (b < a) & (border > 0.5) & (border < 1 - 2.0**-20) & (off > 2.0**-10.5) & (off < 2.0**-9.5)
        rows += [(a[i], b[i], t[i], np.rint(border[i] * 2.0**24) / 2.0**24) for i in np.flatnonzero(ok)]
    assert len(rows) >= n
    return rows[:n]


def share(d):
    return 1 / (1 + np.exp(-d))


def logits(rows, first, second, vocab=20000):
    x = torch.full((len(rows), vocab), -np.inf)
    for r, (a, b, _, _) in enumerate(rows):
        x[r, first], x[r, second] = float(a), float(b)
    return x.cuda()


@pytest.mark.parametrize("place", list(PLACES))
@pytest.mark.parametrize("first,second", [(5, 9), (77, 19000), (8192, 8191), (19999, 0)])
@pytest.mark.parametrize("filters", [{}, dict(top_k=3), dict(min_p=1e-6), dict(top_k=2, top_p=0.9999999)])
def test_random_numbers_near_a_border(place, first, second, filters):
    rows = near_borders(*PLACES[place], share, seed=first)
    x = logits(rows, first, second)
    numbers = [s if first < second else 1 - s for _, _, _, s in rows]
    check(x, numbers, temperature=[float(t) for _, _, t, _ in rows], **filters)


@pytest.mark.parametrize("place", list(PLACES))
@pytest.mark.parametrize("first,second", [(5, 9), (77, 19000), (19999, 0)])
def test_top_p_near_a_border(place, first, second):
    rows = near_borders(*PLACES[place], share, seed=second + 1)
    x = logits(rows, first, second)
    for u in (0.0, 1 - 2.0**-24):
        check(x, [u] * len(rows), temperature=[float(t) for _, _, t, _ in rows], top_p=[float(s) for _, _, _, s in rows])


@pytest.mark.parametrize("place", list(PLACES))
@pytest.mark.parametrize("first,second", [(5, 9), (77, 19000), (19999, 0)])
@pytest.mark.parametrize("filters", [{}, dict(top_k=2), dict(top_p=0.9999999)])
def test_min_p_near_a_border(place, first, second, filters):
    rows = near_borders(*PLACES[place], lambda d: np.exp(-d), seed=second + 2)
    x = logits(rows, first, second)
    for u in (0.0, 1 - 2.0**-24):
        check(x, [u] * len(rows), temperature=[float(t) for _, _, t, _ in rows], min_p=[float(m) for _, _, _, m in rows], **filters)


@pytest.mark.parametrize("filters", [{}, dict(top_k=400), dict(top_p=0.8), dict(min_p=0.02), dict(top_k=900, top_p=0.95, min_p=0.001)])
@pytest.mark.parametrize("offset", [0.0, 2.0**17, -2.0**19, 2.0**21])
def test_a_common_offset_changes_nothing(offset, filters):
    """Logits in steps of 1/4, which fp32 holds with each of these offsets."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    x = (torch.randn((24, 30011), generator=gen, device="cuda") * 12).round() / 4
    u = torch.rand(24, generator=gen, device="cuda").tolist()
    got = check(x + offset, u, temperature=0.37, **filters)
    host = x.double().cpu().numpy()
    f = np.float32
    assert got.tolist() == [draw(host[r], float(f(u[r])), float(f(0.37)), filters.get("top_k", 0), float(f(filters.get("top_p", 1.0))),
                                 float(f(filters.get("min_p", 0.0))))[0] for r in range(24)]


@pytest.mark.parametrize("filters", [{}, dict(top_k=2), dict(top_p=0.5), dict(min_p=0.9), dict(top_k=3, top_p=0.9, min_p=1.0)])
@pytest.mark.parametrize("t", [1e-38, 1e-30, 1e-7, 3e-6, 1e-4])
def test_neighbours_where_nothing_else_weighs(t, filters):
    """The largest logit, some of its equals and its nearest neighbours below, up to places on the scale that 64 bits have no fraction for."""
    vocab = 17000
    for top in (1.0, -1.0, 65504.0, 3.4e38, -3.4e38, 2.0**-126, 0.0):
        a = np.float32(top)
        below = np.nextafter(a, np.float32(-np.inf))
        x = torch.full((4, vocab), float(below))
        for r in range(4):
            x[r, [100 + r, 9000, 16000 + r]] = float(a)
        check(x.cuda(), [0.0, 0.34, 0.66, 1 - 2.0**-24], temperature=t, **filters)
