"""sdvg_rope_positions and sdvg_paged_commit against the definition in 64 bits.

Tolerances, per element: one rounding to the result's type, eps / 2 of the value (e4m3: below 2^-6 half of its 2^-9 step), and
for a rotated element 8 roundings to 32 bits of |a| + |b| (the angle's distance to a quarter turn, sine or cosine to 2
units, gain, product, fma: 6 at most)."""
import numpy as np
import pytest
import torch

from paged_util import i32

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0**-8, "f16": 2.0**-11, "f32": 2.0**-24, "e4m3": 2.0**-4}


def rotated(x, positions, freqs, rot, layout, gain):
    """(x rotated, |a| + |b| of every rotated element) in 64 bits."""
    x = x.double().cpu().numpy()
    # positions and frequencies are exact in 64 bits; their product is reduced there
    ang = positions.cpu().numpy().astype(np.float64)[:, None, None] * freqs.cpu().numpy()
    c, s = np.float32(gain) * np.cos(ang), np.float32(gain) * np.sin(ang)
    i, j = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    y, size = x.copy(), np.zeros_like(x)
    a, b = x[..., i], x[..., j]
    y[..., i], y[..., j] = a * c - b * s, a * s + b * c
    size[..., i] = size[..., j] = (np.abs(a) + np.abs(b)) * gain
    return y, size


# Below its smallest normal number, 2^-14 (f16) or 2^-6 (e4m3), a type's steps are 2^-24 or 2^-9 whatever the value, so half
# a step is 2^-25 or 2^-10 and no share of the value bounds it. (bf16 and f32: 2^-134 and 2^-150, below everything here.)
SMALLEST = {"bf16": 0.0, "f16": 2.0**-25, "f32": 0.0, "e4m3": 2.0**-10}


def assert_close(got, want, size, kind):
    got = got.float().cpu().numpy().astype(np.float64)
    tol = HALF_STEP[kind] * np.abs(want) + 8 * 2.0**-24 * size + SMALLEST[kind]
    excess = float(np.max(np.abs(got - want) - tol))
    assert excess <= 0, excess


def normal(shape, dtype, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def strided(t, how):
    """The same rows as a slice of a wider tensor, or head-major."""
    if how == "wide":
        w = torch.full((t.shape[0], t.shape[1] + 3, 128), 7.0, dtype=t.dtype, device="cuda")
        w[:, 2:-1] = t
        return w[:, 2:-1]
    if how == "head":
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    return t


@pytest.mark.parametrize("n,H,Hy", [(1, 1, 0), (1, 40, 8), (3, 5, 1), (257, 12, 12), (1031, 3, 2), (4099, 1, 0), (1026, 40, 70)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot,kind,how", [(128, "bf16", "plain"), (16, "bf16", "wide"), (48, "f16", "head"), (96, "f32", "wide"),
                                          (112, "f32", "plain")])
def test_rope_positions(n, H, Hy, layout, rot, kind, how):
    import paper_2604_17397_amd as P
    x, y = normal((n, H, 128), DT[kind], n + rot), normal((n, max(Hy, 1), 128), DT[kind], n + rot + 1)
    rng = np.random.default_rng(n + H)
    positions = i32(rng.integers(-(1 << 20), 1 << 20, n))
    positions[0] = 0 if n % 2 else 2**31 - 1
    freqs, gain = P.rope_frequencies(rot, theta=5e5, scaling="yarn", factor=4.0, original=8192)
    xs, ys = strided(x, how), strided(y, how)
    got = P.rope_positions(xs, positions, freqs, y=ys if Hy else None, layout=layout, gain=gain)
    in_place = strided(x.clone(), how)
    P.rope_positions(in_place, positions, freqs, layout=layout, gain=gain, out=in_place)
    torch.cuda.synchronize()
    for src, out in ((x, got[0]), (y, got[1])) if Hy else ((x, got),):
        assert_close(out, *rotated(src, positions, freqs, rot, layout, gain), kind)
        assert torch.equal(out[..., rot:], src[..., rot:])
    assert torch.equal(in_place, got[0] if Hy else got)
    if how == "wide":   # what lies around the slice is left alone
        w = in_place._base
        assert (w[:, :2] == 7).all() and (w[:, -1] == 7).all()


def test_rope_no_token_and_equivalent_layouts():
    import paper_2604_17397_amd as P
    freqs, _ = P.rope_frequencies(64)
    x = normal((0, 3, 128), torch.bfloat16, 1)
    assert P.rope_positions(x, i32([]), freqs).shape == (0, 3, 128)
    x = normal((70, 3, 128), torch.float32, 2)
    pos = i32(np.arange(70) * 31)
    # interleaved is half with the elements dealt out anew
    deal = torch.arange(64, device="cuda").view(32, 2).t().flatten()
    a = P.rope_positions(x, pos, freqs, layout="interleaved")
    z = x.clone()
    z[..., :64] = x[..., deal]
    b = P.rope_positions(z, pos, freqs, layout="half")
    torch.cuda.synchronize()
    assert torch.equal(a[..., deal], b[..., :64]) and torch.equal(a[..., 64:], b[..., 64:])


def test_rope_positions_and_the_pass_with_tables_agree():
    """The same angles through tables (sdvg_rope): at most one step of bf16 apart."""
    import paper_2604_17397_amd as P
    x = normal((300, 7, 128), torch.bfloat16, 3)
    pos = i32(np.arange(300) * 11)
    freqs, _ = P.rope_frequencies(128)
    ang = pos.double()[:, None] * freqs
    a = P.rope(x, torch.cos(ang).float(), torch.sin(ang).float()).float()
    b = P.rope_positions(x, pos, freqs, layout="interleaved").float()
    torch.cuda.synchronize()
    assert ((a - b).abs() <= 2.0**-7 * a.abs() + 2.0**-20).all() and (a != b).float().mean() < 1e-3


@pytest.mark.parametrize("n,H,Hq,P_", [(1, 1, 1, 8), (1, 8, 40, 16), (70, 3, 9, 24), (1030, 2, 4, 64), (1025, 20, 33, 16)])
@pytest.mark.parametrize("kind,cache,rot,layout", [("bf16", "bf16", 128, "half"), ("f16", "f16", 64, "interleaved"),
                                                   ("bf16", "e4m3", 96, "half"), ("f16", "e4m3", 0, "half"), ("bf16", "bf16", 0, "half")])
@pytest.mark.parametrize("pool", ["token", "head", "padded"])
def test_paged_commit(n, H, Hq, P_, kind, cache, rot, layout, pool):
    import paper_2604_17397_amd as S
    t, ct = DT[kind], torch.float8_e4m3fn if cache == "e4m3" else DT[kind]
    pages = -(-n // P_) + 2
    shape = {"token": (pages, P_, H, 128), "head": (H, pages, P_, 128), "padded": (pages, P_ + 1, H, 160)}[pool]

    def storage():
        s = torch.full(shape, 3.5, device="cuda").to(ct)
        return s, (s if pool == "token" else s.permute(1, 2, 0, 3) if pool == "head" else s[:, :P_, :, :128])
    (ks, kc), (vs, vc) = storage(), storage()
    rng = np.random.default_rng(n + P_)
    slots = torch.from_numpy(rng.permutation(pages * P_)[:n].copy()).cuda()
    if n > 3:
        slots[n // 2], slots[1], slots[n - 1] = -1, pages * P_, 2**40     # padded, and past the pools
    wide = normal((n, Hq + 2 * H, 128), t, n)
    q, k, v = wide.split([Hq, H, H], dim=1)
    if n > 8:
        k[5, 0, 1], v[6, 0, 3], v[7, 0, 2] = 1e4, -1e4, float("nan")     # past the largest number of 8 bits
    scale = [None, None]
    if cache == "e4m3":
        scale = [(0.01 + torch.rand(H, device="cuda") / 50) for _ in range(2)]
    c = S.PagedKV(kc, vc, *scale)
    kw, pos, freqs = {}, i32(rng.integers(0, 1 << 17, n)), None
    if rot:
        freqs, _ = S.rope_frequencies(rot, scaling="ntk", factor=2.0)
        kw = dict(positions=pos, freqs=freqs, q=q, layout=layout, gain=1.25)
    got = S.paged_commit(c, k, v, slots, **kw)
    torch.cuda.synchronize()
    ok = (slots >= 0) & (slots < pages * P_)
    at = slots[ok]
    want = {}
    for name, x, sc in (("k", k, scale[0]), ("v", v, scale[1])):
        y, size = rotated(x, pos, freqs, rot, layout, 1.25) if rot and name == "k" else (x.double().cpu().numpy(), np.zeros(tuple(x.shape)))
        if sc is not None:
            d = sc.double().cpu().numpy()[:, None]
            y, size = np.clip(y / d, -448, 448), size / d + np.abs(y / d)     # (the quotient is rounded too)
        want[name] = (y, size)
    for name, x, view, store in (("k", k, kc, ks), ("v", v, vc, vs)):
        y, size = (a[ok.cpu().numpy()] for a in want[name])
        rows = view[at // P_, at % P_].float().cpu().numpy().astype(np.float64) if cache != "e4m3" else \
            view.float()[at // P_, at % P_].cpu().numpy().astype(np.float64)
        bad = np.isnan(y)
        assert np.array_equal(np.isnan(rows), bad)
        if rot == 0 and cache != "e4m3" or name == "v" and cache != "e4m3":
            assert np.array_equal(rows[~bad], y[~bad])
        assert_close(torch.from_numpy(rows[~bad]), y[~bad], size[~bad], cache)
        # everything else in the storage is as it was
        view.view(torch.uint8)[at // P_, at % P_] = torch.full((), 3.5).to(ct).view(1).view(torch.uint8).cuda().repeat(128)
        assert (store.float() == 3.5).all()
    if rot:
        assert_close(got, *rotated(q, pos, freqs, rot, layout, 1.25), kind)
    else:
        assert got is None


def test_paged_commit_of_no_token_and_in_place_q():
    import paper_2604_17397_amd as S
    k = torch.zeros((2, 8, 3, 128), dtype=torch.bfloat16, device="cuda")
    c = S.PagedKV(k, torch.zeros_like(k))
    e = torch.empty((0, 3, 128), dtype=torch.bfloat16, device="cuda")
    S.paged_commit(c, e, e, torch.empty(0, dtype=torch.int64, device="cuda"))
    x, q = normal((5, 3, 128), torch.bfloat16, 8), normal((5, 6, 128), torch.bfloat16, 9)
    freqs, _ = S.rope_frequencies(128)
    pos, slots = i32([4, 0, 9, 2, 7]), torch.tensor([15, 3, 0, -1, 8], device="cuda")
    want = S.rope_positions(q, pos, freqs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert S.paged_commit(c, x, x, slots, positions=pos, freqs=freqs, q=q, q_out=q, stream=side) is q
    side.synchronize()
    assert torch.equal(q, want)
    assert torch.equal(c.v[1, 7], x[0]) and torch.equal(c.k[0, 0], S.rope_positions(x, pos, freqs)[2])
    assert (c.v[1, 1:7] == 0).all()
