"""Clipping of groups too large for the workgroups that run together, which are read twice: against torch in 64 bits, values
exactly as the products of the factors that came back, and the time of one group against that of the same values in several."""
import pytest
import torch

from paper_2011_06495_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GUARD = -12345.5
# fp32 values, 60 MB: more than the 57 that a launch's workgroups hold.  Once and twice as many in each of a call's groups, since
# the workgroups of small calls of this kind add up their group's sums themselves and those of larger ones are left the factor.
LARGE = 15_100_003


@pytest.fixture(autouse=True)
def say(request):
    print("[case] " + request.node.name, flush=True)


def norm64(tensors, kind):
    if not tensors:
        return 0.0
    if kind == B.MV_NORM_MAX:
        return max(float(t.double().abs().max()) for t in tensors)
    return sum(float(t.double().square().sum()) for t in tensors) ** 0.5


def check_norm(got, want, kind):
    # fp64 sums are off by less than 1e-9; then one rounding to fp32
    assert got == want if kind == B.MV_NORM_MAX else abs(got - want) <= want * (2.0 ** -24 + 1e-9), (got, want)


def factor(norm, max_norm):
    c = torch.tensor(max_norm, dtype=torch.float32) / (norm.cpu() + torch.tensor(1e-6, dtype=torch.float32))
    return torch.where(c >= 1.0, torch.ones_like(c), c)


def clip(tensors, out, groups, n_groups, kind, max_norm):
    """Norms and factors, and the norms of mv_clip_norms, which are the same."""
    guarded = [torch.full((n_groups + 1,), GUARD, device="cuda") for _ in range(3)]
    h = B.mv_clip_begin(tensors, out=out, groups=groups, n_groups=n_groups, norm=kind)
    B.mv_clip_norms(h, guarded[2])
    B.mv_clip_grads(h, max_norm, guarded[0], guarded[1])
    torch.cuda.synchronize()
    B.mv_clip_end(h)
    B.mv_clip_release(h)
    assert all(float(g[n_groups]) == GUARD for g in guarded)
    norms, coefs, only = (g[:n_groups] for g in guarded)
    assert torch.equal(norms, only)
    assert torch.equal(coefs.cpu(), factor(norms, max_norm))
    return norms, coefs


@pytest.mark.parametrize("kind", [B.MV_NORM_L2, B.MV_NORM_MAX])
@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("times", [1, 2])
def test_groups_of_all_sizes(times, src, dst, kind):
    """A group of one large tensor and odd small ones, a small group, an empty one and a second large one."""
    gen = torch.Generator(device="cuda").manual_seed(kind)
    large = times * (LARGE if src == "f32" else 2 * LARGE)
    sizes = [large, 5, 70_001, 1, 3, 0, large + 9]
    groups = [0, 0, 1, 1, 4, 0, 4]                    # groups 2 and 3 have no elements
    tensors = [torch.randn(n + 3, generator=gen, device="cuda")[i % 3:i % 3 + n].to(TYPES[src]) for i, n in enumerate(sizes)]
    rows = torch.full((sum(sizes) + 3 * len(sizes),), GUARD, dtype=TYPES[dst], device="cuda")
    places, at = [], 0
    for n in sizes:                                   # any alignment, a guarded value between them
        places.append(rows[at + 1:at + 1 + n])
        at += n + 3
    before = [t.clone() for t in tensors]
    want = [norm64([t for t, g in zip(tensors, groups) if g == k and t.numel()], kind) for k in range(5)]
    max_norm = 0.75 * want[0]
    norms, coefs = clip(tensors, places, groups, 5, kind, max_norm)
    for k in range(5):
        check_norm(float(norms[k]), want[k], kind)
    assert float(coefs[0]) < 1.0 and float(coefs[2]) == 1.0 and float(coefs[3]) == 1.0
    for t, b, o, g in zip(tensors, before, places, groups):
        assert torch.equal(t, b)
        assert torch.equal(o, (b.float() * coefs[g]).to(TYPES[dst]))
    at = 0
    for n in sizes:
        for edge in (at, at + 1 + n, at + 2 + n):
            assert float(rows[edge]) == float(torch.tensor(GUARD, dtype=TYPES[dst]))
        at += n + 3


@pytest.mark.parametrize("times", [1, 2])
def test_types_mixed(times):
    gen = torch.Generator(device="cuda").manual_seed(5)
    kinds = [("f32", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16")]
    tensors = [torch.randn(times * LARGE // 3 + 7 * i, generator=gen, device="cuda").to(TYPES[s]) for i, (s, _) in enumerate(kinds)]
    out = [torch.zeros(t.numel(), dtype=TYPES[d], device="cuda") for t, (_, d) in zip(tensors, kinds)]
    want = norm64(tensors, B.MV_NORM_L2)
    norms, coefs = clip(tensors, out, [0] * 4, 1, B.MV_NORM_L2, 0.3 * want)
    check_norm(float(norms[0]), want, B.MV_NORM_L2)
    for t, o in zip(tensors, out):
        assert torch.equal(o, (t.float() * coefs[0]).to(o.dtype))


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("times", [1, 2])
def test_in_place(times, src):
    """One group's values are clipped where they are, the other's, whose factor is 1, are not touched."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    n = times * (LARGE if src == "f32" else 2 * LARGE)
    tensors = [torch.randn(n, generator=gen, device="cuda").to(TYPES[src]) * s for s in (1.0, 0.25)]
    before = [t.clone() for t in tensors]
    norms, coefs = clip(tensors, tensors, [0, 1], 2, B.MV_NORM_L2, 0.5 * norm64(tensors[:1], B.MV_NORM_L2))
    assert float(coefs[0]) < 1.0 and float(coefs[1]) == 1.0
    for t, b, c in zip(tensors, before, coefs):
        assert torch.equal(t, (b.float() * c).to(t.dtype))


@pytest.mark.parametrize("kind", [B.MV_NORM_L2, B.MV_NORM_MAX])
def test_nan_and_infinity_stay_in_their_group(kind):
    x = [torch.ones(LARGE, device="cuda") for _ in range(3)]
    x[0][LARGE - 1], x[2][17] = float("nan"), float("inf")
    out = [torch.full_like(t, 9.0) for t in x]
    h = B.mv_clip_begin(x, out=out, groups=[0, 1, 2], norm=kind)
    norms, coefs = torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda")
    B.mv_clip_grads(h, 0.5, norms, coefs)
    torch.cuda.synchronize()
    B.mv_clip_end(h)
    B.mv_clip_release(h)
    assert bool(torch.isnan(norms[0])) and bool(torch.isnan(coefs[0])) and bool(torch.isnan(out[0]).all())
    assert bool(torch.isposinf(norms[2])) and float(coefs[2]) == 0.0 and bool(torch.isnan(out[2][17]))
    assert int((out[2] != 0.0).sum()) == 1
    assert bool((out[1] == coefs[1]).all()) and 0.0 < float(coefs[1]) < 1.0


def test_one_large_group_takes_as_long_as_its_values_in_several():
    """2^30 bf16 values as one group and as sixteen, each of which is read twice too: 6 bytes of memory a value either way,
    beside which the sums of its chunks, 16 bytes for each 32 KB, are nothing.  Half as much again is allowed for."""
    n = 1 << 30
    x = torch.randn(n // 16, device="cuda").bfloat16().repeat(16)
    out = torch.empty_like(x)
    least = {}
    for many in (1, 16):
        h = B.mv_clip_begin(list(x.split(n // many)), out=list(out.split(n // many)), groups=range(many))
        norms = torch.zeros(many, device="cuda")
        times = []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            B.mv_clip_grads(h, 1.0, norms)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        least[many] = min(times[1:])
        B.mv_clip_end(h)
        B.mv_clip_release(h)
    print(least, flush=True)
    assert least[1] <= 1.5 * least[16], least
