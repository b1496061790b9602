"""Arguments that the layer norm's and the distillation's calls refuse, all before any device call: the addresses here are made
up."""
import os

import pytest

from paper_2011_06495_amd import binding as B
from paper_2011_06495_amd import build as mv_build

P = 1 << 20            # an address with every alignment


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        mv_build.build_lib()
    return B.load()


def test_sizes(lib):
    for f in (B.mv_layernorm_scratch_bytes, B.mv_distill_scratch_bytes):
        assert f(0, 1) == 0 and f(1, 1 << 31) == 0 and f(-1, 5) == 0
    assert B.mv_layernorm_scratch_bytes(1, 1) > 0
    # neither cut into ranges nor too long to be held
    assert B.mv_distill_scratch_bytes(5000, 65_536) == 0 and B.mv_distill_scratch_bytes(1, 16_384) == 0
    assert B.mv_distill_scratch_bytes(1, 16_385) > 0 and B.mv_distill_scratch_bytes(5000, 70_000) > 0


# every call with good arguments by name, in the order of the C declaration
LISTED = dict(logits=P, dtype=0, ld_z=100, rows=4, n=100, idx=2 * P, ld_idx=5, t=3 * P, t_dtype=0, ld_t=5, top=5, labels=4 * P,
              temperature=2.0, soft=0.5, hard=0.5)
CALLS = {
    "mv_layernorm_forward": dict(x=P, x_dtype=0, ld_x=100, rows=4, n=100, gamma=2 * P, beta=3 * P, weight_dtype=0, eps=1e-5, y=4 * P,
                                 y_dtype=0, ld_y=100, mean=5 * P, rstd=6 * P, stream=None),
    "mv_layernorm_backward": dict(x=P, ld_x=100, dy=2 * P, ld_dy=100, dtype=0, rows=4, n=100, gamma=3 * P, weight_dtype=0, mean=4 * P,
                                  rstd=5 * P, dx=6 * P, dx_dtype=0, ld_dx=100, dgamma=7 * P, dbeta=8 * P, scratch=9 * P,
                                  scratch_bytes=1 << 20, stream=None),
    "mv_distill_loss": dict(LISTED, loss=5 * P, stats=6 * P, grad=7 * P, dz=8 * P, dz_dtype=0, ld_dz=100, scratch=9 * P,
                            scratch_bytes=1 << 20, stream=None),
    "mv_distill_grad": dict(LISTED, stats=6 * P, grad=7 * P, dz=8 * P, dz_dtype=0, ld_dz=100, stream=None),
}
NEEDED = {"mv_layernorm_forward": ("x", "y"), "mv_layernorm_backward": ("x", "dy", "mean", "rstd", "scratch"),
          "mv_distill_loss": ("logits", "idx", "t"), "mv_distill_grad": ("logits", "idx", "t", "stats", "dz")}
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("name", sorted(CALLS))
def test_arguments(lib, name):
    good, call = CALLS[name], getattr(lib, name)

    def status(**change):
        return call(*{**good, **change}.values())

    bad = [{p: 0} for p in NEEDED[name]]
    bad += [{p: v + (8 if p == "scratch" else 2)} for p, v in good.items() if isinstance(v, int) and v >= P and v % P == 0 and p != "scratch_bytes"
            and (p != "scratch" or name == "mv_layernorm_backward")]
    for size in ("rows", "n"):
        bad += [{size: 0}, {size: -1}, {size: 1 << 31}]
    for key in good:
        if key.startswith("ld_"):
            bad += [{key: 0}, {key: good[key] - 1}]
        if key.endswith("dtype"):
            bad += [{key: 2}, {key: -1}]
    if name == "mv_layernorm_forward":
        bad += [{"eps": -1e-9}, {"eps": INF}, {"eps": NAN}, {"y": P, "ld_y": 104}, {"y": P, "y_dtype": 1}]
    if name == "mv_layernorm_backward":
        bad += [{"scratch_bytes": 64}, {"dx": 0, "dgamma": 0, "dbeta": 0}, {"dx": P, "ld_dx": 104}, {"dx": 2 * P, "dx_dtype": 1}]
    if name.startswith("mv_distill"):
        bad += [{"top": -1}, {"top": 4097, "ld_idx": 5000, "ld_t": 5000}, {"temperature": 0.0}, {"temperature": -1.0}, {"temperature": NAN},
                {"temperature": INF}, {"temperature": 1e-30}, {"temperature": 1e30}, {"soft": INF}, {"soft": NAN}, {"hard": -INF},
                {"dz": P, "ld_dz": 104}, {"dz": P, "dz_dtype": 1}]
    if name == "mv_distill_loss":
        long = dict(n=70_000, ld_z=70_000, ld_dz=70_000)
        bad += [{"loss": 0, "dz": 0}, {**long, "scratch": 0}, {**long, "scratch": 9 * P + 8}, {**long, "scratch_bytes": 64}]
    for change in bad:
        assert status(**change) == B.MV_ERR_INVALID_ARG, change
