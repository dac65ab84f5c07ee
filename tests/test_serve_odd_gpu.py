"""Scores and values that are no numbers, among tokens that a query sees, give the same whether its keys are one range or
many that are joined: NaN where the definition's products and sums have one, zeros where every score is -inf."""
import pytest
import torch

from paper_2609_34060_amd import kvc

pytestmark = pytest.mark.gpu
DEV = "cuda"
H, D, BS = 2, 128, 16
INF, NAN = float("inf"), float("nan")

# new tokens and contexts: one range; a few; more than sixteen (single tokens), and the same for rows of many new tokens
LENGTHS = [(1, 100), (1, 1000), (1, 5000), (40, 100), (40, 2000), (40, 5000)]


class Case:
    """Keys whose score is their first feature (queries have a one there and zeros elsewhere)."""

    def __init__(self, kind, new, ctx):
        self.kind, self.new, self.ctx = kind, new, ctx
        nb = -(-ctx // BS)
        g = torch.Generator().manual_seed(1)
        v = torch.randn(nb, BS, H, D, generator=g)
        k = torch.zeros(nb, BS, H, D)
        dt = {"bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8}[kind]
        if kind == "i8":
            v = torch.clamp(torch.round(40 * v), 1, 127)
            self.ks, self.vs = torch.ones(2, nb, BS, H, device=DEV)
        self.k, self.v = k.to(dt).to(DEV), v.to(dt).to(DEV)
        self.dt = torch.float32 if kind == "f32" else torch.bfloat16

    def key(self, t, score):
        """The score of keys t (a slice of the context)."""
        k = self.k.view(-1, H, D)[t]
        if self.kind != "i8":
            k[..., 0] = score
            return
        code = 1 if score != score else 0 if score == 0 else 100 if score > 0 else -1
        k[..., 0] = code
        self.ks.view(-1, H)[t] = score / code if code else 1.0

    def value(self, t, x):
        """Feature 5 of the values of t (in 8 bits every feature: the scale's)."""
        if self.kind == "i8":
            self.vs.view(-1, H)[t] = x
        else:
            self.v.view(-1, H, D)[t][..., 5] = x

    def run(self):
        if self.kind == "i8":
            cache = kvc.Cache([self.k], [self.v], k_scales=[self.ks], v_scales=[self.vs])
        else:
            cache = kvc.Cache([self.k], [self.v])
        q = torch.zeros(self.new, 2 * H, D, dtype=self.dt, device=DEV)
        q[..., 0] = 1
        lse = torch.empty(self.new, 2 * H, device=DEV)
        out = kvc.kvc_attend(cache, kvc.Step([self.new], [self.ctx], device=DEV), q, lse=lse, scale=1.0)
        return out, lse

    def features(self):
        f = torch.zeros(D, dtype=torch.bool, device=DEV)
        f[:] = self.kind == "i8"
        f[5] = True
        return f


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
@pytest.mark.parametrize("new,ctx", LENGTHS)
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_scores_of_minus_infinity_throughout(kind, new, ctx, bad):
    c = Case(kind, new, ctx)
    c.key(slice(0, ctx), -INF)
    c.value(slice(ctx // 3, ctx // 3 + 2), bad)
    out, lse = c.run()
    assert not torch.any(out) and torch.all(lse == -INF)


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
@pytest.mark.parametrize("new,ctx", LENGTHS)
@pytest.mark.parametrize("first", [True, False])
def test_scores_that_are_no_number_far_below_the_largest(kind, new, ctx, first):
    """A NaN score where all others are 200 below the row's largest (a weight of 2^-288)."""
    c = Case(kind, new, ctx)
    top, at = (ctx - new - 5, 10) if first else (10, ctx - new - 5)
    c.key(slice(top, top + 2), 200.0)
    c.key(slice(at, at + 1), NAN)
    out, lse = c.run()
    assert torch.all(out.isnan()) and torch.all(lse.isnan())


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
@pytest.mark.parametrize("new,ctx", LENGTHS)
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("bad", [INF, NAN])
def test_values_that_are_no_number_far_below_the_largest(kind, new, ctx, first, bad):
    c = Case(kind, new, ctx)
    top, at = (ctx - new - 5, 10) if first else (10, ctx - new - 5)
    c.key(slice(top, top + 2), 200.0)
    c.value(slice(at, at + 1), bad)
    out, lse = c.run()
    f = c.features()
    assert torch.all(out[..., f].isnan()) and torch.all(out[..., ~f].isfinite())
    assert torch.all((lse - 200.6931472).abs() < 1e-3)


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
@pytest.mark.parametrize("new,ctx", LENGTHS)
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("bad", [INF, NAN])
def test_values_that_are_no_number_among_scores_of_minus_infinity(kind, new, ctx, first, bad):
    """All but two scores are -inf: whole ranges have no weight, and their values show nevertheless."""
    c = Case(kind, new, ctx)
    top, at = (ctx - new - 5, 10) if first else (10, ctx - new - 5)
    c.key(slice(0, ctx), -INF)
    c.key(slice(top, top + 2), 0.0)
    c.value(slice(at, at + 1), bad)
    out, lse = c.run()
    f = c.features()
    assert torch.all(out[..., f].isnan()) and torch.all(out[..., ~f].isfinite())
    assert torch.all((lse - 0.6931472).abs() < 1e-3)
