"""Every row of the 4-bit precompute against 64 bits, with inputs that no rounding moves.

Where a value lies near a midpoint of codes, fp32 and 64 bits may choose different
ones, and what follows differs by far more than rounding.  Here nothing lies there:

* token rows are +1 and -1 in equal numbers (mean 0, variance 1) and positions 0, so
  that LayerNorm gives +-gain / sqrt(1 + 1e-5), which is +-gain in bf16; gains are
  magnitudes of 4-bit codes, which a block of any of them holds exactly;
* the queries are 0, so that attention is the mean of the values so far.  Rows of w_v
  are eight ones: values are multiples of 1/4 up to 51 (8 bits), a mean of two is exact in
  fp32, and one of three is such a multiple or at least a third of a small power of
  two away from any midpoint of bf16: fp32's rounding decides nothing;
* fc1's biases are +-64 and its sums less than 56 around them (12 of their standard
  deviations, and checked): GELU is the sum itself, or less than 1e-11;
* weights are code magnitudes times a power of two, so that sums are multiples of 2^-13
  below 2^11 and exact in fp32 in any order.

LayerNorm of anything else rounds differently in fp32, so the second one sees either the
token rows ("feed-forward": w_o is 0) or gains of 0 ("attention": its results are its
offsets, for every row the same), and so do both of a second layer.  What is left is
the final LayerNorm in fp32 and its rounding to bf16: of 512 values of fp32, with
roundings of 2^-24 in the mean, the variance, the root and the products, each of at
most 512 steps, 2^-24 * 2 * 512 = 6.1e-5 of values that are 23 (sqrt(512)) at most in
units of the row's deviation, times the gain, 1.5 at most, plus half a bf16 step: of 8
significant bits, neighbours in [1, 2) are 2^-7 apart, so that is 2^-8 of the value."""
import pytest
import torch

import paper_2502_01637_amd as S

pytestmark = pytest.mark.gpu

D, FF, K, V = 512, 640, 3, 44
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def codes(g, shape, scale):
    v = GRID[torch.randint(0, 8, shape, generator=g)]
    return v * (torch.randint(0, 2, shape, generator=g) * 2 - 1) * scale


def parameters(kind, n_layers):
    g = torch.Generator().manual_seed(len(kind) + n_layers)
    P = {"pos": torch.zeros(K, D)}
    for l in range(n_layers):
        ones = torch.zeros(D, D).scatter_(1, torch.rand(D, D, generator=g).argsort(1)[:, :8], 1.0)
        p = {"ln1_g": GRID[torch.randint(1, 8, (D,), generator=g)], "ln1_b": torch.zeros(D),
             "w_qkv": torch.cat([torch.zeros(D, D), codes(g, (D, D), 1 / 8), ones]),
             "b_qkv": torch.cat([torch.zeros(D), codes(g, (2 * D,), 0.5)]),
             "w_o": codes(g, (D, D), 2.0 ** -6), "b_o": codes(g, (D,), 0.25),
             "ln2_g": GRID[torch.randint(1, 8, (D,), generator=g)], "ln2_b": torch.zeros(D),
             "w_fc1": codes(g, (FF, D), 2.0 ** -5),
             "b_fc1": torch.where(torch.arange(FF) % 2 == 0, 64.0, -64.0),
             # where it is the same for every row it is kept small beside what differs
             "w_fc2": codes(g, (D, FF), 2.0 ** (-7 if kind == "feed-forward" else -11)),
             "b_fc2": codes(g, (D,), 0.25)}
        if l > 0:
            p["ln1_b"], p["ln1_g"] = p["ln1_g"], torch.zeros(D)
        if l > 0 or kind == "attention":
            p["ln2_b"], p["ln2_g"] = p["ln2_g"], torch.zeros(D)
        if l == 0 and kind == "feed-forward":
            p["w_o"], p["b_o"] = torch.zeros(D, D), torch.zeros(D)
        P.update({f"l{l}.{k}": v for k, v in p.items()})
    P["lnf_g"] = 0.5 + torch.rand(D, generator=g)
    P["lnf_b"] = torch.randn(D, generator=g)
    return {k: v.bfloat16() for k, v in P.items()}


def rounded(x):
    """What 4-bit rows of x hold, in 64 bits."""
    v = x.reshape(-1, 32)
    scale = torch.exp2((torch.frexp(v.abs().amax(1, keepdim=True))[1] - 3.0).clamp(min=-127.0))
    a = v.abs() / scale
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(a)
    return torch.copysign((torch.round(a / step) * step).clamp(max=6.0) * scale, v).view_as(x)


def norm(x, g, b):
    x = x - x.mean(-1, keepdim=True)
    return x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt() * g + b


def bf16(x):
    return x.float().bfloat16().double()


def forward(P, tok, fgrams, n_layers):
    """F of f-grams of one length [G, n], in 64 bits."""
    n = fgrams.shape[1]
    h = tok[fgrams] + P["pos"][:n]
    for l in range(n_layers):
        p = {k.split(".")[1]: v for k, v in P.items() if k.startswith(f"l{l}.")}
        w = {k: rounded(v) for k, v in p.items() if k.startswith("w_")}
        assert all(torch.equal(w[k], p[k]) for k in w)
        a = bf16(norm(h, p["ln1_g"], p["ln1_b"]))
        assert torch.equal(a, rounded(a))
        q, _, v = bf16(a @ w["w_qkv"].t() + p["b_qkv"]).split(D, -1)
        assert not q.any() and v.abs().max() <= 48 + 3
        # queries of 0: the mean of the values so far
        o = v.cumsum(1) / torch.arange(1, n + 1, device=v.device, dtype=torch.float64)[:, None]
        h = h + rounded(bf16(o)) @ w["w_o"].t() + p["b_o"]
        a = bf16(norm(h, p["ln2_g"], p["ln2_b"]))
        assert torch.equal(a, rounded(a))
        f = a @ w["w_fc1"].t() + p["b_fc1"]
        assert f.abs().min() >= 8
        h = h + rounded(bf16(f.clamp(min=0))) @ w["w_fc2"].t() + p["b_fc2"]
    return norm(h[:, -1], P["lnf_g"], P["lnf_b"])


@pytest.mark.parametrize("n_layers", [1, 2])
@pytest.mark.parametrize("kind", ["attention", "feed-forward"])
@pytest.mark.parametrize("N", [1, 5, 70, 1500, None])
def test_every_row(kind, n_layers, N):
    """All f-grams of two and three of 44 tokens (more states than a chunk holds, the
    last chunk ragged), or a few of them (the products' few-row and small-tile forms)."""
    P = parameters(kind, n_layers)
    g = torch.Generator().manual_seed(9)
    tok = torch.ones(V, D).scatter_(1, torch.rand(V, D, generator=g).argsort(1)[:, :D // 2], -1.0)
    every = torch.cartesian_prod(*[torch.arange(V)] * 3)
    fg = torch.cat([every, torch.cat([every[:V * V, 1:], torch.zeros(V * V, 1)], 1).long()])
    ln = torch.cat([torch.full((V ** 3,), 3), torch.full((V * V,), 2)])
    pick = torch.randperm(len(ln), generator=g)[:N]
    fg, ln = fg[pick].int().cuda(), ln[pick].int().cuda()
    ids = torch.randperm(len(ln), generator=g).int().cuda()
    model = S.FgramModel(P, D, 8, FF, n_layers, K)
    tok16 = tok.bfloat16().cuda()
    rows = torch.zeros((len(ln), D), dtype=torch.bfloat16, device="cuda")
    S.precompute_fgram_rows(S.FgramModelMx4(model), fg, ln, ids, tok16, rows)
    P64 = {k: v.double().cuda() for k, v in P.items()}
    tol = 6.1e-5 * 23 * 1.5
    for n in (2, 3):
        for at in (ln == n).nonzero().flatten().split(20_000):
            if at.numel() == 0:
                continue
            want = forward(P64, tok16.double(), fg[at, :n].long(), n_layers)
            err = (rows[ids[at].long()].double() - want).abs()
            over = (err - (tol + 2.0 ** -8 * (want.abs() + tol))).amax(1)
            bad = (over > 0).nonzero().flatten()
            assert bad.numel() == 0, (n, bad.numel(), fg[at][bad[0]].tolist(), float(over.max()))
