"""The precompute of F with 4-bit linear maps against oracle/mx4.py, which rounds where
the library rounds.

What is left between the two is fp32 against 64 bits, seen through roundings: where the
two sides' values lie on either side of a midpoint the rounded ones differ.  For bf16
that is one step of an element and stays inside the bar that the bf16 model's test
derives (3 eps(L) of a row's norm, eps(L) = 2^-9 sqrt((5 L + 2) / 3), for every element
wrong by its rounding).  A code of 4 bits falls the other way where the value lies within
its bf16 step of a midpoint of codes, about one in a hundred of those whose bf16 differs,
which itself is about one in a thousand: less than one code in a row of 4,096 expected.
So nine rows of ten are held to the bf16 bar.  In the others one code that differs moves
the next product's inputs, by more than their distance from a midpoint for some, and so
on: there any code may be the neighbouring one.  A step is at most max(a / 2, s / 2) for
a magnitude a and scale s, and s at most a quarter of the block's largest magnitude t, so
that a block that is a step off everywhere is off by at most sqrt(1/4 + 32 (t / 8)^2 /
sum a^2) of its norm: with t^2 <= 5 and sum a^2 = 32 rms^2 (normal rows) 0.57, and the
row by no more than its largest block: 0.6.  (The first form of this test allowed 16
codes in any row, without what follows from one: rows at 0.14, 98 in a hundred at
0.0016.)  A wrong matrix, bias or order moves every row."""
import numpy as np
import pytest
import torch

import paper_2502_01637_amd as S
from gpu_util import dev
from oracle import mx4
from test_gpu_fgram_model import as_f64, bf16_dev, eps, random_fgrams
from workloads.fgram_model import ModelConfig, bf16_bits_to_f64, make_params, make_token_rows

pytestmark = pytest.mark.gpu

CASES = [(ModelConfig(512, 8, 1024, 2, 7), 700), (ModelConfig(1024, 16, 4096, 1, 5), 200),
         (ModelConfig(512, 4, 640, 2, 3), 9), (ModelConfig(1536, 12, 1024, 1, 4), 60),
         (ModelConfig(512, 8, 512, 0, 6), 30)]


def inputs(cfg, N, V=300):
    rng = np.random.default_rng(cfg.d + N)
    P, T = make_params(cfg, seed=21), make_token_rows(V, cfg.d, seed=22)
    fg, lengths = random_fgrams(rng, V, N, cfg.max_len)
    return P, T, fg, lengths, (rng.permutation(N) + 5).astype(np.int32)


def models(cfg, P):
    model = S.FgramModel(P, cfg.d, cfg.n_heads, cfg.d_ff, cfg.n_layers, cfg.max_len)
    return model, S.FgramModelMx4(model)


@pytest.mark.parametrize("cfg,N", CASES)
def test_rows_match_the_oracle(cfg, N):
    P, T, fg, lengths, ids = inputs(cfg, N)
    rows = torch.zeros((N + 5, cfg.d), dtype=torch.bfloat16, device="cuda")
    S.precompute_fgram_rows(models(cfg, P)[1], dev(fg), dev(lengths), dev(ids), bf16_dev(T), rows)
    ref = mx4.fgram_forward(fg, lengths, bf16_bits_to_f64(T),
                            {k: bf16_bits_to_f64(v) for k, v in P.items()}, cfg.n_layers,
                            cfg.n_heads)
    got = as_f64(rows)[ids]
    err = np.linalg.norm(got - ref, axis=1) / np.linalg.norm(ref, axis=1)
    bar = 3 * eps(cfg.n_layers)
    assert np.quantile(err, 0.9) <= bar, (np.quantile(err, 0.9), bar)
    assert err.max() <= 0.6, err.max()
    assert not rows[:5].any()


def test_weights_are_the_quantised_rows():
    cfg, N = CASES[2]
    P, *_ = inputs(cfg, N)
    model, four = models(cfg, P)
    at = 0
    for layer in range(cfg.n_layers):
        for name in ("w_qkv", "w_o", "w_fc1", "w_fc2"):
            w = bf16_bits_to_f64(P[f"l{layer}.{name}"])
            want = mx4.quantize(w[:3])
            got = four.weights[at:at + want.size].cpu().numpy().reshape(want.shape)
            assert np.array_equal(got, want), (layer, name)
            at += w.shape[0] * want.shape[1]
    assert at == four.weights.numel()


def test_a_4bit_table_from_a_4bit_model():
    """Token rows and F, precomputed by the 4-bit model, quantised and served."""
    cfg, N = CASES[0]
    P, T, fg, lengths, _ = inputs(cfg, N)
    keep = np.unique(np.array([hash(tuple(f[:n])) for f, n in zip(fg, lengths)]),
                     return_index=True)[1]
    fg, lengths = fg[keep], lengths[keep]
    V, n = len(T), len(keep)
    ids = np.arange(V, V + n, dtype=np.int32)
    rows = torch.empty((V + n, cfg.d), dtype=torch.bfloat16, device="cuda")
    rows[:V] = bf16_dev(T)
    _, four = models(cfg, P)
    S.precompute_fgram_rows(four, dev(fg), dev(lengths), dev(ids), rows[:V], rows)
    table = S.build_fgram_table(dev(fg), dev(lengths), dev(ids))
    q = S.quantize_mx4(rows)
    X = torch.randint(0, V, (4, 50), dtype=torch.int32, device="cuda")
    X[0, :lengths[0]] = dev(fg[0, :lengths[0]])
    want, _ = S.lookup(table, X, cfg.max_len)
    out = S.gather_mx4(want, q)
    S.check_ok()
    values = mx4.values(mx4.quantize(rows[want.flatten()[:60].long()].float().cpu().numpy()), cfg.d)
    assert np.array_equal(out.view(-1, cfg.d)[:60].double().cpu().numpy(), values)


def test_more_than_one_chunk_and_a_stream():
    """More states than a chunk holds give the rows that the f-grams give alone; a side
    stream and a second call give the same bits."""
    cfg = ModelConfig(512, 8, 512, 1, 3)
    N = 40_000
    P, T, fg, lengths, ids = inputs(cfg, N, V=3000)
    _, four = models(cfg, P)
    args = [dev(fg), dev(lengths), dev(ids), bf16_dev(T)]
    rows = [torch.zeros((N + 5, cfg.d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    S.precompute_fgram_rows(four, *args, rows[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    S.precompute_fgram_rows(four, *args, rows[1], stream=side)
    assert torch.equal(rows[0], rows[1])
    some = np.arange(0, N, 997)
    S.precompute_fgram_rows(four, *(dev(x[some]) for x in (fg, lengths, ids)), args[3], rows[2])
    at = torch.from_numpy(ids[some]).long().cuda()
    a, b = rows[0][at].double(), rows[2][at].double()
    # other tiles sum in another order: as against the oracle
    err = (a - b).norm(dim=1) / a.norm(dim=1)
    assert float(err.quantile(0.9)) <= 3 * eps(1) and float(err.max()) <= 0.6
