"""Calls on a stream that is not the current one: where their results live, and chains
whose intermediate results are dropped while the stream still works on them."""
import numpy as np
import pytest
import torch

import paper_2502_01637_amd as S

pytestmark = pytest.mark.gpu


def owner(t):
    """The stream whose memory pool holds the tensor."""
    for seg in torch.cuda.memory._snapshot()["segments"]:
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not torch's memory")


def inputs():
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randn((300, 512), generator=g, device="cuda").bfloat16()
    w = S.quantize_mx4(torch.randn((512, 512), generator=g, device="cuda"))
    ids = torch.randint(0, 300, (300,), generator=g, device="cuda").int()
    torch.cuda.synchronize()
    return x, w, ids


@pytest.mark.parametrize("as_handle", [False, True])
def test_4bit_results_live_on_their_stream(as_handle):
    x, w, ids = inputs()
    side = torch.cuda.Stream()
    st = side.cuda_stream if as_handle else side
    q = S.quantize_mx4(x, stream=st)
    results = [q.data, S.gather_mx4(ids, q, stream=st), S.dequantize_mx4(q, stream=st),
               S.linear_mx4(x, w, stream=st)]
    side.synchronize()
    assert [owner(t) for t in results] == [side.cuda_stream] * 4
    here = torch.cuda.current_stream().cuda_stream
    assert owner(S.linear_mx4(x, w)) == owner(S.linear_mx4(x, w, stream=here)) == here


@pytest.mark.parametrize("as_handle", [False, True])
def test_4bit_chain_of_dropped_results(as_handle):
    """The chain runs on a side stream, the default one stays current and is busy with
    blocks of the same sizes that it gives back."""
    x, w, ids = inputs()

    def chain(stream):
        y = S.gather_mx4(ids, S.quantize_mx4(x, stream=stream), stream=stream)
        for _ in range(3):
            y = S.linear_mx4(S.dequantize_mx4(S.quantize_mx4(y, stream=stream), stream=stream), w,
                             gelu=True, stream=stream)
        return y

    want = chain(None).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(10):
        for _ in range(20):
            for n in (300 * 272, 300 * 1024):
                torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
        got = chain(side.cuda_stream if as_handle else side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)


def test_4bit_chain_captured_over_two_streams():
    """A side stream inside a captured graph, replayed with new inputs."""
    x, w, ids = inputs()
    side = torch.cuda.Stream()

    def run(stream):
        q = S.quantize_mx4(x, stream=stream)
        return S.linear_mx4(S.gather_mx4(ids, q, stream=stream), w, stream=stream)

    run(None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = run(side)
        torch.cuda.current_stream().wait_stream(side)
    for seed in range(4):
        x.copy_(torch.randn(x.shape, generator=torch.Generator("cuda").manual_seed(seed),
                            device="cuda"))
        want = run(None)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), seed
        np.testing.assert_equal(S.check(), S.scone.OK)


@pytest.mark.parametrize("as_handle", [False, True])
def test_4bit_model_made_on_a_side_stream(as_handle):
    """From parameters that the current stream is still copying."""
    from workloads.fgram_model import ModelConfig, make_params
    cfg = ModelConfig(512, 8, 1024, 2, 3)
    P = {k: torch.from_numpy(np.array(v).view(np.int16)).cuda()
         for k, v in make_params(cfg, seed=4).items()}
    want = S.FgramModelMx4(S.FgramModel(P, 512, 8, 1024, 2, 3)).weights
    side = torch.cuda.Stream()
    busy = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        for k in range(20):
            busy.fill_(k)
        model = S.FgramModel(P, 512, 8, 1024, 2, 3)
        four = S.FgramModelMx4(model, stream=side.cuda_stream if as_handle else side)
        assert torch.equal(four.weights, want) and owner(four.weights) == side.cuda_stream


def byte_inputs():
    from gpu_util import build_gpu
    rng = np.random.default_rng(5)
    fg = np.unique(rng.integers(0, 30, (400, 3)), axis=0).astype(np.int32)
    table = build_gpu(fg, np.full(len(fg), 3), np.arange(30, 30 + len(fg)))
    g = torch.Generator("cuda").manual_seed(6)
    rows = torch.randn((30 + len(fg), 256), generator=g, device="cuda")
    tok = torch.randint(0, 30, (20, 100), generator=g, device="cuda").int()
    torch.cuda.synchronize()
    return table, rows, tok


@pytest.mark.parametrize("as_handle", [False, True])
def test_results_of_the_byte_calls_live_on_their_stream(as_handle):
    table, rows, tok = byte_inputs()
    side = torch.cuda.Stream()
    st = side.cuda_stream if as_handle else side
    far = S.HostRows(rows.shape[0] - 30, (256,), torch.float32)
    far.tensor().copy_(rows[30:])
    ws = torch.empty(S.split_workspace_bytes(tok.numel(), 1024), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    ids, lens = S.lookup(table, tok, 3, want_len=True, stream=st)
    results = [ids, lens, S.tag(table, tok, 3, stream=st)[0], S.gather(ids, rows, stream=st),
               S.embed(table, tok, 3, rows, stream=st),
               S.embed_pipelined(table, None, 3, None, ids, rows, stream=st),
               S.gather_split(ids, rows[:30], far, ws, stream=st),
               *S.discover_fgrams(tok, 3, 50, 2, stream=st)]
    count = S.scone.lookup_counted(table, tok, 3, stream=st)
    results += count[:2]
    side.synchronize()
    assert [owner(t) for t in results] == [side.cuda_stream] * len(results)
    want, wlen = S.lookup(table, tok, 3, want_len=True)
    again = S.scone.lookup_counted(table, tok, 3)
    assert torch.equal(ids, want) and torch.equal(lens, wlen) and torch.equal(results[2], wlen)
    assert torch.equal(count[0], want) and torch.equal(count[1], wlen) and count[2] == again[2] > 0
    values = rows[want.long()]
    assert all(torch.equal(t, values) for t in results[3:7])
    assert S.check() == S.scone.OK
    far.close()


def test_chain_of_dropped_ids():
    """A lookup whose ids are dropped behind the gather, on a side stream, under a busy
    current one."""
    table, rows, tok = byte_inputs()
    want = S.embed(table, tok, 3, rows)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        for _ in range(20):
            for n in (tok.numel() * 4, tok.numel() * 1024):
                torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
        got = S.gather(S.lookup(table, tok, 3, stream=side)[0], rows, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)
