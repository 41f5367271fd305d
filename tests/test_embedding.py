"""Embedding lookup and its gradient by sorted tokens, against the plain numpy forms."""
import numpy as np
import pytest
import torch

from paper_2602_04396_b200 import build as lbuild
from paper_2602_04396_b200 import embedding, lordo
from tests import tables_reference as ref

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step, relative


def make_tokens(K, T, V, kind, seed):
    rng = np.random.default_rng(seed)
    if kind == "uniform":
        tok = rng.integers(0, V, (K, T))
    elif kind == "one":
        tok = np.full((K, T), V - 1)
    elif kind == "pads":  # all kinds of padding, a worker with nothing else
        tok = rng.integers(0, V, (K, T))
        tok[rng.random((K, T)) < 0.4] = -1
        tok[rng.random((K, T)) < 0.1] = V
        tok[rng.random((K, T)) < 0.1] = -(2 ** 31)
        tok[0] = 2 ** 31 - 1
    elif kind == "few":
        tok = rng.integers(0, min(V, 3), (K, T))
    else:  # descending
        tok = np.tile(np.arange(T)[::-1] % V, (K, 1))
    return tok


# ---------------------------------------------------------------------------------------------
# no GPU
# ---------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def lib():
    lbuild.build()
    return lordo.load_library()


def test_reference_gradient_is_the_lookups():
    """The plain forms against autograd, padding among the tokens."""
    W = torch.randn(1, 5, 3, dtype=torch.float64, requires_grad=True)
    tok = np.array([[4, -1, 0, 4, 5, 4]])
    safe = torch.from_numpy(np.where((tok >= 0) & (tok < 5), tok, 0))
    inside = torch.from_numpy((tok >= 0) & (tok < 5)).double().unsqueeze(2)
    out = W[0][safe] * 2.5 * inside
    dY = torch.randn_like(out)
    out.backward(dY)
    assert np.allclose(ref.lookup(W.detach().numpy(), tok, 2.5), out.detach().numpy(), atol=1e-14)
    assert np.allclose(ref.table_grad(tok, dY.numpy(), 5, 2.5), W.grad.numpy(), atol=1e-14)


def test_entry_points_refuse_bad_arguments(lib):
    """Checked before anything is launched: the pointers are never followed."""
    p, q = 4096, 8192
    look = lambda W=p, wd=0, K=2, V=10, d=8, tok=p, ix=0, T=4, out=q, od=0: lib.lordo_embedding(W, wd, K, V, d, tok, ix, T, 1.0, out, od, None)
    assert look(wd=2) == 1 and look(od=-1) == 1 and look(ix=2) == 1 and look(K=0) == 1 and look(K=65) == 1 and look(V=0) == 1 and look(d=0) == 1
    assert look(T=-1) == 1 and look(W=None) == 1 and look(tok=None) == 1 and look(out=None) == 1
    assert look(V=2 ** 30 + 1) == 8 and look(T=2 ** 30 + 1) == 8 and look(d=2 ** 24 + 1) == 8
    assert look(W=p + 2) == 3 and look(wd=1, W=p + 1) == 3 and look(tok=p + 2) == 3 and look(ix=1, tok=p + 4) == 3 and look(out=q + 2) == 3
    assert look(T=0, W=None, tok=None, out=None) == 0

    def grad(dY=p, yd=0, tok=p, ix=0, K=2, V=10, d=8, T=4, dW=q, wd=0, acc=0, ws=p, nb=1 << 40):
        return lib.lordo_embedding_grad(dY, yd, tok, ix, K, V, d, T, 1.0, dW, wd, acc, ws, nb, None)

    assert grad(yd=3) == 1 and grad(wd=3) == 1 and grad(ix=5) == 1 and grad(acc=2) == 1 and grad(K=65) == 1 and grad(V=0) == 1 and grad(T=-1) == 1
    assert grad(dY=None) == 1 and grad(tok=None) == 1 and grad(dW=None) == 1 and grad(ws=None) == 1
    assert grad(ws=p + 16) == 3 and grad(dY=p + 2) == 3 and grad(tok=p + 1) == 3 and grad(dW=q + 2) == 3
    assert grad(nb=16) == 5
    assert grad(T=0, acc=1, dY=None, tok=None, ws=None) == 0
    assert lib.lordo_embedding_grad_query_workspace(2, 10, 8, 4, None) == 1


def test_binding_refuses_host_tensors(lib):
    with pytest.raises(ValueError):
        embedding.embedding(torch.zeros(4, 8), torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        embedding.embedding_grad(torch.zeros(3, 8), torch.zeros(3, dtype=torch.int64), 4)


# ---------------------------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------------------------
SHAPES = [(1, 1, 1, 1), (1, 5, 8, 1), (2, 7, 3, 33), (3, 1000, 72, 257), (1, 50000, 16, 1000), (2, 255, 264, 4100), (2, 256, 40, 2049), (1, 70000, 8, 9001),
          (1, 40, 1000, 63), (8, 300, 768, 96), (2, 3000, 8, 20000), (2, 70000, 16, 30001)]


@pytest.mark.gpu
@pytest.mark.parametrize("K,V,d,T", SHAPES)
@pytest.mark.parametrize("dt,odt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("kind", ["uniform", "pads"])
def test_lookup(K, V, d, T, dt, odt, kind):
    """One product in fp32 and one rounding to the output's type: off by half a step of either."""
    W = torch.randn(K, V, d, device="cuda").to(DT[dt])
    tok = make_tokens(K, T, V, kind, V + T)
    want = ref.lookup(ref.to64(W), tok, ref.f32(11.3))
    for ix in (torch.int32, torch.int64):
        out = embedding.embedding(W, torch.from_numpy(tok).to("cuda", ix), scale=11.3, out_dtype=DT[odt])
        assert out.shape == (K, T, d) and out.dtype == DT[odt]
        assert (np.abs(ref.to64(out) - want) <= (HALF["f32"] + HALF[odt] * (1 + HALF["f32"])) * np.abs(want)).all()
    one = embedding.embedding(W[0], torch.from_numpy(tok[0]).cuda(), out_dtype=DT[odt])  # a single table, tokens of any shape
    assert torch.equal(one, embedding.embedding(W[:1], torch.from_numpy(tok[:1]).cuda(), out_dtype=DT[odt])[0])


@pytest.mark.gpu
@pytest.mark.parametrize("K,V,d,T", SHAPES)
@pytest.mark.parametrize("dt,odt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("kind", ["uniform", "one", "pads", "few", "descending"])
def test_gradient(K, V, d, T, dt, odt, kind):
    """A sum of L terms in fp32, whatever its order: off by at most (L - 1) half steps of the sum of the magnitudes, then a product, with
    accumulate a sum, and a rounding to the output's type. Twice the same bits. Accumulating leaves rows without a token as they are."""
    dY = torch.randn(K, T, d, device="cuda").to(DT[dt])
    tok = make_tokens(K, T, V, kind, V + T)
    tokens = torch.from_numpy(tok).to("cuda", torch.int32 if T % 2 else torch.int64)
    y, s = ref.to64(dY), ref.f32(0.7)
    want, size = ref.table_grad(tok, y, V, s), ref.table_grad(tok, np.abs(y), V, abs(s))
    count = ref.table_grad(tok, np.ones_like(y), V, 1.0)
    sums = (np.maximum(count, 1) + 1) * HALF["f32"] * size
    got = embedding.embedding_grad(dY, tokens, V, scale=0.7, K=K, out_dtype=DT[odt])
    assert got.shape == (K, V, d) and got.dtype == DT[odt]
    assert (np.abs(ref.to64(got) - want) <= sums + HALF[odt] * (np.abs(want) + sums)).all()
    assert torch.equal(got, embedding.embedding_grad(dY, tokens, V, scale=0.7, K=K, out_dtype=DT[odt]))
    old = torch.randn(K, V, d, device="cuda").to(DT[odt])
    acc = embedding.embedding_grad(dY, tokens, V, scale=0.7, out=old.clone(), accumulate=True)
    total = want + ref.to64(old)
    off = sums + HALF["f32"] * (np.abs(total) + sums)
    assert (np.abs(ref.to64(acc) - total) <= off + HALF[odt] * (np.abs(total) + off)).all()
    untouched = torch.from_numpy(count[:, :, 0] == 0).cuda()
    assert torch.equal(acc[untouched], old[untouched])
    assert not got[untouched].any()


@pytest.mark.gpu
def test_gradient_of_rows_with_infinities():
    """A padded position's row may hold anything, and a non-finite row reaches its own token only."""
    dY = torch.randn(1, 40, 24, device="cuda")
    tokens = torch.arange(40, device="cuda").view(1, 40) % 8
    dY[0, 3] = float("inf")
    dY[0, 5] = float("nan")
    tokens[0, 5] = -1
    got = embedding.embedding_grad(dY, tokens, 8, K=1)
    assert torch.isinf(got[0, 3]).all() and torch.isfinite(got[0, [0, 1, 2, 4, 5, 6, 7]]).all()


@pytest.mark.gpu
def test_gradient_matches_differences_of_the_lookup():
    """d <dY, lookup(W)> / dW against differences of the lookup itself, fp32. The lookup is linear: a difference of 1 in an element of W
    is exact but for the roundings of `out` (one half step of |scale (w + 1)| <= 24 each)."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    W = torch.randn(2, 6, 5, device="cuda", generator=gen)
    tokens = torch.randint(-1, 6, (2, 9), device="cuda", generator=gen)
    dY = torch.randn(2, 9, 5, device="cuda", generator=gen)
    got = ref.to64(embedding.embedding_grad(dY, tokens, 6, scale=3.0, K=2))
    y, base = ref.to64(dY), ref.to64(embedding.embedding(W, tokens, scale=3.0))
    for k, v, j in [(0, 0, 0), (0, 3, 4), (1, 5, 2), (1, 1, 1)]:
        moved = W.clone()
        moved[k, v, j] += 1.0
        step = float(moved[k, v, j].double() - W[k, v, j].double())
        diff = ((ref.to64(embedding.embedding(moved, tokens, scale=3.0)) - base) * y).sum() / step
        assert abs(diff - got[k, v, j]) <= 9 * 2 * 24 * 2.0 ** -24 * np.abs(y).max() / step + 20 * 2.0 ** -24 * 3 * np.abs(y).sum()


@pytest.mark.gpu
def test_unaligned_rows_and_arrays():
    """Element-aligned addresses: the same values as at aligned ones."""
    flat = torch.randn(2 * 50 * 16 + 1, device="cuda").to(torch.bfloat16)
    W, U = flat[:-1].view(2, 50, 16), flat[1:].view(2, 50, 16)
    tokens = torch.randint(0, 50, (2, 333), device="cuda")
    assert torch.equal(embedding.embedding(U, tokens, scale=2.0), embedding.embedding(U.clone(), tokens, scale=2.0))
    flat = torch.randn(2 * 333 * 16 + 1, device="cuda").to(torch.bfloat16)
    dY = flat[1:].view(2, 333, 16)
    assert torch.equal(embedding.embedding_grad(dY, tokens, 50, K=2), embedding.embedding_grad(dY.clone(), tokens, 50, K=2))
    big = torch.zeros(2 * 50 * 16 + 1, device="cuda")
    out = big[1:].view(2, 50, 16)
    embedding.embedding_grad(dY, tokens, 50, out=out)
    assert torch.equal(out, embedding.embedding_grad(dY, tokens, 50, K=2, out_dtype=torch.float32)) and big[0] == 0


@pytest.mark.gpu
def test_empty_batches():
    W = torch.randn(2, 9, 8, device="cuda")
    none = torch.zeros(2, 0, device="cuda", dtype=torch.int64)
    assert embedding.embedding(W, none).shape == (2, 0, 8)
    dY = torch.zeros(2, 0, 8, device="cuda")
    assert not embedding.embedding_grad(dY, none, 9, out=torch.ones(2, 9, 8, device="cuda")).any()
    assert embedding.embedding_grad(dY, none, 9, out=torch.ones(2, 9, 8, device="cuda"), accumulate=True).all()


@pytest.mark.gpu
def test_rows_behind_two_to_the_32nd():
    """A table of 8 x 70001 x 8192 elements (9.2 GB): rows at its end, read and added to."""
    K, V, d = 8, 70001, 8192
    W = torch.zeros(K, V, d, device="cuda", dtype=torch.bfloat16)
    W[K - 1, V - 1] = torch.randn(d, device="cuda").to(torch.bfloat16)
    tok = torch.full((K, 40), V - 1, device="cuda", dtype=torch.int32)
    tok[:, ::3] = 0
    out = embedding.embedding(W, tok)
    assert torch.equal(out[K - 1, 1], W[K - 1, V - 1]) and not out[:K - 1].any() and not out[:, 0].any()
    dY = torch.ones(K, 40, d, device="cuda", dtype=torch.bfloat16)
    was = W[K - 1, V - 1].clone()
    embedding.embedding_grad(dY, tok, V, out=W, accumulate=True)
    assert torch.equal(W[K - 1, V - 1], (was.float() + 26.0).to(torch.bfloat16)) and (W[K - 1, 0] == 14).all() and not W[:, 1:V - 1].any()
    embedding.embedding_grad(dY, tok, V, out=W)
    assert (W[:, V - 1] == 26).all() and (W[:, 0] == 14).all() and not W[:, 1:V - 1].any()


@pytest.mark.gpu
def test_streams_and_graphs():
    """On a stream of its own, and captured twice and replayed in turn on other inputs: the eager call's bits."""
    V, T = 700, 5000
    W = torch.randn(2, V, 40, device="cuda").to(torch.bfloat16)
    sets = [(torch.randint(-1, V, (2, T), device="cuda"), torch.randn(2, T, 40, device="cuda").to(torch.bfloat16)) for _ in range(3)]
    eager = [(embedding.embedding(W, t, scale=3.0), embedding.embedding_grad(y, t, V, K=2)) for t, y in sets]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = [(embedding.embedding(W, t, scale=3.0, stream=side), embedding.embedding_grad(y, t, V, K=2, stream=side)) for t, y in sets]
    torch.cuda.synchronize()
    for a, b in zip(eager, on_side):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    graphs = []
    for _ in range(2):
        tok, dY = sets[0][0].clone(), sets[0][1].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, grad = embedding.embedding(W, tok, scale=3.0), embedding.embedding_grad(dY, tok, V, K=2)
        graphs.append((graph, tok, dY, out, grad))
    for i in (0, 1, 2, 1):
        for graph, tok, dY, out, grad in graphs:
            tok.copy_(sets[i][0])
            dY.copy_(sets[i][1])
            graph.replay()
        for graph, tok, dY, out, grad in graphs:
            assert torch.equal(out, eager[i][0]) and torch.equal(grad, eager[i][1])


@pytest.mark.gpu
def test_binding_refusals():
    W = torch.zeros(2, 9, 8, device="cuda")
    tok = torch.zeros(2, 3, device="cuda", dtype=torch.int64)
    dY = torch.zeros(2, 3, 8, device="cuda")
    bad = [lambda: embedding.embedding(W, tok.to(torch.int16)), lambda: embedding.embedding(W, tok[:1]), lambda: embedding.embedding(W, tok.cpu()),
           lambda: embedding.embedding(W.transpose(1, 2), tok), lambda: embedding.embedding(W, tok, out=torch.zeros(2, 3, 9, device="cuda")),
           lambda: embedding.embedding(W.half(), tok), lambda: embedding.embedding(W[0, 0], tok),
           lambda: embedding.embedding_grad(dY, tok[:, :2], 9, K=2), lambda: embedding.embedding_grad(dY, tok, 9, K=3),
           lambda: embedding.embedding_grad(dY, tok, 9, accumulate=True), lambda: embedding.embedding_grad(dY, tok, 8, out=W),
           lambda: embedding.embedding_grad(dY, tok, 9, out=W, out_dtype=torch.bfloat16), lambda: embedding.embedding_grad(dY, tok, 9, out=W.cpu())]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(lordo.LordoError):
        embedding.embedding_grad(dY, tok, 0, K=2)


@pytest.mark.gpu
def test_inputs_given_back_before_their_stream_has_come_to_them():
    """Calls on a stream that is still busy with earlier work (a tenth of a second), their inputs dropped at once and their memory taken and
    overwritten on the current stream: the bits of calls whose inputs were kept."""
    K, V, d, T = 2, 900, 256, 700

    def make(s):
        gen = torch.Generator(device="cuda").manual_seed(s)
        return (torch.randn(K, V, d, device="cuda", generator=gen), torch.randint(-1, V, (K, T), device="cuda", generator=gen),
                torch.randn(K, T, d, device="cuda", generator=gen), torch.randint(-1, V, (K, T), device="cuda", generator=gen, dtype=torch.int32))

    kept = [make(s) for s in range(4)]
    want = [(embedding.embedding(W, t), embedding.embedding_grad(dY, u, V, K=K)) for W, t, dY, u in kept]
    added = [embedding.embedding_grad(dY, u, V, out=W.clone(), accumulate=True) for W, _, dY, u in kept]
    side, got, junk = torch.cuda.Stream(), [], [[torch.full_like(x, -1) for x in kept[0]]]  # its kernels are loaded by now
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    for s in range(4):
        W, t, dY, u = make(s)
        torch.cuda.current_stream().synchronize()
        first = embedding.embedding(W, t, stream=side), embedding.embedding_grad(dY, u, V, K=K, stream=side)
        del t
        got.append(first)
        with torch.cuda.stream(side):  # a copy that is made where the table is still whole
            embedding.embedding_grad(dY, u, V, out=W, accumulate=True, stream=side)
            got[-1] += (W.clone(),)
        del W, dY, u
        junk.append([torch.full_like(x, -1 if x.dtype in (torch.int32, torch.int64) else float("nan")) for x in kept[s]])
    torch.cuda.synchronize()
    for g, w, a in zip(got, want, added):
        assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1]) and torch.equal(g[2], a)


@pytest.mark.gpu
def test_a_stream_of_another_device():
    """Refused, not replaced by the current stream of the tensors' device."""
    class Other:
        device, cuda_stream = torch.device("cuda", 1), 0

    W, tok = torch.zeros(9, 8, device="cuda:0"), torch.tensor([1, 3], device="cuda:0")
    with pytest.raises(ValueError, match="stream"):
        embedding.embedding(W, tok, stream=Other())
    with pytest.raises(ValueError, match="stream"):
        embedding.embedding_grad(torch.zeros(2, 8, device="cuda:0"), tok, 9, stream=Other())


@pytest.mark.gpu
def test_a_table_that_requires_a_gradient():
    """The lookup is no part of autograd: where a gradient would be lost in silence the call is refused."""
    W, tok = torch.randn(9, 8, device="cuda", requires_grad=True), torch.tensor([1, 3], device="cuda")
    with pytest.raises(ValueError, match="detach"):
        embedding.embedding(W, tok)
    want = W.detach()[tok]
    assert torch.equal(embedding.embedding(W.detach(), tok), want)
    with torch.no_grad():
        assert torch.equal(embedding.embedding(W, tok), want)


@pytest.mark.gpu
def test_no_workers():
    tok = torch.zeros(0, 3, device="cuda", dtype=torch.int64)
    with pytest.raises(ValueError, match="worker"):
        embedding.embedding(torch.zeros(0, 9, 8, device="cuda"), tok)
    with pytest.raises(ValueError, match="worker"):
        embedding.embedding_grad(torch.zeros(0, 3, 8, device="cuda"), tok, 9, K=0)
    with pytest.raises(ValueError, match="worker"):
        embedding.embedding_grad(torch.zeros(0, 3, 8, device="cuda"), tok, 9, out=torch.zeros(0, 9, 8, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("K,V,d,T", SHAPES)
@pytest.mark.parametrize("kind", ["uniform", "one", "pads", "few", "descending"])
def test_gradient_from_fp32_into_bf16(K, V, d, T, kind):
    """As test_gradient, four columns a lane and two bytes each in the table."""
    test_gradient(K, V, d, T, "f32", "bf16", kind)


@pytest.mark.gpu
@pytest.mark.parametrize("K,V,d", [(2, 30000, 1000), (2, 90000, 333), (3, 30000, 768), (3, 130001, 96)])
@pytest.mark.parametrize("dt,odt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_rows_without_a_token_of_a_large_table(K, V, d, dt, odt):
    """Tables above 100 MB, whose rows without a token are zeroed in three parts: one while the tokens are sorted, one beside the windows, one beside
    the joining. `out` holds NaN before the call; tokens lie on both sides of where the parts meet (64 MB from the front, 128 MB from the end) and at the
    ends of their 32 and 256 rows. Every row against the fp64 sums, bounds as in test_gradient."""
    row = K * d * (4 if odt == "f32" else 2)
    T, first, last = 1500, (64 << 20) // row, V - (128 << 20) // row
    gen = torch.Generator(device="cuda").manual_seed(V)
    tokens = torch.randint(0, V, (K, T), device="cuda", generator=gen)
    at = [x + y for x in (0, first, first + 32, first + 256, max(first, last), V - 1) for y in (-2, -1, 0, 1)]
    tokens[:, :len(at)] = torch.tensor(at, device="cuda")
    tokens[:, -200:] = V // 3  # a token of more than one window
    dY = torch.randn(K, T, d, device="cuda", generator=gen).to(DT[dt])
    out = torch.full((K, V, d), float("nan"), device="cuda", dtype=DT[odt])
    assert embedding.embedding_grad(dY, tokens, V, scale=0.5, out=out) is out
    for k in range(K):
        inside = (tokens[k] >= 0) & (tokens[k] < V)
        ids, y = tokens[k][inside], dY[k][inside].double()
        want = torch.zeros(V, d, device="cuda", dtype=torch.float64).index_add_(0, ids, y) * 0.5
        size = torch.zeros(V, d, device="cuda", dtype=torch.float64).index_add_(0, ids, y.abs()) * 0.5
        count = torch.zeros(V, 1, device="cuda", dtype=torch.float64).index_add_(0, ids, torch.ones(len(ids), 1, device="cuda", dtype=torch.float64))
        sums = (count.clamp(min=1) + 1) * HALF["f32"] * size
        assert ((out[k].double() - want).abs() <= sums + HALF[odt] * (want.abs() + sums)).all()
        assert not out[k][count[:, 0] == 0].any()


@pytest.mark.gpu
def test_a_captured_call_on_a_forked_stream():
    """A branch of a captured graph, its inputs recorded on the branch's stream and dropped within the capture: replayed, the eager call's bits."""
    V, T = 300, 700
    W = torch.randn(2, V, 24, device="cuda")
    tok, dY = torch.randint(-1, V, (2, T), device="cuda"), torch.randn(2, T, 24, device="cuda")
    want = embedding.embedding(W, tok, scale=2.0), embedding.embedding_grad(dY * 3.0, tok, V, K=2)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        larger = dY * 3.0
        side.wait_stream(torch.cuda.current_stream())
        out, grad = embedding.embedding(W, tok, scale=2.0, stream=side), embedding.embedding_grad(larger, tok, V, K=2, stream=side)
        del larger
        other = torch.full_like(dY, float("nan"))
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(2):
        out.zero_(), grad.zero_()
        graph.replay()
        assert torch.equal(out, want[0]) and torch.equal(grad, want[1])
