"""hsadmm_embedding, hsadmm_embedding_gradient and hsadmm_dropout against their formulas in 64 bits (tests/ref_tokens.py derives the
bounds)."""
import numpy as np
import pytest
import torch

import paper_2512_14628_amd as pkg
from tests import ref_tokens as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = pkg.TYPE_F32, pkg.TYPE_BF16, pkg.TYPE_F16
NAMES = {F32: "fp32", BF16: "bf16", F16: "fp16"}
NAN = float("nan")


def say(*what):
    print(*what, flush=True)


def table(D, V, before=4):
    """Three layers, the middle one of V rows of D, others around it."""
    after = before + V * D + (-(V * D)) % 4
    return pkg.Plan({"elem_off": [0, before, after], "c_out": [1, V, 1], "c_in": [before, D, 5], "khw": [1, 1, 2], "mode": [0, 0, 0],
                     "k": [1, V, 1]})


def rows(n, D, pad, dtype, gen=None, sigma=1.0):
    """Rows with a gap of NaN between them, and two rows of NaN behind the last."""
    x = torch.full((n + 2, D + pad), NAN, dtype=dtype, device=DEV)
    if gen is not None:
        x[:n, :D] = (torch.randn((n, D), generator=gen) * sigma).to(dtype).to(DEV)
    return x


def untouched(x, n, D):
    assert torch.isnan(x[n:]).all() and torch.isnan(x[:, D:]).all()


def tokens(n, V, gen, kind, bits=64):
    if kind == "spread":
        ids = torch.randint(0, V, (n,), generator=gen)
    elif kind == "one":
        ids = torch.full((n,), V // 2)
    elif kind == "two":
        ids = torch.where(torch.rand(n, generator=gen) < 0.5, 0, V - 1)
    elif kind == "none":
        ids = torch.full((n,), -1)
    else:                                                    # the r-th token about 1 / r as often as the first; some are none
        ids = (float(V) ** torch.rand(n, generator=gen, dtype=torch.float64)).long() - 1
        ids = ids.clamp(0, V - 1)
        ids[torch.rand(n, generator=gen) < 0.1] = -100
        ids[torch.rand(n, generator=gen) < 0.05] = V
    return ids.to(torch.int64 if bits == 64 else torch.int32).to(DEV)


SIZES = [(1, 1, 1), (1, 2048, 5), (3, 7, 2), (5, 8, 100), (64, 64, 64), (65, 100, 1000), (300, 1001, 50), (1000, 4, 70000), (2000, 24, 3)]


@pytest.mark.parametrize("kind", [F32, BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", SIZES)
@pytest.mark.parametrize("pad", [0, 5, 8])
def test_embedding(kind, n, D, V, pad):
    say("embedding", NAMES[kind], n, D, V, pad)
    gen = torch.Generator().manual_seed(n + D + V)
    plan, dtype = table(D, V), ref.TYPES[kind]
    W = torch.full((plan.arena_elems,), NAN, dtype=dtype, device=DEV)
    w = W[4:4 + V * D].view(V, D)
    w.copy_(torch.randn((V, D), generator=gen).to(dtype))
    ids = tokens(n, V, gen, "common", 64 if pad else 32)
    out = rows(n, D, pad, dtype)
    pkg.hsadmm_embedding(plan, 1, W, ids, out[:n, :D], scale=3.7, type=kind, index_bits=64 if pad else 32)
    torch.cuda.synchronize()
    ref.close(out[:n, :D], *ref.embedding_reference(kind, w, ids.long(), np.float32(3.7).item()), "out")
    untouched(out, n, D)
    # a scale of one copies
    pkg.hsadmm_embedding(plan, 1, W, ids, out[:n, :D], type=kind, index_bits=64 if pad else 32)
    torch.cuda.synchronize()
    token = (ids >= 0) & (ids < V)
    assert torch.equal(out[:n, :D], torch.where(token[:, None], w[torch.where(token, ids, 0).long()], torch.zeros((), dtype=dtype, device=DEV)))


def gradient(plan, kind, ids, dY, G, scale=1.0, accumulate=False, bits=64, stream=None):
    nbytes = pkg.hsadmm_embedding_workspace(plan, 1, ids.numel())
    ws = torch.full((nbytes + 512,), 255, dtype=torch.uint8, device=DEV)
    pkg.hsadmm_embedding_gradient(plan, 1, ids, dY, G, ws, workspace_bytes=nbytes, scale=scale, accumulate=accumulate, type=kind,
                                  index_bits=bits, stream=stream)
    torch.cuda.synchronize()
    assert (ws[nbytes:] == 255).all()


def check_gradient(kind, n, D, V, spread, pad=0, accumulate=False, bits=64, scale=2.5):
    say("gradient", NAMES[kind], n, D, V, spread, pad)
    gen = torch.Generator().manual_seed(n * 7 + D + V)
    plan, dtype = table(D, V), ref.TYPES[kind]
    dY = rows(n, D, pad, dtype, gen)
    ids = tokens(n, V, gen, spread, bits)
    token = (ids >= 0) & (ids < V)
    dY[:n, :D][~token] = NAN                                  # (not read)
    G = torch.full((plan.arena_elems,), NAN, dtype=dtype, device=DEV)
    g = G[4:4 + V * D].view(V, D)
    if accumulate:
        g.copy_(torch.randn((V, D), generator=gen).to(dtype))
    before = g.clone()
    gradient(plan, kind, ids, dY[:n, :D], G, scale, accumulate, bits)
    value, bound = ref.embedding_gradient_reference(V, dY[:n, :D], ids.long(), scale)
    if accumulate:
        value, bound = value + before.double(), bound + ref.U * (value.abs() + before.double().abs())
    ref.close(g, value, ref.rounded(kind, value, bound), "G")
    if accumulate:
        idle = torch.ones(V, dtype=torch.bool, device=DEV)
        idle[ids[token].long()] = False
        assert torch.equal(g[idle], before[idle])
    assert torch.isnan(G[:4]).all() and torch.isnan(G[4 + V * D:]).all()
    first = g.clone()
    if accumulate:
        g.copy_(before)
    gradient(plan, kind, ids, dY[:n, :D], G, scale, accumulate, bits)
    assert torch.equal(first, g)                              # the same bits from run to run


@pytest.mark.parametrize("kind", [F32, BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", SIZES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_embedding_gradient(kind, n, D, V, accumulate):
    check_gradient(kind, n, D, V, "common", pad=(n + D) % 3 * 4, accumulate=accumulate, bits=32 if accumulate else 64)


@pytest.mark.parametrize("spread", ["spread", "one", "two", "none", "common"])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 128, 129, 1000, 32768, 32769, 70001])
def test_tokens_of_all_frequencies(spread, n):
    """Stretches of one token that begin, end and lie inside the sums' parts; one tile of the sort, and several."""
    check_gradient(F32, n, 12, 777, spread)


@pytest.mark.parametrize("kind,D", [(F32, 1023), (F32, 1025), (F32, 1027), (F32, 2049), (BF16, 2047), (BF16, 2049), (F16, 2055), (BF16, 4099), (F32, 259),
                                    (BF16, 515), (F16, 7), (F16, 9)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_rows_that_end_inside_a_piece(kind, D, accumulate):
    """Ends next to a wave's pieces: the last piece is moved back and shares columns with the one before it."""
    check_gradient(kind, 500, D, 30, "common", accumulate=accumulate)


@pytest.mark.parametrize("V", [1, 2, 511, 512, 513, 262143, 262144])
def test_vocabularies_around_whole_digits(V):
    check_gradient(BF16, 3000, 8, V, "spread")
    check_gradient(BF16, 40000, 8, V, "common")


def test_no_tokens():
    plan = table(8, 20)
    G = torch.full((plan.arena_elems,), 3.0, device=DEV)
    none, dY = torch.zeros(0, dtype=torch.int64, device=DEV), torch.zeros((0, 8), device=DEV)
    gradient(plan, F32, none, dY, G, accumulate=True)
    assert (G == 3).all()
    gradient(plan, F32, none, dY, G)
    assert (G[4:164] == 0).all() and (G[:4] == 3).all() and (G[164:] == 3).all()
    assert pkg.hsadmm_embedding(plan, 1, G, none, dY, index_bits=64) == 0


def test_embedding_is_the_gradients_transpose():
    """<embedding(W), dY> = <W, gradient(dY)>: both sides in 64 bits from fp32 outputs whose rounding is below 2^-23 of the terms."""
    gen = torch.Generator().manual_seed(3)
    V, D, n = 300, 36, 2000
    plan = table(D, V)
    W = torch.randn((plan.arena_elems,), generator=gen).to(DEV)
    dY = torch.randn((n, D), generator=gen).to(DEV)
    ids = tokens(n, V, gen, "common")
    out, G = torch.zeros((n, D), device=DEV), torch.zeros_like(W)
    pkg.hsadmm_embedding(plan, 1, W, ids, out, scale=0.5, index_bits=64)
    gradient(plan, F32, ids, dY, G, scale=0.5)
    terms = out.double() * dY.double()
    got = (W[4:4 + V * D].double() * G[4:4 + V * D].double()).sum()
    assert abs(got - terms.sum()) <= (n + 8) * ref.U * terms.abs().sum()


# ------------------------------------------------------------------ dropout

def drop(plan, kind, X, Y, p, seed, call, residual=None, **more):
    pkg.hsadmm_dropout(plan, X, Y, p, seed, call, residual=residual, type=kind, **more)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", [F32, BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D", [(1, 1), (1, 7), (1, 8), (3, 5), (7, 16), (33, 100), (128, 513), (1000, 24)])
@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("with_residual", [False, True])
def test_dropout(kind, n, D, pad, with_residual):
    say("dropout", NAMES[kind], n, D, pad, with_residual)
    plan, dtype = table(4, 4), ref.TYPES[kind]
    gen = torch.Generator().manual_seed(n + D)
    X, Y = rows(n, D, pad, dtype, gen), rows(n, D, pad, dtype)
    R = rows(n, D, pad, dtype, gen, 3.0) if with_residual else None
    for p, seed, call in ((0.0, 1, 0), (0.1, 2 ** 63 + 12345, 7), (0.5, 0, 2 ** 64 - 1), (0.999999, 9, 2 ** 33)):
        kept, factor = ref.dropout_kept(n * D, p, seed, call)
        kept = torch.from_numpy(kept).view(n, D).to(DEV)
        X[:n, :D][~kept] = NAN                            # (what is dropped may hold anything)
        X[:n, :D][kept] = torch.randn(int(kept.sum()), generator=gen).to(dtype).to(DEV)
        drop(plan, kind, X[:n, :D], Y[:n, :D], p, seed, call, None if R is None else R[:n, :D])
        x = torch.where(kept, X[:n, :D], torch.zeros((), dtype=dtype, device=DEV))
        ref.close(Y[:n, :D], *ref.dropout_reference(kind, x, kept, factor, None if R is None else R[:n, :D]), "Y")
        untouched(Y, n, D)


def test_dropped_share_and_independence():
    """Shares within five standard deviations of t / 65536; masks of two calls and two seeds agree as chance has it."""
    n = 1 << 20
    plan, x = table(4, 4), torch.ones((1, 1 << 20), device=DEV)
    for p in (0.1, 0.5, 0.9):
        masks = []
        for seed, call in ((5, 1), (5, 2), (6, 1)):
            y = torch.empty_like(x)
            drop(plan, F32, x, y, p, seed, call)
            masks.append((y == 0).double())
        t = np.floor(65536 * p + 0.5) / 65536
        for m in masks:
            assert abs(m.mean() - t) <= 5 * (t * (1 - t) / n) ** 0.5
        for a, b in ((0, 1), (0, 2), (1, 2)):
            assert abs((masks[a] * masks[b]).mean() - t * t) <= 5 * (t * t * (1 - t * t) / n) ** 0.5


def test_dropout_in_place_and_its_gradient():
    """In place on the input or the residual; the gradient is the same call on the output's gradient."""
    plan = table(4, 4)
    gen = torch.Generator().manual_seed(1)
    x, r, dy = (torch.randn((50, 40), generator=gen).to(DEV) for _ in range(3))
    want = torch.empty_like(x)
    drop(plan, F32, x, want, 0.3, 4, 5, r)
    a, b = x.clone(), r.clone()
    drop(plan, F32, a, a, 0.3, 4, 5, r)
    drop(plan, F32, x, b, 0.3, 4, 5, b)
    assert torch.equal(a, want) and torch.equal(b, want)
    dx = torch.empty_like(x)
    drop(plan, F32, dy, dx, 0.3, 4, 5)
    # linear in x: the difference of two outputs is the mask's factor times the inputs' difference
    kept, factor = ref.dropout_kept(x.numel(), 0.3, 4, 5)
    kept = torch.from_numpy(kept).view(50, 40).to(DEV)
    ref.close(dx, *ref.dropout_reference(F32, dy, kept, factor), "dX")
    # against differences: (Y(x + h dy) - Y(x - h dy)) / 2 h with everything but the mask linear; h a power of two
    h = 0.25
    up, down = torch.empty_like(x), torch.empty_like(x)
    drop(plan, F32, x + h * dy, up, 0.3, 4, 5, r)
    drop(plan, F32, x - h * dy, down, 0.3, 4, 5, r)
    off = (up.double() - down.double()) / (2 * h) - dx.double()
    size = (x.abs() + h * dy.abs()).double() * factor + r.abs().double()
    assert (off.abs() <= 8 * ref.U * size / h).all()


def test_the_calls_number_on_the_device_follows_replays():
    plan = table(4, 4)
    x = torch.randn((64, 72), generator=torch.Generator().manual_seed(2)).to(DEV)
    y, number = torch.empty_like(x), torch.zeros(1, dtype=torch.int64, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pkg.hsadmm_dropout(plan, x, y, 0.4, 77, 0, call_device=number)
    for call in (0, 1, 5, 2 ** 40):
        number.fill_(call)
        graph.replay()
        want = torch.empty_like(x)
        drop(plan, F32, x, want, 0.4, 77, call)
        assert torch.equal(y, want)


def test_captured_embedding_and_gradient():
    gen = torch.Generator().manual_seed(4)
    V, D, n = 500, 40, 900
    plan = table(D, V)
    W, dY = torch.randn((plan.arena_elems,), generator=gen).to(DEV), torch.randn((n, D), generator=gen).to(DEV)
    ids, out, G = tokens(n, V, gen, "common"), torch.zeros((n, D), device=DEV), torch.zeros(plan.arena_elems, device=DEV)
    ws = torch.zeros(pkg.hsadmm_embedding_workspace(plan, 1, n), dtype=torch.uint8, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pkg.hsadmm_embedding(plan, 1, W, ids, out, scale=2.0, index_bits=64)
        pkg.hsadmm_embedding_gradient(plan, 1, ids, dY, G, ws, index_bits=64)
    for i in range(3):
        ids.copy_(tokens(n, V, gen, ("spread", "one", "common")[i]))
        graph.replay()
        want_out, want_G = torch.zeros_like(out), torch.zeros_like(G)
        pkg.hsadmm_embedding(plan, 1, W, ids, want_out, scale=2.0, index_bits=64)
        gradient(plan, F32, ids, dY, want_G)
        assert torch.equal(out, want_out) and torch.equal(G[4:4 + V * D], want_G[4:4 + V * D])


def test_refusals():
    plan = table(20, 30)
    W, G = (torch.zeros(plan.arena_elems, device=DEV) for _ in range(2))
    ids, out = torch.zeros(6, dtype=torch.int32, device=DEV), torch.zeros((6, 20), device=DEV)

    def look(layer=1, W=W, ids=ids, out=out, **more):
        return pkg.hsadmm_embedding(plan, layer, W, ids, out, check=False, **more)

    assert look() == 0
    assert look(layer=-1) == -1 and look(layer=3) == -1 and look(layer=2, out=16) == -4
    assert look(type=5) == -4 and look(index_bits=8) == -4
    assert look(W=None) == -1 and look(out=None) == -1 and look(ids=ids.long()) == -1 and look(ids=ids, index_bits=64) == -1
    assert look(out=out[:, :19]) == -1 and look(out=out[:5]) == -1 and look(out=out.half()) == -1 and look(W=W[:-1]) == -1
    assert look(W=W.data_ptr() + 4) == -1 and look(ids=ids.data_ptr()) == -1 and look(ids=ids.data_ptr() + 2, n=2) == -1
    assert look(out=W[:120].view(6, 20)) == -1                        # written and read
    assert look(ids=ids.data_ptr(), n=-1, out=out.data_ptr()) == -1 and look(ids=16, n=2 ** 27 + 1, out=16) == -4

    nbytes = pkg.hsadmm_embedding_workspace(plan, 1, 6)
    ws = torch.zeros(nbytes + 256, dtype=torch.uint8, device=DEV)

    def back(layer=1, ids=ids, dY=out, G=G, workspace=ws, **more):
        return pkg.hsadmm_embedding_gradient(plan, layer, ids, dY, G, workspace, check=False, **more)

    assert back() == 0
    assert back(layer=7) == -1 and back(layer=2, dY=16) == -4 and back(type=3) == -4 and back(index_bits=1) == -4
    assert back(workspace_bytes=nbytes - 1) == -2 and back(workspace=ws[16:]) == -1 and back(workspace=None, workspace_bytes=nbytes) == -1
    assert back(G=None) == -1 and back(G=W[1:]) == -1 and back(dY=G[:120].view(6, 20)) == -1 and back(dY=None) == -1
    assert back(dY=out[:1].expand(6, 20)) == -1

    def drop_(X=out, Y=None, p=0.1, seed=1, call=1, **more):
        return pkg.hsadmm_dropout(plan, X, torch.zeros_like(out) if Y is None else Y, p, seed, call, check=False, **more)

    assert drop_() == 0
    assert drop_(p=1.0) == -1 and drop_(p=-0.1) == -1 and drop_(p=float("nan")) == -1 and drop_(type=9) == -4
    assert drop_(X=out.half()) == -1 and drop_(Y=out[:5]) == -1 and drop_(residual=out[:5]) == -1
    wide = torch.zeros((6, 30), device=DEV)
    assert drop_(X=wide[:, :20], Y=wide[:, 4:24]) == -1               # overlaps in part
    assert drop_(X=wide[:, :20], Y=wide[:, :20]) == 0
    assert drop_(residual=wide[:, :20], Y=wide[:, 4:24]) == -1
    assert drop_(X=8) == -1                                           # no rows, no width
    assert drop_(call_device=torch.zeros(1, dtype=torch.int32, device=DEV)) == -1
    empty = torch.zeros((0, 20), device=DEV)
    assert drop_(X=empty, Y=empty) == 0
    torch.cuda.synchronize()


def test_tensors_elsewhere_are_refused():
    plan = table(20, 30)
    W, ids, out = torch.zeros(plan.arena_elems, device=DEV), torch.zeros(6, dtype=torch.int32, device=DEV), torch.zeros((6, 20), device=DEV)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    cpu = lambda t: t.cpu()                                           # noqa: E731
    assert pkg.hsadmm_embedding(plan, 1, cpu(W), ids, out, check=False) == -1
    assert pkg.hsadmm_embedding(plan, 1, W, cpu(ids), out, check=False) == -1
    assert pkg.hsadmm_embedding_gradient(plan, 1, ids, cpu(out), W, ws, check=False) == -1
    assert pkg.hsadmm_embedding_gradient(plan, 1, ids, out, W, cpu(ws), check=False) == -1
    assert pkg.hsadmm_dropout(plan, out, cpu(out), 0.5, 1, 1, check=False) == -1
    loss = torch.zeros(6, device=DEV)
    assert pkg.hsadmm_softmax_loss(plan, 1, W, out, ids, workspace=ws, loss=cpu(loss), check=False) == -1
    with pytest.raises(pkg.HsadmmError, match="device"):
        pkg.hsadmm_embedding(plan, 1, W, ids, cpu(out))


@pytest.mark.parametrize("kind,n,D,V", [(F32, 5, 3, 9), (BF16, 300, 65, 400), (F16, 5000, 24, 3000)])
def test_addresses_stand_for_rows_without_gaps(kind, n, D, V):
    """Integer addresses in the place of tensors give what the tensors give."""
    gen = torch.Generator().manual_seed(5)
    plan, dtype = table(D, V), ref.TYPES[kind]
    W = torch.randn(plan.arena_elems, generator=gen).to(dtype).to(DEV)
    ids, x = tokens(n, V, gen, "common", 32), torch.randn((n, D), generator=gen).to(dtype).to(DEV)
    ws = torch.zeros(max(pkg.hsadmm_embedding_workspace(plan, 1, n), pkg.hsadmm_softmax_loss_workspace(plan, 1, n, kind)), dtype=torch.uint8, device=DEV)
    both = []
    for at in (lambda t: t, lambda t: t.data_ptr()):
        y, G, dX, total = torch.zeros_like(x), torch.zeros_like(W), torch.zeros_like(x), torch.zeros(2, device=DEV)
        pkg.hsadmm_embedding(plan, 1, at(W), at(ids), at(y), type=kind, n=n)
        pkg.hsadmm_softmax_loss(plan, 1, at(W), at(x), at(ids), workspace=at(ws), workspace_bytes=ws.numel(), total=at(total), dX=at(dX), G=at(G),
                                type=kind, n=n)
        pkg.hsadmm_embedding_gradient(plan, 1, at(ids), at(x), at(G), at(ws), workspace_bytes=ws.numel(), type=kind, n=n, accumulate=True)
        z = torch.zeros_like(x)
        pkg.hsadmm_dropout(plan, at(x), at(z), 0.5, 1, 2, type=kind, rows=n, width=D, residual=at(y))
        torch.cuda.synchronize()
        both.append((y, G, dX, total, z))
    for a, b in zip(*both):
        assert torch.equal(a, b)


def test_the_largest_offsets():
    """A layer that begins behind 2^31 elements of its arena, rows whose offsets pass 32 bits in bytes and in elements."""
    D, V, off = 2048, 3, 2 ** 31 + 8
    plan = pkg.Plan({"elem_off": [0, off], "c_out": [1, V], "c_in": [8, D], "khw": [1, 1], "mode": [0, 0], "k": [1, V]})
    gen = torch.Generator().manual_seed(6)
    W = torch.zeros(plan.arena_elems, dtype=torch.bfloat16, device=DEV)
    w = W[off:].view(V, D)
    w.copy_(torch.randn((V, D), generator=gen).to(torch.bfloat16))
    n, pad = 1100, 2 ** 21 - D                                # (n rows of 2^21 elements: 2.3 G elements)
    big = torch.zeros((n, D + pad), dtype=torch.bfloat16, device=DEV)
    ids = torch.randint(0, V, (n,), generator=gen, dtype=torch.int32).to(DEV)
    pkg.hsadmm_embedding(plan, 1, W, ids, big[:, :D], type=BF16)
    ref.close(big[:, :D], *ref.embedding_reference(BF16, w, ids.long(), 1.0), "rows far apart")
    near = big[:, :D].contiguous()
    G = torch.zeros_like(W)
    ws = torch.zeros(max(pkg.hsadmm_embedding_workspace(plan, 1, n), pkg.hsadmm_softmax_loss_workspace(plan, 1, n, BF16)), dtype=torch.uint8, device=DEV)
    g = G[off:].view(V, D)
    for rows_ in (big[:, :D], near):
        pkg.hsadmm_embedding_gradient(plan, 1, ids, rows_, G, ws, type=BF16)
        value, bound = ref.embedding_gradient_reference(V, near, ids.long(), 1.0)
        ref.close(g, value, ref.rounded(BF16, value, bound), "G")
    totals = [torch.zeros(2, device=DEV) for _ in range(2)]
    outs = []
    # (a row of W against itself has a logit of about 2048, so its own label a softmax of 1 and no gradient at all: the next one)
    labels = (ids + 1) % V
    for rows_, total in zip((big[:, :D], near), totals):
        pkg.hsadmm_softmax_loss(plan, 1, W, rows_, labels, workspace=ws, total=total, G=G, type=BF16)
        outs.append(g.clone())
    assert torch.equal(*totals) and torch.equal(*outs) and outs[0].abs().max() > 0
    y = torch.zeros_like(near)
    pkg.hsadmm_dropout(plan, big[:, :D], y, 0.5, 3, 4, type=BF16)
    z = torch.zeros_like(near)
    pkg.hsadmm_dropout(plan, near, z, 0.5, 3, 4, type=BF16)
    assert torch.equal(y, z)


def test_dropout_beyond_two_to_the_thirty_two_elements():
    """The element's number is counted in 64 bits: its last groups against the generator."""
    n = 2 ** 32 + 1000
    plan, x = table(4, 4), torch.ones((1, n), dtype=torch.float16, device=DEV)
    if n > 2 ** 31:                                           # (a row is at most 2^31 - 1 wide: as rows of a power of two)
        x = x[:, :2 ** 32].view(2 ** 12, 2 ** 20)
    y = x
    drop(plan, F16, x, y, 0.5, 21, 22)
    last = y.view(-1)[-5003:]
    kept, factor = ref.dropout_kept(5003, 0.5, 21, 22, first=y.numel() - 5003)
    assert torch.equal(last.cpu(), torch.from_numpy(kept * factor).half())
