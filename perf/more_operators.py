"""The two ends of a language model's local training, beside the network's layers that the other calls take: what turns tokens
into activations and the last layer's products into a loss, with the gradients that hsadmm_gradient_norms and hsadmm_adamw read.

A case is one call on one [V, D] layer of a table (V rows of D weights, one row a class or a token):

  loss        hsadmm_softmax_loss: softmax cross entropy of x W^T against labels: every row's loss and the logarithm of its sum
              of exponentials, the mean loss and the number of targets; with the gradients of x and W (`gradients`) or without.
              A label outside [0, V) is no target: its row has loss 0, logarithm 0 and no gradient.
  embed       hsadmm_embedding: rows of W times a scale, zeros for a token outside [0, V)
  embed_grad  hsadmm_embedding_gradient: every row of W receives the scaled sum of its tokens' gradients (0 without tokens)
  dropout     hsadmm_dropout: y = x / (1 - p) where the element's random number says so, else 0; plus a residual

Random numbers of dropout.  Element i (row-major, counted without strides) takes 16 bits of Philox4x32-10 (Salmon, Moraes, Dror
and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): counter (i / 8 as 64 bits, call as 64 bits), key the seed's 64
bits; of the four words it gives, the halves in ascending order belong to elements 8 (i / 8) ... + 7.  An element stays where its
16 bits are at least t = round(65536 p), and the kept ones are multiplied by 65536 / (65536 - t).
"""
import math

import numpy as np
import torch

own = False

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
SIZES = {"float32": 4, "bfloat16": 2, "float16": 2}
PHILOX_M, PHILOX_W = (0xD2511F53, 0xCD9E8D57), (0x9E3779B9, 0xBB67AE85)
LOW32 = 0xFFFFFFFF


# ------------------------------------------------------------------ cases

def listed():
    def loss(name, N, D, V, dtype, gradients, ignored=0.0, pad=0, scale=1.0):
        return {"name": name, "op": "loss", "N": N, "D": D, "V": V, "dtype": dtype, "gradients": gradients,
                "ignored": ignored, "pad": pad, "scale": scale}

    def embed(name, op, N, D, V, dtype, scale, ignored=0.0, pad=0):
        return {"name": name, "op": op, "N": N, "D": D, "V": V, "dtype": dtype, "scale": scale, "ignored": ignored, "pad": pad}

    def dropout(name, N, D, dtype, p, residual, pad=0):
        return {"name": name, "op": "dropout", "N": N, "D": D, "dtype": dtype, "p": p, "residual": residual, "pad": pad}

    return [
        # the smallest training batch: the last layer of a small CNN, where launches are all there is
        loss("loss_tiny", 32, 64, 10, "float32", True),
        # the benchmark's network: its classifier under a batch of images, fp32 as its arenas are
        loss("loss_resnet50", 256, 2048, 1000, "float32", True),
        # language modelling in mixed precision, a tenth of the batch is padding
        loss("loss_tokens", 4096, 2048, 32768, "bfloat16", True, ignored=0.1),
        # odd sizes everywhere, rows with a stride, half precision under loss scaling, prompts masked out
        loss("loss_ragged", 1537, 1441, 20011, "float16", True, ignored=0.4, pad=7, scale=1024.0),
        # the largest: more logits than are held at once
        loss("loss_wide", 8192, 4096, 65536, "bfloat16", True),
        # evaluation of a single token
        loss("loss_one", 1, 2048, 131072, "bfloat16", False),
        # the first layer for one token, and for a batch
        embed("embed_one", "embed", 1, 2048, 131072, "bfloat16", 1.0),
        embed("embed_batch", "embed", 32768, 2048, 131072, "bfloat16", 45.254834, ignored=0.05),
        # its gradient: a small odd layer, and a batch over a large vocabulary
        embed("embed_grad_ragged", "embed_grad", 777, 1001, 20011, "float32", 1.0, ignored=0.2, pad=3),
        embed("embed_grad_batch", "embed_grad", 32768, 2048, 131072, "bfloat16", 45.254834, ignored=0.05),
        # dropout of a small batch's activations, and of a large one's on their way into the residual stream
        dropout("dropout_small", 32, 512, "float32", 0.5, False),
        dropout("dropout_batch", 16384, 4096, "bfloat16", 0.1, True),
    ]


def draw(rng):
    """Any of the operators over its range: from one row to tens of thousands, odd sizes and padded rows among them."""
    def log(a, b):
        return int(round(a * (b / a) ** rng.random()))

    case = {"op": rng.choice(["loss", "loss", "loss", "embed", "embed_grad", "embed_grad", "dropout"]),
            "dtype": rng.choice(["float32", "bfloat16", "bfloat16", "float16"])}
    if case["op"] == "loss":
        N, D, V = log(1, 8192), log(16, 4096), log(10, 65536)
        if rng.random() < 0.5:
            D = max(8, D - D % 8)
        if case["dtype"] == "float32":
            N, V = min(N, 2048), min(V, 32768)
        case.update(N=N, D=D, V=V, gradients=rng.random() < 0.75, scale=1024.0 if case["dtype"] == "float16" else 1.0)
    elif case["op"] == "dropout":
        case.update(N=log(1, 16384), D=log(8, 4096), p=round(rng.uniform(0.02, 0.6), 3), residual=rng.random() < 0.5)
    else:
        case.update(N=log(1, 32768), D=log(8, 4096), V=log(10, 65536), scale=round(rng.uniform(0.5, 50.0), 3))
    if case["op"] != "dropout":
        case["ignored"] = rng.choice([0.0, 0.1, round(rng.random() * 0.9, 3)])
    case["pad"] = rng.choice([0, 0, 8, rng.randint(1, 9)])
    return case


# ------------------------------------------------------------------ what a program has in hand

def _rows(gen, N, D, pad, dtype, sigma=1.0):
    """N rows of D numbers that lie D + pad elements apart."""
    return torch.randn((N, D + pad), generator=gen, device=gen.device).mul_(sigma).to(dtype)[:, :D]


def _tokens(gen, N, V, ignored):
    """Tokens as they occur: the r-th most frequent one about 1 / r as often as the first; some rows have none."""
    t = (float(V) ** torch.rand(N, generator=gen, device=gen.device, dtype=torch.float64)).long() - 1
    t = t.clamp_(0, V - 1)
    return torch.where(torch.rand(N, generator=gen, device=gen.device) < ignored, torch.full_like(t, -100), t)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(int(seed))
    N, D, dtype = case["N"], case["D"], TYPES[case["dtype"]]
    if case["op"] == "dropout":
        x = {"X": _rows(gen, N, D, case["pad"], dtype)}
        if case["residual"]:
            x["R"] = _rows(gen, N, D, case["pad"], dtype, 3.0)
        return x
    V = case["V"]
    x = {"ids": _tokens(gen, N, V, case["ignored"])}
    if case["op"] != "embed_grad":
        x["W"] = (torch.randn((V, D), generator=gen, device=gen.device) * D ** -0.5).to(dtype)
    if case["op"] == "loss":
        x["X"] = _rows(gen, N, D, case["pad"], dtype, 2.0)
    if case["op"] == "embed_grad":
        x["dY"] = _rows(gen, N, D, case["pad"], dtype, 1e-2)
    return x


def prepare(case, seed):
    s = {"case": case, "dtype": TYPES[case["dtype"]], "seed": (int(seed) * 0x9E3779B97F4A7C15 + 12345) & (2 ** 64 - 1), "call": 3 + int(seed)}
    s.update(_inputs(case, seed))
    if not own:
        return s
    import paper_2512_14628_amd as hs
    op, N, D, dev = case["op"], case["N"], case["D"], torch.device("cuda:0")
    V = case.get("V", 1)
    s["hs"], s["type"] = hs, {"float32": hs.TYPE_F32, "bfloat16": hs.TYPE_BF16, "float16": hs.TYPE_F16}[case["dtype"]]
    s["plan"] = plan = hs.Plan({"elem_off": [0], "c_out": [V], "c_in": [D], "khw": [1], "mode": [hs.MODE_NONE], "k": [V]})

    def rows(N):
        return torch.zeros((N, D + case["pad"]), dtype=s["dtype"], device=dev)[:, :D]

    nbytes = 0
    if op in ("dropout", "embed"):
        s["Y"] = rows(N)
    if op == "embed_grad" or (op == "loss" and case["gradients"]):
        s["G"] = torch.zeros((V, D), dtype=s["dtype"], device=dev)
    if op == "embed_grad":
        nbytes = hs.hsadmm_embedding_workspace(plan, 0, N)
    if op == "loss":
        s["loss"], s["lse"], s["total"] = torch.zeros(N, device=dev), torch.zeros(N, device=dev), torch.zeros(2, device=dev)
        if case["gradients"]:
            s["dX"] = rows(N)
        nbytes = hs.hsadmm_softmax_loss_workspace(plan, 0, N, s["type"], case["gradients"])
    s["ws"] = torch.zeros(max(nbytes, 256), dtype=torch.uint8, device=dev)
    return s


# ------------------------------------------------------------------ the operators in plain form

def _loss(s):
    W, X, ids = s["W"].float(), s["X"].float(), s["ids"]
    V = W.shape[0]
    target = (ids >= 0) & (ids < V)
    at = torch.where(target, ids, 0)[:, None]
    logits = X @ W.T
    top = logits.amax(1, keepdim=True)
    picked = logits.gather(1, at)
    e = logits.sub_(top).exp_()
    total = e.sum(1, keepdim=True)
    loss = torch.where(target, (top + total.log() - picked)[:, 0], 0.0)
    lse = (top + total.log())[:, 0]
    count = target.sum().clamp(min=1)
    out = {"loss": loss, "lse": torch.where(target, lse, 0.0), "total": torch.stack((loss.double().sum() / count, target.double().sum())).float()}
    if s["case"]["gradients"]:
        p = e.div_(total)
        p.scatter_add_(1, at, torch.full_like(picked, -1.0))
        p.masked_fill_(~target[:, None], 0.0)
        g = s["case"]["scale"] / count
        out["dX"] = ((p @ W) * g).to(s["dtype"])
        out["G"] = ((p.T @ X) * g).to(s["dtype"])
    return out


def _embed(s):
    ids, V = s["ids"], s["W"].shape[0]
    token = (ids >= 0) & (ids < V)
    y = s["W"][torch.where(token, ids, 0)].float() * s["case"]["scale"]
    return torch.where(token[:, None], y, 0.0).to(s["dtype"])


def _embed_grad(s):
    ids, V = s["ids"], s["case"]["V"]
    token = (ids >= 0) & (ids < V)
    total = torch.zeros((V + 1, s["case"]["D"]), device=ids.device)
    total.index_add_(0, torch.where(token, ids, V), s["dY"].float())
    return (total[:V] * s["case"]["scale"]).to(s["dtype"])


def _philox(groups, call, seed, device):
    """Philox4x32-10 of the counters (0 .. groups - 1, call): [groups, 4] words."""
    g = torch.arange(groups, dtype=torch.int64, device=device)
    c = [g & LOW32, g >> 32, torch.full_like(g, call & LOW32), torch.full_like(g, call >> 32)]
    k = [seed & LOW32, seed >> 32]
    for _ in range(10):
        # (the products' 64 bits, as two's complement: the shift's sign bits are cut off)
        a, b = c[0] * PHILOX_M[0], c[2] * PHILOX_M[1]
        c = [((b >> 32) & LOW32) ^ c[1] ^ k[0], b & LOW32, ((a >> 32) & LOW32) ^ c[3] ^ k[1], a & LOW32]
        k = [(k[0] + PHILOX_W[0]) & LOW32, (k[1] + PHILOX_W[1]) & LOW32]
    return torch.stack(c, 1)


def _dropout(s):
    X, case = s["X"], s["case"]
    n = X.numel()
    words = _philox(-(-n // 8), s["call"], s["seed"], X.device)
    bits = torch.stack((words & 0xFFFF, words >> 16), 2).view(-1)[:n].view(X.shape)
    t = int(math.floor(65536 * case["p"] + 0.5))
    y = torch.where(bits >= t, X.float() * (65536 / (65536 - t)), 0.0)
    return ((y + s["R"].float()) if case["residual"] else y).to(s["dtype"])


def run(s):
    op, case = s["case"]["op"], s["case"]
    if not own:
        return {"loss": _loss, "embed": _embed, "embed_grad": _embed_grad, "dropout": _dropout}[op](s)
    hs, plan, kind = s["hs"], s["plan"], s["type"]
    if op == "loss":
        hs.hsadmm_softmax_loss(plan, 0, s["W"], s["X"], s["ids"], type=kind, index_bits=64, loss=s["loss"], lse=s["lse"],
                               total=s["total"], dX=s.get("dX"), G=s.get("G"), mean=True, scale=case["scale"], workspace=s["ws"])
        return {k: s[k] for k in ("loss", "lse", "total", "dX", "G") if k in s}
    if op == "embed":
        hs.hsadmm_embedding(plan, 0, s["W"], s["ids"], s["Y"], scale=case["scale"], type=kind, index_bits=64)
        return s["Y"]
    if op == "embed_grad":
        hs.hsadmm_embedding_gradient(plan, 0, s["ids"], s["dY"], s["G"], s["ws"], scale=case["scale"], type=kind, index_bits=64)
        return s["G"]
    hs.hsadmm_dropout(plan, s["X"], s["Y"], case["p"], s["seed"], s["call"], residual=s.get("R"), type=kind)
    return s["Y"]


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Each input read once and each output written once; of the table's rows those that the tokens name."""
    N, D, size = case["N"], case["D"], SIZES[case["dtype"]]
    if case["op"] == "dropout":
        return {"bytes": N * D * size * (3 if case["residual"] else 2), "flops": 2 * N * D}
    V, rows = case["V"], N * (1 - case["ignored"])
    if case["op"] == "embed":
        return {"bytes": 8 * N + size * D * (min(rows, V) + N), "flops": N * D}
    if case["op"] == "embed_grad":
        return {"bytes": 8 * N + size * D * (rows + V), "flops": rows * D + V * D}
    products = 3 if case["gradients"] else 1
    nbytes = size * D * (V + rows) + 12 * N + (size * D * (V + N) if case["gradients"] else 0)
    return {"bytes": nbytes, "flops": 2 * rows * V * D * products}


# ------------------------------------------------------------------ the same pass in 64 bits

def _exact_loss(case, x):
    f = torch.float64
    V, ids = case["V"], x["ids"]
    valid = ((ids >= 0) & (ids < V)).nonzero()[:, 0]
    W, X = x["W"].to(f), x["X"].to(f)[valid]
    logits = torch.mm(X, W.t())
    lse = torch.zeros(case["N"], dtype=f, device=ids.device)
    lse[valid] = torch.logsumexp(logits, dim=1)
    logp = torch.log_softmax(logits, dim=1)
    row = torch.arange(valid.numel(), device=ids.device)
    loss = torch.zeros(case["N"], dtype=f, device=ids.device)
    loss[valid] = -logp[row, ids[valid]]
    n = float(valid.numel())
    out = {"loss": loss, "lse": lse, "total": torch.stack((loss.sum() / max(1.0, n), loss.new_tensor(n)))}
    if case["gradients"]:
        p = logp.exp_()
        p[row, ids[valid]] -= 1.0
        p *= case["scale"] / max(1, valid.numel())
        out["dX"] = torch.zeros((case["N"], case["D"]), dtype=f, device=ids.device)
        out["dX"][valid] = torch.mm(p, W)
        out["G"] = torch.mm(p.t(), X)
    return out


def _exact_kept(case, seed, call):
    """Which elements stay, with numpy's 64-bit words."""
    n = case["N"] * case["D"]
    word = np.arange(-(-n // 8), dtype=np.uint64)
    low, half = np.uint64(LOW32), np.uint64(32)
    x0, x1 = word & low, word >> half
    x2, x3 = np.full_like(word, call % 2 ** 32), np.full_like(word, call // 2 ** 32)
    for r in range(10):
        k0, k1 = ((np.uint64((seed >> sh) % 2 ** 32 + r * w) & low) for sh, w in zip((0, 32), PHILOX_W))
        a, b = x0 * np.uint64(PHILOX_M[0]), x2 * np.uint64(PHILOX_M[1])
        x0, x1, x2, x3 = (b >> half) ^ x1 ^ k0, b & low, (a >> half) ^ x3 ^ k1, a & low
    halves = np.stack((x0, x1, x2, x3), 1).astype("<u4").view("<u2").reshape(-1)[:n]
    return halves.reshape(case["N"], case["D"]) >= math.floor(65536 * case["p"] + 0.5)


def exact(case, seed):
    """What `run` returns for these inputs, from the definitions in 64 bits."""
    x, f = _inputs(case, seed), torch.float64
    if case["op"] == "loss":
        return _exact_loss(case, x)
    if case["op"] == "dropout":
        s = (int(seed) * 0x9E3779B97F4A7C15 + 12345) & (2 ** 64 - 1)
        kept = torch.from_numpy(_exact_kept(case, s, 3 + int(seed))).to(x["X"].device)
        share = 1 - math.floor(65536 * case["p"] + 0.5) / 65536
        y = x["X"].to(f) / share * kept
        return y + x["R"].to(f) if case["residual"] else y
    V, ids = case["V"], x["ids"]
    named = ((ids >= 0) & (ids < V)).nonzero()[:, 0]
    if case["op"] == "embed":
        y = torch.zeros((case["N"], case["D"]), dtype=f, device=ids.device)
        y[named] = torch.index_select(x["W"], 0, ids[named]).to(f) * case["scale"]
        return y
    y = torch.zeros((V, case["D"]), dtype=f, device=ids.device)
    return y.index_add_(0, ids[named], x["dY"].to(f)[named]).mul_(case["scale"])
