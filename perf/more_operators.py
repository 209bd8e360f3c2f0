"""What the speed of the operators around the dense-document layer is measured on: what it is trained by and
how it is served.

    loss      softmax cross entropy of documents against a map's units (or any large set of classes), without
              keeping the scores, and its gradients; the scores are som_product's, so that squared distances to a
              codebook are one choice of alpha and bias
    quantise  dense rows or weights into 8 bits (E4M3) with a factor for each block of 128
    blocks    the matrix product of such operands, with the epilogue of som_product
    ortho     an update of weights orthogonalised by Newton-Schulz steps

Formulas (sums, statistics and activations in 32 bits or more):

    loss      v = alpha x W + b;  lse_m = log sum_n exp v_mn;  loss_m = lse_m - v_m,label
    back      g = dloss_m (exp(v - lse_m) - [n = label_m]);  dx = alpha g W^T;  dW = alpha x^T g;  db_n = sum_m g
              (a label outside [0, N): loss 0, g 0)
    quantise  s = max |x| / 448 over a block of 1 x 128 or 128 x 128 (1 where that is 0);  q = x / s, rounded to E4M3
    blocks    pre = alpha sum_b sx_mb sw_nb sum_{k in block b} x_mk W_kn + bias_n;  y = act(pre) + res
    ortho     X = G / |G|;  each step A = X X^T, X = a X + (b A + c A A) X  (tall G: of its transpose)
"""

import math

import torch

own = False

E4M3_MAX = 448.0
BLOCK = 128
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
QUINTIC = (3.4445, -4.7750, 2.0315)

# multiply-adds of the largest listed loss, product and orthogonalisation step: no drawn case has more
LARGEST = 8192 * 4096 * 65536
LARGEST_BLOCKS = 8192 * 4096 * 16384
LARGEST_STEP = 4096 ** 3


def listed():
    return [
        # One document against a 256 x 256 map (its surprise at the unit it was given): the units' bytes.
        dict(name="loss-1x2048x65536", op="loss", M=1, K=2048, N=65536, type="bf16", layout="unit", scores="dot",
             ignored=0.0, pad=0),
        # A batch of documents softly assigned to a 128 x 128 map in half precision: squared distances.
        dict(name="loss-4096x2048x16384", op="loss", M=4096, K=2048, N=16384, type="f16", layout="feature",
             scores="distance", ignored=0.0, pad=64),
        # The largest: a training batch against 65,536 classes.
        dict(name="loss-8192x4096x65536", op="loss", M=8192, K=4096, N=65536, type="bf16", layout="unit", scores="dot",
             ignored=0.1, pad=0),
        # Ragged everything, a third of the documents without a label.
        dict(name="lossback-1001x500x777", op="loss_back", M=1001, K=500, N=777, type="f16", layout="feature",
             scores="distance", ignored=0.33, pad=3),
        # The gradients of a training batch against a 256 x 256 map.
        dict(name="lossback-8192x2048x65536", op="loss_back", M=8192, K=2048, N=65536, type="bf16", layout="unit",
             scores="dot", ignored=0.1, pad=0),
        # Ragged rows of a wider array into 8 bits.
        dict(name="quantise-4999x1023", op="quantise", rows=4999, cols=1023, type="f16", block_rows=1, transpose=False,
             pad=6),
        # The gradient of a large batch, transposed for the weights' gradient.
        dict(name="quantise-16384x8192-t", op="quantise", rows=16384, cols=8192, type="bf16", block_rows=1,
             transpose=True, pad=0),
        # One document's state served in 8 bits.
        dict(name="blocks-1x4096x4096", op="blocks", M=1, K=4096, N=4096, w_rows=128, out="bf16", act="silu", bias=True,
             residual=True, alpha=1.0, pad=0),
        # A few documents, odd sizes.
        dict(name="blocks-37x8191x2047", op="blocks", M=37, K=8191, N=2047, w_rows=128, out="f16", act="none", bias=True,
             residual=True, alpha=1.0, pad=0),
        # A large batch through a wide projection in 8 bits.
        dict(name="blocks-8192x4096x16384", op="blocks", M=8192, K=4096, N=16384, w_rows=128, out="bf16", act="gelu",
             bias=True, residual=False, alpha=1.0, pad=0),
        # The update of a small projection: a chain of small products.
        dict(name="ortho-1024x512", op="ortho", rows=1024, cols=512, type="f32", steps=5, pad=0),
        # The update of a large square projection.
        dict(name="ortho-4096x4096", op="ortho", rows=4096, cols=4096, type="bf16", steps=5, pad=0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, odd=1 / 3):
    """Log-uniform in [lo, hi]: an odd number, or (mostly) 1, 1.25 or 1.75 times a power of two."""
    n = _log_uniform(rng, lo, hi)
    if n < 64 or rng.random() < odd:
        return min(n | 1, hi)
    return max(v for k in range(6, 18) for v in (1 << k, 5 << k - 2, 7 << k - 2) if v <= n)


def draw(rng):
    op = rng.choice(["loss", "loss", "loss_back", "loss_back", "quantise", "blocks", "blocks", "ortho"])
    pad = rng.choice([0, 0, 0, 8, 64, 1])
    if op in ("loss", "loss_back"):
        K, N = _size(rng, 64, 8192), _size(rng, 64, 131072)
        most = LARGEST // 2 if op == "loss_back" else LARGEST
        return dict(op=op, M=_size(rng, 1, min(16384, most // (K * N))), K=K, N=N,
                    type=rng.choice(["bf16", "bf16", "f16"]), layout=rng.choice(["feature", "unit"]),
                    scores=rng.choice(["dot", "dot", "distance"]), ignored=rng.choice([0.0, 0.1, 0.5]), pad=pad)
    if op == "quantise":
        cols = _size(rng, 64, 16384)
        return dict(op=op, rows=_size(rng, 1, min(65536, 16384 * 8192 // cols)), cols=cols,
                    type=rng.choice(["bf16", "bf16", "f16", "f32"]), block_rows=rng.choice([1, 1, 128]),
                    transpose=rng.random() < 0.4, pad=pad)
    if op == "blocks":
        K, N = _size(rng, 64, 16384), _size(rng, 64, 16384)
        return dict(op=op, M=_size(rng, 1, min(16384, LARGEST_BLOCKS // (K * N))), K=K, N=N,
                    w_rows=rng.choice([128, 128, 1]), out=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), bias=rng.random() < 0.6,
                    residual=rng.random() < 0.4, alpha=rng.choice([1.0, 1.0, -2.0]), pad=rng.choice([0, 0, 16, 1]))
    short = _size(rng, 128, 4096)
    long = max(short, _size(rng, 128, min(16384, LARGEST_STEP // (short * short))))
    rows, cols = (short, long) if rng.random() < 0.5 else (long, short)
    return dict(op=op, rows=rows, cols=cols, type=rng.choice(["f32", "bf16", "f16"]), steps=rng.choice([3, 4, 5, 5, 6]),
                pad=pad)


def _rows(g, rows, cols, dtype, pad=0, scale=None, spread=1.0):
    """Random rows in a wider array, as a view of `cols` columns; `scale`: one factor per column."""
    wide = torch.empty((rows, cols + pad), dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // max(1, cols + pad))
    for a in range(0, rows, step):
        b = min(rows, a + step)
        part = torch.randn((b - a, cols + pad), generator=g, device="cuda") * spread
        if scale is not None:
            part[:, :cols] *= scale
        wide[a:b] = part.to(dtype)
    return wide[:, :cols]


def _blocked(t, block_rows):
    """(codes, factors, values that the codes stand for) of a matrix in blocks, made block by block of rows."""
    rows, cols = t.shape
    kb = -(-cols // BLOCK)
    full = torch.zeros((-(-rows // block_rows) * block_rows, kb * BLOCK), device=t.device)
    full[:rows, :cols] = t.float()
    full = full.view(-1, block_rows, kb, BLOCK)
    scale = full.abs().amax((1, 3)) / E4M3_MAX
    scale = torch.where(scale > 0, scale, torch.ones_like(scale))
    q = (full / scale[:, None, :, None]).to(torch.float8_e4m3fn).view(-1, kb * BLOCK)[:rows, :cols]
    return q, scale


def _padded(q, pad):
    """The same rows in a wider array, as a view."""
    wide = torch.zeros((q.shape[0], q.shape[1] + pad), dtype=torch.uint8, device="cuda").view(q.dtype)
    wide[:, :q.shape[1]] = q
    return wide[:, :q.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    c, op, pad = case, case["op"], case["pad"]
    st = dict(case=dict(case))
    if op in ("loss", "loss_back"):
        M, K, N, dt = c["M"], c["K"], c["N"], TYPES[c["type"]]
        label = torch.randint(0, N, (M,), generator=g, device="cuda")
        if c["scores"] == "dot":      # weights of an output layer; documents lean to their class
            Wu = _rows(g, N, K, dt, spread=2.0 * K ** -0.5)
            x = torch.randn((M, K), generator=g, device="cuda") + 0.5 * Wu[label].float()
            bias = 0.1 * torch.randn(N, generator=g, device="cuda")
            st["alpha"] = 1.0
        else:                         # a codebook; documents near their unit, scores -t |x - w|^2 but for |x|^2
            Wu = torch.rand((N, K), generator=g, device="cuda").to(dt)
            x = Wu[label].float() + 0.3 * torch.randn((M, K), generator=g, device="cuda")
            t = 16.0 / K
            bias = -t * (Wu.float() ** 2).sum(1)
            st["alpha"] = 2.0 * t
        Wm = Wu if c["layout"] == "unit" else Wu.t()
        W = torch.empty((Wm.shape[0], Wm.shape[1] + pad), dtype=dt, device="cuda")[:, :Wm.shape[1]]
        W.copy_(Wm)
        st["W"] = W.t() if c["layout"] == "unit" else W
        st["x"] = torch.empty((M, K + pad), dtype=dt, device="cuda")[:, :K]
        st["x"].copy_(x)
        st["bias"] = bias
        label[torch.rand(M, generator=g, device="cuda") < c["ignored"]] = -1
        st["labels"] = label.int()
        if op == "loss_back":
            st["dloss"] = (0.5 + torch.rand(M, generator=g, device="cuda")) / M
            v = _scores(st)           # what the forward pass has returned
            st["lse"] = torch.logsumexp(v, 1)
    elif op == "quantise":
        col = torch.exp(0.5 * torch.randn(c["cols"], generator=g, device="cuda"))
        col[torch.randint(0, c["cols"], (max(1, c["cols"] // 512),), generator=g, device="cuda")] *= 20.0
        st["x"] = _rows(g, c["rows"], c["cols"], TYPES[c["type"]], pad, col)
    elif op == "blocks":
        M, K, N = c["M"], c["K"], c["N"]
        col = torch.exp(0.5 * torch.randn(K, generator=g, device="cuda"))
        x, st["sx"] = _blocked(_rows(g, M, K, torch.bfloat16, 0, col), 1)
        W, st["sw"] = _blocked(_rows(g, N, K, torch.bfloat16, spread=K ** -0.5), c["w_rows"])
        st["sx"] = st["sx"].t().contiguous().t()         # the factors of one block of k lie together
        st["x"], st["W"] = _padded(x, pad), _padded(W, pad).t()
        st["bias"] = 0.1 * torch.randn(N, generator=g, device="cuda") if c["bias"] else None
        st["res"] = _rows(g, M, N, TYPES[c["out"]], pad) if c["residual"] else None
    else:
        # a gradient: noise, and a few directions of the whole batch
        rows, cols, r = c["rows"], c["cols"], 8
        a = torch.randn((rows, r), generator=g, device="cuda") * torch.linspace(1.0, 4.0, r, device="cuda")
        b = torch.randn((r, cols), generator=g, device="cuda")
        G = torch.randn((rows, cols), generator=g, device="cuda") + 0.3 * (a @ b)
        st["G"] = torch.empty((rows, cols + pad), dtype=TYPES[c["type"]], device="cuda")[:, :cols]
        st["G"].copy_(1e-3 * G)
    return st


# The plain forms.

def _act(name, v):
    if name == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if name == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    if name == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _scores(st):
    return st["alpha"] * (st["x"].float() @ st["W"].float()) + st["bias"]


def _values(q, scale, block_rows):
    """What codes in blocks stand for, in 32 bits."""
    wide = scale.repeat_interleave(BLOCK, 1)[:, :q.shape[1]]
    return q.float() * wide.repeat_interleave(block_rows, 0)[:q.shape[0]]


def _plain(st):
    c, op = st["case"], st["case"]["op"]
    if op in ("loss", "loss_back"):
        v = _scores(st)
        some = st["labels"] >= 0
        label = torch.where(some, st["labels"], torch.zeros_like(st["labels"])).long()
        if op == "loss":
            most = v.amax(1)
            lse = most + torch.log(torch.exp(v - most[:, None]).sum(1))
            loss = lse - v.gather(1, label[:, None])[:, 0]
            return {"loss": torch.where(some, loss, torch.zeros_like(loss)), "lse": lse}
        g = torch.exp(v - st["lse"][:, None])
        g.scatter_add_(1, label[:, None], torch.full_like(label[:, None], -1.0, dtype=torch.float32))
        g *= torch.where(some, st["dloss"], torch.zeros_like(st["dloss"]))[:, None]
        dt = st["x"].dtype
        dx = st["alpha"] * (g @ st["W"].float().t())
        if c["layout"] == "unit":
            dW = (st["alpha"] * (g.t() @ st["x"].float())).to(dt).t()
        else:
            dW = (st["alpha"] * (st["x"].float().t() @ g)).to(dt)
        return {"dx": dx.to(dt), "dW": dW, "dbias": g.sum(0)}
    if op == "quantise":
        q, scale = _blocked(st["x"].t() if c["transpose"] else st["x"], c["block_rows"])
        return {"q": q, "scale": scale}
    if op == "blocks":
        pre = c["alpha"] * (_values(st["x"], st["sx"], 1) @ _values(st["W"].t(), st["sw"], c["w_rows"]).t())
        if c["bias"]:
            pre = pre + st["bias"]
        y = _act(c["act"], pre)
        if c["residual"]:
            y = y + st["res"].float()
        return {"y": y.to(TYPES[c["out"]])}
    G = st["G"].float()
    X = G.t() if c["rows"] > c["cols"] else G
    X = X / torch.sqrt((X * X).sum())
    for _ in range(c["steps"]):
        A = X @ X.t()
        X = QUINTIC[0] * X + (QUINTIC[1] * A + QUINTIC[2] * (A @ A)) @ X
    return {"y": (X.t() if c["rows"] > c["cols"] else X).to(torch.bfloat16)}


def _own(st):
    import paper_2609_05138_amd as som
    c, op = st["case"], st["case"]["op"]
    if op == "loss":
        loss, lse = som.som_cross_entropy(st["x"], st["W"], st["labels"], bias=st["bias"], alpha=st["alpha"])
        return {"loss": loss, "lse": lse}
    if op == "loss_back":
        dx, dW, dbias = som.som_cross_entropy_backward(st["dloss"], st["x"], st["W"], st["labels"], st["lse"],
                                                       bias=st["bias"], alpha=st["alpha"])
        return {"dx": dx, "dW": dW, "dbias": dbias}
    if op == "quantise":
        q, scale = som.som_quantise(st["x"], block_rows=c["block_rows"], transpose=c["transpose"])
        return {"q": q, "scale": scale}
    if op == "blocks":
        return {"y": som.som_product_blocks(st["x"], st["sx"], st["W"], st["sw"], bias=st["bias"], act=c["act"],
                                            residual=st["res"], alpha=c["alpha"], dtype=TYPES[c["out"]])}
    return {"y": som.som_orthogonalise(st["G"], steps=c["steps"], coefficients=QUINTIC)}


def run(st):
    return _own(st) if own else _plain(st)


def work(case):
    c, op = case, case["op"]
    if op in ("loss", "loss_back"):
        M, K, N, t = c["M"], c["K"], c["N"], BYTES[c["type"]]
        once = (M * K + K * N) * t + 4 * N + 4 * M
        if op == "loss":
            return {"bytes": once + 8 * M, "flops": 2 * M * K * N}
        return {"bytes": once + 8 * M + (M * K + K * N) * t + 4 * N, "flops": 6 * M * K * N}
    if op == "quantise":
        n = c["rows"] * c["cols"]
        blocks = -(-n // (BLOCK * c["block_rows"]))
        return {"bytes": n * (BYTES[c["type"]] + 1) + 4 * blocks, "flops": 3 * n}
    if op == "blocks":
        M, K, N, o = c["M"], c["K"], c["N"], BYTES[c["out"]]
        kb = -(-K // BLOCK)
        b = M * K + K * N + 4 * kb * (M + -(-N // c["w_rows"])) + M * N * o * (1 + c["residual"]) + 4 * N * c["bias"]
        return {"bytes": b, "flops": 2 * M * K * N}
    m, n = sorted((c["rows"], c["cols"]))
    # of the two symmetric products one half
    return {"bytes": m * n * (BYTES[c["type"]] + 2), "flops": c["steps"] * (3 * m * m * n + m * m * m)}


# The definitions in 64 bits.

def exact(case, seed):
    st = prepare(case, seed)
    c, op = case, case["op"]
    if op in ("loss", "loss_back"):
        x, W = st["x"].double(), st["W"].double().contiguous()
        v = torch.mm(x, W)
        v *= st["alpha"]
        v += st["bias"].double()
        has = (st["labels"] >= 0).double()
        label = st["labels"].long().clamp(min=0)
        rows = torch.arange(c["M"], device="cuda")
        if op == "loss":
            lse = torch.logsumexp(v, 1)
            return {"loss": (lse - v[rows, label]) * has, "lse": lse}
        v -= st["lse"].double()[:, None]
        v.exp_()
        v[rows, label] -= 1.0
        v *= (st["dloss"].double() * has)[:, None]
        return {"dx": st["alpha"] * torch.mm(v, W.t().contiguous()),
                "dW": st["alpha"] * torch.mm(x.t().contiguous(), v), "dbias": v.sum(0)}
    if op == "quantise":
        x = st["x"].double()
        x = (x.t() if c["transpose"] else x).contiguous()
        r, k, br = x.shape[0], x.shape[1], c["block_rows"]
        R, KB = -(-r // br), -(-k // BLOCK)
        amax = torch.zeros((R * br, KB * BLOCK), dtype=torch.float64, device="cuda")
        amax[:r, :k] = x.abs()
        scale = amax.view(R, br, KB, BLOCK).amax(3).amax(1) / E4M3_MAX
        row, col = torch.arange(r, device="cuda") // br, torch.arange(k, device="cuda") // BLOCK
        return {"q": x / scale[row][:, col], "scale": scale}
    if op == "blocks":
        M, K, N = c["M"], c["K"], c["N"]
        col = torch.arange(K, device="cuda") // BLOCK
        unit = torch.arange(N, device="cuda") // c["w_rows"]
        a = st["x"].double() * st["sx"].double()[:, col]
        b = st["W"].t().double() * st["sw"].double()[unit][:, col]
        v = c["alpha"] * torch.mm(a, b.t().contiguous())
        if c["bias"]:
            v += st["bias"].double()
        y = {"none": lambda: v, "relu": lambda: v.clamp(min=0.0), "silu": lambda: v * torch.sigmoid(v),
             "gelu": lambda: v * torch.special.ndtr(v),
             "gelu_tanh": lambda: v * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))}[c["act"]]()
        return {"y": y + st["res"].double() if c["residual"] else y}
    G = st["G"].double()
    tall = c["rows"] > c["cols"]
    X = G / torch.linalg.vector_norm(G)
    a, b, k = QUINTIC
    for _ in range(c["steps"]):
        # the same polynomial from the other side where that is shorter
        S = torch.mm(X.t().contiguous(), X) if tall else torch.mm(X, X.t().contiguous())
        S = b * S + k * torch.mm(S, S)
        X = a * X + (torch.mm(X, S) if tall else torch.mm(S, X))
    return {"y": X}
