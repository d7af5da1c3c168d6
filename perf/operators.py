"""Timed cases of the operators for training with little memory: the softmax
cross entropy over many classes that keeps no logits (``gcn_class_loss``), the
8-bit activation checkpoints and the backward pass that reads them
(``gcn_rows8_pack``, ``gcn_rows8_weight_grad``), and the product of 8-bit rows
with 8-bit weights, one scale for each block of 128 (``gcn_rows8_product``).

With ``own`` false, ``run`` computes a case in plain torch operations in 32
bits; with ``own`` true it makes the library's calls.  ``exact`` repeats a case
in float64.  Inputs are made on the GPU from the seed alone.

8-bit rows.  The row block x of 128 columns with the largest finite magnitude
a = m 2^k (1 <= m < 2) has the power-of-two scale 2^e, e = k - 8 where
m <= 1.75 and k - 7 above (448 is the largest e4m3 value), e within -126 ..
127; a block of zeros has e = 0.  It is held as q = e4m3(x 2^-e), round to
nearest even, a value other than zero keeping its sign (as +-2^-9 where it
would round to zero), a value that is not finite as NaN.  A scale is held as
the byte e + 127.  Weights have one scale for each block of 128 x 128.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 128
FLOAT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # a few labelled vertices of a many-class problem: the smallest training call of the head
        {"name": "loss_bf16_17x128_c1009", "op": "loss", "type": "bf16", "n": 17, "f": 128, "C": 1009, "grad": True,
         "bias": True},
        # a sampled subgraph with ten thousand classes, float32 throughout
        {"name": "loss_f32_2000x256_c10007", "op": "loss", "type": "f32", "n": 2000, "f": 256, "C": 10007,
         "grad": True, "bias": True},
        # evaluation: the loss and every row's loss, no gradient
        {"name": "loss_bf16_5003x600_c50021_eval", "op": "loss", "type": "bf16", "n": 5003, "f": 600, "C": 50021,
         "grad": False, "bias": False},
        # the largest head: 4.3 GB of bfloat16 logits, were they kept
        {"name": "loss_bf16_16384x1024_c131072", "op": "loss", "type": "bf16", "n": 16384, "f": 1024, "C": 131072,
         "grad": True, "bias": True},
        # one row through a wide layer: answering a single request
        {"name": "product_bf16_1x4096x4096", "op": "product", "type": "bf16", "n": 1, "K": 4096, "N": 4096,
         "bias": True, "relu": True, "transpose": False},
        # the Reddit-shaped first layer of the training loop: odd rows, 602 attributes
        {"name": "product_f32_6205x602x512", "op": "product", "type": "f32", "n": 6205, "K": 602, "N": 512,
         "bias": True, "relu": True, "transpose": False},
        # an input gradient on an ordinary subgraph: dZ W^T
        {"name": "product_bf16_8000x512x1024_t", "op": "product", "type": "bf16", "n": 8000, "K": 512, "N": 1024,
         "bias": False, "relu": False, "transpose": True},
        # the largest transform
        {"name": "product_bf16_16384x4096x8192", "op": "product", "type": "bf16", "n": 16384, "K": 4096, "N": 8192,
         "bias": True, "relu": True, "transpose": False},
        # a small subgraph's checkpoint (PPI attributes): the launch is what counts
        {"name": "pack_f32_2000x50", "op": "pack", "type": "f32", "n": 2000, "f": 50},
        # an inner layer's checkpoint at the largest subgraph
        {"name": "pack_bf16_65536x1024", "op": "pack", "type": "bf16", "n": 65536, "f": 1024},
        # the backward pass of a small layer, float32 gradients from above
        {"name": "weight_grad_f32_2003x300x128", "op": "weight_grad", "type": "f32", "n": 2003, "f": 300, "N": 128},
        # the backward pass of one branch of an inner layer at the largest subgraph
        {"name": "weight_grad_bf16_65536x1024x512", "op": "weight_grad", "type": "bf16", "n": 65536, "f": 1024,
         "N": 512},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Half of the widths are multiples of 64, as layers have them; the others are any."""
    w = _log_int(rng, lo, hi)
    return max(64, w // 64 * 64) if rng.random() < 0.5 and hi >= 64 else w


def draw(rng):
    op = rng.choice(["loss", "loss", "product", "product", "pack", "weight_grad", "weight_grad"])
    t = rng.choice(["f32", "bf16", "bf16"])
    if op == "loss":
        if t == "f32":    # float32 products cost several times as much
            n, f, C = _log_int(rng, 1, 4096), _width(rng, 16, 512), _log_int(rng, 3, 20000)
        else:
            n, f, C = _log_int(rng, 1, 16384), _width(rng, 16, 1024), _log_int(rng, 3, 131072)
        return {"op": op, "type": t, "n": n, "f": f, "C": C, "grad": rng.random() < 0.75, "bias": rng.random() < 0.5}
    if op == "product":
        transpose = rng.random() < 0.4
        return {"op": op, "type": t, "n": _log_int(rng, 1, 16384), "K": _width(rng, 16, 4096),
                "N": _width(rng, 16, 8192), "bias": not transpose and rng.random() < 0.7,
                "relu": not transpose and rng.random() < 0.7, "transpose": transpose}
    if op == "pack":
        return {"op": op, "type": t, "n": _log_int(rng, 1, 65536), "f": _width(rng, 16, 1024)}
    return {"op": op, "type": t, "n": _log_int(rng, 1, 65536), "f": _width(rng, 16, 1024),
            "N": _width(rng, 16, 512)}


# ------------------------------------------------------------------ 8-bit rows, plain
def _exponent(a):
    """e of a block whose largest finite magnitude is a (float32, any shape)."""
    m, k = torch.frexp(a)                        # a = m 2^k, 0.5 <= m < 1
    e = k - 9 + (m > 0.875).to(k.dtype)
    return torch.where(a == 0, torch.zeros_like(e), e).clamp(-126, 127)


def _power_of_two(k):
    """2^k in float32 (whole numbers k, -126 to 127), from its bits: exact everywhere."""
    return ((k.to(torch.int32) + 127) << 23).view(torch.float32)


def _held(x, e):
    """e4m3 of x 2^-e (float32 x, e of x's shape)."""
    q = (x * _power_of_two(-e)).to(torch.float8_e4m3fn).to(torch.float32)
    q = torch.where((q == 0) & (x != 0), torch.copysign(torch.full_like(x, 2.0 ** -9), x), q)
    return torch.where(torch.isfinite(x), q, torch.full_like(q, math.nan)).to(torch.float8_e4m3fn)


def _padded(x, multiple_r, multiple_c):
    r, c = x.shape
    return torch.nn.functional.pad(x, (0, -c % multiple_c, 0, -r % multiple_r))


def _pack_rows(x):
    """q [n x f] float8_e4m3fn and the scale bytes [n x ceil(f / 128)] of x."""
    n, f = x.shape
    x = _padded(x.to(torch.float32), 1, BLOCK).view(n, -1, BLOCK)
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(dim=2)
    e = _exponent(a)
    q = _held(x, e.unsqueeze(2).expand_as(x)).view(n, -1)[:, :f]
    return q, (e + 127).to(torch.uint8)


def _pack_weights(w):
    """q [K x N] float8_e4m3fn and the scale bytes [ceil(K / 128) x ceil(N / 128)] of w."""
    K, N = w.shape
    p = _padded(w.to(torch.float32), BLOCK, BLOCK)
    v = p.view(p.shape[0] // BLOCK, BLOCK, p.shape[1] // BLOCK, BLOCK)
    a = v.abs().amax(dim=(1, 3))
    e = _exponent(a)
    q = _held(v, e[:, None, :, None].expand_as(v)).reshape(p.shape)[:K, :N].contiguous()
    return q, (e + 127).to(torch.uint8)


def _values_rows(q, s):
    """What 8-bit rows stand for, in float32."""
    scale = _power_of_two(s.to(torch.int32) - 127)
    return q.to(torch.float32) * scale.repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _values_weights(q, s):
    scale = _power_of_two(s.to(torch.int32) - 127)
    scale = scale.repeat_interleave(BLOCK, 0)[:q.shape[0]].repeat_interleave(BLOCK, 1)[:, :q.shape[1]]
    return q.to(torch.float32) * scale


# ------------------------------------------------------------------ inputs
def _inputs(case, seed):
    """The operator's inputs as plain tensors."""
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)
    t = FLOAT[case["type"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    n = case["n"]
    if case["op"] == "loss":
        f, C = case["f"], case["C"]
        # activations after a ReLU; weights of a partly trained head (logits of
        # standard deviation about 2); one vertex in twenty has no label
        labels = torch.randint(0, C, (n,), generator=g, device=DEV, dtype=torch.int32)
        labels[torch.rand(n, generator=g, device=DEV) < 0.05] = -1
        if n > 1:
            labels[0] = C - 1
        return {"HL": torch.relu(normal(n, f)).to(t), "W": (normal(f, C) * (2.8 / math.sqrt(f))).to(t),
                "b": normal(C) * 0.5 if case["bias"] else None, "labels": labels}
    if case["op"] == "product":
        K, N = case["K"], case["N"]
        x = normal(n, K) * torch.exp(normal(n, 1))
        q, s = _pack_rows(x if case["transpose"] else torch.relu(x))
        w = normal(N, K) / math.sqrt(K) if case["transpose"] else normal(K, N) / math.sqrt(K)
        wq, ws = _pack_weights(w)
        # weights are kept in both orientations, for a layer's two directions
        return {"q": _laid_out(q), "s": s, "wq": _laid_out(wq), "wqT": _laid_out(wq.T), "ws": ws,
                "b": normal(N) * 0.1 if case["bias"] else None}
    if case["op"] == "pack":
        # a layer's output after the ReLU, rows of unlike sizes
        return {"X": (torch.relu(normal(n, case["f"])) * torch.exp(normal(n, 1))).to(t)}
    f, N = case["f"], case["N"]
    q, s = _pack_rows(torch.relu(normal(n, f)))
    yq, _ = _pack_rows(torch.relu(normal(n, N)))
    dY = (normal(n, N) * 1e-3 * torch.exp(normal(n, 1))).to(t)
    return {"q": _laid_out(q), "s": s, "yq": _laid_out(yq), "dY": dY}


def _laid_out(q):
    """8-bit values as they are kept: in rows of whole blocks, the columns past the last one zero."""
    rows, cols = q.shape
    kept = torch.zeros((rows, -(-cols // BLOCK) * BLOCK), dtype=torch.uint8, device=q.device)
    kept[:, :cols] = q.view(torch.uint8)
    return kept.view(torch.float8_e4m3fn)[:, :cols]


def prepare(case, seed):
    """The inputs, and the output buffers that a training program keeps; for
    the library its handles of the 8-bit operands and a workspace."""
    x = _inputs(case, seed)
    state = {"case": case, "in": x}
    if own:
        from paper_1810_11899_amd import binding as B
        state["B"], state["work"] = B, B.Workspace(DEV)
        t, n = FLOAT[case["type"]], case["n"]

        def empty(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=DEV)

        if case["op"] == "loss":
            state["loss"], state["rows"] = empty(1), empty(n)
            if case["grad"]:
                state["dHL"], state["dW"] = empty(n, case["f"], dtype=t), empty(case["f"], case["C"], dtype=t)
                state["db"] = empty(case["C"])
        elif case["op"] == "product":
            state["X8"] = B.Rows8.of(x["q"], x["s"])
            state["W8"] = B.Weights8.of(x["wq"], x["wqT"], x["ws"])
            state["Y"] = empty(n, case["N"], dtype=t)
        elif case["op"] == "pack":
            state["X8"] = B.Rows8(n, case["f"], DEV)
        else:
            state["X8"] = B.Rows8.of(x["q"], x["s"])
            state["dZ8"] = B.Rows8(n, case["N"], DEV)
            state["dW"], state["db"] = empty(case["f"], case["N"]), empty(case["N"])
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if own:
        return {"loss": _own_loss, "product": _own_product, "pack": _own_pack,
                "weight_grad": _own_weight_grad}[case["op"]](state, case)
    return {"loss": _plain_loss, "product": _plain_product, "pack": _plain_pack,
            "weight_grad": _plain_weight_grad}[case["op"]](state["in"], case)


def _own_loss(st, case):
    x = st["in"]
    st["B"].gcn_class_loss(x["HL"], x["W"], x["b"], x["labels"], st["loss"], st["work"], row_loss=st["rows"],
                           dHL=st.get("dHL"), dW_pred=st.get("dW"), db_pred=st.get("db"))
    return {k: st[k] for k in ("loss", "rows", "dHL", "dW", "db") if k in st}


def _own_product(st, case):
    st["B"].gcn_rows8_product(st["X8"], st["W8"], st["Y"], st["work"], bias=st["in"]["b"], relu=case["relu"],
                              transpose=case["transpose"])
    return {"Y": st["Y"]}


def _own_pack(st, case):
    st["B"].gcn_rows8_pack(st["in"]["X"], st["X8"])
    return {"q": st["X8"].values, "scale": st["X8"].scale}


def _own_weight_grad(st, case):
    st["B"].gcn_rows8_weight_grad(st["X8"], st["in"]["dY"], st["dW"], st["work"], db=st["db"], mask=st["in"]["yq"],
                                  dZ8=st["dZ8"])
    return {"dW": st["dW"], "db": st["db"], "q": st["dZ8"].values, "scale": st["dZ8"].scale}


def _plain_loss(x, case):
    W = x["W"].to(torch.float32)
    H = x["HL"].to(torch.float32)
    X = H @ W
    if x["b"] is not None:
        X += x["b"]
    has = (x["labels"] >= 0) & (x["labels"] < case["C"])
    at = torch.where(has, x["labels"], 0).to(torch.int64).unsqueeze(1)
    top = X.amax(dim=1, keepdim=True)
    picked = X.gather(1, at)
    X = torch.exp(X - top)
    total = X.sum(dim=1, keepdim=True)
    rows = torch.where(has, (torch.log(total) + top - picked).squeeze(1), 0.0)
    count = has.sum().clamp(min=1).to(torch.float32)
    out = {"loss": (rows.sum() / count).reshape(1), "rows": rows}
    if case["grad"]:
        G = X * (has.unsqueeze(1) / total)
        G.scatter_add_(1, at, -has.to(torch.float32).unsqueeze(1))
        G /= count
        out |= {"dHL": (G @ W.T).to(x["HL"].dtype), "dW": (H.T @ G).to(x["W"].dtype), "db": G.sum(dim=0)}
    return out


def _plain_product(x, case):
    W = _values_weights(x["wq"], x["ws"])
    Y = _values_rows(x["q"], x["s"]) @ (W.T if case["transpose"] else W)
    if x["b"] is not None:
        Y += x["b"]
    if case["relu"]:
        Y = torch.relu(Y)
    return {"Y": Y.to(FLOAT[case["type"]])}


def _plain_pack(x, case):
    q, s = _pack_rows(x["X"])
    return {"q": q, "scale": s}


def _plain_weight_grad(x, case):
    dZ = x["dY"].to(torch.bfloat16).to(torch.float32) * (x["yq"].to(torch.float32) > 0)
    q, s = _pack_rows(dZ)
    return {"dW": _values_rows(x["q"], x["s"]).T @ dZ, "db": dZ.sum(dim=0), "q": q, "scale": s}


# ------------------------------------------------------------------ the work
def work(case):
    e = 4 if case["type"] == "f32" else 2
    n = case["n"]
    if case["op"] == "loss":
        f, C = case["f"], case["C"]
        moved = e * (n * f + f * C) + 4 * (C if case["bias"] else 0) + 8 * n
        if case["grad"]:   # the three products of the definition
            return {"bytes": moved + e * (n * f + f * C) + 4 * C, "flops": 6.0 * n * f * C}
        return {"bytes": moved, "flops": 2.0 * n * f * C}
    if case["op"] == "product":
        K, N = case["K"], case["N"]
        blocks = (K + BLOCK - 1) // BLOCK
        moved = n * (K + blocks) + K * N + blocks * ((N + BLOCK - 1) // BLOCK) + (4 * N if case["bias"] else 0)
        return {"bytes": moved + e * n * N, "flops": 2.0 * n * K * N}
    if case["op"] == "pack":
        f = case["f"]
        return {"bytes": n * (e * f + f + (f + BLOCK - 1) // BLOCK), "flops": 0}
    f, N = case["f"], case["N"]
    moved = n * (f + (f + BLOCK - 1) // BLOCK) + n * N * (e + 1)
    return {"bytes": moved + 4 * (f * N + N) + n * (N + (N + BLOCK - 1) // BLOCK), "flops": 2.0 * n * f * N}


# ------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    x = _inputs(case, seed)
    d = torch.float64
    if case["op"] == "loss":
        n, C = case["n"], case["C"]
        H, W = x["HL"].to(d), x["W"].to(d)
        b = torch.zeros(C, dtype=d, device=DEV) if x["b"] is None else x["b"].to(d)
        labels = x["labels"].to(torch.int64)
        lab = torch.nonzero((labels >= 0) & (labels < C)).squeeze(1)
        rows = torch.zeros(n, dtype=d, device=DEV)
        dH, dW, db = torch.zeros_like(H), torch.zeros_like(W), torch.zeros_like(b)
        for part in torch.split(lab, 2048):     # the rows without a label add nothing
            h = H.index_select(0, part)
            logp = torch.log_softmax(torch.addmm(b, h, W), dim=1)
            y = labels.index_select(0, part)
            k = torch.arange(part.numel(), device=DEV)
            rows[part] = -logp[k, y]
            if case["grad"]:
                G = logp.exp_()
                G[k, y] -= 1.0
                G.mul_(1.0 / lab.numel())
                dH[part] = G.mm(W.t())
                dW.addmm_(h.t(), G)
                db += G.sum(0)
        out = {"loss": (rows.sum() / max(1, lab.numel())).reshape(1), "rows": rows}
        return out | {"dHL": dH, "dW": dW, "db": db} if case["grad"] else out
    if case["op"] == "product":
        w = _exact_values(x["wq"], x["ws"], BLOCK)
        v = _exact_values(x["q"], x["s"], 1)
        y = v.mm(w.t() if case["transpose"] else w)
        if x["b"] is not None:
            y = y + x["b"].to(d)
        return {"Y": y.clamp(min=0.0) if case["relu"] else y}
    if case["op"] == "pack":
        q, e = _exact_rows8(x["X"].to(d))
        return {"q": q, "scale": e}
    z = torch.where(x["yq"].to(d) > 0, x["dY"].to(torch.bfloat16).to(d), torch.zeros((), dtype=d, device=DEV))
    q, e = _exact_rows8(z)
    return {"dW": _exact_values(x["q"], x["s"], 1).t().mm(z), "db": z.sum(0), "q": q, "scale": e}


def _exact_power(k):
    """2^k in float64, exactly."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_values(q, s, rows):
    """The float64 values of q under one scale byte for each `rows` rows x 128 columns."""
    r, c = q.shape
    i = torch.arange(r, device=q.device) // rows
    j = torch.arange(c, device=q.device) // BLOCK
    return q.to(torch.float64) * _exact_power(s.to(torch.int64) - 127).index_select(0, i).index_select(1, j)


def _exact_rows8(z):
    """The values q of the 8-bit rows of z, and the scale bytes, by the e4m3 grid: steps of an eighth of the
    binade from 2^-6 up, of 2^-9 below."""
    qs, es = [], []
    for block in torch.split(z, BLOCK, dim=1):
        a = block.abs().amax(dim=1, keepdim=True)
        k = _exact_binade(a)
        e = torch.where(a > 1.75 * _exact_power(k), k - 7, k - 8)
        e = torch.where(a > 0, e, torch.zeros_like(e)).clamp(-126, 127)
        v = block * _exact_power(-e)
        step = _exact_power(_exact_binade(v.abs().clamp(min=2.0 ** -6)) - 3)
        q = torch.round(v / step) * step            # halves to the even multiple
        qs.append(torch.where((q == 0) & (v != 0), torch.sign(v) * 2.0 ** -9, q))
        es.append((e + 127).to(torch.uint8))
    return torch.cat(qs, dim=1), torch.cat(es, dim=1)


def _exact_binade(a):
    """k with 2^k <= a < 2^(k + 1), from the bits of the float64 a (0 where a is 0)."""
    return torch.where(a > 0, ((a.view(torch.int64) >> 52) & 2047) - 1023, 0)
