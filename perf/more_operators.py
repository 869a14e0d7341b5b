"""Performance cases of the root-mean-square norm with the residual's addition and of the softmax cross entropy of a vocabulary
projection, through the binding's public entry points, and the same operators in plain form.

  norm      S = X + R, Y = S / rms(S) * w: in bf16, in 32 bits, or in blocks of 32 numbers of 4 or 8 bits with one power
            of two each (flux_norm; those are read back here, flux_mx4_dequantize and flux_mx8_dequantize)
  norm_bwd  the gradients of S and w from that of Y, the stream's own gradient added (flux_norm_backward)
  loss      log-sum-exp, target's logit and loss of every row of X W^T, W [V,K], without keeping X W^T (flux_loss)
  loss_bwd  dX and dW of it (flux_loss_backward)

Where `own` is false `run` is the plain form: elementary torch operations in 32 bits, rounded once at the end.
"""
import functools

import torch

own = False

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-5
NOT_COUNTED = -100                     # target of a token that the loss leaves out


# ---- cases --------------------------------------------------------------------------------------------------------
def _norm(name, M, K, *, out="bf16", stream="bf16", keep=False):
    c = {"op": "norm", "M": M, "K": K, "out": out, "stream": stream, "keep": keep}
    return c if name is None else {"name": name, **c}


def _norm_bwd(name, M, K, *, stream="bf16"):
    c = {"op": "norm_bwd", "M": M, "K": K, "stream": stream}
    return c if name is None else {"name": name, **c}


def _loss(name, op, M, V, K, *, shards=1):
    """One of `shards` equal parts of a vocabulary: V columns of it."""
    c = {"op": op, "M": M, "V": V, "K": K, "shards": shards}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # serving, one token of one sequence: the stream of the Llama-2-70B-like layer
        _norm("norm_token", 1, 8192),
        # a decode batch on its way to the 4-bit gated block
        _norm("norm_decode_mx4", 64, 8192, out="mx4"),
        # an odd width, the stream in 32 bits, the result in 8 bits as it is gathered from the ranks
        _norm("norm_ragged_mx8", 1496, 5111, out="mx8", stream="f32"),
        # training, 8192 tokens of the GPT-3-175B-like layer: 1 / rms is kept for the backward pass
        _norm("norm_train", 8192, 12288, keep=True),
        # backward with an odd width and the stream in 32 bits
        _norm_bwd("norm_bwd_ragged", 1496, 5111, stream="f32"),
        # backward, 8192 tokens of the Llama-2-70B-like layer
        _norm_bwd("norm_bwd_train", 8192, 8192),
        # how likely one token was: one row against the whole vocabulary
        _loss("loss_token", "loss", 1, 32000, 8192),
        # evaluation of as many tokens as a text happens to have, a vocabulary that nothing divides
        _loss("loss_ragged", "loss", 1496, 50257, 5112),
        # training, 8192 tokens, one rank's eighth of the vocabulary
        _loss("loss_train_shard", "loss", 8192, 4000, 8192, shards=8),
        # backward with nothing a multiple of a tile: an eighth of 50257 columns, rounded up
        _loss("loss_bwd_ragged", "loss_bwd", 1496, 6283, 5112, shards=8),
        # backward of that rank's eighth
        _loss("loss_bwd_shard", "loss_bwd", 8192, 4000, 8192, shards=8),
        # backward, 8192 tokens, the whole vocabulary
        _loss("loss_bwd_train", "loss_bwd", 8192, 32000, 8192),
    ]


def draw(rng):
    """A case of the same ranges: 1 to 8192 rows; widths of 64 to 12288 (norm: odd ones too); 256 to 50257 columns of a vocabulary."""
    while True:
        op = rng.choice(["norm", "norm", "norm_bwd", "loss", "loss_bwd"])
        M = int(round(8192 ** rng.random()))                              # log-uniform, 1 .. 8192
        K = 8 * int(round(8 * 192 ** rng.random()))                       # log-uniform, 64 .. 12288
        if rng.random() < 0.4:                                            # sizes that tiles divide, as most models have them
            M, K = (M // 256 * 256 if M >= 256 else M), max(64, K // 256 * 256)
        if op in ("norm", "norm_bwd"):
            K -= rng.choice([0, 0, 0, 1, 5])
            stream = rng.choice(["bf16", "bf16", "f32"])
            if op == "norm_bwd":
                return _norm_bwd(None, M, K, stream=stream)
            return _norm(None, M, K, out=rng.choice(["bf16", "bf16", "f32", "mx4", "mx8"]), stream=stream, keep=rng.random() < 0.5)
        V = int(round(256 * (50257 / 256) ** rng.random()))               # log-uniform, 256 .. 50257, odd ones too
        if rng.random() < 0.4:
            V = max(256, V // 256 * 256)
        if M * V * K <= 8192 * 32000 * 8192:
            return _loss(None, op, M, V, K, shards=rng.choice([1, 1, 8]))


# ---- inputs -------------------------------------------------------------------------------------------------------
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": dict(case)}
    op, M, K = case["op"], case["M"], case["K"]
    if op in ("norm", "norm_bwd"):
        stream = TORCH[case["stream"]]
        loud = torch.exp(0.5 * _randn(gen, 1, K))                         # a few large channels
        s["w"] = (1.0 + 0.1 * _randn(gen, K)).to(torch.bfloat16)
        if op == "norm":
            s["X"], s["R"] = _randn(gen, M, K).to(torch.bfloat16), (_randn(gen, M, K) * loud).to(stream)
            return s
        s["S"] = (_randn(gen, M, K) * loud).to(stream)
        # what the forward pass kept
        s["rstd"] = torch.rsqrt(s["S"].float().square().mean(1) + EPS)
        s["dY"], s["dS"] = _randn(gen, M, K).to(torch.bfloat16), _randn(gen, M, K).to(stream)
        return s
    V, shards = case["V"], case["shards"]
    s["v0"] = V * (shards // 2)                                           # this part's first column
    s["X"], s["W"] = _randn(gen, M, K).to(torch.bfloat16), (0.02 * _randn(gen, V, K)).to(torch.bfloat16)
    target = torch.randint(0, V * shards, (M,), generator=gen, device=DEV)
    counts = torch.rand(M, generator=gen, device=DEV) < 0.9               # the others are a prompt's, or padding
    counts[0] = True
    s["target"] = torch.where(counts, target, NOT_COUNTED)
    if op == "loss_bwd":
        # what the forward pass kept, over the whole vocabulary; the mean's gradient
        s["lse"] = torch.logsumexp(s["X"].float() @ s["W"].float().t(), 1) + torch.log(torch.tensor(float(shards), device=DEV))
        s["dloss"] = counts.float() / counts.sum()
    return s


# ---- plain form ---------------------------------------------------------------------------------------------------
def _in_blocks(y, bits):
    """What blocks of 32 numbers of 4 (E2M1) or 8 bits (E4M3) stand for, in 32 bits."""
    M, K = y.shape
    x = torch.cat((y, y.new_zeros(M, -K % 32)), 1).view(M, -1, 32)
    e = ((x.abs().amax(2).view(torch.int32) >> 23) - (2 if bits == 4 else 8)).clamp(1, 253)[..., None]      # (biased)
    a = (x.abs() * ((254 - e) << 23).view(torch.float32)).clamp(max=6.0 if bits == 4 else 448.0)
    if bits == 8:
        a = a.to(torch.float8_e4m3fn).float()
    else:
        step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
        a = torch.round(a / step) * step
    return (torch.copysign(a, x) * (e << 23).view(torch.float32)).view(M, -1)[:, :K]


def _values(t, out):
    """4-bit values as numbers of 8 bits, which hold them, 8-bit ones as bf16."""
    return t.to(torch.float8_e4m3fn) if out == "mx4" else t.to(torch.bfloat16).contiguous()


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op == "norm":
        stream = (s["X"].float() + s["R"].float()).to(TORCH[c["stream"]])
        x = stream.float()
        rstd = torch.rsqrt(x.square().mean(1) + EPS)
        y = x * rstd[:, None] * s["w"].float()
        out = {"S": stream, "Y": _values(_in_blocks(y, int(c["out"][2:])), c["out"]) if c["out"] in ("mx4", "mx8") else y.to(TORCH[c["out"]])}
        return {**out, "rstd": rstd} if c["keep"] else out
    if op == "norm_bwd":
        x, dy, w = s["S"].float() * s["rstd"][:, None], s["dY"].float(), s["w"].float()
        g = dy * w
        ds = s["rstd"][:, None] * (g - x * (g * x).mean(1, keepdim=True)) + s["dS"].float()
        return {"dS": ds.to(TORCH[c["stream"]]), "dw": (dy * x).sum(0)}
    V = c["V"]
    x, w = s["X"].float(), s["W"].float()
    z = x @ w.t()
    at = s["target"] - s["v0"]
    here, counts = (at >= 0) & (at < V), s["target"] >= 0
    at = at.clamp(0, V - 1)[:, None]
    if op == "loss":
        top = z.amax(1)
        lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
        logit = torch.where(here, z.gather(1, at)[:, 0], 0.0)
        return {"lse": lse, "logit": logit, "loss": torch.where(counts, lse - logit, 0.0)}
    p = torch.exp(z - s["lse"][:, None])
    p.scatter_add_(1, at, -here.float()[:, None])
    p *= torch.where(counts, s["dloss"], 0.0)[:, None]
    return {"dX": (p @ w).to(torch.bfloat16), "dW": (p.t() @ x).to(torch.bfloat16)}


# ---- the framework's operators ------------------------------------------------------------------------------------
_workspaces = {}          # one per operator, as a program keeps it from step to step


def _workspace(kind, nbytes):
    if nbytes == 0:
        return None
    ws = _workspaces.get(kind)
    if ws is None or ws.numel() < nbytes:
        _workspaces.pop(kind, None)
        ws = _workspaces[kind] = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)
    return ws


@functools.lru_cache(maxsize=None)
def _problem(op, M, K, *more):
    """The problem's description and its workspace's size: made once, as a layer makes it."""
    from paper_2406_06858_amd import loss, norm
    if op in ("norm", "norm_bwd"):
        out, stream = more
        p = norm.norm_problem(M, K, x_dtype="bf16", s_dtype=stream, out=out, w_dtype="bf16", eps=EPS)
        return p, norm.flux_norm_workspace_bytes(p) if op == "norm_bwd" else 0
    V, shards, v0 = more
    p = loss.loss_problem(M, V, K, v0=v0, vocab=V * shards)
    return p, loss.flux_loss_workspace_bytes(loss.FLUX_LOSS_FORWARD if op == "loss" else loss.FLUX_LOSS_BACKWARD, p)


def _run_own(s):
    from paper_2406_06858_amd import ffn, loss, norm
    c = s["case"]
    op, M, K = c["op"], c["M"], c["K"]
    if op == "norm":
        p, _ = _problem(op, M, K, c["out"], c["stream"])
        S = torch.empty_like(s["R"])
        rstd = torch.empty(M, dtype=torch.float32, device=DEV) if c["keep"] else None
        if c["out"] in ("mx4", "mx8"):
            row = (ffn.flux_mx4_row_bytes if c["out"] == "mx4" else norm.flux_mx8_row_bytes)(K)
            q = torch.empty(M, row, dtype=torch.uint8, device=DEV)
            scales = torch.empty(M, ffn.flux_mx4_scale_row_bytes(K), dtype=torch.uint8, device=DEV)
            norm.flux_norm(p, s["X"], s["R"], s["w"], S, q, scales, rstd)
            Y = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
            (ffn.flux_mx4_dequantize if c["out"] == "mx4" else norm.flux_mx8_dequantize)(q, scales, Y)
            out = {"S": S, "Y": _values(Y, c["out"])}
        else:
            Y = torch.empty(M, K, dtype=TORCH[c["out"]], device=DEV)
            norm.flux_norm(p, s["X"], s["R"], s["w"], S, Y, None, rstd)
            out = {"S": S, "Y": Y}
        return {**out, "rstd": rstd} if c["keep"] else out
    if op == "norm_bwd":
        p, nbytes = _problem(op, M, K, "bf16", c["stream"])
        ds, dw = torch.empty_like(s["S"]), torch.empty(K, dtype=torch.float32, device=DEV)
        norm.flux_norm_backward(p, s["dY"], s["S"], s["w"], s["rstd"], s["dS"], ds, None, dw, _workspace(op, nbytes))
        return {"dS": ds, "dw": dw}
    p, nbytes = _problem(op, M, K, c["V"], c["shards"], s["v0"])
    ws = _workspace(op, nbytes)
    if op == "loss":
        lse, logit, value = (torch.empty(M, dtype=torch.float32, device=DEV) for _ in range(3))
        loss.flux_loss(p, s["X"], s["W"], s["target"], lse, logit, value, ws)
        return {"lse": lse, "logit": logit, "loss": value}
    dX, dW = torch.empty_like(s["X"]), torch.empty_like(s["W"])
    loss.flux_loss_backward(p, s["X"], s["W"], s["target"], s["lse"], s["dloss"], dX, dW, ws)
    return {"dX": dX, "dW": dW}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    op, M, K = case["op"], case["M"], case["K"]
    if op == "norm":
        n, blocks = M * K, M * ((K + 31) // 32)
        # blocks are written, read back and come out as numbers of 8 or 16 bits
        y = n * SIZE[case["out"]] if case["out"] in SIZE else 34 * blocks + n if case["out"] == "mx4" else 66 * blocks + 2 * n
        return {"bytes": n * (2 + 2 * SIZE[case["stream"]]) + y + 2 * K + (4 * M if case["keep"] else 0), "flops": 5 * n}
    if op == "norm_bwd":
        return {"bytes": M * K * (2 + 3 * SIZE[case["stream"]]) + 6 * K + 4 * M, "flops": 10 * M * K}
    V = case["V"]
    if op == "loss":
        return {"bytes": 2 * (M * K + V * K) + 20 * M, "flops": 2 * M * V * K}
    return {"bytes": 4 * (M * K + V * K) + 16 * M, "flops": 6 * M * V * K}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        stream = torch.add(s["X"].double(), s["R"].double())
        x = stream.to(TORCH[case["stream"]]).double()                     # the norm is that of the stream as it is stored
        rms = torch.sqrt(torch.linalg.vector_norm(x, dim=1) ** 2 / case["K"] + EPS)
        # (a number next to the border of two 4- or 8-bit values has either of them)
        y = None if case["out"] in ("mx4", "mx8") else x / rms[:, None] * s["w"].double()
        return {"S": stream, "Y": y, "rstd": 1.0 / rms} if case["keep"] else {"S": stream, "Y": y}
    if op == "norm_bwd":
        r, w, dy, x = s["rstd"].double()[:, None], s["w"].double(), s["dY"].double(), s["S"].double()
        along = torch.linalg.vecdot(dy * w, x)[:, None] / case["K"]
        return {"dS": s["dS"].double() + dy * w * r - x * along * r ** 3, "dw": torch.mv(x.mul_(dy).t(), s["rstd"].double())}
    x, w, target = s["X"].double(), s["W"].double(), s["target"]
    own_column = (target - s["v0"])[:, None] == torch.arange(case["V"], device=DEV)
    z = torch.mm(x, w.t())
    if op == "loss":
        lse, logit = torch.logsumexp(z, 1), (z * own_column).sum(1)
        return {"lse": lse, "logit": logit, "loss": (lse - logit) * (target != NOT_COUNTED)}
    dz = torch.exp(z.sub_(s["lse"].double()[:, None])) - own_column.double()
    dz *= (s["dloss"].double() * (target != NOT_COUNTED))[:, None]
    return {"dX": torch.mm(dz, w), "dW": torch.mm(dz.t(), x)}
