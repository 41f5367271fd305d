"""Performance cases of the operators for the parameters outside the low-rank path.

A model that trains with ``paper_2602_04396_b200.lordo.Lordo`` has parameters that are no weight matrices of the low-rank
path: the embedding table, norm gains, biases. Their operators are

* ``step``     one ``adamw.AdamW.step`` over a list of tensors, K workers' replicas each, moments in 32 or in 8 bits
* ``tokens``   the same step, the first tensor's gradient given by its tokens (``adamw.TokenGrad``)
* ``outer``    one ``adamw.AdamW.outer_step``: mean of the workers' moments, pseudo-gradient, Nesterov, broadcast
* ``embed``    one ``embedding.embedding``: rows of a table by tokens, scaled
* ``grad``     one ``embedding.embedding_grad``: the table's gradient, by sorted tokens

``sizes`` lists the tensors of a group as ``<elements>`` or ``<rows>x<columns>``, with ``*<count>`` for repetitions. Arrays of one
kind lie in one flat buffer, each tensor's [K][n] from a multiple of 128 elements on; 8-bit moments have a scale for each 256
elements of one worker's tensor, a tensor's scales lie from a multiple of 128 on too.
"""
from __future__ import annotations

import re
from typing import Dict, List

import torch

own = False  # True: the library's operators, False: their plain form

BETA1, BETA2, EPS = 0.9, 0.999, 1e-8
LR, DECAY = 1e-3, 0.1
ETA, MU = 0.7, 0.9  # outer rate and momentum
SEED = 11           # of the generator that rounds the 8-bit moments
BLOCK = 256         # elements per scale of the 8-bit moments
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def listed() -> List[dict]:
    step = dict(op="step", states="f32", dtype="bf16", omega=1.0, rho=1.0)
    table = dict(op="embed", dtype="bf16", index="i64", scale=1.0)
    return [
        # norm gains and biases of a stack of 12 layers of 768: many small tensors, all latency
        dict(step, name="step32_gains_768", sizes="768*37", K=8),
        # the table of a 1B-shaped stack, four workers: HBM rate
        dict(step, name="step32_table_2048", sizes="32000x2048,2048*49", K=4, omega=0.9),
        # a toy model's leftovers in fp32, sizes that fill no block and no vector
        dict(step, name="step8_ragged_f32", sizes="1003x333,50257,4097,1001*3,256,31,7,1", K=3, states="8bit", dtype="f32"),
        # the tables and gains of a 125M-shaped stack, eight workers
        dict(step, name="step8_table_768", sizes="50304x768,2048x768,768*25", K=8, states="8bit"),
        # the same with the embedding's gradient given by its tokens
        dict(step, name="tokens32_table_768", op="tokens", sizes="50304x768,2048x768,768*25", K=8, T=8192, index="i64", scale=1.0, pads=0.02),
        # a short batch on a large table, scaled by the root of the width
        dict(step, name="tokens8_table_2048", op="tokens", sizes="32000x2048,2048*49", K=4, T=2048, index="i32", scale=45.25, states="8bit", pads=0.0),
        # synchronisation of eight workers
        dict(step, name="outer32_table_768", op="outer", sizes="50304x768,768*25", K=8),
        # the same of 8-bit moments, ragged, few elements
        dict(step, name="outer8_ragged", op="outer", sizes="4001x333,50257,1001*7,31,1", K=4, states="8bit", dtype="f32"),
        # the rows of a few sequences' next tokens: latency
        dict(table, name="embed_next_token", V=32000, d=2048, K=1, T=8, scale=45.25, pads=0.0),
        # a training batch of eight workers
        dict(table, name="embed_batch_768", V=50304, d=768, K=8, T=16384, pads=0.02),
        # its gradient
        dict(table, name="grad_batch_768", op="grad", V=50304, d=768, K=8, T=16384, pads=0.02, accumulate=False),
        # a tied table's second share of its gradient, odd sizes, many tokens on few rows
        dict(table, name="grad_tied_odd_f32", op="grad", V=1003, d=333, K=2, T=5001, dtype="f32", index="i32", scale=18.25, pads=0.3, accumulate=True),
    ]


def draw(rng) -> dict:
    """One more case: operator, number and sizes of the tensors, workers, types and options drawn."""
    op = rng.choices(["step", "tokens", "outer", "embed", "grad"], [4, 2, 2, 2, 2])[0]
    dtype = rng.choice(["bf16", "bf16", "f32"])

    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    K = rng.choice([1, 2, 3, 4, 8])
    if op in ("embed", "grad"):
        d = log(8, 4096) if rng.random() < 0.3 else max(8, log(8, 4096) // 8 * 8)
        V = max(2, min(log(64, 130000), int(2.6e8 / (d * K))))
        T = max(1, min(log(1, 65536), int(1e8 / (d * K))))
        case = dict(op=op, dtype=dtype, V=V, d=d, K=K, T=T, index=rng.choice(["i64", "i32"]), scale=rng.choice([1.0, 11.3, 32.0]),
                    pads=rng.choice([0.0, 0.02, 0.5]))
        return dict(case, accumulate=rng.random() < 0.4) if op == "grad" else case
    budget = 10 ** rng.uniform(4.0, 8.3)  # elements of all workers
    sizes, total = [], 0
    if op == "tokens" or rng.random() < 0.5:
        d = log(8, 4096) if rng.random() < 0.2 else max(8, log(8, 4096) // 8 * 8)
        V = max(2, min(log(64, 130000), int(budget / (d * K))))
        sizes.append(f"{V}x{d}")
        total += V * d * K
    for _ in range(rng.randint(1, 5)):
        n, many = log(1, 3e6), rng.choice([1, 1, 3, 12])
        if total + n * many * K <= budget or not sizes:
            n = min(n, max(1, int(budget / (many * K))))
            sizes.append(f"{n}*{many}" if many > 1 else str(n))
            total += n * many * K
    case = dict(op=op, sizes=",".join(sizes), K=K, dtype=dtype, states=rng.choice(["f32", "8bit"]), omega=rng.choice([1.0, 0.94]),
                rho=rng.choice([0.0, 0.5, 1.0]))
    if op == "tokens":
        case.update(T=max(1, min(log(1, 32768), int(5e7 / (d * K)))), index=rng.choice(["i64", "i32"]), scale=rng.choice([1.0, 11.3, 32.0]),
                    pads=rng.choice([0.0, 0.02, 0.5]))
    return case


def _shapes(text: str) -> List[tuple]:
    out = []
    for part in text.split(","):
        shape, count = re.fullmatch(r"([\dx]+)(?:\*(\d+))?", part).groups()
        out += [tuple(int(x) for x in shape.split("x"))] * int(count or 1)
    return out


def _numel(shape: tuple) -> int:
    return shape[0] * (shape[1] if len(shape) == 2 else 1)


def _offsets(counts: List[int]) -> List[int]:
    at = [0]
    for c in counts:
        at.append(at[-1] + (c + 127) // 128 * 128)
    return at


def _distinct(V: int, T: int, pads: float) -> float:
    """Expected number of distinct tokens of one worker (see _tokens)."""
    edge = torch.arange(1, V + 2, dtype=torch.float64).log() / torch.tensor(float(V + 1), dtype=torch.float64).log()
    p = (edge[1:] - edge[:-1]) * (1.0 - pads)
    return float((1.0 - (1.0 - p) ** T).sum())


def work(case: dict) -> Dict[str, float]:
    e = 2 if case["dtype"] == "bf16" else 4
    K = case["K"]
    if case["op"] in ("embed", "grad"):
        V, d, T = case["V"], case["d"], case["T"]
        rows, ids = _distinct(V, T, case["pads"]), 8 if case["index"] == "i64" else 4
        if case["op"] == "embed":
            return {"bytes": K * (T * d * e + rows * d * e + T * ids), "flops": K * T * d}
        table = 2 * rows * d * e if case["accumulate"] else V * d * e
        return {"bytes": K * (T * (1 - case["pads"]) * d * e + table + T * ids), "flops": K * T * d}
    n = [_numel(s) for s in _shapes(case["sizes"])]
    total = K * sum(n)
    if case["op"] == "outer":
        return {"bytes": total * (2 * e + (16 if case["states"] == "f32" else 4)) + 16 * sum(n), "flops": 10 * total}
    moved = total * (2 * e + (16 if case["states"] == "f32" else 4)) + (total - (K * n[0] if case["op"] == "tokens" else 0)) * e
    if case["op"] == "tokens":
        moved += K * case["T"] * ((1 - case["pads"]) * _shapes(case["sizes"])[0][1] * e + (8 if case["index"] == "i64" else 4))
    return {"bytes": moved, "flops": 16 * total}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _tokens(case: dict, V: int, gen) -> torch.Tensor:
    """[K][T] tokens whose frequency falls with their number (P(t) = log((t+2)/(t+1)) / log(V+1)), a share of them padding (-1)."""
    K, T = case["K"], case["T"]
    u = torch.rand(K, T, device="cuda", dtype=torch.float64, generator=gen)
    tok = ((float(V + 1) ** u).floor() - 1).clamp_(0, V - 1).to(torch.int64)
    pad = torch.rand(K, T, device="cuda", generator=gen) < case["pads"]
    return tok.masked_fill_(pad, -1).to(torch.int64 if case["index"] == "i64" else torch.int32)


def prepare(case: dict, seed: int) -> Dict:
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, K = DTYPE[case["dtype"]], case["K"]

    def normal(*shape, std=1.0):
        return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(0.0, std, generator=gen)

    if case["op"] in ("embed", "grad"):
        V, d = case["V"], case["d"]
        st = dict(case=case, tokens=_tokens(case, V, gen))
        if case["op"] == "embed":
            st["W"] = normal(K, V, d, std=0.02).to(dt)
        else:
            st["dY"] = normal(K, case["T"], d, std=0.01).to(dt)
            st["dW"] = normal(K, V, d, std=0.01).to(dt) if case["accumulate"] else torch.empty(K, V, d, device="cuda", dtype=dt)
        return st

    shapes = _shapes(case["sizes"])
    n = [_numel(s) for s in shapes]
    nb = [(x + BLOCK - 1) // BLOCK for x in n]
    at, bat, xat = (_offsets(c) for c in ([K * x for x in n], [K * x for x in nb], n))
    sigma = max(case["rho"], 0.5) / sum(n) ** 0.5  # the norm of a worker's gradient is about twice the radius

    def flat(offsets, counts, fill, dtype):
        """A flat buffer, zero between the tensors."""
        buf = torch.zeros(offsets[-1], device="cuda", dtype=dtype)
        for o, c in zip(offsets, counts):
            buf[o:o + c] = fill(c).to(dtype)
        return buf

    Kn, Kb = [K * x for x in n], [K * x for x in nb]
    store = {"W": flat(at, Kn, lambda c: normal(c, std=0.02), dt)}
    if case["states"] == "f32":
        store["m"] = flat(at, Kn, lambda c: normal(c, std=0.3 * sigma), torch.float32)
        store["v"] = flat(at, Kn, lambda c: (normal(c).square_() + 0.2).mul_(sigma * sigma), torch.float32)
    else:  # codes of up to 255 on scales that put a block's largest near 3 sigma
        top = torch.tensor(3.0 * sigma / 255.0).log2().round().int().item() + 127

        def scales(c):
            return torch.randint(top - 1, top + 2, (c,), device="cuda", generator=gen, dtype=torch.int32)

        store["m"] = flat(at, Kn, lambda c: normal(c, std=25.0).clamp_(-255.0, 255.0), torch.float8_e4m3fn)
        store["v"] = flat(at, Kn, lambda c: normal(c, std=60.0).abs_().add_(8.0).clamp_(max=255.0), torch.float8_e4m3fn)
        store["ms"] = flat(bat, Kb, scales, torch.uint8).view(torch.float8_e8m0fnu)
        store["vs"] = flat(bat, Kb, scales, torch.uint8).view(torch.float8_e8m0fnu)
    if case["op"] == "outer":
        store["X0"] = flat(xat, n, lambda c: normal(c, std=0.02), torch.float32)
        store["B"] = flat(xat, n, lambda c: normal(c, std=0.002), torch.float32)
    st = dict(case=case, shapes=shapes, n=n, nb=nb, at=at, bat=bat, xat=xat, store=store, steps=100, outers=3)
    if case["op"] != "outer":
        st["G"] = [normal(K, *s, std=2.0 * sigma).to(dt) for s in (shapes[1:] if case["op"] == "tokens" else shapes)]
    if case["op"] == "tokens":
        V, d = shapes[0]
        st["tokens"] = _tokens(case, V, gen)
        st["dY"] = normal(K, case["T"], d, std=2.0 * sigma * (V / case["T"]) ** 0.5 / case["scale"]).to(dt)
    if own:
        st["handle"] = _handle(case, st)
    return st


def _handle(case: dict, st: Dict):
    """The group of a training program that stands at step 100, its arrays filled as the state's."""
    from paper_2602_04396_b200 import adamw, lordo
    dt = DTYPE[case["dtype"]]
    W0 = [torch.zeros(s, device="cuda", dtype=dt) for s in st["shapes"]]
    opt = adamw.AdamW(W0, case["K"], g_dtype=dt, states=case["states"], weight_decay=[DECAY if len(s) == 2 else 0.0 for s in st["shapes"]],
                      beta2=BETA2, eps=EPS, clip_rho=case["rho"], outer=lordo.OUTER_NESTEROV if case["op"] == "outer" else None,
                      outer_lr=ETA, outer_momentum=MU, seed=SEED, tables={0: case["T"]} if case["op"] == "tokens" else None)
    for name, buf in st["store"].items():
        opt.storage[name].copy_(buf)
    st["store"] = opt.storage
    opt.set_counters([st["steps"], st["outers"]])
    if case["op"] == "tokens":
        st["G"] = [adamw.TokenGrad(st["tokens"], st["dY"], case["scale"])] + st["G"]
    return opt


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------
_GOLDEN, _M1, _M2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB
_MASK = (1 << 64) - 1


def _signed(x: int) -> int:
    x &= _MASK
    return x - (1 << 64) if x >> 63 else x


def _mix(x: int) -> int:
    x = ((x ^ (x >> 30)) * _M1) & _MASK
    x = ((x ^ (x >> 27)) * _M2) & _MASK
    return x ^ (x >> 31)


def _stream_key(seed: int, purpose: int, index: int) -> int:
    """The library's generator: a key chained from (seed, purpose, matrix 0, index, replica 0)."""
    k = _mix((seed + _GOLDEN) & _MASK)
    for f in (purpose, 0, index, 0):
        k = _mix((k + _GOLDEN * (f + 1)) & _MASK)
    return k


def _bits16(key: int, n: int) -> torch.Tensor:
    """Sixteen random bits for each of n elements: four of them share a word of the generator."""
    x = torch.arange(1, (n + 3) // 4 + 1, device="cuda", dtype=torch.int64) * _signed(_GOLDEN) + _signed(key)
    x = (x ^ ((x >> 30) & (_MASK >> 30))) * _signed(_M1)
    x = (x ^ ((x >> 27) & (_MASK >> 27))) * _signed(_M2)
    x = x ^ ((x >> 31) & (_MASK >> 31))
    return torch.stack([(x >> s) & 0xFFFF for s in (0, 16, 32, 48)], dim=1).view(-1)[:n]


def _rounding(purpose: int, index: int, tensor: int, K: int, n: int):
    """[K][n] random bits for a tensor's first moments, and those for its second."""
    first = _stream_key(SEED, purpose, index)
    u = torch.stack([_bits16(_mix((first + _GOLDEN * (tensor * K + k + 1)) & _MASK), n) for k in range(K)])
    return u, (u * 40503) & 0xFFFF


def _wide(codes: torch.Tensor, scales: torch.Tensor) -> torch.Tensor:
    """[K][n] values of 8-bit codes with a scale for each 256."""
    return codes.float() * scales.float().repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]


def _round8(x: torch.Tensor, u: torch.Tensor, positive: bool):
    """8-bit codes and scales of [K][n] values: the scale is the power of two that puts a block's largest magnitude into [128, 256)
    (at least 2^-126), codes are E4M3, rounded up or down with 16 random bits each. Positive values do not become zero."""
    K, n = x.shape
    blocks = torch.nn.functional.pad(x.abs(), (0, -n % BLOCK)).view(K, -1, BLOCK)
    top = blocks.amax(dim=2)
    e = torch.where(top > 0, torch.frexp(top).exponent - 8, -126).clamp(-126, 127)
    t = torch.ldexp(x.abs(), -e.repeat_interleave(BLOCK, dim=1)[:, :n])
    step = torch.ldexp(torch.ones_like(t), (torch.frexp(t).exponent - 1).clamp(min=-6) - 3)
    q = torch.floor(t / step + (u.float() + 0.5) / 65536.0) * step
    if positive:
        q = torch.where(x > 0, q.clamp(min=2.0 ** -9), q)
    return torch.copysign(q, x).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _views(st: Dict, name: str, counts: List[int], offsets: List[int], K: int) -> List[torch.Tensor]:
    buf = st["store"][name]
    return [buf[o:o + K * c].view(K, c) for o, c in zip(offsets, counts)]


def _table_grad(tokens, dY, scale, V):
    """[K][V][d] in fp32: the sum of the rows of dY that belong to each token."""
    K, T, d = dY.shape
    tok = tokens.to(torch.int64)
    rows = torch.where((tok >= 0) & (tok < V), tok + V * torch.arange(K, device="cuda").view(K, 1), K * V)
    out = torch.zeros(K * V + 1, d, device="cuda", dtype=torch.float32)
    out.index_add_(0, rows.view(-1), dY.reshape(K * T, d).float())
    return (out[:K * V] * scale).view(K, V, d)


def _plain_step(st: Dict):
    case, store, K = st["case"], st["store"], st["case"]["K"]
    st["steps"] += 1
    s, w, rho = st["steps"], case["omega"], case["rho"]
    bc1, bc2 = 1.0 - BETA1 ** s, 1.0 - BETA2 ** s
    G = [g.reshape(K, -1).float() for g in st["G"]]
    if case["op"] == "tokens":
        G = [_table_grad(st["tokens"], st["dY"], case["scale"], st["shapes"][0][0]).view(K, -1)] + G
    coef = torch.ones(K, device="cuda")
    if rho > 0:
        norm = torch.stack([g.square().sum(dim=1, dtype=torch.float64) for g in G]).sum(dim=0).sqrt()
        coef = (rho / (norm + 1e-6)).clamp(max=1.0).float()
    W, m, v = (_views(st, x, st["n"], st["at"], K) for x in ("W", "m", "v"))
    small = case["states"] == "8bit"
    if small:
        ms, vs = (_views(st, x, st["nb"], st["bat"], K) for x in ("ms", "vs"))
    for i, g in enumerate(G):
        g = g * coef.view(K, 1)
        m0 = _wide(m[i], ms[i]) if small else m[i]
        v0 = _wide(v[i], vs[i]).square() if small else v[i]
        m1 = BETA1 * m0 + (1.0 - BETA1) * g
        v1 = BETA2 * v0 + (1.0 - BETA2) * g * g
        mh = m1 / bc1
        up = (w * mh + (1.0 - w) * g) / ((v1 / bc2).sqrt() + EPS)
        x = W[i].float()
        W[i].copy_(x - LR * (up + (DECAY if len(st["shapes"][i]) == 2 else 0.0) * x))
        if small:
            um, uv = _rounding(3, s, i, K, st["n"][i])
            for code, scale, val, u, positive in ((m[i], ms[i], m1, um, False), (v[i], vs[i], v1.sqrt(), uv, True)):
                c8, s8 = _round8(val, u, positive)
                code.copy_(c8)
                scale.copy_(s8)
        else:
            m[i].copy_(m1)
            v[i].copy_(v1)
    return store


def _plain_outer(st: Dict):
    case, store, K = st["case"], st["store"], st["case"]["K"]
    W, m, v = (_views(st, x, st["n"], st["at"], K) for x in ("W", "m", "v"))
    X0, B = (_views(st, x, st["n"], st["xat"], 1) for x in ("X0", "B"))
    small = case["states"] == "8bit"
    if small:
        ms, vs = (_views(st, x, st["nb"], st["bat"], K) for x in ("ms", "vs"))
    for i in range(len(W)):
        if small:
            um, uv = _rounding(4, st["outers"], i, 1, st["n"][i])
            c8, s8 = _round8(_wide(m[i], ms[i]).mean(dim=0, keepdim=True), um, False)
            m[i].copy_(c8.expand(K, -1))
            ms[i].copy_(s8.expand(K, -1))
            c8, s8 = _round8(_wide(v[i], vs[i]).square().mean(dim=0, keepdim=True).sqrt(), uv, True)
            v[i].copy_(c8.expand(K, -1))
            vs[i].copy_(s8.expand(K, -1))
        else:
            m[i].copy_(m[i].mean(dim=0, keepdim=True).expand(K, -1))
            v[i].copy_(v[i].mean(dim=0, keepdim=True).expand(K, -1))
        delta = X0[i] - W[i].float().mean(dim=0, keepdim=True)
        B[i].copy_(MU * B[i] + delta)
        X0[i].copy_(X0[i] - ETA * (delta + MU * B[i]))
        W[i].copy_(X0[i].expand(K, -1))
    st["outers"] += 1
    return store


def run(st: Dict):
    case = st["case"]
    op = case["op"]
    if own:
        if op in ("step", "tokens"):
            st["handle"].step(st["G"], LR, BETA1, case["omega"])
            return st["store"]
        if op == "outer":
            st["handle"].outer_step()
            return st["store"]
        from paper_2602_04396_b200 import embedding
        if op == "embed":
            return embedding.embedding(st["W"], st["tokens"], scale=case["scale"])
        return embedding.embedding_grad(st["dY"], st["tokens"], case["V"], scale=case["scale"], out=st["dW"], accumulate=case["accumulate"])
    if op in ("step", "tokens"):
        return _plain_step(st)
    if op == "outer":
        return _plain_outer(st)
    V, d, K = case["V"], case["d"], case["K"]
    if op == "embed":
        tok = st["tokens"].to(torch.int64)
        inside = (tok >= 0) & (tok < V)
        rows = torch.where(inside, tok, 0) + V * torch.arange(K, device="cuda").view(K, 1)
        out = st["W"].view(K * V, d)[rows].float() * case["scale"]
        return (out * inside.unsqueeze(2)).to(st["W"].dtype)
    g = _table_grad(st["tokens"], st["dY"], case["scale"], V)
    st["dW"].copy_(st["dW"].float() + g if case["accumulate"] else g)
    return st["dW"]


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------
def _words(key: int, count: int) -> torch.Tensor:
    """The generator's words 1 .. count as four 16-bit pieces, computed in 32-bit halves."""
    def mul(hi, lo, c):
        c_hi, c_lo = c >> 32, c & 0xFFFFFFFF
        a, b = lo & 0xFFFF, lo >> 16
        low = a * c_lo
        mid = b * c_lo + (low >> 16)
        return ((mid >> 16) + lo * (c_hi & 0xFFFF) + ((lo * (c_hi >> 16) & 0xFFFF) << 16) + hi * (c_lo & 0xFFFF)
                + ((hi * (c_lo >> 16) & 0xFFFF) << 16)) & 0xFFFFFFFF, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)

    def fold(hi, lo, s):
        if s < 32:
            return hi ^ (hi >> s), lo ^ (((hi << (32 - s)) | (lo >> s)) & 0xFFFFFFFF)
        return hi, lo ^ (hi >> (s - 32))

    j = torch.arange(1, count + 1, device="cuda", dtype=torch.int64)
    hi, lo = mul(j >> 32, j & 0xFFFFFFFF, _GOLDEN)
    lo = lo + (key & 0xFFFFFFFF)
    hi, lo = (hi + (key >> 32) + (lo >> 32)) & 0xFFFFFFFF, lo & 0xFFFFFFFF
    hi, lo = mul(*fold(hi, lo, 30), _M1)
    hi, lo = mul(*fold(hi, lo, 27), _M2)
    hi, lo = fold(hi, lo, 31)
    return torch.stack([lo & 0xFFFF, lo >> 16, hi & 0xFFFF, hi >> 16], dim=1).view(-1)


def _code64(x: torch.Tensor, u: torch.Tensor, positive: bool):
    """One worker's values as (codes, scales), both as 64-bit numbers."""
    n = x.numel()
    a = torch.zeros(-(-n // BLOCK) * BLOCK, device="cuda", dtype=torch.float64)
    a[:n] = x.abs()
    a = a.view(-1, BLOCK)
    top = a.max(dim=1).values
    scale = torch.pow(2.0, torch.where(top > 0, top.clamp(min=1e-300).log2().floor() - 7.0, torch.full_like(top, -126.0)).clamp(-126.0, 127.0))
    over = top / scale  # log2 may be one off next to a power of two
    scale = torch.where(over >= 256.0, scale * 2.0, torch.where((over < 128.0) & (scale > 2.0 ** -126), scale / 2.0, scale))
    t = (a / scale.view(-1, 1)).view(-1)[:n]
    step = torch.full_like(t, 2.0 ** -9)
    for e in range(-5, 9):
        step[t >= 2.0 ** e] = 2.0 ** (e - 3)
    q = ((t / step) + (u.double() + 0.5) / 65536.0).floor() * step
    if positive:
        q[(t > 0) & (q == 0)] = 2.0 ** -9
    return q * torch.where(x < 0, -1.0, 1.0), scale


def exact(case: dict, seed: int):
    """What ``run`` returns, in 64 bits: one tensor and one worker at a time."""
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    K, op = case["K"], case["op"]
    if op in ("embed", "grad"):
        V, d = case["V"], case["d"]
        if op == "embed":
            table = torch.cat([st["W"].double(), torch.zeros(K, 1, d, device="cuda", dtype=torch.float64)], dim=1)
            tok = st["tokens"].long()
            tok = torch.where((tok < 0) | (tok >= V), V, tok)
            return torch.stack([case["scale"] * table[k].index_select(0, tok[k]) for k in range(K)])
        return torch.stack([_grad64(st["tokens"][k], st["dY"][k], V) * case["scale"] + (st["dW"][k].double() if case["accumulate"] else 0.0)
                            for k in range(K)])
    out = {name: torch.zeros_like(buf, dtype=torch.float64) for name, buf in st["store"].items()}
    out.update({name: st["store"][name].double() for name in ("ms", "vs") if name in out})
    store, small = st["store"], case["states"] == "8bit"

    def piece(buf, offsets, i, k, c):
        return buf[offsets[i] + k * c:offsets[i] + (k + 1) * c]

    def moments(i, k):
        n, nb = st["n"][i], st["nb"][i]
        m, v = (piece(store[x], st["at"], i, k, n).double() for x in ("m", "v"))
        if not small:
            return m, v
        sm, sv = (piece(store[x], st["bat"], i, k, nb).double().view(nb, 1).expand(nb, BLOCK).reshape(-1)[:n] for x in ("ms", "vs"))
        return m * sm, (v * sv) ** 2

    def keep(i, k, m, v, u):
        n, nb = st["n"][i], st["nb"][i]
        if small:
            pairs = (("m", "ms", m, u, False), ("v", "vs", v.sqrt(), (u * 40503) % 65536, True))
            for code, scale, x, bits, positive in pairs:
                c, s = _code64(x, bits, positive)
                piece(out[code], st["at"], i, k, n).copy_(c)
                piece(out[scale], st["bat"], i, k, nb).copy_(s)
        else:
            piece(out["m"], st["at"], i, k, n).copy_(m)
            piece(out["v"], st["at"], i, k, n).copy_(v)

    def bits(purpose, index, number, n):
        key = _mix((_stream_key(SEED, purpose, index) + _GOLDEN * (number + 1)) & _MASK)
        return _words(key, (n + 3) // 4)[:n] if small else None

    if op == "outer":
        for i, n in enumerate(st["n"]):
            each = [moments(i, k) for k in range(K)]
            m, v = (sum(x[j] for x in each) / K for j in (0, 1))
            u = bits(4, st["outers"], i, n)
            x0, b = (piece(store[x], st["xat"], i, 0, n).double() for x in ("X0", "B"))
            delta = x0 - sum(piece(store["W"], st["at"], i, k, n).double() for k in range(K)) / K
            b = delta + b * MU
            x0 = x0 - (delta * ETA + b * (ETA * MU))
            piece(out["X0"], st["xat"], i, 0, n).copy_(x0)
            piece(out["B"], st["xat"], i, 0, n).copy_(b)
            for k in range(K):
                keep(i, k, m, v, u)
                piece(out["W"], st["at"], i, k, n).copy_(x0)
        return out

    s, w = st["steps"] + 1, case["omega"]

    def grads(k):
        got = [g[k].reshape(-1).double() for g in st["G"]]
        if op == "tokens":
            got = [_grad64(st["tokens"][k], st["dY"][k], st["shapes"][0][0]).view(-1) * case["scale"]] + got
        return got

    for k in range(K):
        G = grads(k)
        c = 1.0
        if case["rho"] > 0:
            c = min(1.0, case["rho"] / (sum(float((g * g).sum()) for g in G) ** 0.5 + 1e-6))
        for i, g in enumerate(G):
            n = st["n"][i]
            m, v = moments(i, k)
            g = g * c
            m, v = m + (g - m) * (1.0 - BETA1), v + (g * g - v) * (1.0 - BETA2)
            ratio = (m * (w / (1.0 - BETA1 ** s)) + g * (1.0 - w)) / (EPS + (v / (1.0 - BETA2 ** s)) ** 0.5)
            x = piece(store["W"], st["at"], i, k, n).double()
            piece(out["W"], st["at"], i, k, n).copy_(x * (1.0 - LR * (DECAY if len(st["shapes"][i]) == 2 else 0.0)) - ratio * LR)
            keep(i, k, m, v, bits(3, s, i * K + k, n))
    return out


def _grad64(tokens: torch.Tensor, dY: torch.Tensor, V: int) -> torch.Tensor:
    """One worker's sums by token, [V][d]."""
    inside = (tokens >= 0) & (tokens < V)
    out = torch.zeros(V, dY.shape[1], device="cuda", dtype=torch.float64)
    return out.index_put_((tokens[inside].long(),), dY[inside].double(), accumulate=True)
