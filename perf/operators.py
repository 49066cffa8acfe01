"""The work that the 4-bit (MXFP4) operators and the norms around the MLP do,
as cases that can be timed, each with its plain form.

* ``quantize``: rows to MXFP4 and back (``quantize_rows_mxfp4``,
  ``dequantize_rows_mxfp4``): what loading weights and checking them does, and
  what a prompt's activations go through.  The 4-bit values are returned as the
  values they stand for.
* ``linear``: ``x W^T`` with MXFP4 weights and fp16 or bf16 activations
  (``linear_mxfp4``).
* ``gated``: ``ReLU(x W_gate^T) * (x W_up^T)``, Eq. (1) steps 1-3 of a prompt
  (``gated_linear_mxfp4``).
* ``linear_a4``: ``Q(x) W^T`` with the activations quantized to MXFP4 as well
  (``quantize_rows_mxfp4``, ``linear_mxfp4_a4``).
* ``sparse``: the predicted sparse MLP of 1 to 8 tokens with MXFP4 weights
  (``predict_sparse_mlp_mxfp4``).
* ``norm``: what stands between two blocks' products: the norm of a branch, its
  gate and residual scale, the residual, and the next norm
  (``norm_residual``).

MXFP4: 32 consecutive values of a row share the scale ``2^X`` with
``X = floor(log2(max |v|)) - 2`` (at least -127); a value is held as the
nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale, ties to the even code,
larger ones as 6, with its sign.  Rows are padded to whole 128 values.

``own`` False computes the plain forms with elementary torch operations in
float32; True makes the framework's calls.  Weights are laid out once, as a
program does at load: the plain form keeps them as float32.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}


# ---- cases ------------------------------------------------------------------

def _quantize(name, rows, n, dtype):
    return {"name": name, "op": "quantize", "rows": rows, "n": n, "dtype": dtype}


def _linear(name, op, m, rows, n, dtype):
    return {"name": name, "op": op, "m": m, "rows": rows, "n": n, "dtype": dtype}


def _sparse(name, d, k, b, s, alpha):
    return {"name": name, "op": "sparse", "d": d, "k": k, "b": b, "s": s, "alpha": alpha}


def _norm(name, tokens, d, stream, branch, post, gates, pre, x):
    return {"name": name, "op": "norm", "tokens": tokens, "d": d, "stream": stream, "branch": branch, "post": post,
            "gates": gates, "pre": pre, "x": x}


def listed():
    return [
        # the activations of a prompt of 2048 tokens in front of a 4-bit product
        _quantize("quantize-prompt", 2048, 4096, "f16"),
        # a weight matrix at load, with rows that end inside a block of 32
        _quantize("quantize-weights-odd", 11008, 4100, "bf16"),
        # a projection of one token: the 7B-shaped down-projection, latency and weight bytes
        _linear("linear-1tok", "linear", 1, 4096, 11008, "f16"),
        # the same projection of a prompt
        _linear("linear-prompt", "linear", 2048, 4096, 11008, "f16"),
        # gate and up of a few drafted tokens, 13B-shaped, an odd number of them
        _linear("gated-37tok", "gated", 37, 13824, 5120, "bf16"),
        # gate and up of a prompt, 7B-shaped
        _linear("gated-prompt", "gated", 1024, 11008, 4096, "f16"),
        # 4-bit activations: a short chunk of a prompt ...
        _linear("linear-a4-chunk", "linear_a4", 200, 4096, 4096, "f16"),
        # ... and a long one at the 13B shape, the largest case
        _linear("linear-a4-prompt", "linear_a4", 4096, 13824, 5120, "bf16"),
        # decoding one sequence, 7B-shaped layer
        _sparse("sparse-7b-1tok", 4096, 11008, 1, 0.9, 1.0),
        # a few sequences at once, 13B-shaped layer
        _sparse("sparse-13b-4tok", 5120, 13824, 4, 0.88, 1.02),
        # between two blocks of one decoded token: the smallest call
        _norm("norm-1tok", 1, 4096, "f32", "f32", True, 1, True, "f16"),
        # the same for two prompts of 2048 tokens, a gate for each
        _norm("norm-prompt", 4096, 5120, "bf16", "bf16", True, 2, True, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above; odd sizes among them, and never more
    work than the largest listed case of its operator."""
    op = rng.choice(["quantize", "linear", "gated", "linear_a4", "sparse", "norm"])
    cap = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        if op == "quantize":
            c = _quantize(None, _log(rng, 1, 16384), _log(rng, 32, 16384), rng.choice(["f16", "bf16", "f32"]))
        elif op == "sparse":
            c = _sparse(None, 128 * _log(rng, 1, 64), _log(rng, 256, 20000), rng.randint(1, 8),
                        round(rng.uniform(0.8, 0.97), 3), rng.choice([1.0, 1.01, 1.02, 1.03]))
        elif op == "norm":
            tokens = _log(rng, 1, 8192)
            gates = rng.choice([0, 1, tokens])
            c = _norm(None, tokens, _log(rng, 64, 12288), rng.choice(["f16", "bf16", "f32"]),
                      rng.choice(["f16", "bf16", "f32"]), rng.random() < 0.7, gates, rng.random() < 0.8,
                      rng.choice(["f16", "bf16"]))
        else:
            n = _log(rng, 128, 16384)
            if rng.random() < 0.7:
                n = (n + 127) // 128 * 128
            c = _linear(None, op, _log(rng, 1, 4096), _log(rng, 64, 16384), n, rng.choice(["f16", "bf16"]))
        if _cost(c) <= cap:
            del c["name"]
            return c


def _mx_bytes(rows, n):
    return rows * n * 17 / 32


def work(case):
    op = case["op"]
    if op == "quantize":  # in and out, and the 4-bit form once each way
        values = case["rows"] * case["n"]
        return {"bytes": 2 * SIZE[case["dtype"]] * values + 2 * _mx_bytes(case["rows"], case["n"]), "flops": 0}
    if op in ("linear", "gated", "linear_a4"):
        m, rows, n = case["m"], case["rows"], case["n"]
        two = 2 if op == "gated" else 1
        e = SIZE[case["dtype"]]
        return {"bytes": two * _mx_bytes(rows, n) + e * m * n + e * m * rows, "flops": 2 * two * m * rows * n}
    if op == "sparse":
        d, k, b = case["d"], case["k"], case["b"]
        kept = (1 - case["s"]) * k
        return {"bytes": k * d / 8 + 3 * _mx_bytes(kept, d) + 2 * b * d + 4 * b * d, "flops": 6 * b * kept * d}
    t, d = case["tokens"], case["d"]
    per_value = 2 * SIZE[case["stream"]] + SIZE[case["branch"]] + (SIZE[case["x"]] if case["pre"] else 0)
    params = 4 * d * (case["gates"] + (1 if case["post"] else 0) + (1 if case["pre"] else 0))
    return {"bytes": t * d * per_value + params, "flops": 0}


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 1e15


# ---- MXFP4, plain -----------------------------------------------------------

def _blocks(v):
    """``[rows][n]`` -> ``[rows][blocks][32]``, the last block padded with zeros."""
    rows, n = v.shape
    return torch.nn.functional.pad(v, (0, -n % 32)).view(rows, -1, 32)


def _round_mx(v):
    """float32 rows -> (magnitude code values with signs, exponents X), blocked."""
    b = _blocks(v)
    amax = b.abs().amax(dim=2)
    _, e = torch.frexp(amax)  # amax = f 2^e with f in [0.5, 1)
    x = torch.where(amax > 0, (e - 3).clamp(-127, 127), torch.full_like(e, -127))
    r = torch.ldexp(b, -x.unsqueeze(2).float())
    a = r.abs().clamp(max=6.0)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = torch.round(a / step) * step  # ties to even
    return torch.copysign(q, b), x


def _values(q, x, n):
    v = torch.ldexp(q, x.unsqueeze(2).float())
    return v.flatten(1)[:, :n].contiguous()


def _pack(q, x):
    """The stored form: two codes a byte (the first in the low half), a byte a
    scale (X + 127), rows padded to 128 values."""
    rows = q.shape[0]
    a = q.abs()
    # codes 0 .. 7 of 0, 0.5, 1, 1.5, 2, 3, 4, 6
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = code | (torch.signbit(q).to(torch.uint8) << 3)
    nb = x.shape[1]
    code = torch.nn.functional.pad(code.view(rows, -1), (0, 32 * (-nb % 4)))
    packed = code[:, 0::2] | (code[:, 1::2] << 4)
    scale = torch.nn.functional.pad((x + 127).to(torch.uint8), (0, -nb % 4))
    return packed.contiguous(), scale.contiguous()


# ---- inputs -----------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _activations(g, m, n):
    """Unit-size values, with a few channels that are larger in every token."""
    channel = 1.0 + 15.0 * (torch.rand(n, generator=g, device=DEV) < 0.005).float()
    return _randn(g, m, n) * channel


def _weights(g, rows, n, extra=None):
    """MXFP4 weights: their stored form and the values it stands for."""
    w = 0.02 * _randn(g, rows, n)
    if extra is not None:
        w = w + 0.02 * extra
    q, x = _round_mx(w.half().float())
    packed, scale = _pack(q, x)
    return packed, scale, _values(q, x, n)


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    st = {"op": op}
    if op == "quantize":
        st["w"] = _activations(g, case["rows"], case["n"]).to(DTYPES[case["dtype"]])
    elif op in ("linear", "gated", "linear_a4"):
        m, rows, n = case["m"], case["rows"], case["n"]
        st["x"] = _activations(g, m, n).to(DTYPES[case["dtype"]])
        st["q"], st["s"], st["w"] = _weights(g, rows, n)
        if op == "gated":
            st["qu"], st["su"], st["wu"] = _weights(g, rows, n)
    elif op == "sparse":
        d, k, b = case["d"], case["k"], case["b"]
        # tokens around one direction; each gate row leans towards it (active) or away from it
        u = _randn(g, d)
        lean = torch.where(torch.rand(k, generator=g, device=DEV) < case["s"], -1.0, 1.0) * min(7.0 / math.sqrt(d), 0.5)
        st["x"] = (u + 0.4 * _randn(g, b, d)).half()
        st["qg"], st["sg"], st["wg"] = _weights(g, k, d, extra=lean[:, None] * u)
        st["qu"], st["su"], st["wu"] = _weights(g, k, d)
        st["qd"], st["sd"], st["wd"] = _weights(g, k, d)  # W_down^T
        st["alpha"] = case["alpha"]
        # signs of the stored gate codes, as the predictor reads them
        codes = torch.stack([st["qg"] & 8, st["qg"] >> 4 & 8], dim=2).flatten(1)[:, :d]
        st["sign"] = torch.where(codes != 0, -1.0, 1.0)
        if own:
            import paper_2411_12692_amd as si
            st["signs"] = si.pack_signs_mxfp4(st["qg"])
            st["ws"] = si.new_workspace_mxfp4(k, d, b)
    else:
        t, d = case["tokens"], case["d"]
        st["h"] = (4.0 * _activations(g, t, d)).to(DTYPES[case["stream"]])
        st["branch"] = (0.5 * _activations(g, t, d)).to(DTYPES[case["branch"]])
        st["post"] = 1.0 + 0.1 * _randn(g, d) if case["post"] else None
        st["gate"] = 0.5 + 0.2 * _randn(g, case["gates"], d) if case["gates"] else None
        st["pre"] = 1.0 + 0.1 * _randn(g, d) if case["pre"] else None
        st["scale"] = 0.22
        st["x_dtype"] = DTYPES[case["x"]]
    return st


# ---- one pass ---------------------------------------------------------------

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    import paper_2411_12692_amd as si
    op = st["op"]
    if op == "quantize":
        w = st["w"]
        q, s = si.quantize_rows_mxfp4(w)
        return si.dequantize_rows_mxfp4(q, s, w.shape[1], w.dtype)
    if op == "linear":
        return si.linear_mxfp4(st["x"], st["q"], st["s"])
    if op == "gated":
        return si.gated_linear_mxfp4(st["x"], st["q"], st["s"], st["qu"], st["su"])
    if op == "linear_a4":
        xq, xs = si.quantize_rows_mxfp4(st["x"])
        return si.linear_mxfp4_a4(xq, xs, st["q"], st["s"], st["x"].dtype)
    if op == "sparse":
        return si.predict_sparse_mlp_mxfp4(st["signs"], st["qg"], st["sg"], st["qu"], st["su"], st["qd"], st["sd"],
                                           st["x"], st["alpha"], st["ws"])
    h, x = si.norm_residual(st["h"], st["branch"], post_w=st["post"], gate=st["gate"], scale=st["scale"],
                            pre_w=st["pre"], eps=EPS, x_dtype=st["x_dtype"])
    return (h, x) if st["pre"] is not None else h


def _rms(v):
    return v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS)


def _run_plain(st):
    op = st["op"]
    if op == "quantize":
        w = st["w"]
        q, x = _round_mx(w.float())
        return _values(q, x, w.shape[1]).to(w.dtype)
    if op == "linear":
        return (st["x"].float() @ st["w"].t()).to(st["x"].dtype)
    if op == "gated":
        x = st["x"].float()
        return (torch.relu(x @ st["w"].t()) * (x @ st["wu"].t())).to(st["x"].dtype)
    if op == "linear_a4":
        q, e = _round_mx(st["x"].float())
        return (_values(q, e, st["x"].shape[1]) @ st["w"].t()).to(st["x"].dtype)
    if op == "sparse":
        x = st["x"].float()
        d = x.shape[1]
        n_neg = (d - torch.where(torch.signbit(x), -1.0, 1.0) @ st["sign"].t()).double() / 2
        alpha = float(np.float32(st["alpha"]))
        keep = (alpha * (d - n_neg) >= n_neg).any(dim=0)
        h = torch.relu(x @ st["wg"].t()) * (x @ st["wu"].t()) * keep
        return h @ st["wd"]
    branch = st["branch"].float()
    if st["post"] is not None:
        branch = _rms(branch) * st["post"]
    if st["gate"] is not None:
        branch = branch * st["gate"].repeat_interleave(branch.shape[0] // st["gate"].shape[0], dim=0)
    h = st["h"].float() + st["scale"] * branch
    if st["pre"] is None:
        return h.to(st["h"].dtype)
    return h.to(st["h"].dtype), (_rms(h) * st["pre"]).to(st["x_dtype"])


# ---- the definition in 64 bits ----------------------------------------------

_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _decode(packed, scale, n):
    """Stored MXFP4 rows -> float64 values."""
    table = torch.tensor(_E2M1 + [-v for v in _E2M1], dtype=torch.float64, device=packed.device)
    v = torch.empty(packed.shape[0], 2 * packed.shape[1], dtype=torch.float64, device=packed.device)
    v[:, 0::2] = table[(packed & 15).long()]
    v[:, 1::2] = table[(packed >> 4).long()]
    v *= torch.exp2(scale.double() - 127.0).repeat_interleave(32, dim=1)
    return v[:, :n]


def _nearest(v):
    """MXFP4 values of float64 rows, from the definition: the scale from the
    block's largest value, then the candidates one after another."""
    rows, n = v.shape
    pad = torch.zeros(rows, -n % 32, dtype=v.dtype, device=v.device)
    b = torch.cat([v, pad], dim=1).reshape(rows, -1, 32)
    top = b.abs().max(dim=2, keepdim=True).values
    x = torch.floor(torch.log2(top.clamp_min(2.0 ** -126)))
    x = torch.where(torch.exp2(x) > top, x - 1, x)      # log2 rounded up across a power of two
    x = torch.where(torch.exp2(x + 1) <= top, x + 1, x)  # or down
    unit = torch.exp2((x - 2).clamp_min(-127.0))
    a = b.abs() / unit
    best = torch.zeros_like(a)
    for i in range(1, 8):
        border = (_E2M1[i - 1] + _E2M1[i]) / 2
        up = a >= border if i % 2 == 0 else a > border  # a tie goes to the even code
        best = torch.where(up, torch.full_like(a, _E2M1[i]), best)
    out = torch.where(torch.signbit(b), -best, best) * unit
    return out.reshape(rows, -1)[:, :n]


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        return torch.cat([_nearest(part.double()) for part in st["w"].split(2048)])
    if op == "linear":
        return torch.matmul(st["x"].double(), _decode(st["q"], st["s"], case["n"]).t().contiguous())
    if op == "gated":
        x = st["x"].double()
        g = torch.matmul(x, _decode(st["q"], st["s"], case["n"]).t().contiguous())
        u = torch.matmul(x, _decode(st["qu"], st["su"], case["n"]).t().contiguous())
        return g.clamp_min(0) * u
    if op == "linear_a4":
        x = torch.cat([_nearest(part.double()) for part in st["x"].split(2048)])
        return torch.matmul(x, _decode(st["q"], st["s"], case["n"]).t().contiguous())
    if op == "sparse":
        d = case["d"]
        x = st["x"].double()
        gate = _decode(st["qg"], st["sg"], d)
        y = torch.zeros(case["b"], d, dtype=torch.float64, device=DEV)
        kept = torch.zeros(case["k"], dtype=torch.bool, device=DEV)
        for t in range(case["b"]):  # Eq. (2) token by token; the kept rows are shared
            opposite = (torch.signbit(gate) != torch.signbit(x[t])).sum(dim=1)
            kept |= ~(np.float64(np.float32(case["alpha"])) * (d - opposite) < opposite)
        rows = kept.nonzero().flatten()
        gate = gate[rows]
        up = _decode(st["qu"][rows], st["su"][rows], d)
        down = _decode(st["qd"][rows], st["sd"][rows], d)
        for t in range(case["b"]):
            h = (gate @ x[t]).clamp_min(0) * (up @ x[t])
            y[t] = h @ down
        return y
    v = st["branch"].double()
    if case["post"]:
        v = v / torch.sqrt(v.square().sum(dim=1, keepdim=True) / case["d"] + EPS) * st["post"].double()
    if case["gates"]:
        per = case["tokens"] // case["gates"]
        v = (v.view(case["gates"], per, -1) * st["gate"].double()[:, None, :]).view_as(v)
    h = st["h"].double() + st["scale"] * v
    if not case["pre"]:
        return h
    return h, h / torch.sqrt(h.square().sum(dim=1, keepdim=True) / case["d"] + EPS) * st["pre"].double()
