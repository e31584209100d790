"""The 8-bit operators of this library as cases that can be timed and compared: rows quantised to int8 with one scale each
(behind a residual addition and an RMSNorm, or as they are), the int8 matrix product with a scale for each token and each
channel, and the transformer MLP block that the three make together.

``run`` computes a case's operator in elementary fp32 torch operations, or, where ``own`` is true, through the public Python
entry points of ``paper_2608_03537_b200``.  A user's program keeps the quantised weights and the output buffers, so ``prepare``
makes them.  Values: activations N(0, 1) with one channel in 64 twenty times as large, as transformers have them; weights
N(0, 1 / fan-in); biases U(-0.1, 0.1); gains N(1, 0.02).  The int8 rows are returned as the values that they stand for, in
bf16, as the library's bf16 kernels would take them.

    rows     h = x + residual;  y = h * rsqrt(mean(h^2) + eps) * gamma  (or y = x);  s = max|y| / 127;  q = rint(y / s)
    product  Y = act(sa[i] * sb[j] * sum_k A[i, k] * B[j, k] + bias[j]) + residual
    mlp      rows (norm) -> product (bias, GELU) -> rows -> product (bias, residual h)
"""
import math

import torch

own = False

EPS = 1e-5
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # the norm in front of a layer, one token: the latency of a call
        {"name": "norm_token", "path": "rows", "M": 1, "N": 4096, "dtype": "bf16", "norm": True, "residual": True},
        # a short prompt through a layer whose width fits nothing, fp16
        {"name": "norm_ragged", "path": "rows", "M": 777, "N": 1000, "dtype": "f16", "norm": True, "residual": False},
        # the norm in front of a layer, 8192 tokens of prefill
        {"name": "norm_prefill", "path": "rows", "M": 8192, "N": 4096, "dtype": "bf16", "norm": True, "residual": True},
        # one decoding step's hidden layer of a wide MLP, kept in fp32
        {"name": "quantize_step_f32", "path": "rows", "M": 40, "N": 16384, "dtype": "f32", "norm": False, "residual": False},
        # the hidden layer of an MLP, prefill
        {"name": "quantize_hidden", "path": "rows", "M": 8192, "N": 16384, "dtype": "bf16", "norm": False, "residual": False},
        # a linear layer for one token: the weights are all there is to move
        {"name": "product_token", "path": "product", "batch": 1, "M": 1, "N": 4096, "K": 4096, "dtype": "bf16", "act": "none", "bias": False, "residual": False},
        # a decoding step of 40 sequences through the wide layer of an MLP
        {"name": "product_step", "path": "product", "batch": 1, "M": 40, "N": 16384, "K": 4096, "dtype": "bf16", "act": "gelu_tanh", "bias": True, "residual": False},
        # a few hundred tokens, sizes that fit nothing, fp16
        {"name": "product_ragged", "path": "product", "batch": 1, "M": 333, "N": 2824, "K": 1032, "dtype": "f16", "act": "none", "bias": True, "residual": True},
        # scores of 8 sequences x 12 heads over 504 positions, a scale for each query and key, fp32 for the softmax behind
        {"name": "product_scores", "path": "product", "batch": 96, "M": 504, "N": 504, "K": 64, "dtype": "f32", "act": "none", "bias": False, "residual": False},
        # a linear layer, 8192 tokens of prefill
        {"name": "product_prefill", "path": "product", "batch": 1, "M": 8192, "N": 4096, "K": 4096, "dtype": "bf16", "act": "gelu_tanh", "bias": True, "residual": True},
        # an MLP block of a transformer, one decoding step of 40 sequences
        {"name": "mlp_step", "path": "mlp", "M": 40, "N": 4096, "H": 16384, "dtype": "bf16"},
        # the same block, 4096 tokens of prefill
        {"name": "mlp_prefill", "path": "mlp", "M": 4096, "N": 4096, "H": 16384, "dtype": "bf16"},
    ]


def _log(rng, lo, hi, step=1):
    """An integer multiple of `step` in [lo, hi], spread evenly over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(v / step)) * step))


def draw(rng):
    path = rng.choice(["rows", "rows", "product", "product", "product", "mlp"])
    flag = lambda: rng.random() < 0.5  # noqa: E731
    if path == "rows":
        m = _log(rng, 1, 8192)
        n = _log(rng, 64, min(65536, (1 << 27) // m), rng.choice([1, 8, 8, 64]))
        norm = flag()
        return {"path": path, "M": m, "N": n, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "norm": norm, "residual": norm and flag()}
    if path == "product":
        batch = 1 if rng.random() < 0.7 else _log(rng, 2, 96)
        m = _log(rng, 1, 8192 if batch == 1 else 1024)
        n = _log(rng, 64, 16384 if batch == 1 else 1024, rng.choice([1, 8, 8, 64]))
        k = _log(rng, 32, 16384 if batch == 1 else 256, rng.choice([1, 8, 8, 64]))
        n = max(64, min(n, (1 << 36) // (m * k * batch)))
        return {"path": path, "batch": batch, "M": m, "N": n, "K": k, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]),
                "act": rng.choice(["none", "none", "relu", "gelu_tanh", "tanh", "sigmoid"]), "bias": flag(), "residual": flag()}
    return {"path": path, "M": _log(rng, 1, 4096), "N": _log(rng, 256, 4096, 8), "H": _log(rng, 256, 16384, 8), "dtype": rng.choice(["bf16", "bf16", "f16"])}


class _Make:
    """Device tensors from one seeded generator."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape, mean=0.0, std=1.0):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=self.g)

    def uniform(self, n, lo=-0.1, hi=0.1):
        return torch.empty(n, dtype=torch.float32, device="cuda").uniform_(lo, hi, generator=self.g)

    def activations(self, *shape):
        """N(0, 1) with one channel in 64 twenty times as large."""
        x = self.normal(*shape)
        loud = torch.empty(shape[-1], dtype=torch.float32, device="cuda").uniform_(0, 1, generator=self.g) < 1 / 64
        return x.mul_(torch.where(loud, 20.0, 1.0))

    def quantized(self, x):
        """int8 rows with a leading dimension that is a multiple of 16 bytes, and their fp32 scales."""
        scale = x.abs().amax(-1) / 127
        q = torch.zeros(*x.shape[:-1], (x.shape[-1] + 15) // 16 * 16, dtype=torch.int8, device="cuda")[..., : x.shape[-1]]
        q.copy_((x / scale.unsqueeze(-1)).round_())
        return q, scale

    def weights(self, *shape):
        return self.quantized(self.normal(*shape, std=shape[-1] ** -0.5))


def _rows(m, n, dtype, batch=None):
    """An uninitialised [m, n] (or [batch, m, n]) buffer whose rows start on 16-byte boundaries."""
    per = 16 // torch.empty((), dtype=dtype).element_size()
    lead = (m,) if batch is None else (batch, m)
    return torch.empty(*lead, (n + per - 1) // per * per, dtype=dtype, device="cuda")[..., :n]


def prepare(case, seed):
    g, t = _Make(seed), _TYPES[case["dtype"]]
    s = {"case": case}

    def put(x):
        return _rows(x.shape[-2], x.shape[-1], t, x.shape[0] if x.dim() == 3 else None).copy_(x)

    if case["path"] == "rows":
        M, N = case["M"], case["N"]
        s["x"] = put(g.activations(M, N))
        s["residual"] = put(g.activations(M, N)) if case["residual"] else None
        s["gamma"] = g.normal(N, mean=1.0, std=0.02).to(t) if case["norm"] else None
        s["h"] = _rows(M, N, t) if case["residual"] else None
        s["q"], s["scale"], s["values"] = _rows(M, N, torch.int8), torch.empty(M, dtype=torch.float32, device="cuda"), _rows(M, N, torch.bfloat16)
        return s
    if case["path"] == "product":
        batch, M, N, K = case["batch"], case["M"], case["N"], case["K"]
        lead = () if batch == 1 else (batch,)
        s["A"], s["scale_a"] = g.quantized(g.activations(*lead, M, K))
        s["B"], s["scale_b"] = g.weights(*lead, N, K)
        s["bias"] = g.uniform(N).to(t) if case["bias"] else None
        s["residual"] = put(g.activations(*lead, M, N)) if case["residual"] else None
        s["Y"] = _rows(M, N, t, batch if lead else None)
        return s
    M, N, H = case["M"], case["N"], case["H"]
    s["x"], s["residual"], s["gamma"] = put(g.activations(M, N)), put(g.activations(M, N)), g.normal(N, mean=1.0, std=0.02).to(t)
    s["W1"], s["scale_1"] = g.weights(H, N)
    s["W2"], s["scale_2"] = g.weights(N, H)
    s["b1"], s["b2"] = g.uniform(H).to(t), g.uniform(N).to(t)
    s["h"], s["hidden"], s["Y"] = _rows(M, N, t), _rows(M, H, t), _rows(M, N, t)
    s["q"], s["scale_q"] = _rows(M, N, torch.int8), torch.empty(M, dtype=torch.float32, device="cuda")
    s["p"], s["scale_p"] = _rows(M, H, torch.int8), torch.empty(M, dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _norm(h, gamma):
    return h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * gamma.float()


def _quantize(y):
    """(whole numbers as fp32, scale) of fp32 rows."""
    scale = y.abs().amax(-1, keepdim=True) / 127
    return torch.where(scale > 0, torch.round(y / scale), 0.0), scale


def _act(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "tanh":
        return torch.tanh(z)
    return 1 / (1 + torch.exp(-z)) if name == "sigmoid" else z


def _product(a, scale_a, b, scale_b, bias, residual, act):
    z = (a @ b.float().mT) * scale_a * scale_b.unsqueeze(-2)
    if bias is not None:
        z = z + bias.float()
    z = _act(z, act)
    return z if residual is None else z + residual


def _plain(s):
    case = s["case"]
    t = _TYPES[case["dtype"]]
    if case["path"] == "rows":
        h = s["x"].float()
        if case["residual"]:
            h = h + s["residual"].float()
        q, scale = _quantize(_norm(h, s["gamma"]) if case["norm"] else h)
        return {"h": h.to(t) if case["residual"] else None, "values": (q * scale).to(torch.bfloat16), "scale": scale.squeeze(-1)}
    if case["path"] == "product":
        r = None if s["residual"] is None else s["residual"].float()
        return _product(s["A"].float(), s["scale_a"].unsqueeze(-1), s["B"], s["scale_b"], s["bias"], r, case["act"]).to(t)
    h = s["x"].float() + s["residual"].float()
    q, scale = _quantize(_norm(h, s["gamma"]))
    h = h.to(t)
    hidden = _product(q, scale, s["W1"], s["scale_1"], s["b1"], None, "gelu_tanh").to(t)
    q, scale = _quantize(hidden.float())
    return {"h": h, "Y": _product(q, scale, s["W2"], s["scale_2"], s["b2"], h.float(), "none").to(t)}


# ---------------------------------------------------------------------------------------------- the library's entry points
def _library(s):
    import paper_2608_03537_b200 as cf
    case = s["case"]
    if case["path"] == "rows":
        if case["norm"]:
            cf.rmsnorm_quantize_rows(s["x"], s["q"], s["scale"], residual=s["residual"], gamma=s["gamma"], h=s["h"], values=s["values"], eps=EPS)
        else:
            cf.quantize_rows(s["x"], s["q"], s["scale"], values=s["values"])
        return {"h": s["h"], "values": s["values"], "scale": s["scale"]}
    if case["path"] == "product":
        return cf.gemm_q8(s["A"], s["scale_a"], s["B"], s["scale_b"], s["Y"], bias=s["bias"], residual=s["residual"], activation=case["act"])
    cf.rmsnorm_quantize_rows(s["x"], s["q"], s["scale_q"], residual=s["residual"], gamma=s["gamma"], h=s["h"], eps=EPS)
    cf.gemm_q8(s["q"], s["scale_q"], s["W1"], s["scale_1"], s["hidden"], bias=s["b1"], activation="gelu_tanh")
    cf.quantize_rows(s["hidden"], s["p"], s["scale_p"])
    cf.gemm_q8(s["p"], s["scale_p"], s["W2"], s["scale_2"], s["Y"], bias=s["b2"], residual=s["h"])
    return {"h": s["h"], "Y": s["Y"]}


def run(state):
    if own:
        return _library(state)
    return _plain(state)


def work(case):
    e, M, N = _BYTES[case["dtype"]], case["M"], case["N"]
    if case["path"] == "rows":   # x, residual, h; the 8-bit rows and the values that they stand for; gains, scales
        return {"bytes": M * N * (e * (3 if case["residual"] else 1) + 1 + 2) + (e * N if case["norm"] else 0) + 4 * M, "flops": 8 * M * N}
    if case["path"] == "product":
        batch, K = case["batch"], case["K"]
        per = M * K + N * K + 4 * (M + N) + M * N * e * (2 if case["residual"] else 1)
        return {"bytes": batch * per + (e * N if case["bias"] else 0), "flops": 2 * batch * M * N * K}
    H = case["H"]   # the rows between the four calls stay out: a larger fusion would not move them
    return {"bytes": 2 * N * H + 4 * (N + H) + e * (2 * N + H) + 4 * M * N * e, "flops": 4 * M * N * H}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    if 4 * case["M"] * case["N"] * case.get("H", 0) + 2 * case.get("batch", 1) * case["M"] * case["N"] * case.get("K", 0) > 3e12:
        return None
    s = prepare(case, seed)
    f = lambda name: None if s.get(name) is None else s[name].to(torch.float64)  # noqa: E731

    def rows(y):
        top = torch.linalg.vector_norm(y, ord=math.inf, dim=-1)
        step = top / 127
        codes = torch.zeros_like(y)
        some = top > 0
        codes[some] = torch.round(127 * y[some] / top[some, None])
        return codes, step

    def normed(v):
        return v / torch.sqrt((v * v).sum(-1) / v.shape[-1] + EPS)[:, None] * f("gamma")

    def gelu(z):
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))

    def linear(codes, step, w, step_w):
        return torch.einsum("...ik,...jk->...ij", codes, w) * (step[..., :, None] * step_w[..., None, :])

    if case["path"] == "rows":
        v = f("x") + (f("residual") if case["residual"] else 0)
        codes, step = rows(normed(v) if case["norm"] else v)
        return {"h": v if case["residual"] else None, "values": codes * step[:, None], "scale": step}
    if case["path"] == "product":
        z = linear(f("A"), f("scale_a"), f("B"), f("scale_b"))
        if case["bias"]:
            z += f("bias")
        act = {"none": lambda v: v, "relu": lambda v: torch.where(v > 0, v, 0.0), "gelu_tanh": gelu, "tanh": torch.tanh, "sigmoid": torch.sigmoid}[case["act"]]
        z = act(z)
        return z + f("residual") if case["residual"] else z
    v = f("x") + f("residual")
    hidden = gelu(linear(*rows(normed(v)), f("W1"), f("scale_1")) + f("b1")).to(s["x"].dtype)   # a tensor of the block: held in its type
    h = v.to(s["x"].dtype).to(torch.float64)
    return {"h": v, "Y": linear(*rows(hidden.to(torch.float64)), f("W2"), f("scale_2")) + f("b2") + h}
