"""Cases of the 8-bit integer layers with scales for each token and channel, and of the log probabilities of given tokens.

Codes are int8 rows at a pitch that is a multiple of 16 bytes, scales float32 for each row: weights have a row for each channel, activations
one for each token.  A row's scale is max|x| / 127, its codes round(x / scale), the product float(sum of codes) * channel's scale *
token's scale.  The plain forms compute in 32 bits with elementary torch operations and round once (quotients in 64 bits: codes next to a
border); `exact` does the same in 64 bits from the formulas.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ACTS = {"identity": 0, "relu": 1, "silu": 2, "gelu": 3, "sigmoid": 4}


def listed():
    return [
        # a small test layer's weights: the call's latency
        dict(name="quantize_256x256", op="quantize", R=256, N=256, I=256, src="fp32", gather=False),
        # an LLM projection's weights from a 16-bit checkpoint, each channel its scale
        dict(name="quantize_11008x4096", op="quantize", R=11008, N=11008, I=4096, src="bf16", gather=False),
        # a batch of tokens in the order of their experts, some chosen several times
        dict(name="quantize_t1001_k6_gathered", op="quantize", R=1001, N=6006, I=1408, src="fp16", gather=True),
        # decoding: one token, whose codes several projections share
        dict(name="linear_4096_11008_t1", op="linear", O=11008, I=4096, T=1, dtype="bf16", bias=False, act="identity", from_x=False),
        # a small batch of requests through the other projection, quantized on the way
        dict(name="linear_11008_4096_t13", op="linear", O=4096, I=11008, T=13, dtype="fp16", bias=True, act="identity", from_x=True),
        # the head on a batch of positions: logits in 32 bits
        dict(name="linear_4096_32000_t200_fp32", op="linear", O=32000, I=4096, T=200, dtype="fp32", bias=False, act="identity", from_x=True),
        # a prompt
        dict(name="linear_4096_11008_t4096", op="linear", O=11008, I=4096, T=4096, dtype="bf16", bias=True, act="silu", from_x=False),
        # decoding with many small experts: 8 requests, 6 experts each
        dict(name="expert_64x2048_1408_t8", op="expert", E=64, O=1408, I=2048, T=8, k=6, dtype="bf16", bias=False, act="silu"),
        # prompts over a few large experts
        dict(name="expert_8x4096_11008_t4096", op="expert", E=8, O=11008, I=4096, T=4096, k=2, dtype="bf16", bias=False, act="silu"),
        # one position of one request, some alternatives
        dict(name="logprobs_t1_v32000", op="logprobs", T=1, V=32000, dtype="bf16", n=1, top=5, entropy=True, masked=False, scale=1.0),
        # several candidates for each of some positions, an odd vocabulary, masked tokens, at a temperature
        dict(name="logprobs_t201_v50001_masked", op="logprobs", T=201, V=50001, dtype="fp32", n=4, top=20, entropy=True, masked=True, scale=1.25),
        # scoring long texts
        dict(name="logprobs_t2048_v128000", op="logprobs", T=2048, V=128000, dtype="bf16", n=1, top=10, entropy=True, masked=False, scale=1.0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "expert", "expert", "logprobs", "logprobs"])
    dtype, bias, act = rng.choice(["bf16", "fp16", "fp32"]), rng.random() < 0.5, rng.choice(list(ACTS))
    if op == "quantize":
        gather = rng.random() < 0.5
        R = _log(rng, 1, 11008)
        return dict(op=op, R=R, N=_log(rng, 1, 11008) if gather else R, I=_log(rng, 1, 4096), src=dtype, gather=gather)
    if op == "linear":
        return dict(op=op, O=_log(rng, 1, 11008), I=_log(rng, 16, 4096), T=_log(rng, 1, 4096), dtype=dtype, bias=bias, act=act, from_x=rng.random() < 0.5)
    if op == "expert":
        E = _log(rng, 2, 64)
        return dict(op=op, E=E, O=_log(rng, 33, 2048), I=_log(rng, 33, 2048), T=_log(rng, 1, 2048), k=rng.randint(1, min(8, E)), dtype=dtype, bias=bias, act=act)
    return dict(op=op, T=_log(rng, 1, 2048), V=_log(rng, 2, 128000), dtype=dtype, n=rng.randint(1, 8), top=rng.randint(0, 20), entropy=rng.random() < 0.5,
                masked=rng.random() < 0.5, scale=rng.choice([1.0, 0.5, 1.25]))


# ---- inputs -----------------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 6007 + 29)
    return g


def _pitched(shape, dtype=torch.int8):
    """An array whose rows lie at a multiple of 16 values."""
    return torch.zeros((*shape[:-1], -(-shape[-1] // 16) * 16), dtype=dtype, device=DEV)[..., :shape[-1]]


def _weights(gen, R, I):
    """Rows of different size, as trained projections have."""
    return torch.randn((R, I), generator=gen, device=DEV) * 0.02 * torch.exp2(torch.rand((R, 1), generator=gen, device=DEV) * 4 - 2)


def _acts(gen, T, I, h):
    x = torch.randn((T, I), generator=gen, device=DEV)
    many = torch.rand((I,), generator=gen, device=DEV) < 0.005
    return torch.where(many, x * 20, x).to(h)


def _in_codes(x):
    """scale and codes (as numbers) of rows x."""
    x = x.double()
    s = (x.abs().amax(-1) / 127).float()
    d = torch.where(s == 0, 1, s.double())[..., None]
    return s, torch.where(s[..., None] == 0, 0, torch.round(x / d).clamp(-127, 127)).float()


def _held(gen, c):
    """A layer as a checkpoint holds it."""
    E, O, I = c.get("E", 1), c["O"], c["I"]
    codes, scales = _pitched((E, O, I)), torch.empty((E, O), dtype=torch.float32, device=DEV)
    for e in range(E):
        s, q = _in_codes(_weights(gen, O, I))
        codes[e], scales[e] = q.to(torch.int8), s
    return codes, scales


def _choice(gen, T, k, E):
    """k different experts per token, some of them more popular than others."""
    liking = torch.randn((E,), generator=gen, device=DEV) * 0.7
    gumbel = -torch.log(-torch.log(torch.rand((T, E), generator=gen, device=DEV).clamp(1e-7, 1 - 1e-7)))
    return (gumbel + liking).topk(k, dim=1).indices


def prepare(case, seed):
    gen, c = _gen(seed), case
    s = {"case": case}
    if c["op"] == "quantize":
        s["x"] = _weights(gen, c["R"], c["I"]).to(TYPES[c["src"]])
        s["rows"] = torch.randint(0, c["R"], (c["N"],), generator=gen, device=DEV, dtype=torch.int32) if c["gather"] else None
        s["xq"], s["sx"] = _pitched((c["N"], c["I"])), torch.empty(c["N"], dtype=torch.float32, device=DEV)
        s["values"] = torch.empty((c["N"], c["I"]), dtype=torch.float32, device=DEV)
    elif c["op"] == "linear":
        h = TYPES[c["dtype"]]
        s["codes"], s["scales"] = _held(gen, c)
        s["bias"] = (torch.randn((c["O"],), generator=gen, device=DEV) * 0.1).to(h) if c["bias"] else None
        s["x"] = _acts(gen, c["T"], c["I"], h)
        s["xq"], s["sx"] = _pitched((c["T"], c["I"])), torch.empty(c["T"], dtype=torch.float32, device=DEV)
        if not c["from_x"]:   # another call has quantized them
            s["sx"], q = _in_codes(s.pop("x"))
            s["xq"].copy_(q)
        s["y"] = torch.empty((c["T"], c["O"]), dtype=h, device=DEV)
    elif c["op"] == "expert":
        h, N = TYPES[c["dtype"]], c["T"] * c["k"]
        s["codes"], s["scales"] = _held(gen, c)
        s["bias"] = (torch.randn((c["E"], c["O"]), generator=gen, device=DEV) * 0.1).to(h) if c["bias"] else None
        s["x"] = _acts(gen, c["T"], c["I"], h)
        choice = _choice(gen, c["T"], c["k"], c["E"]).reshape(-1)
        s["offsets"] = torch.zeros(c["E"] + 1, dtype=torch.int32, device=DEV)
        s["offsets"][1:] = torch.bincount(choice, minlength=c["E"]).cumsum(0)
        s["rows"] = (torch.sort(choice, stable=True).indices // c["k"]).to(torch.int32)
        s["most"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())   # (only the plain form pads to it)
        s["xq"], s["sx"] = _pitched((N, c["I"])), torch.empty(N, dtype=torch.float32, device=DEV)
        s["y"] = torch.empty((N, c["O"]), dtype=h, device=DEV)
    else:
        T, V, h = c["T"], c["V"], TYPES[c["dtype"]]
        l = torch.randn((T, V), generator=gen, device=DEV) * 2.5
        sure = torch.randint(0, V, (T,), generator=gen, device=DEV)
        l[torch.arange(T, device=DEV), sure] += torch.rand((T,), generator=gen, device=DEV) * 16
        s["tokens"] = torch.randint(0, V, (T, c["n"]), generator=gen, device=DEV)
        s["tokens"][:, 0] = torch.where(torch.rand((T,), generator=gen, device=DEV) < 0.6, sure, s["tokens"][:, 0])
        if c["masked"]:   # a grammar's mask, a padded vocabulary, positions that are padding
            l[torch.rand((T, V), generator=gen, device=DEV) < 0.3] = -math.inf
            l[:, V - V // 50:] = -math.inf
            if T > 3:
                l[T - 2] = -math.inf
                s["tokens"][T - 1] = -1
        s["logits"], s["tokens"] = l.to(h), s["tokens"].to(torch.int32)
        s["logprobs"] = torch.empty((T, c["n"]), dtype=torch.float32, device=DEV)
        s["entropy"] = torch.empty(T, dtype=torch.float32, device=DEV) if c["entropy"] else None
        s["top"] = torch.empty((T, c["top"]), dtype=torch.int32, device=DEV) if c["top"] else None
        s["top_logprobs"] = torch.empty((T, c["top"]), dtype=torch.float32, device=DEV) if c["top"] else None
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------------------
def _act32(v, act):
    if act == "relu":
        return torch.clamp(v, min=0)
    if act == "silu":
        return v / (1 + torch.exp(-v))
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * 0.7071067811865476))
    if act == "sigmoid":
        return 1 / (1 + torch.exp(-v))
    return v


def _plain_quantize(s):
    x = s["x"] if s["rows"] is None else s["x"][s["rows"].long()]
    scales, q = _in_codes(x)
    return {"values": q * scales[:, None], "scales": scales}


def _plain_linear(s):
    sx, q = _in_codes(s["x"]) if s["case"]["from_x"] else (s["sx"], s["xq"].float())
    v = q @ s["codes"][0].float().t() * s["scales"][0] * sx[:, None]
    if s["bias"] is not None:
        v = v + s["bias"].float()
    return _act32(v, s["case"]["act"]).to(s["y"].dtype)


def _plain_expert(s):
    c, off = s["case"], s["offsets"]
    N = c["T"] * c["k"]
    slot = torch.arange(N, device=DEV)
    e = (slot[:, None] >= off[None, 1:]).sum(1)
    at = slot - off[e].long()
    sx, q = _in_codes(s["x"])
    padded = torch.zeros((c["E"], s["most"], c["I"]), dtype=torch.float32, device=DEV)
    padded[e, at] = q[s["rows"].long()]
    v = torch.bmm(padded, s["codes"].float().transpose(1, 2))[e, at] * s["scales"][e] * sx[s["rows"].long(), None]
    if s["bias"] is not None:
        v = v + s["bias"].float()[e]
    return _act32(v, c["act"]).to(s["y"].dtype)


def _plain_logprobs(s):
    c, l = s["case"], s["logits"].float()
    none = torch.isneginf(l).all(1, keepdim=True)
    m = torch.where(none, 0, l.amax(1, keepdim=True))
    d = (l - m) * c["scale"]
    e = torch.exp(d)
    total = torch.where(none, 1, e.sum(1, keepdim=True))
    log_total = torch.log(total)
    out = {}
    tokens = s["tokens"].long()
    inside = (tokens >= 0) & (tokens < c["V"])
    out["logprobs"] = torch.where(inside, torch.gather(d, 1, torch.where(inside, tokens, 0)) - log_total, 0)
    if c["entropy"]:
        terms = torch.where(e == 0, 0, e * d).sum(1, keepdim=True)
        out["entropy"] = torch.where(none, 0, log_total - terms / total)[:, 0]
    if c["top"]:
        values, ids = torch.sort(l, dim=1, descending=True, stable=True)
        pad = max(0, c["top"] - c["V"])
        values = torch.nn.functional.pad(values[:, :c["top"]], (0, pad), value=-math.inf)
        ids = torch.nn.functional.pad(ids[:, :c["top"]], (0, pad), value=-1)
        out["top"] = torch.where(torch.isneginf(values), -1, ids).to(torch.int32)
        out["top_logprobs"] = (values - m) * c["scale"] - log_total
    return out


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2311_15806_b200 import binding as B
        if c["op"] == "quantize":
            B.pipe_int8_quantize(s["x"], s["xq"], s["sx"], rows=s["rows"], values=s["values"])
            return {"values": s["values"], "scales": s["sx"]}
        if c["op"] == "logprobs":
            B.pipe_token_logprobs(s["logits"], s["tokens"], s["logprobs"], entropy=s["entropy"], top=s["top"], top_logprobs=s["top_logprobs"], scale=c["scale"])
            return {k: s[k] for k in ("logprobs", "entropy", "top", "top_logprobs") if s[k] is not None}
        if "desc" not in s:   # a program keeps the layer's descriptor
            s["desc"] = B.make_int8_desc(c["O"], c["I"], dtype=TYPES[c["dtype"]], experts=c.get("E", 1))
        if c["op"] == "linear":
            if c["from_x"]:
                B.pipe_int8_quantize(s["x"], s["xq"], s["sx"])
            B.pipe_int8_linear(s["desc"], s["codes"], s["scales"], s["xq"], s["sx"], s["y"], bias=s["bias"], activation=ACTS[c["act"]])
            return s["y"]
        B.pipe_int8_quantize(s["x"], s["xq"], s["sx"], rows=s["rows"])
        B.pipe_int8_expert_linear(s["desc"], s["codes"], s["scales"], s["xq"], s["sx"], s["offsets"], s["y"], bias=s["bias"], activation=ACTS[c["act"]])
        return s["y"]
    return {"quantize": _plain_quantize, "linear": _plain_linear, "expert": _plain_expert, "logprobs": _plain_logprobs}[c["op"]](s)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------------------
def work(case):
    c = case
    size = lambda t: 4 if t == "fp32" else 2  # noqa: E731
    if c["op"] == "quantize":
        read = min(c["R"], c["N"])
        return {"bytes": read * c["I"] * size(c["src"]) + c["N"] * (c["I"] * 5 + 4) + (4 * c["N"] if c["gather"] else 0), "flops": 4 * c["N"] * c["I"]}
    if c["op"] == "logprobs":
        return {"bytes": c["T"] * (c["V"] * size(c["dtype"]) + 8 * c["n"] + 8 * c["top"] + (4 if c["entropy"] else 0)), "flops": 4 * c["T"] * c["V"]}
    E, O, I, h = c.get("E", 1), c["O"], c["I"], size(c["dtype"])
    layer = O * I + 4 * O + (h * O if c["bias"] else 0)
    if c["op"] == "linear":
        x = c["T"] * I * h if c["from_x"] else c["T"] * (I + 4)
        return {"bytes": layer + x + c["T"] * O * h, "flops": 2 * c["T"] * I * O}
    n = c["T"] * c["k"]
    # the experts that some row has chosen, were all equally liked
    used = min(E, max(1, round(E * (1 - (1 - c["k"] / E) ** c["T"]))))
    return {"bytes": used * layer + c["T"] * I * h + n * O * h + 4 * (E + 1) + 4 * n, "flops": 2 * n * I * O}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------------------
def _act64(v, act):
    if act == "relu":
        return v.clamp(min=0)
    if act == "gelu":
        return v * torch.special.ndtr(v)
    if act == "sigmoid":
        return torch.special.expit(v)
    return v * torch.special.expit(v) if act == "silu" else v


def _codes64(x):
    """float64 codes and scales of rows: the least whole number that is not below x / s - 1/2, an odd tie one lower."""
    s = torch.true_divide(x.abs().max(1).values.double(), 127.0).to(torch.float32).double()
    q = (x.double() / s[:, None]).nan_to_num(0)
    up = torch.ceil(q - 0.5)
    up = torch.where((up - q == -0.5) & (torch.remainder(up, 2) == 1), up + 1, up)
    return torch.minimum(torch.maximum(up, up.new_tensor(-127.0)), up.new_tensor(127.0)), s


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "quantize":
        q, sc = _codes64(s["x"] if s["rows"] is None else s["x"].index_select(0, s["rows"].long()))
        return {"values": q * sc[:, None], "scales": sc}
    if c["op"] == "logprobs":
        z = s["logits"].double() * c["scale"]
        alive = (z > -math.inf).any(1)
        norm = torch.logsumexp(z, 1)                       # -inf for a row of nothing
        lp = torch.where(alive[:, None], z - norm[:, None], -math.inf)
        out = {"logprobs": torch.zeros((c["T"], c["n"]), dtype=torch.float64, device=DEV)}
        for j in range(c["n"]):
            t = s["tokens"][:, j].long()
            ok = (t >= 0) & (t < c["V"])
            out["logprobs"][ok, j] = lp[ok].gather(1, t[ok, None])[:, 0]
        if c["entropy"]:
            out["entropy"] = torch.special.entr(torch.exp(lp)).sum(1)
        if c["top"]:
            out["top"] = torch.full((c["T"], c["top"]), -1, dtype=torch.int32, device=DEV)
            out["top_logprobs"] = torch.full((c["T"], c["top"]), -math.inf, dtype=torch.float64, device=DEV)
            left = s["logits"].double()
            for j in range(min(c["top"], c["V"])):         # the largest that is left, the first of equal ones
                best = left.amax(1)
                at = (left == best[:, None]).int().argmax(1)
                some = best > -math.inf
                out["top"][some, j] = at[some].int()
                out["top_logprobs"][some, j] = lp[some].gather(1, at[some, None])[:, 0]
                left.scatter_(1, at[:, None], -math.inf)
        return out
    if c["op"] == "linear":
        q, sx = _codes64(s["x"]) if c["from_x"] else (s["xq"].double(), s["sx"].double())
        v = torch.einsum("ti,oi->to", q, s["codes"][0].double()) * torch.outer(sx, s["scales"][0].double())
        return _act64(v + s["bias"].double() if s["bias"] is not None else v, c["act"])
    off, out = s["offsets"].tolist(), torch.empty(s["y"].shape, dtype=torch.float64, device=DEV)
    q, sx = _codes64(s["x"])
    for e in range(c["E"]):
        a, b = off[e], off[e + 1]
        if b > a:
            r = s["rows"][a:b].long()
            v = q[r] @ s["codes"][e].double().t() * torch.outer(sx[r], s["scales"][e].double())
            out[a:b] = _act64(v + s["bias"][e].double() if s["bias"] is not None else v, c["act"])
    return out
