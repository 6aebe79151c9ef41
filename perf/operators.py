"""Cases that the transformer-block operators of this library are measured on: matrix products with an epilogue, the gated
feed-forward block and attention to an encoder's states, forwards and backwards, beside the convolutions of perf/cases.py.

``own`` false: every operator in its plain form, elementary torch operations in fp32, rounded once at the end.  ``own`` true:
the calls that a program makes of ``paper_2412_05781_amd.binding``, with outputs and workspaces kept between the calls.

    linear      y = act(x w^T + bias) + residual                                x[M,K] w[N,K] bias[N] residual,y[M,N]
    glu         h = (x wu^T + bu) * act(x wg^T + bg), w = [wu; wg], bias = [bu; bg]     x[M,K] w[2N,K] bias[2N] h[M,N]
    attention   o = softmax(q k^T / sqrt(D)) v over the valid keys of a row of the batch; no valid key: zero
                q,o[B,Sq,H,D] k,v[B,Skv,Hkv,D], query head h reads key head h // (H // Hkv)
and their gradients.  bias is fp32, everything else of the case's type; key lengths are int32 [B], key masks uint8 [B,Skv].
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = ("none", "silu", "gelu", "gelu_tanh")
DEV = "cuda:0"


def _linear(name, M, K, N, dtype, act="none", residual=False, backward=False):
    return _named(name, dict(op="linear", backward=backward, M=M, K=K, N=N, dtype=dtype, act=act, residual=residual))


def _glu(name, M, K, N, dtype, act="gelu", backward=False):
    return _named(name, dict(op="glu", backward=backward, M=M, K=K, N=N, dtype=dtype, act=act))


def _attention(name, B, Sq, Skv, H, Hkv, D, dtype, keys="all", backward=False):
    return _named(name, dict(op="attention", backward=backward, B=B, Sq=Sq, Skv=Skv, H=H, Hkv=Hkv, D=D, dtype=dtype, keys=keys))


def _named(name, case):
    return dict(case, name=name) if name else case


def listed():
    return [
        # time embedding of a guidance batch: two rows against a square weight, latency and a stream of weights
        _linear("time_embedding", 2, 1280, 1280, "f16", act="silu"),
        # output projection of an attention at full latent size (64x64, guidance batch), skip connection in the epilogue
        _linear("attention_out_64", 2 * 4096, 320, 320, "f16", residual=True),
        # second product of the feed-forward block on 32x32 latents, fp32 storage, a 416x624 image's ragged token count
        _linear("feed_forward_out_f32", 2 * 26 * 39, 2560, 640, "f32", residual=True),
        # training: key projection of an encoder's 77 states, wide input features
        _linear("key_projection_backward", 8 * 77, 2048, 1280, "bf16", backward=True),
        # one token through the gated feed-forward of the deepest level
        _glu("feed_forward_token", 1, 1280, 5120, "bf16"),
        # the gated feed-forward at full latent size
        _glu("feed_forward_64", 2 * 4096, 320, 1280, "f16"),
        # training: the gated feed-forward at the middle level, guidance-free batch of four
        _glu("feed_forward_32_backward", 4 * 1024, 640, 2560, "bf16", backward=True),
        # image tokens attending to an encoder's 77 states, padded to the longest prompt
        _attention("cross_64", 2, 4096, 77, 8, 8, 40, "f16", keys="lengths"),
        # the block's other attention, over the image's own tokens (128x128 latent, one level down)
        _attention("self_64", 2, 4096, 4096, 10, 10, 64, "bf16"),
        # one query a sequence against long encoder states of ragged lengths, heads that share keys
        _attention("one_query_long", 8, 1, 15000, 32, 8, 128, "bf16", keys="lengths"),
        # training: image tokens attending to an encoder's states with masked keys
        _attention("cross_32_backward", 4, 1024, 154, 10, 10, 64, "f16", keys="mask", backward=True),
        # training: image tokens of a 32x32 latent among each other, two levels down, wide heads
        _attention("self_32_backward", 4, 1024, 1024, 8, 8, 80, "bf16", backward=True),
    ]


MAX_PRODUCT = 6.0 * 4096 * 640 * 2560 * 2        # multiply-adds of the largest listed products, doubled into flops
MAX_SCORES = 2.0 * 10 * 4096 * 4096              # scores of the largest listed attention
MAX_SCORES_BACKWARD = 4.0 * 8 * 1024 * 1024
MAX_KEYS = 8.0 * 15000 * 8 * 128                 # elements of the largest listed keys


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _features(rng, lo, hi):
    """Feature counts: mostly whole groups of 32 or 8 channels, now and then odd ones."""
    v, kind = int(_log(rng, lo, hi + 1)), rng.random()
    return v if kind < 0.12 else max(8, v // 8 * 8) if kind < 0.4 else max(32, v // 32 * 32)


def _draw_once(rng):
    op, dtype, backward = rng.choice(["linear", "glu", "attention", "attention"]), rng.choice(["f16", "bf16", "f16", "bf16", "f32"]), rng.random() < 0.4
    if op == "linear":
        M = int(_log(rng, 1, 16385))
        return _linear(None, M, _features(rng, 64, 5120), _features(rng, 64, 2560), dtype, rng.choice(ACTS), not backward and rng.random() < 0.5, backward)
    if op == "glu":
        return _glu(None, int(_log(rng, 1, 16385)), _features(rng, 64, 1280), _features(rng, 64, 5120), dtype, rng.choice(ACTS[1:]), backward)
    kind = rng.choice(["cross", "cross", "self", "few"])
    D, Hkv = rng.choice([40, 64, 64, 80, 128, 160, 8 * rng.randint(3, 20)]), rng.choice([1, 2, 4, 5, 8, 10])
    H, B = Hkv * rng.choice([1, 1, 1, 2, 4]), rng.choice([1, 2, 2, 3, 4, 8])
    keys = rng.choice(["all", "lengths", "mask"])
    if kind == "cross":
        # (with one key alone the gradients of q and k are zero, and their rounding errors nothing to compare)
        return _attention(None, B, int(_log(rng, 16, 4097)), int(_log(rng, 16 if backward else 1, 700)), H, Hkv, D, dtype, keys, backward)
    if kind == "self":
        S = int(_log(rng, 64, 4097))
        return _attention(None, B, S, S, H, Hkv, D, dtype, keys, backward)
    return _attention(None, B, rng.choice([1, 1, 2, 3, 5, 8]), int(_log(rng, 64, 16385)), H, Hkv, D, dtype, keys, False)


def _fits(c):
    if c["op"] == "attention":
        scores = c["B"] * c["H"] * c["Sq"] * c["Skv"] * (2.0 if c["dtype"] == "f32" else 1.0)
        return scores <= (MAX_SCORES_BACKWARD if c["backward"] else MAX_SCORES) and c["B"] * c["Skv"] * c["Hkv"] * c["D"] <= MAX_KEYS
    return work(c)["flops"] * (2.0 if c["dtype"] == "f32" else 1.0) <= MAX_PRODUCT


def draw(rng):
    while True:
        case = _draw_once(rng)
        if _fits(case):
            return case


def work(case):
    """Each input read once, each output written once; keys that a mask or a length takes out are counted all the same (their share is an
    accident of the seed).  Products: two flops a multiply-add; a backward pass makes z, or u and g, again where an activation needs them."""
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "attention":
        q, k = c["B"] * c["Sq"] * c["H"] * c["D"], c["B"] * c["Skv"] * c["Hkv"] * c["D"]
        pairs = 2.0 * c["B"] * c["H"] * c["Sq"] * c["Skv"] * c["D"]
        masks = {"all": 0, "lengths": 4 * c["B"], "mask": c["B"] * c["Skv"]}[c["keys"]]
        lse = 4 * c["B"] * c["H"] * c["Sq"]
        return ({"bytes": 4 * (q + k) * e + lse + masks, "flops": 5 * pairs} if c["backward"] else {"bytes": 2 * (q + k) * e + masks, "flops": 2 * pairs})
    M, K, N = c["M"], c["K"], c["N"]
    W = N if c["op"] == "linear" else 2 * N
    product = 2.0 * M * K * W
    if not c["backward"]:
        return {"bytes": (M * K + W * K + M * N * (2 if c.get("residual") else 1)) * e + 4 * W, "flops": product}
    again = c["op"] == "glu" or c["act"] != "none"
    return {"bytes": (2 * M * K + 2 * W * K + M * N) * e + (8 if again else 4) * W, "flops": product * (3 if again else 2)}


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    td = TORCH[c["dtype"]]

    def randn(shape, std=1.0, dtype=td):
        return (torch.randn(shape, device=DEV, generator=g, dtype=torch.float32) * std).to(dtype)

    s = {"case": c}
    if c["op"] == "attention":
        B, Sq, Skv, H, Hkv, D = (c[n] for n in ("B", "Sq", "Skv", "H", "Hkv", "D"))
        s["q"], s["k"], s["v"] = randn((B, Sq, H, D), 1.5), randn((B, Skv, Hkv, D)), randn((B, Skv, Hkv, D))
        s["kv_len"] = s["key_mask"] = None
        if c["keys"] == "lengths":          # prompts from none to all of the states; the last row of a batch is whole
            s["kv_len"] = torch.randint(0, Skv + 1, (B,), device=DEV, generator=g, dtype=torch.int32)
            s["kv_len"][-1] = Skv
        if c["keys"] == "mask":
            s["key_mask"] = (torch.rand((B, Skv), device=DEV, generator=g) < 0.7).to(torch.uint8)
        if c["backward"]:                   # what the forward pass of a training step left behind
            s["do"] = randn((B, Sq, H, D))
            p, lse = _probabilities(s)
            s["o"] = _heads_back(p @ _keys(s, s["v"]), H).to(td)
            s["lse"] = lse.view(B, H, Sq).contiguous()
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in ("q", "k", "v"))
        else:
            s["o"] = torch.empty((B, Sq, H, D), dtype=td, device=DEV)
        return s
    M, K, N = c["M"], c["K"], c["N"]
    W = N if c["op"] == "linear" else 2 * N
    s["x"], s["w"], s["bias"] = randn((M, K)), randn((W, K), 1.0 / math.sqrt(K)), randn((W,), 0.1, torch.float32)
    s["residual"] = randn((M, N)) if c.get("residual") else None
    if c["backward"]:
        s["dy"] = randn((M, N))
        s["dx"], s["dw"], s["dbias"] = torch.empty_like(s["x"]), torch.empty_like(s["w"]), torch.empty_like(s["bias"])
    else:
        s["y"] = torch.empty((M, N), dtype=td, device=DEV)
    return s


# ---- the plain forms: elementary operations in fp32 -------------------------------------------------------------------------------
def _act(z, act):
    """act(z) and act'(z)."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return z * p, p * (1.0 + z * (1.0 - p))
    if act == "gelu":
        p = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * p, p + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    a, b = math.sqrt(2.0 / math.pi), 0.044715
    t = torch.tanh(a * (z + b * z * z * z))
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * a * (1.0 + 3.0 * b * z * z)


def _heads(t):
    """[B,S,H,D] -> fp32 [B,H,S,D]"""
    return t.float().permute(0, 2, 1, 3).contiguous()


def _heads_back(t, H):
    """[B,Hkv,H/Hkv * Sq,D] -> [B,Sq,H,D]"""
    B, D = t.shape[0], t.shape[-1]
    return t.reshape(B, H, -1, D).permute(0, 2, 1, 3).contiguous()


def _valid(s):
    """[B,1,1,Skv] truth values, or None"""
    if s["kv_len"] is not None:
        return (torch.arange(s["k"].shape[1], device=DEV)[None, :] < s["kv_len"][:, None])[:, None, None, :]
    return None if s["key_mask"] is None else (s["key_mask"] != 0)[:, None, None, :]


def _queries(s, t):
    """The query heads that share a key head, one after the other: [B,Hkv,H/Hkv * Sq,D]"""
    return _heads(t).view(t.shape[0], s["k"].shape[2], -1, t.shape[3])


def _keys(s, t):
    """[B,Hkv,Skv,D], zero where no query may look"""
    valid = _valid(s)
    return _heads(t) if valid is None else torch.where(valid.transpose(2, 3), _heads(t), 0.0)


def _probabilities(s):
    """p [B,Hkv,H/Hkv * Sq,Skv] and the logarithm of the sum under it"""
    scores = _queries(s, s["q"]) @ _keys(s, s["k"]).transpose(2, 3)
    scores *= s["q"].shape[3] ** -0.5
    valid = _valid(s)
    if valid is not None:
        scores.masked_fill_(~valid, -math.inf)
    top = scores.amax(3, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = scores.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    return p.div_(torch.where(total > 0, total, 1.0)), top + torch.log(total)


def _plain(s):
    c = s["case"]
    td = TORCH[c["dtype"]]
    if c["op"] == "attention":
        H, scale = c["H"], c["D"] ** -0.5
        p, _ = _probabilities(s)
        if not c["backward"]:
            return _heads_back(p @ _keys(s, s["v"]), H).to(td)
        do = _queries(s, s["do"])
        dp = do @ _keys(s, s["v"]).transpose(2, 3)
        dv = p.transpose(2, 3) @ do
        ds = p * (dp - (p * dp).sum(3, keepdim=True)) * scale
        dq, dk = ds @ _keys(s, s["k"]), ds.transpose(2, 3) @ _queries(s, s["q"])
        return _heads_back(dq, H).to(td), dk.permute(0, 2, 1, 3).contiguous().to(td), dv.permute(0, 2, 1, 3).contiguous().to(td)
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t() + s["bias"]
    if c["op"] == "linear":
        a, slope = _act(z, c["act"])
        if not c["backward"]:
            return (a if s["residual"] is None else a + s["residual"].float()).to(td)
        dz = s["dy"].float() * slope
    else:
        u, (a, slope) = z[:, :c["N"]], _act(z[:, c["N"]:], c["act"])
        if not c["backward"]:
            return (u * a).to(td)
        dh = s["dy"].float()
        dz = torch.cat([dh * a, dh * u * slope], 1)
    return (dz @ w).to(td), (dz.t() @ x).to(td), dz.sum(0)


# ---- the library's calls ----------------------------------------------------------------------------------------------------------
def _library(s):
    from paper_2412_05781_amd import binding as lib
    c = s["case"]
    if "ws" not in s:                       # the workspace that a program allocates once and keeps
        s["ws"] = _workspace(lib, c)
    ws = s["ws"]
    if c["op"] == "attention":
        if c["backward"]:
            return lib.wino_attention_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"],
                                               kv_len=s["kv_len"], key_mask=s["key_mask"], workspace=ws)
        return lib.wino_attention(s["q"], s["k"], s["v"], s["o"], kv_len=s["kv_len"], key_mask=s["key_mask"], workspace=ws)
    act = _act_code(lib, c)
    if c["op"] == "linear":
        if c["backward"]:
            return lib.wino_linear_backward(s["x"], s["w"], s["bias"], s["dy"], s["dx"], s["dw"], s["dbias"], act, workspace=ws)
        return lib.wino_linear(s["x"], s["w"], s["bias"], s["y"], act, residual=s["residual"], workspace=ws)
    if c["backward"]:
        return lib.wino_glu_backward(s["x"], s["w"], s["bias"], s["dy"], s["dx"], s["dw"], s["dbias"], act, workspace=ws)
    return lib.wino_glu(s["x"], s["w"], s["bias"], s["y"], act, workspace=ws)


def _act_code(lib, c):
    return getattr(lib, "WINO_ACT_" + c["act"].upper())


def _workspace(lib, c):
    dt = lib.DTYPE_OF[TORCH[c["dtype"]]]
    if c["op"] == "attention":
        size = lib.wino_attention_backward_workspace_bytes if c["backward"] else lib.wino_attention_workspace_bytes
        n = size(c["B"], c["Sq"], c["Skv"], c["H"], c["Hkv"], c["D"], dt)
    else:
        size = {("linear", False): lib.wino_linear_workspace_bytes, ("linear", True): lib.wino_linear_backward_workspace_bytes,
                ("glu", False): lib.wino_glu_workspace_bytes, ("glu", True): lib.wino_glu_backward_workspace_bytes}[c["op"], c["backward"]]
        n = size(c["M"], c["N"], c["K"], dt, _act_code(lib, c))
    return torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


def run(state):
    return _library(state) if own else _plain(state)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------------
def _exact_gate(z, act):
    """(phi, phi') of the activation z * phi(z): a logistic, normal or tanh distribution function."""
    if act == "none":
        return torch.ones_like(z), torch.zeros_like(z)
    if act == "silu":
        p = torch.sigmoid(z)
        return p, p * (1 - p)
    if act == "gelu":
        return torch.special.ndtr(z), torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    inner, slope = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3), math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z.square())
    p = torch.sigmoid(2 * inner)            # (1 + tanh(t)) / 2
    return p, 2 * slope * p * (1 - p)


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] != "attention":
        x, w, N = s["x"].double(), s["w"].double(), c["N"]
        z = torch.addmm(s["bias"].double(), x, w.mT)
        gate = z[:, -N:]
        phi, dphi = _exact_gate(gate, c["act"])
        if not c["backward"]:
            y = gate * phi if c["op"] == "linear" else z[:, :N] * gate * phi
            return y if s["residual"] is None else y + s["residual"].double()
        dy = s["dy"].double()
        dgate = dy * (phi + gate * dphi)
        dz = dgate if c["op"] == "linear" else torch.hstack([dy * gate * phi, dgate * z[:, :N]])
        return dz @ w, dz.mT @ x, dz.sum(0)
    B, H, group, scale = c["B"], c["H"], c["H"] // c["Hkv"], 1 / math.sqrt(c["D"])
    o, dq, dk, dv = (torch.zeros(s[n].shape, dtype=torch.float64, device=DEV) for n in ("q", "q", "k", "v"))
    for b in range(B):
        if s["kv_len"] is not None:
            seen = torch.arange(c["Skv"], device=DEV)[: int(s["kv_len"][b])]
        else:
            seen = torch.arange(c["Skv"], device=DEV) if s["key_mask"] is None else s["key_mask"][b].nonzero()[:, 0]
        if seen.numel() == 0:
            continue
        for h in range(H):
            q, k, v = s["q"][b, :, h].double(), s["k"][b, seen, h // group].double(), s["v"][b, seen, h // group].double()
            p = torch.softmax(q @ k.mT * scale, 1)
            o[b, :, h] = p @ v
            if c["backward"]:
                do = s["do"][b, :, h].double()
                ds = p * ((do @ v.mT) - (do * o[b, :, h]).sum(1, keepdim=True))
                dq[b, :, h] = ds @ k * scale
                dk[b, seen, h // group] += ds.mT @ q * scale
                dv[b, seen, h // group] += p.mT @ do
    return (dq, dk, dv) if c["backward"] else o
