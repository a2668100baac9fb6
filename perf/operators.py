"""The operators around the policy's log-probs, as cases whose time and results can be measured.

What lies between the last layer of a policy and the distribution that its tokens are drawn from, in rollouts and in
training: the final norm (forward and backward), the LM head with 4-bit weights of a rollout, and the adjustment of logits
(penalties for repeated tokens, biases, grammar masks, temperature) with the log-probs of the adjusted policy and the
gradient back through it.  Every case is one call of one entry point:
  norm_fwd     layer norm or its root-mean-square form over rows of hidden states
  norm_bwd     its gradient: dx of every row, the sums over rows for weight and bias
  adjust       logits -> logits of the policy that is sampled from, their log-sum-exp, log-probs of chosen tokens
  adjust_bwd   gradient with respect to the adjusted logits -> gradient with respect to the logits
  w4_linear    a few tokens' hidden states times a weight held as 4-bit codes with a scale per group
Sizes are those of the workloads in synth/ and bench.py (vocabulary 151,936 and 32,000, hidden sizes 1,536 and 4,096,
batches up to 65,536 tokens) and generic odd ones.
"""
import math

import torch

own = False  # plain torch operations; True: the library's operators

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # the final norm of one decoding step of 64 sequences: latency
        {"name": "norm_decode_64", "op": "norm_fwd", "T": 64, "H": 1536, "kind": "rms", "x": "bf16", "y": "bf16"},
        # a micro-batch of an fp32 residual stream of odd width, normed into the bfloat16 states that the head takes
        {"name": "norm_f32_odd", "op": "norm_fwd", "T": 10240, "H": 2049, "kind": "layer", "x": "f32", "y": "bf16"},
        # backward pass of a small micro-batch at the 1.5B-scale hidden size, fp32 residual stream
        {"name": "norm_bwd_1000", "op": "norm_bwd", "T": 1000, "H": 1536, "kind": "rms", "x": "f32", "y": "bf16"},
        # backward pass of the 8B-scale batch in one call
        {"name": "norm_bwd_65536", "op": "norm_bwd", "T": 65536, "H": 4096, "kind": "layer", "x": "bf16", "y": "bf16"},
        # one sequence that decodes alone, under every adjustment: latency
        {"name": "adjust_decode_1", "op": "adjust", "T": 1, "V": 151936, "z": "bf16", "u": "f32", "history": 3000,
         "shape": "decode", "mask": True, "bias": True, "write": True},
        # a decoding step of 64 sequences with long ragged contexts
        {"name": "adjust_decode_64", "op": "adjust", "T": 64, "V": 151936, "z": "bf16", "u": "f32", "history": 16384,
         "shape": "decode", "mask": True, "bias": False, "write": True},
        # scoring a micro-batch under the adjusted policy (rows of one sequence share its growing history): log-probs
        # only, a vocabulary that is no multiple of anything
        {"name": "adjust_score_odd", "op": "adjust", "T": 8192, "V": 50001, "z": "bf16", "u": "bf16", "history": 2048,
         "shape": "prefix", "mask": False, "bias": False, "write": False},
        # gradient of a small fp32 micro-batch
        {"name": "adjust_bwd_300", "op": "adjust_bwd", "T": 300, "V": 32000, "z": "f32", "u": "f32", "history": 256,
         "shape": "prefix", "mask": True, "bias": False},
        # gradient of a training micro-batch at the full vocabulary
        {"name": "adjust_bwd_8192", "op": "adjust_bwd", "T": 8192, "V": 151936, "z": "bf16", "u": "bf16", "history": 2048,
         "shape": "prefix", "mask": True, "bias": False},
        # the head of one decoding sequence, 1.5B scale
        {"name": "w4_1x1536", "op": "w4_linear", "T": 1, "H": 1536, "V": 151936, "group": 128, "scale": "bf16",
         "zeros": False, "out": "bf16"},
        # the head of 16 decoding sequences, 8B scale
        {"name": "w4_16x4096", "op": "w4_linear", "T": 16, "H": 4096, "V": 151936, "group": 128, "scale": "bf16",
         "zeros": False, "out": "f32"},
        # a batch of 50 short rollouts, finer groups with zero points
        {"name": "w4_50x4096_zeros", "op": "w4_linear", "T": 50, "H": 4096, "V": 151936, "group": 32, "scale": "f32",
         "zeros": True, "out": "f32"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _vocab(rng):
    """A vocabulary of 16,000 to 200,000 entries: a common size, a multiple of 64, or any odd number."""
    how = rng.randrange(3)
    if how == 0:
        return rng.choice([32000, 50264, 65536, 100352, 128256, 151936])
    v = _log_int(rng, 16000, 200000)
    return v // 64 * 64 if how == 1 else v | 1


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "adjust", "adjust", "adjust_bwd", "w4_linear", "w4_linear"])
    if op in ("norm_fwd", "norm_bwd"):
        H = rng.choice([896, 1536, 2048, 4096, _log_int(rng, 65, 8192), _log_int(rng, 65, 8192) | 1])
        T = _log_int(rng, 1, min(65536, 65536 * 4096 // H))
        x, y = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        if x == "f32":
            T = (T + 2) // 3
        return {"op": op, "T": T, "H": H, "kind": rng.choice(["rms", "layer"]), "x": x, "y": y}
    if op == "w4_linear":
        group = rng.choice([32, 64, 128])
        H = rng.choice([896, 1536, 2048, 4096, _log_int(rng, 2, 32) * 128 + rng.choice([0, 128 - group if group < 128 else 0])])
        return {"op": op, "T": _log_int(rng, 1, 50), "H": H, "V": _vocab(rng) * 3 // 4, "group": group,
                "scale": rng.choice(["bf16", "f32"]), "zeros": rng.random() < 0.4, "out": rng.choice(["bf16", "f32"])}
    V = _vocab(rng)
    z, u = rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
    d = {"op": op, "V": V, "z": z, "u": u, "mask": rng.random() < 0.5, "bias": rng.random() < 0.4}
    if op == "adjust" and rng.random() < 0.5:
        return {**d, "T": _log_int(rng, 1, 256), "history": _log_int(rng, 16, 16384), "shape": "decode", "write": True}
    d.update(T=_log_int(rng, 16, min(8192, int(4e8) // V)), history=_log_int(rng, 64, 2048), shape="prefix")
    return {**d, "write": rng.random() < 0.5} if op == "adjust" else d


# ---- inputs ------------------------------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(0x0B5E + 7919 * int(seed))
    return g


def _norm_inputs(case, g):
    T, H = case["T"], case["H"]
    xt, yt = DTYPES[case["x"]], DTYPES[case["y"]]
    # a residual stream: a spread of row scales, a small common offset, a few wide channels
    x = torch.randn(T, H, generator=g, device="cuda") * (0.5 + 3.0 * torch.rand(T, 1, generator=g, device="cuda"))
    x = ((x + 0.3) * (1.0 + 9.0 * (torch.rand(H, generator=g, device="cuda") < 0.01))).to(xt)
    d = {"x": x, "weight": (1.0 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(xt), "bias": None, "mean": None}
    if case["kind"] == "layer":
        d["bias"] = (0.1 * torch.randn(H, generator=g, device="cuda")).to(xt)
    if case["op"] == "norm_fwd":
        d["out"] = torch.empty(T, H, device="cuda", dtype=yt)
        return d
    d["dy"] = (1e-2 * torch.randn(T, H, generator=g, device="cuda")).to(yt)
    # what the forward pass left behind
    xf = x.float()
    mean = xf.mean(1) if case["kind"] == "layer" else torch.zeros(T, device="cuda")
    xf -= mean[:, None]
    d["rstd"] = torch.rsqrt(xf.square_().mean(1) + EPS)
    d["mean"] = mean if case["kind"] == "layer" else None
    d["out"] = torch.empty_like(x)
    return d


def _policy(case, g):
    """The rows' histories and the adjustments' strengths: `decode` rows are sequences with a context of their own,
    `prefix` rows are the tokens of sequences, each with the sequence's tokens before it as its history."""
    T, V, most = case["T"], case["V"], case["history"]
    dev = "cuda"
    if case["shape"] == "decode":
        lengths = torch.randint((most + 1) // 2, most + 1, (T,), generator=g, device=dev)
        start = torch.cumsum(lengths, 0) - lengths
        prompt = (lengths * torch.rand(T, generator=g, device=dev)).long()
        total = T * most
        seq = torch.arange(T, device=dev)
    else:
        # packed sequences of `most` tokens (the last one shorter), the first eighth of each a prompt
        t = torch.arange(T, device=dev)
        seq = t // most
        start, lengths = seq * most, t % most
        prompt = torch.minimum(lengths, torch.full_like(lengths, most // 8))
        total = T
    # token ids are drawn as a text's are: few of them often, most of them rarely
    ids = (V * torch.rand(total, generator=g, device=dev).pow(4)).long().clamp_(max=V - 1).to(torch.int32)
    one = lambda lo, hi: (lo + (hi - lo) * torch.rand(int(seq[-1]) + 1, generator=g, device=dev))[seq].contiguous()
    p = {"history": ids, "hist_start": start, "hist_len": lengths.to(torch.int32), "prompt_len": prompt.to(torch.int32),
         "repetition": one(1.0, 1.3), "frequency": one(0.0, 0.3), "presence": one(0.0, 0.5), "temperature": one(0.6, 1.2),
         "bias": None, "allowed": None}
    if case["bias"]:
        p["bias"] = 4.0 * torch.randn(V, generator=g, device=dev) * (torch.rand(V, generator=g, device=dev) < 0.05)
    if case["mask"]:
        # a quarter of the rows is inside a grammar that lets one token in 16 through, the others may take any
        words = lambda: torch.randint(-2 ** 31, 2 ** 31, (T, (V + 31) // 32), generator=g, device=dev).to(torch.int32)
        free = (torch.rand(T, 1, generator=g, device=dev) < 0.75).to(torch.int32)
        p["allowed"] = (words() & words() & words() & words()) | -free
    return p


def _adjust_inputs(case, g):
    T, V = case["T"], case["V"]
    z = torch.randn(T, V, generator=g, device="cuda", dtype=DTYPES[case["z"]]).mul_(3.0)
    d = {"z": z, "policy": _policy(case, g), "chosen": None, "out": None}
    ut = DTYPES[case["u"]]
    if case["op"] == "adjust_bwd":
        # dz of a clipped surrogate: g (1[chosen] - p)
        du = torch.softmax(z.float(), 1)
        du *= -torch.randn(T, 1, generator=g, device="cuda")
        rows = torch.arange(T, device="cuda")
        du[rows, torch.randint(0, V, (T,), generator=g, device="cuda")] += 0.5
        d["du"] = du.to(ut)
        d["out"] = torch.empty_like(z)
        return d
    if case["write"]:
        d["out"] = torch.empty(T, V, device="cuda", dtype=ut)
    if case["shape"] == "prefix":  # scoring: the tokens are known
        chosen = torch.randint(0, V, (T,), generator=g, device="cuda")
        allowed = d["policy"]["allowed"]
        if allowed is not None:  # (a token that was drawn is one that was allowed)
            word = chosen // 32
            bit = torch.bitwise_left_shift(torch.ones_like(chosen), chosen % 32)
            rows = torch.arange(T, device="cuda")
            allowed[rows, word] = ((allowed[rows, word].long() & 0xFFFFFFFF) | bit).to(torch.int32)
        d["chosen"] = chosen.to(torch.int32)
    return d


def _w4_inputs(case, g):
    T, H, V, G = case["T"], case["H"], case["V"], case["group"]
    w = torch.randn(V, H, generator=g, device="cuda").mul_(2.5).add_(8.5).clamp_(0.0, 15.99).to(torch.uint8)
    d = {"x": torch.randn(T, H, generator=g, device="cuda", dtype=torch.bfloat16),
         "codes": w[:, 0::2] | (w[:, 1::2] << 4),
         "scales": (0.008 * (0.5 + torch.rand(V, H // G, generator=g, device="cuda"))).to(DTYPES[case["scale"]]),
         "zeros": None, "group": G,
         "out": torch.empty(T, V, device="cuda", dtype=DTYPES[case["out"]])}
    if case["zeros"]:
        d["zeros"] = torch.randint(5, 12, (V, H // G), generator=g, device="cuda").to(torch.uint8)
    return d


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    make = _norm_inputs if op.startswith("norm") else _adjust_inputs if op.startswith("adjust") else _w4_inputs
    d = make(case, g)
    d["case"] = case
    return d


# ---- one pass ----------------------------------------------------------------------------------------------------


def run(state):
    op = state["case"]["op"]
    return (_OWN if own else _PLAIN)[op](state)


def _own_norm_fwd(s):
    import paper_2512_06547_amd as a3po
    kind = a3po.A3PO_NORM_LAYER if s["case"]["kind"] == "layer" else a3po.A3PO_NORM_RMS
    y, mean, rstd = a3po.norm_fwd(s["x"], s["weight"], s["bias"], eps=EPS, kind=kind, out=s["out"])
    return {"y": y, "rstd": rstd} if mean is None else {"y": y, "mean": mean, "rstd": rstd}


def _own_norm_bwd(s):
    import paper_2512_06547_amd as a3po
    layer = s["case"]["kind"] == "layer"
    out = a3po.norm_bwd(s["dy"], s["x"], s["weight"], s["rstd"], mean=s["mean"], want_dbias=layer,
                        kind=a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS, dx=s["out"])
    return {k: out[k] for k in (("dx", "dweight", "dbias") if layer else ("dx", "dweight"))}


def _own_adjust(s):
    import paper_2512_06547_amd as a3po
    out = a3po.adjust_logits(s["z"], chosen=s["chosen"], out=s["out"], write=s["case"]["write"], **s["policy"])
    return {k: out[k] for k in ("out", "lse", "logp") if out[k] is not None}


def _own_adjust_bwd(s):
    import paper_2512_06547_amd as a3po
    return a3po.adjust_logits_bwd(s["du"], s["z"], dlogits=s["out"], **s["policy"])


def _own_w4(s):
    import paper_2512_06547_amd as a3po
    return a3po.w4_linear(s["x"], s["codes"], s["scales"], zeros=s["zeros"], group=s["group"], out=s["out"])


def _norm_of(x, kind):
    """(xhat, mean, rstd) in the type of x."""
    mean = x.mean(1) if kind == "layer" else None
    c = x if mean is None else x - mean[:, None]
    rstd = 1.0 / torch.sqrt((c * c).mean(1) + EPS)
    return c * rstd[:, None], mean, rstd


def _plain_norm_fwd(s):
    xhat, mean, rstd = _norm_of(s["x"].float(), s["case"]["kind"])
    y = xhat * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = y.to(s["out"].dtype)
    return {"y": y, "rstd": rstd} if mean is None else {"y": y, "mean": mean, "rstd": rstd}


def _plain_norm_bwd(s):
    x, dy = s["x"].float(), s["dy"].float()
    layer = s["case"]["kind"] == "layer"
    xhat = (x - s["mean"][:, None] if layer else x) * s["rstd"][:, None]
    g = dy * s["weight"].float()
    inner = g - xhat * (g * xhat).mean(1, keepdim=True)
    if layer:
        inner = inner - g.mean(1, keepdim=True)
    out = {"dx": (inner * s["rstd"][:, None]).to(s["x"].dtype), "dweight": (dy * xhat).sum(0)}
    return {**out, "dbias": dy.sum(0)} if layer else out


def _counts(p, T, V):
    """How often each token is in the output part of each row's history, and whether it is in the history at all."""
    length = p["hist_len"].long()
    rows = torch.repeat_interleave(torch.arange(T, device="cuda"), length)
    at = torch.arange(rows.numel(), device="cuda") - (torch.cumsum(length, 0) - length)[rows]
    token = rows * V + p["history"][p["hist_start"][rows] + at].long()
    output = at >= p["prompt_len"][rows]
    n = torch.zeros(T * V, dtype=torch.int32, device="cuda")
    n.index_add_(0, token, output.to(torch.int32))
    seen = torch.zeros(T * V, dtype=torch.bool, device="cuda")
    seen[token] = True
    return n.view(T, V), seen.view(T, V)


def _allowed(words, V):
    bits = (words[:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    return bits.reshape(words.shape[0], -1)[:, :V].bool()


def _plain_adjust(s):
    case, p = s["case"], s["policy"]
    z = s["z"].float()
    n, seen = _counts(p, *z.shape)
    rep = p["repetition"][:, None]
    u = torch.where(seen, torch.where(z > 0, z / rep, z * rep), z)
    u = u - p["frequency"][:, None] * n - p["presence"][:, None] * (n > 0)
    if p["bias"] is not None:
        u = u + p["bias"]
    u = u / p["temperature"][:, None]
    if p["allowed"] is not None:
        u = torch.where(_allowed(p["allowed"], case["V"]), u, torch.full_like(u, -math.inf))
    m = u.amax(1)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    lse = m + torch.log(torch.exp(u - m[:, None]).sum(1))
    out = {"out": u.to(s["out"].dtype)} if case["write"] else {}
    out["lse"] = lse
    if s["chosen"] is not None:
        out["logp"] = u.gather(1, s["chosen"].long()[:, None])[:, 0] - lse
    return out


def _plain_adjust_bwd(s):
    p, z = s["policy"], s["z"].float()
    _, seen = _counts(p, *z.shape)
    rep = p["repetition"][:, None]
    dz = s["du"].float() / p["temperature"][:, None]
    dz = torch.where(seen, torch.where(z > 0, dz / rep, dz * rep), dz)
    if p["allowed"] is not None:
        dz = torch.where(_allowed(p["allowed"], z.shape[1]), dz, torch.zeros_like(dz))
    return dz.to(s["z"].dtype)


def _plain_w4(s):
    V, half = s["codes"].shape
    q = torch.stack([s["codes"] & 15, s["codes"] >> 4], dim=2).view(V, -1, s["group"]).float()
    q -= 8.0 if s["zeros"] is None else s["zeros"].float()[:, :, None]
    w = (q * s["scales"].float()[:, :, None]).view(V, 2 * half)
    return (s["x"].float() @ w.t()).to(s["out"].dtype)


_OWN = {"norm_fwd": _own_norm_fwd, "norm_bwd": _own_norm_bwd, "adjust": _own_adjust, "adjust_bwd": _own_adjust_bwd,
        "w4_linear": _own_w4}
_PLAIN = {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "adjust": _plain_adjust,
          "adjust_bwd": _plain_adjust_bwd, "w4_linear": _plain_w4}


# ---- what a pass cannot do without -------------------------------------------------------------------------------


def _size(name):
    return 4 if name == "f32" else 2


def work(case):
    T = case["T"]
    if case["op"].startswith("norm"):
        H, x, y = case["H"], _size(case["x"]), _size(case["y"])
        layer = case["kind"] == "layer"
        if case["op"] == "norm_fwd":
            return {"bytes": T * H * (x + y) + H * x * (1 + layer) + 4 * T * (1 + layer), "flops": T * H * 7}
        return {"bytes": T * H * (2 * x + y) + H * (x + 4 + 4 * layer) + 4 * T * (1 + layer), "flops": T * H * 13}
    V = case["V"]
    if case["op"] == "w4_linear":
        H, groups = case["H"], case["H"] // case["group"]
        return {"bytes": V * H // 2 + V * groups * (_size(case["scale"]) + case["zeros"]) + T * H * 2
                + T * V * _size(case["out"]), "flops": 2 * T * V * H}
    z, u = _size(case["z"]), _size(case["u"])
    # every row's tokens once: sequences' own contexts, or the packed tokens that the rows share
    side = 4 * (T * (case["history"] * 3 // 4) if case["shape"] == "decode" else T) + 32 * T
    side += (T * ((V + 31) // 32) * 4 if case["mask"] else 0) + (4 * V if case["bias"] else 0)
    if case["op"] == "adjust":
        return {"bytes": T * V * (z + (u if case["write"] else 0)) + side + 8 * T, "flops": T * V * 6}
    return {"bytes": T * V * (z + u) + side, "flops": T * V * 2}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return {"norm_fwd": _exact_norm_fwd, "norm_bwd": _exact_norm_bwd, "adjust": _exact_adjust,
                "adjust_bwd": _exact_adjust_bwd, "w4_linear": _exact_w4}[case["op"]](s)


def _blocks(T, width, values=1 << 25):
    step = max(1, values // width)
    return [slice(a, min(T, a + step)) for a in range(0, T, step)]


def _exact_norm_fwd(s):
    w = s["weight"].double()
    b = torch.zeros_like(w) if s["bias"] is None else s["bias"].double()
    T, H = s["x"].shape
    ys, means, rstds = [], [], []
    for rows in _blocks(T, H):
        x = s["x"][rows].double()
        mu = x.sum(1) / H if s["case"]["kind"] == "layer" else x.new_zeros(x.shape[0])
        var = ((x - mu[:, None]) ** 2).sum(1) / H
        r = (var + EPS) ** -0.5
        ys.append(((x - mu[:, None]) * r[:, None] * w + b))
        means.append(mu)
        rstds.append(r)
    y, mean, rstd = torch.cat(ys), torch.cat(means), torch.cat(rstds)
    return {"y": y, "mean": mean, "rstd": rstd} if s["case"]["kind"] == "layer" else {"y": y, "rstd": rstd}


def _exact_norm_bwd(s):
    w = s["weight"].double()
    T, H = s["x"].shape
    dx, dw, db = [], w.new_zeros(H), w.new_zeros(H)
    for rows in _blocks(T, H):
        x, dy, r = s["x"][rows].double(), s["dy"][rows].double(), s["rstd"][rows].double()[:, None]
        n = x * r if s["mean"] is None else (x - s["mean"][rows].double()[:, None]) * r
        a = dy * w
        along = (a * n).sum(1, keepdim=True) / H
        level = a.sum(1, keepdim=True) / H if s["mean"] is not None else 0.0
        dx.append(r * (a - level - n * along))
        dw += (dy * n).sum(0)
        db += dy.sum(0)
    out = {"dx": torch.cat(dx), "dweight": dw}
    return out if s["mean"] is None else {**out, "dbias": db}


def _exact_rows(s):
    """Per row: (row, factor that the repetition penalty multiplies with, what frequency and presence take off, allowed)."""
    p, V = s["policy"], s["case"]["V"]
    host = {k: p[k].tolist() for k in ("hist_start", "hist_len", "prompt_len", "repetition", "frequency", "presence")}
    ids = p["history"].long()
    every = torch.arange(V, device="cuda")
    for t in range(s["z"].shape[0]):
        a, n, k = host["hist_start"][t], host["hist_len"][t], host["prompt_len"][t]
        z = s["z"][t].double()
        factor = torch.ones_like(z)
        tokens = ids[a:a + n]
        rep = host["repetition"][t]
        factor[tokens] = torch.where(z[tokens] > 0, 1.0 / rep, rep).double()
        count = torch.zeros_like(z)
        count.index_put_((tokens[k:],), torch.ones((), dtype=torch.float64, device="cuda"), accumulate=True)
        off = host["frequency"][t] * count + host["presence"][t] * (count != 0).double()
        ok = None
        if p["allowed"] is not None:
            ok = ((p["allowed"][t].long() & 0xFFFFFFFF)[every // 32] >> (every % 32)) % 2 == 1
        yield t, z, factor, off, ok


def _exact_adjust(s):
    p, (T, V) = s["policy"], s["z"].shape
    u_all = torch.empty(T, V, dtype=torch.float64, device="cuda") if s["case"]["write"] else None
    lse, logp = torch.empty(T, dtype=torch.float64, device="cuda"), torch.empty(T, dtype=torch.float64, device="cuda")
    for t, z, factor, off, ok in _exact_rows(s):
        u = z * factor - off
        if p["bias"] is not None:
            u = u + p["bias"].double()
        u = u / p["temperature"][t].double()
        if ok is not None:
            u[~ok] = -math.inf
        lse[t] = torch.logsumexp(u, 0)
        if u_all is not None:
            u_all[t] = u
        if s["chosen"] is not None:
            logp[t] = u[s["chosen"][t]] - lse[t]
    out = {} if u_all is None else {"out": u_all}
    out["lse"] = lse
    return out if s["chosen"] is None else {**out, "logp": logp}


def _exact_adjust_bwd(s):
    p, (T, V) = s["policy"], s["z"].shape
    dz = torch.empty(T, V, dtype=torch.float64, device="cuda")
    for t, _, factor, _, ok in _exact_rows(s):
        dz[t] = s["du"][t].double() * factor / p["temperature"][t].double()
        if ok is not None:
            dz[t, ~ok] = 0.0
    return dz


def _exact_w4(s):
    V, G = s["codes"].shape[0], s["group"]
    x = s["x"].double()
    out = torch.empty(x.shape[0], V, dtype=torch.float64, device="cuda")
    for rows in _blocks(V, x.shape[1]):
        c = s["codes"][rows].long()
        w = torch.empty(c.shape[0], x.shape[1], dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = (c % 16).double(), (c // 16).double()
        zero = 8.0 if s["zeros"] is None else s["zeros"][rows].double().repeat_interleave(G, 1)
        w = (w - zero) * s["scales"][rows].double().repeat_interleave(G, 1)
        out[:, rows] = x @ w.t()
    return out
