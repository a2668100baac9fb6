"""The operators that close the policy's loop, as cases whose time and results can be measured.

A rollout draws a token from every row of logits, training updates the weights with the gradients that the loss leaves, and
the updated head is laid out in 4 bits again for the next rollouts.  Every case is one call of one entry point, or the two
calls of an optimizer step:
  sample       logits -> a drawn token of the policy cut by top-k, top-p and min-p, its log-prob, optionally the entries kept
  adamw        (global norm of all gradients ->) a step of AdamW over many tensors, states in 32 bits or in 8
  w4_quantize  the head's weight -> 4-bit codes with a scale, and maybe a zero point, per group
Sizes are those of the workloads in synth/ and bench.py (vocabulary 151,936 and 32,000, hidden sizes 1,536 and 4,096) and
generic odd ones.
"""
import math

import torch

own = False  # plain torch operations; True: the library's operators

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LR, BETA1, BETA2, EPS, DECAY, STEP, MAX_NORM, SEED = 8.5e-6, 0.9, 0.999, 1e-8, 0.017, 300, 1.0, 20251206


def listed():
    return [
        # one sequence that decodes alone, nucleus sampling: latency
        {"name": "sample_1_nucleus", "op": "sample", "T": 1, "V": 32000, "z": "f32", "shape": "peaked", "tau": True, "k": 0,
         "p": 0.95, "min_p": 0.0, "full": True, "allowed": False},
        # a decoding step of 64 sequences on adjusted logits
        {"name": "sample_64_nucleus", "op": "sample", "T": 64, "V": 151936, "z": "f32", "shape": "peaked", "tau": True, "k": 0,
         "p": 0.95, "min_p": 0.0, "full": True, "allowed": False},
        # a step of 300 sequences under all three cuts whose kept entries training sees again, a vocabulary that is no
        # multiple of anything
        {"name": "sample_300_all_odd", "op": "sample", "T": 300, "V": 50001, "z": "f32", "shape": "peaked", "tau": True, "k": 50,
         "p": 0.9, "min_p": 0.02, "full": False, "allowed": True},
        # flat rows early in training: nuclei of tens of thousands of entries, many of them equal in bfloat16
        {"name": "sample_256_flat", "op": "sample", "T": 256, "V": 151936, "z": "bf16", "shape": "flat", "tau": False, "k": 0,
         "p": 0.9, "min_p": 0.0, "full": True, "allowed": True},
        # the paper's rollouts, uncut (temperature 1, top-p 1, all entries): 256 prompts x 4 samples decode together
        {"name": "sample_1024_uncut", "op": "sample", "T": 1024, "V": 151936, "z": "bf16", "shape": "peaked", "tau": False, "k": 0,
         "p": 1.0, "min_p": 0.0, "full": False, "allowed": False},
        # norms' gains and small matrices of a policy: latency
        {"name": "adamw_small", "op": "adamw", "tensors": 24, "n": 2 ** 20, "sizes": "mixed", "param": "f32", "grad": "f32",
         "state": "f32", "copy": False, "clip": True},
        # the head at the 1.5B-scale hidden size: fp32 weights, their bfloat16 copy for the forward pass, clipped gradients
        {"name": "adamw_head", "op": "adamw", "tensors": 1, "n": 151936 * 1536, "sizes": "even", "param": "f32", "grad": "bf16",
         "state": "f32", "copy": True, "clip": True},
        # the same head with both states in 8 bits
        {"name": "adamw_head_8bit", "op": "adamw", "tensors": 1, "n": 151936 * 1536, "sizes": "even", "param": "f32",
         "grad": "bf16", "state": "8bit", "copy": True, "clip": True},
        # many tensors of odd sizes, bfloat16 weights without a copy in fp32 (rounded stochastically), 8-bit states
        {"name": "adamw_odd_8bit", "op": "adamw", "tensors": 300, "n": 5 * 10 ** 7, "sizes": "odd", "param": "bf16",
         "grad": "bf16", "state": "8bit", "copy": False, "clip": False},
        # the odd tensors in 32 bits
        {"name": "adamw_odd", "op": "adamw", "tensors": 300, "n": 5 * 10 ** 7, "sizes": "odd", "param": "f32",
         "grad": "f32", "state": "f32", "copy": False, "clip": True},
        # the bfloat16 head, 1.5B scale, laid out for the next rollouts
        {"name": "w4_quantize_1536", "op": "w4_quantize", "H": 1536, "V": 151936, "group": 128, "w": "bf16", "scale": "bf16",
         "zeros": False},
        # an fp32 head, 8B-scale hidden size, fine groups with zero points
        {"name": "w4_quantize_zeros", "op": "w4_quantize", "H": 4096, "V": 32001, "group": 32, "w": "f32", "scale": "f32",
         "zeros": True},
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
    op = rng.choice(["sample", "sample", "sample", "adamw", "adamw", "w4_quantize"])
    if op == "sample":
        V = _vocab(rng)
        return {"op": op, "T": _log_int(rng, 1, 1024 * 151936 // max(V, 151936)), "V": V, "z": rng.choice(["f32", "bf16"]),
                "shape": rng.choice(["peaked", "peaked", "flat"]), "tau": rng.random() < 0.6,
                "k": rng.choice([0, 0, 1, _log_int(rng, 2, 1000)]), "p": rng.choice([1.0, round(rng.uniform(0.5, 0.99), 3)]),
                "min_p": rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.2), 3)]), "full": rng.random() < 0.5,
                "allowed": rng.random() < 0.4}
    if op == "adamw":
        tensors = rng.choice([1, _log_int(rng, 2, 400)])
        return {"op": op, "tensors": tensors, "n": max(_log_int(rng, 10 ** 5, 2 * 10 ** 8), 64 * tensors),
                "sizes": rng.choice(["mixed", "even", "odd"]), "param": rng.choice(["f32", "f32", "bf16"]),
                "grad": rng.choice(["f32", "bf16"]), "state": rng.choice(["f32", "8bit"]), "copy": rng.random() < 0.4,
                "clip": rng.random() < 0.7}
    group = rng.choice([32, 64, 128])
    H = rng.choice([896, 1536, 2048, 4096, _log_int(rng, 2, 32) * 128 + rng.choice([0, 128 - group if group < 128 else 0])])
    return {"op": op, "H": H, "V": min(_vocab(rng), 151936 * 1536 // H), "group": group, "w": rng.choice(["f32", "bf16"]),
            "scale": rng.choice(["bf16", "f32"]), "zeros": rng.random() < 0.5}


# ---- inputs ------------------------------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(0x5A3D + 7919 * int(seed))
    return g


def _sample_inputs(case, g):
    T, V, dev = case["T"], case["V"], "cuda"
    rand = lambda *s: torch.rand(*s, generator=g, device=dev)
    z = torch.randn(T, V, generator=g, device=dev)
    if case["shape"] == "flat":
        z *= 0.4 + 0.6 * rand(T, 1)
    else:
        # a bulk of unlikely tokens and, for each row, 200 that its context raises, by little in some rows and much in others
        z *= 1.5 + 2.0 * rand(T, 1)
        at = torch.randint(0, V, (T, 200), generator=g, device=dev)
        z.scatter_add_(1, at, 16.0 * rand(T, 1) * rand(T, 200) ** 2)
    d = {"z": z.to(DTYPES[case["z"]]), "uniform": rand(T), "temperature": None, "top_k": None, "top_p": None, "min_p": None}
    if case["tau"]:
        d["temperature"] = 0.6 + 0.7 * rand(T)
    if case["k"]:
        # requests of one batch have strengths of their own
        d["top_k"] = torch.randint((case["k"] + 1) // 2, case["k"] + 1, (T,), generator=g, device=dev).to(torch.int32)
    if case["p"] < 1.0:
        d["top_p"] = case["p"] - 0.1 * rand(T) * (rand(T) < 0.5)
    if case["min_p"]:
        d["min_p"] = case["min_p"] * (0.5 + 0.5 * rand(T))
    return d


def _sizes(case):
    """Elements of each tensor; all together about case["n"]."""
    k, n = case["tensors"], case["n"]
    if k == 1:
        return [n | 1 if case["sizes"] == "odd" else n]
    if case["sizes"] == "even":
        return [max(1, n // k // 64) * 64] * k
    if case["sizes"] == "mixed":  # half of them gains of a norm, the others matrices
        small = max(64, min(1536, n // k // 8 // 64 * 64))
        return [small if i % 2 else max(64, (2 * n // k - small) // 64 * 64) for i in range(k)]
    # odd sizes from a few elements to many
    part = [(1 + i % 17) ** 2 for i in range(k)]
    return [max(1, n * p // sum(part)) | 1 for p in part]


PAD = 64  # elements that each tensor's place in the common storage is a multiple of


def _views(flat, sizes):
    """The tensors, each at its own place of the common storage `flat`."""
    got, at = [], 0
    for n in sizes:
        got.append(flat[at:at + n])
        at += -(-n // PAD) * PAD
    return got


def _adamw_inputs(case, g):
    sizes = _sizes(case)
    places = torch.tensor([-(-n // PAD) * PAD for n in sizes])
    total = int(places.sum())
    dev = "cuda"
    which = torch.repeat_interleave(torch.arange(len(sizes), device=dev), places.to(dev), output_size=total)
    at = torch.arange(total, device=dev) - (torch.cumsum(places, 0) - places).to(dev)[which]
    inside = at < torch.tensor(sizes, device=dev)[which]
    randn = lambda: torch.randn(total, generator=g, device=dev)
    # tensors with scales of their own, elements of one tensor over a few powers of ten
    spread = torch.exp(1.5 * randn()) * torch.exp(1.0 * torch.randn(len(sizes), generator=g, device=dev))[which] * inside
    grad = (3e-4 * randn() * spread).to(DTYPES[case["grad"]])
    m = 6e-5 * randn() * spread
    v = 1e-7 * (0.5 + torch.rand(total, generator=g, device=dev)) * spread * spread
    param = (0.02 * randn() * inside).to(DTYPES[case["param"]])
    d = {"param": param, "grad": grad, "copy": param.to(torch.bfloat16) if case["copy"] else None, "which": which.to(torch.int32), "at": at}
    if case["state"] == "f32":
        d.update(m=m, v=v, scales=None)
    else:
        # held as what an earlier step left: float8 values and, per 32 elements, a power of two
        m8, ms = _to_blocks(m, torch.float8_e4m3fn, 7)
        v8, vs = _to_blocks(v, torch.float8_e5m2, 14)
        d.update(m=m8, v=v8, scales=torch.stack([ms, vs]))
    del spread, m, v, inside
    d["params"], d["grads"], d["ms"], d["vs"] = (_views(d[k], sizes) for k in ("param", "grad", "m", "v"))
    d["copies"] = _views(d["copy"], sizes) if case["copy"] else None
    d["scale_rows"] = None
    if d["scales"] is not None:
        rows, first = [], 0
        for n in sizes:
            rows.append((d["scales"][0, first:first + -(-n // 32)], d["scales"][1, first:first + -(-n // 32)]))
            first += -(-n // PAD) * PAD // 32
        d["scale_rows"] = rows
    if case["state"] == "f32" and case["param"] == "f32":
        del d["which"], d["at"]  # nothing is rounded by chance
    return d


def _w4_inputs(case, g):
    w = torch.randn(case["V"], case["H"], generator=g, device="cuda").mul_(0.02)
    w *= 0.5 + torch.rand(case["V"], 1, generator=g, device="cuda")
    if case["zeros"]:
        w += 0.004
    return {"w": w.to(DTYPES[case["w"]])}


def prepare(case, seed):
    g = _generator(seed)
    make = {"sample": _sample_inputs, "adamw": _adamw_inputs, "w4_quantize": _w4_inputs}[case["op"]]
    d = make(case, g)
    d["case"] = case
    return d


# ---- one pass ----------------------------------------------------------------------------------------------------


def run(state):
    op = state["case"]["op"]
    return (_OWN if own else _PLAIN)[op](state)


def _own_sample(s):
    import paper_2512_06547_amd as a3po
    out = a3po.sample(s["z"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                      want_logp_full=s["case"]["full"], want_allowed=s["case"]["allowed"], want_kept=True)
    return {k: out[k] for k in ("token", "logp", "logp_full", "kept", "allowed") if out[k] is not None}


def _own_adamw(s):
    import paper_2512_06547_amd as a3po
    norm = a3po.grad_norm(s["grads"]) if s["case"]["clip"] else None
    a3po.adamw_step(s["params"], s["grads"], s["ms"], s["vs"], scales=s["scale_rows"], copies=s["copies"], step=STEP, lr=LR,
                    beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, norm=norm, max_norm=MAX_NORM, seed=SEED)
    return _adamw_outputs(s, norm)


def _own_w4(s):
    import paper_2512_06547_amd as a3po
    c = s["case"]
    codes, scales, zeros = a3po.w4_quantize(s["w"], group=c["group"], scale_dtype=DTYPES[c["scale"]], zeros=c["zeros"])
    return {"codes": codes, "scales": scales, "zeros": zeros} if c["zeros"] else {"codes": codes, "scales": scales}


def _adamw_outputs(s, norm):
    """What the step leaves: weights, their copy and the states, 8-bit ones as float8 values with their powers of two."""
    out = {k: s[k] for k in ("param", "copy", "m", "v") if s[k] is not None}
    if s["scales"] is not None:
        out["scales"] = s["scales"].view(torch.float8_e8m0fnu)
    return out if norm is None else {**out, "norm": norm}


def _plain_sample(s):
    c, z = s["case"], s["z"]
    T, V = z.shape
    # 64 bits: a token is the entry in whose part of the sum the drawn number falls, and its neighbour's begins at its end
    u = z.double()
    if s["temperature"] is not None:
        u = u / s["temperature"].double()[:, None]
    x = u - u.amax(1, keepdim=True)
    w = torch.exp(x)
    kept = z > -math.inf
    if s["top_k"] is not None or s["top_p"] is not None:
        # the order of the cuts: larger first, the lower index first among equals
        order = torch.sort(z, dim=1, descending=True, stable=True).indices
        before = torch.cumsum(w.gather(1, order), 1)
        rank = torch.arange(V, device=z.device)
        among = torch.ones_like(kept)
        total = before[:, -1:]
        if s["top_k"] is not None:
            k = s["top_k"].long()[:, None].clamp(max=V)
            among = rank < k
            total = before.gather(1, k - 1)
        if s["top_p"] is not None:
            # the fewest whose mass reaches top_p of what top_k left: an entry stays if those ahead of it do not
            mass = torch.zeros_like(before)
            mass[:, 1:] = before[:, :-1]
            among = among & ((mass < s["top_p"].double()[:, None] * total) | (rank == 0))
        kept &= torch.zeros_like(kept).scatter_(1, order, among)
    if s["min_p"] is not None:
        kept &= w >= s["min_p"].double()[:, None]
    sums = torch.cumsum(w * kept, 1)
    total = sums[:, -1]
    token = (sums <= (s["uniform"].double() * total)[:, None]).sum(1)
    at = x.gather(1, token[:, None])[:, 0]
    out = {"token": token.to(torch.int32), "logp": (at - torch.log(total)).float(), "kept": kept.sum(1).to(torch.int32)}
    if c["full"]:
        out["logp_full"] = (at - torch.log(w.sum(1))).float()
    if c["allowed"]:
        out["allowed"] = _words(kept)
    return out


def _words(kept):
    """32 entries a word, the first in its lowest bit."""
    T, V = kept.shape
    bits = torch.zeros(T, -(-V // 32) * 32, dtype=torch.int64, device=kept.device)
    bits[:, :V] = kept
    return (bits.view(T, -1, 32) << torch.arange(32, device=kept.device)).sum(2).to(torch.int32)


def _mix(x):
    """32 bits of chance for every whole number: two multiplications and three shifted sums without carry."""
    x = x ^ (x >> 16)
    x = (x * 0x85EBCA6B) & 0xFFFFFFFF
    x = x ^ (x >> 13)
    x = (x * 0xC2B2AE35) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _chance(which, at):
    """The 32 random bits of element `at` of tensor `which` under SEED (which fits 32 bits, as `at` does)."""
    key = _mix((which.long() + 1) * 0x9E3779B9 + SEED & 0xFFFFFFFF)
    return _mix(at ^ key)


def _exponents(x):
    """For every 32 values, the biased exponent of the largest, as int32."""
    top = x.view(-1, 32).abs().amax(1)
    return top.view(torch.int32) >> 23


def _to_blocks(x, dtype, top):
    """(float8 values, powers of two): the largest of 32 values gets the exponent `top`; round to nearest."""
    e = (_exponents(x) - top).clamp_(min=1)
    up = ((254 - e) << 23).view(torch.float32)
    return (x.view(-1, 32) * up[:, None]).reshape(-1).to(dtype), e.to(torch.uint8)


def _from_blocks(x8, scales):
    e = scales.to(torch.int32)
    return (x8.float().view(-1, 32) * (e << 23).view(torch.float32)[:, None]).reshape(-1)


def _by_chance_e5m2(x, bits):
    """x >= 0 in units of its block as float8 e5m2, up or down by 21 random bits so that the mean is x; what is not zero
    stays so."""
    code = ((x.view(torch.int32) + bits) >> 21) - 448
    low = torch.floor(x * 65536.0 + bits.float() * 2.0 ** -21).to(torch.int32)
    code = torch.where(x < 2.0 ** -14, low, code)
    code = torch.where(x > 0, code.clamp(min=1), code)
    return code.to(torch.uint8).view(torch.float8_e5m2)


def _by_chance_bf16(x, bits):
    """x as bfloat16, to or from zero by 16 random bits so that the mean is x."""
    return ((x.view(torch.int32) + bits) & -65536).view(torch.float32).to(torch.bfloat16)


def _plain_adamw(s):
    c = s["case"]
    g = s["grad"].float()
    norm, go = None, None
    if c["clip"]:
        norm = torch.sqrt(g.double().square().sum()).float().view(1)
        go = torch.isfinite(norm)
        g = g * torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    m, v, p = s["m"], s["v"], s["param"].float()
    if s["scales"] is not None:
        m, v = _from_blocks(m, s["scales"][0]), _from_blocks(v, s["scales"][1])
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    root = torch.sqrt(v) * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS
    p = p * (1 - LR * DECAY) - (LR / (1 - BETA1 ** STEP)) * (m / root)
    chance = _chance(s["which"], s["at"]) if "which" in s else None
    if c["param"] == "bf16":
        p = _by_chance_bf16(p, (chance >> 16).to(torch.int32))
    new = {"param": p}
    if c["copy"]:
        new["copy"] = p.to(torch.bfloat16)
    if s["scales"] is None:
        new.update(m=m, v=v)
    else:
        new["m"], ms = _to_blocks(m, torch.float8_e4m3fn, 7)
        vs = (_exponents(v) - 14).clamp_(min=1)
        up = ((254 - vs) << 23).view(torch.float32)
        new["v"] = _by_chance_e5m2((v.view(-1, 32) * up[:, None]).reshape(-1), (chance & 0x1FFFFF).to(torch.int32))
        new["scales"] = torch.stack([ms, vs.to(torch.uint8)])
    for k, x in new.items():
        bits = torch.uint8 if "float8" in str(x.dtype) else x.dtype
        now = s[k].view(bits)
        now.copy_(x.view(bits) if go is None else torch.where(go, x.view(bits), now))
    return _adamw_outputs(s, norm)


def _plain_w4(s):
    c = s["case"]
    w = s["w"].float().view(c["V"], c["H"] // c["group"], c["group"])
    hi, lo = w.amax(2), w.amin(2)
    if c["zeros"]:
        # 0 is among the values that codes stand for
        hi, lo = hi.clamp(min=0.0), lo.clamp(max=0.0)
        scale = ((hi - lo) * (1.0 / 15.0)).to(DTYPES[c["scale"]])
    else:
        scale = torch.maximum(hi * (1.0 / 7.0), lo * (-1.0 / 8.0)).to(DTYPES[c["scale"]])
    inverse = torch.where(scale > 0, 1.0 / scale.float(), torch.zeros_like(hi))
    zero = torch.round(-lo * inverse).clamp(0.0, 15.0) if c["zeros"] else torch.full_like(hi, 8.0)
    code = (torch.round(w * inverse[:, :, None]) + zero[:, :, None]).clamp_(0.0, 15.0).to(torch.uint8).view(c["V"], c["H"])
    out = {"codes": code[:, 0::2] | (code[:, 1::2] << 4), "scales": scale}
    return {**out, "zeros": zero.to(torch.uint8)} if c["zeros"] else out


_OWN = {"sample": _own_sample, "adamw": _own_adamw, "w4_quantize": _own_w4}
_PLAIN = {"sample": _plain_sample, "adamw": _plain_adamw, "w4_quantize": _plain_w4}


# ---- in 64 bits --------------------------------------------------------------------------------------------------


def exact(case, seed):
    """What run() returns, from the definitions in 64 bits; None for whole numbers, which have no value in between."""
    s = prepare(case, seed)
    return {"sample": _exact_sample, "adamw": _exact_adamw, "w4_quantize": _exact_w4}[case["op"]](s)


def _exact_sample(s):
    case, V = s["case"], s["z"].shape[1]
    logp, full = [], []
    for t in range(s["z"].shape[0]):
        z = s["z"][t].double()
        x = (z - z.max()) / (1.0 if s["temperature"] is None else s["temperature"][t].double())
        order = torch.argsort(-z, stable=True)
        mass = torch.exp(x[order])
        n = V if s["top_k"] is None else min(V, int(s["top_k"][t]))
        if s["top_p"] is not None:
            reached = torch.cumsum(mass[:n], 0)
            n = min(n, 1 + int(torch.searchsorted(reached, s["top_p"][t].double() * reached[-1])))
        if s["min_p"] is not None:
            n = min(n, int((x >= torch.log(s["min_p"][t].double())).sum()))
        at = torch.sort(order[:n]).values
        upto = torch.cumsum(torch.exp(x[at]), 0)
        y = at[torch.searchsorted(upto, s["uniform"][t].double() * upto[-1], right=True)]
        logp.append(x[y] - torch.log(upto[-1]))
        full.append(x[y] - torch.logsumexp(x, 0))
    out = {"token": None, "logp": torch.stack(logp), "kept": None}
    if case["full"]:
        out["logp_full"] = torch.stack(full)
    return {**out, "allowed": None} if case["allowed"] else out


def _grid(x, bits, lowest):
    """The distance of the floating-point numbers around x that have `bits` bits, exponents not below `lowest`."""
    return torch.exp2(torch.clamp(torch.frexp(x).exponent.double() - 1, min=lowest) - (bits - 1))


def _exact_adamw(s):
    case, d = s["case"], torch.float64
    g, m, v, p = s["grad"].to(d), s["m"].to(d), s["v"].to(d), s["param"].to(d)
    out = {}
    if s["scales"] is not None:
        unit = torch.exp2(s["scales"].to(d) - 127.0).repeat_interleave(32, 1)
        m, v = m * unit[0], v * unit[1]
    if case["clip"]:
        norm = torch.linalg.vector_norm(g)
        out["norm"] = norm.view(1)
        if norm + 1e-6 > MAX_NORM:
            g = g * (MAX_NORM / (norm + 1e-6))
    m += (1.0 - BETA1) * (g - m)
    v += (1.0 - BETA2) * (g * g - v)
    p -= LR * (DECAY * p + m / (1.0 - BETA1 ** STEP) / (torch.sqrt(v / (1.0 - BETA2 ** STEP)) + EPS))
    if "which" in s:
        seeds = torch.tensor([(0x9E3779B9 * (i + 1) + SEED) % 2 ** 32 for i in range(case["tensors"])], device="cuda")
        for shift, factor in ((16, 0x85EBCA6B), (13, 0xC2B2AE35), (16, 1)):
            seeds = (seeds ^ (seeds >> shift)) * factor % 2 ** 32
        chance = s["at"] ^ seeds[s["which"].long()]
        for shift, factor in ((16, 0x85EBCA6B), (13, 0xC2B2AE35), (16, 1)):
            chance = (chance ^ (chance >> shift)) * factor % 2 ** 32
    if case["param"] == "bf16":
        step = _grid(p, 8, -126.0)
        p = torch.sign(p) * torch.floor(p.abs() / step + (chance // 65536).to(d) / 65536.0) * step
    out["param"] = p
    if case["copy"]:
        out["copy"] = p
    if s["scales"] is None:
        return {**out, "m": m, "v": v}
    # the largest of a block goes to the exponent 7 or 14; numbers of 4 and 3 bits
    for x, top in ((m, 7.0), (v, 14.0)):
        unit = _grid(x.view(-1, 32).abs().amax(1), 1, -126.0 + top + 1) * 2.0 ** -top
        x /= unit.repeat_interleave(32)
    step = _grid(m, 4, -6.0)
    out["m"] = torch.round(m / step) * step
    step = _grid(v, 3, -14.0)
    r = torch.floor(v / step + (chance % 2 ** 21).to(d) / 2.0 ** 21) * step
    out["v"] = torch.where((v > 0) & (r == 0), torch.full_like(r, 2.0 ** -16), r)
    return {**out, "scales": None}


def _exact_w4(s):
    c = s["case"]
    w = s["w"].double().view(c["V"], -1, c["group"])
    top, low = w.max(2).values, w.min(2).values
    if c["zeros"]:
        scale = (top.clamp(min=0.0) - low.clamp(max=0.0)) / 15.0
    else:
        scale = torch.maximum(top / 7.0, -low / 8.0)
    out = {"codes": None, "scales": scale}
    return {**out, "zeros": None} if c["zeros"] else out


def work(case):
    if case["op"] == "sample":
        n = case["T"] * case["V"]
        return {"bytes": n * (2 if case["z"] == "bf16" else 4) + (n / 8 if case["allowed"] else 0) + 24 * case["T"], "flops": 4.0 * n}
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        each = 2 * size[case["param"]] + size[case["grad"]] + (16 if case["state"] == "f32" else 4 + 4 / 32) + (2 if case["copy"] else 0)
        return {"bytes": n * each, "flops": 14.0 * n}
    n = case["V"] * case["H"]
    return {"bytes": n * (size[case["w"]] + 0.5 + (size[case["scale"]] + case["zeros"]) / case["group"]), "flops": 5.0 * n}
