"""Operators of sampling and training around the vocabulary head whose speed is measured: draws from truncated laws, the
cross-entropy of the head with its gradients, and the AdamW step.

"draw": B sequences x K slots of logits x of V tokens.  y = x * (1 / tau) in float32; tokens with y below -2e38 do not exist, a row
without tokens, or with a NaN or +inf, has no law (nothing kept, token -1, confidence 0, log-sum-exp -inf).  Tokens are ordered by y
descending, then by id ascending, with weights w = exp(y - max y).  Kept is the shortest of three beginnings of that order: the first top_k
tokens; the fewest tokens whose mass reaches top_p of the mass top_k leaves; the tokens with w >= min_p.  The token drawn is the smallest
kept id at which the kept mass up to it, in the order of the ids, reaches u times the kept mass.  Outputs: y of what is kept and -inf
elsewhere, the log-sum-exp, the number of tokens kept, the token and its probability.

"grad": z[r, v] = (1 / tau) sum_k h[r, k] w[v, k], ce[r] = log sum_v exp z[r, v] - z[r, label r] (0 where the label is negative), and the
gradients of sum_r g[r] ce[r] in h and w.

"adamw": one step t over a list of tensors, with g the gradient: m <- b1 m + (1 - b1) g, v <- b2 v + (1 - b2) g^2,
p <- p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps), where p is a float32 copy of bf16 parameters if there is one.
States in 8 bits hold m and sqrt(v) of 256 elements at a time as e4m3 codes under one float32 scale, the largest magnitude / 448 (0 for
one below 2^-100), and a positive sqrt(v) never becomes 0 under a scale.
"""
import math

import torch

own = False

_LOWEST = -2e38
_LR, _B1, _B2, _EPS, _WD = 1e-4, 0.9, 0.95, 1e-8, 0.1


def listed():
    return [
        # one token of a toy model: latency is all it costs
        dict(name="draw_toy", op="draw", B=1, K=1, V=5000, dtype="f32", tau=1.0, top_k=50, top_p=0.9, min_p=0.0, masked=False),
        # the window of one sequence of an 8B model, nucleus sampling: what a round is given
        dict(name="draw_llada_b1", op="draw", B=1, K=8, V=126464, dtype="f32", tau=0.8, top_k=0, top_p=0.95, min_p=0.0, masked=False),
        # a few sequences, logits as a model in bf16 returns them (many are equal), behind a grammar, with all three limits
        dict(name="draw_ragged", op="draw", B=7, K=5, V=100003, dtype="bf16", tau=1.0, top_k=1000, top_p=0.98, min_p=0.02, masked=True),
        # batched serving of windows with everything
        dict(name="draw_dream_b32", op="draw", B=32, K=16, V=151936, dtype="f32", tau=0.7, top_k=200, top_p=0.95, min_p=0.01, masked=True),
        # the toy model's own training step, in float32
        dict(name="grad_toy", op="grad", R=61, d=64, V=1000, dtype="f32", tau=1.0),
        # one short sequence through an 8B model's head: W is read and its gradient written
        dict(name="grad_llada_r48", op="grad", R=48, d=4096, V=126464, dtype="bf16", tau=1.0),
        # a few hundred positions of a smaller model, nothing a round number
        dict(name="grad_ragged", op="grad", R=333, d=2048, V=50257, dtype="bf16", tau=0.9),
        # a batch of 2048 positions of an 8B model: three large products
        dict(name="grad_llada_r2048", op="grad", R=2048, d=4096, V=126464, dtype="bf16", tau=1.0),
        # the toy model's parameters, float32 all through: latency
        dict(name="adamw_toy", op="adamw", sizes="64000 4096 4096 4096 4096 64 64 16384 256 16384 64", dtype="f32", state="f32", master=False),
        # parameters of one block of an 8B model in bf16 with float32 copies and float32 states
        dict(name="adamw_block", op="adamw", sizes="16777216 16777216 16777216 16777216 50331648 50331648 50331648 4096 4096", dtype="bf16",
             state="f32", master=True),
        # the same kind of step with states in 8 bits, tensors that end inside a block of 256
        dict(name="adamw_8bit_ragged", op="adamw", sizes="10000019 4096 777 33554432 1 5000003 255", dtype="bf16", state="8bit", master=True),
        # an 8B model's head with states in 8 bits
        dict(name="adamw_8bit_head", op="adamw", sizes="517996544", dtype="bf16", state="8bit", master=True),
    ]


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    op = rng.choice(["draw", "grad", "adamw"])
    if op == "draw":
        while True:
            c = dict(op="draw", B=log(1, 64), K=rng.choice([1, 4, 8, 16, rng.randint(1, 32)]),
                     V=rng.choice([126464, 151936, log(200, 152000), log(8000, 152000)]), dtype=rng.choice(["f32", "f32", "bf16"]),
                     tau=rng.choice([0.5, 0.8, 1.0, 1.0]), top_k=rng.choice([0, 1, log(2, 5000), log(2, 200)]),
                     top_p=rng.choice([0.0, 1.0, round(rng.uniform(0.5, 0.999), 3), round(rng.uniform(0.8, 0.99), 3)]),
                     min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.2), 4)]), masked=rng.random() < 0.5)
            if c["B"] * c["K"] * c["V"] <= 32 * 16 * 151936:
                return c
    if op == "grad":
        while True:
            c = dict(op="grad", R=log(1, 4096), d=64 * log(1, 64), V=rng.choice([126464, 151936, log(200, 152000), log(8000, 152000)]),
                     dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), tau=rng.choice([0.8, 1.0, 1.0]))
            if c["R"] * c["d"] * c["V"] * (4 if c["dtype"] == "f32" else 1) <= 2048 * 4096 * 126464:
                return c
    sizes = [log(1, 40_000_000) for _ in range(rng.randint(1, 9))]
    dtype = rng.choice(["bf16", "bf16", "f32"])
    return dict(op="adamw", sizes=" ".join(str(n) for n in sizes), dtype=dtype, state=rng.choice(["f32", "8bit"]),
                master=dtype == "bf16" and rng.random() < 0.8)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + 54321) & 0x7FFFFFFFFFFFFFFF)
    return g


def _blocks(x):
    """x in rows of 256, the last one filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.numel() % 256)).view(-1, 256)


def _coded(x, positive):
    """e4m3 codes of x and the scales of its blocks of 256."""
    rows = _blocks(x)
    top = rows.abs().amax(1)
    top = torch.where(top < 2.0 ** -100, torch.zeros_like(top), top)
    y = rows * torch.where(top > 0, 448.0 / top, torch.zeros_like(top))[:, None]
    if positive:
        y = torch.where((rows > 0) & (y < 2.0 ** -9), torch.full((), 2.0 ** -9, device=x.device), y)
    return y.to(torch.float8_e4m3fn).view(-1)[:x.numel()], top / 448.0


def prepare(case, seed):
    c, g = case, _gen(seed)

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    kind = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    if c["op"] == "draw":
        B, K, V = c["B"], c["K"], c["V"]
        # slots from nearly sure to nearly flat; a few tokens stand out of a gaussian mass
        x = randn(B, K, V) * (1.0 + 2.0 * rand(B, K, 1))
        some = torch.randint(0, V, (B, K, 12), generator=g, device="cuda")
        x.scatter_(2, some, 6.0 + 10.0 * rand(B, K, 12))
        if c["masked"]:
            # grammars: one slot in three allows a few tokens, one in three about half, the others all; one in fifty leaves nothing
            share = rand(B, K, 1)
            allowed = rand(B, K, V) < torch.where(share < 0.33, 0.01, torch.where(share < 0.67, 0.5, 1.0))
            x = torch.where(allowed & (share < 0.98), x, torch.full((), -math.inf, device="cuda"))
        s = dict(c=c, logits=x.to(kind), uniforms=torch.randint(0, 1 << 23, (B, K), generator=g, device="cuda").add(0.5) * 2.0 ** -23)
        s["limits"] = {}
        if c["top_k"]:  # every request brings its own limits; some want none
            k = (c["top_k"] * (0.5 + rand(B))).int().clamp(min=1)
            s["limits"]["top_k"] = torch.where(rand(B) < 0.1, torch.zeros_like(k), k)
        if c["top_p"] < 1.0:
            s["limits"]["top_p"] = (c["top_p"] + (1.0 - c["top_p"]) * 0.5 * rand(B)).float()
        if c["min_p"]:
            s["limits"]["min_p"] = c["min_p"] * (0.5 + rand(B))
        if own:
            from paper_2605_14305_amd import binding as fb
            s["call"] = fb.DrawLogits(B, K, V, dtype=c["dtype"])
        return s
    if c["op"] == "grad":
        # a gaussian head; rows that point at a predicted token, which is the label in two of three rows, on top of noise
        R, d, V = c["R"], c["d"], c["V"]
        W = randn(V, d).mul_(0.02)
        label = torch.randint(0, V, (R,), generator=g, device="cuda")
        near = W[label]
        h = randn(R, d) * (2.0 / (0.02 * math.sqrt(d)))
        h = (h + near * ((math.log(V) + 3.0 * rand(R, 1)) / near.square().sum(-1, keepdim=True))) * c["tau"]
        label = torch.where(rand(R) < 0.33, torch.randint(0, V, (R,), generator=g, device="cuda"), label)
        if R > 4:  # positions of the prompt do not count
            label = torch.where(rand(R) < 0.1, torch.full_like(label, -1), label)
        s = dict(c=c, h=h.to(kind), W=W.to(kind), labels=label.to(torch.int32), weights=(0.5 + rand(R)) / R)
        if own:
            from paper_2605_14305_amd import binding as fb
            s["call"] = fb.HeadCrossEntropyGrad(R, d, V, dtype=c["dtype"])
        return s
    sizes = [int(n) for n in c["sizes"].split()]
    master = [randn(n).mul_(0.02) for n in sizes]
    s = dict(c=c, t=100, params=[x.to(kind) for x in master], m=[], v=[], m_scale=[], v_scale=[])
    s["master"] = master if c["master"] else None
    s["grads"] = [(randn(n) * 1e-3).to(kind) for n in sizes]
    for n in sizes:  # a hundred steps into training: the spread of the gradients differs from element to element
        r = torch.exp(randn(n)) * 1e-3
        m = randn(n) * r * 0.3
        if c["state"] == "f32":
            s["m"].append(m)
            s["v"].append(r * r)
        else:
            for key, x in (("m", m), ("v", r)):
                code, scale = _coded(x, key == "v")
                s[key].append(code)
                s[key + "_scale"].append(scale)
    if own:
        from paper_2605_14305_amd import binding as fb
        s["call"] = fb.AdamW(s["params"], s["grads"], lr=_LR, betas=(_B1, _B2), eps=_EPS, weight_decay=_WD, master=s["master"],
                             states={"8bit": "8bit-reciprocal"}.get(c["state"], c["state"]),  # the states above are elementwise torch's
                             m=s["m"], v=s["v"], m_scale=s["m_scale"], v_scale=s["v_scale"], step=s["t"])
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def _plain_draw(s):
    c = s["c"]
    B, K, V = c["B"], c["K"], c["V"]
    none = torch.full((), -math.inf, device="cuda")
    y = s["logits"].float() * (1.0 / torch.tensor(c["tau"], dtype=torch.float32)).item()
    law = ~((y == math.inf) | y.isnan()).any(2, keepdim=True)
    y = torch.where(law & (y >= _LOWEST), y, none)
    top = y.amax(2, keepdim=True)
    law = top > -math.inf
    # which tokens are kept hangs on sums next to a border: 64 bits
    order_y, order = torch.sort(y, dim=2, descending=True, stable=True)
    w = torch.exp(order_y.double() - torch.where(law, top, torch.zeros_like(top)).double())
    at = torch.arange(V, device="cuda")
    keep = order_y > -math.inf
    if "top_k" in s["limits"]:
        k = s["limits"]["top_k"][:, None, None]
        keep = keep & ((at < k) | (k <= 0))
    if "top_p" in s["limits"]:
        mass = torch.cumsum(torch.where(keep, w, torch.zeros_like(w)), 2)
        p = s["limits"]["top_p"].double()[:, None, None]
        before = torch.nn.functional.pad(mass, (1, 0))[:, :, :V]
        keep = keep & ((before < p * mass[:, :, -1:]) | (at == 0) | (p >= 1))
    if "min_p" in s["limits"]:
        keep = keep & ((w >= s["limits"]["min_p"].double()[:, None, None]) | (at == 0))
    kept = keep.sum(2).int()
    w = torch.zeros_like(w).scatter_(2, order, torch.where(keep, w, torch.zeros_like(w)))
    keep = torch.zeros_like(keep).scatter_(2, order, keep)
    out = torch.where(keep, y, none)
    mass = torch.cumsum(w, 2)
    total = mass[:, :, -1]
    lse = torch.where(law[:, :, 0], torch.log(total) + top[:, :, 0].double(), none.double()).float()
    reached = (mass >= s["uniforms"].double()[:, :, None] * total[:, :, None]) & (w > 0)
    token = torch.where(law[:, :, 0], reached.int().argmax(2), -1)
    conf = torch.where(law[:, :, 0], torch.gather(w, 2, token.clamp(min=0)[:, :, None])[:, :, 0] / total, torch.zeros_like(total)).float()
    return {"logits": out, "lse": lse, "kept": kept, "tokens": token.int(), "conf": conf}


def _plain_grad(s):
    c = s["c"]
    kind = s["h"].dtype
    h, W, inv = s["h"].float(), s["W"].float(), 1.0 / c["tau"]
    z = (h @ W.t()) * inv
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    label = s["labels"].long()
    counts = label >= 0
    at = label.clamp(min=0)[:, None]
    ce = torch.where(counts, (torch.log(total) + top - z.gather(1, at))[:, 0], torch.zeros_like(s["weights"]))
    p = e / total
    p.scatter_add_(1, at, torch.full_like(total, -1.0))
    p *= torch.where(counts, s["weights"] * inv, torch.zeros_like(s["weights"]))[:, None]
    return {"ce": ce, "loss": ce.sum(), "grad_h": (p @ W).to(kind), "grad_w": (p.t() @ h).to(kind)}


def _cat(tensors):
    return tensors[0] if len(tensors) == 1 else torch.cat(tensors)


def _back(tensors, x):
    torch._foreach_copy_(tensors, list(torch.split(x, [t.numel() for t in tensors])))


def _plain_adamw(s):
    c, t = s["c"], s["t"]
    n = [x.numel() for x in s["params"]]
    eight = c["state"] == "8bit"

    def decoded(key):
        if not eight:
            return _cat(s[key])
        return _cat([(_blocks(code.float()) * scale[:, None]).view(-1)[:code.numel()] for code, scale in zip(s[key], s[key + "_scale"])])

    def held(key, x):
        if not eight:
            return _back(s[key], x)
        coded = [_coded(part, key == "v") for part in torch.split(x, n)]
        torch._foreach_copy_([code.view(torch.uint8) for code in s[key]], [code.view(torch.uint8) for code, _ in coded])
        torch._foreach_copy_(s[key + "_scale"], [scale for _, scale in coded])

    g, p = _cat(s["grads"]).float(), _cat(s["master"] or s["params"]).float()
    m = decoded("m") * _B1 + g * (1.0 - _B1)
    v = decoded("v")
    v = (v * v if eight else v) * _B2 + g * g * (1.0 - _B2)
    r = torch.sqrt(v)
    p = p * (1.0 - _LR * _WD) - m / (r * (1.0 / math.sqrt(1.0 - _B2 ** t)) + _EPS) * (_LR / (1.0 - _B1 ** t))
    held("m", m)
    held("v", r if eight else v)
    if s["master"]:
        _back(s["master"], p)
    _back(s["params"], p)


def _state_of(s):
    keys = ("params", "m", "v") + (("master",) if s["master"] else ()) + (("m_scale", "v_scale") if s["c"]["state"] == "8bit" else ())
    return {k: s[k] for k in keys}


def run(s):
    c = s["c"]
    if c["op"] == "draw":
        if not own:
            return _plain_draw(s)
        tokens, conf, kept, lse, out = s["call"](s["logits"], s["uniforms"], temperature=c["tau"], **s["limits"])
        return {"logits": out, "lse": lse, "kept": kept, "tokens": tokens, "conf": conf}
    if c["op"] == "grad":
        if not own:
            return _plain_grad(s)
        ce, loss, grad_h, grad_w = s["call"](s["h"], s["W"], s["labels"], s["weights"], temperature=c["tau"])
        return {"ce": ce, "loss": loss[0], "grad_h": grad_h, "grad_w": grad_w}
    s["t"] += 1
    if own:
        s["call"].step()
    else:
        _plain_adamw(s)
    return _state_of(s)


def work(case):
    """Inputs read once and outputs written once."""
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "draw":
        rows = c["B"] * c["K"]
        return {"bytes": rows * (c["V"] * (e + 4) + 20) + 12 * c["B"], "flops": 8 * rows * c["V"]}
    if c["op"] == "grad":
        R, d, V = c["R"], c["d"], c["V"]
        return {"bytes": 2 * e * (V * d + R * d) + 12 * R, "flops": 6 * R * d * V}
    n = sum(int(x) for x in c["sizes"].split())
    state = 16 if c["state"] == "f32" else 4 + 16 / 256
    return {"bytes": n * (2 * e + e + (8 if c["master"] else 0) + state) - (e * n if c["master"] else 0), "flops": 16 * n}


# ------------------------------------------------------------------------------------------------
# the same in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_draw(s):
    """Row by row: the existing tokens alone are sorted, and the three limits are lengths of that list."""
    c = s["c"]
    B, K, V = c["B"], c["K"], c["V"]
    scaled = s["logits"].float().mul(float(torch.tensor(1.0) / torch.tensor(c["tau"])))
    out = torch.full((B, K, V), -math.inf, dtype=torch.float64, device="cuda")
    lse = torch.full((B, K), -math.inf, dtype=torch.float64)
    kept, tokens, conf = torch.zeros(B, K, dtype=torch.int32), torch.full((B, K), -1, dtype=torch.int32), torch.zeros(B, K, dtype=torch.float64)
    limit = {k: v.double().cpu().tolist() for k, v in s["limits"].items()}
    us = s["uniforms"].double().cpu()
    for b in range(B):
        for m in range(K):
            row = scaled[b, m].double()
            ids = torch.nonzero(row >= _LOWEST)[:, 0]
            if ids.numel() == 0 or not bool((row < math.inf).all()):
                continue
            rank = ids[torch.argsort(-row[ids], stable=True)]
            weight = (row[rank] - row[rank[0]]).exp()
            length = rank.numel()
            k = int(limit["top_k"][b]) if "top_k" in limit else 0
            if k > 0:
                length = min(length, k)
            of_k = length
            if "top_p" in limit and limit["top_p"][b] < 1:
                sums = weight[:of_k].cumsum(0)
                length = min(length, int((sums < limit["top_p"][b] * sums[-1]).sum()) + 1)
            if "min_p" in limit:
                length = max(1, min(length, int((weight[:of_k] >= limit["min_p"][b]).sum())))
            chosen, by_id = torch.sort(rank[:length])
            mass = weight[:length][by_id]
            sums = mass.cumsum(0)
            j = int(torch.nonzero((sums >= us[b, m].item() * sums[-1]) & (mass > 0))[0, 0])
            out[b, m, chosen] = row[chosen]
            lse[b, m] = (row[rank[0]] + sums[-1].log()).item()
            kept[b, m], tokens[b, m], conf[b, m] = length, int(chosen[j]), (mass[j] / sums[-1]).item()
    return {"logits": out, "lse": lse, "kept": kept, "tokens": tokens, "conf": conf}


def _exact_grad(s):
    """Row block by row block: ce by torch's own log-sum-exp in 64 bits, gradients from probabilities exp(z - lse)."""
    c = s["c"]
    R, tau = c["R"], c["tau"]
    W, h = s["W"].double(), s["h"].double()
    ce = torch.zeros(R, dtype=torch.float64, device="cuda")
    grad_h, grad_w = torch.zeros_like(h), torch.zeros_like(W)
    for a in range(0, R, 512):
        some = slice(a, min(R, a + 512))
        z = (h[some] / tau) @ W.t().contiguous()
        lse = torch.logsumexp(z, 1)
        label = s["labels"][some].long()
        rows = torch.nonzero(label >= 0)[:, 0]
        ce[some][rows] = lse[rows] - z[rows, label[rows]]
        z = (z - lse[:, None]).exp_()
        z[rows, label[rows]] -= 1.0
        z *= ((label >= 0).double() * s["weights"][some].double() / tau)[:, None]
        grad_h[some] = z @ W
        grad_w += z.t().contiguous() @ h[some]
    return {"ce": ce, "loss": ce.sum(), "grad_h": grad_h, "grad_w": grad_w}


def _exact_adamw(s):
    """Tensor by tensor; what 8 bits hold is given before its rounding, in units of the scale."""
    t, eight = s["t"] + 1, s["c"]["state"] == "8bit"
    found = {"params": [], "m": [], "v": [], "master": [], "m_scale": [], "v_scale": []}
    for i, param in enumerate(s["params"]):
        g = s["grads"][i].double()
        p = (s["master"][i] if s["master"] else param).double()
        first, second = s["m"][i].double(), s["v"][i].double()
        if eight:
            first = first * s["m_scale"][i].double().repeat_interleave(256)[:g.numel()]
            second = (second * s["v_scale"][i].double().repeat_interleave(256)[:g.numel()]) ** 2
        first = first + (1.0 - _B1) * (g - first)
        second = second + (1.0 - _B2) * (g ** 2 - second)
        p = p - _LR * _WD * p - _LR * (first / (1.0 - _B1 ** t)) / ((second / (1.0 - _B2 ** t)) ** 0.5 + _EPS)
        found["params"].append(p)
        found["master"].append(p)
        if not eight:
            found["m"].append(first)
            found["v"].append(second)
            continue
        for key, x in (("m", first), ("v", second ** 0.5)):
            scale = torch.nn.functional.pad(x.abs(), (0, -x.numel() % 256)).view(-1, 256).amax(1) / 448.0
            found[key].append(x / scale.repeat_interleave(256)[:x.numel()])
            found[key + "_scale"].append(scale)
    return {k: found[k] for k in _state_of(s)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"draw": _exact_draw, "grad": _exact_grad, "adamw": _exact_adamw}[case["op"]](s)
