"""The operators around the vocabulary head whose speed is measured: logits from a 4-bit head, and logits edited by
penalties, biases and grammar masks.

"mx4": logits[r, v] = (1 / tau) sum_k h[r, k] w[v, k] with w in the OCP MX 4-bit form: e2m1 codes, two per byte (the low
nibble is the even k), and one power-of-two scale (e8m0 byte) per 32 codes of a row.

"edit": B sequences x K window slots of logits.  For slot m of sequence b a token v has been generated n times if it occurs n
times in history[b, prompt_len[b] : history_len[b]] and prefix[b, : m] together, and it has been seen if n > 0 or it occurs
in the prompt history[b, : prompt_len[b]].  A logit x becomes: x / repetition if x > 0 else x * repetition, where seen;
minus frequency * n, minus presence where n > 0; plus the biases of the token; times 1 / tau; -inf where the slot's bit
mask does not allow the token.  Beside the edited logits the row's log-sum-exp (-inf for a row that leaves nothing).
"""
import math

import torch

own = False

_LUT = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # one token of a toy model: latency is all it costs
        dict(name="mx4_toy", op="mx4", R=1, d=512, V=5000, dtype="bf16", tau=1.0),
        # one token of an 8B model: the matrix-vector product itself
        dict(name="mx4_one_row", op="mx4", R=1, d=4096, V=126464, dtype="bf16", tau=1.0),
        # the draft half of a round of one sequence, window of 8
        dict(name="mx4_llada_b1", op="mx4", R=8, d=4096, V=126464, dtype="bf16", tau=1.0),
        # a few sequences in flight, nothing a round number
        dict(name="mx4_ragged", op="mx4", R=55, d=2560, V=100003, dtype="bf16", tau=0.8),
        # fp32 hidden states of a small model
        dict(name="mx4_f32", op="mx4", R=16, d=1024, V=32000, dtype="f32", tau=1.0),
        # the draft half of batched serving: 32 sequences, window of 16, the larger vocabulary
        dict(name="mx4_dream_b32", op="mx4", R=512, d=3584, V=151936, dtype="bf16", tau=1.0),
        # one token of a small model with a short history
        dict(name="edit_one_row", op="edit", B=1, K=1, V=32000, ld=32000, dtype="f32", history=300, prefix=False, penalties=True,
             n_bias=8, mask="none", tau=0.7),
        # a window of an 8B model: penalties, a bias list and a grammar
        dict(name="edit_llada_b1", op="edit", B=1, K=8, V=126464, ld=126464, dtype="f32", history=1024, prefix=True, penalties=True,
             n_bias=64, mask="slots", tau=1.0),
        # a few sequences, logits as a model in bf16 returns them, rows that end anywhere
        dict(name="edit_ragged", op="edit", B=5, K=11, V=100003, ld=100003, dtype="bf16", history=777, prefix=True, penalties=True,
             n_bias=17, mask="slots", tau=0.8),
        # long documents: 64 thousand tokens of history each
        dict(name="edit_long", op="edit", B=8, K=4, V=126464, ld=126464, dtype="f32", history=65536, prefix=False, penalties=True,
             n_bias=300, mask="none", tau=1.0),
        # constrained decoding and nothing else: a grammar per slot, some of which leave nothing
        dict(name="edit_grammar_b16", op="edit", B=16, K=8, V=126464, ld=126464, dtype="f32", history=0, prefix=False, penalties=False,
             n_bias=0, mask="slots", tau=1.0),
        # batched serving with everything
        dict(name="edit_dream_b32", op="edit", B=32, K=16, V=151936, ld=151936, dtype="f32", history=2048, prefix=True, penalties=True,
             n_bias=64, mask="slots", tau=1.0),
    ]


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    tau = rng.choice([0.5, 0.8, 1.0, 1.0])
    if rng.random() < 0.5:
        while True:
            # toy heads to those of 8B models; one row to a batch of windows
            c = dict(op="mx4", R=log(1, 512), d=64 * log(1, 64), V=rng.choice([126464, 151936, log(200, 152000), log(8000, 152000)]),
                     dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), tau=tau)
            if c["R"] * (3 if c["dtype"] == "f32" else 1) * c["d"] * c["V"] <= 512 * 3584 * 151936:
                return c
    while True:
        V = rng.choice([126464, 151936, log(200, 152000), log(8000, 152000)])
        c = dict(op="edit", B=log(1, 64), K=rng.choice([1, 4, 8, 16, rng.randint(1, 32)]), V=V, ld=V + rng.choice([0, 0, 1, 61]),
                 dtype=rng.choice(["f32", "f32", "bf16"]), history=rng.choice([0, log(1, 65536), log(100, 8000)]), prefix=rng.random() < 0.5,
                 penalties=rng.random() < 0.8, n_bias=rng.choice([0, 1, log(2, 300)]), mask=rng.choice(["none", "slots", "sequences"]), tau=tau)
        if c["B"] * c["K"] * V <= 32 * 16 * 151936 and c["B"] * c["history"] <= 8 * 65536:
            return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + 54321) & 0x7FFFFFFFFFFFFFFF)
    return g


def _quantised(W):
    """Codes and scales of a head, as a checkpoint in this form holds them: the smallest power of two whose sevenfold reaches the
    largest magnitude of 32, and the nearest of the 16 values."""
    V, d = W.shape
    X = W.view(V, d // 32, 32)
    mantissa, exponent = torch.frexp(X.abs().amax(2, keepdim=True))  # amax = mantissa 2^exponent, mantissa in [0.5, 1)
    e = (exponent - 3 + (mantissa > 0.875).int()).clamp(-126, 127)
    code = torch.bucketize((X * torch.exp2(-e.float())).abs(), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=W.device),
                           out_int32=True)
    code = (code + 8 * (X < 0).int()).view(V, d // 2, 2).to(torch.uint8)
    return code[:, :, 0] | (code[:, :, 1] << 4), (e + 127).to(torch.uint8).view(V, d // 32)


def prepare(case, seed):
    c, g = case, _gen(seed)
    V = c["V"]
    if c["op"] == "mx4":
        # a gaussian head; rows that each point at a predicted token on top of noise over the whole vocabulary
        R, d = c["R"], c["d"]
        W = torch.randn(V, d, generator=g, device="cuda").mul_(0.02)
        w = W[torch.randint(0, V, (R,), generator=g, device="cuda")]
        h = torch.randn(R, d, generator=g, device="cuda") * (2.0 / (0.02 * math.sqrt(d)))
        h = (h + w * ((math.log(V) + 7.0) / w.square().sum(-1, keepdim=True))) * c["tau"]
        codes, scales = _quantised(W)
        s = dict(c=c, h=h.to(torch.bfloat16 if c["dtype"] == "bf16" else torch.float32), codes=codes, scales=scales)
        if own:
            from paper_2605_14305_amd import binding as fb
            s["call"] = fb.Mx4Logits(R, d, V, dtype=c["dtype"])
        return s
    B, K, H = c["B"], c["K"], c["history"]
    logits = torch.randn(B, K, c["ld"], generator=g, device="cuda") * 3.0
    logits = logits.to(torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)[:, :, :V]
    x = {}
    if H:
        # few tokens make up most of a text: u^4 over the vocabulary, turned so that the frequent ones lie anywhere
        u = torch.rand(B, H, generator=g, device="cuda")
        x["history"] = (((u ** 4 * V).long() * 7919 + 13) % V).to(torch.int32)
        x["history_len"] = (H - torch.randint(0, H // 4 + 1, (B,), generator=g, device="cuda")).to(torch.int32)
        x["prompt_len"] = torch.randint(0, H // 2 + 1, (B,), generator=g, device="cuda").to(torch.int32)
    if c["prefix"]:
        x["prefix"] = torch.randint(0, V, (B, K), generator=g, device="cuda").to(torch.int32)
    if c["penalties"]:
        plain = torch.rand(B, generator=g, device="cuda") < 0.2  # requests that ask for none
        for name, low, high, none in (("repetition", 1.05, 1.4, 1.0), ("presence", -0.2, 1.0, 0.0), ("frequency", 0.0, 0.3, 0.0)):
            p = torch.rand(B, generator=g, device="cuda") * (high - low) + low
            x[name] = torch.where(plain, torch.full_like(p, none), p)
    if c["n_bias"]:
        ids = torch.randint(0, V, (B, c["n_bias"]), generator=g, device="cuda")
        used = torch.arange(c["n_bias"], device="cuda") < torch.randint(0, c["n_bias"] + 1, (B, 1), generator=g, device="cuda")
        x["bias_ids"] = torch.where(used, ids, torch.full_like(ids, -1)).to(torch.int32)
        x["bias_values"] = torch.randn(B, c["n_bias"], generator=g, device="cuda") * 4.0
    if c["mask"] != "none":
        # grammars: one slot in three allows a few tokens, one in three about half, the others all; one in fifty leaves nothing
        M, words = (K if c["mask"] == "slots" else 1), (V + 31) // 32
        kind = torch.rand(B, M, 1, generator=g, device="cuda")
        a, b, e, f, h = (torch.randint(-2 ** 31, 2 ** 31, (B, M, words), generator=g, device="cuda").to(torch.int32) for _ in range(5))
        allowed = torch.where(kind < 0.33, a & b & e & f & h, torch.where(kind < 0.67, a, torch.full_like(a, -1)))
        x["allowed"] = torch.where(kind > 0.98, torch.zeros_like(a), allowed)
    s = dict(c=c, logits=logits, x=x)
    if own:
        from paper_2605_14305_amd import binding as fb
        s["edits"] = fb.Edits(**x)
        s["call"] = fb.EditLogits(B, K, V, dtype=c["dtype"])
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def _plain_mx4(s):
    lut = torch.tensor(_LUT + tuple(-x for x in _LUT), device="cuda")
    codes, scales, V, d = s["codes"], s["scales"], s["c"]["V"], s["c"]["d"]
    w = torch.stack((lut[(codes & 15).int()], lut[(codes >> 4).int()]), 2).view(V, d // 32, 32)
    w = (w * torch.exp2(scales.float() - 127.0)[:, :, None]).view(V, d)
    return (s["h"].float() @ w.t()) * (1.0 / s["c"]["tau"])


def _plain_edit(s):
    c, x = s["c"], s["x"]
    B, K, V, H = c["B"], c["K"], c["V"], c["history"]
    y = s["logits"].float()
    n = torch.zeros(B, K, V + 1, device="cuda")  # column V takes what does not count
    seen = torch.zeros(B, 1, V + 1, device="cuda")
    if H:
        at = torch.arange(H, device="cuda")[None]
        ids = x["history"].long()
        prompt = (at < x["prompt_len"][:, None]) & (at < x["history_len"][:, None])
        later = (at >= x["prompt_len"][:, None]) & (at < x["history_len"][:, None])
        seen[:, 0].scatter_add_(1, torch.where(prompt, ids, torch.full_like(ids, V)), torch.ones(B, H, device="cuda"))
        count = torch.zeros(B, V + 1, device="cuda").scatter_add_(1, torch.where(later, ids, torch.full_like(ids, V)), torch.ones(B, H, device="cuda"))
        n += count[:, None]
    if "prefix" in x:
        earlier = torch.arange(K, device="cuda")[None, :] < torch.arange(K, device="cuda")[:, None]  # [slot, token of the prefix]
        ids = torch.where(earlier[None], x["prefix"].long()[:, None, :], torch.full((), V, device="cuda"))
        n.scatter_add_(2, ids, torch.ones(B, K, K, device="cuda"))
    n, seen = n[:, :, :V], seen[:, :, :V]
    if c["penalties"]:
        rep = x["repetition"][:, None, None]
        y = torch.where((n > 0) | (seen > 0), torch.where(y > 0, y / rep, y * rep), y)
        y = y - x["frequency"][:, None, None] * n
        y = y - x["presence"][:, None, None] * (n > 0)
    if c["n_bias"]:
        ids = x["bias_ids"].long()
        bias = torch.zeros(B, V + 1, device="cuda").scatter_add_(1, torch.where(ids < 0, torch.full_like(ids, V), ids), x["bias_values"])
        y = y + bias[:, None, :V]
    y = y * (1.0 / c["tau"])
    if c["mask"] != "none":
        bits = (x["allowed"][..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        y = torch.where(bits.flatten(2)[:, :, :V] != 0, y, torch.full((), -math.inf, device="cuda"))
    top = y.amax(2, keepdim=True)
    lse = torch.log(torch.exp(y - torch.where(top > -math.inf, top, torch.zeros_like(top))).sum(2)) + top[:, :, 0]
    return y, lse


def run(s):
    if s["c"]["op"] == "mx4":
        if own:
            return {"logits": s["call"](s["h"], s["codes"], s["scales"], temperature=s["c"]["tau"])}
        return {"logits": _plain_mx4(s)}
    if own:
        out, lse = s["call"](s["logits"], s["edits"], temperature=s["c"]["tau"])
    else:
        out, lse = _plain_edit(s)
    return {"logits": out, "lse": lse}


def work(case):
    """Codes, scales and hidden states (or logits, history, masks and lists) read once, the logits written once."""
    c = case
    if c["op"] == "mx4":
        nbytes = c["V"] * (c["d"] // 2 + c["d"] // 32) + c["R"] * c["d"] * (2 if c["dtype"] == "bf16" else 4) + 4 * c["R"] * c["V"]
        return {"bytes": nbytes, "flops": 2 * c["R"] * c["d"] * c["V"]}
    rows = c["B"] * c["K"]
    nbytes = rows * c["V"] * ((2 if c["dtype"] == "bf16" else 4) + 4) + 4 * rows + 4 * c["B"] * c["history"] + 8 * c["B"] * c["n_bias"]
    nbytes += {"none": 0, "slots": rows, "sequences": c["B"]}[c["mask"]] * ((c["V"] + 31) // 32) * 4
    return {"bytes": nbytes, "flops": 8 * rows * c["V"]}


# ------------------------------------------------------------------------------------------------
# the same in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_mx4(s):
    """Each code by its fields: exponent e and mantissa bit m stand for (1 + m / 2) 2^(e - 1), for m / 2 where e is zero."""
    c = s["c"]
    out = torch.empty(c["R"], c["V"], dtype=torch.float64, device="cuda")
    h = s["h"].double()
    for v in range(0, c["V"], 16384):
        byte = s["codes"][v:v + 16384].long()
        w = torch.empty(byte.shape[0], c["d"], dtype=torch.float64, device="cuda")
        for half in (0, 1):
            q = (byte >> (4 * half)) & 15
            e, m = ((q >> 1) & 3).double(), (q & 1).double()
            w[:, half::2] = torch.where(e > 0, (1.0 + m / 2) * 2.0 ** (e - 1), m / 2) * (1.0 - 2.0 * (q >> 3).double())
        w *= (2.0 ** (s["scales"][v:v + 16384].double() - 127.0)).repeat_interleave(32, 1)
        out[:, v:v + 16384] = h @ w.t().contiguous()
    return {"logits": out / c["tau"]}


def _exact_edit(s):
    """Sequence by sequence, the tokens that an edit touches found by counting the lists on the host."""
    c, x = s["c"], s["x"]
    B, K, V = c["B"], c["K"], c["V"]
    out = s["logits"].double()
    host = {k: v.cpu() for k, v in x.items() if k != "allowed"}
    column = torch.arange(V, device="cuda")
    for b in range(B):
        prompt, generated = torch.zeros(0, dtype=torch.long), torch.zeros(0, dtype=torch.long)
        if c["history"]:
            total, first = int(host["history_len"][b]), min(int(host["prompt_len"][b]), int(host["history_len"][b]))
            prompt, generated = host["history"][b, :first].long(), host["history"][b, first:total].long()
        for m in range(K):
            row = out[b, m]
            if c["penalties"]:
                g = generated if "prefix" not in host else torch.cat((generated, host["prefix"][b, :m].long()))
                n = torch.bincount(g, minlength=V).double().cuda()
                seen = (torch.bincount(prompt, minlength=V).cuda() > 0) | (n > 0)
                rep, pres, freq = (float(host[k][b]) for k in ("repetition", "presence", "frequency"))
                row = torch.where(seen, torch.where(row > 0, row / rep, row * rep), row) - freq * n - pres * (n > 0).double()
            if c["n_bias"]:
                used = host["bias_ids"][b] >= 0
                row = row + torch.bincount(host["bias_ids"][b][used].long(), weights=host["bias_values"][b][used].double(), minlength=V).cuda()
            row = row / c["tau"]
            if c["mask"] != "none":
                words = x["allowed"][b, m if c["mask"] == "slots" else 0].long()
                row = row.masked_fill(((words[column // 32] >> (column % 32)) & 1) == 0, -math.inf)
            out[b, m] = row
    return {"logits": out, "lse": torch.logsumexp(out, 2)}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_mx4(s) if case["op"] == "mx4" else _exact_edit(s)
