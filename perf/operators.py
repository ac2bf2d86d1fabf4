"""Work whose time is measured for the operators behind the training step: attention under a rule (score cap, distance bias, document
and prefix masks) with its gradients, and the GELU whose input is kept in 8 bits for the backward pass.

`run(state)` computes a case in its plain form, elementary torch operations in 32 bits, or, where `own` is true, by the
framework's calls.  `exact(case, seed)` gives the same results in 64 bits.

Fields of a case:
  op        "attn" or "gelu8"
  direction attn: "fwd" (the output) or "train" (output and the gradients of q, k, v);
            gelu8: "train" (activation, then from its checkpoint the input's gradient and the activation again) or "bwd" (the latter
            two alone, from a checkpoint in hand)
  dtype     "bf16" or "f32"
  attn:   nb, Sq, Sk, H, Hkv, dh; q0: the position of query 0 among the keys; order: "full", "causal" or "prefix" (a key behind the
          query is seen when it is among the sample's first tokens); cap: 0, or c of c tanh(s / c); slopes: a bias of
          -slope_h |i - j|; docs: "none", "padded" (one document and padding) or "packed" (several documents, then padding);
          layout: "packed" ([tokens, heads of q | k | v] in one tensor) or "heads" ([sample, head, token, :])
  gelu8:  T rows of F values
"""
import math
import random

import torch

own = False

BLOCK = 32      # values that share one exponent in an 8-bit checkpoint
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attn(name, nb, S, H, dh, direction="train", dtype="bf16", **over):
    c = dict(op="attn", direction=direction, dtype=dtype, nb=nb, Sq=S, Sk=S, H=H, Hkv=H, dh=dh, q0=0, order="full", cap=0.0, slopes=False,
             docs="none", layout="packed")
    if name:
        c["name"] = name
    c.update(over)
    return c


def _gelu8(name, T, F, direction="train", dtype="bf16"):
    c = dict(op="gelu8", direction=direction, dtype=dtype, T=T, F=F)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One short fp32 sequence of the smallest model, scores capped: launch latency.
        _attn("attn_fwd_tiny_f32", 1, 17, 4, 16, "fwd", "f32", cap=20.0),
        # A handful of padded sentences in a small model: few tokens, every tile ragged.
        _attn("attn_train_small_padded", 3, 77, 4, 64, docs="padded"),
        # The fine-tuning batch of BERT-base, question and passage padded to one length.
        _attn("attn_train_base_padded", 32, 384, 12, 64, docs="padded"),
        # Short texts packed into full rows of BERT-large: a token sees its own document, nearer tokens more.
        _attn("attn_train_large_packed_bias", 32, 512, 16, 64, docs="packed", slopes=True),
        # Long packed rows with capped scores, every sample with a prefix that all its tokens see.
        _attn("attn_train_long_prefix_cap", 4, 2048, 16, 64, order="prefix", cap=30.0, docs="packed"),
        # Evaluation on one long causal row whose key heads are shared by four query heads each, head-major tensors.
        _attn("attn_fwd_8k_shared_heads", 1, 8192, 16, 128, "fwd", Hkv=4, order="causal", layout="heads"),
        # fp32 mode, ragged, packed documents with a distance bias.
        _attn("attn_train_f32_packed", 4, 203, 6, 64, "train", "f32", docs="packed", slopes=True),
        # The class token's attention alone over long sequences: one query for each sample and head.
        _attn("attn_fwd_first_token", 64, 1024, 12, 64, "fwd", Sq=1, docs="padded"),
        # The MLP activation of a few sentences.
        _gelu8("gelu8_train_small", 231, 1024),
        # The MLP activation of BERT-large on 32768 tokens, both directions.
        _gelu8("gelu8_train_large", 32768, 4096),
        # The backward half alone, of a width whose last block is short.
        _gelu8("gelu8_bwd_ragged", 12608, 1540, "bwd"),
        # fp32 mode.
        _gelu8("gelu8_bwd_f32", 1576, 1536, "bwd", "f32"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if rng.random() < 0.25:
        F = 4 * _logint(rng, 1, 2048)
        most = min(131072, (1 << 27) // F)
        return _gelu8("", _logint(rng, 1, most), F, rng.choice(["train", "bwd"]), dtype)
    dh = rng.choice([64, 64, 64, 128, 8 * rng.randint(1, 16)])
    Hkv = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
    H = Hkv * (rng.choice([2, 3, 4, 8]) if rng.random() < 0.3 and Hkv <= 6 else 1)
    S = _logint(rng, 1, 4096)
    over = dict(Hkv=Hkv, order=rng.choice(["full", "full", "causal", "prefix"]), docs=rng.choice(["none", "padded", "packed", "packed"]),
                layout=rng.choice(["packed", "packed", "heads"]), slopes=rng.random() < 0.3)
    if rng.random() < 0.3:
        over["cap"] = float(rng.choice([5, 15, 20, 30, 50]))
    kind = rng.random()
    if kind < 0.1:          # the first token alone
        over.update(Sq=1, order="full")
    elif kind < 0.2:        # the last tokens of a longer row
        over.update(Sq=_logint(rng, 1, S))
        over["q0"] = S - over["Sq"]
    # as many samples as keep the scores below the largest listed case
    most = max(1, min(64, int((1 << 28) * (64 / dh) * (0.25 if dtype == "f32" else 1) / (H * S * over.get("Sq", S)))))
    return _attn("", _logint(rng, 1, most), S, H, dh, rng.choice(["fwd", "train", "train"]), dtype, **over)


def _documents(case, seed):
    """For each sample the document of every key (-1: padding), as nested lists of lengths turned into ids; None without documents."""
    if case["docs"] == "none":
        return None
    rng = random.Random(int(seed) * 7919 + case["Sk"])
    S, rows = case["Sk"], []
    for _ in range(case["nb"]):
        used = max(1, int(S * rng.uniform(0.5 if case["docs"] == "padded" else 0.85, 1.0)))
        row, doc = [], 0
        while len(row) < used:
            n = used if case["docs"] == "padded" else max(1, min(used - len(row), int(S * rng.uniform(0.05, 0.45))))
            row += [doc] * n
            doc += 1
        rows.append(row + [-1] * (S - used))
    return rows


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(gen, *shape, std=1.0):
    return torch.empty(*shape, device="cuda").normal_(0.0, std, generator=gen)


def prepare(case, seed):
    c, gen, t = case, _generator(seed), DTYPES[case["dtype"]]
    if c["op"] == "gelu8":
        # pre-activations as an MLP has them: each column with a spread of its own, a few far out
        h = (_randn(gen, c["T"], c["F"]) * (0.3 + _randn(gen, 1, c["F"]).abs())).to(t)
        st = dict(case=c, h=h, dg=_randn(gen, c["T"], c["F"], std=1e-3).to(t))
        if c["direction"] == "bwd":     # the checkpoint that the forward pass left
            st["codes"], st["exps"] = _plain_pack(h)
            del st["h"]
        return st
    nb, Sq, Sk, H, Hkv, dh = (c[k] for k in ("nb", "Sq", "Sk", "H", "Hkv", "dh"))
    st = dict(case=c)
    if c["layout"] == "packed" and Sq == Sk:
        st["qkv"] = _randn(gen, nb, Sq, (H + 2 * Hkv) * dh, std=1.2).to(t)
        st["do"] = _randn(gen, nb, Sq, H, dh, std=0.02).to(t)
    elif c["layout"] == "packed":       # fewer queries than keys: q apart, k and v in one tensor
        st["q"] = _randn(gen, nb, Sq, H * dh, std=1.2).to(t)
        st["kv"] = _randn(gen, nb, Sk, 2 * Hkv * dh, std=1.2).to(t)
        st["do"] = _randn(gen, nb, Sq, H, dh, std=0.02).to(t)
    else:
        st["q"] = _randn(gen, nb, H, Sq, dh, std=1.2).to(t)
        st["k"], st["v"] = (_randn(gen, nb, Hkv, Sk, dh, std=1.2).to(t) for _ in range(2))
        st["do"] = _randn(gen, nb, H, Sq, dh, std=0.02).to(t).transpose(1, 2)
    docs = _documents(c, seed)
    st["docs"] = None if docs is None else torch.tensor(docs, dtype=torch.int32).cuda()
    st["q_docs"] = None if docs is None else st["docs"][:, c["q0"]:c["q0"] + Sq].contiguous()
    st["slopes"] = 2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda", dtype=torch.float32) / H) if c["slopes"] else None
    st["prefix"] = (torch.rand(nb, device="cuda", generator=gen) * 0.5 * Sk).to(torch.int32) if c["order"] == "prefix" else None
    return st


def _views(st):
    """q, k, v as [nb, tokens, heads, dh]."""
    c = st["case"]
    nb, Sq, Sk, H, Hkv, dh = (c[k] for k in ("nb", "Sq", "Sk", "H", "Hkv", "dh"))
    if "qkv" in st:
        heads = st["qkv"].view(nb, Sq, H + 2 * Hkv, dh)
        return heads[:, :, :H], heads[:, :, H:H + Hkv], heads[:, :, H + Hkv:]
    if "kv" in st:
        heads = st["kv"].view(nb, Sk, 2 * Hkv, dh)
        return st["q"].view(nb, Sq, H, dh), heads[:, :, :Hkv], heads[:, :, Hkv:]
    return st["q"].transpose(1, 2), st["k"].transpose(1, 2), st["v"].transpose(1, 2)


def _own_attn(st):
    from paper_2102_03161_amd import binding
    c = st["case"]
    q, k, v = _views(st)
    rule = binding.AttentionRule(order=c["order"], cap=c["cap"], slopes=st["slopes"], documents=st["docs"], q_documents=st["q_docs"],
                                 prefix=st["prefix"], q0=c["q0"])
    if c["direction"] == "fwd":
        return binding.attention_forward(q, k, v, rule, want_lse=False)[0]
    o, lse = binding.attention_forward(q, k, v, rule)
    return (o, *binding.attention_backward(q, k, v, o, lse, st["do"], rule))


def _own_gelu8(st):
    from paper_2102_03161_amd import binding
    if st["case"]["direction"] == "bwd":
        return binding.gelu8_backward(st["codes"], st["exps"], st["dg"])
    g, codes, exps = binding.gelu8_forward(st["h"])
    return (g, *binding.gelu8_backward(codes, exps, st["dg"]))


def _plain_pack(h):
    """Codes (int8) and biased exponents (uint8): blocks of 32 along the row, a block's step the least power of two that holds its
    largest value in 127 steps."""
    T, F = h.shape
    n = -(-F // BLOCK)
    x = torch.nn.functional.pad(h.float(), (0, n * BLOCK - F)).view(T, n, BLOCK)
    top = x.abs().amax(-1)
    e = torch.ceil(torch.log2(top.double() / 127.0)).clamp(min=-126.0)
    step = torch.pow(2.0, e).float().unsqueeze(-1)
    codes = torch.round(x / step).to(torch.int8).view(T, n * BLOCK)[:, :F].contiguous()
    return codes, (e + 127.0).to(torch.uint8)


def _plain_unpack(codes, exps):
    step = torch.pow(2.0, exps.double() - 127.0).float()
    return codes.float() * step.repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]


def _plain_gelu8(st):
    c, dg = st["case"], st["dg"]
    out = []
    if c["direction"] == "train":
        h = st["h"].float()
        out.append((0.5 * h * torch.erfc(h * -math.sqrt(0.5))).to(dg.dtype))
        codes, exps = _plain_pack(st["h"])
    else:
        codes, exps = st["codes"], st["exps"]
    x = _plain_unpack(codes, exps)
    cdf = 0.5 * torch.erfc(x * -math.sqrt(0.5))
    slope = cdf + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))
    return (*out, (dg.float() * slope).to(dg.dtype), (x * cdf).to(dg.dtype))


def _allowed(st):
    """Which key each query sees, [nb, 1, 1, Sq, Sk], or None."""
    c = st["case"]
    i = torch.arange(c["Sq"], device="cuda").view(-1, 1) + c["q0"]
    j = torch.arange(c["Sk"], device="cuda").view(1, -1)
    see = None
    if c["order"] == "causal":
        see = (j <= i).view(1, 1, 1, c["Sq"], c["Sk"])
    elif c["order"] == "prefix":
        see = ((j <= i) | (j < st["prefix"].view(-1, 1, 1))).view(c["nb"], 1, 1, c["Sq"], c["Sk"])
    if st["docs"] is not None:
        a, b = st["q_docs"].view(c["nb"], 1, 1, -1, 1), st["docs"].view(c["nb"], 1, 1, 1, -1)
        same = (a == b) & (a >= 0)
        see = same if see is None else see & same
    return see


def _plain_attn(st):
    c = st["case"]
    nb, Sq, Sk, H, Hkv, dh = (c[k] for k in ("nb", "Sq", "Sk", "H", "Hkv", "dh"))
    G, t = H // Hkv, st["do"].dtype
    scale = 1.0 / math.sqrt(dh)

    def heads(x, n):        # [nb, tokens, Hkv * n, dh] -> [nb, Hkv, n * tokens, dh]
        return x.float().view(nb, x.shape[1], Hkv, n, dh).permute(0, 2, 3, 1, 4).reshape(nb, Hkv, n * x.shape[1], dh)

    def back(x, n):
        tokens = x.shape[2] // n
        return x.view(nb, Hkv, n, tokens, dh).permute(0, 3, 1, 2, 4).reshape(nb, tokens, Hkv * n, dh).to(t)

    q, k, v = _views(st)
    q, k, v = heads(q, G), heads(k, 1), heads(v, 1)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).view(nb, Hkv, G, Sq, Sk) * scale
    bent = None
    if c["cap"]:
        bent = torch.tanh(s / c["cap"])
        s = c["cap"] * bent
    if c["slopes"]:
        i = torch.arange(Sq, device="cuda").view(-1, 1) + c["q0"]
        far = (i - torch.arange(Sk, device="cuda").view(1, -1)).abs().float()
        s = s - st["slopes"].view(1, Hkv, G, 1, 1) * far
    see = _allowed(st)
    if see is not None:
        s = s.masked_fill(~see, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = back(torch.matmul(p.view(nb, Hkv, G * Sq, Sk), v), G)
    if c["direction"] == "fwd":
        return o
    do = heads(st["do"], G)
    dv = torch.matmul(p.view(nb, Hkv, G * Sq, Sk).transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous()).view(nb, Hkv, G, Sq, Sk)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    if c["cap"]:
        ds = ds * (1.0 - bent * bent)
    ds = (ds * scale).view(nb, Hkv, G * Sq, Sk)
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    return o, back(dq, G), back(dk, 1), back(dv, 1)


def run(state):
    if own:
        return _own_attn(state) if state["case"]["op"] == "attn" else _own_gelu8(state)
    return _plain_attn(state) if state["case"]["op"] == "attn" else _plain_gelu8(state)


def work(case):
    c, e = case, 4 if case["dtype"] == "f32" else 2
    if c["op"] == "gelu8":
        n = c["T"] * c["F"]
        per = 3 * e + (1 + 1 / BLOCK if c["direction"] == "bwd" else 2 * e)     # dg, dh, g; and the checkpoint, or h and its g
        return {"bytes": n * per, "flops": (40 if c["direction"] == "bwd" else 70) * n}
    nb, Sq, Sk, H, Hkv, dh = (c[k] for k in ("nb", "Sq", "Sk", "H", "Hkv", "dh"))
    # the pairs of a query and a key that it sees (document lengths as one seed has them, prefixes of a quarter)
    rows = _documents(c, 1) or [[0] * Sk] * nb
    pairs = 0
    for row in rows:
        first, count = {}, {}
        for j, d in enumerate(row):
            first.setdefault(d, j)
            count[d] = count.get(d, 0) + 1
        for i in range(c["q0"], c["q0"] + Sq):
            d = row[i]
            if d >= 0:
                last = Sk if c["order"] == "full" else max(i + 1, Sk // 4 if c["order"] == "prefix" else 0)
                pairs += min(count[d], max(0, last - first[d]))
    qo, kv = nb * Sq * H * dh * e, nb * Sk * Hkv * dh * e
    if c["direction"] == "fwd":
        return {"bytes": 2 * qo + 2 * kv, "flops": 4 * dh * H * pairs}
    return {"bytes": 4 * qo + 4 * kv, "flops": 14 * dh * H * pairs}


def exact(case, seed):
    """The definition in 64 bits, head by head; gradients by automatic differentiation."""
    c, st = case, prepare(case, seed)
    if c["op"] == "gelu8":
        def gelu(x):
            return x * torch.special.ndtr(x)

        out = []
        if c["direction"] == "train":
            h = st["h"].double()
            out.append(gelu(h))
            n = -(-c["F"] // BLOCK)
            x = torch.cat([h, h.new_zeros(c["T"], n * BLOCK - c["F"])], 1).view(-1, BLOCK)
            m, power = torch.frexp(x.abs().max(1).values)       # largest = m 2^power, m in [1/2, 1)
            power = torch.where(m <= 127.0 / 128.0, power - 7, power - 6).clamp(min=-126)
            x = torch.ldexp(torch.ldexp(x, -power.view(-1, 1)).round(), power.view(-1, 1)).view(c["T"], -1)[:, :c["F"]]
        else:
            block = torch.arange(c["F"], device="cuda") // BLOCK
            x = torch.ldexp(st["codes"].double(), st["exps"].to(torch.int32)[:, block] - 127)
        x = x.contiguous().requires_grad_()
        g = gelu(x)
        g.backward(st["dg"].double())
        return (*out, x.grad, g.detach())
    nb, Sq, Sk, H, Hkv, dh = (c[k] for k in ("nb", "Sq", "Sk", "H", "Hkv", "dh"))
    train = c["direction"] == "train"
    q, k, v = (x.double().detach().requires_grad_(train) for x in _views(st))
    o = torch.zeros(nb, Sq, H, dh, dtype=torch.float64, device="cuda")
    at, key = torch.arange(c["q0"], c["q0"] + Sq, device="cuda"), torch.arange(Sk, device="cuda")
    for b in range(nb):
        hidden = torch.zeros(Sq, Sk, dtype=torch.bool, device="cuda")
        if c["order"] != "full":
            hidden |= key[None, :] > at[:, None]
        if c["order"] == "prefix":
            hidden &= (key >= st["prefix"][b])[None, :]
        if st["docs"] is not None:
            hidden |= (st["q_docs"][b][:, None] != st["docs"][b][None, :]) | (st["docs"][b] < 0)[None, :]
        seeing = ~hidden.all(1)
        for h in range(H):
            s = (q[b, :, h] @ k[b, :, h * Hkv // H].T) / math.sqrt(dh)
            if c["cap"]:
                s = torch.tanh(s / c["cap"]) * c["cap"]
            if c["slopes"]:
                s = s - float(st["slopes"][h]) * (at[:, None] - key[None, :]).abs()
            s = s[seeing].masked_fill(hidden[seeing], -math.inf)
            part = (s - torch.logsumexp(s, 1, keepdim=True)).exp() @ v[b, :, h * Hkv // H]
            o[b, seeing, h] = part.detach()
            if train:
                (part * st["do"][b, seeing, h].double()).sum().backward()
    return (o, q.grad, k.grad, v.grad) if train else o
