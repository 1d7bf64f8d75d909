"""Operators of a training iteration over packed sequences, each as cases of its own.

Three operators: attention over sequences that lie one behind the other without padding, with as many heads of keys and
values as the caller has (forward, and the gradient of queries, keys and values), and an update of a model's matrices
whose step is made orthogonal by Newton-Schulz products.  A pass is one call as a training loop makes it.  Heads,
widths, batches and lengths are those of `synthdata.WORKLOADS` (2 heads of 32, 12 or 16 of 64; sequences
of 16 to 1024 tokens, batches of 4 to 32), and generic ones beside them: heads of 128, four or eight query heads to one of
keys, sequences of up to 4096.

Fields of a case
  op        "attention", "attention_bwd" or "muon"
  dtype     storage type of the rows, or of the model: "bf16" or "fp32"
attention
  heads, kv_heads, head   query heads, heads of keys and values, head size
  batch, shortest, length   sequences, of evenly spread lengths from `shortest` to `length` in an order drawn from the seed
  behind    rows behind the last sequence, which belong to none
  causal    whether a row sees those before it and itself, or all of its sequence
update
  layers, hidden, kv, ffn   the model whose matrices are updated: projections of hidden x hidden (two) and kv x hidden
            (two), and a feed-forward block's two
  decay     weight decay
"""
import math

import torch

own = False

MUON = dict(lr=2e-5, momentum=0.95, rms=0.2, eps=1e-7)
POLYNOMIAL = (3.4445, -4.7750, 2.0315)
ITERATIONS = 5


def _attention(name, op, dtype, heads, kv_heads, head, batch, shortest, length, causal=True, behind=0):
    return {"name": name, "op": op, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "head": head, "batch": batch,
            "shortest": shortest, "length": length, "causal": causal, "behind": behind}


def _update(name, dtype, layers, hidden, kv, ffn, decay=0.01):
    return {"name": name, "op": "muon", "dtype": dtype, "layers": layers, "hidden": hidden, "kv": kv, "ffn": ffn, "decay": decay}


def listed():
    return [
        # scoring one short answer: latency
        _attention("attention_one_answer", "attention", "bf16", 16, 16, 64, 1, 17, 17),
        # the median batch of a causal model, four query heads to one of keys, packed
        _attention("attention_median", "attention", "bf16", 16, 4, 64, 16, 128, 661),
        # an encoder's batch, every row sees its whole sequence; a few rows are left at the buffer's end
        _attention("attention_encoder", "attention", "bf16", 12, 12, 64, 32, 153, 512, causal=False, behind=5),
        # long documents, heads of 128
        _attention("attention_long", "attention", "bf16", 16, 4, 128, 6, 1000, 4096),
        # the smallest configuration in full precision: launches
        _attention("attention_bwd_tiny_fp32", "attention_bwd", "fp32", 2, 1, 32, 4, 16, 64),
        _attention("attention_bwd_median", "attention_bwd", "bf16", 16, 4, 64, 16, 128, 661),
        # full precision, a batch of 12 packed samples
        _attention("attention_bwd_fp32", "attention_bwd", "fp32", 12, 12, 64, 12, 153, 397, causal=False, behind=3),
        _attention("attention_bwd_long", "attention_bwd", "bf16", 16, 4, 128, 6, 1000, 4096),
        # matrices of the smallest configuration: latency
        _update("muon_tiny_fp32", "fp32", 2, 64, 64, 256),
        # odd widths
        _update("muon_odd", "bf16", 5, 301, 77, 999, decay=0.0),
        # the two real models
        _update("muon_bert_base", "bf16", 12, 768, 768, 3072),
        _update("muon_gpt2_medium", "bf16", 24, 1024, 256, 4096),
    ]


def draw(rng):
    spread = lambda lo, hi: min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))  # noqa: E731
    op = rng.choice(["attention", "attention", "attention_bwd", "attention_bwd", "muon"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op == "muon":
        hidden = spread(48, 1024)
        c = _update("", dtype, spread(1, 12), hidden, max(8, hidden // rng.choice([1, 1, 4, 8])), rng.randint(hidden, 4 * hidden),
                    rng.choice([0.0, 0.01]))
    else:
        head = rng.choice([32, 64, 64, 128])
        kv_heads = rng.choice([1, 2, 4, 8])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 8] if kv_heads < 4 else [1, 2])
        causal = rng.random() < 0.7
        length = spread(1, 512 if dtype == "fp32" else 4096 if causal else 2048)
        batch = spread(1, max(1, min(32, 12000 // length)))
        c = _attention("", op, dtype, heads, kv_heads, head, batch, max(1, round(length * rng.uniform(0.05, 1.0))), length,
                       causal=causal, behind=rng.choice([0, 0, 1, 37]))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
class _State:
    pass


def _lengths(case):
    B, lo, hi = case["batch"], case["shortest"], case["length"]
    return [round(lo + (hi - lo) * b / (B - 1)) for b in range(B)] if B > 1 else [hi]


def _prepare_attention(case, seed):
    s, g = _State(), torch.Generator(device="cuda").manual_seed(seed)
    s.case = case
    h, hk, d = case["heads"], case["kv_heads"], case["head"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    lengths = torch.tensor(_lengths(case), device="cuda")[torch.randperm(case["batch"], generator=g, device="cuda")]
    ends = lengths.cumsum(0)
    s.rows = int(ends[-1])
    s.T = T = s.rows + case["behind"]
    s.starts, s.lengths, s.ends = ends - lengths, lengths, ends.to(torch.int32)
    # a projection's output: queries, keys and values of a token beside each other, and a bias that a head shares
    width = (h + 2 * hk) * d
    x = torch.randn(T, width, generator=g, device="cuda")
    x[:, :(h + hk) * d] += 0.3 * torch.randn(width, generator=g, device="cuda")[:(h + hk) * d]
    s.qkv = x.to(dt)
    s.q, s.k, s.v = s.qkv[:, :h * d], s.qkv[:, h * d:(h + hk) * d], s.qkv[:, (h + hk) * d:]
    s.scale = 1.0 / math.sqrt(d)
    s.out, s.lse = torch.zeros(T, h * d, dtype=dt, device="cuda"), torch.zeros(h, T, device="cuda")
    if case["op"] == "attention_bwd":
        _plain_attention(s)                                 # what the forward pass left
        s.dout = torch.randn(T, h * d, generator=g, device="cuda").to(dt)
        s.dqkv = torch.zeros_like(s.qkv)
        s.dq, s.dk, s.dv = s.dqkv[:, :h * d], s.dqkv[:, h * d:(h + hk) * d], s.dqkv[:, (h + hk) * d:]
        if own:                                             # scratch that a training loop keeps
            import paper_2209_02478_amd as mi
            nbytes = mi.mimose_op_packed_attention_bwd_workspace_bytes(T, h, hk, d)
            s.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return s


def _shapes(case):
    """(how many, rows, columns) of a model's matrices."""
    n, H, K, F = case["layers"], case["hidden"], case["kv"], case["ffn"]
    return [(2 * n, H, H), (2 * n, K, H), (n, F, H), (n, H, F)]


def _prepare_update(case, seed):
    """Matrices of one shape stand one behind the other, each on a whole number of 16 bytes."""
    s, g = _State(), torch.Generator(device="cuda").manual_seed(seed)
    s.case = case
    s.master, s.grad, s.momentum, s.lowp = [], [], [], []

    def stack(n, r, c, dt=torch.float32):
        return torch.zeros(n, -(-r * c // 8) * 8, dtype=dt, device="cuda")[:, :r * c].unflatten(1, (r, c))

    for n, r, c in _shapes(case):
        normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
        # a gradient: few directions that the batch agrees on, and noise; matrices differ by orders of magnitude
        size = torch.exp(normal(n, 1, 1) * 1.5 - 9.0)
        rank = max(1, min(r, c) // 16)

        def gradient():
            return (torch.matmul(normal(n, r, rank), normal(n, rank, c)) * (0.5 / math.sqrt(rank)) + normal(n, r, c)) * size

        w, gr, mo = stack(n, r, c), stack(n, r, c), stack(n, r, c)
        w.copy_(normal(n, r, c) * 0.02), gr.copy_(gradient()), mo.copy_(gradient() * 3.0)
        s.master.append(w), s.grad.append(gr), s.momentum.append(mo)
        if case["dtype"] == "bf16":
            s.lowp.append(stack(n, r, c, torch.bfloat16).copy_(w))
    s.hyper = {k: float(torch.tensor(x, dtype=torch.float32)) for k, x in (MUON | {"weight_decay": case["decay"]}).items()}
    if own:                                                 # the table of all matrices and its scratch, which a training loop keeps
        import paper_2209_02478_amd as mi
        s.table = mi.MuonTable([dict(master=s.master[k][i], lowp=s.lowp[k][i] if s.lowp else None, grad=s.grad[k][i], momentum=s.momentum[k][i])
                                for k in range(len(s.master)) for i in range(len(s.master[k]))])
    return s


def prepare(case, seed):
    return _prepare_update(case, seed) if case["op"] == "muon" else _prepare_attention(case, seed)


# ------------------------------------------------------------------ the plain forms
def _padded(s, x, heads):
    """[sequence, head, row, head size] in 32 bits, rows behind a sequence's end copied from its last."""
    at = s.starts[:, None] + torch.minimum(torch.arange(s.case["length"], device="cuda"), s.lengths[:, None] - 1)
    return x.float()[at].unflatten(2, (heads, s.case["head"])).transpose(1, 2)


def _grouped(s, x):
    """Query heads of one head of keys one behind the other: [sequence, kv head, group * row, head size]."""
    c = s.case
    return x.unflatten(1, (c["kv_heads"], c["heads"] // c["kv_heads"])).flatten(2, 3)


def _inside(s):
    return torch.arange(s.case["length"], device="cuda") < s.lengths[:, None]


def _scores(s, q, k):
    """Scaled scores, minus infinity where a row does not see another: [sequence, kv head, group, row, row]."""
    c, L = s.case, s.case["length"]
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s.scale).unflatten(2, (-1, L))
    seen = _inside(s)[:, None, :]
    if c["causal"]:
        seen = seen & torch.ones(L, L, dtype=torch.bool, device="cuda").tril()
    return x.masked_fill_(~seen[:, None, None], -math.inf)


def _unpad(s, x, out):
    """Rows of the sequences, into their places of `out`: x [sequence, head, row, head size]."""
    out[:s.rows] = x.transpose(1, 2)[_inside(s)].flatten(1).to(out.dtype)


def _plain_attention(s):
    c = s.case
    q, k, v = _grouped(s, _padded(s, s.q, c["heads"])), _padded(s, s.k, c["kv_heads"]), _padded(s, s.v, c["kv_heads"])
    x = _scores(s, q, k)
    top = x.amax(4, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(4, keepdim=True)
    lse = (total.log() + top).squeeze(4).flatten(1, 2)      # [sequence, head, row]
    o = torch.matmul(p.div_(total).flatten(2, 3), v)
    _unpad(s, o.unflatten(2, (-1, c["length"])).flatten(1, 2), s.out)
    s.lse[:, :s.rows] = lse.transpose(1, 2)[_inside(s)].t()


def _plain_attention_bwd(s):
    c, L = s.case, s.case["length"]
    q, k, v = _grouped(s, _padded(s, s.q, c["heads"])), _padded(s, s.k, c["kv_heads"]), _padded(s, s.v, c["kv_heads"])
    o, do = _padded(s, s.out, c["heads"]), _padded(s, s.dout, c["heads"])
    do = do * _inside(s)[:, None, :, None]                  # copies of the last row pass nothing back
    delta = _grouped(s, (o * do).sum(3, keepdim=True))
    at = s.starts[:, None] + torch.minimum(torch.arange(L, device="cuda"), s.lengths[:, None] - 1)
    lse = _grouped(s, s.lse.t()[at].transpose(1, 2)[..., None])
    do = _grouped(s, do)
    p = _scores(s, q, k).flatten(2, 3).sub_(lse).exp_()
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3)).sub_(delta).mul_(p)
    dq = torch.matmul(ds, k).mul_(s.scale)
    dk = torch.matmul(ds.transpose(2, 3), q).mul_(s.scale)
    _unpad(s, dq.unflatten(2, (-1, L)).flatten(1, 2), s.dq)
    _unpad(s, dk, s.dk)
    _unpad(s, dv, s.dv)


def _plain_muon(s):
    h, (a, b, c) = s.hyper, POLYNOMIAL
    for k, (w, g, m) in enumerate(zip(s.master, s.grad, s.momentum)):
        m.mul_(h["momentum"]).add_(g)
        x = g + m * h["momentum"]
        # the norm of gradients as small as 1e-20 needs the exponents of 64 bits
        x = x / (x.double().square().sum((1, 2), keepdim=True).sqrt() + h["eps"]).float()
        r, n = x.shape[1:]
        if r > n:
            x = x.transpose(1, 2).contiguous()
        for _ in range(ITERATIONS):
            A = torch.matmul(x, x.transpose(1, 2))
            B = A * b + torch.matmul(A, A) * c
            x = x * a + torch.matmul(B, x)
        if r > n:
            x = x.transpose(1, 2)
        w.sub_((x * (h["rms"] * math.sqrt(max(r, n))) + w * h["weight_decay"]) * h["lr"])
        if s.lowp:
            s.lowp[k].copy_(w)


def _muon_out(s):
    out = {"master": s.master, "momentum": s.momentum}
    if s.lowp:
        out["lowp"] = s.lowp
    return out


# ------------------------------------------------------------------ a pass
def _own_pass(s):
    import paper_2209_02478_amd as mi
    c = s.case
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "muon":
        mi.mimose_op_muon_step(s.table, **MUON, weight_decay=c["decay"], nesterov=1, iterations=ITERATIONS, stream=stream)
        return _muon_out(s)
    dt, ld, ldo = 1 if c["dtype"] == "bf16" else 0, s.qkv.stride(0), s.out.stride(0)
    heads = (s.ends, c["batch"], s.T, c["heads"], c["kv_heads"], c["head"], int(c["causal"]), s.scale)
    if c["op"] == "attention":
        mi.mimose_op_packed_attention_fwd(dt, s.q, ld, s.k, ld, s.v, ld, s.out, ldo, s.lse, *heads, stream=stream)
        return {"out": s.out, "lse": s.lse}
    mi.mimose_op_packed_attention_bwd(dt, s.q, ld, s.k, ld, s.v, ld, s.out, ldo, s.lse, s.dout, ldo, s.dq, ld, s.dk, ld, s.dv, ld, *heads,
                                      workspace=s.workspace, workspace_bytes=s.workspace.numel(), stream=stream)
    return {"dqkv": s.dqkv}


def run(s):
    if own:
        return _own_pass(s)
    if s.case["op"] == "muon":
        _plain_muon(s)
        return _muon_out(s)
    if s.case["op"] == "attention":
        _plain_attention(s)
        return {"out": s.out, "lse": s.lse}
    _plain_attention_bwd(s)
    return {"dqkv": s.dqkv}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_attention(case, s):
    """A sequence and a head of keys at a time."""
    h, hk, d, T = case["heads"], case["kv_heads"], case["head"], s.T
    per = h // hk
    q, k, v = (x.double().view(T, -1, d) for x in (s.q.contiguous(), s.k.contiguous(), s.v.contiguous()))
    out, lse = torch.zeros(T, h, d, dtype=torch.float64, device="cuda"), torch.zeros(h, T, dtype=torch.float64, device="cuda")
    back = case["op"] == "attention_bwd"
    if back:
        o, do = s.out.double().view(T, h, d), s.dout.double().view(T, h, d)
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for first, n in zip(s.starts.tolist(), s.lengths.tolist()):
        rows = slice(first, first + n)
        hidden = torch.full((n, n), -math.inf, dtype=torch.float64, device="cuda").triu(1) if case["causal"] else 0.0
        for head in range(h):
            kh, vh, qh = k[rows, head // per], v[rows, head // per], q[rows, head]
            x = qh @ kh.T / math.sqrt(d) + hidden
            if not back:
                lse[head, rows] = torch.logsumexp(x, 1)
                out[rows, head] = torch.softmax(x, 1) @ vh
                continue
            p = torch.exp(x - s.lse[head, rows].double()[:, None])
            g = do[rows, head]
            ds = p * (g @ vh.T - (g * o[rows, head]).sum(1, keepdim=True)) / math.sqrt(d)
            dq[rows, head] = ds @ kh
            dk[rows, head // per] += ds.T @ qh
            dv[rows, head // per] += p.T @ g
    if back:
        return {"dqkv": torch.cat([x.flatten(1) for x in (dq, dk, dv)], 1)}
    return {"out": out.flatten(1), "lse": lse}


def _exact_update(case, s):
    h, mu = s.hyper, s.hyper["momentum"]
    out = {"master": [], "momentum": []}
    for w, g, m in zip(s.master, s.grad, s.momentum):
        r, n = w.shape[1:]
        ms, ws = [], []
        for i in range(len(w)):
            buf = mu * m[i].double() + g[i].double()
            u = g[i].double() + mu * buf
            x = u / (torch.linalg.norm(u) + h["eps"])
            for _ in range(ITERATIONS):                     # an odd polynomial of the matrix, from the side that is cheaper
                gram = x.T @ x if r > n else x @ x.T
                poly = POLYNOMIAL[0] * torch.eye(len(gram), dtype=torch.float64, device="cuda") + POLYNOMIAL[1] * gram + POLYNOMIAL[2] * gram @ gram
                x = x @ poly if r > n else poly @ x
            ms.append(buf)
            ws.append((1 - h["lr"] * h["weight_decay"]) * w[i].double() - h["lr"] * h["rms"] * math.sqrt(max(r, n)) * x)
        out["momentum"].append(torch.stack(ms)), out["master"].append(torch.stack(ws))
    if s.lowp:
        out["lowp"] = out["master"]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_update(case, s) if case["op"] == "muon" else _exact_attention(case, s)


def work(case):
    """Attention: rows read and written once, the products of the pairs that see each other (two forward, five backward).
    Update: gradient read, momentum and weights read and written; of the products that are symmetric one half."""
    if case["op"] == "muon":
        size = 4 + 8 + 8 + (2 if case["dtype"] == "bf16" else 0)
        values = sum(n * r * c for n, r, c in _shapes(case))
        flops = sum(n * ITERATIONS * (3.0 * min(r, c) ** 2 * max(r, c) + 1.0 * min(r, c) ** 3) for n, r, c in _shapes(case))
        return {"bytes": float(values * size), "flops": flops}
    lengths = _lengths(case)
    h, hk, d, T = case["heads"], case["kv_heads"], case["head"], sum(lengths)
    pairs = sum(n * (n + 1) / 2 if case["causal"] else n * n for n in lengths)
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "attention":
        return {"bytes": float(T * (2 * h + 2 * hk) * d * size + 4 * T * h), "flops": 4.0 * d * h * pairs}
    return {"bytes": float(T * (4 * h + 4 * hk) * d * size + 4 * T * h), "flops": 10.0 * d * h * pairs}
