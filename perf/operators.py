"""The operators of a fine-tuning iteration behind the model's forward, each as cases of its own.

Four operators: log-probabilities of given tokens (scoring by a reference model or an older policy),
a preference loss on pairs of sequences and a clipped policy loss with a KL term, both with their
gradient on the logits, and an AdamW step over all tensors of a model with its state in 8 bits or in
32.  A pass is one call as a training loop makes it.  Vocabularies, batches and lengths are those of
`synthdata.WORKLOADS` (a vocabulary of 1000, 30522 or 50257 entries, rows padded to a multiple of 64;
sequences of up to 1024 tokens, batches of 12 to 16) and what lies between; the tensors that the
update runs over are those of the same models.

Fields of a case
  op        "logprob", "preference", "policy" or "adamw"
  dtype     storage type of the logits, or of the model: "bf16" or "fp32"
losses
  vocab, batch, length   logits of `batch` sequences of up to `length` tokens (preference: batch / 2 pairs)
  shortest  0: every sequence has `length` rows; else the rows are packed, and the sequences have evenly
            spread lengths from `shortest` to `length`, in an order drawn from the seed
  prompt    part of a sequence, at its start, that is not scored
  smoothing part of the preferences that are taken to be the wrong way round
  kl        weight of the KL term
update
  layers, hidden, ffn, vocab, positions   the model whose tensors are updated
  state_bits   8 or 32
  step      number of the update
"""
import math

import torch

own = False

BETA = 0.1                      # of the preference loss
CLIP_LOW, CLIP_HIGH = 0.2, 0.28
ADAMW = dict(lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
BLOCK = 256                     # elements that share a scale where a state is held in 8 bits


def _loss(name, op, dtype, vocab, batch, length, shortest=0, prompt=0.0, smoothing=0.0, kl=0.0):
    return {"name": name, "op": op, "dtype": dtype, "vocab": vocab, "batch": batch, "length": length, "shortest": shortest,
            "prompt": prompt, "smoothing": smoothing, "kl": kl}


def _update(name, dtype, layers, hidden, ffn, vocab, positions, state_bits, step):
    return {"name": name, "op": "adamw", "dtype": dtype, "layers": layers, "hidden": hidden, "ffn": ffn, "vocab": vocab,
            "positions": positions, "state_bits": state_bits, "step": step}


def listed():
    return [
        # scoring one short answer: a handful of rows, latency
        _loss("logprob_one_answer", "logprob", "bf16", 50257, 1, 17),
        # the reference model's pass over a whole batch, its prompts left out
        _loss("logprob_batch", "logprob", "bf16", 50257, 16, 1024, prompt=0.25),
        # the smallest configuration, two pairs, odd length: launches
        _loss("preference_tiny_fp32", "preference", "fp32", 1000, 4, 33, prompt=0.3, smoothing=0.1),
        # eight pairs around the median length, packed
        _loss("preference_median", "preference", "bf16", 50257, 16, 397, shortest=128, prompt=0.4),
        # the longest batch, every row scored but the last of a sequence
        _loss("preference_longest", "preference", "bf16", 50257, 16, 1024),
        # one sampled answer, few rows of a long vocabulary
        _loss("policy_one_answer", "policy", "bf16", 50257, 1, 17, kl=0.04),
        # full precision, batch of 12 packed answers
        _loss("policy_fp32", "policy", "fp32", 30522, 12, 397, shortest=153, prompt=0.2, kl=0.04),
        # the longest batch
        _loss("policy_longest", "policy", "bf16", 50257, 16, 1024, prompt=0.25, kl=0.04),
        # tensors of the smallest configuration: latency
        _update("adamw8_tiny_fp32", "fp32", 2, 64, 256, 1000, 64, 8, 3),
        # the two real models, state in 8 bits
        _update("adamw8_bert_base", "bf16", 12, 768, 3072, 30522, 512, 8, 150),
        _update("adamw8_gpt2_medium", "bf16", 24, 1024, 4096, 50257, 1024, 8, 1),
        # state in 32 bits
        _update("adamw32_bert_base", "bf16", 12, 768, 3072, 30522, 512, 32, 150),
    ]


def draw(rng):
    spread = lambda lo, hi: min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))  # noqa: E731
    op = rng.choice(["logprob", "preference", "preference", "policy", "policy", "adamw", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op == "adamw":
        hidden = 8 * spread(8, 128)
        c = _update("", dtype, spread(1, 24), hidden, 8 * rng.randint(hidden // 8, hidden // 2), spread(500, 50257), spread(64, 1024),
                    rng.choice([8, 8, 32]), spread(1, 10000))
    else:
        vocab = rng.choice([1000, 30522, 50257, spread(300, 50257)])
        batch = 2 * spread(1, 8)
        length = spread(4, 1024) if dtype == "bf16" else spread(4, 512)
        c = _loss("", op, dtype, vocab, batch, length, shortest=max(2, round(length * rng.uniform(0.1, 0.9))) if rng.random() < 0.5 else 0,
                  prompt=rng.choice([0.0, 0.1, 0.3, 0.6]), smoothing=rng.choice([0.0, 0.1]) if op == "preference" else 0.0,
                  kl=rng.choice([0.0, 0.04]) if op == "policy" else 0.0)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
class _State:
    pass


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _lengths(case):
    B, lo, hi = case["batch"], case["shortest"], case["length"]
    if not lo:
        return [hi] * B
    return [round(lo + (hi - lo) * b / (B - 1)) for b in range(B)] if B > 1 else [hi]


def _prompt(case, length):
    return min(length - 1, round(case["prompt"] * length))


def _prepare_loss(case, seed):
    s, g = _State(), _generator(seed)
    s.case, V = case, case["vocab"]
    s.ld = (V + 63) // 64 * 64
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    lengths = torch.tensor(_lengths(case), device="cuda")[torch.randperm(case["batch"], generator=g, device="cuda")]
    ends = lengths.cumsum(0)
    s.T = T = int(ends[-1])
    s.lengths, s.starts = lengths, ends - lengths
    s.ends = ends.to(torch.int32) if case["shortest"] else None
    row = torch.arange(T, device="cuda")
    s.seq = torch.searchsorted(ends, row, right=True)
    at = row - s.starts[s.seq]
    # a model's logits: spread by about 2.5, and the sampled tokens well above the mean
    s.logits = torch.randn(T, s.ld, generator=g, device="cuda", dtype=dt).mul_(2.5)
    labels = torch.randint(V, (T,), generator=g, device="cuda")
    lift = torch.rand(T, generator=g, device="cuda") * 12.0 + 2.0
    s.logits[row, labels] = lift.to(dt)
    prompt = torch.tensor([_prompt(case, n) for n in lengths.tolist()], device="cuda")
    # the rows of the prompt predict nothing that is scored, nor does a sequence's last row
    scored = (at >= prompt[s.seq]) & ((at < lengths[s.seq] - 1) | (lengths[s.seq] == 1))
    s.labels = torch.where(scored, labels, -1).to(torch.int32)
    s.n_valid = max(1, int(scored.sum()))
    s.logp = torch.empty(T, device="cuda")
    if own:                                                 # scratch that a training loop keeps
        import paper_2209_02478_amd as mi
        s.workspace = torch.empty(mi.mimose_op_token_loss_workspace_bytes(T), dtype=torch.uint8, device="cuda")
    if case["op"] == "logprob":
        return s
    s.dlogits = torch.empty_like(s.logits)
    if case["op"] == "preference":
        # the reference model's sums lie near the model's own: its answers differ by little in each token
        lp = _segment_sums(s, _logp(s)[0])
        s.ref = lp + torch.randn(case["batch"], generator=g, device="cuda") * lengths.float().sqrt()
        s.pairs = case["batch"] // 2
        s.seq_logp, s.margin, s.loss = torch.empty(2 * s.pairs, device="cuda"), torch.empty(s.pairs, device="cuda"), torch.empty(1, device="cuda")
    else:
        # the policy has moved by a few updates since it sampled; its ratios are kept off the two
        # bounds by 1e-3, so that no rounding decides which side of a bound a token is on
        lp = _logp(s)[0]
        move = torch.randn(T, generator=g, device="cuda") * 0.2
        for bound in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
            move = torch.where((move - bound).abs() < 1e-3, bound + 2e-3, move)
        s.old = lp - move
        s.ref = lp + torch.randn(T, generator=g, device="cuda") * 0.3
        s.advantage = torch.randn(case["batch"], generator=g, device="cuda")[s.seq]
        # mean over the tokens of each answer, then over the answers
        count = torch.zeros(case["batch"], device="cuda").index_put_((s.seq,), scored.float(), accumulate=True)
        s.weight = 1.0 / count.clamp(min=1.0)[s.seq]
        s.scale = 1.0 / case["batch"]
        s.rows, s.stats = torch.empty(T, 4, device="cuda"), torch.empty(3, device="cuda")
    return s


def _tensors(case):
    """Element count of each tensor, and whether it decays: a table of words and one of positions, each layer's
    projections, biases and norms."""
    H, F = case["hidden"], case["ffn"]
    out = [(case["vocab"] * H, 1), (case["positions"] * H, 1)]
    for _ in range(case["layers"]):
        out += [(3 * H * H, 1), (3 * H, 0), (H * H, 1), (H, 0), (H, 0), (H, 0), (F * H, 1), (F, 0), (H * F, 1), (H, 0), (H, 0), (H, 0)]
    return out + [(H, 0), (H, 0), (case["vocab"], 0)]


def _prepare_update(case, seed):
    """The tensors stand one behind the other in one buffer of each kind, each on a whole block of 256 elements."""
    s, g = _State(), _generator(seed)
    s.case = case
    counts = _tensors(case)
    pitch = [-(-n // BLOCK) * BLOCK for n, _ in counts]
    total = sum(pitch)
    blocks = torch.tensor([p // BLOCK for p in pitch], device="cuda")
    start = torch.tensor([sum(pitch[:k]) for k in range(len(pitch))], device="cuda")
    s.decay = torch.tensor([float(d) for _, d in counts], device="cuda").repeat_interleave(blocks)[:, None]
    s.start = start.repeat_interleave(blocks)[:, None]      # first element of a block's tensor
    real = torch.tensor([n for n, _ in counts], device="cuda").repeat_interleave(blocks)[:, None]
    index = torch.arange(total, device="cuda").view(-1, BLOCK)
    real = (index - s.start) < real
    draw_ = lambda: torch.randn(total // BLOCK, BLOCK, generator=g, device="cuda")  # noqa: E731
    # gradients of a block differ by orders of magnitude, and the words that a batch lacks have none
    scale = torch.exp(torch.randn(total // BLOCK, 1, generator=g, device="cuda") * 1.5 - 9.0)
    scale *= torch.rand(total // BLOCK, 1, generator=g, device="cuda") > 0.15
    s.grad = draw_() * scale * real
    s.master = draw_() * 0.02 * real
    s.lowp = s.master.to(torch.bfloat16) if case["dtype"] == "bf16" else None
    if s.lowp is not None and case["step"] == 1:
        s.master.copy_(s.lowp)                              # freshly loaded weights
    first = case["step"] == 1                               # before the first update there is no state
    m, v = draw_() * (scale * (0.0 if first else 0.3)) * real, (draw_() * (scale * (0.0 if first else 1.0))).square() * real
    s.m_scale = s.v_scale = None
    if case["state_bits"] == 8:
        s.m, s.m_scale = _to_8bit(m, _dither(s, index, 0xC13FA9A9, 0))
        s.v, s.v_scale = _to_8bit(v.sqrt(), _dither(s, index, 0x91E10DA5, 0))
    else:
        s.m, s.v = m, v
    s.hyper = {k: float(torch.tensor(x, dtype=torch.float32)) for k, x in ADAMW.items()}
    if own:                                                 # the table of all tensors, which a training loop keeps
        import paper_2209_02478_amd as mi
        part = lambda buf, k: None if buf is None else buf.view(-1)[sum(pitch[:k]):sum(pitch[:k]) + counts[k][0]]  # noqa: E731
        scales = lambda buf, k: None if buf is None else buf.view(-1)[sum(pitch[:k]) // BLOCK:sum(pitch[:k + 1]) // BLOCK]  # noqa: E731
        s.table = mi.AdamWTable([dict(master=part(s.master, k), lowp=part(s.lowp, k), grad=part(s.grad, k), m=part(s.m, k), v=part(s.v, k),
                                      m_scale=scales(s.m_scale, k), v_scale=scales(s.v_scale, k), decay=counts[k][1])
                                 for k in range(len(counts))], case["state_bits"])
    return s


def prepare(case, seed):
    return _prepare_update(case, seed) if case["op"] == "adamw" else _prepare_loss(case, seed)


# ------------------------------------------------------------------ the plain forms
def _logp(s):
    """log-probability of each row's label (0 where there is none), and the exponentials and their sums."""
    x = s.logits[:, :s.case["vocab"]].float()
    top = x.amax(1, keepdim=True)
    label = s.labels.long().clamp(min=0)[:, None]
    picked = x.gather(1, label) - top
    e = x.sub_(top).exp_() if x.data_ptr() != s.logits.data_ptr() else (x - top).exp_()
    total = e.sum(1, keepdim=True)
    return torch.where(s.labels >= 0, (picked - total.log())[:, 0], 0.0), e, total


def _segment_sums(s, per_row):
    """Sum over the rows of each sequence, in the order of the rows."""
    at = s.starts[:, None] + torch.arange(s.case["length"], device="cuda")
    inside = torch.arange(s.case["length"], device="cuda") < s.lengths[:, None]
    return (per_row[at.clamp(max=s.T - 1)] * inside).sum(1)


def _gradient(s, dlogp, e, total):
    """dlogits = dlogp * (onehot - softmax), zeros in the columns behind the vocabulary."""
    d = e.mul_(-dlogp[:, None] / total)
    row, label = torch.arange(s.T, device="cuda"), s.labels.long().clamp(min=0)
    d[row, label] += dlogp
    out = torch.zeros_like(s.logits)
    out[:, :s.case["vocab"]] = d
    return out


def _plain_preference(s):
    logp, e, total = _logp(s)
    lp = _segment_sums(s, logp)
    h = (lp - s.ref).view(-1, 2)
    z = BETA * (h[:, 0] - h[:, 1])
    eps, P = s.case["smoothing"], s.pairs
    softplus = lambda t: t.clamp(min=0.0) + (-t.abs()).exp().log1p()  # noqa: E731
    loss = ((1 - eps) * softplus(-z) + eps * softplus(z)).sum() / P
    g = BETA / P * ((1 - eps) / (1 + z.exp()) - eps / (1 + (-z).exp()))
    dlp = torch.stack((g, -g), 1).view(-1)
    dlogp = torch.where(s.labels >= 0, -dlp[s.seq], 0.0)
    return {"loss": loss.view(1), "logp": logp, "seq_logp": lp, "margin": z, "dlogits": _gradient(s, dlogp, e, total)}


def _plain_policy(s):
    logp, e, total = _logp(s)
    w = torch.where(s.labels >= 0, s.scale * s.weight, 0.0)
    ratio, A = (logp - s.old).exp(), s.advantage
    free, held = ratio * A, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A
    d = s.ref - logp
    kl = torch.expm1(d) - d
    kb = s.case["kl"]
    row_loss = w * (kb * kl - torch.minimum(free, held))
    clipped = (free > held).float()
    dlogp = w * (kb * (1 - d.exp()) - torch.where(free <= held, free, 0.0))
    rows = torch.stack((logp, row_loss, w * kl, w * clipped), 1)
    return {"stats": rows[:, 1:].sum(0), "rows": rows, "dlogits": _gradient(s, dlogp, e, total)}


def _dither(s, index, by_element, step):
    """A number below 2^20 for each element: a Weyl sequence over the updates."""
    return (((index - s.start) * by_element + step * 0x9E3779B9) & 0xFFFFFFFF) >> 12


def _to_8bit(x, dither):
    """e4m3 codes and a scale for each block: the scale puts the block's largest value at 448, the dither is
    added below the last of the bits that are kept; a value above zero that would become none is the smallest."""
    fine = x.isfinite()
    top = torch.where(fine, x.abs(), 0.0).amax(1, keepdim=True)
    scale = top.clamp(min=2.0 ** -100) * float(torch.tensor(1.0 / 448.0, dtype=torch.float32))
    y = (x.abs() * scale.reciprocal()).clamp(max=448.0)
    y = torch.where(fine, y, 0.0)
    normal = (y.view(torch.int32).long() + dither >> 20) - 960
    small = (y * 2.0 ** 29).long() + dither >> 20
    code = torch.where(y >= 2.0 ** -6, normal, small)
    code = torch.where(fine, code, 127) + 128 * (x < 0)
    return code.to(torch.uint8).view(torch.float8_e4m3fn), scale[:, 0]


def _plain_adamw(s):
    c, h = s.case, s.hyper
    one = torch.tensor(1.0)
    rest = [float(one - torch.tensor(h[k])) for k in ("beta1", "beta2")]
    inv_c1, inv_c2 = 1.0 / (1.0 - h["beta1"] ** c["step"]), 1.0 / (1.0 - h["beta2"] ** c["step"])
    eight = c["state_bits"] == 8
    m = s.m.float() * s.m_scale[:, None] if eight else s.m
    m = m * h["beta1"] + s.grad * rest[0]
    if eight:
        v = (s.v.float() * s.v_scale[:, None]).square()
    else:
        v = s.v
    v = v * h["beta2"] + s.grad * rest[1] * s.grad
    root = v.sqrt()
    step = m * inv_c1 / (root * math.sqrt(inv_c2) + h["eps"]) + s.master * (s.decay * h["weight_decay"])
    s.master.sub_(step * h["lr"])
    if eight:
        index = torch.arange(s.master.numel(), device="cuda").view(-1, BLOCK)
        code, scale = _to_8bit(m, _dither(s, index, 0xC13FA9A9, c["step"]))
        s.m.copy_(code), s.m_scale.copy_(scale)
        code, scale = _to_8bit(root, _dither(s, index, 0x91E10DA5, c["step"]))
        code = torch.where((root > 0) & (code.view(torch.uint8) == 0), 1, code.view(torch.uint8)).view(torch.float8_e4m3fn)
        s.v.copy_(code), s.v_scale.copy_(scale)
    else:
        s.m.copy_(m), s.v.copy_(v)
    if s.lowp is not None:
        s.lowp.copy_(s.master)


def _state_out(s):
    out = {"master": s.master, "m": s.m, "v": s.v}
    if s.lowp is not None:
        out["lowp"] = s.lowp
    if s.m_scale is not None:
        out |= {"m_scale": s.m_scale, "v_scale": s.v_scale}
    return out


# ------------------------------------------------------------------ a pass
def _own_pass(s):
    import paper_2209_02478_amd as mi
    c = s.case
    dt = 1 if c["dtype"] == "bf16" else 0
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "adamw":
        mi.mimose_op_adamw_step(s.table, c["step"], **ADAMW, stream=stream)
        return _state_out(s)
    scratch = dict(workspace=s.workspace, workspace_bytes=s.workspace.numel(), stream=stream)
    if c["op"] == "logprob":
        mi.mimose_op_token_logprob(dt, s.logits, s.ld, s.labels, s.logp, s.T, c["vocab"], **scratch)
        return {"logp": s.logp}
    if c["op"] == "preference":
        mi.mimose_op_preference_loss(dt, s.logits, s.ld, s.labels, s.ends, s.pairs, c["length"], s.ref, BETA, c["smoothing"], s.dlogits,
                                     s.logp, s.seq_logp, s.margin, s.loss, s.T, c["vocab"], **scratch)
        return {"loss": s.loss, "logp": s.logp, "seq_logp": s.seq_logp, "margin": s.margin, "dlogits": s.dlogits}
    mi.mimose_op_policy_loss(dt, s.logits, s.ld, s.labels, s.old, s.ref, s.advantage, s.weight, s.scale, CLIP_LOW, CLIP_HIGH, c["kl"],
                             s.dlogits, s.rows, s.stats, s.T, c["vocab"], **scratch)
    return {"stats": s.stats, "rows": s.rows, "dlogits": s.dlogits}


def run(s):
    if own:
        return _own_pass(s)
    op = s.case["op"]
    if op == "adamw":
        _plain_adamw(s)
        return _state_out(s)
    if op == "logprob":
        return {"logp": _logp(s)[0]}
    return _plain_preference(s) if op == "preference" else _plain_policy(s)


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_loss(case, s):
    """The losses written as such, their gradient by differentiation, a sequence at a time."""
    V, T = case["vocab"], s.T
    y = s.labels.long()
    scored = y >= 0
    out = torch.zeros(T, s.ld, dtype=torch.float64, device="cuda") if case["op"] != "logprob" else None
    logp = torch.zeros(T, dtype=torch.float64, device="cuda")
    firsts, counts = s.starts.tolist(), s.lengths.tolist()

    def rows(b):
        return slice(firsts[b], firsts[b] + counts[b])

    def of_sequence(b, grad):
        x = s.logits[rows(b), :V].double().requires_grad_(grad)
        own_rows = scored[rows(b)].nonzero()[:, 0]
        lp = torch.log_softmax(x[own_rows], 1)[torch.arange(len(own_rows), device="cuda"), y[rows(b)][own_rows]]
        return x, own_rows, lp

    for b in range(case["batch"]):
        _, own_rows, lp = of_sequence(b, False)
        logp[firsts[b] + own_rows] = lp
    if case["op"] == "logprob":
        return {"logp": logp}
    if case["op"] == "preference":
        lp = torch.stack([logp[rows(b)].sum() for b in range(case["batch"])]).requires_grad_()
        z = BETA * ((lp[0::2] - s.ref[0::2].double()) - (lp[1::2] - s.ref[1::2].double()))
        eps = case["smoothing"]
        loss = -((1 - eps) * torch.nn.functional.logsigmoid(z) + eps * torch.nn.functional.logsigmoid(-z)).mean()
        loss.backward()
        found = {"loss": loss.detach().view(1), "logp": logp, "seq_logp": lp.detach(), "margin": z.detach()}
        dlogp = lp.grad[s.seq]
    else:
        q = logp.clone().requires_grad_()
        w = s.scale * s.weight.double() * scored
        ratio, A, d = torch.exp(q - s.old.double()), s.advantage.double(), s.ref.double() - q
        gain = torch.min(ratio * A, torch.clamp(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH) * A)
        kl = torch.exp(d) - d - 1
        terms = torch.stack((q, w * (case["kl"] * kl - gain), w * kl, w * (ratio * A > gain)), 1)
        terms[:, 1].sum().backward()
        found = {"stats": terms[:, 1:].detach().sum(0), "rows": terms.detach()}
        dlogp = q.grad
    for b in range(case["batch"]):
        x, own_rows, lp = of_sequence(b, True)
        if len(own_rows):
            lp.backward(dlogp[rows(b)][own_rows])
            out[rows(b), :V] = x.grad
    return found | {"dlogits": out}


def _exact_update(case, s):
    h = {k: v for k, v in s.hyper.items()}
    t, eight = case["step"], case["state_bits"] == 8
    index = torch.arange(s.master.numel(), device="cuda").view(-1, BLOCK) - s.start
    g, p = s.grad.double(), s.master.double()
    m, v = s.m.double(), s.v.double()
    if eight:
        m, v = m * s.m_scale.double()[:, None], (v * s.v_scale.double()[:, None]) ** 2
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    mean, var = m / (1 - h["beta1"] ** t), v / (1 - h["beta2"] ** t)
    p = p - h["lr"] * (mean / (var.sqrt() + h["eps"]) + h["weight_decay"] * s.decay * p)
    out = {"master": p, "m": m, "v": v}
    if s.lowp is not None:
        out["lowp"] = p

    def held(x, by_element):
        """Values of three bits behind the first one, from 448 down to 2^-6, and evenly spaced below."""
        scale = x.abs().amax(1).clamp(min=2.0 ** -100) / 448
        a = x.abs() / scale[:, None]
        space = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
        part = ((index * by_element + t * 0x9E3779B9) % 2 ** 32 // 2 ** 12).double() / 2 ** 20
        return torch.floor(a / space + part) * space * x.sign(), scale

    if eight:
        out["m"], out["m_scale"] = held(m, 0xC13FA9A9)
        root = v.sqrt()
        code, out["v_scale"] = held(root, 0x91E10DA5)
        out["v"] = torch.where((root > 0) & (code == 0), 2.0 ** -9, code)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_update(case, s) if case["op"] == "adamw" else _exact_loss(case, s)


def work(case):
    """Losses: every scored row of logits read, every row of the gradient written.  Update: gradient read; weights and
    states read and written."""
    if case["op"] == "adamw":
        n = sum(c for c, _ in _tensors(case))
        state = 4 + 16.0 / BLOCK if case["state_bits"] == 8 else 16
        return {"bytes": n * (4 + 8 + (2 if case["dtype"] == "bf16" else 0) + state), "flops": 15.0 * n}
    lengths = _lengths(case)
    scored = sum(max(1, n - 1 - _prompt(case, n)) if n == 1 else n - 1 - _prompt(case, n) for n in lengths)
    size = 2 if case["dtype"] == "bf16" else 4
    rows = scored + (0 if case["op"] == "logprob" else sum(lengths))
    return {"bytes": float(rows * case["vocab"] * size), "flops": 4.0 * scored * case["vocab"]}
