"""Performance cases of the learning operators: token log-probabilities, the clipped policy loss with its
gradient, and AdamW over many tensors.

Each is given twice: as the framework's calls (own) and in elementary torch operations.  Sizes are those of
the engine's vocabularies (4096, 32000), drafter factors and layers, and generic ones around them.
"""
import math
from types import SimpleNamespace

import torch

own = False

CLIP = (0.2, 0.28)              # clip_low, clip_high
C_KL, C_ENT = 0.1, 0.01
REF_T = 1.25                    # temperature of the reference distribution
LR, BETAS, EPS, DECAY, MAX_NORM, SEED = 1e-3, (0.9, 0.999), 1e-8, 0.01, 1.0, 20250
BLOCK = 256                     # elements of a tensor that share the scales of its 8-bit states
FP8 = torch.float8_e4m3fn


def listed():
    return [
        # The four drafts of one step, scored while serving: latency.
        dict(name="logp_4x32000_f32", op="logp", rows=4, vocab=32000, dtype="f32", pad=0, masked=0.0, banned=0.0, temp=0.7),
        # Scoring a batch of rollouts once, for the ratios of the steps that follow.
        dict(name="logp_8192x32000_bf16", op="logp", rows=8192, vocab=32000, dtype="bf16", pad=0, masked=0.1, banned=0.0,
             temp=1.0),
        # Odd vocabulary in rows of a padded buffer, part of it forbidden by a grammar.
        dict(name="logp_1500x65521_bf16", op="logp", rows=1500, vocab=65521, dtype="bf16", pad=15, masked=0.0, banned=0.3,
             temp=1.0),
        # The smallest model's replay rows after a few steps: latency.
        dict(name="policy_16x4096_f32", op="policy", rows=16, vocab=4096, dtype="f32", pad=0, masked=0.0, banned=0.0,
             temp=1.0, ref="tokens"),
        # A partly filled and a full replay ring: KL to the verifier's logits.
        dict(name="policy_48x32000_f32", op="policy", rows=48, vocab=32000, dtype="f32", pad=0, masked=0.0, banned=0.0,
             temp=1.0, ref="logits"),
        dict(name="policy_256x32000_f32", op="policy", rows=256, vocab=32000, dtype="f32", pad=0, masked=0.0, banned=0.0,
             temp=1.0, ref="logits"),
        # Rollouts of different lengths in one padded batch.
        dict(name="policy_4096x32000_bf16", op="policy", rows=4096, vocab=32000, dtype="bf16", pad=0, masked=0.25, banned=0.0,
             temp=1.0, ref="tokens"),
        # A large vocabulary against a reference's whole distribution.
        dict(name="policy_2048x131072_bf16", op="policy", rows=2048, vocab=131072, dtype="bf16", pad=0, masked=0.0,
             banned=0.0, temp=1.0, ref="logits"),
        # The drafter's two factors at 7B widths, gradient clipping on: latency.
        dict(name="adamw_lora_f32", op="adamw", kind="lora", n=1, d=4096, ffn=0, vocab=32000, dtype="f32", bits=32, clip=True),
        # The same at 13B widths with states in 8 bits.
        dict(name="adamw_lora_8bit", op="adamw", kind="lora", n=1, d=5120, ffn=0, vocab=32000, dtype="f32", bits=8, clip=True),
        # Two layers at 1B widths in bf16 with 32-bit masters, every projection a tensor of its own.
        dict(name="adamw_1b_bf16", op="adamw", kind="layers", n=2, d=2048, ffn=8192, vocab=0, dtype="bf16", bits=32, clip=True),
        # A layer at 7B widths, states in 8 bits.
        dict(name="adamw_7b_8bit", op="adamw", kind="layers", n=1, d=4096, ffn=11008, vocab=0, dtype="bf16", bits=8, clip=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logp", "policy", "policy", "adamw", "adamw"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "adamw":
        kind = rng.choice(["lora", "layers", "odd"])
        c = dict(op=op, kind=kind, n=1, d=_log_int(rng, 128, 5120), ffn=0, vocab=0, dtype=dtype, bits=rng.choice([8, 32]),
                 clip=rng.random() < 0.5)
        if kind == "lora":
            c["vocab"] = _log_int(rng, 1000, 131072)
        elif kind == "layers":
            c["d"] = _log_int(rng, 64, 2048)
            c["ffn"], c["n"] = int(c["d"] * rng.uniform(2, 4)), rng.randint(1, 3)
        else:
            c["n"] = _log_int(rng, 1, 60)
        return c
    vocab = _log_int(rng, 128, 131072)
    most = int(2e8 // vocab) if op == "policy" else int(2.4e8 // vocab)
    c = dict(op=op, rows=_log_int(rng, 1, min(8192, most)), vocab=vocab, dtype=dtype, pad=rng.choice([0, 0, 1, 8, 37]),
             masked=rng.choice([0.0, 0.0, 0.3]), banned=rng.choice([0.0, 0.0, 0.5]), temp=rng.choice([0.6, 1.0, 1.0, 1.4]))
    if dtype == "f32" and c["rows"] * vocab > 1e8:
        c["rows"] = max(1, int(1e8 // vocab))
    if op == "policy":
        c["ref"] = rng.choice(["none", "tokens", "logits"])
    return c


# ------------------------------------------------------------------ inputs
def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _gen(seed, stream):
    return torch.Generator(_device()).manual_seed((int(seed) * 1000003 + stream * 7919 + 77) % (1 << 62))


def _normal(seed, stream, std, shape):
    return torch.empty(shape, dtype=torch.float32, device=_device()).normal_(0.0, std, generator=_gen(seed, stream))


def _uniform(seed, stream, shape):
    return torch.empty(shape, dtype=torch.float32, device=_device()).uniform_(generator=_gen(seed, stream))


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(case, seed):
    """Logits [rows, vocab] (rows of a wider buffer where pad > 0) of a model that has one likely token a
    row, the tokens it sampled, and which rows count."""
    n, V = case["rows"], case["vocab"]
    z = _normal(seed, 1, 2.0, (n, V + case["pad"]))
    likely = (_uniform(seed, 2, (n, 1)) * V).long().clamp_(max=V - 1)
    z.scatter_add_(1, likely, 5.0 + 2.0 * _normal(seed, 3, 1.0, (n, 1)))
    if case["banned"]:
        out = _uniform(seed, 4, (V,)) < case["banned"]
        out[0] = False
        z[:, :V].masked_fill_(out, -math.inf)
    buffer = z.to(_dtype(case))
    noise = _uniform(seed, 5, (n, V)).clamp_(1e-7, 1 - 1e-7).log_().neg_().log_().neg_()
    tokens = noise.add_(z[:, :V], alpha=1.0 / case["temp"]).argmax(-1).to(torch.int32)
    live = _uniform(seed, 6, (n,)) >= case["masked"]
    live[0] = True
    return buffer[:, :V], torch.where(live, tokens, -1).to(torch.int32), live


def _sizes(case):
    d, f, rank = case["d"], case["ffn"], 16
    if case["kind"] == "lora":
        return [case["vocab"] * rank, rank * d]
    if case["kind"] == "layers":
        return [d, d * d, d * d, d * d, d * d, d, d * f, d * f, f * d] * case["n"]
    return [1 + (d * d * (i + 1) * 7919) % (d * 97 + 13) for i in range(case["n"])]


def _segments(case):
    """Where each tensor starts in a flat buffer of whole blocks, and the buffer's length."""
    at, starts = 0, []
    for s in _sizes(case):
        starts.append(at)
        at += -(-s // BLOCK) * BLOCK
    return starts, at


def _tensors(case, seed):
    """Parameters, gradients and the states of a run that has gone on for a while, as flat buffers of whole
    blocks whose tails hold zeros."""
    (starts, total), sizes = _segments(case), _sizes(case)
    inside = torch.zeros(total, device=_device())
    for a, s in zip(starts, sizes):
        inside[a:a + s] = 1.0
    master = _normal(seed, 11, 0.02, (total,)) * inside
    grad = _normal(seed, 12, 1e-3, (total,)) * inside
    m, r = _normal(seed, 13, 3e-4, (total,)) * inside, (5e-4 + 1e-3 * _uniform(seed, 14, (total,))) * inside
    t = dict(grad=grad.to(_dtype(case)))
    if case["bits"] == 8:
        for name, x in (("m", m), ("r", r)):
            scale = x.view(-1, BLOCK).abs().amax(1) / 448.0
            t[name] = (x.view(-1, BLOCK) / scale[:, None]).nan_to_num_(0.0).to(FP8).view(-1)
            t[name + "_scale"] = scale
    else:
        t["m"], t["v"] = m, r * r
    t["param"] = master.to(_dtype(case))
    if case["dtype"] == "bf16":
        t["master"] = master
    return t


def prepare(case, seed):
    s = SimpleNamespace(case=case)
    if case["op"] == "adamw":
        (starts, _), sizes = _segments(case), _sizes(case)
        s.flat, s.step = _tensors(case, seed), 1000
        if own:
            from paper_2510_05421_amd import learn

            def cut(x, per=1):
                return [x[a // per:a // per + -(-n // per)] for a, n in zip(starts, sizes)]

            f = s.flat
            states = {k: cut(f[k], BLOCK if k.endswith("scale") else 1) for k in f if k not in ("param", "grad")}
            s.grads = cut(f["grad"])
            s.opt = learn.AdamW(cut(f["param"]), lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY,
                                max_norm=MAX_NORM if case["clip"] else 0.0, state_bits=case["bits"], seed=SEED, states=states,
                                step_count=s.step)
        return s
    s.logits, s.tokens, live = _rows(case, seed)
    if case["op"] == "logp":
        return s
    n, T = case["rows"], case["temp"]
    lp = torch.empty(n, device=_device())
    for i in range(0, n, 1024):
        z = s.logits[i:i + 1024].float() / T
        lp[i:i + 1024] = z.gather(1, s.tokens[i:i + 1024, None].clamp(min=0).long())[:, 0] - z.logsumexp(-1)
    # the policy has moved a little since the tokens were drawn; a ratio within a rounding of the border
    # would fall on either side of it in any arithmetic, so those are moved off it
    moved = _normal(seed, 21, 0.15, (n,))
    for border in (math.log(1 - CLIP[0]), math.log(1 + CLIP[1])):
        moved = torch.where((moved - border).abs() < 5e-4, border + 1e-3, moved)
    s.old = lp - moved
    s.adv = _normal(seed, 22, 1.0, (n,))
    s.weights = live.float() / live.sum()
    s.ref_logits = s.ref_logp = None
    if case["ref"] == "tokens":
        s.ref_logp = lp + _normal(seed, 23, 0.1, (n,))
    elif case["ref"] == "logits":
        s.ref_logits = (s.logits.float() + _normal(seed, 24, 0.3, tuple(s.logits.shape))).to(_dtype(case))
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    case = s.case
    if own:
        from paper_2510_05421_amd import learn
        if case["op"] == "logp":
            lp, ent = learn.token_logprobs(s.logits, s.tokens, temperature=case["temp"], entropy=True)
            return {"logp": lp, "entropy": ent}
        if case["op"] == "policy":
            out = learn.policy_loss(s.logits, s.tokens, s.adv, s.old, s.weights, ref_logits=s.ref_logits, ref_logp=s.ref_logp,
                                    temperature=case["temp"], ref_temperature=REF_T, clip_low=CLIP[0], clip_high=CLIP[1],
                                    c_kl=C_KL if case["ref"] != "none" else 0.0, c_ent=C_ENT)
            return {"terms": out.terms, "logp": out.logp, "grad": out.grad}
        s.opt.step(s.grads)
        return _updated(s, s.opt.grad_norm[0] if case["clip"] else None)
    if case["op"] == "logp":
        return _plain_logp(s)
    if case["op"] == "policy":
        return _plain_policy(s)
    return _plain_adamw(s)


def _updated(s, norm):
    out = {k: v for k, v in s.flat.items() if k != "grad"}
    if s.case["clip"]:
        out["grad_norm"] = norm
    return out


def _softmax_rows(z):
    """p, log p and the log of the sum (in 64 bits) of every row; rows without a logit: zeros."""
    top = z.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    e = torch.exp(z - top)
    lse = top[:, 0].double() + e.sum(-1, dtype=torch.float64).log()
    lg = z - lse[:, None].float()
    return torch.exp(lg), lg, lse


def _times(p, x):
    return torch.where(p > 0, p * x, 0.0)


def _plain_logp(s):
    V = s.logits.shape[1]
    z = s.logits.float() / s.case["temp"]
    p, lg, lse = _softmax_rows(z)
    live = (s.tokens >= 0) & (s.tokens < V) & (lse > -math.inf)
    at = s.tokens.clamp(0, V - 1).long()[:, None]
    lp = z.gather(1, at)[:, 0].double() - lse
    ent = -_times(p, lg).sum(-1)
    return {"logp": torch.where(live, lp.float(), 0.0), "entropy": torch.where(live, ent, 0.0)}


def _plain_policy(s):
    case, V, T = s.case, s.logits.shape[1], s.case["temp"]
    z = s.logits.float() / T
    p, lg, lse = _softmax_rows(z)
    live = (s.tokens >= 0) & (s.tokens < V) & (lse > -math.inf) & (s.weights != 0)
    at = s.tokens.clamp(0, V - 1).long()[:, None]
    lp = z.gather(1, at)[:, 0].double() - lse
    ratio = torch.exp(lp - s.old)
    adv = s.adv.double()
    plain, clipped = ratio * adv, ratio.clamp(1 - CLIP[0], 1 + CLIP[1]) * adv
    pol, cut = -torch.minimum(plain, clipped), clipped < plain
    by_lp = torch.where(cut, 0.0, -plain)
    ent = -_times(p, lg).sum(-1)
    kl, c_kl = torch.zeros_like(lp), C_KL if case["ref"] != "none" else 0.0
    by_z = C_ENT * _times(p, lg + ent[:, None])
    if case["ref"] == "tokens":
        r = s.ref_logp - lp
        kl = torch.exp(r) - r - 1
        by_lp = by_lp + c_kl * (1 - torch.exp(r))
    elif case["ref"] == "logits":
        _, lq, _ = _softmax_rows(s.ref_logits.float() / REF_T)
        apart = lg - lq
        kl = _times(p, apart).sum(-1)
        by_z = by_z + c_kl * _times(p, apart - kl[:, None])
        kl = kl.double()
    grad = by_z - by_lp.float()[:, None] * p
    grad.scatter_add_(1, at, by_lp.float()[:, None])
    grad = torch.where(live[:, None], grad * (s.weights / T)[:, None], 0.0)
    w = s.weights.double()
    rows = torch.stack([pol, kl, ent.double(), cut.double()])
    rows = torch.where(live, rows, 0.0)
    pol, kl, ent, cut = (rows * torch.where(live, w, 0.0)).sum(-1)
    terms = torch.stack([pol + c_kl * kl - C_ENT * ent, pol, kl, ent, cut])
    return {"terms": terms.float(), "logp": torch.where(live, lp, 0.0).float(), "grad": grad.to(s.logits.dtype)}


MASK32 = 0xFFFFFFFF


def _keys(seed, step):
    """The step's two 32-bit keys: one 64-bit mix of the seed and the step."""
    x = (seed + step * 0x9E3779B97F4A7C15) & 0xFFFFFFFFFFFFFFFF
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & 0xFFFFFFFFFFFFFFFF
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & 0xFFFFFFFFFFFFFFFF
    x ^= x >> 31
    return x & MASK32, x >> 32


def _random_bits(count, keys):
    """32 random bits for every element of the flat buffer (fewer than 2^32 elements)."""
    h = torch.arange(count, device=_device()) ^ keys[0]
    h = ((h ^ (h >> 16)) * 0x7FEB352D) & MASK32
    h = ((h ^ (h >> 15)) * 0x846CA68B) & MASK32
    h = (((h ^ (h >> 16)) + keys[1]) * 0x9E3779B1) & MASK32
    return h ^ (h >> 15)


def _to_fp8(x, bits):
    """x >= 0, at most 448, rounded to e4m3 up or down by 16 random bits."""
    small = x < 2.0 ** -6
    t = torch.where(small, x + 2.0 ** -6, x)   # the spacing of e4m3 below 2^-6 is that of the next binade
    t = ((t.view(torch.int32) + (bits << 4).to(torch.int32)) & -(1 << 20)).view(torch.float32)
    return torch.where(small, t - 2.0 ** -6, t)


def _plain_adamw(s):
    case, f = s.case, s.flat
    s.step += 1
    b1, b2 = BETAS
    g = f["grad"].float()
    norm = None
    if case["clip"]:
        norm = f["grad"].double().square().sum().sqrt()
        g = g * torch.clamp(MAX_NORM / norm, max=1.0).float()
        norm = norm.float()
    eight = case["bits"] == 8
    m, v = f["m"], f.get("v")
    if eight:
        m = (f["m"].float().view(-1, BLOCK) * f["m_scale"][:, None]).view(-1)
        v = (f["r"].float().view(-1, BLOCK) * f["r_scale"][:, None]).view(-1).square()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    r = v.sqrt()
    master = f.get("master", f["param"])
    rate, root = LR / (1 - b1 ** s.step), 1 / math.sqrt(1 - b2 ** s.step)
    new = master * (1 - LR * DECAY) - rate * m / (r * root + EPS)
    master.copy_(new)
    if "master" in f:
        f["param"].copy_(new)
    if not eight:
        f["m"].copy_(m)
        f["v"].copy_(v)
        return _updated(s, norm)
    bits = _random_bits(m.numel(), _keys(SEED, s.step))
    for name, x, part in (("m", m, bits & 0xFFFF), ("r", r, bits >> 16)):
        top = x.view(-1, BLOCK).abs().amax(1)
        top = torch.where(top < 2.0 ** -100, 0.0, top)
        inverse = torch.where(top > 0, 448.0 / top, 0.0)
        y = (x.view(-1, BLOCK).abs() * inverse[:, None]).view(-1).clamp(max=448.0)
        t = _to_fp8(y, part)
        if name == "r":
            t = torch.where(y > 0, t.clamp(min=2.0 ** -9), t)   # a root that is not zero stays so
        f[name].copy_(torch.copysign(t, x).to(FP8))
        f[name + "_scale"].copy_(top / 448.0)
    return _updated(s, norm)


# ------------------------------------------------------------------ work
def work(case):
    if case["op"] == "adamw":
        n = float(sum(_sizes(case)))
        es, state = (2 if case["dtype"] == "bf16" else 4), (2 * case["bits"] / 8)
        per = es + 2 * state + (es + 8 if case["dtype"] == "bf16" else 8)   # gradient; states; parameter and master
        return {"bytes": n * per, "flops": 20 * n}
    es = 2 if case["dtype"] == "bf16" else 4
    live = max(1.0, round(case["rows"] * (1 - case["masked"])))
    cells, all_cells = live * case["vocab"], float(case["rows"]) * case["vocab"]
    if case["op"] == "logp":
        return {"bytes": es * cells + 12.0 * case["rows"], "flops": 6 * cells}
    reads = 2 if case["ref"] == "logits" else 1
    return {"bytes": es * (reads * cells + all_cells) + 24.0 * case["rows"], "flops": (18 if reads == 2 else 12) * cells}


# ------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    if case["op"] == "adamw":
        return _exact_adamw(case, seed)
    s = prepare(case, seed)
    n, V, T = case["rows"], case["vocab"], case["temp"]
    out = {k: [] for k in (("logp", "entropy") if case["op"] == "logp" else ("logp", "grad"))}
    sums = torch.zeros(5, dtype=torch.float64, device=s.logits.device)
    for i in range(0, n, 256):
        part = _exact_rows(case, s, slice(i, min(n, i + 256)), T, sums)
        for k in out:
            out[k].append(part[k])
    out = {k: torch.cat(v) for k, v in out.items()}
    return out if case["op"] == "logp" else dict(out, terms=sums)


def _exact_rows(case, s, at, T, sums):
    """Some rows by the definition; the gradient by differentiating the loss."""
    z = s.logits[at].double()
    z = torch.where(z == -math.inf, -1e6, z).requires_grad_()   # exp(-1e6) is 0 in 64 bits too
    tok = s.tokens[at].long()
    live = tok >= 0
    lg = torch.log_softmax(z / T, -1)
    p = lg.exp()
    ent = -(p * lg).sum(-1)
    lp = lg[torch.arange(len(tok), device=z.device), tok.clamp(min=0)]
    if case["op"] == "logp":
        return {"logp": (lp * live).detach(), "entropy": (ent * live).detach()}
    w = s.weights[at].double()
    adv = s.adv[at].double()
    ratio = (lp - s.old[at].double()).exp()
    held = ratio.clamp(1 - CLIP[0], 1 + CLIP[1])
    cut = held * adv < ratio * adv
    pol = -torch.where(cut, held * adv, ratio * adv)
    kl, c_kl = 0 * lp, C_KL
    if case["ref"] == "tokens":
        r = s.ref_logp[at].double() - lp
        kl = r.exp() - r - 1
    elif case["ref"] == "logits":
        q = s.ref_logits[at].double()
        kl = (p * (lg - torch.log_softmax(torch.where(q == -math.inf, -1e6, q) / REF_T, -1))).sum(-1)
    else:
        c_kl = 0.0
    w = torch.where(live, w, 0.0)
    loss = (w * (pol + c_kl * kl - C_ENT * ent)).sum()
    loss.backward()
    sums += torch.stack([x.detach() for x in (loss, (w * pol).sum(), (w * kl).sum(), (w * ent).sum(), (w * cut).sum())])
    return {"logp": (lp * live).detach(), "grad": z.grad}


def _exact_adamw(case, seed):
    f = {k: v.double() for k, v in _tensors(case, seed).items()}
    t, (b1, b2) = 1001, BETAS
    g = f["grad"]
    norm = float(g.norm())
    if case["clip"]:
        g = g * min(1.0, MAX_NORM / norm)
    blocks = g.view(-1, BLOCK)
    if case["bits"] == 8:
        m0 = f["m"].view(-1, BLOCK) * f["m_scale"][:, None]
        v0 = (f["r"].view(-1, BLOCK) * f["r_scale"][:, None]) ** 2
    else:
        m0, v0 = f["m"].view(-1, BLOCK), f["v"].view(-1, BLOCK)
    m, v = b1 * m0 + (1 - b1) * blocks, b2 * v0 + (1 - b2) * blocks ** 2
    p = f.get("master", f["param"]).view(-1, BLOCK)
    p = p - LR * DECAY * p - LR * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + EPS)
    out = {"param": p.view(-1)}
    if "master" in f:
        out["master"] = p.view(-1)
    if case["clip"]:
        out["grad_norm"] = norm
    if case["bits"] == 32:
        return dict(out, m=m.view(-1), v=v.view(-1))
    bits = _random_bits(g.numel(), _keys(SEED, t)).view(-1, BLOCK)
    for name, x, part in (("m", m, bits % 65536), ("r", v.sqrt(), bits // 65536)):
        scale = x.abs().amax(1, keepdim=True) / 448
        y = (x.abs() / scale).nan_to_num(0.0).clamp(max=448.0)
        # the spacing of e4m3 at y, then up by chance: where the fraction and the random bits reach one
        gap = 2.0 ** (torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
        code = torch.floor(y / gap + part.double() / 65536) * gap
        if name == "r":
            code = torch.where((y > 0) & (code == 0), 2.0 ** -9, code)
        out[name], out[name + "_scale"] = (code * x.sign()).view(-1), scale.view(-1)
    return out
