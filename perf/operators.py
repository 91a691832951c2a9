"""Performance cases of the operators at both ends of the vocabulary: from tokens to vectors, from hidden states to logits, and
from the logits of drafted tokens to the tokens that are kept.

Where `own` is false, `run` computes each operator from elementary torch operations; where it is true it calls the library.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
ESIZE = {"fp32": 4, "bf16": 2}
BLOCK = 256  # entries that share one uniform when the last token is drawn
GROUP = 128  # entries that share one scale
E4M3 = torch.float8_e4m3fn
CHUNK = 1 << 28  # logits made at a time


def _verify(seqs, drafts, vocab, dtype, model, ragged=False, greedy=0.0):
    return {"op": "verify", "seqs": seqs, "drafts": drafts, "vocab": vocab, "dtype": dtype, "model": model, "ragged": ragged,
            "greedy": greedy}


def _embed(tokens, vocab, width, dtype, pad=0.0):
    return {"op": "embed", "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype, "pad": pad}


def _embed_backward(tokens, vocab, width, dtype, pad=0.0):
    return {"op": "embed backward", "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype, "pad": pad}


def _quantize(rows, width, dtype, table):
    return {"op": "quantize", "rows": rows, "width": width, "dtype": dtype, "table": table}


def _project(rows, vocab, width, dtype):
    return {"op": "project", "rows": rows, "vocab": vocab, "width": width, "dtype": dtype}


def listed():
    return [
        # the tail of a rollout: a few sequences left, drafts of different lengths, some greedy, rows that begin anywhere
        dict(_verify(8, 5, 33333, "fp32", True, True, 0.25), name="verify few odd"),
        # one step of 64 prompts, four tokens each from a small model with its own distributions
        dict(_verify(64, 4, 151936, "bf16", True), name="verify rollout"),
        # the headline batch of 512 rollouts, three tokens each copied from the prompt: no distribution of the draft
        dict(_verify(512, 3, 151936, "bf16", False), name="verify lookup batch"),
        # the input of one decode step of the headline batch
        dict(_embed(512, 151936, 2048, "bf16"), name="embed decode"),
        # the input of a training pass over 64 responses of 2,048 tokens
        dict(_embed(131072, 151936, 1536, "bf16"), name="embed training"),
        # the table's gradient from that pass
        dict(_embed_backward(131072, 151936, 1536, "bf16"), name="embed backward training"),
        # the table's gradient from a short padded batch, odd sizes, fp32
        dict(_embed_backward(3001, 33333, 1001, "fp32", 0.1), name="embed backward odd"),
        # hidden states of one decode step of the headline batch, a scale for 128 entries of a row
        dict(_quantize(512, 2048, "bf16", False), name="quantize hidden"),
        # the table after an update of the policy, a scale for 128 x 128 entries
        dict(_quantize(151936, 2048, "bf16", True), name="quantize table"),
        # logits of the last group of 8 that is still decoding: the table is what counts
        dict(_project(8, 151936, 2048, "bf16"), name="project few rows"),
        # logits of one decode step of the headline batch
        dict(_project(512, 151936, 2048, "bf16"), name="project rollout"),
        # odd sizes, fp32 logits
        dict(_project(77, 33333, 1000, "fp32"), name="project odd"),
    ]


MOST = {"verify": 512 * 4 * 151936, "embed": 131072 * 1536, "quantize": 151936 * 2048, "project": 512 * 151936 * 2048}


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    def a_vocab():  # padded to a multiple of 64 as most are, or whatever the tokenizer has
        v = spread(8000, 256000)
        return v // 64 * 64 if rng.random() < 0.5 else v

    def a_width(most=4096):
        d = spread(64, max(64, min(4096, most)))
        return max(64, d // 64 * 64) if rng.random() < 0.6 else d

    dtype = rng.choice(("bf16", "bf16", "fp32"))
    op = rng.choice(("verify", "verify", "embed", "embed backward", "quantize", "project", "project"))
    if op == "verify":
        vocab, drafts = a_vocab(), rng.randint(1, 8)
        most = MOST["verify"] * 2 // ESIZE[dtype] // vocab // (drafts + 1)
        model = rng.random() < 0.6
        return _verify(spread(1, min(512, most // (1 + model))), drafts, vocab, dtype, model, rng.random() < 0.5, rng.choice((0.0, 0.0, 0.2)))
    if op in ("embed", "embed backward"):
        vocab = a_vocab()
        width = a_width(2 * MOST["embed"] // ESIZE[dtype] // vocab)
        tokens = spread(1, min(131072, 2 * MOST["embed"] // ESIZE[dtype] // width))
        return (_embed if op == "embed" else _embed_backward)(tokens, vocab, width, dtype, rng.choice((0.0, 0.1)))
    if op == "quantize":
        table = rng.random() < 0.5
        rows = a_vocab() if table else spread(1, 4096)
        return _quantize(rows, a_width(2 * MOST["quantize"] // ESIZE[dtype] // rows), dtype, table)
    vocab, width = a_vocab(), a_width()
    return _project(spread(1, min(4096, max(1, MOST["project"] // vocab // width))), vocab, width, dtype)


# ------------------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _logits(g, rows, vocab):
    """Rows as a language model gives them: a Gaussian body and a Zipf-like bias over a random ranking."""
    z = torch.randn((rows, vocab), generator=g, device=DEVICE)
    return z.mul_(3.0).sub_(torch.rand((rows, vocab), generator=g, device=DEVICE).mul_(vocab).log1p_().mul_(1.2))


def _tokens(g, n, vocab, pad):
    """Token numbers as text has them: frequency about one over the rank, ranks scattered over the vocabulary; -1 where padded."""
    rank = torch.exp(torch.rand(n, generator=g, device=DEVICE, dtype=torch.float64) * math.log(vocab + 1.0)).long().clamp_(1, vocab) - 1
    tok = torch.randperm(vocab, generator=g, device=DEVICE)[rank]
    return torch.where(torch.rand(n, generator=g, device=DEVICE) < pad, -1, tok).to(torch.int32)


def _prepare_verify(case, g):
    n, k, v, dt = case["seqs"], case["drafts"], case["vocab"], DTYPES[case["dtype"]]
    s = {}
    tau = torch.rand(n, generator=g, device=DEVICE) * 0.8 + 0.6
    s["temps"] = torch.where(torch.rand(n, generator=g, device=DEVICE) < case["greedy"], torch.zeros_like(tau), tau)
    lens = torch.randint(0, k + 1, (n,), generator=g, device=DEVICE) if case["ragged"] else torch.full((n,), k, device=DEVICE)
    s["draft_len"] = lens.to(torch.int32) if case["ragged"] else None
    s["logits"] = torch.empty((n * (k + 1), v), dtype=dt, device=DEVICE)
    if case["model"]:
        s["draft_logits"] = torch.empty((n * k, v), dtype=dt, device=DEVICE)
        s["draft_temps"] = tau
        s["draft_logp"] = torch.empty((n, k), device=DEVICE)
    else:
        s["draft_logits"] = s["draft_temps"] = s["draft_logp"] = None
    s["draft_tok"] = torch.empty((n, k), dtype=torch.int32, device=DEVICE)
    step = max(1, CHUNK // (v * (k + 1)))
    for lo in range(0, n, step):
        m = min(step, n - lo)
        z = _logits(g, m * (k + 1), v).view(m, k + 1, v)
        t = tau[lo:lo + m, None, None]
        if case["model"]:  # a smaller model: the target's logits with an error, drafts drawn from it
            y = (z[:, :k] + 0.7 * torch.randn((m, k, v), generator=g, device=DEVICE)).to(dt)
            s["draft_logits"][lo * k:(lo + m) * k] = y.view(m * k, v)
            y = y.float() / t
            gumbel = -torch.empty((m, k, v), device=DEVICE).exponential_(1.0, generator=g).log_()
            d = (y + gumbel).argmax(-1)
            s["draft_logp"][lo:lo + m] = y.gather(-1, d[..., None]).squeeze(-1) - y.logsumexp(-1)
        else:  # text that repeats: at most places the model agrees with the copied token
            d = torch.randint(0, v, (m, k), generator=g, device=DEVICE)
            agrees = torch.rand((m, k), generator=g, device=DEVICE) < 0.8
            high = z[:, :k].logsumexp(-1) + 1.0
            z[:, :k].scatter_(-1, d[..., None], torch.where(agrees, high, z[:, :k].gather(-1, d[..., None]).squeeze(-1))[..., None])
        s["draft_tok"][lo:lo + m] = d.to(torch.int32)
        s["logits"][lo * (k + 1):(lo + m) * (k + 1)] = z.view(m * (k + 1), v)
    # drafts behind a sequence's last are padding
    s["draft_tok"].masked_fill_(torch.arange(k, device=DEVICE) >= lens[:, None], -1)
    s["uniforms"] = torch.rand((n, k + -(-v // BLOCK) + 1), generator=g, device=DEVICE, dtype=torch.float64)
    return s


def _hidden(g, rows, width):
    """Activations: Gaussian entries, some channels and some rows much larger than the rest."""
    x = torch.randn((rows, width), generator=g, device=DEVICE)
    x *= torch.exp(torch.randn(width, generator=g, device=DEVICE))
    return x * torch.exp(0.5 * torch.randn((rows, 1), generator=g, device=DEVICE))


def _eight_bits(x, rows_per_scale):
    """e4m3 values and their scales, any positive scale: what some other program may have made."""
    rows, width = x.shape
    nr, nc = -(-rows // rows_per_scale), -(-width // GROUP)
    full = x.new_zeros((nr * rows_per_scale, nc * GROUP))
    full[:rows, :width] = x
    amax = full.view(nr, rows_per_scale, nc, GROUP).abs().amax((1, 3))
    scale = (amax / 400.0).clamp_min(1e-30)
    each = scale.repeat_interleave(rows_per_scale, 0)[:rows].repeat_interleave(GROUP, 1)[:, :width]
    q = torch.zeros((rows, -(-width // 16) * 16), device=DEVICE).to(E4M3)
    q[:, :width] = (x / each).to(E4M3)
    return q[:, :width], scale


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    op = case["op"]
    if op == "verify":
        s.update(_prepare_verify(case, g))
    elif op == "embed":
        s["table"] = torch.randn((case["vocab"], case["width"]), generator=g, device=DEVICE).to(DTYPES[case["dtype"]])
        s["tok"] = _tokens(g, case["tokens"], case["vocab"], case["pad"])
    elif op == "embed backward":
        s["g"] = torch.randn((case["tokens"], case["width"]), generator=g, device=DEVICE).to(DTYPES[case["dtype"]])
        s["tok"] = _tokens(g, case["tokens"], case["vocab"], case["pad"])
    elif op == "quantize":
        s["x"] = _hidden(g, case["rows"], case["width"]).to(DTYPES[case["dtype"]])
    else:
        s["x"], s["x_scale"] = _eight_bits(_hidden(g, case["rows"], case["width"]), 1)
        s["w"], s["w_scale"] = _eight_bits(torch.randn((case["vocab"], case["width"]), generator=g, device=DEVICE) * 0.03, GROUP)
    return s


def _scale_of(case):
    return math.sqrt(case["width"])


# --------------------------------------------------------------------------------------------------------------- what is run
def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2505_18573_b200 import binding as e3

        if op == "verify":
            return e3.e3_verify_drafts(s["logits"], s["temps"], s["draft_tok"], s["uniforms"], draft_len=s["draft_len"],
                                       draft_logits=s["draft_logits"], draft_temps=s["draft_temps"], draft_logp=s["draft_logp"])
        if op == "embed":
            return e3.e3_embed_tokens(s["table"], s["tok"], scale=_scale_of(s["case"]))
        if op == "embed backward":
            return e3.e3_embed_tokens_backward(s["g"], s["tok"], s["case"]["vocab"], scale=_scale_of(s["case"]))
        if op == "quantize":
            return e3.e3_quantize(s["x"], block_rows=GROUP if s["case"]["table"] else 1)
        return e3.e3_project_vocab(s["x"], s["x_scale"], s["w"], s["w_scale"], dtype=DTYPES[s["case"]["dtype"]])
    return {"verify": _plain_verify, "embed": _plain_embed, "embed backward": _plain_embed_backward, "quantize": _plain_quantize,
            "project": _plain_project}[op](s)


def _plain_verify(s):
    """All positions at once, in 64 bits: a draw is compared with borders that 32 bits put elsewhere."""
    n, k = s["draft_tok"].shape
    v = s["logits"].shape[1]
    z = s["logits"].view(n, k + 1, v).double()
    tau = s["temps"].double()[:, None, None]
    greedy = tau == 0
    x = z / torch.where(greedy, torch.ones_like(tau), tau)
    x -= x.amax(-1, keepdim=True)
    total = torch.exp(x).sum(-1, keepdim=True)
    x -= total.log()  # ln p
    ent = -(torch.exp(x) * x.clamp_min(-1e300)).sum(-1)
    best = z.argmax(-1, keepdim=True)
    del z
    one_hot = torch.full_like(x, -math.inf).scatter_(-1, best, 0.0) if s["case"]["greedy"] else x
    lp = torch.where(greedy, one_hot, x)
    ent = torch.where(greedy[..., 0], torch.zeros_like(ent), ent)
    d = s["draft_tok"].long().clamp_min(0)
    live = s["draft_tok"] >= 0
    lq = s["draft_logp"].double() if s["draft_logp"] is not None else torch.zeros((n, k), device=DEVICE, dtype=torch.float64)
    u = s["uniforms"]
    kept = live & (u[:, :k] * lq.exp() < lp[:, :k].gather(-1, d[..., None]).squeeze(-1).exp())
    a = torch.cumprod(kept.long(), 1).sum(1)
    seq = torch.arange(n, device=DEVICE)
    p = lp[seq, a].exp()
    at = a.clamp_max(k - 1)
    refused = (a < k) & live[seq, at]
    da = d[seq, at][:, None]
    if s["draft_logits"] is not None:
        y = s["draft_logits"].view(n, k, v)[seq, at].double()
        q = torch.exp((y - y.gather(-1, da)) / s["draft_temps"].double()[:, None] + lq[seq, at][:, None])
    else:
        q = torch.zeros_like(p).scatter_(-1, da, 1.0)
    r = torch.where(refused[:, None], (p - q).clamp_min(0.0), p)
    r = torch.where(r.sum(-1, keepdim=True) > 0, r, p)
    nb = -(-v // BLOCK)
    r = torch.nn.functional.pad(r, (0, nb * BLOCK - v)).view(n, nb, BLOCK)
    score = r.sum(-1).log() - (-(u[:, k:k + nb].log())).log()
    b = score.argmax(-1)
    prefix = r[seq, b].cumsum(-1)
    last = (b * BLOCK + (prefix > u[:, k + nb:] * prefix[:, -1:]).int().argmax(-1))[:, None]
    place = torch.arange(k + 1, device=DEVICE)
    tok = torch.where(place < a[:, None], torch.nn.functional.pad(d, (0, 1)), last)
    emitted = place <= a[:, None]
    logp = torch.where(emitted, lp.gather(-1, tok[..., None]).squeeze(-1), 0.0)
    return (torch.where(emitted, tok, -1).to(torch.int32), a.to(torch.int32), logp.float(), torch.where(emitted, ent, 0.0).float())


def _plain_embed(s):
    live = s["tok"] >= 0
    rows = s["table"][s["tok"].long().clamp_min(0)].float() * _scale_of(s["case"])
    return torch.where(live[:, None], rows, 0.0).to(s["table"].dtype)


def _plain_embed_backward(s):
    live = s["tok"] >= 0
    rows = torch.where(live[:, None], s["g"].float() * _scale_of(s["case"]), 0.0)
    out = torch.zeros((s["case"]["vocab"], s["case"]["width"]), device=DEVICE)
    return out.index_add_(0, s["tok"].long().clamp_min(0), rows).to(s["g"].dtype)


def _plain_quantize(s):
    x, per = s["x"].float(), GROUP if s["case"]["table"] else 1
    rows, width = x.shape
    nr, nc = -(-rows // per), -(-width // GROUP)
    full = torch.nn.functional.pad(x, (0, nc * GROUP - width, 0, nr * per - rows)).view(nr, per, nc, GROUP)
    amax = full.abs().amax((1, 3))
    fraction, exponent = torch.frexp(amax)  # 448 = 0.875 * 2^9
    scale = torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), exponent - 9 + (fraction > 0.875).int()), 1.0)
    q = (full / scale[:, None, :, None]).view(nr * per, nc * GROUP)[:rows, :width]
    return q.to(E4M3), scale


def _plain_project(s):
    def values(q, scale, per):
        rows, width = q.shape
        each = scale.repeat_interleave(per, 0)[:rows].repeat_interleave(GROUP, 1)[:, :width]
        return q.float() * each

    return (values(s["x"], s["x_scale"], 1) @ values(s["w"], s["w_scale"], GROUP).t()).to(DTYPES[s["case"]["dtype"]])


# ------------------------------------------------------------------------------------------------------------------- sizes
def _distinct(tokens, vocab):
    """About how many different numbers `_tokens` gives: ranks in steps of a tenth, each seen with its own probability."""
    seen, lo = 0.0, 1
    while lo <= vocab:
        hi = min(vocab + 1, max(lo + 1, int(lo * 1.1)))
        share = math.log(hi / lo) / math.log(vocab + 1.0) / (hi - lo)
        seen += (hi - lo) * -math.expm1(-tokens * share)
        lo = hi
    return seen


def work(case):
    op = case["op"]
    if op == "verify":
        n, k, v = case["seqs"], case["drafts"], case["vocab"]
        keeps = 0.74 if case["model"] else 0.65  # how often a draft of these inputs is kept, where every one before it was
        lens = range(k + 1) if case["ragged"] else (k,)
        rows = sum(sum(keeps ** j for j in range(m + 1)) for m in lens) / len(lens)
        refused = sum(1 - keeps ** m for m in lens) / len(lens)
        drafts = refused if case["model"] else 0.0
        return {"bytes": n * (rows + drafts) * v * ESIZE[case["dtype"]] + n * (8.0 * (-(-v // BLOCK) + 1) + 20.0 * k + 16 + 12.0 * k),
                "flops": 5.0 * n * (rows + 2) * v}
    if op == "embed":
        t, d, e = case["tokens"], case["width"], ESIZE[case["dtype"]]
        return {"bytes": _distinct(t * (1 - case["pad"]), case["vocab"]) * d * e + t * d * e + 4.0 * t, "flops": 1.0 * t * d}
    if op == "embed backward":
        t, d, e = case["tokens"], case["width"], ESIZE[case["dtype"]]
        return {"bytes": (t * (1 - case["pad"]) + case["vocab"]) * d * e + 4.0 * t, "flops": 2.0 * t * d}
    if op == "quantize":
        r, d = case["rows"], case["width"]
        return {"bytes": r * d * (ESIZE[case["dtype"]] + 1.0) + 4.0 * -(-r // (GROUP if case["table"] else 1)) * -(-d // GROUP), "flops": 3.0 * r * d}
    r, v, d = case["rows"], case["vocab"], case["width"]
    return {"bytes": 1.0 * (r + v) * d + 4.0 * (r + -(-v // GROUP)) * -(-d // GROUP) + 1.0 * r * v * ESIZE[case["dtype"]], "flops": 2.0 * r * v * d}


# ----------------------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"verify": _exact_verify, "embed": _exact_embed, "embed backward": _exact_embed_backward, "quantize": _exact_quantize,
            "project": _exact_project}[case["op"]](s)


def _exact_verify(s):
    """One sequence after the other, one position after the other, as the definition reads."""
    n, k = s["draft_tok"].shape
    lens = s["draft_len"].tolist() if s["draft_len"] is not None else [k] * n
    drafts, taus, u = s["draft_tok"].tolist(), s["temps"].tolist(), s["uniforms"].cpu()
    tok = torch.full((n, k + 1), -1, dtype=torch.int32)
    logp, ent = torch.zeros((n, k + 1), dtype=torch.float64), torch.zeros((n, k + 1), dtype=torch.float64)
    count = torch.zeros(n, dtype=torch.int32)
    for i in range(n):
        for j in range(lens[i] + 1):
            row = s["logits"][i * (k + 1) + j].to(torch.float64)
            if taus[i] == 0:
                p = torch.zeros_like(row)
                p[int(torch.nonzero(row == row.max())[0])] = 1.0
                h = 0.0
            else:
                p = torch.softmax(row / taus[i], 0)
                h = float(torch.special.entr(p).sum())
            left = p
            if j < lens[i]:
                d = drafts[i][j]
                if s["draft_logits"] is not None:
                    y = s["draft_logits"][i * k + j].to(torch.float64)
                    q = torch.exp((y - y[d]) / s["draft_temps"][i].to(torch.float64) + s["draft_logp"][i, j].to(torch.float64))
                else:
                    q = torch.zeros_like(p)
                    q[d] = 1.0
                if float(u[i, j]) * float(q[d]) < float(p[d]):
                    tok[i, j], logp[i, j], ent[i, j] = d, math.log(float(p[d])), h
                    count[i] += 1
                    continue
                left = torch.relu(p - q)
                if float(left.sum()) == 0.0:
                    left = p
            sums = _sums(left)
            noise = -torch.log(-torch.log(u[i, k:k + len(sums)])).to(DEVICE)
            b = int(torch.argmax(torch.log(sums) + noise))
            part = left[b * BLOCK:(b + 1) * BLOCK].cpu().numpy()
            target, seen, at = float(u[i, -1]) * float(part.sum()), 0.0, len(part) - 1
            for e, w in enumerate(part):
                seen += float(w)
                if seen > target:
                    at = e
                    break
            t = b * BLOCK + at
            tok[i, j], logp[i, j], ent[i, j] = t, math.log(float(p[t])), h
            break
    return tok, count, logp, ent


def _sums(left):
    whole = left.numel() // BLOCK * BLOCK
    sums = left[:whole].reshape(-1, BLOCK).sum(1)
    return torch.cat([sums, left[whole:].sum().reshape(1)]) if whole < left.numel() else sums


def _exact_embed(s):
    padded = torch.cat([s["table"], s["table"].new_zeros((1, s["table"].shape[1]))])
    tok = torch.where(s["tok"] < 0, s["table"].shape[0], s["tok"].long())
    return torch.index_select(padded, 0, tok).to(torch.float64) * _scale_of(s["case"])


def _exact_embed_backward(s):
    """Sorted tokens, their running sums, and the differences of these at the ends of each token's run; a slice of columns at a time."""
    v = s["case"]["vocab"]
    order = torch.sort(s["tok"].long(), stable=True)
    ends = torch.searchsorted(order.values, torch.arange(-1, v, device=DEVICE), right=True)
    out = []
    for g in s["g"].split(256, 1):
        running = torch.nn.functional.pad(torch.cumsum(g[order.indices].to(torch.float64), 0), (0, 0, 1, 0))
        out.append((running[ends[1:]] - running[ends[:-1]]) * _scale_of(s["case"]))
    return torch.cat(out, 1)


def _exact_quantize(s):
    x, per = s["x"].to(torch.float64), GROUP if s["case"]["table"] else 1
    q, scales = torch.empty_like(x), []
    for c in range(0, x.shape[1], GROUP):
        part = x[:, c:c + GROUP]
        top = part.abs().amax(1)
        top = torch.nn.functional.pad(top, (0, -len(top) % per)).view(-1, per).amax(1)
        scale = torch.where(top > 0, torch.exp2(torch.ceil(torch.log2(top / 448.0))), 1.0)
        scale = torch.where(top > 448.0 * scale, 2 * scale, torch.where((top > 0) & (top <= 224.0 * scale), scale / 2, scale))
        t = part / scale.repeat_interleave(per)[:len(part), None]
        # four significant bits, no finer than 2^-9, half to even
        step = torch.exp2(torch.floor(torch.log2(t.abs().clamp_min(2.0 ** -6))) - 3)
        q[:, c:c + GROUP] = torch.round(t / step) * step
        scales.append(scale)
    return q, torch.stack(scales, 1)


def _exact_project(s):
    """Block after block of the inner axis, as the scales are laid out."""
    x, w = s["x"], s["w"]
    out = torch.zeros((x.shape[0], w.shape[0]), dtype=torch.float64, device=DEVICE)
    for k in range(s["x_scale"].shape[1]):
        a = x[:, k * GROUP:(k + 1) * GROUP].to(torch.float64) * s["x_scale"][:, k, None].to(torch.float64)
        b = w[:, k * GROUP:(k + 1) * GROUP].to(torch.float64) * s["w_scale"][:, k].to(torch.float64).repeat_interleave(GROUP)[:w.shape[0], None]
        out.addmm_(a, b.t())
    return out
