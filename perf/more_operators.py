"""The calls at the end of a network over tokens whose speed matters to a user, as
measurable cases.

A network over tokens ends in logits: n rows of d numbers, one per token of the
vocabulary.  A case is an operator, its sizes and its types:

  logprob       log probability of each row's given token, the row's entropy and its
                `top` most probable tokens
  logprob_grad  the gradient of a loss of those log probabilities (and entropies) for
                the logits, beside the log probabilities themselves
  distill       how far each row is from a teacher's `top` saved logits (relative entropy)
  distill_grad  its gradient for the logits, beside the distances

A token number of -1 pads a ragged batch: its log probability is 0, and it takes part in
no gradient and no distance.
"""

import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
TEXT = 47236                 # columns of the sparse-text workload


def _case(name, op, n, d, kind, top=0, id_bits=64, entropy=False, scale=1.0, padded=0.0, gap=0,
          masked="none", whole=False):
    """n rows of d logits; entropy: whether it is wanted (logprob) or has a part in the loss
    (logprob_grad); scale: 1 / temperature; padded: share of token numbers that are -1; gap:
    columns between a row's end and the next row's start; masked: "none", or a third of the
    columns at minus infinity ("inf") or at the type's lowest value ("low"); whole: the
    teacher's logits come with the logarithm of their whole row's sum."""
    return dict(name=name, op=op, n=n, d=d, kind=kind, top=top, id_bits=id_bits, entropy=entropy,
                scale=scale, padded=padded, gap=gap, masked=masked, whole=whole)


def listed():
    return [
        # serving one token: its log probability beside five alternatives (latency)
        _case("score_token", "logprob", 1, TEXT, "bf16", top=5),
        # a decoding step of 64 requests, at a temperature, under a grammar's mask
        _case("score_step", "logprob", 64, TEXT, "bf16", top=20, entropy=True, scale=1.25,
              masked="inf"),
        # the tokens of whole texts scored
        _case("score_texts", "logprob", 8192, TEXT, "bf16", entropy=True, padded=0.03),
        # an odd vocabulary, rows of a wider matrix, the largest token beside the given one
        _case("score_odd", "logprob", 1001, 9973, "f16", top=1, id_bits=32, gap=19),
        # one token of each of a mini-batch's 250 texts, binary32
        _case("grad_batch", "logprob_grad", 250, TEXT, "f32", id_bits=32),
        # tokens of a small categorical vocabulary: many short rows
        _case("grad_short", "logprob_grad", 18750, 900, "f16", id_bits=32, padded=0.03),
        # a large training step, ragged texts padded with -1
        _case("grad_train", "logprob_grad", 8192, TEXT, "bf16", padded=0.03),
        # a policy's step with a bonus for entropy, a long vocabulary
        _case("grad_policy", "logprob_grad", 512, 200003, "bf16", entropy=True),
        # a request's tokens compared with a teacher's eight
        _case("distill_few", "distill", 16, TEXT, "bf16", top=8, id_bits=32),
        # a large evaluation against 64 saved logits a token
        _case("distill_eval", "distill", 8192, TEXT, "bf16", top=64, scale=0.5, padded=0.1),
        # a mini-batch's step in binary32
        _case("distill_batch", "distill_grad", 250, TEXT, "f32", top=20, whole=True),
        # a large training step at temperature 2
        _case("distill_train", "distill_grad", 8192, TEXT, "bf16", top=64, id_bits=32, scale=0.5,
              padded=0.1),
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["logprob", "logprob_grad", "distill", "distill_grad"])
    kind = rng.choice(["f32", "bf16", "bf16", "f16"])
    d = log(100, 262144)
    if rng.random() < 0.4:
        d = max(100, d // 64 * 64)
    n = min(log(1, 20000), 8192 * TEXT * 2 // SIZE[kind] // d)
    top, masked = 0, "none"
    if op == "logprob":
        top = rng.choice([0, 0, 1, log(2, 64)])
        if top:
            n = min(n, (1 << 25) // d)
    elif op.startswith("distill"):
        top = log(2, 100)
        n = min(n, (1 << 22) // top)
    if rng.random() < 0.3:
        masked = rng.choice(["inf", "low"])
    return dict(op=op, n=max(1, n), d=d, kind=kind, top=top, id_bits=rng.choice([32, 64]),
                entropy=op.startswith("logprob") and rng.random() < 0.5,
                scale=rng.choice([1.0, 1.0, 0.5, rng.uniform(0.3, 2.0)]),
                padded=rng.choice([0.0, 0.05]), gap=rng.choice([0, 0, 0, 8, rng.randint(1, 40)]),
                masked=masked, whole=op.startswith("distill") and rng.random() < 0.5)


# --- inputs -------------------------------------------------------------------


def _given(shape, d, case, g):
    """Token numbers, some of them -1."""
    ids = torch.randint(0, d, shape, generator=g, device=DEVICE)
    if case["padded"]:
        ids[torch.rand(shape, generator=g, device=DEVICE) < case["padded"]] = -1
    return ids


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    op, n, d, top, kind = case["op"], case["n"], case["d"], case["top"], TYPES[case["kind"]]
    ints = torch.int32 if case["id_bits"] == 32 else torch.int64
    Z = torch.empty((n, d + case["gap"]), dtype=kind, device=DEVICE)[:, :d]
    block = max(1, (1 << 27) // d)
    for r in range(0, n, block):
        rows = torch.randn((min(block, n - r), d), generator=g, device=DEVICE) * 2.5
        if case["masked"] != "none":
            low = -math.inf if case["masked"] == "inf" else torch.finfo(kind).min
            rows[torch.rand(rows.shape, generator=g, device=DEVICE) < 1 / 3] = low
        Z[r:r + block] = rows.to(kind)
    s = dict(case=case, Z=Z)
    if op.startswith("logprob"):
        s["ids"] = _given((n,), d, case, g)
    else:
        # a row's teacher: `top` different tokens (fewer where d is), its largest logit first
        first = torch.randint(0, d, (n, 1), generator=g, device=DEVICE)
        apart = max(1, d // top)
        s["ids"] = (first + apart * torch.arange(top, device=DEVICE)) % d
        s["ids"] = torch.where(_given((n, top), d, case, g) < 0, -1, s["ids"])
        if top > d:
            s["ids"][:, d:] = -1
        s["T"] = (9.0 - torch.rand((n, top), generator=g, device=DEVICE).cumsum(1)
                  * (8.0 / top)).to(kind)
    # the given tokens are likely ones, and no mask holds them
    for a in range(1 if s["ids"].dim() == 1 else top):
        one = s["ids"] if s["ids"].dim() == 1 else s["ids"][:, a]
        row = torch.arange(n, device=DEVICE)[one >= 0]
        height = 4.0 + 2.0 * torch.randn(n, generator=g, device=DEVICE)
        Z[row, one[row]] = height[row].to(kind)
    s["ids"] = s["ids"].to(ints)

    # a row's share of the mean loss; binary16 gradients are kept off its smallest numbers
    share = (4096.0 if case["kind"] == "f16" else 1.0) / n

    def blank(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=DEVICE)

    if op == "logprob":
        s["logp"] = blank(n)
        s["entropy"] = blank(n) if case["entropy"] else None
        s["top_ids"] = blank(n, top, dtype=ints) if top else None
        s["top_logp"] = blank(n, top) if top else None
    elif op == "logprob_grad":
        # a policy's advantages, or the mean's share with a weight a token
        s["dlogp"] = torch.randn(n, generator=g, device=DEVICE) * share
        s["dentropy"] = blank(n).fill_(0.01 * share) if case["entropy"] else None
        s["logp"] = blank(n)
        s["entropy"] = blank(n) if case["entropy"] else None
    else:
        s["loss"] = blank(n)
        # the rest of the teacher's row: a tenth to a half as much as the sum of its saved part
        s["T_lse"] = None
        if case["whole"]:
            e = torch.exp(case["scale"] * s["T"].double()).sum(1)
            more = 0.1 + 0.4 * torch.rand(n, generator=g, device=DEVICE)
            s["T_lse"] = torch.log(e * (1.0 + more)).float()
        if op == "distill_grad":
            s["dloss"] = torch.rand(n, generator=g, device=DEVICE) * share
    if op.endswith("grad"):
        s["dZ"] = torch.empty((n, d), dtype=kind, device=DEVICE)
    if own:
        # the workspace that a program keeps for all its steps
        import paper_1702_06943_amd as T
        size = T.toc_logits_workspace_size(n, d, top if op == "logprob" else 0)
        s["ws"] = blank(max(size, 16), dtype=torch.uint8)
    return s


# --- the operators in plain form ------------------------------------------------


def _softmax(s):
    """(scaled logits below their row's largest, exponentials, their sums)."""
    z = s["Z"].float()
    x = (z - z.amax(1, keepdim=True)) * s["case"]["scale"]
    e = torch.exp(x)
    return x, e, e.sum(1, keepdim=True)


def _entropy(x, e, total):
    return (torch.log(total) - torch.where(e > 0, e * x, 0.0).sum(1, keepdim=True) / total)[:, 0]


def _at(x, ids):
    """x at the rows' given tokens, and which of these are tokens."""
    ok = (ids >= 0) & (ids < x.shape[1])
    return x.gather(1, torch.where(ok, ids, 0)), ok


def _top(x, log_total, top, ints):
    """The largest of each row, again and again; the lowest column of equal ones."""
    x, number = x.clone(), torch.arange(x.shape[1], device=DEVICE, dtype=ints)
    ids, logp = [], []
    for _ in range(top):
        best = x.amax(1, keepdim=True)
        at = torch.where(x == best, number, x.shape[1]).amin(1, keepdim=True)
        x.scatter_(1, at.long(), -math.inf)
        none = best == -math.inf
        ids.append(torch.where(none, -1, at).to(ints))
        logp.append(torch.where(none, -math.inf, best - log_total))
    return torch.cat(ids, 1), torch.cat(logp, 1)


def _teacher(s, ok):
    """(the teacher's log probabilities, its probabilities): 0 where there is no token."""
    t = torch.where(ok, s["T"].float() * s["case"]["scale"], -math.inf)
    if s["T_lse"] is not None:
        log_q = t - s["T_lse"][:, None]
    else:
        top = torch.where(ok.any(1, keepdim=True), t.amax(1, keepdim=True), 0.0)
        log_q = t - top - torch.log(torch.exp(t - top).sum(1, keepdim=True))
    return log_q, torch.where(ok, torch.exp(log_q), 0.0)


def _plain(s):
    case, ids = s["case"], s["ids"].long()
    kind, scale = TYPES[case["kind"]], case["scale"]
    x, e, total = _softmax(s)
    log_total = torch.log(total)
    if case["op"].startswith("logprob"):
        there, ok = _at(x, ids[:, None])
        out = {"logp": torch.where(ok, there - log_total, 0.0)[:, 0]}
        if case["entropy"]:
            out["entropy"] = _entropy(x, e, total)
        if case["op"] == "logprob":
            if case["top"]:
                out["top_ids"], out["top_logp"] = _top(x, log_total, case["top"], s["ids"].dtype)
            return out
        p = e / total
        dl = torch.where(ok, s["dlogp"][:, None], 0.0)
        dz = p * -dl
        if case["entropy"]:
            inner = torch.where(p > 0, x - log_total + out["entropy"][:, None], 0.0)
            dz = dz - s["dentropy"][:, None] * p * inner
        dz.scatter_add_(1, torch.where(ok, ids[:, None], 0), dl)
        out["dz"] = (dz * scale).to(kind)
        return out
    there, ok = _at(x, ids)
    log_q, q = _teacher(s, ok)
    out = {"loss": torch.where(q > 0, q * (log_q - there + log_total), 0.0).sum(1)}
    if case["op"] == "distill_grad":
        dz = e * (q.sum(1, keepdim=True) / total)
        dz.scatter_add_(1, torch.where(ok, ids, 0), -q)
        out["dz"] = (dz * (s["dloss"][:, None] * scale)).to(kind)
    return out


def run(s):
    if not own:
        return _plain(s)
    import paper_1702_06943_amd as T
    case = s["case"]
    op, scale = case["op"], case["scale"]
    if op == "logprob":
        T.toc_logprob(s["Z"], s["ids"], s["logp"], entropy=s["entropy"], top_ids=s["top_ids"],
                      top_logp=s["top_logp"], scale=scale, ws=s["ws"])
        names = ["logp", "entropy", "top_ids", "top_logp"]
    elif op == "logprob_grad":
        T.toc_logprob_grad(s["Z"], s["dZ"], s["ids"], dlogp=s["dlogp"], dentropy=s["dentropy"],
                           logp=s["logp"], entropy=s["entropy"], scale=scale, ws=s["ws"])
        names = ["logp", "entropy"]
    elif op == "distill":
        T.toc_distill(s["Z"], s["ids"], s["T"], s["loss"], scale=scale, top_scale=scale,
                      top_lse=s["T_lse"], ws=s["ws"])
        names = ["loss"]
    else:
        T.toc_distill_grad(s["Z"], s["dZ"], s["ids"], s["T"], s["dloss"], loss=s["loss"],
                           scale=scale, top_scale=scale, top_lse=s["T_lse"], ws=s["ws"])
        names = ["loss"]
    out = {name: s[name] for name in names if s[name] is not None}
    if "dZ" in s:
        out["dz"] = s["dZ"]
    return out


# --- what a pass cannot do without ----------------------------------------------


def work(case):
    n, d, size, top, op = case["n"], case["d"], SIZE[case["kind"]], case["top"], case["op"]
    each = 5 + (2 if case["entropy"] else 0)
    count, small = n * d * size, n * 4 * (2 if case["entropy"] else 1)
    if op.startswith("logprob"):
        small += n * case["id_bits"] // 8
    if op == "logprob":
        small += n * top * (case["id_bits"] // 8 + 4)
    if op.startswith("distill"):
        small += n * top * (case["id_bits"] // 8 + size) + (4 * n if case["whole"] else 0)
    if op.endswith("grad"):
        small += 4 * n * (2 if case["entropy"] else 1)
        return {"bytes": 2 * count + small, "flops": (each + 2) * n * d}
    return {"bytes": count + small, "flops": each * n * d}


# --- the definition in 64 bits --------------------------------------------------


def _exact_rows(case, s, r):
    """The definition for the rows r (a slice): probabilities from the logarithm of the
    whole sum, one-hot targets, losses as sums over a row."""
    a = case["scale"]
    z = s["Z"][r].double() * a
    lse = torch.logsumexp(z, 1, keepdim=True)
    log_p = z - lse
    p = log_p.exp()
    ids = s["ids"][r].long()
    ids = ids[:, None] if ids.dim() == 1 else ids
    ok = ids >= 0
    safe = ids.clamp(min=0)
    out = {}
    if case["op"].startswith("logprob"):
        out["logp"] = (log_p.gather(1, safe) * ok)[:, 0]
        plogp = torch.where(p > 0, p * log_p, 0.0)
        h = -plogp.sum(1, keepdim=True)
        if case["entropy"]:
            out["entropy"] = h[:, 0]
        if case["op"] == "logprob" and case["top"]:
            order = torch.sort(z, dim=1, descending=True, stable=True)
            most = min(case["top"], case["d"])
            values, numbers = order.values[:, :most] - lse, order.indices[:, :most]
            numbers = torch.where(values == -math.inf, -1, numbers)
            pad = (0, case["top"] - most)
            out["top_ids"] = torch.nn.functional.pad(numbers, pad, value=-1)
            out["top_logp"] = torch.nn.functional.pad(values, pad, value=-math.inf)
        if case["op"] == "logprob_grad":
            dl = s["dlogp"][r].double()[:, None] * ok
            dz = torch.zeros_like(p).scatter_add_(1, safe, dl) - dl * p
            if case["entropy"]:
                dz -= s["dentropy"][r].double()[:, None] * (plogp + p * h)
            out["dz"] = a * dz
        return out
    w = torch.exp(a * s["T"][r].double()) * ok
    if s["T_lse"] is not None:
        q = w / torch.exp(s["T_lse"][r].double())[:, None]
    else:
        q = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    log_q = torch.where(q > 0, q, 1.0).log()
    out["loss"] = (q * torch.where(q > 0, log_q - log_p.gather(1, safe), 0.0)).sum(1)
    if case["op"] == "distill_grad":
        target = torch.zeros_like(p).scatter_add_(1, safe, q)
        out["dz"] = a * s["dloss"][r].double()[:, None] * (q.sum(1, keepdim=True) * p - target)
    return out


def exact(case, seed):
    n, d = case["n"], case["d"]
    s = prepare(case, seed)
    block = max(1, (1 << 25) // d)
    parts = [_exact_rows(case, s, slice(r, r + block)) for r in range(0, n, block)]
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
