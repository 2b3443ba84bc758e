"""Performance cases of the vocabulary operators: what a mixed batch's rows of logits [rows, vocab] become.

A case is a dict of plain values.  `listed()` gives the fixed ones, `draw(rng)` one more of the same ranges.
`prepare(case, seed)` makes what a program holds before the call, `run(state)` is one pass through one operator,
`work(case)` the bytes and operations the pass cannot do without, `exact(case, seed)` the outputs in 64 bits.  Where the
module's `own` is false, `run` computes the plain form in torch operations; where it is true, it calls the library.

Kinds:
  sample  one token for each inference row: temperature, top-k, top-p and min-p, each row with its own, from one uniform
          number a row.  The kept tokens are a prefix of the falling order of the logits (lowest index first among equals):
          the first k; of those, a token stays while the weight before it is below p times their sum; of those, weights of
          at least min_p times the largest.  The token is the first, in that order, whose running sum exceeds u times the
          sum of the kept.  Returns the tokens and the logarithms of the probabilities they were drawn with.
  top     the K largest logits of a teacher's rows, their places, and the log-sum-exp of row / temperature.
  loss    distillation from a teacher's K logits a row, forward alone: loss[row] = kd_weight tau^2 KL(p || softmax(z / tau)) +
          ce_weight CE(z, label).  p: softmax of the K over tau, or ("tail") their true probabilities by the teacher's
          log-sum-exp, with the remaining mass against the student's mass outside the K.
  train   the same forward and backward by two calls, the gradient of each row's loss given: loss and dlogits.
  step    the same by the one call that gives loss and dlogits at once.

`rows`: the tensor holds the rows of a mixed batch, of which an index list names those of the operator's kind.
"""
import math

import torch

own = False

WORKSPACE = 16 << 20  # bytes of device memory that a program keeps for these calls
CELLS = 8192 * 128256  # rows times vocabulary of the largest listed case


# ----------------------------------------------------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------------------------------------------------
def _sample(name, n, vocab, dtype, params, rows=False):
    return {"name": name, "kind": "sample", "n": n, "vocab": vocab, "dtype": dtype, "params": params, "rows": rows}


def _top(name, n, vocab, dtype, k, temperature, rows=False):
    return {"name": name, "kind": "top", "n": n, "vocab": vocab, "dtype": dtype, "k": k, "temperature": temperature, "rows": rows}


def _distill(name, kind, n, vocab, dtype, k, temperature, tail, labels, rows=False):
    return {"name": name, "kind": kind, "n": n, "vocab": vocab, "dtype": dtype, "k": k, "temperature": temperature, "tail": tail,
            "labels": labels, "rows": rows}


def listed():
    return [
        # the smallest call: one request's next token
        _sample("sample_1", 1, 32000, "bf16", "top_k_p"),
        # a decode step of 256 requests, each with sampling parameters of its own, among the rows of a mixed batch
        _sample("sample_256_mixed", 256, 128256, "bf16", "mixed", rows=True),
        # logits widened to fp32, a vocabulary that is no multiple of anything, some requests
        _sample("sample_200_f32_odd", 200, 50257, "f32", "mixed"),
        # the largest decode step: nucleus sampling of 1024 requests
        _sample("sample_1024_top_p", 1024, 128256, "bf16", "top_p"),
        # a teacher's record of a short training sequence, fp32
        _top("top_32_f32", 32, 32000, "f32", 20, 1.0),
        # a teacher's record of one step's training tokens (three sequences and a ragged one)
        _top("top_3277", 3277, 128256, "bf16", 64, 2.0),
        # odd vocabulary, wide record, the training rows of a mixed batch
        _top("top_205_odd", 205, 50257, "bf16", 250, 1.0, rows=True),
        # evaluation: the loss alone
        _distill("loss_1792", "loss", 1792, 32000, "bf16", 32, 2.0, False, False),
        # fp32, odd vocabulary, teacher's true probabilities and labels: forward and backward by two calls
        _distill("train_205_f32_odd", "train", 205, 50257, "f32", 48, 1.0, True, True),
        # the same two calls over the training rows of a mixed batch
        _distill("train_1024", "train", 1024, 128256, "bf16", 64, 2.0, True, False, rows=True),
        # a small training step: one short sequence beside decoding
        _distill("step_32", "step", 32, 32000, "bf16", 16, 1.0, False, True),
        # the largest: four sequences of 2048 tokens, loss and gradient at once
        _distill("step_8192", "step", 8192, 128256, "bf16", 64, 2.0, True, True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "top", "loss", "train", "step"])
    vocab = _log_uniform(rng, 8000, 160000)
    if rng.random() < 0.5:
        vocab = (vocab + 31) // 64 * 64
    most = {"sample": 1024, "top": 4096, "loss": 8192, "train": 4096, "step": 8192}[kind]
    cells = CELLS // {"sample": 8, "top": 2, "loss": 1, "train": 2, "step": 1}[kind]
    n = _log_uniform(rng, 1, max(1, min(most, cells // vocab)))
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if dtype == "f32":
        n = (n + 1) // 2
    rows = rng.random() < 0.3
    temperature = rng.choice([1.0, 1.0, 2.0, 1.5, 4.0])
    if kind == "sample":
        return {"kind": kind, "n": n, "vocab": vocab, "dtype": dtype, "params": rng.choice(["mixed", "top_p", "top_k_p", "plain"]),
                "rows": rows}
    k = _log_uniform(rng, 1, 256)
    if kind == "top":
        return {"kind": kind, "n": n, "vocab": vocab, "dtype": dtype, "k": k, "temperature": temperature, "rows": rows}
    return {"kind": kind, "n": n, "vocab": vocab, "dtype": dtype, "k": k, "temperature": temperature, "tail": rng.random() < 0.5,
            "labels": rng.random() < 0.5, "rows": rows}


def work(case):
    n, v = case["n"], case["vocab"]
    cells, e = n * v, 2 if case["dtype"] == "bf16" else 4
    index = 4 * n if case["rows"] else 0
    if case["kind"] == "sample":
        # one comparison a logit; parameters, random number, token and logarithm
        return {"bytes": cells * e + 28 * n + index, "flops": cells}
    if case["kind"] == "top":
        return {"bytes": cells * e + 8 * n * case["k"] + 4 * n + index, "flops": 4 * cells}
    record = 8 * n * case["k"] + (4 * n if case["tail"] else 0) + (4 * n if case["labels"] else 0) + 4 * n + index
    two = case["labels"] and case["temperature"] != 1.0  # softmaxes a row
    if case["kind"] == "loss":
        return {"bytes": cells * e + record, "flops": cells * (8 if two else 4)}
    return {"bytes": 2 * cells * e + record + 4 * n, "flops": cells * (14 if two else 7)}


# ----------------------------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------------------------
KD_WEIGHT, CE_WEIGHT = 0.7, 0.3


def _logits(g, n, vocab, dtype):
    """Rows as a language model's: words by rank (Zipf), noise, and a few candidates that stand out."""
    z = torch.randn((n, vocab), generator=g, device="cuda", dtype=torch.float32)
    z *= 1.5
    rank = torch.randperm(vocab, generator=g, device="cuda").float()
    z -= (rank + 2.0).log()
    at = torch.randint(0, vocab, (n, 12), generator=g, device="cuda")
    z.scatter_add_(1, at, 5.0 + 5.0 * torch.rand((n, 12), generator=g, device="cuda"))
    return z.to(torch.bfloat16) if dtype == "bf16" else z


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    pick = lambda choice, n: torch.tensor(choice, device="cuda")[torch.randint(0, len(choice), (n,), generator=g, device="cuda")]  # noqa: E731
    n, vocab = case["n"], case["vocab"]
    held = n + n // 8 + 1 if case["rows"] else n  # rows of the tensor
    s = {"case": case, "logits": _logits(g, held, vocab, case["dtype"]), "rows": None,
         "workspace": torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")}
    if case["rows"]:
        s["rows"] = torch.randperm(held, generator=g, device="cuda")[:n].sort().values.to(torch.int32)
    if case["kind"] == "sample":
        # every eighth request answers under a grammar that leaves a hundredth of the vocabulary
        for r in range(3, held, 8):
            s["logits"][r].masked_fill_(rand(vocab) > 0.01, -math.inf)
        how = case["params"]
        s["u"] = rand(n)
        s["temperature"] = (pick([0.0, 0.6, 0.7, 0.8, 1.0, 1.3], n) if how == "mixed" else pick([0.7, 0.8, 1.0], n)).float()
        s["top_k"] = s["top_p"] = s["min_p"] = None
        if how in ("mixed", "top_k_p"):
            s["top_k"] = (pick([0, 0, 1, 20, 50, 200], n) if how == "mixed" else pick([40, 50], n)).to(torch.int32)
        if how in ("mixed", "top_k_p", "top_p"):
            s["top_p"] = (pick([1.0, 1.0, 0.95, 0.9, 0.5], n) if how == "mixed" else pick([0.9, 0.95], n)).float()
        if how == "mixed":
            s["min_p"] = pick([0.0, 0.0, 0.0, 0.05], n).float()
        s["token"] = torch.empty(n, dtype=torch.int32, device="cuda")
        s["logprob"] = torch.empty(n, dtype=torch.float32, device="cuda")
        return s
    k = case["k"]
    if case["kind"] == "top":
        s["values"] = torch.empty((n, k), dtype=torch.float32, device="cuda")
        s["indices"] = torch.empty((n, k), dtype=torch.int32, device="cuda")
        s["lse"] = torch.empty(n, dtype=torch.float32, device="cuda")
        return s
    # the teacher agrees with the student up to noise; its record was made elsewhere, by torch here
    values, indices, lse = [], [], []
    for lo in range(0, n, 1024):
        hi = min(n, lo + 1024)
        z = s["logits"][lo:hi] if s["rows"] is None else s["logits"][s["rows"][lo:hi].long()]
        t = z.float() + 0.7 * torch.randn((hi - lo, vocab), generator=g, device="cuda")
        v, i = t.topk(min(k, vocab), dim=1)
        values.append(v)
        indices.append(i.to(torch.int32))
        lse.append(torch.logsumexp(t / case["temperature"], 1))
    s["t_values"], s["t_indices"] = torch.cat(values), torch.cat(indices)
    s["t_lse"] = torch.cat(lse) if case["tail"] else None
    # some rows have a shorter record, a few (padding of the batch) none
    s["t_indices"][5::16, k - k // 4:] = -1
    s["t_indices"][7::32] = -1
    s["labels"] = None
    if case["labels"]:
        s["labels"] = torch.where(rand(n) < 0.1, -100, s["t_indices"][:, 0].clone()).to(torch.int32)
    s["dloss"] = torch.full((n,), 1.0 / n, device="cuda") * (0.5 + rand(n))
    s["loss"] = torch.empty(n, dtype=torch.float32, device="cuda")
    if case["kind"] != "loss":
        s["stats"] = torch.empty((n, 8), dtype=torch.float32, device="cuda")
        s["dlogits"] = torch.zeros_like(s["logits"])
    return s


# ----------------------------------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _library(s)
    kind = s["case"]["kind"]
    return _plain_sample(s) if kind == "sample" else _plain_top(s) if kind == "top" else _plain_distill(s)


def _library(s):
    from paper_2604_16400_amd import binding

    c = s["case"]
    common = {"rows": s["rows"], "workspace": s["workspace"]}
    if c["kind"] == "sample":
        binding.collm_sample(s["logits"], s["u"], s["token"], s["logprob"], temperature=s["temperature"], top_k=s["top_k"],
                             top_p=s["top_p"], min_p=s["min_p"], **common)
        return s["token"], s["logprob"]
    if c["kind"] == "top":
        binding.collm_top_logits(s["logits"], s["values"], s["indices"], s["lse"], temperature=c["temperature"], **common)
        return s["values"], s["indices"], s["lse"]
    common.update(t_lse=s["t_lse"], labels=s["labels"], temperature=c["temperature"], kd_weight=KD_WEIGHT, ce_weight=CE_WEIGHT)
    teacher = (s["t_values"], s["t_indices"])
    if c["kind"] == "step":
        binding.collm_distill_fwd_bwd(s["logits"], *teacher, s["dloss"], s["loss"], s["dlogits"], **common)
        return s["loss"], s["dlogits"]
    if c["kind"] == "loss":
        binding.collm_distill_fwd(s["logits"], *teacher, s["loss"], **common)
        return s["loss"]
    binding.collm_distill_fwd(s["logits"], *teacher, s["loss"], s["stats"], **common)
    binding.collm_distill_bwd(s["logits"], *teacher, s["stats"], s["dloss"], s["dlogits"], **common)
    return s["loss"], s["dlogits"]


def _chosen(s):
    z = s["logits"] if s["rows"] is None else s["logits"][s["rows"].long()]
    return z.float()


def _plain_sample(s):
    z = _chosen(s)
    z = torch.where(z.isnan(), -math.inf, z)
    n, vocab = z.shape
    z, order = z.sort(dim=1, descending=True, stable=True)
    t = s["temperature"].double()[:, None]
    greedy = ~(t > 0)
    # weights in 64 bits: a token changes where a running sum passes a border by the least amount
    y = (z.double() - z[:, :1].double()) / torch.where(greedy, 1.0, t)
    w = torch.where(z == z[:, :1], 1.0, y.exp())
    w = torch.where(z == -math.inf, 0.0, w)
    place = torch.arange(vocab, device=z.device)[None, :]
    kept = (z > -math.inf) & ((place == 0) | ~greedy)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        kept &= (place < k) | (k <= 0)
    w = w * kept
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        run_ = w.cumsum(1)
        kept &= (run_ - w < p * run_[:, -1:]) | ~(p < 1) | (place == 0)
    if s["min_p"] is not None:
        kept &= ~(w < s["min_p"].double()[:, None].clamp(max=1.0))
    w = w * kept
    run_ = w.cumsum(1)
    total = run_[:, -1:]
    last = kept.sum(1, keepdim=True) - 1
    at = (run_ <= s["u"].double()[:, None] * total).sum(1, keepdim=True).minimum(last)
    none = last[:, 0] < 0
    at = at.clamp(min=0)
    token = order.gather(1, at)[:, 0].masked_fill(none, -1)
    logprob = (w.gather(1, at) / total).log()[:, 0].masked_fill(none, -math.inf)
    return token.to(torch.int32), logprob.float()


def _plain_top(s):
    c = s["case"]
    z = _chosen(s)
    z = torch.where(z.isnan(), -math.inf, z)
    n, vocab = z.shape
    # unique keys whose order is (value falling, place rising): the value's bits, then the place from behind
    bits = torch.where(z == 0, 0.0, z).view(torch.int32).long()
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 32) + (vocab - 1 - torch.arange(vocab, device=z.device))
    best = key.topk(min(c["k"], vocab), dim=1).values
    indices = vocab - 1 - (best & 0xFFFFFFFF)
    values = z.gather(1, indices)
    indices = indices.masked_fill(values == -math.inf, -1)
    pad = c["k"] - indices.shape[1]
    values = torch.nn.functional.pad(values, (0, pad), value=-math.inf)
    indices = torch.nn.functional.pad(indices, (0, pad), value=-1)
    m = z.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    total = ((z - m) / c["temperature"]).exp().sum(1, dtype=torch.float64)
    return values, indices.to(torch.int32), (m[:, 0].double() / c["temperature"] + total.log()).float()


def _plain_distill(s):
    c = s["case"]
    tau = c["temperature"]
    z = _chosen(s)
    n, vocab = z.shape
    valid = (s["t_indices"] >= 0) & (s["t_indices"] < vocab) & (s["t_values"] > -math.inf)
    at = torch.where(valid, s["t_indices"], 0).long()
    t = torch.where(valid, s["t_values"], -math.inf).double() / tau
    if s["t_lse"] is None:
        t = t - torch.where(valid.any(1, keepdim=True), t.amax(1, keepdim=True), 0.0)
        log_p = t - t.exp().sum(1, keepdim=True).log()
    else:
        log_p = t - s["t_lse"].double()[:, None]
    p = torch.where(valid, log_p.exp(), 0.0)
    some = valid.any(1)
    m = z.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = ((z - m) / tau).exp()
    total = e.sum(1, dtype=torch.float64)
    mark = torch.zeros((n, vocab + 1), dtype=torch.bool, device=z.device)
    mark.scatter_(1, torch.where(valid, at, vocab), True)
    inside = mark[:, :vocab]
    rest = torch.where(inside, 0.0, e).sum(1, dtype=torch.float64)
    r = (1.0 - p.sum(1)).clamp(min=0.0) if s["t_lse"] is not None else torch.zeros(n, dtype=torch.float64, device=z.device)
    r = torch.where(some & (rest > 0), r, 0.0)
    log_q = (z.gather(1, at) - m).double() / tau - total.log()[:, None]
    kd = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
    kd = kd + torch.where(r > 0, r * (r.log() - (rest / total).log()), 0.0)
    live = total != 0
    loss = KD_WEIGHT * tau * tau * torch.where(some, kd, 0.0)
    has = None
    if s["labels"] is not None:
        label = s["labels"].long()
        has = (label >= 0) & (label < vocab)
        label = torch.where(has, label, 0)
        e1 = e if tau == 1.0 else (z - m).exp()
        total1 = e1.sum(1, dtype=torch.float64)
        ce = total1.log() - (z.gather(1, label[:, None]) - m)[:, 0].double()
        loss = loss + CE_WEIGHT * torch.where(has, ce, 0.0)
    loss = torch.where(live, loss, 0.0).float()
    if c["kind"] == "loss":
        return loss
    scale = torch.where(live, s["dloss"].double(), 0.0)
    kd_scale = torch.where(some, scale, 0.0) * KD_WEIGHT * tau
    mass = p.sum(1) + r
    in_coef = kd_scale * mass / total
    out_coef = in_coef - torch.where(r > 0, kd_scale * r / rest, 0.0)
    grad = e * torch.where(inside, in_coef.float()[:, None], out_coef.float()[:, None])
    grad = grad.scatter_add_(1, at, (-(kd_scale[:, None] * p)).float())
    if has is not None:
        ce_scale = torch.where(has, scale, 0.0) * CE_WEIGHT
        grad += e1 * (ce_scale / total1).float()[:, None]
        grad.scatter_add_(1, label[:, None], (-ce_scale).float()[:, None])
    grad = torch.where(live[:, None], grad, 0.0).to(s["logits"].dtype)
    if s["rows"] is None:
        return loss, grad
    whole = torch.zeros_like(s["logits"])
    whole[s["rows"].long()] = grad
    return loss, whole


# ----------------------------------------------------------------------------------------------------------------------
# in 64 bits
# ----------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    z = s["logits"] if s["rows"] is None else s["logits"].index_select(0, s["rows"].long())
    if case["kind"] == "sample":
        one = lambda name, r, off: off if s[name] is None else s[name][r].item()  # noqa: E731
        logprob = [_exact_sample(z[r].double(), s["u"][r].item(), s["temperature"][r].item(), one("top_k", r, 0), one("top_p", r, 1.0),
                                 one("min_p", r, 0.0)) for r in range(case["n"])]
        return None, torch.tensor(logprob, dtype=torch.float64)
    step = max(1, (1 << 26) // case["vocab"])
    parts = [range(lo, min(case["n"], lo + step)) for lo in range(0, case["n"], step)]
    if case["kind"] == "top":
        values, lse = [], []
        for part in parts:
            x = z[part.start:part.stop].double()
            values.append(x.sort(dim=1, descending=True).values[:, :case["k"]])
            lse.append(torch.logsumexp(x / case["temperature"], 1))
        return torch.cat(values), None, torch.cat(lse)
    loss, grad = [], []
    for part in parts:
        cut = slice(part.start, part.stop)
        one, two = _exact_distill(case, z[cut].double(), s["t_values"][cut].double(), s["t_indices"][cut].long(),
                                  None if s["t_lse"] is None else s["t_lse"][cut].double(),
                                  None if s["labels"] is None else s["labels"][cut].long(), s["dloss"][cut].double())
        loss.append(one)
        grad.append(two)
    if case["kind"] == "loss":
        return torch.cat(loss)
    grad = torch.cat(grad)
    if s["rows"] is None:
        return torch.cat(loss), grad
    whole = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
    whole[s["rows"].long()] = grad
    return torch.cat(loss), whole


def _exact_sample(z, u, temperature, top_k, top_p, min_p):
    """log of the probability with which the row's token is drawn."""
    if not temperature > 0:
        return 0.0
    order = torch.argsort(-z, stable=True)
    finite = int((z > -math.inf).sum())
    order = order[:min(top_k, finite) if top_k > 0 else finite]
    w = torch.exp((z[order] - z[order[0]]) / temperature)
    run_ = torch.cumsum(w, 0)
    count = len(w)
    if top_p < 1:
        before = torch.cat([run_.new_zeros(1), run_[:-1]])
        count = max(1, int((before < top_p * run_[-1]).sum()))
    if min_p > 0:
        count = min(count, int((w >= min(min_p, 1.0)).sum()))
    total = run_[count - 1]
    at = min(count - 1, int(torch.searchsorted(run_[:count], u * total, right=True)))
    return float(torch.log(w[at] / total))


def _exact_distill(case, z, t, at, t_lse, label, dloss):
    tau, vocab = case["temperature"], z.shape[1]
    valid = at >= 0
    some = valid.any(1)
    t = (t / tau).masked_fill(~valid, -math.inf)
    p = torch.exp(t - (torch.logsumexp(t, 1) if t_lse is None else t_lse)[:, None]).masked_fill(~some[:, None], 0.0)
    teacher = torch.zeros_like(z).scatter_add_(1, at.clamp(min=0), p)
    top = torch.zeros_like(z).scatter_add_(1, at.clamp(min=0), valid.double()) > 0
    log_q = torch.log_softmax(z / tau, 1)
    loss = torch.special.xlogy(p, p).sum(1) - (teacher * log_q).sum(1)
    grad = torch.exp(log_q) * teacher.sum(1)[:, None] - teacher
    if t_lse is not None:
        r = (1.0 - p.sum(1)).clamp(min=0.0) * some
        log_rest = torch.logsumexp(log_q.masked_fill(top, -math.inf), 1)
        loss += torch.special.xlogy(r, r) - r * log_rest
        grad += r[:, None] * (torch.exp(log_q) - torch.exp(log_q - log_rest[:, None]).masked_fill(top, 0.0))
    loss, grad = KD_WEIGHT * tau * tau * loss, KD_WEIGHT * tau * grad
    if label is not None:
        has = (label >= 0).double()
        label = label.clamp(min=0)[:, None]
        log_s = torch.log_softmax(z, 1)
        loss -= CE_WEIGHT * has * log_s.gather(1, label)[:, 0]
        grad += CE_WEIGHT * has[:, None] * torch.exp(log_s).scatter_add_(1, label, torch.full_like(log_s[:, :1], -1.0))
    return loss, grad * dloss[:, None]
