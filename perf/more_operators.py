"""The work of the token operators, as a list of cases that can be timed and compared.

Three operators at the two ends of a token student, in their plain form (elementary torch operations in 32 bits) and through the
framework's entry points:

  op "embed"    lookup of tokens in a table, times a scale.  mode "forward": the lookup; mode "train": lookup, and the table's gradient
  op "head"     softmax cross entropy of h W^T against labels, over the whole vocabulary.  mode "score": losses and log-sums only;
                mode "train": losses and the gradients of h and W
  op "distill"  distillation from a teacher's top logits: T^2 KL(softmax of the teacher's top / T, softmax of the student's logits / T).
                mode "score": losses only; mode "train": losses and the gradient of the student's logits

rows         tokens (embed), rows of h (head), rows of logits (distill)
vocab, d     size of the vocabulary, width of the table (embed) and of h (head)
dtype        type of the table and activations (embed), of h and W (head), of the logits (distill)
top          distill: how many of the teacher's logits are known;  teacher: their type
index        type of tokens, labels or places ("i32", "i64")
ragged       embed: some tokens are padding; head: some labels are to be ignored; distill: rows know fewer of the teacher's logits, some none
accumulate   embed, train: the gradient is added to what the table's gradient holds, as with a table that is the head's weight too

Tokens and labels are distributed as words are, most of them few.  Sizes are generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32, "i64": torch.int64}
NONE = float("-inf")


# ------------------------------------------------------------------------------------------------------------- the cases
def _embed(name, mode, rows, vocab, d, dtype="bf16", index="i64", ragged=False, accumulate=False):
    return {"name": name, "op": "embed", "mode": mode, "rows": rows, "vocab": vocab, "d": d, "dtype": dtype, "index": index, "ragged": ragged,
            "accumulate": accumulate}


def _head(name, mode, rows, vocab, d, dtype="bf16", index="i64", ragged=False):
    return {"name": name, "op": "head", "mode": mode, "rows": rows, "vocab": vocab, "d": d, "dtype": dtype, "index": index, "ragged": ragged}


def _distill(name, mode, rows, vocab, top, dtype="bf16", teacher="bf16", index="i64", ragged=False):
    return {"name": name, "op": "distill", "mode": mode, "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "teacher": teacher, "index": index,
            "ragged": ragged, "temperature": 2.0}


def listed():
    return [
        # serving: a token for each of 64 sequences; latency
        _embed("embed_token", "forward", 64, 32768, 2048),
        # the usual training batch of a token student, both directions
        _embed("embed_train", "train", 32768, 65536, 2048),
        # the largest table and batch; the gradient goes on top of the head's, whose weight the table is
        _embed("embed_train_tied", "train", 65536, 131072, 4096, index="i32", accumulate=True),
        # a small odd vocabulary and width in 32 bits, padded texts: every row of the table has many tokens
        _embed("embed_train_odd_f32", "train", 5003, 777, 515, "f32", ragged=True),
        # serving: how likely the next token of each of 32 sequences is
        _head("head_score_token", "score", 32, 65536, 2048),
        # a small model in the framework's own 32 bits, odd sizes, some labels ignored: latency of a training step
        _head("head_train_odd_f32", "train", 500, 1013, 515, "f32", ragged=True),
        # the usual training batch of a token student
        _head("head_train", "train", 4096, 65536, 2048),
        # a large vocabulary under a wide model
        _head("head_train_large", "train", 8192, 131072, 4096, index="i32", ragged=True),
        # the last batch of an epoch: few rows, few known logits; latency
        _distill("distill_train_small", "train", 48, 16384, 16),
        # the usual training batch of a student that learns from stored logits of its teacher
        _distill("distill_train", "train", 8192, 65536, 64),
        # 32 bits, an odd vocabulary, rows that know little or nothing of the teacher
        _distill("distill_train_odd_f32", "train", 1023, 50021, 20, "f32", "f32", "i32", ragged=True),
        # how far the student is from the teacher, on held-out text
        _distill("distill_score_f16", "score", 4095, 131071, 100, "f16", "f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _round(rng, n):
    """n, or as often a multiple of 64 near it."""
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


_MOST = {}


def draw(rng):
    """One more case: any operator, any mode, over the whole range of sizes."""
    if not _MOST:
        for c in listed():
            for k, v in work(c).items():
                _MOST[c["op"], k] = max(_MOST.get((c["op"], k), 0), v)
    while True:
        op, dtype, index, ragged = rng.choice(["embed", "head", "distill"]), rng.choice(["bf16", "bf16", "f32", "f16"]), rng.choice(["i32", "i64"]), rng.random() < 0.4
        if op == "embed":
            mode = rng.choice(["forward", "train", "train"])
            c = _embed("", mode, _log(rng, 1, 131072), _round(rng, _log(rng, 16, 262144)), _round(rng, _log(rng, 16, 8192)), dtype, index, ragged,
                       mode == "train" and rng.random() < 0.3)
        elif op == "head":
            c = _head("", rng.choice(["score", "train", "train"]), _log(rng, 1, 16384), _round(rng, _log(rng, 100, 262144)), _round(rng, _log(rng, 64, 8192)), dtype, index, ragged)
        else:
            c = _distill("", rng.choice(["score", "train", "train"]), _log(rng, 1, 16384), _round(rng, _log(rng, 100, 262144)), _log(rng, 1, 512), dtype,
                         rng.choice([dtype, "f32"]), index, ragged)
            c["top"], c["temperature"] = min(c["top"], c["vocab"]), rng.choice([1.0, 2.0, 4.0])
        del c["name"]
        if all(v <= _MOST[op, k] for k, v in work(c).items()):
            return c


def work(case):
    size, isize = (4 if case["dtype"] == "f32" else 2), (4 if case["index"] == "i32" else 8)
    n, v = case["rows"], case["vocab"]
    if case["op"] == "embed":
        d, known = case["d"], min(case["rows"], case["vocab"])      # rows of the table that occur: at most these
        if case["mode"] == "forward":
            return {"bytes": (n + known) * d * size + n * isize, "flops": n * d}
        # tokens, table -> y; later tokens, dy -> the table's gradient, or what of it occurs
        return {"bytes": (2 * n + known + (2 * known if case["accumulate"] else v)) * d * size + 2 * n * isize, "flops": 3 * n * d}
    if case["op"] == "head":
        d, train = case["d"], case["mode"] == "train"
        # a product for the logits, and one for each gradient
        return {"bytes": (2 if train else 1) * (n + v) * d * size + n * (isize + 12), "flops": (6 if train else 2) * n * v * d}
    teacher = 4 if case["teacher"] == "f32" else 2
    return {"bytes": (2 if case["mode"] == "train" else 1) * n * v * size + n * case["top"] * (teacher + isize) + 8 * n, "flops": 6 * n * v}


# ------------------------------------------------------------------------------------------------------------ the inputs
def _randn(gen, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


def _words(gen, n, vocab, dtype):
    """n tokens, token k about as often as 1 / (k + 1)."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp(0, vocab - 1).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": case, "stream": torch.cuda.current_stream()}
    n, v, dt, it = case["rows"], case["vocab"], TYPES[case["dtype"]], TYPES[case["index"]]
    if case["op"] in ("embed", "head"):
        d = case["d"]
        words = _words(gen, n, v, it)
        if case["ragged"]:
            words = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.15, torch.tensor(-100, device="cuda", dtype=it), words)
        st["weight"] = _randn(gen, v, d, scale=2.0 * d ** -0.5 if case["op"] == "head" else d ** -0.5, dtype=dt)
    if case["op"] == "embed":
        st["tokens"], st["scale"] = words, math.sqrt(d)
        st["y"] = torch.empty(n, d, device="cuda", dtype=dt)
        if case["mode"] == "train":
            st["dy"] = _randn(gen, n, d, dtype=dt)
            st["dweight"] = _randn(gen, v, d, dtype=dt) if case["accumulate"] else torch.empty(v, d, device="cuda", dtype=dt)
        return st
    if case["op"] == "head":
        st["h"], st["labels"] = _randn(gen, n, d, dtype=dt), words
        st["loss"], st["lse"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        if case["mode"] == "train":
            st["row_weight"] = (0.5 + torch.rand(n, generator=gen, device="cuda")) / n
            st["dh"], st["dweight"] = torch.empty_like(st["h"]), torch.empty_like(st["weight"])
        return st
    # the teacher's top logits lie where some of the student's are; the student is on its way to them
    top, tt = case["top"], TYPES[case["teacher"]]
    st["logits"] = _randn(gen, n, v, scale=2.0, dtype=dt)
    first = torch.randint(0, v, (n, 1), generator=gen, device="cuda")
    at = (first + torch.arange(top, device="cuda") * max(1, v // top)) % v          # all different
    st["teacher"] = (torch.sort(torch.randn(n, top, generator=gen, device="cuda") * 2.0 + 6.0, dim=1, descending=True).values).to(tt)
    st["logits"].scatter_add_(1, at, (0.5 * st["teacher"].float()).to(dt))
    if case["ragged"]:
        known = torch.randint(0, top + 1, (n, 1), generator=gen, device="cuda")
        known[0] = 0
        at = torch.where(torch.arange(top, device="cuda") < known, at, -1)
    st["at"] = at.to(it)
    st["loss"] = torch.empty(n, device="cuda")
    if case["mode"] == "train":
        st["row_weight"] = (0.5 + torch.rand(n, generator=gen, device="cuda")) / n
        st["dlogits"] = torch.empty_like(st["logits"])
    return st


# ------------------------------------------------------------------------------------------------------- the plain forms
def _plain_embed(st):
    case, w, tokens, scale = st["case"], st["weight"], st["tokens"], st["scale"]
    live = (tokens >= 0) & (tokens < case["vocab"])
    at = torch.where(live, tokens, 0).long()
    y = torch.where(live[:, None], w[at].float() * scale, 0.0).to(w.dtype)
    if case["mode"] == "forward":
        return {"y": y}
    total = torch.zeros(case["vocab"], case["d"], device="cuda")
    total.index_add_(0, at, torch.where(live[:, None], st["dy"].float(), 0.0))
    total = total * scale
    if not case["accumulate"]:
        return {"y": y, "dweight": total.to(w.dtype)}
    st["dweight"].copy_(st["dweight"].float() + total)
    return {"y": y, "dweight": st["dweight"]}


def _plain_head(st):
    case, labels = st["case"], st["labels"]
    h, w = st["h"].float(), st["weight"].float()
    live = (labels >= 0) & (labels < case["vocab"])
    at = torch.where(live, labels, 0).long()[:, None]
    z = torch.mm(h, w.t())
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    loss = torch.where(live, (lse - z.gather(1, at))[:, 0], 0.0)
    if case["mode"] == "score":
        return {"loss": loss, "lse": lse[:, 0]}
    g = torch.where(live, st["row_weight"], 0.0)[:, None]
    dz = e * (g / total)
    dz.scatter_add_(1, at, -g)
    return {"loss": loss, "lse": lse[:, 0], "dh": torch.mm(dz, w).to(st["h"].dtype), "dweight": torch.mm(dz.t(), h).to(st["weight"].dtype)}


def _plain_distill(st):
    case, at, temperature = st["case"], st["at"].long(), st["case"]["temperature"]
    t = st["teacher"].float()
    known = (at >= 0) & (at < case["vocab"]) & (t > NONE)
    some = known.any(1, keepdim=True)
    at = torch.where(known, at, 0)
    t = torch.where(known, t * (1.0 / temperature), NONE)
    t = t - torch.where(some, t.amax(1, keepdim=True), 0.0)
    q = torch.exp(t)
    share = torch.where(some, q.sum(1, keepdim=True), 1.0)
    q = q / share
    z = st["logits"].float() * (1.0 / temperature)
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    far = t - torch.log(share) - z.gather(1, at) + top + torch.log(total)
    loss = torch.where(q > 0, q * far, 0.0).sum(1) * temperature ** 2
    if case["mode"] == "score":
        return {"loss": loss}
    g = torch.where(some, st["row_weight"][:, None] * temperature, 0.0)
    dz = e * (g / total)
    dz.scatter_add_(1, at, -g * q)
    return {"loss": loss, "dlogits": dz.to(st["logits"].dtype)}


# ------------------------------------------------------------------------------------------- through the framework's calls
def _own_embed(st):
    case = st["case"]
    if "pb" not in st:
        from paper_2012_03096_amd import binding
        st["pb"] = binding
        if case["mode"] == "train":
            st["workspace"] = torch.empty(binding.embed_workspace_bytes(case["rows"], case["vocab"], case["d"]), device="cuda", dtype=torch.uint8)
    pb, stream = st["pb"], st["stream"]
    pb.embed_forward(st["tokens"], st["weight"], st["y"], scale=st["scale"], stream=stream)
    if case["mode"] == "forward":
        return {"y": st["y"]}
    pb.embed_backward(st["tokens"], st["dy"], st["dweight"], st["workspace"], scale=st["scale"], accumulate=case["accumulate"], stream=stream)
    return {"y": st["y"], "dweight": st["dweight"]}


def _own_head(st):
    case, train = st["case"], st["case"]["mode"] == "train"
    if "pb" not in st:
        from paper_2012_03096_amd import binding
        st["pb"] = binding
        st["workspace"] = torch.empty(binding.head_loss_workspace_bytes(case["rows"], case["vocab"], case["d"], TYPES[case["dtype"]], gradients=train),
                                      device="cuda", dtype=torch.uint8)
    pb, stream = st["pb"], st["stream"]
    if not train:
        pb.head_loss(st["h"], st["weight"], st["labels"], st["loss"], st["workspace"], lse=st["lse"], stream=stream)
        return {"loss": st["loss"], "lse": st["lse"]}
    pb.head_loss(st["h"], st["weight"], st["labels"], st["loss"], st["workspace"], lse=st["lse"], row_weight=st["row_weight"], dh=st["dh"],
                 dweight=st["dweight"], stream=stream)
    return {"loss": st["loss"], "lse": st["lse"], "dh": st["dh"], "dweight": st["dweight"]}


def _own_distill(st):
    case = st["case"]
    if "pb" not in st:
        from paper_2012_03096_amd import binding
        st["pb"] = binding
    pb, stream = st["pb"], st["stream"]
    if case["mode"] == "score":
        pb.topk_distill(st["logits"], st["teacher"], st["at"], st["loss"], temperature=case["temperature"], stream=stream)
        return {"loss": st["loss"]}
    pb.topk_distill(st["logits"], st["teacher"], st["at"], st["loss"], temperature=case["temperature"], row_weight=st["row_weight"], dlogits=st["dlogits"],
                    stream=stream)
    return {"loss": st["loss"], "dlogits": st["dlogits"]}


def run(st):
    op = st["case"]["op"]
    if own:
        return (_own_embed if op == "embed" else _own_head if op == "head" else _own_distill)(st)
    return (_plain_embed if op == "embed" else _plain_head if op == "head" else _plain_distill)(st)


# ------------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return (_exact_embed if case["op"] == "embed" else _exact_head if case["op"] == "head" else _exact_distill)(case, st)


def _exact_embed(case, st):
    v, w = case["vocab"], st["weight"]
    tokens = st["tokens"].long()
    live = ((tokens >= 0) & (tokens < v)).nonzero()[:, 0]
    y = torch.zeros(case["rows"], case["d"], dtype=torch.float64, device="cuda")
    y[live] = torch.index_select(w, 0, tokens[live]).double() * st["scale"]
    if case["mode"] == "forward":
        return {"y": y}
    # the rows of dy in the order of their tokens; a token's sum is the sum of a range of them
    order = live[torch.argsort(tokens[live], stable=True)]
    counts = torch.bincount(tokens[live], minlength=v)
    parts = []
    for i in range(0, case["d"], 1024):                         # a range of columns at a time
        rows = st["dy"][:, i:i + 1024][order].double()
        parts.append(torch.segment_reduce(rows, "sum", lengths=counts, axis=0, unsafe=True, initial=0.0))
    dw = torch.cat(parts, 1) * st["scale"]
    return {"y": y, "dweight": dw + st["dweight"].double() if case["accumulate"] else dw}


def _exact_head(case, st):
    n, v, train = case["rows"], case["vocab"], case["mode"] == "train"
    w, labels = st["weight"].double(), st["labels"].tolist()
    step = max(1, (1 << 27) // v)                               # a range of rows at a time
    loss, lse, dh = [], [], []
    dw = torch.zeros_like(w) if train else None
    for i in range(0, n, step):
        h = st["h"][i:i + step].double()
        logits = torch.mm(h, w.t().contiguous()) if n < 64 else h @ w.t()
        norm = torch.logsumexp(logits, 1)
        lse.append(norm)
        rows = [r for r in range(h.shape[0]) if 0 <= labels[i + r] < v]
        cols = [labels[i + r] for r in rows]
        part = torch.zeros_like(norm)
        part[rows] = norm[rows] - logits[rows, cols]
        loss.append(part)
        if train:
            p = torch.softmax(logits, 1)
            del logits
            p[rows, cols] -= 1.0
            g = torch.zeros_like(norm)
            g[rows] = st["row_weight"][i:i + step].double()[rows]
            p *= g[:, None]
            dh.append(p @ w)
            dw += p.t() @ h
    out = {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    return {**out, "dh": torch.cat(dh), "dweight": dw} if train else out


def _exact_distill(case, st):
    n, v, temperature, train = case["rows"], case["vocab"], case["temperature"], case["mode"] == "train"
    step = max(1, (1 << 27) // v)                               # a range of rows at a time
    loss, dz = [], []
    for i in range(0, n, step):
        z = torch.log_softmax(st["logits"][i:i + step].double() / temperature, 1)
        # the teacher's distribution, written out over the whole vocabulary
        at, t = st["at"][i:i + step].long(), st["teacher"][i:i + step].double()
        place = torch.where((at >= 0) & (at < v), at, v)
        full = torch.full((z.shape[0], v + 1), NONE, dtype=torch.float64, device="cuda").scatter_(1, place, t)[:, :v]
        some = (full > NONE).any(1)
        log_q = torch.log_softmax(full / temperature, 1)
        q = torch.where(some[:, None], torch.exp(log_q), 0.0)
        loss.append(torch.where(q > 0, q * (log_q - z), 0.0).sum(1) * temperature ** 2)
        if train:
            g = torch.where(some, st["row_weight"][i:i + step].double(), 0.0) * temperature
            dz.append((torch.exp(z) - q) * g[:, None])
    return {"loss": torch.cat(loss), "dlogits": torch.cat(dz)} if train else {"loss": torch.cat(loss)}
