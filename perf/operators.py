"""The float work on both ends of an exchange of answers, as cases that can be timed.

The nodes of a neighbourhood answer the same examples: for every example (a row of logits) the log-probabilities
of k classes are encoded, encrypted, summed and decrypted like any other vector, and every node moves its model
towards the mean.  Five kinds of pass:

``top``       the k most probable classes of every row and their log-probabilities: the positions that are exchanged
``at``        a member's log-probabilities at given positions: the vector that it encodes
``loss``      distillation loss of every row against the neighbourhood's mean answer
``step``      the loss and, in the same pass, its gradient with respect to the logits
``backward``  the gradient alone, from the row statistics that an earlier ``loss`` returned

Numbers of classes run from the ten of the repository's image classifiers to vocabularies of language models.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# ---- cases ------------------------------------------------------------------------------------------------

def listed():
    return [
        # a mini-batch of 256 of the repository's ten-class classifiers: all classes are exchanged
        {"name": "step_10", "kind": "step", "rows": 256, "classes": 10, "pad": 0, "k": 10, "dtype": "f32", "members": 4,
         "temperature": 1.0, "masked": False},
        # an ordinary training step of a small language model; the end of the batch is padding
        {"name": "step_32768", "kind": "step", "rows": 2048, "classes": 32768, "pad": 0, "k": 64, "dtype": "bf16",
         "members": 5, "temperature": 2.0, "masked": True},
        # a large batch with a large vocabulary
        {"name": "step_131072", "kind": "step", "rows": 4096, "classes": 131072, "pad": 0, "k": 128, "dtype": "bf16",
         "members": 8, "temperature": 1.0, "masked": False},
        # the last few examples of an exchange, logits in 32 bits
        {"name": "step_few_rows", "kind": "step", "rows": 16, "classes": 131072, "pad": 0, "k": 64, "dtype": "f32",
         "members": 7, "temperature": 1.5, "masked": True},
        # evaluation of a held-out set: an odd vocabulary, so that rows start at any multiple of two bytes
        {"name": "loss_50001", "kind": "loss", "rows": 777, "classes": 50001, "pad": 0, "k": 33, "dtype": "f16",
         "members": 7, "temperature": 1.0, "masked": True},
        # backward pass of its own, a thousand image classes
        {"name": "backward_1000", "kind": "backward", "rows": 16384, "classes": 1000, "pad": 24, "k": 16, "dtype": "bf16",
         "members": 5, "temperature": 4.0, "masked": True},
        # backward pass of its own, long rows of 32 bits at odd addresses
        {"name": "backward_65537", "kind": "backward", "rows": 512, "classes": 65537, "pad": 0, "k": 250, "dtype": "f32",
         "members": 8, "temperature": 1.0, "masked": False},
        # the positions of a large exchange
        {"name": "top_131072", "kind": "top", "rows": 4096, "classes": 131072, "pad": 0, "k": 64, "dtype": "bf16"},
        # one example by itself
        {"name": "top_one_row", "kind": "top", "rows": 1, "classes": 50001, "pad": 0, "k": 16, "dtype": "f32"},
        # very many short rows
        {"name": "top_100", "kind": "top", "rows": 65536, "classes": 100, "pad": 4, "k": 5, "dtype": "f16"},
        # a member's answers for an ordinary batch, and for the ten-class classifiers
        {"name": "at_32768", "kind": "at", "rows": 2048, "classes": 32768, "pad": 0, "k": 64, "dtype": "bf16"},
        {"name": "at_10", "kind": "at", "rows": 256, "classes": 10, "pad": 0, "k": 10, "dtype": "f32"},
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    case = {"kind": rng.choice(["top", "at", "loss", "step", "step", "backward"]), "classes": _spread(rng, 2, 131072),
            "k": _spread(rng, 1, 256), "dtype": rng.choice(["f32", "f16", "bf16"]),
            "pad": rng.choice([0, 0, rng.randint(1, 40)])}
    case["rows"] = _spread(rng, 1, min(65536, (1 << 27) // case["classes"]))
    if case["kind"] in ("loss", "step", "backward"):
        case["members"] = rng.randint(2, 32)
        case["temperature"] = rng.choice([1.0, 1.5, 2.0, 4.0])
        case["masked"] = rng.random() < 0.5
    return case


def _live_rows(case):
    """Rows that are no padding of the batch: a masked case ends with padding."""
    return case["rows"] - (case["rows"] // 16 if case.get("masked") else 0)


def work(case):
    rows, live, V, k = case["rows"], _live_rows(case), case["classes"], case["k"]
    word = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("top", "at"):
        return {"bytes": rows * V * word + 8 * rows * k, "flops": 4 * rows * V}
    read = live * V * word + 8 * live * k + 4 * rows
    if case["kind"] == "loss":
        return {"bytes": read + 8 * rows, "flops": 4 * live * V + 12 * live * k}
    return {"bytes": read + rows * V * word + 8 * rows, "flops": (8 if case["kind"] == "step" else 5) * live * V + 12 * live * k}


# ---- what a program holds before the pass -----------------------------------------------------------------

def _logits(case, gen):
    """[rows][classes + pad]: a few classes far above the rest, as models answer; what pads a row is no number."""
    V, stride = case["classes"], case["classes"] + case["pad"]
    bias = -1.5 * torch.log1p(torch.randperm(V, generator=gen, device=DEV).float())
    buf = torch.empty((case["rows"], stride), dtype=DTYPES[case["dtype"]], device=DEV)
    part = max(1, (1 << 26) // stride)
    for r in range(0, case["rows"], part):
        rows = min(part, case["rows"] - r)
        z = torch.randn((rows, V), generator=gen, device=DEV)
        shift = torch.randn((rows, 1), generator=gen, device=DEV)
        buf[r:r + rows, :V] = z * 2 + bias + shift
        buf[r:r + rows, V:] = float("nan")
    return buf


def _positions(case, gen):
    """k different classes of every row, in no order; slots that a row cannot fill hold -1."""
    rows, V, k = case["rows"], case["classes"], case["k"]
    used = min(k, V)
    at = torch.arange(used, device=DEV)
    lo, hi = at * V // used, (at + 1) * V // used
    u = torch.rand((rows, used), generator=gen, device=DEV)
    index = torch.minimum(lo + (u * (hi - lo)).long(), hi - 1)
    index = index[:, torch.randperm(used, generator=gen, device=DEV)]
    full = torch.full((rows, k), -1, dtype=torch.int32, device=DEV)
    full[:, :used] = index.int()
    return full


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rows, V, k, kind = case["rows"], case["classes"], case["k"], case["kind"]
    s = {"case": case, "logits": _logits(case, gen)}
    if kind != "top":
        s["index"] = _positions(case, gen)
    if kind in ("loss", "step", "backward"):
        K = case["members"]
        # decoded sums are multiples of the fixed point's last bit
        s["sum"] = -torch.round(torch.rand((rows, k), generator=gen, device=DEV) * 8 * K * 256) / 256
        live = _live_rows(case)
        s["weight"] = torch.zeros(rows, device=DEV)        # gradients of 16 bits and five exponent bits are scaled up
        s["weight"][:live] = case["temperature"] ** 2 / live * (1024 if case["dtype"] == "f16" else 1)
        if case["masked"]:                                 # rows of fewer filled slots, among them none at all
            filled = torch.randint(0, k + 1, (rows, 1), generator=gen, device=DEV)
            short = torch.rand((rows, 1), generator=gen, device=DEV) < 0.25
            s["index"][short & (torch.arange(k, device=DEV) >= filled)] = -1
    if kind == "backward":
        s["lse"] = torch.empty(rows, device=DEV)
        part = max(1, (1 << 25) // V)
        for r in range(0, rows, part):
            s["lse"][r:r + part] = torch.logsumexp(s["logits"][r:r + part, :V].double() / case["temperature"], 1).float()
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    from paper_2207_04604_amd import binding
    case = s["case"]
    rows, V, k = case["rows"], case["classes"], case["k"]
    dtype = {"f32": binding.F32, "f16": binding.F16, "bf16": binding.BF16}[case["dtype"]]
    s["z"] = binding.make_logits(s["logits"], dtype, rows, V, row_stride=V + case["pad"])
    s["bytes"] = binding.logits_scratch_bytes(s["z"], k)
    s["scratch"] = torch.empty(s["bytes"] // 8, dtype=torch.int64, device=DEV)
    if case["kind"] == "top":
        s["index"] = torch.empty((rows, k), dtype=torch.int32, device=DEV)
    if case["kind"] in ("top", "at"):
        s["logprobs"] = torch.empty((rows, k), device=DEV)
        return
    s["teacher"] = binding.make_teacher(s["index"], s["sum"], k, case["members"], temperature=case["temperature"],
                                        weight=s["weight"])
    if case["kind"] != "backward":
        s["loss"], s["lse"] = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    if case["kind"] != "loss":
        s["grad"] = torch.empty((rows, V), dtype=DTYPES[case["dtype"]], device=DEV)


# ---- one pass ---------------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2207_04604_amd import binding
    kind, V, k = s["case"]["kind"], s["case"]["classes"], s["case"]["k"]
    stream = torch.cuda.current_stream().cuda_stream
    if kind == "top":
        binding.top_logprobs(s["z"], k, s["index"], s["logprobs"], s["scratch"], s["bytes"], stream)
        return {"index": s["index"], "logprobs": s["logprobs"]}
    if kind == "at":
        binding.logprobs_at(s["z"], s["index"], k, s["logprobs"], s["scratch"], s["bytes"], stream)
        return {"logprobs": s["logprobs"]}
    if kind == "loss":
        binding.distill(s["z"], s["teacher"], s["loss"], s["lse"], None, 0, s["scratch"], s["bytes"], stream)
        return {"loss": s["loss"], "lse": s["lse"]}
    if kind == "step":
        binding.distill(s["z"], s["teacher"], s["loss"], s["lse"], s["grad"], V, s["scratch"], s["bytes"], stream)
        return {"loss": s["loss"], "lse": s["lse"], "grad": s["grad"]}
    binding.distill_backward(s["z"], s["teacher"], s["lse"], s["grad"], V, stream)
    return {"grad": s["grad"]}


def _run_plain(s):
    case = s["case"]
    kind, V, k, rows = case["kind"], case["classes"], case["k"], case["rows"]
    z = s["logits"][:, :V].float()
    if kind == "top":
        # the order of the values as whole numbers, then the lower class first: no two keys are alike
        bits = (z + 0.0).view(torch.int32)
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = (bits << 32) + (V - 1 - torch.arange(V, device=DEV))
        best = torch.topk(key, min(k, V), dim=1).values
        index = V - 1 - (best & 0xFFFFFFFF)
        logprobs = torch.gather(z, 1, index) - _lse(z)
        full = torch.full((rows, k), -1, dtype=torch.int32, device=DEV)
        out = torch.zeros((rows, k), device=DEV)
        full[:, :index.shape[1]], out[:, :index.shape[1]] = index.int(), logprobs
        return {"index": full, "logprobs": out}
    filled = s["index"] >= 0
    index = s["index"].clamp(min=0).long()
    if kind == "at":
        return {"logprobs": torch.where(filled, torch.gather(z, 1, index) - _lse(z), 0.0)}
    T = case["temperature"]
    z = z / T
    lse = _lse(z) if kind != "backward" else s["lse"][:, None]
    t = torch.where(filled, s["sum"] / case["members"] / T, -math.inf)
    some = filled.any(1, keepdim=True)
    p = torch.exp(t - torch.where(some, t.amax(1, keepdim=True), 0.0))
    total = torch.where(some, p.sum(1, keepdim=True), 1.0)
    p = p / total
    weight = torch.where(some, s["weight"][:, None], 0.0)          # rows of weight 0 and of no filled slot: all 0
    out = {}
    if kind != "backward":
        logp = torch.where(filled, t - t.amax(1, keepdim=True) - torch.log(total), 0.0)
        out["loss"] = (weight * (p * (logp - (torch.gather(z, 1, index) - lse))).sum(1, keepdim=True))[:, 0]
        out["lse"] = torch.where(weight != 0, lse, 0.0)[:, 0]
    if kind != "loss":
        grad = torch.exp(z - lse)
        grad.scatter_add_(1, index, -p)
        out["grad"] = (grad * (weight / T)).to(s["logits"].dtype)
    return out


def _lse(z):
    top = z.amax(1, keepdim=True)
    return top + torch.log(torch.exp(z - top).sum(1, keepdim=True))


# ---- the definition in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    V, k, rows = case["classes"], case["k"], case["rows"]
    parts = []
    step = max(1, (1 << 26) // V)
    for lo in range(0, rows, step):
        z = s["logits"][lo:lo + step, :V].double()
        if case["kind"] == "top":
            order = torch.sort(z, dim=1, descending=True, stable=True)
            n = min(k, V)
            index = torch.full((z.shape[0], k), -1, dtype=torch.int32, device=DEV)
            logprobs = torch.zeros((z.shape[0], k), dtype=torch.float64, device=DEV)
            index[:, :n] = order.indices[:, :n].int()
            logprobs[:, :n] = order.values[:, :n] - torch.logsumexp(z, 1, keepdim=True)
            parts.append({"index": index, "logprobs": logprobs})
            continue
        slots = s["index"][lo:lo + step]
        full = torch.cat([z, torch.zeros_like(z[:, :1])], 1)          # column V stands for an empty slot
        column = torch.where(slots < 0, V, slots.long())
        if case["kind"] == "at":
            got = torch.log_softmax(z, 1)
            got = torch.cat([got, torch.zeros_like(z[:, :1])], 1)
            parts.append({"logprobs": torch.gather(got, 1, column)})
            continue
        T = case["temperature"]
        # the lse of a backward pass is an input, given in 32 bits
        lse = torch.logsumexp(z / T, 1) if case["kind"] != "backward" else s["lse"][lo:lo + step].double()
        answer = s["sum"][lo:lo + step].double() / (case["members"] * T)
        answer[slots < 0] = -math.inf
        logp = torch.log_softmax(answer, 1)
        p = torch.nan_to_num(torch.exp(logp), nan=0.0)
        weight = s["weight"][lo:lo + step].double() * (slots >= 0).any(1)
        part = {}
        if case["kind"] != "backward":
            student = torch.gather(full, 1, column) / T - lse[:, None]
            part["loss"] = weight * torch.where(p > 0, p * (logp - student), 0.0).sum(1)
            part["lse"] = lse * (weight != 0)
        if case["kind"] != "loss":
            teacher = torch.zeros_like(full).scatter_add_(1, column, p)[:, :V]
            part["grad"] = (torch.exp(z / T - lse[:, None]) - teacher) * (weight / T)[:, None]
        parts.append(part)
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
