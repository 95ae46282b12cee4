"""Timed cases of the operators on token ids, through the Python entry points.

They lie at both ends of the policy that the trainer's operators learn from.  Each case is one of four things:

``embed``       the table's rows of the tokens that go in, scaled (``sr_embed_tokens``).
``embed_grad``  the table's gradient, every row of it (``sr_embed_tokens_backward``).
``adjust``      the logits that come out, adjusted by what the sampler was set to: penalties for tokens that were seen before, biases,
                and the mask of the tokens that a grammar or an environment allows (``sr_adjust_logits``).  In the form ``step`` every row
                is one rollout's next token with a history of its own; in the form ``rollouts`` rows are all tokens of whole
                rollouts, each seeing the prompt and the tokens before it: the distribution that the policy's loss has to be taken of.
``adjust_grad`` its gradient (``sr_adjust_logits_backward``).

Vocabularies are those of the repository's workloads (4096 actions, 151 936 tokens) or generic, and rollouts have the lengths of its
token-level workload.  Tokens are drawn as in text: the logarithm of an id is uniform, so that a few are taken thousands of times
and most never.
"""
import math

import numpy as np
import torch

own = False             # set from outside: the plain forms, or the framework's entry points

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
MOST_LOGITS = {"adjust": 4096 * 151936 * 2, "adjust_grad": 2048 * 151936 * 2}     # bytes of logits
MOST_TABLE = 151936 * 2048 * 2                                                    # bytes of a table
MOST_OUT = 65536 * 2048 * 2                                                       # bytes of embedded tokens
ROWS_AT_ONCE = 512      # of logits in the plain forms


def listed():
    return [
        # the eight rollouts of one group choose their next token; the sampler's three penalties, no grammar
        {"name": "adjust-step", "kind": "adjust", "form": "step", "T": 8, "V": 151936, "pad": 0, "dtype": "bf16", "prompt": 512, "longest": 1024, "penalties": "rpf", "biases": 0, "masks": 0},
        # all rollouts of 64 groups, each with its settings, a few hundred biases and the state of its grammar
        {"name": "adjust-rollouts-live", "kind": "adjust", "form": "step", "T": 512, "V": 151936, "pad": 0, "dtype": "bf16", "prompt": 512, "longest": 1024, "penalties": "rpf", "biases": 300, "masks": 64},
        # an odd vocabulary in a padded buffer
        {"name": "adjust-odd", "kind": "adjust", "form": "rollouts", "T": 601, "V": 50021, "pad": 3, "dtype": "f16", "prompt": 99, "longest": 75, "penalties": "rf", "biases": 17, "masks": 5},
        # a chunk of rollouts that were sampled with penalties, as the trainer scores them
        {"name": "adjust-rollouts", "kind": "adjust", "form": "rollouts", "T": 4096, "V": 151936, "pad": 0, "dtype": "bf16", "prompt": 512, "longest": 640, "penalties": "rp", "biases": 0, "masks": 0},
        # action-level policy head: what the environment does not allow has no gradient
        {"name": "adjust-grad-actions", "kind": "adjust_grad", "form": "rollouts", "T": 1200, "V": 4096, "pad": 0, "dtype": "f32", "prompt": 0, "longest": 30, "penalties": "r", "biases": 0, "masks": 240},
        # a chunk of rollouts that were sampled with penalties and a grammar
        {"name": "adjust-grad-rollouts", "kind": "adjust_grad", "form": "rollouts", "T": 2048, "V": 151936, "pad": 0, "dtype": "bf16", "prompt": 512, "longest": 640, "penalties": "r", "biases": 0, "masks": 64},
        # the last tokens of the eight rollouts of one group
        {"name": "embed-step", "kind": "embed", "T": 8, "V": 151936, "D": 2048, "dtype": "bf16", "table": "bf16", "scaled": False, "padding": 0.0},
        # a chunk of rollouts
        {"name": "embed-rollouts", "kind": "embed", "T": 65536, "V": 151936, "D": 2048, "dtype": "bf16", "table": "bf16", "scaled": True, "padding": 0.0},
        # an odd width, a quarter of a padded batch, a table held in 32 bits
        {"name": "embed-odd", "kind": "embed", "T": 5003, "V": 50021, "D": 1001, "dtype": "f16", "table": "f32", "scaled": True, "padding": 0.25},
        # the paper's iteration at action level
        {"name": "embed-grad-actions", "kind": "embed_grad", "T": 1200, "V": 4096, "D": 256, "dtype": "f32", "table": "f32", "scaled": False, "padding": 0.0},
        # gradients kept in 32 bits, a quarter of a padded batch
        {"name": "embed-grad-wide", "kind": "embed_grad", "T": 8192, "V": 50021, "D": 1000, "dtype": "bf16", "table": "f32", "scaled": True, "padding": 0.25},
        # a chunk of rollouts
        {"name": "embed-grad-rollouts", "kind": "embed_grad", "T": 65536, "V": 151936, "D": 2048, "dtype": "bf16", "table": "bf16", "scaled": True, "padding": 0.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["adjust", "adjust", "adjust_grad", "embed", "embed_grad"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind in ("embed", "embed_grad"):
        table = rng.choice([dtype, dtype, "f32"])
        V = rng.choice([151936, 4096, _log_int(rng, 500, 151936), _log_int(rng, 500, 151936) | 1])
        D = rng.choice([2048, _log_int(rng, 64, 4096), 64 * rng.randint(1, 64)])
        D = max(32, min(D, MOST_TABLE // (V * BYTES[table])))
        T = _log_int(rng, 1 if kind == "embed" else 32, max(64, min(1 << 17, MOST_OUT // (D * BYTES[dtype]))))
        return {"kind": kind, "T": T, "V": V, "D": D, "dtype": dtype, "table": table, "scaled": rng.random() < 0.5, "padding": rng.choice([0.0, 0.0, 0.25]) if T >= 16 else 0.0}
    V = rng.choice([151936, 4096, _log_int(rng, 500, 151936), _log_int(rng, 500, 151936) | 1])
    pad = rng.choice([0, 0, rng.randint(1, 64), -V % 64])
    form = rng.choice(["step", "rollouts"]) if kind == "adjust" else "rollouts"
    T = _log_int(rng, 1 if form == "step" else 16, max(32, min(4096, MOST_LOGITS[kind] // ((V + pad) * BYTES[dtype]))))
    return {"kind": kind, "form": form, "T": T, "V": V, "pad": pad, "dtype": dtype, "prompt": rng.choice([0, _log_int(rng, 8, 2000)]), "longest": _log_int(rng, 8, 2000),
            "penalties": rng.choice(["rpf", "rp", "pf", "r", ""]) if kind == "adjust" else rng.choice(["r", "r", ""]), "biases": rng.choice([0, 0, 300, rng.randint(1, 50)]) if kind == "adjust" else 0,
            "masks": rng.choice([0, 1, 64, rng.randint(1, T)])}


# ------------------------------------------------------------------------------ inputs
def _tokens(n, V, g):
    """Ids as in text."""
    u = torch.rand(n, generator=g, device=g.device, dtype=torch.float64)
    return (torch.exp(u * math.log(V + 1)) - 1).long().clamp(0, V - 1).to(torch.int32)


def _histories(case, g):
    """Ids of all prompts and rollouts back to back, and for every row where its history begins, how long it is and how much of
    that is the prompt."""
    T, V, dev = case["T"], case["V"], g.device
    if case["form"] == "step":
        prompt = torch.randint(case["prompt"] // 2, case["prompt"] + 1, (T,), generator=g, device=dev)
        length = prompt + torch.randint(0, case["longest"] + 1, (T,), generator=g, device=dev)
        end = length.cumsum(0)
        return _tokens(int(end[-1]), V, g), end - length, length.to(torch.int32), prompt.to(torch.int32)
    rollouts = -(-T // case["longest"])
    first = (torch.arange(rollouts + 1, device=dev) * T) // rollouts            # of its rows
    prompt = torch.randint(case["prompt"] // 2, case["prompt"] + 1, (rollouts,), generator=g, device=dev)
    end = (prompt + first[1:] - first[:-1]).cumsum(0)
    row = torch.searchsorted(first, torch.arange(T, device=dev), right=True) - 1
    start = torch.cat([end.new_zeros(1), end[:-1]])[row]
    return _tokens(int(end[-1]), V, g), start, (prompt[row] + torch.arange(T, device=dev) - first[row]).to(torch.int32), prompt[row].to(torch.int32)


def _allowed(masks, V, g):
    """Bits of allowed tokens, 32 to a word: every other state of the grammar allows nearly all, the others a handful."""
    words = (V + 31) // 32
    rows = []
    for m in range(masks):
        share = 0.98 if m % 2 else 50.0 / V
        bits = torch.rand(words * 32, generator=g, device=g.device) < share
        bits[m % V] = True
        rows.append((bits.view(words, 32).long() << torch.arange(32, device=g.device)).sum(1))
    return torch.stack(rows).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev, kind, T, V = g.device, case["kind"], case["T"], case["V"]
    dtype = DTYPES[case["dtype"]]
    if kind in ("embed", "embed_grad"):
        tokens = _tokens(T, V, g)
        tokens[torch.randperm(T, generator=g, device=dev)[:int(case["padding"] * T)]] = -1
        D, table = case["D"], DTYPES[case["table"]]
        s = {"kind": kind, "tokens": tokens, "scale": math.sqrt(D) if case["scaled"] else 1.0, "V": V}
        if kind == "embed":
            s.update(table=(0.02 * torch.randn(V, D, generator=g, device=dev)).to(table), out=torch.empty(T, D, dtype=dtype, device=dev))
        else:
            s.update(d_out=(1e-3 * torch.randn(T, D, generator=g, device=dev)).to(dtype), d_table=torch.empty(V, D, dtype=table, device=dev))
        return s
    x = torch.randn(T, V + case["pad"], generator=g, device=dev).mul_(2.0)
    likely = torch.randint(0, V, (T, 8), generator=g, device=dev)
    x.scatter_(1, likely, 4.0 + 8.0 * torch.rand(T, 8, generator=g, device=dev))
    x = x.to(dtype)[:, :V]
    history, start, length, prompt = _histories(case, g)
    s = {"kind": kind, "x": x, "out": torch.empty(T, V + case["pad"], dtype=dtype, device=dev)[:, :V], "history": history, "start": start, "length": length, "prompt": prompt}
    one = case["form"] == "rollouts"                    # one setting for a batch that is trained on
    for name, letter, values in (("repetition", "r", (1.1, 1.0, 1.3)), ("presence", "p", (0.5, 0.0, 1.2)), ("frequency", "f", (0.3, 0.0, 0.05))):
        pick = torch.randint(0, 1 if one else 3, (T,), generator=g, device=dev)
        s[name] = torch.tensor(values, device=dev)[pick].contiguous() if letter in case["penalties"] else None
    n = min(case["biases"], V)
    s["bias_token"] = s["bias_value"] = s["bias_start"] = s["bias_len"] = None
    if n:                                               # one list of the batch, or one of each row
        lists = 1 if one else T
        s["bias_token"] = torch.cat([torch.randperm(V, generator=g, device=dev)[:n] for _ in range(lists)]).to(torch.int32)
        s["bias_value"] = 4.0 * torch.randn(n * lists, generator=g, device=dev)
        s["bias_start"] = n * (torch.zeros(T, dtype=torch.int64, device=dev) if one else torch.arange(T, device=dev))
        s["bias_len"] = torch.full((T,), n, dtype=torch.int32, device=dev)
    s["allowed"] = _allowed(case["masks"], V, g) if case["masks"] else None
    s["mask_row"] = torch.randint(0, case["masks"], (T,), generator=g, device=dev, dtype=torch.int32) if case["masks"] else None
    if kind == "adjust_grad":
        s["d"] = torch.empty(T, V + case["pad"], dtype=dtype, device=dev)[:, :V]
        for a in range(0, T, ROWS_AT_ONCE):
            s["d"][a:a + ROWS_AT_ONCE] = (torch.softmax(x[a:a + ROWS_AT_ONCE].float(), 1) * torch.randn(x[a:a + ROWS_AT_ONCE].shape[0], 1, generator=g, device=dev) / T).to(dtype)
    return s


# ------------------------------------------------------------------------- plain forms
def _seen(s, r):
    """For a slice of rows: which tokens stand in the history, and how often behind the prompt."""
    V, dev = s["x"].shape[1], s["x"].device
    at = torch.arange(max(1, int(s["most"])), device=dev)
    inside = at < s["length"][r, None]
    token = s["history"][torch.where(inside, s["start"][r, None] + at, 0)].long()
    slot = torch.where(inside, token, V)                # one slot more for what is not there
    rows = slot.shape[0]
    seen = torch.zeros(rows, V + 1, device=dev).scatter_(1, slot, 1.0)[:, :V] > 0
    count = torch.zeros(rows, V + 1, device=dev).scatter_add_(1, slot, (at >= s["prompt"][r, None]).float())[:, :V]
    return seen, count


def _is_allowed(s, r):
    v = torch.arange(s["x"].shape[1], device=s["x"].device)
    return ((s["allowed"][s["mask_row"][r].long()][:, v >> 5] >> (v & 31)) & 1) != 0


def _adjust(s, r):
    x = s["x"][r].float()
    y = x
    if s["repetition"] is not None or s["presence"] is not None or s["frequency"] is not None:
        seen, count = _seen(s, r)
        if s["repetition"] is not None:
            by = s["repetition"][r, None]
            y = torch.where(seen, torch.where(x > 0, x / by, x * by), x)
        if s["frequency"] is not None:
            y = y - s["frequency"][r, None] * count
        if s["presence"] is not None:
            y = y - torch.where(count > 0, s["presence"][r, None], 0.0)
    if s["bias_value"] is not None:
        n = s["bias_value"].numel() if s["bias_shared"] else s["bias_value"].numel() // s["x"].shape[0]
        at = s["bias_start"][r, None] + torch.arange(n, device=x.device)
        y = y.scatter_add(1, s["bias_token"][at].long(), s["bias_value"][at])
    if s["allowed"] is not None:
        y = torch.where(_is_allowed(s, r), y, -math.inf)
    return y.to(s["x"].dtype)


def _adjust_gradient(s, r):
    d = s["d"][r].float()
    if s["repetition"] is not None:
        by = s["repetition"][r, None]
        d = torch.where(_seen(s, r)[0], torch.where(s["x"][r].float() > 0, d / by, d * by), d)
    if s["allowed"] is not None:
        d = torch.where(_is_allowed(s, r), d, 0.0)
    return d.to(s["d"].dtype)


def _in_chunks(s, form):
    if "most" not in s:                                 # sizes that a user's program knows
        s["most"] = int(s["length"].max())
        s["bias_shared"] = s["bias_value"] is not None and s["bias_value"].numel() == int(s["bias_len"][0])
    T = s["x"].shape[0]
    return torch.cat([form(s, slice(a, min(a + ROWS_AT_ONCE, T))) for a in range(0, T, ROWS_AT_ONCE)])


def _embed(s):
    e = s["table"][s["tokens"].clamp(min=0).long()].float() * s["scale"]
    return torch.where(s["tokens"][:, None] >= 0, e, 0.0).to(s["out"].dtype)


def _embed_gradient(s):
    d = torch.where(s["tokens"][:, None] >= 0, s["d_out"].float(), 0.0)
    total = torch.zeros(s["d_table"].shape, device=d.device).index_add_(0, s["tokens"].clamp(min=0).long(), d)
    return (total * s["scale"]).to(s["d_table"].dtype)


def run(s):
    kind = s["kind"]
    if not own:
        return _embed(s) if kind == "embed" else _embed_gradient(s) if kind == "embed_grad" else _in_chunks(s, _adjust if kind == "adjust" else _adjust_gradient)
    import paper_2605_05802_b200 as sr
    if kind == "embed":
        sr.sr_embed_tokens(s["table"], s["tokens"], s["scale"], out=s["out"])
        return s["out"]
    if kind == "embed_grad":
        if "ws" not in s:                               # a workspace that the program allocates once
            bytes_of = sr.sr_embed_tokens_backward_workspace_bytes(s["tokens"].numel(), s["V"], s["d_table"].shape[1])
            s["ws"] = torch.empty(max(bytes_of, 1), dtype=torch.uint8, device="cuda")
        sr.sr_embed_tokens_backward(s["d_out"], s["tokens"], s["scale"], d_table=s["d_table"], workspace=s["ws"])
        return s["d_table"]
    if kind == "adjust":
        sr.sr_adjust_logits(s["x"], history=s["history"], history_start=s["start"], history_len=s["length"], prompt_len=s["prompt"], repetition=s["repetition"],
                            presence=s["presence"], frequency=s["frequency"], bias_token=s["bias_token"], bias_value=s["bias_value"], bias_start=s["bias_start"],
                            bias_len=s["bias_len"], allowed=s["allowed"], mask_row=s["mask_row"], out=s["out"])
        return s["out"]
    sr.sr_adjust_logits_backward(s["d"], s["x"], history=s["history"], history_start=s["start"], history_len=s["length"], repetition=s["repetition"],
                                 allowed=s["allowed"], mask_row=s["mask_row"], d_logits=s["out"])
    return s["out"]


def work(case):
    T, V, kind = case["T"], case["V"], case["kind"]
    e = BYTES[case["dtype"]]
    if kind in ("embed", "embed_grad"):
        D, t = case["D"], BYTES[case["table"]]
        taken = T - int(case["padding"] * T)
        if kind == "embed_grad":
            return {"bytes": float(taken * D * e + V * D * t + 4 * T), "flops": float(taken * D)}
        v = np.arange(V, dtype=np.float64)              # rows of the table that are read at all
        distinct = float((1.0 - (1.0 - np.log1p(1.0 / (v + 1)) / math.log(V + 1)) ** taken).sum())
        return {"bytes": distinct * D * t + T * D * e + 4.0 * T, "flops": float(taken * D)}
    rows = T if case["form"] == "step" else -(-T // case["longest"])
    history = rows * 0.75 * case["prompt"] + (T * case["longest"] / 2 if case["form"] == "step" else T)
    rules = 4.0 * history * bool(case["penalties"]) + 4.0 * T * len(case["penalties"]) + 8.0 * case["biases"] * (T if case["form"] == "step" else 1) + case["masks"] * V / 8.0
    return {"bytes": 2.0 * T * V * e + rules, "flops": float(T * V)}


# ------------------------------------------------------------- the definition, 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    kind, T, V = case["kind"], case["T"], case["V"]
    if kind == "embed":
        out = torch.zeros(T, case["D"], dtype=torch.float64, device="cuda")
        real = torch.nonzero(s["tokens"] >= 0)[:, 0]
        out[real] = s["scale"] * torch.index_select(s["table"], 0, s["tokens"][real].long()).double()
        return out
    if kind == "embed_grad":
        order = torch.argsort(s["tokens"].long(), stable=True)
        token, runs = torch.unique_consecutive(s["tokens"][order], return_counts=True)
        out = torch.zeros(V, case["D"], dtype=torch.float64, device="cuda")
        ends = torch.cat([runs.new_zeros(1), runs.cumsum(0)])
        for c in range(0, case["D"], 256):              # sums of runs as differences of running sums
            before = torch.nn.functional.pad(s["d_out"][:, c:c + 256].double()[order].cumsum(0), (0, 0, 1, 0))
            sums = before[ends[1:]] - before[ends[:-1]]
            out[token[token >= 0].long(), c:c + 256] = s["scale"] * sums[token >= 0]
        return out
    parts = []
    for a in range(0, T, 256):
        b = min(a + 256, T)
        x = s["x"][a:b].double()
        lengths, starts, prompts = (s[k][a:b].tolist() for k in ("length", "start", "prompt"))
        spans = [torch.arange(at, at + n, device="cuda") for at, n in zip(starts, lengths)]
        row = torch.repeat_interleave(torch.arange(b - a, device="cuda"), s["length"][a:b].long())
        keys = row * V + s["history"][torch.cat(spans)].long()
        late = torch.cat([torch.arange(n, device="cuda") >= p for n, p in zip(lengths, prompts)])
        seen = torch.unique(keys)
        again, times = torch.unique(keys[late], return_counts=True)
        y = (x if kind == "adjust" else s["d"][a:b].double()).clone().view(-1)
        if s["repetition"] is not None:
            by = s["repetition"][a:b].double()[seen // V]
            y[seen] *= torch.where(x.view(-1)[seen] > 0, 1 / by, by)
        if kind == "adjust":
            for name, amount in (("presence", torch.ones_like(times)), ("frequency", times)):
                if s[name] is not None:
                    y[again] -= s[name][a:b].double()[again // V] * amount
            if s["bias_value"] is not None:
                for t in range(a, b):
                    here = slice(int(s["bias_start"][t]), int(s["bias_start"][t]) + int(s["bias_len"][t]))
                    y[(t - a) * V + s["bias_token"][here].long()] += s["bias_value"][here].double()
        y = y.view(b - a, V)
        if s["allowed"] is not None:
            words = s["allowed"][s["mask_row"][a:b].long()].cpu().numpy().astype("<i4").view(np.uint8)
            bits = torch.from_numpy(np.unpackbits(words, axis=1, bitorder="little")[:, :V]).cuda()
            y = y.masked_fill(bits == 0, -math.inf if kind == "adjust" else 0.0)
        parts.append(y)
    return torch.cat(parts)
