"""Workloads of the attention operators: what a pipeline stage computes between the product behind its norm and its second product.

The product in front gives every token its queries, keys and values side by side.  Queries and keys are rotated by their
position; in training the tokens of a batch, or of sequences of different lengths packed behind each other, attend to their own
sequence, causally, and the gradients come back the same way; in serving keys and values go into a cache of pages, and
new tokens (one of each sequence, a chunk of a prompt, or a tree of drafted tokens) attend to everything that is there.  Query heads may
share key heads.  Sizes run from one token to sequences of 16384 and batches of long contexts, with odd and ragged ones among them.

ops
  rotate          accept_rotate: queries and keys by their position, or their gradients back
  append          accept_cache_append: keys and values into their pages, keys and queries rotated on the way
  attend          accept_attention: causal or not, and the logarithms of the sums that the backward pass takes
  attend_back     accept_attention_backward: gradients of queries, keys and values
  cached          accept_cache_attention: few tokens a sequence over its cache, causal or as a tree

Descriptors are made once, as a training loop or a server keeps them; outputs are allocated by each call.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
CHUNK = 1 << 29  # scores held at a time
MOST = {"bf16": 8e11, "f32": 1e11}  # operations of a drawn case


# ---------------------------------------------------------------------------------- the cases
def _rotate(name, tokens, heads, head, rotated, dtype="bf16", neighbours=False, inverse=False, first=0):
    """`first`: position of the first token (positions are given where it is not 0)."""
    return {"name": name, "op": "rotate", "tokens": tokens, "heads": heads, "head": head, "rotated": rotated, "dtype": dtype,
            "neighbours": neighbours, "inverse": inverse, "first": first}


def _attend(name, op, tokens, sequences, mix, heads, kv_heads, head, dtype="bf16", causal=True):
    """`mix` 0: sequences of one length; otherwise the seed of their lengths."""
    return {"name": name, "op": op, "tokens": tokens, "sequences": sequences, "mix": mix, "heads": heads, "kv_heads": kv_heads,
            "head": head, "dtype": dtype, "causal": causal}


def _cache(name, op, sequences, context, new, mix, heads, kv_heads, head, page, dtype="bf16", rotated=0, neighbours=False, tree=False):
    """Contexts of `context` tokens on average, `new` tokens a sequence on average; mix 0: all alike."""
    return {"name": name, "op": op, "sequences": sequences, "context": context, "new": new, "mix": mix, "heads": heads,
            "kv_heads": kv_heads, "head": head, "page": page, "dtype": dtype, "rotated": rotated, "neighbours": neighbours, "tree": tree}


def listed():
    return [
        # Queries and keys of a batch's hidden states (16 x 509 tokens) in front of the attention.
        _rotate("rotate_hidden", 8144, 16, 64, 64),
        # Their gradients back in float32, of a long sequence's end, where only half of a head is rotated.
        _rotate("rotate_far_back", 20000, 40, 128, 64, dtype="f32", neighbours=True, inverse=True, first=1000000),
        # One new token of one sequence.
        _cache("append_token", "append", 1, 4001, 1, 0, 32, 8, 128, 16, rotated=128),
        # Prompts of different lengths into an empty cache.
        _cache("append_prompts", "append", 12, 0, 1361, 5, 32, 8, 128, 64, rotated=128),
        # Hidden states of a batch (16 x 509 x 768): 12 heads of 64.
        _attend("attend_hidden", "attend", 8144, 16, 0, 12, 12, 64),
        # Sequences of different lengths packed behind each other, four query heads to a key head.
        _attend("attend_packed", "attend", 16384, 11, 3, 32, 8, 128),
        # One long sequence.
        _attend("attend_long", "attend", 16384, 1, 0, 16, 2, 128),
        # The batch's backward pass.
        _attend("attend_back_hidden", "attend_back", 8144, 16, 0, 12, 12, 64),
        # Backward of packed sequences with shared key heads.
        _attend("attend_back_packed", "attend_back", 12288, 7, 4, 32, 8, 128),
        # The next token of one sequence.
        _cache("cached_token", "cached", 1, 4001, 1, 0, 32, 8, 128, 16),
        # A served batch, one token of each sequence, contexts of different lengths.
        _cache("cached_batch", "cached", 48, 5000, 1, 2, 32, 8, 128, 64),
        # Trees of 40 drafted tokens over the contexts of a smaller batch.
        _cache("cached_tree", "cached", 6, 9000, 40, 7, 32, 8, 128, 32, tree=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend", "attend", "attend_back", "attend_back", "cached", "cached", "cached"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    head = rng.choice([64, 64, 128, 128, 128, 32, 80, 96, 256])
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
    mix = rng.choice([0, rng.randrange(1, 1000)])
    if op == "rotate":
        tokens = _log(rng, 1, max(16, (1 << 26) // (heads * head)))
        case = _rotate("", tokens, heads, head, rng.choice([head, head // 2]), dtype, rng.random() < 0.5, rng.random() < 0.5,
                       rng.choice([0, rng.randrange(1, 1 << 20)]))
    elif op in ("attend", "attend_back"):
        sequences, length, causal = _log(rng, 1, 64), _log(rng, 1, 8192), rng.random() < 0.8
        while True:
            case = _attend("", op, sequences * length, sequences, mix, heads, kv_heads, head, dtype, causal)
            if sequences * length <= 32768 and work(case)["flops"] <= MOST[dtype]:
                break
            sequences, length = max(1, sequences * 2 // 3), max(1, length * 3 // 4)
    else:
        sequences, context, new = _log(rng, 1, 128), _log(rng, 1, 32768), 1
        tree = op == "cached" and rng.random() < 0.4
        if tree:
            new = _log(rng, 2, 64)
        elif rng.random() < 0.4:
            new = _log(rng, 2, 512)
        page, neighbours = rng.choice([16, 32, 64, 128]), rng.random() < 0.5
        rotated = rng.choice([0, head // 2, head, head]) if op == "append" else 0
        while True:
            case = _cache("", op, sequences, context, new, mix, heads, kv_heads, head, page, dtype, rotated, neighbours, tree)
            if sequences * (context + new) * kv_heads * head <= 1 << 28 and work(case)["flops"] <= MOST[dtype] / 8:
                break
            sequences, context, new = max(1, sequences * 2 // 3), max(1, context * 3 // 4), max(1 + tree, new * 3 // 4)
    del case["name"]
    return case


def _lengths(total, count, mix, least=0):
    """`count` lengths that come to `total`: equal ones (mix 0), or some long and many short (log-normal, and none below `least`)."""
    if mix == 0:
        return [total // count] * count
    rng = random.Random(mix)
    weights = [math.exp(rng.gauss(0, 0.8)) for _ in range(count)]
    lengths = [max(least, int(total * w / sum(weights))) for w in weights]
    lengths[lengths.index(max(lengths))] += total - sum(lengths)
    return lengths


def _new(case):
    """New tokens of every sequence of a cache."""
    if case["new"] == 1 or case["tree"]:
        return [case["new"]] * case["sequences"]
    return _lengths(case["new"] * case["sequences"], case["sequences"], case["mix"])


def _contexts(case):
    return _lengths(case["context"] * case["sequences"], case["sequences"], case["mix"] + 1 if case["mix"] else 0)


def _pairs(queries, keys, causal):
    """Keys that the queries of a sequence see, in all; the last query sees the last key."""
    if not causal:
        return queries * keys
    return sum(max(0, i + 1 + keys - queries) for i in range(queries))


def work(case):
    size, head = SIZE[case["dtype"]], case["head"]
    if case["op"] == "rotate":
        values = case["tokens"] * case["heads"] * head
        return {"bytes": 2 * values * size + 2 * case["rotated"] + (4 * case["tokens"] if case["first"] else 0),
                "flops": 3 * case["tokens"] * case["heads"] * case["rotated"]}
    heads, kv_heads = case["heads"], case["kv_heads"]
    if case["op"] == "append":
        tokens = sum(_new(case))
        return {"bytes": 2 * tokens * (heads + 2 * kv_heads) * head * size, "flops": 3 * tokens * (heads + kv_heads) * case["rotated"]}
    if case["op"] == "cached":
        new, contexts = _new(case), _contexts(case)
        keys = sum(c + n for c, n in zip(contexts, new) if n)
        if case["tree"]:
            trees = _trees(case)
            pairs = sum(n * c + sum(bin(m).count("1") for m in t) for n, c, t in zip(new, contexts, trees))
        else:
            pairs = sum(n * c + n * (n + 1) // 2 for n, c in zip(new, contexts))
        return {"bytes": size * head * (2 * keys * kv_heads + 2 * sum(new) * heads), "flops": 4 * pairs * heads * head}
    lengths = _lengths(case["tokens"], case["sequences"], case["mix"])
    pairs = sum(_pairs(n, n, case["causal"]) for n in lengths) * heads * head
    values = case["tokens"] * head
    if case["op"] == "attend":
        return {"bytes": size * values * 2 * (heads + kv_heads) + 4 * case["tokens"] * heads, "flops": 4 * pairs}
    # scores and their gradients again, three gradients
    return {"bytes": size * values * 4 * (heads + kv_heads) + 4 * case["tokens"] * heads, "flops": 10 * pairs}


# ------------------------------------------------------------------------------------- inputs
def _normal(g, *size):
    return torch.randn(*size, generator=g, device=DEVICE)


def _channels(g, heads, head):
    """Every channel of a head has a size of its own, a few large ones among them."""
    return torch.exp(0.4 * _normal(g, heads, head))


def _projected(g, tokens, heads, kv_heads, head, dtype):
    """(q, k, v) as they lie side by side in a product's result."""
    both = heads + 2 * kv_heads
    held = torch.empty(tokens, both * head, dtype=TYPES[dtype], device=DEVICE)
    whole = held.view(tokens, both, head)
    whole.copy_(_normal(g, tokens, both, head) * _channels(g, both, head))
    return whole[:, :heads], whole[:, heads:heads + kv_heads], whole[:, heads + kv_heads:]


def _frequencies(rotated):
    return (10000.0 ** (-torch.arange(0, rotated, 2, dtype=torch.float64) / max(rotated, 1))).float().to(DEVICE)


def _offsets(lengths):
    ends = [0]
    for n in lengths:
        ends.append(ends[-1] + n)
    return ends


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _trees(case):
    """For every sequence the nodes that each drafted token sees, as bits: itself and what it continues."""
    trees = []
    for s in range(case["sequences"]):
        rng, masks = random.Random(1000 * case["mix"] + s), []
        for j in range(case["new"]):
            parent = rng.randrange(max(0, j - 6), j + 1) - 1 if j else -1
            masks.append((masks[parent] if parent >= 0 else 0) | 1 << j)
        trees.append(masks)
    return trees


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    op, dtype = case["op"], case["dtype"]
    state = {"case": dict(case), "desc": None}
    if op == "rotate":
        size = (case["tokens"], case["heads"], case["head"])
        state["x"] = (_normal(g, *size) * _channels(g, *size[1:])).to(TYPES[dtype])
        state["frequencies"] = _frequencies(case["rotated"])
        first = case["first"]
        state["positions"] = torch.arange(first, first + case["tokens"], dtype=torch.int32, device=DEVICE) if first else None
        return state
    heads, kv_heads, head = case["heads"], case["kv_heads"], case["head"]
    if op in ("attend", "attend_back"):
        state["ends"] = _offsets(_lengths(case["tokens"], case["sequences"], case["mix"]))
        state["offsets"] = _ints(state["ends"]) if case["mix"] else None
        state["q"], state["k"], state["v"] = _projected(g, case["tokens"], heads, kv_heads, head, dtype)
        if op == "attend_back":
            out = _plain_attention(state)
            state["o"], state["lse"] = out["o"], out["lse"]
            state["do"] = (1e-3 * _normal(g, case["tokens"], heads, head)).to(TYPES[dtype])
        return state
    new, contexts, page = _new(case), _contexts(case), case["page"]
    state["ends"], state["contexts"] = _offsets(new), contexts
    state["offsets"] = None if len(set(new)) == 1 else _ints(state["ends"])
    state["lengths"] = _ints(contexts)
    each = [-(-(c + n) // page) for c, n in zip(contexts, new)]
    pages = sum(each) + 3
    # pages as they were free when they were needed: in no order
    free = torch.randperm(pages, generator=g, device=DEVICE).to(torch.int32)
    state["table"] = torch.zeros(case["sequences"], max(max(each), 1), dtype=torch.int32, device=DEVICE)
    taken = 0
    for s, n in enumerate(each):
        state["table"][s, :n] = free[taken:taken + n]
        taken += n
    size = (pages, kv_heads, page, head)
    state["k_cache"] = (_normal(g, *size) * _channels(g, kv_heads, head)[:, None]).to(TYPES[dtype])
    state["v_cache"] = _normal(g, *size).to(TYPES[dtype])
    state["q"], state["k"], state["v"] = _projected(g, state["ends"][-1], heads, kv_heads, head, dtype)
    state["frequencies"] = _frequencies(case["rotated"]) if case["rotated"] else None
    state["tree"] = None
    if case["tree"]:
        masks = [m - (1 << 64) if m >> 63 else m for t in _trees(case) for m in t]
        state["tree"] = torch.tensor(masks, dtype=torch.int64, device=DEVICE).view(-1, 1)
    return state


# --------------------------------------------------------------------- the operators, in plain form
def _plain_rotation(x, positions, frequencies, neighbours, inverse=False):
    """x (tokens, heads, head) in float32; the angles in 64 bits, where far positions lose nothing."""
    rotated = 2 * frequencies.numel()
    angle = positions.double()[:, None] * frequencies.double()[None, :]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if inverse:
        sin = -sin
    y = x.clone()
    if neighbours:
        a, b = x[..., 0:rotated:2], x[..., 1:rotated:2]
        y[..., 0:rotated:2], y[..., 1:rotated:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :rotated // 2], x[..., rotated // 2:rotated]
        y[..., :rotated // 2], y[..., rotated // 2:rotated] = a * cos - b * sin, a * sin + b * cos
    return y


def _plain_scores(q, k, scale, seen):
    """Of (group, queries, head) and (keys, head); what is not seen is minus infinity."""
    scores = torch.matmul(q, k.t()) * scale
    return scores if seen is None else scores.masked_fill_(~seen, float("-inf"))


def _plain_seen(queries, keys, causal):
    if not causal:
        return None
    i, j = torch.arange(queries, device=DEVICE), torch.arange(keys, device=DEVICE)
    return j[None, :] <= i[:, None] + (keys - queries)


def _pieces(state):
    """(first token, end, query heads, key head, scale) of every sequence and every part of a group that fits."""
    case = state["case"]
    group = case["heads"] // case["kv_heads"]
    for begin, end in zip(state["ends"], state["ends"][1:]):
        if begin == end:
            continue
        some = max(1, min(group, CHUNK // (end - begin) ** 2))
        for kv in range(case["kv_heads"]):
            for h in range(kv * group, (kv + 1) * group, some):
                yield begin, end, slice(h, min(h + some, (kv + 1) * group)), kv, case["head"] ** -0.5


def _plain_attention(state):
    case = state["case"]
    o = torch.zeros(case["tokens"], case["heads"], case["head"], dtype=TYPES[case["dtype"]], device=DEVICE)
    lse = torch.full((case["heads"], case["tokens"]), float("-inf"), device=DEVICE)
    for begin, end, hs, kv, scale in _pieces(state):
        q = state["q"][begin:end, hs].transpose(0, 1).float()
        k, v = state["k"][begin:end, kv].float(), state["v"][begin:end, kv].float()
        scores = _plain_scores(q, k, scale, _plain_seen(end - begin, end - begin, case["causal"]))
        largest = scores.amax(-1, keepdim=True)
        p = torch.exp_(scores.sub_(largest))
        total = p.sum(-1, keepdim=True)
        o[begin:end, hs] = (torch.matmul(p, v) / total).transpose(0, 1).to(o.dtype)
        lse[hs, begin:end] = (largest + torch.log(total))[..., 0]
    return {"o": o, "lse": lse}


def _plain_gradients(state):
    case = state["case"]
    size = (case["tokens"], case["kv_heads"], case["head"])
    dq = torch.zeros(case["tokens"], case["heads"], case["head"], device=DEVICE)
    dk, dv = torch.zeros(size, device=DEVICE), torch.zeros(size, device=DEVICE)
    for begin, end, hs, kv, scale in _pieces(state):
        q, o, do = (state[name][begin:end, hs].transpose(0, 1).float() for name in ("q", "o", "do"))
        k, v = state["k"][begin:end, kv].float(), state["v"][begin:end, kv].float()
        scores = _plain_scores(q, k, scale, _plain_seen(end - begin, end - begin, case["causal"]))
        p = torch.exp_(scores.sub_(state["lse"][hs, begin:end, None]))
        ds = torch.matmul(do, v.t()).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
        dq[begin:end, hs] = torch.matmul(ds, k).transpose(0, 1)
        dk[begin:end, kv] += torch.matmul(ds.flatten(0, 1).t(), q.flatten(0, 1))
        dv[begin:end, kv] += torch.matmul(p.flatten(0, 1).t(), do.flatten(0, 1))
    dtype = TYPES[case["dtype"]]
    return {"dq": dq.to(dtype), "dk": dk.to(dtype), "dv": dv.to(dtype)}


def _slots(state, s, first, end):
    """(pages, places in them) of a sequence's tokens first .. end-1."""
    at = torch.arange(first, end, device=DEVICE)
    page = state["case"]["page"]
    return state["table"][s].long()[at // page], at % page


def _plain_append(state):
    case, q, k = state["case"], state["q"].float(), state["k"].float()
    if case["rotated"]:
        positions = torch.cat([torch.arange(c, c + e - b, device=DEVICE)
                               for b, e, c in zip(state["ends"], state["ends"][1:], state["contexts"])])
        q = _plain_rotation(q, positions, state["frequencies"], case["neighbours"])
        k = _plain_rotation(k, positions, state["frequencies"], case["neighbours"])
    dtype = TYPES[case["dtype"]]
    for s, (b, e, c) in enumerate(zip(state["ends"], state["ends"][1:], state["contexts"])):
        page, place = _slots(state, s, c, c + e - b)
        state["k_cache"][page, :, place] = k[b:e].to(dtype)
        state["v_cache"][page, :, place] = state["v"][b:e]
    return {"q": q.to(dtype), "k_cache": state["k_cache"], "v_cache": state["v_cache"]}


def _plain_cached(state):
    case = state["case"]
    o = torch.zeros(state["ends"][-1], case["heads"], case["head"], dtype=TYPES[case["dtype"]], device=DEVICE)
    group, scale = case["heads"] // case["kv_heads"], case["head"] ** -0.5
    for s, (b, e, c) in enumerate(zip(state["ends"], state["ends"][1:], state["contexts"])):
        if b == e:
            continue
        n = e - b
        page, place = _slots(state, s, 0, c + n)
        k, v = state["k_cache"][page, :, place].float(), state["v_cache"][page, :, place].float()  # keys, heads, head
        seen = _plain_seen(n, c + n, True)
        if case["tree"]:
            bits = state["tree"][b:e, 0, None] >> torch.arange(n, device=DEVICE) & 1
            seen = torch.cat((torch.ones(n, c, dtype=torch.bool, device=DEVICE), bits == 1), 1)
        for kv in range(case["kv_heads"]):
            hs = slice(kv * group, (kv + 1) * group)
            scores = _plain_scores(state["q"][b:e, hs].transpose(0, 1).float(), k[:, kv], scale, seen)
            p = torch.exp_(scores - scores.amax(-1, keepdim=True))
            o[b:e, hs] = (torch.matmul(p, v[:, kv]) / p.sum(-1, keepdim=True)).transpose(0, 1).to(o.dtype)
    return {"o": o}


def _run_plain(state):
    case = state["case"]
    if case["op"] == "rotate":
        positions = state["positions"] if case["first"] else torch.arange(case["tokens"], device=DEVICE)
        y = _plain_rotation(state["x"].float(), positions, state["frequencies"], case["neighbours"], case["inverse"])
        return {"y": y.to(TYPES[case["dtype"]])}
    return {"append": _plain_append, "attend": _plain_attention, "attend_back": _plain_gradients, "cached": _plain_cached}[case["op"]](state)


# --------------------------------------------------------------------- the framework's operators
def _describe(state):
    import paper_2311_05827_amd as A

    case = state["case"]
    code = {"f32": A.F32, "bf16": A.BF16}[case["dtype"]]
    pairs = A.ROTATE_NEIGHBOURS if case.get("neighbours") else A.ROTATE_HALVES
    if case["op"] == "rotate":
        return A.make_rotate_desc(case["tokens"], case["heads"], case["head"], rotated=case["rotated"], dtype=code, pairs=pairs,
                                  inverse=case["inverse"])
    stride = state["q"].stride(0)
    heads = (case["heads"], case["kv_heads"], case["head"])
    if case["op"] in ("attend", "attend_back"):
        return A.make_attention_desc(case["tokens"], case["tokens"], *heads, sequences=case["sequences"], dtype=code, causal=case["causal"],
                                     q_stride=stride, k_stride=stride, v_stride=stride)
    return A.make_cache_desc(state["ends"][-1], case["sequences"], *heads, page_size=case["page"], pages=state["k_cache"].shape[0],
                             table_pages=state["table"].shape[1], dtype=code, rotated=case["rotated"], pairs=pairs,
                             tree_words=1 if case["tree"] else 0, q_stride=stride, k_stride=stride, v_stride=stride)


def _run_own(state):
    import paper_2311_05827_amd as A

    case = state["case"]
    if state["desc"] is None:
        state["desc"] = _describe(state)
    desc = state["desc"]
    if case["op"] == "rotate":
        return {"y": A.accept_rotate(desc, state["x"], state["frequencies"], positions=state["positions"])}
    if case["op"] == "attend":
        o, lse = A.accept_attention(desc, state["q"], state["k"], state["v"], q_offsets=state["offsets"], k_offsets=state["offsets"])
        return {"o": o, "lse": lse}
    if case["op"] == "attend_back":
        dq, dk, dv = A.accept_attention_backward(desc, state["do"], state["q"], state["k"], state["v"], state["o"], state["lse"],
                                                 q_offsets=state["offsets"], k_offsets=state["offsets"])
        return {"dq": dq, "dk": dk, "dv": dv}
    if case["op"] == "append":
        q = A.accept_cache_append(desc, state["q"], state["k"], state["v"], state["k_cache"], state["v_cache"], state["table"],
                                  state["lengths"], offsets=state["offsets"], frequencies=state["frequencies"])
        return {"q": q, "k_cache": state["k_cache"], "v_cache": state["v_cache"]}
    return {"o": A.accept_cache_attention(desc, state["q"], state["k_cache"], state["v_cache"], state["table"], state["lengths"],
                                          offsets=state["offsets"], tree=state["tree"])}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------- in 64 bits, from the definitions
def _exact_turned(x, positions, case):
    """Every pair of values is a complex number, times that of its position's angle."""
    rotated = case["rotated"]
    half = rotated // 2
    x = x.double()
    head, rest = x[..., :rotated], x[..., rotated:]
    pairs = head.unflatten(-1, (half, 2)) if case["neighbours"] else torch.stack((head[..., :half], head[..., half:]), -1)
    number = torch.view_as_complex(pairs.contiguous())
    angle = torch.outer(positions.double(), _frequencies(rotated).double())
    if case.get("inverse"):
        angle = -angle
    turned = torch.view_as_real(number * torch.polar(torch.ones_like(angle), angle)[:, None, :])
    head = turned.flatten(-2) if case["neighbours"] else torch.cat((turned[..., 0], turned[..., 1]), -1)
    return torch.cat((head, rest), -1)


def _exact_weights(q, k, scale, first):
    """Probabilities of (queries, head) over (keys, head), and the logarithm of each row's sum; query i sees keys up to first + i (all
    where that is None)."""
    s = (q @ k.transpose(0, 1).contiguous()) * scale
    if first is not None:
        hidden = torch.ones_like(s, dtype=torch.bool).triu_(first + 1)
        s[hidden] = float("-inf")
    lse = torch.logsumexp(s, 1)
    return torch.exp(s - lse[:, None]), lse


def _exact_attention(state):
    case = state["case"]
    group = case["heads"] // case["kv_heads"]
    o = torch.zeros(case["tokens"], case["heads"], case["head"], dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(case["heads"], case["tokens"], dtype=torch.float64, device=DEVICE)
    for b, e in zip(state["ends"], state["ends"][1:]):
        for h in range(case["heads"] if e > b else 0):
            q, k, v = state["q"][b:e, h].double(), state["k"][b:e, h // group].double(), state["v"][b:e, h // group].double()
            for at in range(0, e - b, 4096):  # rows at a time
                w, part = _exact_weights(q[at:at + 4096], k, 1 / math.sqrt(case["head"]), at if case["causal"] else None)
                o[b + at:b + at + w.shape[0], h] = w @ v
                lse[h, b + at:b + at + w.shape[0]] = part
    return {"o": o, "lse": lse}


def _exact_gradients(state):
    case = state["case"]
    group, scale = case["heads"] // case["kv_heads"], 1 / math.sqrt(case["head"])
    out = {name: torch.zeros(state[name[1:]].shape, dtype=torch.float64, device=DEVICE) for name in ("dq", "dk", "dv")}
    for b, e in zip(state["ends"], state["ends"][1:]):
        for h in range(case["heads"] if e > b else 0):
            kv = h // group
            k, v = state["k"][b:e, kv].double(), state["v"][b:e, kv].double()
            for at in range(b, e, 4096):
                to = min(e, at + 4096)
                q, o, do = (state[name][at:to, h].double() for name in ("q", "o", "do"))
                s = (q @ k.transpose(0, 1).contiguous()) * scale
                if case["causal"]:
                    s = s.where(torch.ones_like(s, dtype=torch.bool).tril_(at - b), torch.full_like(s, float("-inf")))
                p = (s - state["lse"][h, at:to].double()[:, None]).exp()
                along = (do * o).sum(1, keepdim=True)
                ds = p * (do @ v.transpose(0, 1).contiguous() - along) * scale
                out["dq"][at:to, h] = ds @ k
                out["dk"][b:e, kv] += ds.transpose(0, 1).contiguous() @ q
                out["dv"][b:e, kv] += p.transpose(0, 1).contiguous() @ do
    return out


def _exact_append(state):
    case = state["case"]
    out = {name: state[name].double() for name in ("q", "k_cache", "v_cache")}
    page = case["page"]
    for s, (b, e) in enumerate(zip(state["ends"], state["ends"][1:])):
        if b == e:
            continue
        position = state["contexts"][s] + torch.arange(e - b, device=DEVICE)
        k = state["k"][b:e].double()
        if case["rotated"]:
            k = _exact_turned(state["k"][b:e], position, case)
            out["q"][b:e] = _exact_turned(state["q"][b:e], position, case)
        at = state["table"][s, torch.div(position, page, rounding_mode="floor")].long() * page + position % page
        for name, values in (("k_cache", k), ("v_cache", state["v"][b:e].double())):
            flat = out[name].transpose(1, 2).reshape(-1, case["kv_heads"], case["head"])  # page by page, place by place
            flat[at] = values
            out[name] = flat.unflatten(0, (-1, page)).transpose(1, 2).contiguous()
    return out


def _exact_cached(state):
    case = state["case"]
    group, page = case["heads"] // case["kv_heads"], case["page"]
    o = torch.zeros(state["ends"][-1], case["heads"], case["head"], dtype=torch.float64, device=DEVICE)
    trees = _trees(case) if case["tree"] else None
    for s, (b, e) in enumerate(zip(state["ends"], state["ends"][1:])):
        n, c = e - b, state["contexts"][s]
        if n == 0:
            continue
        pages = state["table"][s, :-(-(c + n) // page)].long()
        for kv in range(case["kv_heads"]):
            k, v = (state[name][pages, kv].reshape(-1, case["head"])[:c + n].double() for name in ("k_cache", "v_cache"))
            for h in range(kv * group, (kv + 1) * group):
                q = state["q"][b:e, h].double()
                if trees is None:
                    w, _ = _exact_weights(q, k, 1 / math.sqrt(case["head"]), c)
                else:
                    s_all = q @ k.transpose(0, 1).contiguous() / math.sqrt(case["head"])
                    for i, m in enumerate(trees[s]):
                        unseen = [c + j for j in range(n) if not m >> j & 1]
                        s_all[i, unseen] = float("-inf")
                    w = torch.softmax(s_all, 1)
                o[b:e, h] = w @ v
    return {"o": o}


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "rotate":
        positions = torch.arange(case["first"], case["first"] + case["tokens"], device=DEVICE)
        return {"y": _exact_turned(state["x"], positions, case)}
    return {"append": _exact_append, "attend": _exact_attention, "attend_back": _exact_gradients, "cached": _exact_cached}[case["op"]](state)
