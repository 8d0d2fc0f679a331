"""The measured cases of the operators for serving the layer around the lattice memory, and for training it with rotary
positions: the rotation itself, a paged key-value cache with the append that rotates, attention of new tokens over its
pages, and eviction from it by accumulated attention weight.

``run`` computes a case with the package's kernels where ``own`` is true and in plain form, elementary torch operations
in 32 bits (angles in 64), where it is false.  ``exact`` computes it from the definitions in 64 bits, sequence by sequence.

Definitions.  Rotation: pair i of a head, (x[2i], x[2i+1]) interleaved or (x[i], x[i+n]) in halves, turns by the angle
a = 2 pi position frequency_i: m (x1 cos a - x2 sin a), m (x1 sin a + x2 cos a); the head's dimensions past 2n stay.

Cache.  Of each sequence table[b] names the pages, used[b] counts its keys and seen[b] the tokens that it has had; its
newest rows are the last nq of both.  With E = 16 bytes of elements, F = E / 4, key slot t of a page is element
[t / 16, d / E, t % 16, d % E] of k[page, head] and [t / (16 F), d / 16, t % 16 / 4, d % 16, t % (16 F) / 16 * 4 + t % 4]
of v[page, head]; position[page, head, t] is its token's place in the text, weight[page, head, t] the attention weight
that it has gathered.

Attention: query i of a sequence, at position p_i = seen - nq + i, sees the used keys of position p_j <= p_i;
s_ij = q_i . k_j / sqrt(D) + W[head, bucket(p_j - p_i)], o_i = sum_j softmax_j(s_ij) v_j, and weight_j grows by the sum
of softmax_j(s_ij) over the sequence's queries and the heads that share the key.

Eviction to a budget: of each key head stay the keys of the ``recent`` newest positions and, of the others, those of the
largest weight, at equal weights the lowest position; those that stay from slot ``budget`` on move, in their order, to
the slots below it that are left.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BUCKETS, REACH = 32, 128  # of the relative position bias
BASE, FACTOR, LENGTH = 10000.0, 8.0, 2048  # of the frequencies; scaled: for texts 8 times as long as those of training
LOW, HIGH = 1.0, 32.0  # turns over LENGTH up to which a frequency is divided by FACTOR, and from which on it stays


def _times(n, length):
    return ",".join([str(length)] * n)


def _rotary(name, lengths, heads, kv_heads, dim, pairs, interleaved, scaled, far, dtype, train):
    """far: the first token's position."""
    return {"name": name, "kind": "rotary", "queries": lengths, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "pairs": pairs, "interleaved": interleaved, "scaled": scaled, "far": far, "dtype": dtype, "train": train}


def _cache(name, kind, queries, used, heads, kv_heads, dim, page, dtype, pairs=0, interleaved=False, bias=False,
           weigh=False, budget=0, recent=0):
    """queries: the sequences' new rows; used: the keys that they have with these (a step: before it)."""
    return {"name": name, "kind": kind, "queries": queries, "used": used, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "page": page, "dtype": dtype, "pairs": pairs, "interleaved": interleaved, "bias": bias,
            "weigh": weigh, "budget": budget, "recent": recent}


def listed():
    ragged = ",".join(str(256 + (i * 2741) % 7937) for i in range(32))  # 256 ... 8192 tokens
    return [
        # one token of the 512-wide model that answers: the latency of a call
        _rotary("rotary-token", "1", 8, 8, 64, 32, False, False, 777, "bf16", False),
        # a training step of the paper's model: 32 sequences of 256 tokens, 8 heads of 64
        _rotary("rotary-train", _times(32, 256), 8, 8, 64, 32, True, False, 0, "bf16", True),
        # long texts at width 4096, frequencies scaled for them
        _rotary("rotary-long", _times(2, 8192), 32, 8, 128, 64, False, True, 0, "bf16", True),
        # 17 pairs of each head, where no half starts on a vector's boundary; far positions; single precision
        _rotary("rotary-part", "5003", 12, 4, 64, 17, False, False, 1000003, "f32", True),
        # the next token of 32 users into their caches
        _cache("append-tokens", "append", _times(32, 1), ragged, 32, 8, 128, 64, "bf16", pairs=64),
        # prompts of different lengths into a cache, at width 2048
        _cache("append-prompts", "append", "1,37,255,1024,2049,4321,8,505", "1,40,300,1024,2049,8000,8,505", 16, 8, 128, 64,
               "bf16", pairs=32, interleaved=True),
        # one token for one user: the latency of a call, with the learned bias
        _cache("attend-token", "attend", "1", "777", 8, 8, 64, 32, "bf16", bias=True),
        # the next token of 32 users over their caches
        _cache("attend-batch", "attend", _times(32, 1), ragged, 32, 8, 128, 64, "bf16"),
        # one token over one long text, whose keys gather weights
        _cache("attend-long", "attend", "1", "131072", 32, 8, 128, 256, "bf16", weigh=True),
        # a few tokens at once (drafts that are checked), odd lengths, bias and weights, single precision
        _cache("attend-few", "attend", "1,3,4,2,7", "129,1000,77,2500,611", 8, 4, 64, 32, "f32", bias=True, weigh=True),
        # a decoding step of 32 users under a budget: evict, append, attend
        _cache("step-budget", "step", _times(32, 1), _times(32, 2049), 32, 8, 128, 64, "bf16", pairs=64, weigh=True,
               budget=2048, recent=64),
        # prompts that are stored and cut down to a budget
        _cache("fill-budget", "fill", "8192,1000,5003,512,2049,4096,7777,1025", "8192,1000,5003,512,2049,4096,7777,1025", 32, 8,
               128, 128, "bf16", pairs=64, weigh=True, budget=1024, recent=32),
    ]


def _log_int(rng, low, high):
    return min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f32"])
    dim = rng.choice([32, 64, 128])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 2, 3, 4, 8])
    pairs = rng.choice([dim // 2, dim // 2, dim // 4, rng.randint(1, dim // 2)])
    kind = rng.choice(["rotary", "append", "attend", "attend", "step", "fill"])
    text = lambda lengths: ",".join(map(str, lengths))  # noqa: E731
    if kind == "rotary":
        total = _log_int(rng, 1, min(16384, (1 << 26) // ((heads + kv) * dim)))
        lengths = []
        while sum(lengths) < total and len(lengths) < 24:
            lengths.append(_log_int(rng, 1, total - sum(lengths)))
        c = _rotary("", text(lengths), heads, kv, dim, pairs, rng.random() < 0.5, rng.random() < 0.4,
                    rng.choice([0, 0, _log_int(rng, 1, 2000000)]), dtype, rng.random() < 0.7)
        del c["name"]
        return c
    page = rng.choice([32, 64, 128, 256])
    n = _log_int(rng, 1, 32)
    most = min(65536, (1 << 26) // (n * kv * dim))  # keys of a sequence: at most half of the largest case's elements
    rows = min(most, 8192, (1 << 26) // (n * (heads + 2 * kv) * dim))  # new ones of a sequence
    budget = recent = 0
    weigh = rng.random() < 0.5
    if kind == "append":
        queries = [_log_int(rng, 1, rows) for _ in range(n)] if rng.random() < 0.5 else [1] * n
        used = [nq + _log_int(rng, 1, max(1, most - nq)) - 1 for nq in queries]
    elif kind == "attend":
        what = rng.choice([1, 1, 8, 256])
        queries = [1 if what == 1 else _log_int(rng, 1, min(what, max(1, (1 << 26) // (n * heads * most)))) for _ in range(n)]
        used = [max(nq, _log_int(rng, 1, most)) for nq in queries]
    elif kind == "step":
        budget = _log_int(rng, 16, max(16, min(4096, most)))
        recent = _log_int(rng, 1, budget)
        queries, used = [1] * n, [budget + 1] * n
        weigh = True
    else:
        queries = [_log_int(rng, 1, rows) for _ in range(n)]
        used = queries
        budget = _log_int(rng, 16, 4096)
        recent = _log_int(rng, 1, budget)
        weigh = True
    c = _cache("", kind, text(queries), text(used), heads, kv, dim, page, dtype,
               0 if kind == "attend" else pairs, rng.random() < 0.5, kind == "attend" and rng.random() < 0.4, weigh, budget,
               recent)
    del c["name"]
    return c


def _lengths(text):
    return [int(n) for n in text.split(",")]


def _bucket_list():
    """Bucket of each distance -REACH ... REACH (key minus query): half of the buckets one distance each, the others growing
    as powers up to REACH; keys behind the query are met by none."""
    near = BUCKETS // 2
    n = BUCKETS - near

    def one(a):  # near + floor(log(a / near) / log(REACH / near) n), at most BUCKETS - 1, in whole numbers
        return a if a < near else near + sum(a ** n * near ** c >= near ** n * REACH ** c for c in range(1, n))

    return [one(max(-d, 0)) for d in range(-REACH, REACH + 1)]


def _frequencies(case):
    """(radians a token of each pair, in 64 bits; the factor of the rotated dimensions)."""
    n = case["pairs"]
    f = BASE ** (-np.arange(n, dtype=np.float64) / n)
    if not case.get("scaled"):
        return f, 1.0
    stays = np.clip((LENGTH * f / (2 * math.pi) - LOW) / (HIGH - LOW), 0, 1)
    return f * (stays + (1 - stays) / FACTOR), 0.1 * math.log(FACTOR) + 1


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = TYPES[case["dtype"]]
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]

    def new(*shape, dtype=dt, scale=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0, scale, generator=g)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32).cuda()

    nq = _lengths(case["queries"])
    s = {"case": case, "nq": ints(nq)}
    # slices of one projection's output
    x = new(sum(nq), (hq + 2 * hk) * d, scale=1.3)
    s["q"] = x[:, :hq * d].unflatten(1, (hq, d))
    s["xk"] = x[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
    s["xv"] = x[:, (hq + hk) * d:].unflatten(1, (hk, d))
    if case["pairs"]:
        f, s["magnitude"] = _frequencies(case)
        s["frequency"] = torch.from_numpy(f).cuda()
        # the same as turns a token in 64 bits behind the point
        turns = [int(t) % (1 << 64) for t in (float(v) / (2 * math.pi) * 2.0 ** 64 for v in f)]
        s["turns"] = torch.tensor([t - (1 << 64) if t >= 1 << 63 else t for t in turns]).cuda()
    if case["kind"] == "rotary":
        at = torch.cat([torch.arange(n, dtype=torch.int32) for n in nq]) + case["far"]
        s["at"] = at.cuda()
        if case["train"]:
            s["gq"], s["gk"] = new(sum(nq), hq, d), new(sum(nq), hk, d)
        return s
    used, page = _lengths(case["used"]), case["page"]
    most = max(used) + (1 if case["kind"] == "step" else 0)
    start = ints(np.concatenate([[0], np.cumsum(nq)]).tolist())
    s["plan"] = {"start_q": start, "start_k": start, "max_q": max(nq), "max_k": most}
    each = [-(-(n + (1 if case["kind"] == "step" else 0)) // page) for n in used]
    pages = torch.randperm(sum(each), generator=g, device="cuda").to(torch.int32).cpu()  # as they come free
    table = torch.full((len(used), max(each)), -1, dtype=torch.int32)
    first = np.concatenate([[0], np.cumsum(each)])
    for b, n in enumerate(each):
        table[b, :n] = pages[first[b]:first[b + 1]]
    s["table"] = table.cuda()
    elements = 128 // torch.finfo(dt).bits
    parts = 4 * elements
    s["k"] = new(sum(each), hk, page // 16, d // elements, 16, elements)
    s["v"] = new(sum(each), hk, page // parts, d // 16, 4, 16, elements)
    s["used"], s["seen"] = ints(used), ints(used)
    slots = torch.arange(max(each) * page, dtype=torch.int32, device="cuda")
    at = slots.expand(len(used), hk, -1)  # the order of the text, as long as nothing was evicted
    if case["kind"] == "step":  # what stayed of texts four times as long, the newest keys among it
        n, text = used[0], 4 * used[0]
        rank = torch.rand((len(used), hk, text), generator=g, device="cuda")
        rank[:, :, text - case["recent"]:] = 2
        at = at.clone()
        at[:, :, :n] = rank.argsort(2, descending=True)[:, :, torch.randperm(n, generator=g, device="cuda")].to(torch.int32)
        s["seen"] = ints([text] * len(used))
    s["position"] = torch.zeros((sum(each), hk, page), dtype=torch.int32, device="cuda")
    # what keys have gathered: nothing much at first, and sums over the steps before
    s["weight"] = torch.rand(s["position"].shape, generator=g, device="cuda") * (4.0 / most)
    mine = s["table"] >= 0
    s["position"][s["table"][mine].long()] = at.unflatten(2, (-1, page)).transpose(1, 2)[mine]
    if case["kind"] == "step":  # no two alike, so that a rounding decides nothing
        rank = torch.rand((hk, sum(each) * page), generator=g, device="cuda").argsort(1).float() / 1024
        s["weight"] = rank.unflatten(1, (-1, page)).transpose(0, 1).contiguous()
    if case["kind"] == "fill":  # a few keys get most of the weight, and many the same little
        s["given"] = (torch.exp(2 * torch.randn((sum(nq), hk), generator=g, device="cuda")) * 4).floor_() / 4
    if case["bias"]:
        s["w"] = new(hq, BUCKETS, scale=0.5)
        s["bucket"] = ints(_bucket_list())
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2107_03474_amd as lram

    case = s["case"]
    rotary = lram.Rotary(s["turns"], case["interleaved"], s["magnitude"]) if case["pairs"] else None
    if case["kind"] == "rotary":
        q, k = lram.rotary_forward(s["q"], s["xk"], s["at"], rotary)
        got = {"q": q, "k": k}
        if case["train"]:
            got["dq"], got["dk"] = lram.rotary_backward(s["gq"], s["gk"], s["at"], rotary)
        return got
    keys = lram.PagedKeys(s["k"], s["v"], s["position"], s["weight"])
    table = lram.PageTable(s["table"], s["used"], s["seen"])
    seqs = lram.Packed(**s["plan"])
    if case["kind"] == "attend":
        rel = lram.RelativeBias(s["w"], s["bucket"]) if case["bias"] else None
        got = {"out": lram.paged_attention(s["q"], keys, table, seqs, rel=rel, weigh=case["weigh"])}
        if case["weigh"]:
            got["weight"] = s["weight"]
        return got
    got = {"k": s["k"], "v": s["v"], "position": s["position"], "weight": s["weight"], "used": s["used"], "seen": s["seen"]}
    if case["kind"] == "append":
        got["q"] = lram.paged_append(s["xk"], s["xv"], keys, table, seqs, q=s["q"], rotary=rotary)
    elif case["kind"] == "step":
        lram.paged_evict(keys, table, case["budget"], case["recent"])
        lram.paged_shrink(table, case["budget"])
        lram.paged_extend(table, seqs)
        q = lram.paged_append(s["xk"], s["xv"], keys, table, seqs, q=s["q"], rotary=rotary)
        got["out"] = lram.paged_attention(q, keys, table, seqs, weigh=True)
    else:
        s["used"].zero_()  # new texts in the places of old ones
        s["seen"].zero_()
        lram.paged_extend(table, seqs)
        got["q"] = lram.paged_append(s["xk"], s["xv"], keys, table, seqs, q=s["q"], rotary=rotary, weight=s["given"])
        lram.paged_evict(keys, table, case["budget"], case["recent"])
        lram.paged_shrink(table, case["budget"])
    return got


def _turned(x, at, s, sign=1):
    """x [rows, heads, D] at these positions, rotated (backward: sign = -1)."""
    case = s["case"]
    n = case["pairs"]
    if not n:
        return x
    angle = sign * at.double()[:, None, None] * s["frequency"]
    c, z = (torch.cos(angle) * s["magnitude"]).float(), (torch.sin(angle) * s["magnitude"]).float()
    y = x.float()
    if case["interleaved"]:
        a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
        turned = torch.stack([a * c - b * z, a * z + b * c], -1).flatten(-2)
    else:
        a, b = y[..., :n], y[..., n:2 * n]
        turned = torch.cat([a * c - b * z, a * z + b * c], -1)
    return torch.cat([turned, y[..., 2 * n:]], -1).to(x.dtype)


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "rotary":
        got = {"q": _turned(s["q"], s["at"], s), "k": _turned(s["xk"], s["at"], s)}
        if case["train"]:
            got["dq"], got["dk"] = _turned(s["gq"], s["at"], s, -1), _turned(s["gk"], s["at"], s, -1)
        return got
    if case["kind"] == "attend":
        got = {"out": _plain_attention(s, s["q"])}
        if case["weigh"]:
            got["weight"] = s["weight"]
        return got
    got = {"k": s["k"], "v": s["v"], "position": s["position"], "weight": s["weight"], "used": s["used"], "seen": s["seen"]}
    if case["kind"] == "append":
        got["q"] = _plain_append(s, None)
    elif case["kind"] == "step":
        _plain_evict(s)
        s["used"] += s["nq"]
        s["seen"] += s["nq"]
        got["out"] = _plain_attention(s, _plain_append(s, None))
    else:
        s["used"].copy_(s["nq"])
        s["seen"].copy_(s["nq"])
        got["q"] = _plain_append(s, s["given"])
        _plain_evict(s)
    return got


def _v_parts(v):
    """The values with the last dimension in its two: [page, head, block, d / 16, part, d % 16, half, 4]."""
    return v.unflatten(-1, (-1, 4))


def _plain_append(s, given):
    page, dev = s["case"]["page"], s["q"].device
    nq, start = s["nq"].long(), s["plan"]["start_q"].long()
    row = torch.arange(s["q"].shape[0], device=dev)
    b = torch.searchsorted(start, row, right=True) - 1
    back = nq[b] - (row - start[b])  # rows from here to the sequence's end
    place, at = s["used"][b] - back, s["seen"][b] - back
    q, k = _turned(s["q"], at, s), _turned(s["xk"], at, s)
    p, t = s["table"][b, place // page].long(), place % page
    s["k"][p, :, t // 16, :, t % 16] = k.unflatten(2, (s["k"].shape[3], -1))
    v = _v_parts(s["v"])
    width = 16 * v.shape[6]
    v[p, :, t // width, :, t % 16 // 4, :, t % width // 16, t % 4] = s["xv"].unflatten(2, (-1, 16))
    s["position"][p, :, t] = at[:, None].to(torch.int32)
    s["weight"][p, :, t] = 0 if given is None else given
    return q


def _plain_keys(s, where):
    """(k, v [B, heads, keys, D] in 32 bits, position [B, heads, keys]) of these pages [B, n]."""
    at = s["position"][where].transpose(1, 2).flatten(2)
    k = s["k"][where].float().permute(0, 2, 1, 3, 5, 4, 6).flatten(5, 6).flatten(2, 4)
    v = _v_parts(s["v"])[where].float().permute(0, 2, 1, 3, 7, 5, 8, 4, 6).flatten(7, 8).flatten(2, 6)
    return k, v, at


def _plain_attention(s, q):
    """All sequences at once, each padded to the longest."""
    case, dev = s["case"], q.device
    hq, hk, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    group, start, nq = hq // hk, s["plan"]["start_q"].long(), s["nq"].long()
    where = s["table"].clamp(min=0).long()
    k, v, at = _plain_keys(s, where)
    j = torch.arange(k.shape[2], device=dev)
    i = torch.arange(s["plan"]["max_q"], device=dev)
    has_q, has_k = i < nq[:, None], j < s["used"][:, None]
    v.masked_fill_(~has_k[:, None, :, None], 0)
    rows = (start[:-1, None] + i).clamp(max=q.shape[0] - 1)
    x = (q[rows].float() * has_q[:, :, None, None]).unflatten(2, (hk, group)).permute(0, 2, 3, 1, 4)  # [B, hk, group, i, d]
    z = torch.matmul(x.flatten(2, 3), k.transpose(2, 3)).mul_(1 / math.sqrt(d)).unflatten(2, (group, -1))
    del k
    far = at[:, :, None] - (s["seen"][:, None] - s["nq"][:, None] + i)[:, None, :, None]  # [B, hk, i, j]
    seen = (far <= 0) & has_k[:, None, None, :] & has_q[:, None, :, None]
    if case["bias"]:
        of = s["bucket"].long()[far.clamp(-REACH, REACH) + REACH]
        one = torch.arange(hk, device=dev)[:, None, None, None] * group + torch.arange(group, device=dev)[:, None, None]
        z += s["w"].float()[one, of[:, :, None]]
    z.masked_fill_(~seen[:, :, None], float("-inf"))
    top = z.amax(4, keepdim=True)
    p = torch.exp(z.sub_(torch.where(torch.isfinite(top), top, 0)))
    del z
    total = p.sum(4, keepdim=True)
    p /= torch.where(total > 0, total, 1)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (group, -1)).permute(0, 3, 1, 2, 4).flatten(2, 3)
    if case["weigh"]:
        more = torch.where(has_k[:, None], p.sum((2, 3)), 0).unflatten(2, (-1, page)).transpose(1, 2)  # [B, page, hk, slot]
        mine = s["table"] >= 0
        s["weight"][where[mine]] += more[mine]
    return out[has_q].to(q.dtype)


def _plain_evict(s):
    case, dev = s["case"], s["k"].device
    page, budget, recent = case["page"], case["budget"], case["recent"]
    where = s["table"].clamp(min=0).long()
    at = s["position"][where].transpose(1, 2).flatten(2).long()
    weight = s["weight"][where].transpose(1, 2).flatten(2)
    slot = torch.arange(at.shape[2], device=dev)
    n = s["used"][:, None, None]
    # by newest, weight and position: the bits of what is not negative are in its order
    rank = (at >= s["seen"][:, None, None] - recent).long() << 62
    rank = rank | (weight.view(torch.int32).long() << 31) | ((1 << 31) - 1 - at)
    rank = torch.where(slot < n, rank, -1)
    order = torch.sort(rank, dim=2, descending=True, stable=True)[1]
    stays = torch.zeros_like(rank, dtype=torch.bool).scatter_(2, order[:, :, :budget], True) & (slot < n)
    far = at.shape[2]
    hole = torch.sort(torch.where(~stays & (slot < n) & (slot < budget), slot, far), dim=2)[0]
    moved = torch.sort(torch.where(stays & (slot >= budget), slot, far), dim=2)[0]
    b, h, i = (moved < far).nonzero(as_tuple=True)
    to, of = hole[b, h, i], moved[b, h, i]
    p0, p1, t0, t1 = where[b, of // page], where[b, to // page], of % page, to % page
    s["k"][p1, h, t1 // 16, :, t1 % 16] = s["k"][p0, h, t0 // 16, :, t0 % 16]
    v = _v_parts(s["v"])
    width = 16 * v.shape[6]
    v[p1, h, t1 // width, :, t1 % 16 // 4, :, t1 % width // 16, t1 % 4] = \
        v[p0, h, t0 // width, :, t0 % 16 // 4, :, t0 % width // 16, t0 % 4]
    s["position"][p1, h, t1] = s["position"][p0, h, t0]
    s["weight"][p1, h, t1] = s["weight"][p0, h, t0]
    s["used"].clamp_(max=budget)


# ---------------------------------------------------------------------------
# In 64 bits.

def _exact_turned(x, at, case, sign=1):
    n = case["pairs"]
    x = x.double()
    if not n:
        return x
    f, m = _frequencies(case)
    angle = sign * at.double()[:, None] * torch.from_numpy(f).to(x.device)
    unit = torch.polar(torch.full_like(angle, m), angle)[:, None]
    y = x.clone()
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if case["interleaved"] else (slice(0, n), slice(n, 2 * n))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * unit
    y[..., first], y[..., second] = z.real, z.imag
    return y


class _Store:
    """The pages' contents key by key: k, v [page, head, slot, D] in 64 bits."""

    def __init__(self, s):
        k, v = s["k"].double(), s["v"].double()
        self.shape_k, self.shape_v = k.shape, v.shape
        pages, heads, _, _, _, e = k.shape
        self.k = k.transpose(3, 4).reshape(pages, heads, -1, s["case"]["dim"])
        v = v.reshape(pages, heads, v.shape[2], v.shape[3], 4, 16, e // 4, 4)
        self.v = v.permute(0, 1, 2, 6, 4, 7, 3, 5).reshape(pages, heads, -1, s["case"]["dim"])
        self.weight, self.position = s["weight"].double(), s["position"].clone()

    def keys(self, table, n):
        pages = table.tolist()
        size = self.k.shape[2]
        pages = torch.tensor(pages[:-(-n // size)], device=self.k.device)
        return pages.repeat_interleave(size)[:n], torch.arange(n, device=self.k.device) % size

    def back(self):
        e = self.shape_k[5]
        k = self.k.unflatten(2, (-1, 16)).unflatten(4, (-1, e)).transpose(3, 4)
        v = self.v.unflatten(2, (-1, e // 4, 4, 4)).unflatten(6, (-1, 16)).permute(0, 1, 2, 6, 4, 7, 3, 5)
        return {"k": k.reshape(self.shape_k), "v": v.reshape(self.shape_v), "weight": self.weight, "position": None, "used": None,
                "seen": None}


def _exact_append(s, store, used, seen, given):
    case, typed = s["case"], s["q"].dtype
    got = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, n in enumerate(_lengths(case["queries"])):
        at = torch.arange(seen[b] - n, seen[b], device="cuda")
        got[row:row + n] = _exact_turned(s["q"][row:row + n], at, case)
        page, slot = (t[used[b] - n:] for t in store.keys(s["table"][b], used[b]))
        store.k[page, :, slot] = _exact_turned(s["xk"][row:row + n], at, case)
        store.v[page, :, slot] = s["xv"][row:row + n].double()
        store.position[page, :, slot] = at[:, None].to(torch.int32)
        store.weight[page, :, slot] = 0.0 if given is None else given[row:row + n].double()
        row += n
    return got, got.to(typed).double()  # what attention is given is of the type


def _exact_attention(s, store, q, used, seen, typed):
    case = s["case"]
    group = case["heads"] // case["kv_heads"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, n in enumerate(_lengths(case["queries"])):
        page, slot = store.keys(s["table"][b], used[b])
        at_q = torch.arange(seen[b] - n, seen[b], device="cuda")
        for h in range(case["kv_heads"]):
            k, v = store.k[page, h, slot], store.v[page, h, slot]
            far = store.position[page, h, slot][None] - at_q[:, None]
            x = q[row:row + n, h * group:(h + 1) * group].transpose(0, 1)
            z = x @ k.to(typed).double().t() / math.sqrt(case["dim"])
            if case["bias"]:
                z = z + s["w"][h * group:(h + 1) * group].double()[:, s["bucket"].long()[far.clamp(-REACH, REACH) + REACH]]
            z = z.masked_fill(far > 0, float("-inf"))
            none = torch.isinf(z).all(2, keepdim=True)
            p = torch.softmax(z.masked_fill(none, 0.0), 2).masked_fill(none, 0.0)
            out[row:row + n, h * group:(h + 1) * group] = (p @ v).transpose(0, 1)
            if case["weigh"]:
                store.weight[page, h, slot] += p.sum((0, 1))
        row += n
    return out


def _exact_evict(s, store, used, seen):
    case = s["case"]
    budget, recent = case["budget"], case["recent"]
    for b, n in enumerate(used):
        if n <= budget:
            continue
        page, slot = store.keys(s["table"][b], n)
        for h in range(case["kv_heads"]):
            at = store.position[page, h, slot].cpu().numpy().astype(np.int64)
            weight = store.weight[page, h, slot].cpu().numpy()
            best = np.lexsort((at, -weight, at < seen[b] - recent))[:budget]
            stays = np.zeros(n, bool)
            stays[best] = True
            of = np.nonzero(stays[budget:])[0] + budget
            to = np.nonzero(~stays[:budget])[0]
            of, to = torch.from_numpy(of).cuda(), torch.from_numpy(to).cuda()
            for t in (store.k, store.v, store.weight, store.position):
                t[page[to], h, slot[to]] = t[page[of], h, slot[of]]
    return [min(n, budget) for n in used]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        got = {"q": _exact_turned(s["q"], s["at"], case), "k": _exact_turned(s["xk"], s["at"], case)}
        if case["train"]:
            got["dq"], got["dk"] = _exact_turned(s["gq"], s["at"], case, -1), _exact_turned(s["gk"], s["at"], case, -1)
        return got
    store, typed = _Store(s), s["q"].dtype
    used, seen, nq = s["used"].tolist(), s["seen"].tolist(), _lengths(case["queries"])
    if case["kind"] == "attend":
        got = {"out": _exact_attention(s, store, s["q"].double(), used, seen, typed)}
        if case["weigh"]:
            got["weight"] = store.weight
        return got
    got = {}
    if case["kind"] == "append":
        got["q"] = _exact_append(s, store, used, seen, None)[0]
    elif case["kind"] == "step":
        used = [u + n for u, n in zip(_exact_evict(s, store, used, seen), nq)]
        seen = [u + n for u, n in zip(seen, nq)]
        q = _exact_append(s, store, used, seen, None)[1]
        got["out"] = _exact_attention(s, store, q, used, seen, typed)
    else:
        got["q"] = _exact_append(s, store, used, seen, s["given"])[0]
        _exact_evict(s, store, used, seen)
    return {**got, **store.back()}


def _moved(case, n):
    """Keys of a head that move when n are cut down to the budget, about: as many of those past it stay as of all."""
    budget = case["budget"]
    return 0 if n <= budget else max(1, (n - budget) * budget // n)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    nq = _lengths(case["queries"])
    rows = sum(nq)
    turns = 6 * case["pairs"] * rows * (hq + hk)  # products and sums of a rotation
    if case["kind"] == "rotary":
        both = 2 if case["train"] else 1
        return {"bytes": both * 2 * rows * (hq + hk) * d * size, "flops": both * turns}
    used, kind = _lengths(case["used"]), case["kind"]
    append = {"bytes": 2 * rows * (hq + 2 * hk) * d * size + 8 * rows * hk, "flops": turns}
    if kind == "append":
        return append
    evict = sum(8 * n * hk + _moved(case, n) * hk * (4 * d * size + 16) for n in used if n > case["budget"])
    if kind == "fill":
        return {"bytes": append["bytes"] + 4 * rows * hk + evict, "flops": turns}
    keys = [case["budget"] + 1] * len(used) if kind == "step" else used
    pairs = sum(sum(max(0, n - m + i + 1) for i in range(m)) for m, n in zip(nq, keys)) * hq
    attend = sum(keys) * hk * (2 * d * size + 8 * case["weigh"]) + 2 * rows * hq * d * size
    if kind == "attend":
        return {"bytes": attend, "flops": 4 * d * pairs}
    return {"bytes": append["bytes"] + evict + attend, "flops": 4 * d * pairs + turns}
