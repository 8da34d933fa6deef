"""What the operators of a generated token are measured on, beside its attention.

Text over the compact memory is generated token by token (`KVPages.append`,
`KVPages.attend`).  Around that lie, for a few rows at a time, products with weights
in 4 bits (`PackedWeight.product`: the fused projection whose rows `append` takes, the
output projection with its residual, and the vocabulary's logits), the choice of
the next tokens over beams and vocabulary (`beam_select`), and the pages that
the chosen beams go on with (`KVPages.reorder`: full pages are shared, a partly
filled one that two beams continue is copied).

A case is a dict of plain values:
  op         "product", "select" or "reorder"
"product"    x [rows][k] times the transpose of a weight [n][k]; bias, add (truth
             values): with a bias [n], with a residual [rows][n]; out "bf16" or "fp32"
"select"     seqs, beams, vocab, keep: the keep best continuations of every sequence;
             logits "bf16" or "fp32" in rows `pad` longer than the vocabulary; done: how many
             beams of a sequence have ended
"reorder"    layers, seqs, beams; heads, dim, fmt, page: of the pool; memory: tokens before the
             prompt in the first and the last layer, as text; made: tokens generated so far
"""
import math

import numpy as np
import torch

own = False

END = 2                        # the token that ends a sequence; ended beams repeat it
GROW = 1                       # a token is appended between two reorders


# --------------------------------------------------------------------- cases
def _product(rows, n, k, bias=False, add=False, out="bf16"):
    return dict(op="product", rows=rows, n=n, k=k, bias=bias, add=add, out=out)


def _select(seqs, beams, vocab, keep, logits="bf16", pad=0, done=0):
    return dict(op="select", seqs=seqs, beams=beams, vocab=vocab, keep=keep, logits=logits, pad=pad, done=done)


def _reorder(layers, seqs, beams, heads, dim, fmt, page, memory, made):
    return dict(op="reorder", layers=layers, seqs=seqs, beams=beams, heads=heads, dim=dim, fmt=fmt, page=page,
                memory=memory, made=made)


def listed():
    return [
        # the fused q, k, v projection of one token, 14/2 heads of 64: the smallest product
        dict(_product(1, 1152, 896, bias=True), name="product_qkv_0p5b_1row"),
        # the same of 28/4 heads of 128, for a token of each of 16 streams
        dict(_product(16, 4608, 3584, bias=True), name="product_qkv_7b_16rows"),
        # an output projection with its residual, of odd sizes
        dict(_product(5, 1003, 2236, add=True), name="product_odd_5rows"),
        # a question's 64 tokens through a layer four times as wide
        dict(_product(64, 14336, 3584), name="product_wide_64rows"),
        # the vocabulary's logits for two sequences of four beams: the largest weight
        dict(_product(8, 131072, 3584, out="fp32"), name="product_vocabulary_8rows"),
        # one answer's four beams over a small vocabulary
        dict(_select(1, 4, 32000, 4), name="select_1x4"),
        # odd sizes: rows of a padded vocabulary, ended beams, twice the beams kept
        dict(_select(3, 5, 49999, 10, logits="fp32", pad=17, done=2), name="select_odd_3x5"),
        # 16 answers of eight beams
        dict(_select(16, 8, 131072, 16), name="select_16x8"),
        # 32 answers of 16 beams in 32 bits: the largest choice
        dict(_select(32, 16, 131072, 32, logits="fp32"), name="select_32x16"),
        # one layer's pages of one answer
        dict(_reorder(1, 1, 4, 2, 64, "fp4", 64, "513,513", 21), name="reorder_0p5b_1layer"),
        # small pages in bf16, 24 layers, odd numbers of answers and beams
        dict(_reorder(24, 3, 5, 2, 64, "bf16", 16, "2048,2048", 150), name="reorder_0p5b_24layers"),
        # eight answers of eight beams over the compact memory of 28 layers
        dict(_reorder(28, 8, 8, 4, 128, "fp4", 64, "2048,6144", 100), name="reorder_7b_28layers"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["product", "select", "reorder"])
    if op == "product":
        rows, k = _log(rng, 1, 64), _log(rng, 64, 14336)
        n = _log(rng, 64, min(131072, 14336 * 3584 * 8 // (k * max(rows // 4, 1))))
        return _product(rows, n, k, bias=rng.random() < 0.4, add=rng.random() < 0.3, out=rng.choice(["bf16", "fp32"]))
    if op == "select":
        seqs, beams = _log(rng, 1, 32), rng.randint(1, 16)
        vocab = _log(rng, 100, 131072)
        keep = rng.choice([beams, 2 * beams])
        return _select(seqs, beams, vocab, keep, logits=rng.choice(["bf16", "fp32"]), pad=rng.choice([0, 0, 1, 40]),
                       done=rng.randint(0, beams - 1) if rng.random() < 0.4 else 0)
    heads, dim = rng.choice([(2, 64), (4, 128), (1, 64), (1, 128), (8, 128)])
    layers, seqs, beams = rng.choice([1, 1, 24, 28]), _log(rng, 1, 8), rng.randint(1, 8)
    if heads == 8:
        layers = 1
    first = _log(rng, 1, 6000)
    return _reorder(layers, seqs, beams, heads, dim, rng.choice(["fp4", "fp4", "bf16"]) if heads * dim < 512 else "fp4",
                    rng.choice([16, 32, 64]), f"{first},{first + rng.randint(0, 4000)}", rng.randint(0, 150))


def _lengths(case):
    """Rows of every (layer, sequence): before generation, and now."""
    low, high = (int(x) for x in case["memory"].split(","))
    n = case["layers"]
    start = [[low + (high - low) * i // max(n - 1, 1) + 37 + 11 * s for s in range(case["seqs"])] for i in range(n)]
    return start, [[t + case["made"] for t in row] for row in start]


def _row_bytes(case):
    """Bytes of a stored row of K and V of all heads."""
    d = case["dim"]
    return 2 * case["heads"] * (d // 2 + d // 32 if case["fmt"] == "fp4" else 2 * d)


def work(case):
    if case["op"] == "product":
        m, n, k = case["rows"], case["n"], case["k"]
        size = n * ((k + 31) // 32) * 17 + 2 * m * k + m * n * (2 if case["out"] == "bf16" else 4)
        return {"bytes": size + 2 * n * case["bias"] + 2 * m * n * case["add"], "flops": 2 * m * n * k}
    if case["op"] == "select":
        rows = case["seqs"] * case["beams"]
        live = case["seqs"] * (case["beams"] - case["done"]) * case["vocab"]
        # an element: compared, its difference to the largest, an exponential, added
        return {"bytes": live * (2 if case["logits"] == "bf16" else 4) + 8 * rows + 16 * case["seqs"] * case["keep"],
                "flops": 4 * live}
    b, page = case["beams"], case["page"]
    lens = [t for row in _lengths(case)[1] for t in row]
    entries = sum(2 * -(-(t + GROW) // page) for t in lens) * b
    # of b children of uniform parents, those beyond a parent's first copy its partly filled page
    # (all of them, while the prompt's page is the last one)
    copies = b - (b * (1 - (1 - 1 / b) ** b) if case["made"] > 0 else 0)
    rows = sum(-(-(t % page) // 4) * 4 for t in lens) * copies
    return {"bytes": int(4 * entries + 2 * rows * _row_bytes(case) + 8 * len(lens) * b), "flops": 0}


# -------------------------------------------------------------------- inputs
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1013 + stream)
    return g


def _randn(shape, g, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda") * scale


def _padded(values, width):
    """`values` [rows][n] in rows `width` long, as a view."""
    full = torch.zeros((values.shape[0], width), dtype=values.dtype, device="cuda")
    full[:, :values.shape[1]] = values
    return full[:, :values.shape[1]]


def _product_inputs(case, seed):
    m, n, k = case["rows"], case["n"], case["k"]
    g = _gen(seed, 1)
    s = {"case": case}
    s["weight"] = torch.empty((n, k), dtype=torch.bfloat16, device="cuda")
    for i in range(0, n, 16384):
        j = min(i + 16384, n)
        s["weight"][i:j] = _randn((j - i, k), g, 0.02)
    # normalised activations, a few channels of which stand out
    x = _randn((m, k), g)
    x[:, torch.randint(0, k, (max(k // 256, 1),), generator=g, device="cuda")] *= 12.0
    s["x"] = _padded(x.to(torch.bfloat16), -(-k // 8) * 8)
    s["bias"] = _randn((n,), g, 0.5).to(torch.bfloat16) if case["bias"] else None
    s["add"] = _randn((m, n), g, 2.0).to(torch.bfloat16) if case["add"] else None
    return s


def _select_inputs(case, seed):
    n_seqs, b, v = case["seqs"], case["beams"], case["vocab"]
    g = _gen(seed, 2)
    logits = _randn((n_seqs * b, v), g, 2.0)
    likely = torch.randint(0, v, (n_seqs * b, 24), generator=g, device="cuda")      # a context favours a few tokens
    logits.scatter_add_(1, likely, 4.0 + 6.0 * torch.rand(likely.shape, generator=g, device="cuda"))
    banned = torch.randint(0, v, (max(v // 500, 1),), generator=g, device="cuda")
    logits[:, banned] = -math.inf
    dtype = torch.bfloat16 if case["logits"] == "bf16" else torch.float32
    s = {"case": case, "logits": _padded(logits.to(dtype), v + case["pad"]).unflatten(0, (n_seqs, b))}
    s["score"] = -8.0 - 6.0 * torch.rand((n_seqs, b), generator=g, device="cuda")
    s["done"] = None
    if case["done"] > 0:
        order = torch.rand((n_seqs, b), generator=g, device="cuda").argsort(1)
        s["done"] = (order < case["done"]).to(torch.int32)
    return s


def _reorder_inputs(case, seed):
    """Tables of beams that have a memory and a prompt in common, and then pages of
    their own, or of the beam that they once split from."""
    rng = np.random.default_rng((seed, 3))
    layers, n_seqs, b, page = case["layers"], case["seqs"], case["beams"], case["page"]
    start, now = _lengths(case)
    made = case["made"]
    most = -(-(max(map(max, now)) + GROW) // page)
    tables = np.full((layers, n_seqs, b, most), -1, dtype=np.int32)
    shared = 0                                         # pages outside the rooms: memory, prompts
    for i in range(layers):
        memory = (start[i][0] - 37) // page            # full pages that all answers read
        for s in range(n_seqs):
            have = -(-start[i][s] // page)
            tables[i, s, :, :memory] = np.arange(shared, shared + memory)
            first = shared + memory + 12 * s
            tables[i, s, :, memory:have] = np.arange(first, first + have - memory)
        shared += memory + 12 * n_seqs
    spread = made // page + 2                          # pages that a beam may have for itself
    size = b * (spread + 2)
    room = np.zeros((layers, n_seqs, 2), dtype=np.int32)
    at = shared
    for i in range(layers):
        for s in range(n_seqs):
            room[i, s] = (at, size)
            if made > 0:
                ids = at + rng.permutation(size)
                first, total, used = start[i][s] // page, -(-now[i][s] // page), 0
                for j in range(b):
                    split = first
                    if j > 0:
                        split = int(rng.integers(first, total))
                        tables[i, s, j] = tables[i, s, int(rng.integers(0, j))]
                    n = total - split
                    tables[i, s, j, split:total] = ids[used:used + n]
                    used += n
            at += size
    s = {"case": case}
    s["n_pages"] = at
    s["tables"] = torch.from_numpy(tables).cuda()
    s["room"] = torch.from_numpy(room).cuda()
    lens = np.broadcast_to(np.asarray(now, dtype=np.int32)[:, :, None], (layers, n_seqs, b))
    s["kv_len"] = torch.from_numpy(np.ascontiguousarray(lens)).cuda()
    s["parent"] = torch.from_numpy(rng.integers(0, b, (n_seqs, b)).astype(np.int32)).cuda()
    s["pages"] = torch.randint(0, 120, (at, page * _row_bytes(case)), generator=_gen(seed, 3), dtype=torch.uint8,
                               device="cuda")
    return s


def prepare(case, seed):
    if case["op"] == "product":
        s = _product_inputs(case, seed)
        dense = s.pop("weight")
        if own:
            from paper_2601_14724_amd import hermes
            s["w"] = hermes.PackedWeight(dense)
        else:
            s["codes"], s["scales"] = _quantised(dense)
        return s
    if case["op"] == "select":
        return _select_inputs(case, seed)
    s = _reorder_inputs(case, seed)
    if own:
        from paper_2601_14724_amd import hermes
        fmt = hermes.PAGE_FP4 if case["fmt"] == "fp4" else hermes.PAGE_BF16
        s["pool"] = hermes.KVPages(case["heads"], case["heads"], case["dim"], s["n_pages"], page_rows=case["page"],
                                   fmt=fmt, pages=s["pages"])
    return s


# --------------------------------------------------------------------- a pass
def run(state):
    case = state["case"]
    if not own:
        return {"product": _plain_product, "select": _plain_select, "reorder": _plain_reorder}[case["op"]](state)
    if case["op"] == "product":
        dtype = torch.bfloat16 if case["out"] == "bf16" else torch.float32
        return state["w"].product(state["x"], bias=state["bias"], add=state["add"], dtype=dtype)
    if case["op"] == "select":
        from paper_2601_14724_amd import hermes
        score, parent, token, done = hermes.beam_select(state["logits"], state["score"], case["keep"],
                                                        done=state["done"], end_token=END, pad_token=END)
        return {"score": score, "parent": parent, "token": token, "done": done}
    tables, kv_len = state["pool"].reorder(state["tables"], state["kv_len"], state["parent"], state["room"], grow=GROW)
    return {"tables": tables, "len": kv_len, "pages": state["pages"]}


_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _blocks(w):
    """w [n][k] -> [n][k / 32, rounded up][32], zeros behind the end."""
    n, k = w.shape
    full = torch.zeros((n, -(-k // 32) * 32), dtype=w.dtype, device=w.device)
    full[:, :k] = w
    return full.unflatten(1, (-1, 32))


def _quantised(w):
    """4-bit codes (a byte each) and scale bytes of a weight, 32 inputs a block."""
    n, k = w.shape
    codes = torch.empty((n, -(-k // 32), 32), dtype=torch.uint8, device=w.device)
    scales = torch.empty((n, -(-k // 32)), dtype=torch.uint8, device=w.device)
    for i in range(0, n, 16384):
        b = _blocks(w[i:i + 16384]).float()
        amax = b.abs().amax(-1)
        _, ex = torch.frexp(amax)                      # amax = m 2^ex, m in [1/2, 1)
        e = torch.where(amax <= torch.ldexp(torch.full_like(amax, 7.0), ex - 3), ex - 3, ex - 2)
        e = torch.where(amax == 0, torch.full_like(e, -119), e).clamp(-119, 125)
        m = torch.ldexp(b.abs(), -e.unsqueeze(-1))
        c = (m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)
        codes[i:i + 16384] = c + 8 * torch.signbit(b).to(torch.uint8)
        scales[i:i + 16384] = (e + 127).to(torch.uint8)
    return codes, scales


def _plain_product(s):
    case = s["case"]
    x = s["x"].float()
    out = torch.empty((case["rows"], case["n"]), device="cuda")
    table = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), device="cuda")
    for i in range(0, case["n"], 16384):
        w = torch.ldexp(table[s["codes"][i:i + 16384].int()], s["scales"][i:i + 16384].int().unsqueeze(-1) - 127)
        out[:, i:i + 16384] = x @ w.flatten(1)[:, :case["k"]].T
    if s["bias"] is not None:
        out += s["bias"].float()
    if s["add"] is not None:
        out += s["add"].float()
    return out if case["out"] == "fp32" else out.to(torch.bfloat16)


def _plain_select(s):
    case = s["case"]
    keep, v = case["keep"], case["vocab"]
    score, x = s["score"].double(), s["logits"].double()          # 64 bits: beams meet by their sums
    top = x.amax(-1, keepdim=True)
    lse = (x - top).exp_().sum(-1).log() + top.squeeze(-1)
    value = x + (score - lse).unsqueeze(-1)
    if s["done"] is not None:
        ended = s["done"].bool()
        value[ended] = -math.inf
        value[..., END] = torch.where(ended, score, value[..., END])
    value, index = value.flatten(1).sort(dim=1, descending=True, stable=True)
    value, index = value[:, :keep], index[:, :keep].int()
    parent, token = torch.div(index, v, rounding_mode="floor"), index % v
    none = value == -math.inf
    parent, token = parent.masked_fill(none, -1), token.masked_fill(none, -1)
    done = token == END
    if s["done"] is not None:
        done |= s["done"].gather(1, parent.clamp_min(0).long()).bool() & ~none
    return {"score": value.float(), "parent": parent, "token": token, "done": done.int()}


def _group_of_byte(case, device):
    """Of every byte of a page, which four rows it belongs to."""
    page, d = case["page"], case["dim"]
    row = d // 2 if case["fmt"] == "fp4" else 2 * d
    group = torch.arange(page // 4, device=device)
    parts = [group.repeat_interleave(4 * row)] * 2
    if case["fmt"] == "fp4":
        parts += [group.repeat_interleave(4 * (d // 32))] * 2
    return torch.cat(parts).repeat(case["heads"])


def _plain_reorder(s):
    case = s["case"]
    page, b = case["page"], case["beams"]
    layers, n_seqs, most = case["layers"], case["seqs"], s["tables"].shape[-1]
    parent = s["parent"].long().expand(layers, -1, -1)
    table = s["tables"].long().gather(2, parent.unsqueeze(-1).expand(-1, -1, -1, most)).flatten(0, 1)   # [groups][b][most]
    kv_len = s["kv_len"].gather(2, parent)
    n = kv_len.long().flatten(0, 1)
    full, part = n // page, n % page > 0
    entry = torch.arange(most, device="cuda")
    shared = entry < full.unsqueeze(-1)
    used = torch.zeros(s["n_pages"], dtype=torch.bool, device="cuda")
    used[table[shared]] = True
    first, size = s["room"].long().flatten(0, 1).unbind(-1)
    last = table.gather(2, full.clamp_max(most - 1).unsqueeze(-1)).squeeze(-1)      # the partly filled page
    earlier = torch.ones((b, b), dtype=torch.bool, device="cuda").tril(-1)
    again = ((last.unsqueeze(-1) == last.unsqueeze(-2)) & part.unsqueeze(-2) & earlier).any(-1)
    inside = (last >= first.unsqueeze(-1)) & (last < (first + size).unsqueeze(-1))
    kept = part & inside & ~again & ~used[last.clamp_min(0)]
    used[last[kept]] = True
    need = (n + GROW + page - 1) // page - full - kept.long()
    place = need.cumsum(1) - need
    ids = first.unsqueeze(-1) + torch.arange(int(size.max()), device="cuda")
    free = (ids < (first + size).unsqueeze(-1)) & ~used[ids.clamp_max(s["n_pages"] - 1)]
    ids = torch.where(free, ids, -1).gather(1, (~free).int().sort(dim=1, stable=True).indices)
    own_entry = entry - (full + kept.long()).unsqueeze(-1)                            # which of its new pages
    at = (place.unsqueeze(-1) + own_entry).clamp(0, ids.shape[1] - 1)
    given = ids.gather(1, at.flatten(1)).view_as(at)
    out = torch.where(shared, table, -1)
    out = torch.where(kept.unsqueeze(-1) & (entry == full.unsqueeze(-1)), last.unsqueeze(-1), out)
    out = torch.where((own_entry >= 0) & (own_entry < need.unsqueeze(-1)), given, out)
    copied = part & ~kept
    target = out.gather(2, full.clamp_max(most - 1).unsqueeze(-1)).squeeze(-1)[copied]
    groups = ((n % page + 3) // 4)[copied]
    live = _group_of_byte(case, "cuda").unsqueeze(0) < groups.unsqueeze(-1)
    pages = s["pages"]
    pages[target] = torch.where(live, pages[last[copied]], pages[target])
    return {"tables": out.int().view(layers, n_seqs, b, most), "len": kv_len, "pages": pages}


# ------------------------------------------------------ from the definition, 64 bits
def _nearest(b):
    """What blocks [..][32] of fp64 values stand for in 4 bits: the scale is the least
    power of two of which seven cover the largest magnitude; a value goes to the nearest
    level, a tie to the even one."""
    top = b.abs().amax(-1, keepdim=True)
    step = torch.full_like(top, 2.0 ** -119)
    for e in range(-40, 20):
        step = torch.where(top > 7.0 * 2.0 ** (e - 1), torch.full_like(top, 2.0 ** e), step)
    ratio = b.abs() / step
    best, err = torch.zeros_like(ratio), ratio.clone()
    for i in (2, 4, 6, 1, 3, 5, 7):                    # the even ones first, so that they keep a tie
        gap = (ratio - _LEVELS[i]).abs()
        best, err = torch.where(gap < err, _LEVELS[i], best), torch.minimum(gap, err)
    return best * step * torch.sign(b)


def _exact_product(case, seed):
    s = _product_inputs(case, seed)
    x = s["x"].double()
    out = torch.empty((case["rows"], case["n"]), dtype=torch.float64, device="cuda")
    for i in range(0, case["n"], 4096):
        w = _nearest(_blocks(s["weight"][i:i + 4096]).double()).flatten(1)[:, :case["k"]]
        out[:, i:i + 4096] = torch.mm(w, x.T.contiguous()).T
    for extra in (s["bias"], s["add"]):
        if extra is not None:
            out = out + extra.double()
    return out


def _exact_select(case, seed):
    s = _select_inputs(case, seed)
    n_seqs, b, v, keep = case["seqs"], case["beams"], case["vocab"], case["keep"]
    result = {"score": np.full((n_seqs, keep), -np.inf), "parent": np.full((n_seqs, keep), -1),
              "token": np.full((n_seqs, keep), -1), "done": np.zeros((n_seqs, keep))}
    for q in range(n_seqs):
        found = []
        for j in range(b):
            total = float(s["score"][q, j])
            if s["done"] is not None and int(s["done"][q, j]):
                found.append((-total, j, END, 1))
                continue
            row = s["logits"][q, j].double()
            value = row + (total - float(torch.logsumexp(row, 0)))
            # its keep best with all that tie with the last of them
            edge = float(value.topk(min(keep, v)).values[-1])
            places = torch.nonzero(value >= edge).flatten()
            for t, x in zip(places.tolist(), value[places].tolist()):
                if x > -math.inf:
                    found.append((-x, j, t, int(t == END)))
        for i, (x, j, t, ended) in enumerate(sorted(found)[:keep]):
            result["score"][q, i], result["parent"][q, i], result["token"][q, i] = -x, j, t
            result["done"][q, i] = ended
    return {"score": torch.from_numpy(result["score"]).cuda(),
            **{k: torch.from_numpy(result[k].astype(np.int32)).cuda() for k in ("parent", "token", "done")}}


def _exact_reorder(case, seed):
    s = _reorder_inputs(case, seed)
    page, b, heads, d = case["page"], case["beams"], case["heads"], case["dim"]
    old, room = s["tables"].cpu().numpy(), s["room"].cpu().numpy()
    lens, parent, pages = s["kv_len"].cpu().numpy(), s["parent"].cpu().numpy(), s["pages"]
    out, new_lens = np.full_like(old, -1), np.zeros_like(lens)
    row = d // 2 if case["fmt"] == "fp4" else 2 * d
    sizes = [row, row] + ([d // 32, d // 32] if case["fmt"] == "fp4" else [])        # of a row, part by part
    for i in range(case["layers"]):
        for q in range(case["seqs"]):
            first, size = room[i, q]
            held, tails, copies = set(), {}, []
            for j in range(b):
                new_lens[i, q, j] = n = lens[i, q, parent[q, j]]
                out[i, q, j, :n // page] = old[i, q, parent[q, j], :n // page]
                held.update(out[i, q, j, :n // page].tolist())
            for j in range(b):
                n = new_lens[i, q, j]
                last = int(old[i, q, parent[q, j], n // page]) if n % page else -1
                if n % page and first <= last < first + size and last not in held and last not in tails.values():
                    tails[j] = last
            free = iter(x for x in range(first, first + size) if x not in held and x not in set(tails.values()))
            for j in range(b):
                n = new_lens[i, q, j]
                for e in range(n // page, -(-(n + GROW) // page)):
                    if e == n // page and j in tails:
                        out[i, q, j, e] = tails[j]
                        continue
                    out[i, q, j, e] = next(free)
                    if n % page and e == n // page:
                        copies.append((int(old[i, q, parent[q, j], e]), int(out[i, q, j, e]), -(-(n % page) // 4) * 4))
            for source, target, rows in copies:
                a, c = pages[source].view(heads, -1), pages[target].view(heads, -1)
                at = 0
                for part in sizes:
                    c[:, at:at + rows * part] = a[:, at:at + rows * part]
                    at += page * part
    return {"tables": torch.from_numpy(out).cuda(), "len": torch.from_numpy(new_lens).cuda(), "pages": pages}


def exact(case, seed):
    return {"product": _exact_product, "select": _exact_select, "reorder": _exact_reorder}[case["op"]](case, seed)
