"""Operators between two attention calls of a rollout step, as a rollout program calls them.

* ``pages``: the page table of all segments, grown from their lengths and a list of free pages
  (``page_table``);
* ``slots``: slot word, position and branch of every new token (``slot_map``);
* ``qkv``: norms of queries and keys for each head, the position rotation, and the write of K and V into
  the pool's pages (``qkv_append``);
* ``logits``: penalties for the tokens on a branch's path, biases and grammar masks (``process_logits``).

Head shapes and graph sizes are those of the package's own configurations (trees, merged graphs, long
reasoning, prompts, at 7B and 32B head shapes); vocabularies are generic.  A graph's structure follows
from the case alone, the page placement and all values from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
NAMES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ----------------------------------------------------------------------------------------------
# The cases
# ----------------------------------------------------------------------------------------------

def graph_case(name, op, prompts, fans, root, step, shape=1, **more):
    """A forest: `prompts` roots of up to root tokens, at every level `fans` children of up to step tokens each."""
    c = {"op": op, "prompts": prompts, "fans": fans, "root": root, "step": step, "shape": shape, **more}
    return {"name": name, **c} if name else c


def qkv_case(name, tokens, hq, hkv, dim, dtype, rotary, far, interleaved=False, norm=True, shape=1):
    c = {"op": "qkv", "tokens": tokens, "hq": hq, "hkv": hkv, "dim": dim, "dtype": dtype, "rotary": rotary, "far": far,
         "interleaved": interleaved, "norm": norm, "shape": shape}
    return {"name": name, **c} if name else c


def listed():
    return [
        # A small rollout batch's table before a step: 16 step trees, each segment with the room of its next token.
        graph_case("pages_tree", "pages", 16, "2 2 2", 512, 384, spare=1, known=1.0),
        # The tables of a whole training batch's segments, half of them new, each with room for 256 tokens.
        graph_case("pages_batch", "pages", 512, "2 2 2 2 1", 2048, 1024, spare=256, known=0.5),
        # A decode step's slots: 1024 branches of 64 graphs, one token each.
        graph_case("slots_step", "slots", 64, "2 2 2 2 1 1", 1024, 1024, new=1),
        # Every token of 256 prompts of up to 16384 tokens, for their prefill.
        graph_case("slots_prompts", "slots", 256, "", 16384, 1, new=0),
        # The smallest call: one branch's token, a 7B layer.
        qkv_case("qkv_one_7b", 1, 28, 4, 128, "bf16", 128, 4000),
        # A decode step of 1024 branches, a 7B layer.
        qkv_case("qkv_step_7b", 1024, 28, 4, 128, "bf16", 128, 16384),
        # The prompts of a batch at a 32B layer.
        qkv_case("qkv_prompts_32b", 32768, 40, 8, 128, "bf16", 128, 4096),
        # A model of 64-wide heads in float32, half of the channels rotated in neighbouring pairs, no norms, far positions.
        qkv_case("qkv_f32_d64", 777, 16, 2, 64, "f32", 32, 1000000, interleaved=True, norm=False),
        # One prompt's branch, its next token's logits.
        graph_case("logits_one", "logits", 1, "1 1", 512, 384, vocab=32000, dtype="bf16", wide=True, bias=16, masks=0,
                   drafts=1),
        # 128 branches of 16 trees under grammar masks, a vocabulary of odd size.
        graph_case("logits_tree_odd", "logits", 16, "2 2 2", 512, 384, vocab=50001, dtype="bf16", wide=False, bias=300,
                   masks=40, drafts=1),
        # The training batch's step: 1024 branches, float32 logits, penalties and a few biases.
        graph_case("logits_batch", "logits", 64, "2 2 2 2 1 1", 1024, 1024, vocab=152064, dtype="f32", wide=False, bias=4,
                   masks=0, drafts=1),
        # Four drafted tokens of 256 long branches checked at once.
        graph_case("logits_long_drafts", "logits", 32, "1 1 8 1", 8192, 2700, vocab=65024, dtype="bf16", wide=True, bias=0,
                   masks=8, drafts=4),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(28, 4, 128), (40, 8, 128), (32, 8, 128), (16, 2, 64), (12, 12, 64), (8, 1, 128)]


def draw(rng):
    op = rng.choice(["pages", "slots", "qkv", "qkv", "qkv", "logits", "logits", "logits"])
    shape = rng.randrange(1, 1 << 20)
    if op == "qkv":
        hq, hkv, dim = rng.choice(_HEADS)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rotary = rng.choice([dim, dim, dim // 2, 16, 0])
        return qkv_case("", _spread(rng, 1, 30000 if dtype == "bf16" else 12000), hq, hkv, dim, dtype, rotary,
                        _spread(rng, 10, 1000000), rng.random() < 0.3, rng.random() < 0.7, shape)
    if op == "pages":
        return graph_case("", op, _spread(rng, 1, 450), rng.choice(["", "2", "3 2", "2 2 2 1", "2 2 2 2 1"]),
                          _spread(rng, 1, 2000), _spread(rng, 1, 1000), shape, spare=rng.randrange(0, 250),
                          known=round(rng.random(), 3))
    if op == "slots":
        new = rng.choice([0, 1, _spread(rng, 2, 24)])
        fans = rng.choice(["", "5", "2 2 2", "2 2 2 2 1 1"])
        return graph_case("", op, _spread(rng, 1, 250 if fans == "" else 64), fans, _spread(rng, 1, 16000 if fans == "" else 2000),
                          _spread(rng, 1, 1500), shape, new=new)
    vocab = _spread(rng, 1000, 152064)
    dtype = rng.choice(["f32", "bf16"])
    fans = rng.choice(["", "5", "2 2 2", "1 1 8 1"])
    most = math.prod(int(x) for x in fans.split())
    drafts = rng.choice([1, 1, rng.randrange(2, 6)])
    prompts = _spread(rng, 1, max(1, min(256, 60_000_000 // (vocab * most * drafts))))
    return graph_case("", op, prompts, fans, _spread(rng, 8, 8000), _spread(rng, 8, 2000), shape, vocab=vocab, dtype=dtype,
                      wide=rng.random() < 0.5, bias=rng.choice([0, 1, _spread(rng, 2, 600)]),
                      masks=rng.choice([0, 1, _spread(rng, 2, 64)]), drafts=drafts)


# ----------------------------------------------------------------------------------------------
# Rollout graphs: segment lengths and every branch's segments
# ----------------------------------------------------------------------------------------------

def _structure(case):
    """(lens [S], paths [B, levels]): levels of segments, the first prompts' roots."""
    rng = np.random.default_rng(7919 * case["shape"] + 13)
    width = case["prompts"] * np.cumprod([1] + [int(x) for x in case["fans"].split()])
    first = np.concatenate([[0], np.cumsum(width)])
    leaf = np.arange(width[-1])
    paths = np.stack([first[i] + leaf // (width[-1] // w) for i, w in enumerate(width)], 1)
    # (a segment that the drafted tokens end has at least those)
    lo = case.get("drafts", 1)
    top = np.maximum(np.where(np.arange(first[-1]) < width[0], case["root"], case["step"]), lo)
    return np.maximum(lo, rng.integers((top + 3) // 4, top + 1)).astype(np.int32), paths


def _pages(lens, seed):
    """A seeded placement of whole pages of 16 tokens: offsets [S + 1], pages, pages of the pool."""
    off = np.concatenate([[0], np.cumsum((lens.astype(np.int64) + 15) // 16)])
    total = int(off[-1]) + 3
    return off, np.random.default_rng(seed + 77).permutation(total)[:off[-1]].astype(np.int32), total


def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed(1_000_003 * int(seed) + stream)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _graph(case, seed):
    """The graph on the device, as the calls take it."""
    lens, paths = _structure(case)
    off, pages, total = _pages(lens, seed)
    at = np.arange(len(paths) + 1, dtype=np.int64) * paths.shape[1]
    return {"lens": _dev(lens), "off": _dev(off), "pages": _dev(pages), "total": total, "path_off": _dev(at),
            "paths": _dev(paths.astype(np.int32))}


def _device_graph(g):
    from paper_2606_18954_amd import graphattn as ga
    return ga.DeviceGraph(g["lens"], g["off"], g["pages"], g["path_off"], g["paths"].flatten(), g["total"])


# ----------------------------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------------------------

def _pages_inputs(case, seed):
    """Segment lengths now, the table from before (the first segments, when they were shorter) and free pages."""
    lens, _ = _structure(case)
    known = int(round(case["known"] * len(lens)))
    before = np.maximum(1, lens[:known] - np.random.default_rng(case["shape"]).integers(0, 40, known))
    off = np.concatenate([[0], np.cumsum((before.astype(np.int64) + case["spare"] + 15) // 16)])
    need = int(((lens.astype(np.int64) + case["spare"] + 15) // 16).sum()) + 64
    order = np.random.default_rng(seed + 5).permutation(int(off[-1]) + need).astype(np.int32)
    return {"lens": _dev(lens), "old_off": _dev(off), "old_pages": _dev(order[:off[-1]]), "free": _dev(order[off[-1]:]),
            "spare": case["spare"]}


def _slots_inputs(case, seed):
    st = _graph(case, seed)
    last = st["lens"][st["paths"][:, -1].long()]
    if case["new"] == 0:
        st["counts"] = last.clone()                        # all of them
    else:
        most = np.random.default_rng(case["shape"]).integers(1, case["new"] + 1, len(last), dtype=np.int32)
        st["counts"] = torch.minimum(_dev(most), last)
    # The buffers are those of the largest step: a few rows of padding.
    st["capacity"] = int(st["counts"].sum()) + 8
    return st


def _qkv_inputs(case, seed):
    n, hq, hkv, dim = case["tokens"], case["hq"], case["hkv"], case["dim"]
    dt, g = NAMES[case["dtype"]], _gen(seed, 1)
    # One projection's rows, q, k and v side by side; keys and queries with a spread of channel sizes.
    size = torch.exp(0.3 * torch.randn(hq + 2 * hkv, dim, generator=g, device=DEV))
    rows = (torch.randn(n, hq + 2 * hkv, dim, generator=g, device=DEV) * size).to(dt)
    total = n // 12 + 2
    words = torch.randperm(total * 16, generator=g, device=DEV)[:n].int()
    # A few tokens are on their path already (their queries alone are wanted), a few rows are padding.
    u = torch.rand(n, generator=g, device=DEV)
    words = torch.where(u < 0.01, -1, words)
    pos = torch.randint(0, case["far"], (n,), generator=g, device=DEV, dtype=torch.int32)
    pos = torch.where((u > 0.99) & (n > 1), -1, pos)
    half = case["rotary"] // 2
    st = {"rows": rows, "words": words, "pos": pos, "total": total, "rotary": case["rotary"], "hq": hq, "hkv": hkv,
          "interleaved": case["interleaved"], "q_norm": None, "k_norm": None,
          "freq": 10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / max(half, 1))}
    if case["norm"]:
        st["q_norm"] = 1 + 0.2 * torch.randn(dim, generator=g, device=DEV)
        st["k_norm"] = 1 + 0.2 * torch.randn(dim, generator=g, device=DEV)
    return st


def _logits_inputs(case, seed):
    st = _graph(case, seed)
    B, drafts, vocab = len(st["paths"]), case["drafts"], case["vocab"]
    R, g = B * drafts, _gen(seed, 1)
    st["logits"] = (3.0 * torch.randn(R, vocab, generator=g, device=DEV)).to(NAMES[case["dtype"]])
    # Some tokens come often; a few slots hold none (an image's, say).
    u = torch.rand(st["total"] * 16, generator=g, device=DEV)
    ids = (vocab * u ** 3).int().clamp(max=vocab - 1)
    st["ids"] = torch.where(torch.rand(u.shape, generator=g, device=DEV) < 0.01, -1, ids)
    length = st["lens"][st["paths"].long()].sum(1)
    st["longest"] = int(length.max())
    row = torch.arange(R, device=DEV)
    st["branch"] = (row // drafts).int()
    st["pos"] = (length[row // drafts] - drafts + row % drafts).int()
    st["rep"] = 1 + 0.5 * torch.rand(R, generator=g, device=DEV)
    st["freq"] = 0.5 * torch.rand(R, generator=g, device=DEV)
    st["pres"] = torch.rand(R, generator=g, device=DEV)
    st["temp"] = 0.5 + torch.rand(R, generator=g, device=DEV)
    if case["bias"]:
        n = min(case["bias"], vocab)
        # (ascending tokens: a step of at least one between neighbours)
        gap = torch.rand(R, n, generator=g, device=DEV) * (vocab - n) / n
        st["bias_tokens"] = (gap.cumsum(1).long().clamp(max=vocab - n) + torch.arange(n, device=DEV)).int().flatten()
        st["bias_values"] = 4 * torch.randn(R * n, generator=g, device=DEV)
        st["bias_off"] = torch.arange(R + 1, device=DEV) * n
    if case["masks"]:
        words = (vocab + 31) // 32
        a, b = (torch.randint(-2**31, 2**31, (case["masks"], words), generator=g, device=DEV) for _ in range(2))
        # Grammars that allow a quarter of the tokens or three quarters of them; some rows have none.
        st["masks"] = torch.where(torch.arange(case["masks"], device=DEV)[:, None] % 2 == 0, a & b, a | b).int()
        st["mask_of"] = torch.randint(-1, case["masks"], (R,), generator=g, device=DEV, dtype=torch.int32)
    return st


def prepare(case, seed):
    op = case["op"]
    st = {"pages": _pages_inputs, "slots": _slots_inputs, "qkv": _qkv_inputs, "logits": _logits_inputs}[op](case, seed)
    st["op"] = op
    # What a call writes.
    if op == "pages":
        n = st["old_pages"].numel() + st["free"].numel()
        st["new_off"] = torch.zeros(st["lens"].numel() + 1, dtype=torch.int64, device=DEV)
        st["new_pages"] = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    elif op == "slots":
        st["token_off"] = torch.zeros(st["counts"].numel() + 1, dtype=torch.int32, device=DEV)
        st["out"] = [torch.zeros(st["capacity"], dtype=torch.int32, device=DEV) for _ in range(3)]
    elif op == "qkv":
        dim, dt = case["dim"], NAMES[case["dtype"]]
        st["q_out"] = torch.zeros(case["tokens"], case["hq"], dim, dtype=dt, device=DEV)
        # (a page behind the pool's takes what the plain form writes for tokens that are not stored)
        st["pool"] = torch.zeros(st["total"] + 1, case["hkv"], 2, 16, dim, dtype=dt, device=DEV)
    else:
        wide = case["wide"] or case["dtype"] == "f32"
        st["out"] = torch.zeros_like(st["logits"], dtype=torch.float32 if wide else torch.bfloat16)
        st["prompt_segments"] = 1
    if own:
        from paper_2606_18954_amd import graphattn as ga
        if op in ("slots", "logits"):
            st["graph"] = _device_graph(st)
        elif op == "qkv":
            st["params"] = ga.make_params(case["hq"], case["hkv"], case["dim"], st["total"], case["dtype"])
            st["rope"] = ga.QKTransform(case["dim"], st["freq"], st["interleaved"], q_norm=st["q_norm"],
                                        k_norm=st["k_norm"], eps=EPS)
        if op == "logits":
            st["rules"] = ga.LogitRules(repetition=st["rep"], frequency=st["freq"], presence=st["pres"],
                                        temperature=st["temp"], prompt_segments=1, bias_offsets=st.get("bias_off"),
                                        bias_tokens=st.get("bias_tokens"), bias_values=st.get("bias_values"),
                                        masks=st.get("masks"), row_mask=st.get("mask_of"))
    return st


# ----------------------------------------------------------------------------------------------
# One pass, in elementary operations
# ----------------------------------------------------------------------------------------------

def _run_pages(st):
    lens, old_off = st["lens"].long(), st["old_off"]
    S, known = lens.numel(), old_off.numel() - 1
    start = torch.cat([old_off, old_off[-1:].expand(S - known)])
    had = start[1:] - start[:-1]
    need = torch.maximum(had, (lens + st["spare"] + 15) // 16)
    st["new_off"][1:] = need.cumsum(0)
    off = st["new_off"]
    j = torch.arange(st["new_pages"].numel(), device=DEV)
    s = torch.searchsorted(off[1:], j, right=True).clamp(max=S - 1)
    k = j - off[s]
    free = (off[s] - start[s] + k - had[s]).clamp(0, st["free"].numel() - 1)
    old = (start[s] + k).clamp(max=max(st["old_pages"].numel() - 1, 0))
    page = torch.where(k < had[s], st["old_pages"][old] if st["old_pages"].numel() else -1, st["free"][free])
    st["new_pages"].copy_(torch.where(j < off[-1], page, -1))
    return {"offsets": off, "pages": st["new_pages"]}


def _run_slots(st):
    counts, paths, lens = st["counts"].long(), st["paths"].long(), st["lens"].long()
    B = counts.numel()
    st["token_off"][1:] = counts.cumsum(0)
    off = st["token_off"].long()
    j = torch.arange(st["capacity"], device=DEV)
    b = torch.searchsorted(off[1:], j, right=True).clamp(max=B - 1)
    last = paths[b, -1]
    t = lens[last] - counts[b] + j - off[b]
    page = st["pages"][(st["off"][last] + t // 16).clamp(0, st["pages"].numel() - 1)].long()
    before = lens[paths].sum(1) - lens[paths[:, -1]]
    there = j < off[-1]
    words, pos, branch = st["out"]
    words.copy_(torch.where(there, page * 16 + t % 16, -1))
    pos.copy_(torch.where(there, before[b] + t, -1))
    branch.copy_(torch.where(there, b, -1))
    return {"offsets": st["token_off"], "words": words, "positions": pos, "branches": branch}


def _normed(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w


def _rotated(x, cos, sin, interleaved):
    r = 2 * cos.shape[-1]
    rot, rest = x[..., :r], x[..., r:]
    a, b = (rot[..., 0::2], rot[..., 1::2]) if interleaved else (rot[..., :r // 2], rot[..., r // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    out = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([out, rest], -1)


def _run_qkv(st):
    hq, hkv, rows = st["hq"], st["hkv"], st["rows"]
    x = rows.float()
    angle = (st["pos"].double()[:, None] * st["freq"])[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q = _rotated(_normed(x[:, :hq], st["q_norm"]), cos, sin, st["interleaved"])
    k = _rotated(_normed(x[:, hq:hq + hkv], st["k_norm"]), cos, sin, st["interleaved"])
    real = st["pos"] >= 0
    st["q_out"].copy_(torch.where(real[:, None, None], q.to(rows.dtype), st["q_out"]))
    w = torch.where(real & (st["words"] >= 0), st["words"], st["total"] * 16).long()
    kv = torch.stack([k.to(rows.dtype), rows[:, hq + hkv:]], 2)
    st["pool"][w // 16, :, :, w % 16] = kv
    return {"q": st["q_out"], "pool": st["pool"][:st["total"]]}


def _slots_of_paths(st):
    """[B, longest] slot words of every branch's tokens (0 behind them) and, beside them, whether they are and
    whether they are the prompt's."""
    paths, lens = st["paths"].long(), st["lens"].long()
    n = lens[paths]
    end = n.cumsum(1)
    longest = st["longest"]
    t = torch.arange(longest, device=DEV).expand(len(paths), -1).contiguous()
    level = torch.searchsorted(end, t, right=True).clamp(max=paths.shape[1] - 1)
    s = paths.gather(1, level)
    i = t - (end - n).gather(1, level)
    page = st["pages"][(st["off"][s] + i // 16).clamp(max=st["pages"].numel() - 1)].long()
    return page * 16 + i % 16, t < end[:, -1:], t < end[:, st["prompt_segments"] - 1:st["prompt_segments"]]


def _run_logits(st):
    z = st["logits"].float()
    R, vocab = z.shape
    slot, there, prompt = _slots_of_paths(st)
    b = st["branch"].long()
    token = st["ids"].long()[slot][b]
    t = torch.arange(slot.shape[1], device=DEV)
    seen = there[b] & (t <= st["pos"][:, None]) & (token >= 0)
    said = torch.where(seen & ~prompt[b], token, vocab)
    read = torch.where(seen & prompt[b], token, vocab)
    count = torch.zeros(R, vocab + 1, device=DEV).scatter_add_(1, said, torch.ones_like(said, dtype=torch.float32))[:, :-1]
    was = torch.zeros(R, vocab + 1, dtype=torch.bool, device=DEV).scatter_(1, read, True)[:, :-1] | (count > 0)
    if "bias_off" in st:
        n = st["bias_tokens"].numel() // R
        z = z.scatter_add(1, st["bias_tokens"].long().view(R, n), st["bias_values"].view(R, n))
    rep = st["rep"][:, None]
    z = torch.where(was, torch.where(z > 0, z / rep, z * rep), z)
    z = z - st["freq"][:, None] * count - st["pres"][:, None] * (count > 0)
    z = z / st["temp"][:, None]
    if "masks" in st:
        v = torch.arange(vocab, device=DEV)
        m = st["mask_of"].long()
        allowed = (st["masks"][m.clamp(min=0)][:, v // 32] >> (v % 32)) & 1
        z = z.masked_fill((allowed == 0) & (m >= 0)[:, None], -math.inf)
    st["out"].copy_(z)
    return {"out": st["out"]}


def run(st):
    op = st["op"]
    if own:
        from paper_2606_18954_amd import graphattn as ga
        if op == "pages":
            ga.page_table(st["lens"], st["free"], st["spare"], st["old_off"], st["old_pages"], st["new_off"],
                          st["new_pages"])
            return {"offsets": st["new_off"], "pages": st["new_pages"]}
        if op == "slots":
            words, pos, branch = st["out"]
            ga.slot_map(st["graph"], st["counts"], st["token_off"], words, pos, branch)
            return {"offsets": st["token_off"], "words": words, "positions": pos, "branches": branch}
        if op == "qkv":
            q, k, v = st["rows"].split([st["hq"], st["hkv"], st["hkv"]], 1)
            ga.qkv_append(st["pool"], q, k, v, st["pos"], st["words"], st["rope"], st["params"], st["q_out"])
            return {"q": st["q_out"], "pool": st["pool"][:st["total"]]}
        ga.process_logits(st["logits"], st["rules"], st["graph"], st["ids"], st["branch"], st["pos"], st["out"])
        return {"out": st["out"]}
    return {"pages": _run_pages, "slots": _run_slots, "qkv": _run_qkv, "logits": _run_logits}[op](st)


# ----------------------------------------------------------------------------------------------
# What a pass cannot do without
# ----------------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "qkv":
        elt = 4 if case["dtype"] == "f32" else 2
        values = case["tokens"] * (case["hq"] + 2 * case["hkv"]) * case["dim"]
        return {"bytes": 2 * values * elt + 8 * case["tokens"], "flops": 9 * values}
    lens, paths = _structure(case)
    if case["op"] == "pages":
        known = int(round(case["known"] * len(lens)))
        pages = int(((lens.astype(np.int64) + case["spare"] + 15) // 16).sum())
        return {"bytes": 12 * len(lens) + 8 * known + 8 * pages, "flops": 0}
    graph = 12 * len(lens) + 4 * paths.size + 8 * len(paths)
    if case["op"] == "slots":
        last = lens[paths[:, -1]].astype(np.int64)
        new = last if case["new"] == 0 else np.minimum(last, (1 + case["new"]) / 2)
        return {"bytes": int(graph + 8 * len(paths) + 12 * new.sum() + 4 * (new / 16 + 1).sum()), "flops": 0}
    rows, vocab = len(paths) * case["drafts"], case["vocab"]
    wide = 4 if case["wide"] or case["dtype"] == "f32" else 2
    per = vocab * ((4 if case["dtype"] == "f32" else 2) + wide) + 8 * case["bias"] + 24
    return {"bytes": int(rows * per + graph + 4 * lens.astype(np.int64).sum() + case["masks"] * ((vocab + 31) // 32) * 4),
            "flops": 4 * rows * vocab}


# ----------------------------------------------------------------------------------------------
# The definition, in 64 bits
# ----------------------------------------------------------------------------------------------

def exact(case, seed):
    op = case["op"]
    if op in ("pages", "slots"):
        return None                                      # whole numbers only
    if op == "qkv":
        st = _qkv_inputs(case, seed)
        x = st["rows"].double()
        hq, hkv, half, dim = case["hq"], case["hkv"], case["rotary"] // 2, case["dim"]
        qk = x[:, :hq + hkv]
        if case["norm"]:
            w = torch.cat([st["q_norm"].expand(hq, dim), st["k_norm"].expand(hkv, dim)]).double()
            qk = qk / torch.sqrt((qk ** 2).sum(-1, keepdim=True) / dim + EPS) * w
        # A pair of channels as a complex number, turned by its angle.
        ch = torch.arange(2 * half, device=DEV)
        a, b = (ch[0::2], ch[1::2]) if case["interleaved"] else (ch[:half], ch[half:])
        turn = torch.polar(torch.ones(1, dtype=torch.float64, device=DEV), st["pos"].double()[:, None] * st["freq"])
        z = torch.complex(qk[..., a], qk[..., b]) * turn[:, None]
        qk = qk.clone()
        qk[..., a], qk[..., b] = z.real, z.imag
        real = st["pos"] >= 0
        pool = torch.zeros(st["total"], hkv, 2, 16, dim, dtype=torch.float64, device=DEV)
        j = torch.nonzero(real & (st["words"] >= 0)).flatten()
        w = st["words"][j].long()
        pool[w // 16, :, 0, w % 16] = qk[j, hq:]
        pool[w // 16, :, 1, w % 16] = x[j, hq + hkv:]
        return {"q": qk[:, :hq] * real[:, None, None], "pool": pool}
    st = _logits_inputs(case, seed)
    lens, paths = _structure(case)
    off, pages, _ = _pages(lens, seed)
    vocab, ids = case["vocab"], st["ids"].cpu().numpy()
    out = torch.empty(st["logits"].shape, dtype=torch.float64, device=DEV)
    rep, freq, pres, temp = (st[k].double().tolist() for k in ("rep", "freq", "pres", "temp"))
    mask_of = st["mask_of"].tolist() if case["masks"] else None
    for r in range(len(out)):
        if r % case["drafts"] == 0:
            parts = [ids[(pages[off[s]:off[s + 1], None].astype(np.int64) * 16 + np.arange(16)).reshape(-1)[:lens[s]]]
                     for s in paths[r // case["drafts"]]]
            context = _dev(np.concatenate(parts).astype(np.int64))
            root = len(parts[0])
        n = len(context) - case["drafts"] + r % case["drafts"] + 1
        a, b = context[:min(root, n)], context[root:n]
        count = torch.bincount(b[b >= 0], minlength=vocab)
        old = (torch.bincount(a[a >= 0], minlength=vocab) + count) > 0
        z = st["logits"][r].double()
        if case["bias"]:
            at = slice(*st["bias_off"][r:r + 2].tolist())
            z[st["bias_tokens"][at].long()] += st["bias_values"][at].double()
        z[old] = torch.where(z[old] > 0, z[old] / rep[r], z[old] * rep[r])
        z -= freq[r] * count + pres[r] * (count > 0)
        z /= temp[r]
        if case["masks"] and mask_of[r] >= 0:
            word = st["masks"][mask_of[r]].long() & 0xffffffff
            bits = (word[:, None] >> torch.arange(32, device=DEV)) & 1
            z[bits.flatten()[:vocab] == 0] = -math.inf
        out[r] = z
    return {"out": out}
