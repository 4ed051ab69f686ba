"""The step that README.md shows between two attention calls, run as it is written there: its page table and slots by the
oracle's definitions, everything else as a stand-in that does nothing (CPU)."""
import os
import textwrap
import types

import numpy as np
import pytest

from oracle import step_oracle as S

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def blocks(title):
    """The indented blocks of a section of README.md, in order."""
    with open(os.path.join(ROOT, "README.md"), encoding="utf-8") as f:
        section = f.read().split(f"## {title}\n")[1].split("\n## ")[0]
    out, lines = [], []
    for line in section.splitlines() + ["end"]:
        if line.startswith("    ") or (lines and not line.strip()):
            lines.append(line)
        elif lines:
            out.append(textwrap.dedent("\n".join(lines)))
            lines = []
    return out


class Library:
    """The calls of the step on tensors of the host."""

    DeviceGraph = staticmethod(lambda lens, off, pages, po, ps, n: S.Graph(*(t.numpy() for t in (lens, off, pages, po, ps)), n))

    @staticmethod
    def page_table(seg_len, free_pages, spare=0, old_offsets=None, old_pages=None):
        none = torch.zeros(0, dtype=torch.int32)
        old = none if old_pages is None else old_pages
        off, pages = S.page_table(seg_len.numpy(), spare, (none if old_offsets is None else old_offsets).numpy(), old.numpy(),
                                  free_pages.numpy())
        out = torch.full((old.numel() + free_pages.numel(),), -1, dtype=torch.int32)
        out[:len(pages)] = torch.from_numpy(pages[:len(out)].astype(np.int32))
        return torch.from_numpy(off), out

    @staticmethod
    def slot_map(graph):
        B = len(graph.path_offsets) - 1
        return tuple(torch.from_numpy(x.astype(np.int32)) for x in S.slot_map(graph, None, B))

    QKTransform = LogitRules = staticmethod(lambda *a, **k: None)
    qkv_append = staticmethod(lambda pool, q, *a: q)
    process_logits = staticmethod(lambda logits, *a: logits)


def test_the_step_of_the_readme_gives_every_page_once():
    """Two hundred steps, tables that grow on the way: no page comes twice or is lost, every token has its slot until the
    pool is full, and a branch without a slot stores no token."""
    *once, step = blocks("A step between two attention calls")
    num_pages, lens = 80, np.array([40, 1, 7, 1], np.int32)
    rng = np.random.default_rng(3)
    free = torch.from_numpy(rng.permutation(num_pages).astype(np.int32))
    seg_len = torch.from_numpy(lens)
    offsets, pages = Library.page_table(seg_len, free, 64)
    had = int(offsets[-1])
    space = {
        "ga": Library, "torch": torch, "seg_len": seg_len, "newest": torch.tensor([1, 2, 3]), "num_pages": num_pages,
        "offsets": offsets, "pages": pages[:had], "free": free[had:].clone(),
        # (the last branch has no path: its row is padding)
        "path_offsets": torch.tensor([0, 2, 4, 6, 6]), "path_segs": torch.tensor([0, 1, 0, 2, 0, 3], dtype=torch.int32),
        "x": torch.zeros(4, 8), "w_qkv": torch.zeros(8, 36 * 128), "plan": types.SimpleNamespace(run=lambda *a: None),
        "token_ids": torch.full((16 * num_pages,), -1, dtype=torch.int32),
        **{k: None for k in ("inv_freq", "wq", "wk", "pool", "p", "out", "lse", "r", "f", "t", "grammar", "state", "logits")},
    }
    for block in once:
        exec(block, space)                                   # (what is made once)
    written = {}
    for i in range(200):
        space["tokens"] = torch.arange(4, dtype=torch.int32) + 10 * i
        space["step"] = i
        exec(step, space)
        total = int(space["offsets"][-1])
        given = space["pages"][:total].tolist()
        assert len(set(given)) == total and min(given) >= 0, f"step {i}: a page of two segments"
        assert space["pages"].numel() == total, f"step {i}: the table has entries behind its total"
        assert sorted(given + space["free"].tolist()) == list(range(num_pages)), f"step {i}: pages were lost"
        words = space["words"].tolist()
        assert words[3] == -1 and min(words[:3]) >= 0 and not written.keys() & set(words[:3]), f"step {i}"
        written.update(zip(words[:3], space["tokens"].tolist()))
        assert {w: int(v) for w, v in enumerate(space["token_ids"][:16 * num_pages]) if v >= 0} == written, f"step {i}"
