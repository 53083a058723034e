"""The readme's lines on rotated positions, parts of prompts, windows and drafted tokens, run as they stand there."""
import os
import re

import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2601_16986_amd import ckv
from tests.paged import DEV, bf16, device, pools
from tests.rows import random_tree

pytestmark = pytest.mark.gpu


def lines():
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        text = f.read()
    block = re.search(r"For models that rotate positions.*?:\n\n((?:    .*\n)+)", text).group(1)
    return "".join(line[4:] + "\n" for line in block.splitlines())


def test_a_part_of_a_prompt_and_drafted_tokens():
    """Keys lie turned by where each row stands in the text: parts of prompts by their place in the sequence, drafts by the tokens that they descend from."""
    rng = np.random.default_rng(0)
    batch, rows, T, hq, hkv, ps = 3, 20, 9, 4, 2, 16
    c = pools(batch * 8, hkv, ps, False)
    lengths = torch.tensor([60, 20, 41], dtype=torch.int32, device=DEV)
    before = lengths.tolist()
    trees = np.stack([random_tree(rng, T) for _ in range(batch)])
    parts = {n: bf16(rng.standard_normal((batch, r, h, 128))) for n, r, h in (("q_part", rows, hq), ("k_part", rows, hkv), ("v_part", rows, hkv), ("q_draft", T, hq), ("k_draft", T, hkv), ("v_draft", T, hkv))}
    f = 10000.0 ** (-np.arange(64) / 64)
    s = c.sequences(torch.arange(batch * 8, dtype=torch.int32, device=DEV).view(batch, 8), lengths)
    c.append(s, *(device(rng.standard_normal((batch, 60, hkv, 128))) for _ in range(2)))
    env = dict(torch=torch, ckv=ckv, c=c, s=s, lengths=lengths, T=T, tree=torch.from_numpy(trees).to(DEV), frequencies=torch.from_numpy(f).to(DEV),
               depths=torch.from_numpy(trees.sum(2).astype(np.int32) - 1).to(DEV), **{n: device(x) for n, x in parts.items()})
    exec(compile(lines(), "README.md", "exec"), env)
    assert c.status() == 0 and lengths.tolist() == [n + T for n in before] and torch.isfinite(env["out"]).all()
    k, v = (x.double().cpu().numpy() for x in c.read(s, rows + T))

    def close(got, x, at):
        y = ref.rotate(x, at, f)
        slack = ref.pair_size(x, 64) * (3 * 2.0 ** -24 + 2.0 ** -40)
        assert (np.abs(got - y) <= slack + 2.0 ** -8 * (np.abs(y) + slack)).all()

    first, depth = np.array(before)[:, None], trees.sum(2)
    close(k[:, :rows], parts["k_part"], first - rows + np.arange(rows))
    close(k[:, rows:], parts["k_draft"], first + depth - 1)
    close(env["q"].double().cpu().numpy(), parts["q_draft"], first + depth - 1)
    assert np.array_equal(v[:, rows:], parts["v_draft"])
