"""The example's decoding loop (marked gpu): drafted trees give the tokens that
decoding one by one gives."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_drafts_change_no_token(lib):
    spec = importlib.util.spec_from_file_location("decode_with_drafts", os.path.join(ROOT, "examples", "decode_with_drafts.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, ex.VOCAB, k).tolist() for k in (9, 140)]
    seqs, gained = ex.decode(prompts, 6)
    model = ex.Model("cuda")
    for p, s in zip(prompts, seqs):
        # all at once, in fp32, from the model's weights
        x = model.embed[torch.tensor(s[:-1], device="cuda")]
        n = len(x)
        for w in model.layers:
            q, k, v = ((x @ w["qkv"]).float().split([ex.HEADS * ex.DIM, ex.KV_HEADS * ex.DIM, ex.KV_HEADS * ex.DIM], dim=1))
            q, k, v = (t.view(n, -1, ex.DIM) for t in (q, k, v))
            turned = []
            for t, g in ((q, w["norms"][0]), (k, w["norms"][1])):
                t = torch.nn.functional.rms_norm(t, (ex.DIM,), g, 1e-6)
                a, b = t.chunk(2, -1)
                c, d = model.cos[:n, None], model.sin[:n, None]
                turned.append(torch.cat([a * c - b * d, b * c + a * d], -1).bfloat16().float())
            q, k = turned
            k, v = (t.repeat_interleave(ex.HEADS // ex.KV_HEADS, 1) for t in (k, v))
            sc = torch.einsum("ihd,jhd->hij", q, k) * ex.DIM ** -0.5
            sc = sc.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -torch.inf)
            y = torch.einsum("hij,jhd->ihd", sc.softmax(-1), v).bfloat16()
            x = torch.nn.functional.rms_norm(x + y.reshape(n, -1) @ w["out"], (ex.WIDTH,))
        logits = x.float() @ model.head.float().T
        got = torch.tensor(s[len(p):], device="cuda")
        rows = logits[len(p) - 1:]
        # each token is the best one, or within bf16's rounding of it (a unit of 2^-8 in each of the final state's
        # WIDTH elements, in random directions: 2^-8 of the logits' own spread)
        lag = rows.amax(-1) - rows.gather(1, got[:, None])[:, 0]
        assert (lag <= 2.0 ** -5 * rows.std(-1)).all(), lag
    assert all(k >= 1 for g in gained for k in g) and max(k for g in gained for k in g) > 1
