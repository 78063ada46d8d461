"""The decoding loop of examples/tree_decode.py: what the operators compute together, against a plain forward pass.

The logits that the loop gets for a path's nodes through tree attention, the paged cache and its commits are compared with
those of the whole text run through the model at once with plain attention.  Tolerances: single precision, two layers
of a few hundred fp32 roundings: 2e-4 of the largest logit; bfloat16, about a dozen roundings of 2^-8 to each of the two
layers' contributions: 0.1 of the largest logit.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _plain_logits(model, tokens):
    import torch

    def attend(layer, q, k, v):
        g = model.hq // model.hkv
        q, k, v = (t.float().transpose(1, 2) for t in (q, k.repeat_interleave(g, 2), v.repeat_interleave(g, 2)))
        s = q @ k.transpose(2, 3) / model.dim ** 0.5
        n = s.shape[-1]
        s = s.masked_fill(~torch.ones((n, n), dtype=torch.bool, device=s.device).tril(), float("-inf"))
        return (torch.softmax(s, -1) @ v).transpose(1, 2).to(model.dtype)

    n = tokens.shape[0]
    return model.forward(tokens[None], torch.arange(n, device=tokens.device)[None], attend)[0][0]


@pytest.mark.parametrize("dtype,tol", [("f32", 2e-4), ("bf16", 0.1)])
@pytest.mark.parametrize("batch", [1, 5])
def test_the_loop_computes_what_a_plain_pass_does(dtype, tol, batch):
    import torch
    from examples import tree_decode as td
    model = td.Model(dtype=torch.float32 if dtype == "f32" else torch.bfloat16, V=300)
    dec = td.Decoder(model, td.prompts_for(batch, model.V, seed=batch), most=256)
    seen = []
    deepest = 0
    for _ in range(24):
        before = dec.n_text.clone()
        raw, emitted, n = dec.step()
        seen.append((before.cpu().numpy(), raw.clone(), dec.path.cpu().numpy().copy(), n.cpu().numpy().copy()))
        deepest = max(deepest, int(n.max()))
    assert deepest >= 2 or batch == 1  # some draft was accepted: paths of more than the root (24 steps of one sequence may have none)
    st = dec.stand.stats()
    assert st["bad_tokens"] == 0 and st["wait_timeouts"] == 0
    assert torch.equal(dec.len + 1, dec.n_text)
    lens = torch.zeros(batch, dtype=torch.int64, device="cuda:0")
    assert torch.equal(dec.stand.lens_device(lens), dec.n_text)
    for b in range(batch):
        want = _plain_logits(model, dec.text[b, : int(dec.n_text[b])]).float()
        top = float(want.abs().max())
        for before, raw, path, n in seen:
            for j in range(n[b]):  # the j-th node of the path predicts the text's token before + j
                got = raw[b, path[b, j]].float()
                assert float((got - want[before[b] - 1 + j]).abs().max()) <= tol * top


def test_masked_tokens_are_never_emitted_and_pages_hold():
    import torch
    from examples import tree_decode as td
    model = td.Model(V=1000)
    allowed = np.zeros((1, 1024), np.uint8)
    allowed[0, 100:400] = 1
    mask = torch.from_numpy(np.packbits(allowed, axis=1, bitorder="little").view(np.int32)).to("cuda:0")
    dec = td.Decoder(model, td.prompts_for(3, model.V), most=320, mask=mask)
    for _ in range(40):
        dec.step()
    for b in range(3):
        made = dec.text[b, int(dec.n_prompt[b]): int(dec.n_text[b])].cpu().numpy()
        assert len(made) >= 40 and made.min() >= 100 and made.max() < 400
    used = [int(p) for b in range(3) for p in dec.table[b, : -(-int(dec.len[b]) // dec.page)]]
    rest = [int(p) for p in dec.free[: int(dec.n_free)]]
    assert sorted(used + rest) == list(range(dec.free.numel()))
