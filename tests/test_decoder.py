"""The decoder stack: attention over the 4-bit cache in front of the MoE layer (paper_2509_02753_b200/decoder.py)."""
import pytest
import torch

from paper_2509_02753_b200 import decoder as D
from paper_2509_02753_b200 import synth

pytestmark = pytest.mark.gpu
ATTN = D.Attention(n_heads=4, n_kv_heads=2, head_dim=64, rope_dim=32, k_scale=0.01, v_scale=0.01)


def make(requests=2, max_tokens=64, max_context=64, attn=ATTN, dtype=torch.float32, page_size=16):
    return D.build("tiny", attn, layers=2, dtype=dtype, requests=requests, max_tokens=max_tokens, max_context=max_context, page_size=page_size)


def tokens(n):
    return synth.make_tokens(synth.WORKLOADS["tiny"], n, torch.float32, "cuda")


@pytest.mark.parametrize("attn", [ATTN, D.Attention(4, 2, 64, 32, layout="pairs", window=9, sinks=2, k_scale=0.01, v_scale=0.01)])
def test_prompts_at_once_and_token_by_token_agree(attn):
    """The same tokens in one step, in uneven chunks and one by one: sums of other orders in fp32, so the outputs are near.
    Two layers of a few thousand fp32 additions each: 2^-24 * 4096 * 2 relative at worst, below 1e-3; what is stored in 4
    bits could differ by a code only where a number lies that near to a boundary, and an expert only where two logits do."""
    x = tokens(40)
    n = [23, 17]
    outs = []
    for cuts in ([n], [[5, 0], [1, 16], [17, 1]], [[1, 1]] * 17 + [[1, 0]] * 6):
        dec, at, got = make(attn=attn), [0, 0], [[], []]
        for new in cuts:
            part = torch.cat([x[:23][at[0]: at[0] + new[0]], x[23:][at[1]: at[1] + new[1]]])
            y = dec.step(part, new)
            got[0].append(y[: new[0]])
            got[1].append(y[new[0]:])
            at = [a + b for a, b in zip(at, new)]
        dec.check()
        assert [r.length for r in dec.requests] == n and at == n
        outs.append(torch.cat(got[0] + got[1]))
        dec.close()
    for other in outs[1:]:
        assert (outs[0] - other).abs().max() <= 1e-3 * outs[0].abs().max()


@pytest.mark.parametrize("attn", [ATTN, D.Attention(4, 2, 64, 64, layout="pairs", window=9, sinks=2, k_scale=0.01, v_scale=0.01)])
def test_a_step_against_the_formula(attn):
    """Prompts, then a token each: the turns, the masks and the sums in 64 bits on the numbers that the cache holds (read back), the
    MoE layer as it is.  Tolerance as above: fp32 sums of a few thousand terms."""
    dec, seen = make(attn=attn), [0, 0]
    layer_forward = dec.moe.layer_forward
    for new in ([23, 17], [1, 1], [0, 3]):
        x = tokens(40)[: sum(new)]
        got = dec.step(x, new)
        dec.check()
        positions = torch.cat([torch.arange(s, s + n) for s, n in zip(seen, new)]).cuda()
        seen = [s + n for s, n in zip(seen, new)]
        held = [(dec.table[i, torch.arange(s, device="cuda") // dec.page].long() * dec.page + torch.arange(s, device="cuda") % dec.page) for i, s in enumerate(seen)]
        half = attn.rope_dim // 2
        angle = positions.double().view(-1, 1, 1) * 10000.0 ** (-torch.arange(half, device="cuda").double() / half)
        want = x
        for layer, weights, cache, k_l in zip(dec.layers, dec.weights, dec.caches, dec.k_vec):
            q = (D.rms_norm(want).double() @ layer["qkv"].double().t()).view(len(x), -1, attn.head_dim)[:, : attn.n_heads]
            at = slice(0, half), slice(half, 2 * half)
            if attn.layout == "pairs":
                at = slice(0, 2 * half, 2), slice(1, 2 * half, 2)
            turned = q.clone()
            turned[..., at[0]] = q[..., at[0]] * angle.cos() - q[..., at[1]] * angle.sin()
            turned[..., at[1]] = q[..., at[1]] * angle.cos() + q[..., at[0]] * angle.sin()
            out = []
            for i, s in enumerate(seen):
                keys, values = (t.double().repeat_interleave(attn.n_heads // attn.n_kv_heads, 1)
                                for t in dec.kv.read(cache, held[i], k_scale=attn.k_scale, v_scale=attn.v_scale))
                first = sum(new[:i])
                back = positions[first: first + new[i]].view(-1, 1) - torch.arange(s, device="cuda")
                see = back >= 0
                if attn.window:
                    see &= (back < attn.window) | (torch.arange(s, device="cuda") < attn.sinks)
                w = torch.einsum("thd,khd->htk", turned[first: first + new[i]], keys) / attn.head_dim ** 0.5
                out.append(torch.einsum("htk,khd->thd", torch.softmax(w.masked_fill(~see, float("-inf")), -1), values))
            want = want + (torch.cat(out).flatten(1) @ layer["o"].double().t()).float()
            want = want + layer_forward(D.rms_norm(want), weights, k_l, dec.renorm)
        assert (got - want).abs().max() <= 1e-3 * want.abs().max()
    dec.close()


def test_a_row_serves_another_request_after_finish():
    dec = make()
    x = tokens(40)
    first = dec.step(x, [23, 17])
    free = len(dec.free)
    dec.finish(0)
    assert len(dec.free) == free + 2
    again = dec.step(x[:23], [23, 0])
    dec.check()
    assert (again - first[:23]).abs().max() <= 1e-3 * first.abs().max()
    dec.close()


def test_refusals():
    dec = make()
    with pytest.raises(ValueError):
        dec.step(tokens(65), [65, 0])
    dec.free = dec.free[:1]
    with pytest.raises(MemoryError):
        dec.step(tokens(20), [17, 3])
    assert [r.length for r in dec.requests] == [0, 0]
    dec.close()


def test_a_step_in_which_every_request_pauses():
    dec = make()
    first = dec.step(tokens(20), [17, 3])
    none = dec.step(tokens(1)[:0], [0, 0])
    assert none.shape == (0, first.shape[1]) and [r.length for r in dec.requests] == [17, 3]
    dec.check()
    assert dec.step(tokens(2), [1, 1]).shape == (2, first.shape[1]) and dec.lengths.tolist() == [18, 4]
    dec.check()
    dec.close()


def test_negative_numbers_of_tokens_are_refused():
    dec = make()
    dec.step(tokens(20), [17, 3])
    with pytest.raises(ValueError):
        dec.step(tokens(2), [-1, 3])
    assert [r.length for r in dec.requests] == [17, 3] and dec.lengths.tolist() == [17, 3]
    dec.check()
    dec.close()


def test_bf16_step_runs_and_stays_finite():
    dec = make(dtype=torch.bfloat16, requests=3, max_tokens=200, max_context=100, page_size=32)
    x = synth.make_tokens(synth.WORKLOADS["tiny"], 130, torch.bfloat16, "cuda")
    y = dec.step(x, [90, 0, 40])
    y = torch.cat([y, dec.step(x[:3], [1, 1, 1])])
    dec.check()
    assert bool(torch.isfinite(y.float()).all())
    dec.close()
