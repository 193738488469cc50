"""Language models of several tenants, as paper_1901_10008_amd.decode runs them (norms, products, append, attention, experts, verification, pages), against a
plain decoder in 64 bits."""
import pytest
import torch

import paper_1901_10008_amd as sk
from paper_1901_10008_amd import decode

pytestmark = pytest.mark.gpu

# hidden, heads, window, sinks, vocabulary, experts, chosen, width of an expert and of the shared one
KINDS = [(96, (4, 4, 24), 0, 0, 50, 8, 2, 200, 0), (128, (4, 2, 64), 40, 3, 301, 5, 3, 64, 136), (64, (6, 1, 80), 0, 0, 17, 16, 1, 96, 64)]


def models(children, most):
    return [decode.LanguageModel(h, heads, 2, children + 1, most, vocab, experts, top_k, ffn, shared, window=w, sinks=s, seed=i)
            for i, (h, heads, w, s, vocab, experts, top_k, ffn, shared) in enumerate(KINDS)]


def rms(x, weight):
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.double().cpu()


def attention(t, layer, x, keys, values):
    """x on the keys and values of the tokens before, which it takes up."""
    qkv = (x @ t.w_qkv[layer].double().cpu().T).view(x.shape[0], -1, t.d)
    old, n = keys[layer].shape[0], x.shape[0]
    turned = []
    for part, weight in ((qkv[:, :t.hq], t.q_norm[layer]), (qkv[:, t.hq:t.hq + t.hkv], t.k_norm[layer])):
        y = rms(part, weight)
        co, si = t.cos[old:old + n].double().cpu()[:, None], t.sin[old:old + n].double().cpu()[:, None]
        a, b = y[..., :t.d // 2], y[..., t.d // 2:]
        turned.append(torch.cat([a * co - b * si, b * co + a * si], -1))
    keys[layer] = torch.cat([keys[layer], turned[1]])
    values[layer] = torch.cat([values[layer], qkv[:, t.hq + t.hkv:]])
    pos, j = torch.arange(old, old + n)[:, None], torch.arange(old + n)[None]
    see = j <= pos
    if t.window:
        see &= (pos - j < t.window) | (j < t.sinks)
    out = torch.zeros((n, t.hq, t.d), dtype=torch.float64)
    for h in range(t.hq):
        kv = h // (t.hq // t.hkv)
        score = turned[0][:, h] @ keys[layer][:, kv].T * t.d ** -0.5
        out[:, h] = torch.softmax(score.masked_fill(~see, -float("inf")), -1) @ values[layer][:, kv]
    return out.flatten(1) @ t.w_out[layer].double().cpu().T


def through(x, gate, up, down):
    z = x @ gate.double().cpu().T
    return (z * torch.sigmoid(z) * (x @ up.double().cpu().T)) @ down.double().cpu().T


def experts(t, layer, x, ids):
    """With the choice that the kernels made (which of two experts with scores next to each other it is, roundings before them decide)."""
    s = torch.softmax(x @ t.router[layer].double().cpu().T, -1)
    y = through(x, t.shared_gate[layer], t.shared_up[layer], t.shared_down[layer]) if t.shared else torch.zeros_like(x)
    for r in range(x.shape[0]):
        w = s[r, ids[r]] / s[r, ids[r]].sum()
        for e, we in zip(ids[r].tolist(), w):
            y[r] += we * through(x[r:r + 1], t.gate[layer][e], t.up[layer][e], t.down[layer][e])[0]
        # (and that choice is the best there is, up to those roundings: x is off by some 2 %, a score's logit by that much of its size)
        assert s[r, ids[r]].min() >= 0.8 * torch.topk(s[r], len(ids[r])).values[-1]
    return y


def logits_of(t, tokens, keys, values, chosen):
    x = t.embedding[torch.tensor(tokens)].double().cpu()
    for layer in range(t.layers):
        x = x + attention(t, layer, rms(x, t.norms[2 * layer]), keys, values)
        x = x + experts(t, layer, rms(x, t.norms[2 * layer + 1]), chosen[layer])
    return rms(x, t.norms[-1]) @ t.head.double().cpu().T


def answer(logits, drafted, accept, sample, temperature):
    """What verification makes of a sequence's rows: the tokens, by its definition."""
    tokens = []
    for row in range(len(logits)):
        x = logits[row].double()
        p = torch.softmax(x / temperature, -1) if temperature > 0 else torch.nn.functional.one_hot(x.argmax(), len(x)).double()
        d = int(drafted[row])
        last = row + 1 == len(logits)
        if not last and 0 <= d < len(x):
            if float(accept[row]) < float(p[d]):
                tokens.append(d)
                continue
            p = p.clone()
            p[d] = 0.0
        upto = p.cumsum(0)
        tokens.append(int(((upto > float(sample) * upto[-1]) & (p > 0)).nonzero()[0]))
        return tokens


@pytest.mark.parametrize("temperature", [0.0, 0.6])
def test_prompts_forks_and_drafts_against_a_plain_decoder(temperature):
    children, steps, drafts = 3, 5, 3
    ts = models(children, 150 + steps * (drafts + 1) + 8)
    g = torch.Generator().manual_seed(7)
    # prompts that repeat themselves, so that something is found in them
    prompts = [(torch.randint(0, t.vocab, (n // 4,), generator=g).tolist() * 5)[:n] for n, t in zip((133, 96, 50), ts)]
    held = {}  # (tenant, child): keys and values of the plain decoder
    accepted = [0]

    def seen(step, launches, histories):
        torch.cuda.synchronize()
        for i, t in enumerate(ts):
            chosen, tokens_in = [launches.chosen[layer][i].cpu().long() for layer in range(t.layers)], launches.tokens_in[i].tolist()
            got, made = launches.logits[i].double().cpu(), launches.tokens[i].tolist()
            assert torch.isfinite(got).all()
            sequences = 1 if step == 0 else children
            width, rows = len(tokens_in) // sequences, len(made) // sequences
            for c in range(sequences):
                if step == 0:
                    none = [torch.zeros((0, t.hkv, t.d), dtype=torch.float64) for _ in range(t.layers)]
                    keys, values = list(none), list(none)
                else:
                    keys, values = (list(x) for x in held[i, c if (i, c) in held else 0])
                    assert keys[0].shape[0] == len(histories[i][c]) - 1
                mine = slice(c * width, (c + 1) * width)
                want = logits_of(t, tokens_in[mine], keys, values, [ids[mine] for ids in chosen])[-rows:]
                # As with the decoder without a vocabulary: some dozen roundings to bf16 on the way; the framework's bound for it.
                off = (got[c * rows:(c + 1) * rows] - want).norm() / want.norm()
                assert off <= 2e-2, f"step {step} tenant {i} sequence {c}: {off:.3g}"
                new = answer(got[c * rows:(c + 1) * rows], launches.drafted[i][c * rows:(c + 1) * rows].tolist(), launches.accept[i][c * rows:(c + 1) * rows].tolist(),
                             launches.sample[i][c], temperature)
                assert made[c * rows:(c + 1) * rows] == new + [-1] * (rows - len(new)), f"step {step} tenant {i} sequence {c}"
                assert int(launches.accepted[i][c]) == len(new) - 1
                accepted[0] += len(new) - 1
                upto = len(prompts[i]) if step == 0 else len(histories[i][c]) - 1 + len(new)
                held[i, c] = [k[:upto] for k in keys], [v[:upto] for v in values]
            if step == 0:
                for c in range(1, children):
                    held[i, c] = held[i, 0]

    histories, _, _ = decode.generate(ts, prompts, children, steps, drafts, temperature, torch.cuda.current_stream().cuda_stream, seed=3, seen=seen)
    assert accepted[0] > 0  # drafts were looked up and taken
    for t, hs in zip(ts, histories):
        # no page is held for what was rejected
        assert [sk.sk_pages_state(t.account, c)[0] for c in range(children)] == [len(h) - 1 for h in hs]
        assert all(sum(p >= 0 for p in sk.sk_pages_state(t.account, c)[1]) == -(-(len(h) - 1) // t.page) for c, h in enumerate(hs))
    if temperature == 0.0:
        assert all(h == hs[0] for hs in histories for h in hs)


def test_lookup():
    assert decode.looked_up([1, 2, 3, 1], 2) == [2, 3]
    assert decode.looked_up([5, 5], 3) == [5, -1, -1]
    assert decode.looked_up([1, 2, 3], 2) == [-1, -1]


def test_command(capsys):
    decode.main(["--tenants", "2", "--layers", "1", "--prompt", "40", "--children", "2", "--steps", "2", "--vocab", "60"])
    assert "2 language models" in capsys.readouterr().out
