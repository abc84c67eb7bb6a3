"""Rotation, adapters and scores as `decode_step` runs them with the plan, the products, the cache and the attention: every stage against its
definition applied to what the stage before it gave, and replayed from a graph."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle, step_oracle as o

pytestmark = pytest.mark.gpu

HIDDEN, Q_HEADS, HEADS, DIM, BLOCK, ROT, VOCAB = 96, 6, 2, 40, 16, 32, 500


@pytest.fixture(scope="module")
def b():
    from paper_2103_00130_amd import binding
    assert torch.cuda.is_available()
    return binding


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def within(got, want, tol, what):
    off = ~(np.abs(got - want) <= tol)
    assert not off.any(), f"{what}: {off.sum()} of {got.size} beyond the bound"


def make(b, rng, requests, longest, most_rows, dtype=torch.float32):
    """(layer, scores, plain weights, plain adapters)"""
    from paper_2103_00130_amd import decode_step
    handles, plain, pools, adapters = [], [], [], []
    for n, k in (((Q_HEADS + 2 * HEADS) * DIM, HIDDEN), (HIDDEN, Q_HEADS * DIM), (VOCAB, HIDDEN)):
        W = rng.integers(0, 256, (n, k // 2), dtype=np.uint8)
        scale = torch.full((n, -(-k // 32)), (21.25 * k) ** -0.5)
        bias = scale * -7.5
        handles.append(b.abft_w4_pack(torch.from_numpy(W).cuda(), scale.cuda(), bias.cuda(), K=k, group=32))
        plain.append((W, f64(scale), f64(bias)))
    for w in handles[:2]:
        pools.append(b.LoraPool(3, w.K, w.N, 20, dtype))
        adapters.append([])
        for slot, rank in enumerate((20, 7, 1)):
            A, B = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(dtype).cuda() for s in ((rank, w.K), (w.N, rank)))
            pools[-1].load(slot, A, B, 0.1)
            adapters[-1].append((f64(A), f64(B), 0.1))
    layer = decode_step.DecodeLayer(*handles[:2], Q_HEADS, HEADS, DIM, requests, longest, most_rows, BLOCK, dtype, rotary=b.rotary_table(longest, ROT), adapters=tuple(pools))
    return layer, decode_step.TokenScores(handles[2], most_rows, 4, dtype), plain, adapters


def test_prompts_then_single_tokens(b):
    rng = np.random.default_rng(21)
    steps = [[5, 0, 33, 16], [1, 1, 1, 1], [1, 1, 1, 1], [0, 40, 1, 0], [11, 1, 0, 1]]
    longest = int(np.sum(steps, axis=0).max())
    layer, scores, plain, adapters = make(b, rng, 4, longest, 64)
    table, split = layer.rotary.cpu().numpy(), Q_HEADS * DIM
    parts = [np.zeros((layer.cache.n_blocks, HEADS, BLOCK, DIM), np.int8) for _ in range(2)]
    scales = [np.zeros((layer.cache.n_blocks, HEADS), np.float32) for _ in range(2)]
    held, using = np.zeros(4, np.int64), np.array([2, -1, 0, 1])
    for r, slot in enumerate(using):
        layer.use(r, int(slot))
    for i, new in enumerate(steps):
        if i == 3:
            using[0] = -1
            layer.use(0, -1)
        n = sum(new)
        x = torch.from_numpy(rng.standard_normal((n, HIDDEN)).astype(np.float32)).cuda()
        y = layer.step(x, new)
        held += new
        who = np.repeat(np.arange(4), new)
        where = np.concatenate([np.arange(m - c, m) for m, c in zip(held, new)])
        qkv, slots, blocks = f64(layer.qkv[:n]), layer.slots[:n].cpu().numpy(), layer.table.cpu().numpy()
        assert np.array_equal(slots, blocks[who, where // BLOCK] * BLOCK + where % BLOCK)
        # the projection and the adapters: keys and values as they are in the buffer, queries as they were before they were turned there
        first, first_tol = decode_oracle.w4_product(f64(x), *plain[0], 32, "f32")
        want, tol = o.lora(f64(x), adapters[0], using[who], first, "f32")
        tol = tol + first_tol
        within(qkv[:, split:], want[:, split:], tol[:, split:], "keys and values")
        q, q_tol = (a[:, :split].reshape(n, Q_HEADS, DIM) for a in (want, tol))
        turned = o.rotate(q.astype(np.float32), table, where, False)
        within(qkv[:, :split].reshape(n, Q_HEADS, DIM), turned, 2 * (q_tol + np.roll(q_tol, ROT // 2, 2)) + q_tol.max() + 2.0 ** -22 * np.abs(q).max(), "queries")
        for j in range(2):
            rows = qkv[:, split + j * HEADS * DIM:split + (j + 1) * HEADS * DIM].reshape(n, HEADS, DIM).astype(np.float32)
            decode_oracle.append(parts[j], scales[j], o.rotate(rows, table, where, False) if j == 0 else rows, slots)
        for got, code, gs, ws in zip(layer.cache.codes(), parts, (layer.cache.k_scale, layer.cache.v_scale), scales):
            got = got.cpu().numpy()
            for r in range(4):
                for t in range(int(held[r])):
                    assert np.array_equal(got[blocks[r, t // BLOCK], :, t % BLOCK], code[blocks[r, t // BLOCK], :, t % BLOCK])
            taken = np.concatenate([row[:-(-int(m) // BLOCK)] for row, m in zip(blocks, held)])
            assert np.array_equal(gs.cpu().numpy()[taken], ws[taken])
        mid = f64(layer.mid[:n])
        want, tol, _, _ = decode_oracle.attention(qkv[:, :split].reshape(n, Q_HEADS, DIM), *parts, *scales, blocks, held, np.concatenate([[0], np.cumsum(new)]), DIM ** -0.5, "f32")
        within(mid, want, tol, "attention")
        second, second_tol = decode_oracle.w4_product(mid.reshape(n, -1), *plain[1], 32, "f32")
        want, tol = o.lora(mid.reshape(n, -1), adapters[1], using[who], second, "f32")
        within(f64(y), want, tol + second_tol, "output")
        # scores of what came out
        tokens = rng.integers(0, VOCAB, n).astype(np.int64)
        got = {k: v.cpu().numpy() for k, v in scores(y, torch.from_numpy(tokens).cuda(), temperature=0.8).items()}
        logits = f64(scores.logits[:n])
        within(logits, *decode_oracle.w4_product(f64(y), *plain[2], 32, "f32"), "logits")
        want = o.logprobs(logits, tokens, np.float32(1 / 0.8), 4)
        assert np.array_equal(got["rank"], want["rank"]) and np.array_equal(got["top_index"], want["top_index"])
        for name, tol in (("logprob", "logprob_tol"), ("entropy", "entropy_tol"), ("top_logprob", "top_tol")):
            within(got[name].astype(np.float64), want[name], want[tol], name)


def test_steps_replayed_from_a_graph_are_the_steps_run(b):
    """Replays with other adapters and with work and synchronization of the program's own between them, against the same steps run: the same bits."""
    ran, replayed = (make(b, np.random.default_rng(22), 3, 60, 64, torch.bfloat16)[:2] for _ in range(2))
    rng = np.random.default_rng(23)
    draw = lambda n: torch.from_numpy(rng.standard_normal((n, HIDDEN)).astype(np.float32)).to(torch.bfloat16).cuda()
    prompt = [14, 31, 1]
    x = draw(sum(prompt))
    for layer, _ in (ran, replayed):
        layer.use(1, 2)
    assert torch.equal(ran[0].step(x, prompt), replayed[0].step(x, prompt))
    replayed[0].record()
    tokens = torch.randint(0, VOCAB, (3,), device="cuda")
    hidden = torch.zeros((3, HIDDEN), dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    replayed[1](hidden, tokens)
    with torch.cuda.graph(graph):
        captured = replayed[1](hidden, tokens)
    for i in range(20):
        if i % 4 == 1:
            for layer, _ in (ran, replayed):
                layer.use(i % 3, i % 4 - 1)
        x = draw(3)
        y = torch.empty((3, HIDDEN), dtype=torch.bfloat16, device="cuda")
        layer = ran[0]
        first = layer._take([1, 1, 1])
        # (both with the same estimate of the longest request, so that they are cut alike)
        layer._launch(x, torch.ones(3, dtype=torch.int32, device="cuda"), layer.pool[first:layer.used], y, 1, 60, *layer._positions([1, 1, 1]))
        got = replayed[0].replay(x)
        assert torch.equal(got, y), f"replay {i}"
        hidden.copy_(got)
        graph.replay()
        want = ran[1](y, tokens)
        assert all(torch.equal(captured[k], want[k]) for k in want), f"scores {i}"
        torch.ones(1000, device="cuda").sum().item()
        torch.cuda.synchronize()


def test_calls_agree_with_and_without_their_native_marshalling(b, monkeypatch):
    layers = [make(b, np.random.default_rng(24), 2, 40, 20)[:2] for _ in range(2)]
    x = torch.from_numpy(np.random.default_rng(25).standard_normal((20, HIDDEN)).astype(np.float32)).cuda()
    tokens = torch.arange(20, device="cuda")
    outs = []
    for i, (layer, scores) in enumerate(layers):
        layer.use(0, 1)
        if i:
            for name in ("w4", "plan", "append", "append_rotary", "read", "attention", "lora", "logprobs"):
                monkeypatch.setattr(b._fastcall, name, lambda *a: None)
        y = layer.step(x, [3, 17])
        outs.append((y, {k: v.clone() for k, v in scores(y, tokens).items()}))
    assert torch.equal(outs[0][0], outs[1][0]) and all(torch.equal(outs[0][1][k], outs[1][1][k]) for k in outs[0][1])


def test_layer_refuses_what_does_not_fit(b):
    from paper_2103_00130_amd import decode_step
    layer, scores, _, _ = make(b, np.random.default_rng(26), 2, 20, 30)
    for slot in (-2, 3):
        with pytest.raises(ValueError):
            layer.use(0, slot)
    sizes = (layer.wqkv, layer.wo, Q_HEADS, HEADS, DIM, 2, 20, 30, BLOCK, torch.float32)
    with pytest.raises(ValueError):
        decode_step.DecodeLayer(*sizes, rotary=b.rotary_table(19, ROT))
    with pytest.raises(ValueError):
        decode_step.DecodeLayer(*sizes, adapters=layer.adapters[::-1])
    with pytest.raises(ValueError):
        decode_step.DecodeLayer(*sizes).use(0, 0)
    assert layer.step(torch.zeros((0, HIDDEN), device="cuda"), [0, 0]).shape == (0, HIDDEN)


def test_example_runs(b, capsys):
    from paper_2103_00130_amd import decode_step
    decode_step.main(["--hidden", "256", "--q-heads", "4", "--heads", "2", "--head-dim", "64", "--requests", "3", "--prompt", "20", "--steps", "3", "--vocab", "1000", "--rank", "8"])
    assert "replayed" in capsys.readouterr().out
