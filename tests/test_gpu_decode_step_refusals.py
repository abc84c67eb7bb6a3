"""A decoding layer refuses tables and pools that its steps could not use, and a step that fails leaves it as it was."""
import numpy as np
import pytest
import torch

from test_gpu_around_step_together import BLOCK, DIM, HEADS, HIDDEN, Q_HEADS, ROT, b, make  # noqa: F401 (b: the fixture)

pytestmark = pytest.mark.gpu


def test_tables_and_pools_that_no_step_could_use(b):  # noqa: F811
    from paper_2103_00130_amd import decode_step
    layer, _, _, _ = make(b, np.random.default_rng(31), 2, 20, 30)
    sizes = (layer.wqkv, layer.wo, Q_HEADS, HEADS, DIM, 2, 20, 30, BLOCK, torch.float32)
    table = b.rotary_table(20, ROT)
    wide = torch.zeros((20, DIM + 2), device="cuda")
    for bad in (table[:, :ROT - 1].contiguous(), wide, wide[:, :ROT], table[:, :0], table[0], table[:19]):
        with pytest.raises(ValueError):
            decode_step.DecodeLayer(*sizes, rotary=bad)
    for bad in (table.double(), table.cpu(), table.half()):
        with pytest.raises(TypeError):
            decode_step.DecodeLayer(*sizes, rotary=bad)
    for bad in ((), layer.adapters[:1], layer.adapters + layer.adapters[:1]):
        with pytest.raises(ValueError):
            decode_step.DecodeLayer(*sizes, adapters=bad)


@pytest.mark.parametrize("stage", ["abft_w4_gemv", "abft_lora_gemv", "abft_kv_append_rotary", "abft_kv_attention"])
def test_a_step_that_fails_is_taken_again(b, monkeypatch, stage):  # noqa: F811
    """Whatever call of a step raises: the step called again gives what it gives to a layer of which none failed, and so do the steps behind it."""
    rng = np.random.default_rng(32)
    steps = [[5, 0, 20], [1, 14, 1], [1, 1, 1]]
    layers = [make(b, np.random.default_rng(33), 3, 40, 30)[0] for _ in range(2)]
    for layer in layers:
        layer.use(2, 1)
    for new in steps:
        x = torch.from_numpy(rng.standard_normal((sum(new), HIDDEN)).astype(np.float32)).cuda()
        before = (list(layers[1].lengths), layers[1].used)

        def fails(*a, **kw):
            raise RuntimeError("refused")
        with monkeypatch.context() as m:
            m.setattr(b, stage, fails)
            with pytest.raises(RuntimeError):
                layers[1].step(x, new)
        assert (layers[1].lengths, layers[1].used) == before
        want, got = (layer.step(x, new) for layer in layers)
        assert torch.equal(want, got) and layers[0].lengths == layers[1].lengths and layers[0].used == layers[1].used
