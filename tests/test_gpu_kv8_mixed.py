"""Attention over the 8-bit cache in batches that a server has under load: a long piece of a prompt beside decodes over
long contexts, whole prompts beside requests that bring nothing.  Bounds as in test_gpu_kv8."""
import pytest

from test_gpu_kv8 import Case, check, serve  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,dt", [(64, "f16"), (128, "bf16"), (256, "bf16")])
@pytest.mark.parametrize("window", [0, 700])
def test_a_chunk_beside_long_decodes(serve, D, dt, window):
    c = Case(serve, [2600, 5000, 37, 0, 3001], [260, 1, 1, 0, 1], heads=2, D=D, page=32, dt=dt, seed=80)
    c.fill(2)
    check(c, 4, window=window)


@pytest.mark.parametrize("first", [True, False])
def test_whole_prompts_beside_decodes(serve, first):
    kv, new = [300, 4000, 0, 129, 1], [300, 1, 0, 129, 1]
    order = range(5) if first else range(4, -1, -1)
    c = Case(serve, [kv[i] for i in order], [new[i] for i in order], heads=1, D=128, page=16, dt="bf16", seed=81)
    c.fill(1)
    check(c, 8)
