"""The serving loop with weights of 4 bits, norms and positions of heads, and tokens drawn by chance: each step checked against plain products, and the
definition of judging."""
import pytest
import torch

pytestmark = pytest.mark.gpu

CASES = {
    "bfloat16": dict(requests=5, layers=2, hidden=256, heads=8, kv_heads=2, dim=64, vocab=97, page=16, prompt=70, answer=9, depth=3),
    "float16, odd widths": dict(requests=7, layers=1, hidden=136, heads=3, kv_heads=3, dim=128, vocab=31, page=7, prompt=33, answer=5, depth=4, ranks=(1, 5, 40),
                                dtype=torch.float16),
    "a larger vocabulary": dict(requests=3, layers=2, hidden=512, heads=4, kv_heads=1, dim=128, vocab=40000, page=32, prompt=300, answer=12, depth=6),
    "deep trees": dict(requests=3, layers=1, hidden=128, heads=4, kv_heads=4, dim=64, vocab=5, page=8, prompt=20, answer=64, depth=31),
}


@pytest.mark.parametrize("name", list(CASES))
def test_steps_of_a_server_that_draws_tokens(name):
    from paper_2411_01830_amd.serve import Server
    server = Server(check=True, seed=len(name), rotate=True, four_bit=True, sample=True, **CASES[name])
    tokens = [server.step() for _ in range(8)]
    assert all((got >= 1).all() for got in tokens)
    assert all((got <= 1 + max(server.levels)).all() for got in tokens)
    server.close()


@pytest.mark.parametrize("one", ["rotate", "four_bit", "sample"])
def test_steps_of_a_server_with_one_of_these(one):
    from paper_2411_01830_amd.serve import Server
    server = Server(check=True, seed=3, **CASES["bfloat16"], **{one: True})
    for _ in range(4):
        assert (server.step() >= 1).all()
    server.close()
