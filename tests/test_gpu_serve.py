"""The serving loop: transfers into the pool and the operators on it, each step checked against plain products over a history of its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu

CASES = {
    "bfloat16": dict(requests=5, layers=2, hidden=256, heads=8, kv_heads=2, dim=64, vocab=97, page=16, prompt=70, answer=9, depth=3),
    "float16, odd pages, a head each": dict(requests=7, layers=1, hidden=136, heads=3, kv_heads=3, dim=128, vocab=31, page=7, prompt=33, answer=5, depth=4,
                                            ranks=(1, 5, 40), dtype=torch.float16),
    "one request, long prompt": dict(requests=1, layers=2, hidden=192, heads=4, kv_heads=1, dim=128, vocab=11, page=32, prompt=3001, answer=20, depth=6),
    "deep trees": dict(requests=3, layers=1, hidden=128, heads=4, kv_heads=4, dim=64, vocab=5, page=8, prompt=20, answer=64, depth=31),
}


@pytest.mark.parametrize("name", list(CASES))
def test_steps_of_a_server(name):
    from paper_2411_01830_amd.serve import Server
    case = CASES[name]
    server = Server(check=True, seed=len(name), **case)
    brought = server.bytes_moved
    tokens = [server.step() for _ in range(8)]
    assert all((got >= 1).all() for got in tokens)                                     # each step answers with a token at least
    assert all((got <= 1 + max(server.levels)).all() for got in tokens)
    assert server.bytes_moved > brought or sum(tokens).max() < case["answer"]          # who has their tokens makes room
    server.close()


def test_trees_deeper_than_a_word_are_refused():
    from paper_2411_01830_amd.serve import Server
    with pytest.raises(ValueError):
        Server(depth=32)
