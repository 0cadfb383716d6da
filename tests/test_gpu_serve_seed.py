"""A serving loop's run is its seed's, whatever else has drawn random numbers on the GPU."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", [{}, dict(four_bit=True), dict(sample=True), dict(rotate=True, four_bit=True, sample=True)], ids=lambda h: "-".join(h) or "plain")
def test_two_runs_of_one_seed_are_one(how):
    from paper_2411_01830_amd.serve import Server

    def run(seed, other):
        torch.cuda.manual_seed(other)
        server = Server(seed=seed, requests=8, layers=2, hidden=128, heads=4, kv_heads=2, dim=64, vocab=5, page=16, prompt=40, answer=9, depth=3, **how)
        seen = []
        for _ in range(12):
            seen.append(server.step().tolist())
            seen.append(server.last.tolist())
        weights = [t for w in server.w_qkv + server.w_out for t in server._weights(w)] if how.get("four_bit") else []    # (other memory of the pool holds anything)
        server.close()
        return seen, weights

    (a, wa), (b, wb), (c, _) = run(5, 1), run(5, 2), run(6, 1)
    assert a == b and a != c
    assert len(wa) == len(wb) and all(torch.equal(x, y) for x, y in zip(wa, wb))
