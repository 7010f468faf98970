"""Results that a call allocates for itself come from the pool of the stream that its kernels run on: memory of another stream's pool may
still be in use there."""
import pytest
import torch

import paper_2510_00236_amd as pex

pytestmark = pytest.mark.gpu


def stream_of(t):
    """The stream of the caching allocator's segment that holds a tensor"""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not in the caching allocator")


def tensors_of(x):
    if isinstance(x, torch.Tensor):
        return [x]
    if isinstance(x, dict):
        x = list(x.values())
    return [t for y in x for t in tensors_of(y)] if isinstance(x, (list, tuple)) else []


def calls():
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    X, G, gamma, M, ids = rnd(3, 40, 64), rnd(3, 40, 64), rnd(64), rnd(100, 300), torch.randint(0, 50, (3, 40), device="cuda", generator=g)
    mean, rstd = X.mean(2).contiguous(), torch.rsqrt(X.var(2, correction=0) + 1e-5).contiguous()
    N = rnd(2, 3).abs()
    return {
        "layer_norm": lambda s: pex.pex_layer_norm(X, gamma, stream=s),
        "layer_norm_grad": lambda s: pex.pex_layer_norm_grad(G, X, mean, rstd, gamma, stream=s),
        "orthogonalize": lambda s: pex.pex_orthogonalize(M, stream=s),
        "stat": lambda s: pex.pex_stat(X, G, "square", stream=s),
        "stat_multi": lambda s: pex.pex_stat_multi(X, G, ("identity", "square"), stream=s),
        "token_sq": lambda s: pex.pex_token_sq(X, G, stream=s),
        "vec_stat": lambda s: pex.pex_vec_stat(G, X, stream=s),
        "embed_stat": lambda s: pex.pex_embed_stat(ids, G, 50, ("identity",), stream=s),
        "example_norms": lambda s: pex.pex_example_norms(X, G, stream=s),
        "clip_weights": lambda s: pex.pex_clip_weights(N, 1.0, stream=s),
        "sum_squares": lambda s: pex.pex_sum_squares(M, accumulate=True, stream=s),
    }


@pytest.mark.parametrize("name", ["layer_norm", "layer_norm_grad", "orthogonalize", "stat", "stat_multi", "token_sq", "vec_stat", "embed_stat", "example_norms",
                                  "clip_weights", "sum_squares"])
def test_results_belong_to_the_stream_of_the_call(name):
    call = calls()[name]
    want = tensors_of(call(None))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = tensors_of(call(side))
    torch.cuda.current_stream().wait_stream(side)
    assert len(got) == len(want) > 0
    for a, b in zip(got, want):
        assert torch.equal(a, b) and stream_of(a) == side.cuda_stream != stream_of(b)
