"""GPU: what a call of the worker's operators does to the program around it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_an_earlier_error_of_the_caller_is_neither_this_calls_nor_lost():
    """The runtime keeps a thread's last error until it is asked for: a call that works says so beside one, and leaves it."""
    import paper_2605_01989_amd as dblp
    x, y, w, z = (torch.ones(4, 8, device="cuda") for _ in range(4))
    tok, v, stats, grad = torch.arange(4, device="cuda"), torch.ones(4, device="cuda"), torch.empty(5, device="cuda"), torch.zeros(8, 8, device="cuda")
    big = torch.zeros(600, dtype=torch.int64, device="cuda")
    dy, ws = torch.ones(600, 8, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    half = dblp.Drop(1, 1, 0.5)
    torch.cuda.synchronize()
    hip = dblp.lib()                             # (the runtime's own functions are found through the library that uses them)
    hip.hipGetLastError()
    for call in (lambda: dblp.dropout(x, y, half), lambda: dblp.embed(tok, x, z), lambda: dblp.embed_grad(tok, x, grad, ws), lambda: dblp.embed_grad(big, dy, grad, ws),
                 lambda: dblp.token_logprobs(x, tok, v, ws), lambda: dblp.policy_loss(x, tok, v, v, stats, ws, dlogits=w)):
        pending = hip.hipSetDevice(99)
        assert pending != 0
        try:
            call()
        finally:
            left = hip.hipGetLastError()
        assert left == pending and hip.hipGetLastError() == 0
    torch.cuda.synchronize()
    assert torch.equal(z, x) and float(grad[0, 0]) == 600.0 and float(stats[4]) == 4
