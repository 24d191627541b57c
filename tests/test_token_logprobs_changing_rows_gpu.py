"""Logits that another stream writes to while a call reads them: what the call returns for such rows is not specified, but it ends, its alternatives are tokens of the
vocabulary, and the next call is right."""
import pytest
import torch

from tests.test_token_logprobs_gpu import BF16, F32, check_forward, forward, given, lib  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,v,dtype,top", [(600, 30000, BF16, 128), (2400, 5003, BF16, 32), (1200, 14000, F32, 32), (12, 200001, F32, 64), (64, 1024, BF16, 8)])
def test_rows_that_change_under_the_call(lib, n, v, dtype, top):
    z = torch.ones(n, v, dtype=dtype, device="cuda")             # ties throughout, so that a place in the row has to decide
    tokens = given(n, v, 2, 1).cuda()
    writer, reader = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    results = []
    for i in range(60):
        with torch.cuda.stream(writer):
            z.fill_(float(i % 3))
            z[:, ::7] = 2.0
        with torch.cuda.stream(reader):
            results.append(forward(lib, z, tokens, 1.0, top, stream=reader))
    torch.cuda.synchronize()
    for o in results:
        assert bool(((o["top_ids"] >= -1) & (o["top_ids"] < v)).all())
    z.fill_(1.0)
    o = forward(lib, z, tokens, 1.0, top)
    torch.cuda.synchronize()
    some = slice(0, min(n, 6))
    check_forward({k: x[some] for k, x in o.items()}, z[some].cpu(), tokens[some].cpu(), 1.0, top)
