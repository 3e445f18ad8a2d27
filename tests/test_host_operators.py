"""CPU-only checks of the layer operators' and the log probabilities' entry points: bad arguments are refused before any GPU
call, sizes are host formulas."""
import ctypes

import pytest

from paper_2505_06653_amd import binding

F32, BF16 = 0, 1


def at(address):
    return ctypes.c_void_p(address)


P = at(0x10000)


def logprobs(logits=P, kind=F32, n=4, vocab=100, ld=100, target=P, top=0, lp=P, ent=P, ids=None, top_lp=None, stats=P, ws=P,
             size=1 << 30):
    return binding.lib().bof4_token_logprobs(logits, kind, n, vocab, ld, target, top, lp, ent, ids, top_lp, stats, ws, size,
                                             None)


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(ws=None), dict(kind=2), dict(n=0), dict(vocab=0), dict(n=(1 << 23) + 1), dict(vocab=(1 << 30) + 1, ld=1 << 31),
    dict(ld=99), dict(target=None), dict(lp=None), dict(top=65, ids=P, top_lp=P), dict(top=1), dict(top=1, ids=P),
    dict(top=1, top_lp=P), dict(logits=at(0x10002)), dict(logits=at(0x10001), kind=BF16), dict(target=at(0x10004)),
    dict(ws=at(0x10010)), dict(ent=at(0x10002)), dict(stats=at(0x10002)), dict(top=1, ids=at(0x10004), top_lp=P)])
def test_token_logprobs_refuses(bad):
    assert logprobs(**bad) == binding.BOF4_ERR_ARG
    assert b"bof4_token_logprobs" in binding.lib().bof4_last_error()


def test_token_logprobs_workspace():
    L = binding.lib()
    assert logprobs(size=0) == binding.BOF4_ERR_WORKSPACE
    assert L.bof4_token_logprobs_workspace_bytes(0, 10, 0) == 0 and L.bof4_token_logprobs_workspace_bytes(1, 0, 0) == 0
    assert L.bof4_token_logprobs_workspace_bytes(1, 10, 65) == 0
    for n, vocab in ((1, 1), (1, 128000), (3, 1 << 30), (1000, 50257), (1 << 23, 7)):
        sizes = [L.bof4_token_logprobs_workspace_bytes(n, vocab, top) for top in (0, 1, 20, 64)]
        assert sizes == sorted(sizes) and 0 < sizes[0] and sizes[-1] < 1 << 24


def backward(logits=P, kind=F32, n=4, vocab=100, ld=100, stats=P, target=P, d_lp=P, ent=P, d_ent=P, out=at(0x20000), out_kind=F32,
             ld_out=100):
    return binding.lib().bof4_token_logprobs_backward(logits, kind, n, vocab, ld, stats, target, d_lp, ent, d_ent, out, out_kind,
                                                      ld_out, None)


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(stats=None), dict(out=None), dict(kind=7), dict(out_kind=2), dict(n=0), dict(vocab=0),
    dict(n=(1 << 23) + 1), dict(vocab=(1 << 30) + 1, ld=1 << 31, ld_out=1 << 31), dict(ld=99), dict(ld_out=99), dict(target=None),
    dict(d_lp=None), dict(ent=None), dict(d_ent=None), dict(out=P, out_kind=BF16), dict(out=P, ld_out=101),
    dict(out=at(0x20002)), dict(stats=at(0x10002)), dict(target=at(0x10004)),
    dict(n=1 << 20, vocab=1 << 20, ld=1 << 20, ld_out=1 << 20)])
def test_token_logprobs_backward_refuses(bad):
    assert backward(**bad) == binding.BOF4_ERR_ARG
    assert b"bof4_token_logprobs_backward" in binding.lib().bof4_last_error()
