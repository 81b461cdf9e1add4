"""Workspaces of choosing tokens: what is asked for (host arithmetic), and that a call keeps to it (GPU)."""
import ctypes as C

import pytest
import torch

import paper_2312_04916_amd as ee

GOOD, ARG, CONFIG, NOMEM = 0, -7, -1, -2


def sizes(rows, vocab):
    b, u = C.c_size_t(), C.c_size_t()
    assert ee.lib().ee_sample_bytes(rows, vocab, C.byref(b)) == GOOD and ee.lib().ee_sample_uncut_bytes(rows, vocab, C.byref(u)) == GOOD
    return b.value, u.value


def test_sizes():
    for rows, vocab in ((1, 1), (3, 1024), (64, 50304), (512, 50304), (1024, 262144), (1 << 20, 5), (2000, 100000)):
        cut, uncut = sizes(rows, vocab)
        assert uncut <= 256 + rows * 128 * -(-vocab // 1024)
        # bins and lists are for the rows that several workgroups share
        shared = vocab > 4096 and rows <= 1024
        assert cut == uncut if not shared else rows * (2 * vocab + (36 << 10)) <= cut - uncut <= rows * (2 * vocab + (240 << 10)), (rows, vocab)
    L, b = ee.lib(), C.c_size_t()
    assert L.ee_sample_uncut_bytes(0, 5, C.byref(b)) == GOOD and b.value == 0
    for rows, vocab, p, code in ((-1, 5, C.byref(b), ARG), ((1 << 20) + 1, 5, C.byref(b), ARG), (1, 5, None, ARG), (1, 0, C.byref(b), CONFIG), (1, (1 << 18) + 1, C.byref(b), CONFIG)):
        assert L.ee_sample_uncut_bytes(rows, vocab, p) == code


def test_settings_that_may_cut_need_the_larger_one():
    """Refused for the size of the workspace, or behind that for where it lies: nothing runs."""
    M, rows, vocab = 1 << 24, 4, 50304
    cut, uncut = sizes(rows, vocab)

    def sample(size, kp=None, pp=None, mp=None, k=0, p=1.0, m=0.0):
        return ee.lib().ee_sample(rows, vocab, ee.EE_F32, M, vocab, 4 * M, None, kp, pp, mp, 1.0, k, p, m, 5 * M, None, None, M, size, None)

    assert sample(uncut - 1) == NOMEM and sample(uncut) == ARG
    assert sample(uncut, k=vocab) == ARG
    for one in (dict(k=vocab - 1), dict(p=0.999), dict(m=1e-30), dict(kp=6 * M), dict(pp=6 * M), dict(mp=6 * M)):
        assert sample(uncut, **one) == NOMEM and sample(cut - 1, **one) == NOMEM and sample(cut, **one) == ARG, one


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 1000), (7, 3000), (5, 4097), (2, 50304), (130, 9000), (1100, 5000), (2000, 300)])
@pytest.mark.parametrize("k,p", [(0, 1.0), (0, 0.9), (2500, 0.97)])
def test_a_call_keeps_to_its_workspace(rows, vocab, k, p):
    g = torch.Generator(device="cuda:0").manual_seed(rows + vocab)
    z, u = torch.randn(rows, vocab, device="cuda:0", generator=g), torch.rand(rows, device="cuda:0", generator=g)
    cuts = 0 < k < vocab or p < 1
    need, guard = sizes(rows, vocab)[0 if cuts else 1], 1 << 20
    memory = torch.full((need + 2 * guard,), 0xA5, dtype=torch.uint8, device="cuda:0")
    token, logprob, conf = torch.empty(rows, dtype=torch.int32, device="cuda:0"), torch.empty(rows, device="cuda:0"), torch.empty(rows, device="cuda:0")
    stream = torch.cuda.current_stream().cuda_stream
    assert ee.lib().ee_sample(rows, vocab, ee.EE_F32, z.data_ptr(), vocab, u.data_ptr(), None, None, None, None, 1.0, k, p, 0.0, token.data_ptr(), logprob.data_ptr(),
                              conf.data_ptr(), memory.data_ptr() + guard, need, stream) == GOOD
    torch.cuda.synchronize()
    assert (memory[:guard] == 0xA5).all() and (memory[guard + need:] == 0xA5).all()
    want = ee.sample(z, u, top_k=k, top_p=p, scores=True)
    assert torch.equal(token, want[0]) and torch.equal(logprob, want[1]) and torch.equal(conf, want[2])
    # the settings per row, with which the host does not know that nothing is cut: the same tokens
    per_row = ee.sample(z, u, top_k=torch.full((rows,), k, dtype=torch.int32, device="cuda:0"), top_p=torch.full((rows,), p, device="cuda:0"))
    assert torch.equal(per_row, token)
