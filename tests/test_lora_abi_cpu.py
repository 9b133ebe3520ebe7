"""CPU-only checks of the adapters' calls: refusals before any GPU work, and sizes."""
import ctypes as C
import os

import pytest
import torch

FAKE = C.c_void_p(256)
ODD = C.c_void_p(264)


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2602_10431_amd import build
        build.build(verbose=False)
    pkg.load_library()
    return pkg


def _lora(qt, **how):
    a = dict(down=256, up=256, rank=None, scale=None, n_adapters=4, max_rank=16, N=256, K=512)
    a.update(how)
    return C.byref(qt.qtale_lora(**a))


BAD = [(dict(n_adapters=0), -1), (dict(n_adapters=-1), -1), (dict(max_rank=0), -1), (dict(max_rank=12), -2), (dict(max_rank=136), -3),
       (dict(n_adapters=(1 << 20) + 1), -3), (dict(N=264), -2), (dict(K=520), -2)]
NO_BUFFER = [(dict(down=None), -1), (dict(up=None), -1), (dict(down=264), -1), (dict(up=258), -1)]


@pytest.mark.parametrize("how,code", BAD + NO_BUFFER)
def test_a_bad_adapter_is_refused(qt, how, code):
    lib = qt.load_library()
    w = C.byref(qt.qtale_qlinear(None, None, None, 256, 256, 512))
    bad, good = _lora(qt, **how), _lora(qt)
    size = 1 << 30
    assert lib.qtale_linear_lora_w4a16(w, 4, 128, bad, FAKE, FAKE, 3, FAKE, FAKE, size, None) == code
    assert lib.qtale_swiglu_lora_w4a16(w, w, 4, 128, bad, good, FAKE, FAKE, 3, FAKE, FAKE, size, None) == code
    assert lib.qtale_swiglu_lora_w4a16(w, w, 4, 128, good, bad, FAKE, FAKE, 3, FAKE, FAKE, size, None) == code
    assert lib.qtale_swiglu_lora_w4a16(w, w, 4, 128, None, bad, FAKE, FAKE, 3, FAKE, FAKE, size, None) == code
    if (how, code) in NO_BUFFER:                                  # sizes do not look at the buffers
        assert lib.qtale_lora_workspace_bytes(bad, None, 3) > 0
    elif "N" not in how and "K" not in how:
        assert lib.qtale_lora_workspace_bytes(bad, None, 3) == 0 and lib.qtale_lora_workspace_bytes(good, bad, 3) == 0


def test_calls_refuse(qt):
    lib = qt.load_library()
    lora = _lora(qt)
    linear = lambda N=256, K=512, pre=256: C.byref(qt.qtale_qlinear(None, None, None, pre, N, K))
    size = lib.qtale_lora_workspace_bytes(lora, None, 3)
    pair = lib.qtale_lora_workspace_bytes(lora, lora, 3)
    assert size >= 3 * 16 * 4 and pair >= 2 * (3 * 16 * 4 + 3 * 256 * 2)

    def one(w=linear(), bits=4, group=128, l=lora, ids=FAKE, A=FAKE, M=3, out=FAKE, ws=FAKE, n=size):
        return lib.qtale_linear_lora_w4a16(w, bits, group, l, ids, A, M, out, ws, n, None)

    def two(g=linear(), u=linear(), bits=4, group=128, lg=lora, lu=lora, ids=FAKE, A=FAKE, M=3, out=FAKE, ws=FAKE, n=pair):
        return lib.qtale_swiglu_lora_w4a16(g, u, bits, group, lg, lu, ids, A, M, out, ws, n, None)

    for call in (one, two):
        assert call(bits=5) == -3 and call(group=48) == -3 and call(M=-1) == -1
        for missing in ("ids", "A", "out", "ws"):
            assert call(**{missing: None}) == -1
        assert call(ws=ODD) == -1 and call(A=ODD) == -1 and call(out=ODD) == -1
        assert call(n=100) == -4
        assert call(M=0) == 0
    assert one(w=None) == -1 and one(l=None) == -1 and one(w=linear(pre=None)) == -1 and one(w=linear(K=516)) == -2 and one(w=linear(N=260)) == -2
    assert two(g=None) == -1 and two(u=None) == -1 and two(u=linear(N=264)) == -2 and two(u=linear(pre=None)) == -1 and two(lg=None, lu=None) == -1
    assert lib.qtale_lora_workspace_bytes(None, None, 3) == 0 and lib.qtale_lora_workspace_bytes(lora, None, -1) == 0
    assert lib.qtale_lora_workspace_bytes(lora, _lora(qt, N=264), 3) == 0


def test_python_pads_ranks(qt):
    l = qt.Lora(torch.ones(3, 5, 64, dtype=torch.float16), torch.ones(3, 32, 5, dtype=torch.float16))
    assert (l.max_rank, l.N, l.K, l.n) == (8, 32, 64, 3) and l.rank.tolist() == [5, 5, 5]
    assert l.down.shape == (3, 8, 64) and float(l.down.sum()) == 3 * 5 * 64 and float(l.up.sum()) == 3 * 32 * 5
    with pytest.raises(AssertionError):
        qt.Lora(torch.ones(3, 8, 64, dtype=torch.float16), torch.ones(3, 32, 16, dtype=torch.float16))
    with pytest.raises(AssertionError):
        qt.Lora(torch.ones(3, 8, 64, dtype=torch.float16), torch.ones(3, 32, 8, dtype=torch.float16), rank=torch.ones(3))
