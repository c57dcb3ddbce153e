"""What the entry points of the verification step beside the tree refuse, without a GPU: every argument is
checked before the first HIP call."""
import os

import pytest
import torch

from paper_2606_03819_amd import binding

pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH), reason="libtreeflash.so not built")

P, P2 = 0x10000, 0x20000   # 16-byte aligned non-null dummy pointers: never dereferenced
BF16, F32 = binding.TF_BF16, binding.TF_F32
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
BIG = 1 << 40


def _call(name, defaults, over):
    assert not set(over) - set(defaults), over
    return getattr(binding.lib(), name)(*{**defaults, **over}.values())


SAMPLE = dict(logits=P, ld=1000, b=2, n=3, V=1000, dt=BF16, t=None, k=None, p=None, m=None, u=P, tok=P2, lp=None,
              ws=P, wsb=BIG, st=None)


@pytest.mark.parametrize("over,code", [
    (dict(logits=None), INVALID), (dict(u=None), INVALID), (dict(tok=None), INVALID), (dict(b=0), INVALID),
    (dict(n=0), INVALID), (dict(V=0), INVALID), (dict(V=(1 << 22) + 1, ld=1 << 23), INVALID), (dict(ld=999), INVALID),
    (dict(ld=(1 << 32) + 1), INVALID), (dict(dt=3), INVALID), (dict(logits=P + 1), INVALID),
    (dict(dt=F32, logits=P + 2), INVALID), (dict(t=P + 2), INVALID), (dict(k=P + 1), INVALID), (dict(p=P + 3), INVALID),
    (dict(m=P + 2), INVALID), (dict(u=P + 2), INVALID), (dict(tok=P + 1), INVALID), (dict(lp=P + 2), INVALID),
    (dict(b=1 << 11, n=1 << 10), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=P + 8), WORKSPACE), (dict(wsb=8), WORKSPACE),
])
def test_sample_rejects(over, code):
    assert _call("treeflash_sample", SAMPLE, over) == code


def test_sample_workspace():
    f = binding.treeflash_sample_workspace_bytes
    assert f(0, 1, 10) == f(1, 0, 10) == f(1, 1, 0) == f(1 << 11, 1 << 10, 10) == f(1, 1, (1 << 22) + 1) == 0
    for V in (1, 1000, 151936, 1 << 22):
        sizes = [f(1, n, V) for n in (1, 2, 31, 64, 65, 1000, 1001)]
        assert sizes == sorted(sizes) and sizes[0] > 0
        assert f(31, 1, V) == f(1, 31, V)


SLOTS = dict(ctx=P, add=P, acc=P, free=P, fc=P, b=2, gamma=16, n=33, page=64, cols=10, max_free=100, max_tokens=34,
             table=P, nl=P, nfc=P, start=P, ps=P, slot=P, pos=None, src=None, status=P, st=None)


@pytest.mark.parametrize("over,code", [(dict([(f, None)]), INVALID) for f in
                                       ("ctx", "add", "free", "fc", "table", "nl", "nfc", "start", "ps", "slot", "status")]
                         + [(dict([(f, P + 2)]), INVALID) for f in ("ctx", "acc", "table", "slot", "pos", "src", "status")]
                         + [(dict(b=0), INVALID), (dict(gamma=0), INVALID), (dict(gamma=256), INVALID), (dict(n=0), INVALID),
                            (dict(n=-1), INVALID), (dict(page=0), INVALID), (dict(page=48), UNSUPPORTED),
                            (dict(page=256), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(cols=0), INVALID),
                            (dict(cols=1 << 26), INVALID), (dict(max_free=0), INVALID), (dict(max_tokens=0), INVALID), (dict(max_tokens=(1 << 30) + 1), INVALID)])
def test_slots_rejects(over, code):
    assert _call("treeflash_cache_slots", SLOTS, over) == code


RELEASE = dict(done=P, ctx=P, table=P, fc=P, b=2, page=64, cols=10, max_free=100, free=P, nl=P, nfc=P, st=None)


@pytest.mark.parametrize("over,code", [(dict([(f, None)]), INVALID) for f in ("done", "ctx", "table", "fc", "free", "nl", "nfc")]
                         + [(dict(b=0), INVALID), (dict(page=24), UNSUPPORTED), (dict(cols=0), INVALID),
                            (dict(max_free=0), INVALID), (dict(nl=P + 2), INVALID)])
def test_release_rejects(over, code):
    assert _call("treeflash_cache_release", RELEASE, over) == code


APPEND = dict(k=P, v=P, ld=1024, rows=5, slot=P, src=None, N=5, H=8, D=128, page=64, pages=10, dt=BF16, kc=P, vc=P, ks=P,
              vs=P, st=None)


@pytest.mark.parametrize("over,code", [(dict([(f, None)]), INVALID) for f in ("k", "v", "slot", "kc", "vc", "ks", "vs")]
                         + [(dict(rows=0), INVALID), (dict(N=0), INVALID), (dict(H=0), INVALID), (dict(D=0), INVALID),
                            (dict(D=96), UNSUPPORTED), (dict(D=256, ld=4096), UNSUPPORTED), (dict(page=40), UNSUPPORTED),
                            (dict(pages=0), INVALID), (dict(pages=1 << 26), INVALID), (dict(ld=1023), INVALID),
                            (dict(ld=1028), UNSUPPORTED), (dict(dt=F32, ld=1026), UNSUPPORTED), (dict(dt=9), INVALID),
                            (dict(k=P + 8), UNSUPPORTED), (dict(v=P + 1), INVALID), (dict(kc=P + 4), UNSUPPORTED),
                            (dict(N=1 << 26), UNSUPPORTED), (dict(slot=P + 2), INVALID), (dict(src=P + 1), INVALID), (dict(ks=P + 2), INVALID)])
def test_append_rejects(over, code):
    assert _call("treeflash_cache_append", APPEND, over) == code


ATTEND = dict(q=P, ldq=4096, k=P, v=P, ld=1024, mask=None, nl=None, ctx=P, table=P, kc=P, vc=P, ks=P, vs=P, b=2, n=33,
              Hq=32, H=8, D=128, page=64, cols=100, pages=500, scale=0.1, dt=BF16, out=P2, lse=None, ws=P, wsb=BIG, st=None)


@pytest.mark.parametrize("over,code", [(dict([(f, None)]), INVALID) for f in
                                       ("q", "k", "v", "ctx", "table", "kc", "vc", "ks", "vs", "out")]
                         + [(dict(b=0), INVALID), (dict(n=0), INVALID), (dict(n=4097), INVALID), (dict(Hq=30), INVALID),
                            (dict(Hq=4), INVALID), (dict(H=0), INVALID), (dict(D=80, ldq=8192), UNSUPPORTED),
                            (dict(page=65), UNSUPPORTED), (dict(cols=0), INVALID), (dict(pages=0), INVALID),
                            (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(dt=2), INVALID),
                            (dict(ldq=4095), INVALID), (dict(ldq=4097), UNSUPPORTED), (dict(ld=1000), INVALID),
                            (dict(q=P + 8), UNSUPPORTED), (dict(out=P + 2), UNSUPPORTED), (dict(out=P + 1), INVALID),
                            (dict(vc=P + 8), UNSUPPORTED), (dict(lse=P + 2), INVALID), (dict(nl=P + 1), INVALID),
                            (dict(ctx=P + 2), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=P + 4), WORKSPACE),
                            (dict(wsb=64), WORKSPACE), (dict(b=1 << 10, n=2000), INVALID),
                            (dict(b=200, n=4096, Hq=16, H=8, ldq=2048), UNSUPPORTED)])
def test_attention_rejects(over, code):
    assert _call("treeflash_tree_attention", ATTEND, over) == code


def test_attention_workspace():
    f = binding.treeflash_tree_attention_workspace_bytes
    assert f(1, 1, 32, 8, 128, 64, 100, BF16) > 0 and f(1, 1, 8, 2, 64, 16, 100, F32) > 0
    assert f(1, 1, 30, 8, 128, 64, 100, BF16) == f(1, 1, 32, 8, 96, 64, 100, BF16) == f(1, 1, 32, 8, 128, 60, 100, BF16) == 0
    assert f(0, 1, 32, 8, 128, 64, 100, BF16) == f(1, 5000, 32, 8, 128, 64, 100, BF16) == f(1, 1, 32, 8, 128, 64, 0, BF16) == 0


def test_rows_at_one_distance():
    """Views that the library can read with one row distance, and those that it cannot."""
    class Fake:   # _rows_ptr looks at shape, strides and type; nothing is read
        is_cuda, device = True, "gpu"

        def __new__(cls, t):
            t = t.as_subclass(type("FakeTensor", (torch.Tensor,), {"is_cuda": True, "device": "gpu"}))
            return t

    rows = lambda t, inner=2: binding._rows_ptr(Fake(t), "t", inner, t.dtype, "gpu")[1]  # noqa: E731
    qkv = torch.zeros(2, 3, 10, 64)
    assert rows(qkv[:, :, :4]) == 640 and rows(qkv[:, :, 4:6]) == 640 and rows(qkv[:, 1:2, :4]) == 1920
    assert rows(torch.zeros(1, 1, 4, 64)) == 256 and rows(torch.zeros(5, 17)[:, :9], 1) == 17
    for bad in (qkv[:, :2, :4], qkv[:, :, ::2], qkv[..., ::2], qkv.transpose(0, 1)):
        with pytest.raises(ValueError):
            rows(bad)
