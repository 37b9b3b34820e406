"""What the entry points of the 4-bit cache, the key weights and the eviction refuse, without a GPU: nothing is enqueued, no
pointer is followed."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2410_17980_amd import binding
    return binding.load()


P, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4096 + 8)      # never dereferenced: validation fails first


def test_status_of_overlap():
    from paper_2410_17980_amd import binding
    assert "overlaps" in binding.sb_status_string(-7)


@pytest.mark.parametrize("name", ["sb_attn_kv4_store", "sb_attn_kv4_load"])
def test_rows(lib, name):
    call = getattr(lib, name)
    for i in range(6):
        args = [P] * 7
        args[i] = None
        assert call(*args, 1, 1, 1, 32, 64, None) == -1
        args[i] = ODD
        assert call(*args, 1, 1, 1, 32, 64, None) == -4
    assert call(*[P] * 6, ODD, 1, 1, 1, 32, 64, None) == -4
    for sizes, rc in (((0, 1, 1, 32, 64), -2), ((1, 0, 1, 32, 64), -2), ((1, 1, 0, 32, 64), -2), ((1, 1, 33, 32, 64), -2), ((1, 1, 1, 33, 64), -2),
                      ((1, 1, 1, 0, 64), -2), ((1, 1, 1, 32, 96), -3), ((1, 1, 1, 32, 0), -3), ((256, 256, 1, 32, 64), -2), ((1, 1, 1, 1 << 27, 64), -2),
                      ((60000, 1, 1, 1 << 20, 32), -2)):
        assert call(*[P] * 7, *sizes, None) == rc, sizes


def test_decode(lib):
    need = lib.sb_attn_decode_kv4_workspace_bytes(2, 8, 2, 5000, 5024, 64, 1)
    assert need > lib.sb_attn_decode_kv4_workspace_bytes(2, 8, 2, 5000, 5024, 64, 0) > 0
    def call(ptrs=(), sizes=(2, 8, 2, 5000, 5024, 64), ws=P, nbytes=need):
        args = dict(q=P, kc=P, ks=P, vc=P, vs=P, r=None, lens=None, score=None, score_out=P, o=P, m=None)
        args.update(ptrs)
        return lib.sb_attn_decode_kv4(*args.values(), ws, nbytes, *sizes, None)
    for n in ("q", "kc", "ks", "vc", "vs", "o"):
        assert call({n: None}) == -1
    for n in ("q", "kc", "ks", "vc", "vs", "o", "r", "lens", "score", "score_out", "m"):
        assert call({n: ODD}) == -4
    assert call({"score": P, "score_out": None}) == -1
    assert call(ws=None) == -6 and call(nbytes=need - 1) == -6 and call(ws=ODD) == -4
    for sizes, rc in (((0, 8, 2, 64, 64, 64), -2), ((1, 8, 3, 64, 64, 64), -2), ((1, 8, 0, 64, 64, 64), -2), ((1, 8, 2, 0, 64, 64), -2), ((1, 8, 2, 65, 64, 64), -2),
                      ((1, 8, 2, 64, 65, 64), -2), ((1, 8, 2, 64, 64, 48), -3), ((1, 8, 2, 524289, 524320, 64), -2), ((1, 2048, 1, 64, 64, 64), -2),
                      ((256, 256, 256, 64, 64, 64), -2)):
        assert call(sizes=sizes) == rc, sizes
        B, H, Hkv, T, Tcap, d = sizes
        assert lib.sb_attn_decode_kv4_workspace_bytes(B, H, Hkv, T, Tcap, d, 1) == 0


def test_key_weight(lib):
    need = lib.sb_attn_key_weight_workspace_bytes(2, 6, 2, 100, 300, 64)
    assert need > 0
    def call(ptrs=(), sizes=(2, 6, 2, 100, 300, 310, 64), ws=P, nbytes=need):
        args = dict(q=P, k=P, lens=None, qlens=None, score=None, score_out=P)
        args.update(ptrs)
        return lib.sb_attn_key_weight(*args.values(), ws, nbytes, *sizes, None)
    for n in ("q", "k", "score_out"):
        assert call({n: None}) == -1
    for n in ("q", "k", "lens", "qlens", "score", "score_out"):
        assert call({n: ODD}) == -4
    assert call(ws=None) == -6 and call(nbytes=need - 1) == -6 and call(ws=ODD) == -4
    for sizes, rc in (((0, 6, 2, 1, 8, 8, 64), -2), ((1, 6, 4, 1, 8, 8, 64), -2), ((1, 6, 2, 0, 8, 8, 64), -2), ((1, 6, 2, 9, 8, 8, 64), -2),
                      ((1, 6, 2, 1, 9, 8, 64), -2), ((1, 6, 2, 1, 8, 8, 16), -3), ((1, 6, 2, 1, 524289, 524289, 64), -2), ((1, 6, 2, 1, 0, 8, 64), -2)):
        assert call(sizes=sizes) == rc, sizes


def test_evict(lib):
    KB = 1024
    ptr = lambda *at: (ctypes.c_void_p * len(at))(*at)
    def call(src=(1 << 20,), dst=(2 << 20,), row=(16,), n=1, score=3 << 20, lens=None, score_out=4 << 20, index=5 << 20, lens_out=6 << 20,
             sizes=(1, 1, 8, 8, 8, 4, 1)):
        return lib.sb_attn_evict(score, lens, ptr(*src), ptr(*dst), (ctypes.c_int * len(row))(*row), n, score_out, index, lens_out, *sizes, None)
    for n in ("score", "score_out", "index", "lens_out"):
        assert call(**{n: None}) == -1
        assert call(**{n: 4096 + 8}) == -4
    assert call(src=(None,)) == -1 and call(dst=(None,)) == -1 and call(src=(KB + 8,)) == -4 and call(dst=(KB + 4,)) == -4
    assert lib.sb_attn_evict(P, None, None, None, None, 1, ctypes.c_void_p(1 << 20), P, P, 1, 1, 8, 8, 8, 4, 1, None) == -1
    assert call(n=-1) == -2 and call(n=9) == -2 and call(row=(0,)) == -2 and call(row=(65537,)) == -2
    for sizes in ((0, 1, 8, 8, 8, 4, 1), (1, 0, 8, 8, 8, 4, 1), (1, 1, 0, 8, 8, 4, 1), (1, 1, 9, 8, 8, 4, 1), (1, 1, 8, 8, 3, 4, 1), (1, 1, 8, 8, 8, 0, 0),
                  (1, 1, 8, 8, 8, 4, 5), (1, 1, 8, 8, 8, 4, -1), (256, 256, 8, 8, 8, 4, 1), (1, 1, 8, 1 << 27, 8, 4, 1)):
        assert call(sizes=sizes) == -2, sizes
    # in place, or into one another: 128 bytes of rows, 32 of scores
    assert call(src=(1 << 20,), dst=(1 << 20,)) == -7 and call(src=(1 << 20,), dst=((1 << 20) + 112,)) == -7
    assert call(score=3 << 20, score_out=(3 << 20) + 16) == -7 and call(lens=7 << 20, lens_out=7 << 20) == -7
    assert call(src=(1 << 20, 2 << 20), dst=(3 << 18, (2 << 20) + 64), row=(16, 16), n=2) == -7
    assert call(src=(1 << 20, 2 << 20), dst=(3 << 18, 3 << 18), row=(16, 16), n=2) == -7


def test_python_wants_tensors_on_the_gpu():
    from paper_2410_17980_amd import binding as sb
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    cache = (u8(1, 1, 32, 32), u8(1, 1, 32, 2), u8(1, 1, 32, 32), u8(1, 1, 32, 2))
    x, s = bf(1, 1, 1, 64), torch.zeros(1, 1, 32)
    for call in (lambda: sb.sb_attn_kv4_store(x, x, *cache), lambda: sb.sb_attn_kv4_load(*cache, 1),
                 lambda: sb.sb_attn_decode_kv4(bf(1, 1, 64), *cache), lambda: sb.sb_attn_key_weight(x, bf(1, 1, 32, 64)),
                 lambda: sb.sb_attn_evict(s, [bf(1, 1, 32, 64)], 4)):
        with pytest.raises(sb.SbAttnError, match="must live on the GPU"):
            call()
