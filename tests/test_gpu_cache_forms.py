"""The forms that decode on a 4-bit cache, the key weights and eviction take by their sizes, and their calls on streams of their own."""
import numpy as np
import pytest
import torch

from helpers import to64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24            # half a step of fp32, relative
BUSY = 100_000_000        # clocks: about 0.05 s


@pytest.fixture(scope="module")
def sb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2410_17980_amd import binding
    binding.load(build_if_missing=False)
    return binding


def new_cache(B, Hkv, Tcap, d):
    return [torch.full((B, Hkv, Tcap, w), 0xFF, dtype=torch.uint8, device="cuda") for w in (d // 2, d // 32, d // 2, d // 32)]


def activations(B, H, Hkv, T, d, seed):
    """By kv head in turn: N(0,1), and logits around -6, whose weights reach far."""
    g = torch.Generator().manual_seed(seed)
    q, k, v = torch.randn(B, H, d, generator=g), torch.randn(B, Hkv, T, d, generator=g), torch.randn(B, Hkv, T, d, generator=g)
    far = (6.0 * d ** 0.5) ** 0.5
    k[:, 1::2, :, d - 1] = -far
    q.view(B, Hkv, H // Hkv, d)[:, 1::2, :, d - 1] = far
    return tuple(t.to(torch.bfloat16).cuda() for t in (q, k, v))


# Workgroups of the near launch (entries x kv heads) beyond what the chip holds at once, where half as many waves take a kv head: d = 128 from 257,
# d = 64 and 32 from 513; up to four query heads a kv head; short caches, ends inside a round, and such that need the far launch as well
@pytest.mark.parametrize("want_m", [False, True])
@pytest.mark.parametrize("B,H,Hkv,T,d", [(37, 8, 8, 200, 128), (37, 16, 8, 1000, 128), (33, 32, 8, 300, 128), (70, 8, 8, 33, 64), (65, 32, 8, 1500, 32), (33, 8, 8, 3500, 128),
                                         (33, 40, 8, 300, 128), (66, 16, 8, 3600, 64), (33, 16, 16, 4200, 32), (33, 8, 8, 4200, 64)])
def test_decode_of_many_heads(sb, oracle, B, H, Hkv, T, d, want_m):
    """Against the oracle for a sample of entries, in the bounds of the 4-bit decode's tests: a weight is off by rel = (T + 64) 2^-23 + 8 dz of it,
    o by that, by 2^-16 of the largest value, and by half a step (2^-8); and every entry as it comes out of a call of its own."""
    q, k, v = activations(B, H, Hkv, T, d, seed=B + T)
    cap = (T + 31) // 32 * 32 + 32
    cache = new_cache(B, Hkv, cap, d)
    sb.sb_attn_kv4_store(k, v, *cache)
    lens = [T] * B
    lens[1], lens[2], lens[3], lens[4], lens[B - 1] = 0, 1, min(T, 65), T - 1, T // 2 + 5
    ld = torch.tensor(lens, dtype=torch.int32, device="cuda")
    was = torch.rand(B, Hkv, cap, generator=torch.Generator().manual_seed(2)).cuda()
    got = sb.sb_attn_decode_kv4(q, *cache, T=T, lens=ld, score=was, score_out=torch.full_like(was, -7.0), want_m=want_m)
    torch.cuda.synchronize()
    G = H // Hkv
    held = lambda i, b: oracle.kv4_values(np.stack((cache[i][b].cpu().numpy() & 15, cache[i][b].cpu().numpy() >> 4), -1).reshape(Hkv, cap, d), cache[i + 1][b].cpu().numpy())
    for b in (0, 1, 2, 3, 4, B // 2, B - 1):
        kb, vb, n = held(0, b), held(2, b), lens[b]
        for g in range(Hkv):
            total, rel = np.zeros(n), 0.0
            for h in range(g * G, (g + 1) * G):
                qh = to64(q)[b, h]
                A, left = oracle.row_weights(qh, kb[g, :n])
                dz = d * U * (np.abs(kb[g, :n]) @ np.abs(qh)).max(initial=0.0) / np.sqrt(d)
                rel = max(rel, (n + 64) * 2 * U + 8 * dz)
                want = A @ vb[g, :n]
                tol = 2.0 ** -8 * np.abs(want) + np.abs(vb[g, :n]).max(initial=0.0) * (2.0 ** -16 + rel)
                assert (np.abs(to64(got[0])[b, h] - want) <= tol).all(), (b, h)
                if want_m and left > 1e-290:
                    assert abs(to64(got[1])[b, h] - np.log(left)) <= 2e-3 + 2e-3 * abs(np.log(left)), (b, h)
                total += A
            s, ref = to64(got[-1])[b, g], to64(was)[b, g, :n] + total
            assert (np.abs(s[:n] - ref) <= G * rel + 2 * U * (G + 1) * ref).all(), (b, g)
            assert (s[n:] == -7.0).all()
    # o of the call without scores is the same: scores change nothing else
    plain = sb.sb_attn_decode_kv4(q, *cache, T=T, lens=ld, want_m=want_m)
    assert torch.equal(plain[0] if want_m else plain, got[0])


@pytest.mark.parametrize("kind", ["mixed", "ties", "zeros"])
@pytest.mark.parametrize("T,keep,recent", [(16385, 8000, 100), (40000, 39999, 0), (65536, 20000, 20000), (65536, 1, 0), (65537, 30000, 64)])
def test_eviction_of_long_caches(sb, oracle, T, keep, recent, kind):
    g = torch.Generator().manual_seed(T)
    s = torch.exp(3 * torch.randn(2, 2, T, generator=g) - 4)
    if kind == "ties":
        s = torch.randint(0, 4, s.shape, generator=g).float() * 0.37
    elif kind == "zeros":
        s[:, :, ::3] = 0.0
        s[0] = 0.0
    lens = [T, T - 777]
    k = torch.randint(0, 256, (2, 2, T, 8), generator=g).to(torch.uint8).cuda()
    out, so, lo, ix = sb.sb_attn_evict(s.cuda(), [k], keep, recent=recent, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    assert lo.tolist() == [min(n, keep) for n in lens]
    for b in range(2):
        for h in range(2):
            n, older = lens[b], lens[b] - recent if lens[b] > keep else 0
            order = np.lexsort((np.arange(older), -s[b, h, :older].numpy().astype(np.float64)))[:min(n, keep) - (n - older)]
            want = np.concatenate((np.sort(order), np.arange(older, n)))
            w = torch.tensor(want, device="cuda")
            assert ix[b, h].tolist() == want.tolist() + [-1] * (keep - len(want))
            assert torch.equal(so[b, h, :len(want)], s.cuda()[b, h, w]) and torch.equal(out[0][b, h, :len(want)], k[b, h, w])


@pytest.fixture(scope="module")
def calls(sb):
    """name -> call(stream=...) that leaves every output and workspace to the library"""
    B, H, Hkv, T, d = 2, 6, 2, 4096, 64
    q, k, v = activations(B, H, Hkv, T, d, seed=31)
    qs = torch.randn(B, H, 300, d, generator=torch.Generator().manual_seed(32)).bfloat16().cuda()
    cache = new_cache(B, Hkv, T, d)
    sb.sb_attn_kv4_store(k, v, *cache)
    score = torch.rand(B, Hkv, T, generator=torch.Generator().manual_seed(33)).cuda()
    into = [torch.zeros_like(score) for _ in range(2)]
    torch.cuda.synchronize()
    def evict(**kw):
        out, so, lo, ix = sb.sb_attn_evict(score, cache, 4000, recent=10, **kw)
        return (*out, so, lo, ix)
    return {
        "load": lambda **kw: sb.sb_attn_kv4_load(*cache, 1000, **kw),
        "decode": lambda **kw: sb.sb_attn_decode_kv4(q, *cache, want_m=True, **kw),
        "decode_scores": lambda **kw: sb.sb_attn_decode_kv4(q, *cache, want_m=True, score=score, score_out=into[0], **kw)[:2],
        "key_weight": lambda **kw: (sb.sb_attn_key_weight(qs, k, **kw),),
        "evict": evict,
    }


NAMES = ("load", "decode", "decode_scores", "key_weight", "evict")


def written(name, got):
    """What the call writes: of an eviction's outputs the first rows."""
    return got if name != "evict" else [t[:, :, :4000] if t.dim() > 2 else t for t in got]


def memory_of(stream):
    return [(s["address"], s["address"] + s["total_size"]) for s in torch.cuda.memory_snapshot() if s["stream"] == stream.cuda_stream]


@pytest.mark.parametrize("name", NAMES)
def test_outputs_do_not_take_memory_that_is_still_written(calls, name):
    """Memory freed on the current stream, with a write to it still queued there, is not a result's."""
    call = calls[name]
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    for t in want:                                   # the sizes that the call will ask for
        for _ in range(3):
            torch.empty_like(t).fill_(77)
    got = call(stream=side)
    torch.cuda.synchronize()
    blocks = memory_of(side)
    for a in got:
        assert any(lo <= a.data_ptr() < hi for lo, hi in blocks)
    for a, b in zip(written(name, got), written(name, want)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", NAMES)
def test_dropped_outputs_wait_for_their_readers(calls, name):
    """A result that is dropped while the current stream has a read of it queued is not the next call's memory."""
    call = calls[name]
    want = call()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(BUSY)
    copies = [t.clone() for t in got]
    held = {t.data_ptr() for t in got}
    del got
    again = call(stream=side)
    assert not held & {t.data_ptr() for t in again}
    torch.cuda.synchronize()
    for a, b in zip(written(name, copies), written(name, want)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", NAMES)
def test_two_calls_at_once(calls, name):
    """Calls on two streams, each with a workspace of its own, do not meet."""
    call = calls[name]
    want = [t.clone() for t in written(name, call())]
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for s in sides:
            got.append(call(stream=s))
    torch.cuda.synchronize()
    for x in got:
        for a, b in zip(written(name, x), want):
            assert torch.equal(a, b)


def test_store_goes_to_its_stream(sb):
    """Behind what the stream has queued, not the current one."""
    x = torch.randn(1, 2, 64, 64, generator=torch.Generator().manual_seed(34)).bfloat16().cuda()
    want = new_cache(1, 2, 64, 64)
    sb.sb_attn_kv4_store(x, x, *want)
    cache, y = new_cache(1, 2, 64, 64), torch.zeros_like(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
        y.copy_(x)
    sb.sb_attn_kv4_store(y, y, *cache, stream=side)
    torch.cuda.synchronize()
    for a, b in zip(cache, want):
        assert torch.equal(a, b)


# Two units a wave where the work of all, by the keys that a query sees, is some 7000 whole units of 32 query rows (more where the last 64 keys are few).  Groups whose heads end inside a pair, an odd number of strips,
# windows, padded entries; and fewer units beside them
@pytest.mark.parametrize("B,H,Hkv,Tq,T,d", [(128, 96, 32, 70, 70, 32), (70, 96, 96, 95, 95, 64), (48, 32, 8, 300, 300, 128), (52, 30, 2, 300, 333, 64), (128, 64, 16, 33, 200, 128),
                                              (9, 32, 8, 300, 300, 128)])
def test_key_weights_of_many_units(sb, oracle, B, H, Hkv, Tq, T, d):
    """Every entry as a call of its own gives it (which is held against the oracle elsewhere), and some against the oracle.  A weight is off by
    rel = (T + 64) 2^-23 + 8 dz of it, dz what d products and sums in fp32 are off in a logit of the largest q and k; a key's sum by that share of itself,
    and by a rounding of half a step for each of its Tq G terms: once against the oracle, twice between two calls."""
    g = torch.Generator().manual_seed(B + T)
    G, far = H // Hkv, (6.0 * d ** 0.5) ** 0.5
    q, k = torch.randn(B, H, Tq, d, generator=g), torch.randn(B, Hkv, T, d, generator=g)
    k[:, 1::2, :, d - 1] = -far
    q.view(B, Hkv, G, Tq, d)[:, 1::2, ..., d - 1] = far
    q, k = q.bfloat16(), k.bfloat16()
    lens, qlens = [T] * B, [Tq] * B
    lens[1], lens[2], lens[3], lens[B - 1] = 0, 1, T // 2, T - 3
    qlens[1], qlens[2], qlens[3], qlens[4] = 0, 1, min(Tq, T // 2), Tq - 1
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    qd, kd = q.cuda(), k.cuda()
    for b in range(B):                                   # padding is anything at all
        kd[b, :, lens[b]:], qd[b, :, qlens[b]:] = float("nan"), float("nan")
    was = torch.rand(B, Hkv, T, generator=g).cuda()
    got = sb.sb_attn_key_weight(qd, kd, lens=ints(lens), qlens=ints(qlens), score=was, score_out=torch.full_like(was, -7.0))
    dz = d * U * float(q.abs().max()) * float(k.abs().float().sum(-1).max()) / d ** 0.5 / 4
    rel = (T + 64) * 2 * U + 8 * dz
    bound = lambda want, ref: rel * (1.0 + want) + (Tq * G + 2) * U * ref
    for b in range(B):
        n = lens[b]
        one = sb.sb_attn_key_weight(qd[b:b + 1].clone(), kd[b:b + 1].clone(), lens=ints(lens[b:b + 1]), qlens=ints(qlens[b:b + 1]), score=was[b:b + 1].clone(), score_out=torch.empty_like(was[b:b + 1]))
        a, c, w = to64(got[b, :, :n]), to64(one[0, :, :n]), to64(was[b, :, :n])
        assert (np.abs(a - c) <= 2 * bound(c - w, c)).all(), b
        assert (got[b, :, n:] == -7.0).all()
    for b in (0, 1, 2, 3, 4, B - 1):
        n, m = lens[b], qlens[b]
        want = oracle.key_weight(to64(q)[b:b + 1, :, :m], to64(k)[b:b + 1, :, :n])[0]
        ref = want + to64(was)[b, :, :n]
        assert (np.abs(to64(got)[b, :, :n] - ref) <= bound(want, ref)).all(), b


@pytest.mark.parametrize("T", [131_073, 524_288])
@pytest.mark.parametrize("want_m", [False, True])
def test_decode_of_the_longest_caches(sb, oracle, T, want_m):
    """Logits around -12, so that the last of 524288 keys still counts.  Bounds as in test_decode_of_many_heads."""
    B, H, Hkv, d = 1, 4, 2, 32
    g = torch.Generator().manual_seed(T)
    q, k, v = torch.randn(B, H, d, generator=g), torch.randn(B, Hkv, T, d, generator=g), torch.randn(B, Hkv, T, d, generator=g)
    k[:, 1, :, d - 1], q[:, 2:, d - 1] = -8.0, 12.0 * d ** 0.5 / 8.0
    q, k, v = (t.bfloat16().cuda() for t in (q, k, v))
    cap = (T + 31) // 32 * 32
    cache = new_cache(B, Hkv, cap, d)
    sb.sb_attn_kv4_store(k, v, *cache)
    k4, v4 = (to64(t)[0] for t in sb.sb_attn_kv4_load(*cache, T))
    got = sb.sb_attn_decode_kv4(q, *cache, T=T, score_out=torch.zeros(B, Hkv, cap, device="cuda"), want_m=want_m)
    for h in range(Hkv):
        total, rel = np.zeros(T), 0.0
        for i in (2 * h, 2 * h + 1):
            qi = to64(q)[0, i]
            A, left = oracle.row_weights(qi, k4[h])
            dz = d * U * (np.abs(k4[h]) @ np.abs(qi)).max() / np.sqrt(d)
            rel = max(rel, (T + 64) * 2 * U + 8 * dz)
            want = A @ v4[h]
            assert (np.abs(to64(got[0])[0, i] - want) <= 2.0 ** -8 * np.abs(want) + np.abs(v4[h]).max() * (2.0 ** -16 + rel)).all()
            total += A
        s = to64(got[-1])[0, h, :T]
        assert (np.abs(s - total) <= 2 * rel * total + 6 * U * total + 1e-37).all()          # of each weight itself
        assert h == 0 or total[0] > 1e-8


@pytest.mark.parametrize("Tq", [1, 40])
def test_key_weights_of_the_longest_caches(sb, oracle, Tq):
    T, d = 524_288, 32
    g = torch.Generator().manual_seed(Tq)
    q, k = torch.randn(1, 1, Tq, d, generator=g), torch.randn(1, 1, T, d, generator=g)
    k[..., d - 1], q[..., d - 1] = -8.0, 12.0 * d ** 0.5 / 8.0
    q, k = q.bfloat16(), k.bfloat16()
    got = to64(sb.sb_attn_key_weight(q.cuda(), k.cuda()))[0, 0]
    want = oracle.key_weight(to64(q), to64(k))[0, 0]
    dz = d * U * float(q.abs().float().max()) * float(k.abs().float().sum(-1).max()) / d ** 0.5
    assert (np.abs(got - want) <= ((T + 64) * 2 * U + 8 * dz + (Tq + 2) * U) * want + 1e-37).all() and want[0] > 1e-8


def test_entries_beyond_four_gigabytes(sb):
    """The last of three entries of a cache of 2^25 rows, as the same rows in a small cache give it."""
    big, small, n, d = 1 << 25, 2080, 2048, 64
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("not enough memory")
    q, k, v = activations(1, 2, 1, n, d, seed=40)
    part = new_cache(1, 1, small, d)
    sb.sb_attn_kv4_store(k, v, *part)
    cache = [torch.zeros(3, 1, big, t.shape[-1], dtype=torch.uint8, device="cuda") for t in part]
    for a, b in zip(cache, part):
        a[2, :, :small] = b[0]
    lens = torch.tensor([0, 0, n], dtype=torch.int32, device="cuda")
    q3 = q.expand(3, -1, -1).contiguous()
    score = torch.zeros(3, 1, big, device="cuda")
    o, s = sb.sb_attn_decode_kv4(q3, *cache, T=n, lens=lens, score=score)
    o1, s1 = sb.sb_attn_decode_kv4(q, *part, T=n, score=torch.zeros(1, 1, small, device="cuda"))
    assert torch.equal(o[2], o1[0]) and torch.equal(s[2, 0, :n], s1[0, 0, :n]) and not s[2, 0, n:].any() and not o[:2].any()
    out, so, lo, ix = sb.sb_attn_evict(s, cache, 1000, recent=10, T=n, lens=lens, out=[torch.zeros(3, 1, 1024, t.shape[-1], dtype=torch.uint8, device="cuda") for t in cache])
    out1, so1, _, ix1 = sb.sb_attn_evict(s1, part, 1000, recent=10, T=n)
    assert lo.tolist() == [0, 0, 1000] and torch.equal(ix[2], ix1[0]) and torch.equal(so[2, 0, :1000], so1[0, 0, :1000])
    assert all(torch.equal(a[2, 0, :1000], b[0, 0, :1000]) and not a[:2].any() for a, b in zip(out, out1))
    del cache, score, s, out
    kb = torch.zeros(3, 1, big, d, dtype=torch.bfloat16, device="cuda")
    kb[2, :, :n] = k[0]
    qs = torch.randn(1, 2, 100, d, generator=torch.Generator().manual_seed(41)).bfloat16().cuda()
    w = sb.sb_attn_key_weight(qs.expand(3, -1, -1, -1).contiguous(), kb, T=n, lens=lens)
    w1 = sb.sb_attn_key_weight(qs, k)
    assert torch.allclose(w[2, 0, :n], w1[0, 0], rtol=1e-5, atol=1e-7)
