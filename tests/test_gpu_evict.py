"""Eviction against the oracle (exactly), and the operators of a cache that is kept to a budget one after the other."""
import numpy as np
import pytest
import torch

from helpers import to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2410_17980_amd import binding
    binding.load(build_if_missing=False)
    return binding


def scores(B, Hkv, cap, seed, kind="mixed"):
    g = torch.Generator().manual_seed(seed)
    s = torch.exp(3 * torch.randn(B, Hkv, cap, generator=g) - 4)
    if kind == "zeros":
        s[:] = 0.0
    elif kind == "ties":
        s = torch.randint(0, 4, s.shape, generator=g).float() * 0.37
    elif kind == "signs":                     # both zeros and negative numbers among them
        s = torch.randn(B, Hkv, cap, generator=g) * torch.randint(-1, 2, s.shape, generator=g)
    elif kind == "tiny":                      # subnormal ones
        s *= 1e-39
    else:
        s[:, ::2, :cap // 2] = 0.0
    return s


def rows_of(B, Hkv, cap, widths, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randint(0, 256, (B, Hkv, cap, w), generator=g).to(torch.uint8).cuda() for w in widths]


def check(sb, oracle, s, rows, keep, recent, T=None, lens=None, cap_out=None):
    B, Hkv, cap = s.shape
    cap_out = cap_out or cap
    bound = cap if T is None else T
    at = [min(max(x, 0), bound) for x in lens] if lens is not None else [bound] * B
    sd = s.cuda()
    for b in range(B):                        # what lies behind an entry's rows does not count
        sd[b, :, at[b]:] = float("inf")
    out = [torch.full((B, Hkv, cap_out) + t.shape[3:], 0x77, device="cuda").to(t.dtype) for t in rows]
    clean = [t.clone() for t in out]
    score_out = torch.full((B, Hkv, cap_out), -7.0, device="cuda")
    index = torch.full((B, Hkv, keep), 12345, dtype=torch.int32, device="cuda")
    ld = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens is not None else None
    got, so, lo, ix = sb.sb_attn_evict(sd, rows, keep, recent=recent, T=T, lens=ld, out=out, score_out=score_out, index=index)
    torch.cuda.synchronize()
    assert all(a is b or a.data_ptr() == b.data_ptr() for a, b in zip(got, out)) and so is score_out and ix is index
    assert lo.tolist() == [min(n, keep) for n in at]
    for b in range(B):
        for h in range(Hkv):
            want = oracle.evict(s[b, h].numpy(), at[b], keep, recent)
            n = len(want)
            assert ix[b, h].tolist() == want + [-1] * (keep - n)
            w = torch.tensor(want, dtype=torch.long, device="cuda")
            assert torch.equal(so[b, h, :n], sd[b, h, w]) and (so[b, h, n:] == -7.0).all()
            for a, r, c in zip(got, rows, clean):
                assert torch.equal(a[b, h, :n], r[b, h, w]) and torch.equal(a[b, h, n:], c[b, h, n:])


@pytest.mark.parametrize("kind", ["mixed", "zeros", "ties", "signs", "tiny"])
@pytest.mark.parametrize("T,keep,recent", [(1, 1, 0), (5, 3, 1), (5, 5, 5), (64, 63, 0), (100, 30, 30), (1023, 500, 7), (1025, 1024, 0), (3000, 64, 32), (5000, 4097, 1000)])
def test_selection(sb, oracle, T, keep, recent, kind):
    check(sb, oracle, scores(2, 3, T, T + keep, kind), rows_of(2, 3, T, (16, 1), 1), keep, recent)


@pytest.mark.parametrize("widths", [(), (1,), (2, 4, 8), (16, 64, 256), (3, 12, 48), (20, 5), (64, 4, 64, 4), (1, 2, 3, 4, 5, 6, 7, 8), (1000,)])
def test_rows_of_any_width(sb, oracle, widths):
    check(sb, oracle, scores(2, 2, 300, 2), rows_of(2, 2, 300, widths, 3), 170, 20, cap_out=200)


def test_entries_of_different_lengths(sb, oracle):
    lens = [0, 1, 10, 99, 100, 101, 2000, 2100, 5000, -3]
    s = scores(len(lens), 2, 2100, 4)
    for keep, recent in ((100, 0), (100, 100), (100, 13), (1, 1), (2100, 5)):
        check(sb, oracle, s, rows_of(len(lens), 2, 2100, (32, 2), 5), keep, recent, lens=lens)
    check(sb, oracle, s, rows_of(len(lens), 2, 2100, (32, 2), 5), 700, 50, T=1500, lens=lens, cap_out=704)


def test_more_room_than_rows(sb, oracle):
    check(sb, oracle, scores(1, 2, 50, 6), rows_of(1, 2, 50, (16,), 7), 200, 10, cap_out=224)


def test_nan_and_infinities(sb):
    s = torch.zeros(1, 1, 64, device="cuda")
    s[0, 0, 3], s[0, 0, 9], s[0, 0, 20], s[0, 0, 30] = float("nan"), float("inf"), -float("inf"), 1.0
    pick = lambda keep: sb.sb_attn_evict(s, [], keep)[3][0, 0].tolist()
    assert pick(1) == [3] and pick(2) == [3, 9] and pick(3) == [3, 9, 30] and pick(4) == [0, 3, 9, 30]
    assert 20 not in pick(63)


def test_long_caches(sb, oracle):
    T = 200_000
    s = scores(1, 2, T, 8)
    _, so, _, ix = sb.sb_attn_evict(s.cuda(), [], 60_000, recent=500)
    for h in range(2):
        order = np.lexsort((np.arange(T - 500), -s[0, h, :T - 500].numpy().astype(np.float64)))[:59_500]
        assert np.array_equal(ix[0, h].cpu().numpy(), np.concatenate((np.sort(order), np.arange(T - 500, T))))


def test_outputs_that_are_not_given(sb):
    s = scores(2, 2, 96, 9).cuda()
    k = torch.randn(2, 2, 96, 64, device="cuda").bfloat16()
    c = torch.randint(0, 255, (2, 2, 96, 4, 3), device="cuda", dtype=torch.int32)
    out, so, lo, ix = sb.sb_attn_evict(s, [k, c], 40, recent=8)
    assert [t.shape for t in out] == [k.shape, c.shape] and so.shape == s.shape and ix.shape == (2, 2, 40) and lo.tolist() == [40, 40]
    at = ix.long()
    assert torch.equal(out[0][:, :, :40], torch.gather(k, 2, at[..., None].expand(-1, -1, -1, 64)))
    assert torch.equal(out[1][:, :, :40], torch.gather(c, 2, at[..., None, None].expand(-1, -1, -1, 4, 3)))
    assert torch.equal(so[:, :, :40], torch.gather(s, 2, at))


def test_captured(sb):
    s = scores(2, 3, 3000, 10).cuda()
    k = rows_of(2, 3, 3000, (64,), 11)
    lens = torch.tensor([3000, 1500], dtype=torch.int32, device="cuda")
    out = [torch.zeros_like(k[0])]
    so, lo, ix = torch.zeros_like(s), torch.zeros_like(lens), torch.zeros(2, 3, 1000, dtype=torch.int32, device="cuda")
    step = lambda: sb.sb_attn_evict(s, k, 1000, recent=64, lens=lens, out=out, score_out=so, lens_out=lo, index=ix)
    cases = [(scores(2, 3, 3000, 12 + i).cuda(), n) for i, n in enumerate(([3000, 1500], [900, 2000], [0, 1001]))]
    def once(x, n):
        s.copy_(x)
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        for t in (*out, so, lo, ix):
            t.zero_()
    want = []
    for c in cases:
        once(*c)
        step()
        want.append([t.clone() for t in (*out, so, lo, ix)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(2):
        for c, w in zip(cases, want):
            once(*c)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((*out, so, lo, ix), w))


def test_refusals(sb):
    s = torch.zeros(2, 2, 64, device="cuda")
    k = torch.zeros(2, 2, 64, 64, device="cuda").bfloat16()
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    for call, why in ((lambda: sb.sb_attn_evict(s, [k], 65), "more rows"), (lambda: sb.sb_attn_evict(s, [k], 0), "keep"), (lambda: sb.sb_attn_evict(s, [k], 4, recent=5), "bad shape"),
                      (lambda: sb.sb_attn_evict(s, [k], 4, recent=-1), "bad shape"), (lambda: sb.sb_attn_evict(s, [k], 4, T=65), "bad shape"),
                      (lambda: sb.sb_attn_evict(s, [k], 4, out=[k]), "overlaps"), (lambda: sb.sb_attn_evict(s, [], 4, score_out=s), "overlaps"),
                      (lambda: sb.sb_attn_evict(s, [], 4, lens=lens, lens_out=lens), "overlaps"), (lambda: sb.sb_attn_evict(s, [k[:, :, :63]], 4), "expected"),
                      (lambda: sb.sb_attn_evict(s, [k.transpose(0, 1)], 4), "contiguous"), (lambda: sb.sb_attn_evict(s, [k] * 9, 4), "at most 8"),
                      (lambda: sb.sb_attn_evict(s, [k], 4, out=[]), "as many"), (lambda: sb.sb_attn_evict(s.double(), [k], 4), "must be torch.float32"),
                      (lambda: sb.sb_attn_evict(s, [k.cpu()], 4), "must live on the GPU"), (lambda: sb.sb_attn_evict(s, [k], 4, out=[torch.zeros_like(k).half()]), "must be torch.bfloat16"),
                      (lambda: sb.sb_attn_evict(s, [k], 4, index=torch.zeros(2, 2, 5, dtype=torch.int32, device="cuda")), "has shape")):
        with pytest.raises(sb.SbAttnError, match=why):
            call()


@pytest.mark.parametrize("d", [32, 128])
def test_a_generation_kept_to_a_budget(sb, oracle, d):
    """A padded batch of prompts into a 4-bit cache, the keys' scores from the prompts' queries, then tokens: decode with scores,
    append, and eviction whenever an entry reaches the budget's end.  Every step's o and scores against the oracle on the rows that are left."""
    from paper_2410_17980_amd import inputs as gen
    B, H, Hkv, T, steps, cap, keep, recent = 2, 4, 2, 200, 60, 224, 96, 16
    G = H // Hkv
    q, k, v = gen.gaussian(B, H, T + steps, d, seed=21)
    far = (6.0 * d ** 0.5) ** 0.5
    q[:, G:, :, d - 1], k[:, :, :, d - 1] = far, -far          # the second kv head reaches far
    q, k, v = (t.to(torch.bfloat16) for t in (q, k[:, :Hkv], v[:, :Hkv]))
    n = [200, 131]
    lens = torch.tensor(n, dtype=torch.int32, device="cuda")
    prompt = lambda x: x[:, :, :T].contiguous().cuda()
    cache = [torch.full((B, Hkv, cap, w), 0xFF, dtype=torch.uint8, device="cuda") for w in (d // 2, d // 32, d // 2, d // 32)]
    spare = [t.clone() for t in cache]
    sb.sb_attn_kv4_store(prompt(k), prompt(v), *cache)
    score = torch.zeros(B, Hkv, cap, device="cuda")
    score[:, :, :T] = sb.sb_attn_key_weight(prompt(q), prompt(k), lens=lens, qlens=lens, score=torch.zeros(B, Hkv, T, device="cuda"))
    # the same in 64 bits: rows (values of k and v) and scores as lists
    val = lambda x: oracle.kv4_values(*oracle.kv4(to64(x)))
    kv, vv = val(k), val(v)
    held = [[list(range(n[b])) for _ in range(Hkv)] for b in range(B)]           # the tokens that the rows stand for
    ref = [[list(x[:n[b]]) for x in oracle.key_weight(to64(q)[b:b + 1, :, :n[b]], to64(k)[b:b + 1, :, :n[b]])[0]] for b in range(B)]
    for t in range(steps):
        tok = [n[b] + t for b in range(B)]
        pick = lambda x: torch.stack([x[b, :, tok[b]] for b in range(B)]).cuda()
        o, _ = sb.sb_attn_decode_kv4(pick(q), *cache, lens=lens, score=score)
        sb.sb_attn_kv4_store(pick(k)[:, :, None].contiguous(), pick(v)[:, :, None].contiguous(), *cache, pos=lens)
        score[torch.arange(B), :, lens.long()] = 0.0
        lens += 1
        for b in range(B):
            for h in range(H):
                g = h // G
                A, _ = oracle.row_weights(to64(q)[b, h, tok[b]], kv[b, g, held[b][g]])
                want = A @ vv[b, g, held[b][g]]
                # 64 bits and fp32 part by 2^-8 of o (its rounding) and the weights' errors (2^-16 and some 300 2^-23) times the largest value
                assert (np.abs(to64(o)[b, h] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -13 * np.abs(vv).max()).all(), (t, b, h)
                for i, a in enumerate(A):
                    ref[b][g][i] += a
            for g in range(Hkv):
                held[b][g].append(tok[b])
                ref[b][g].append(0.0)
        if int(lens.max()) >= 210:
            cache_was, kept = [t.clone() for t in cache], lens.clone()
            spare, score, lens, index = sb.sb_attn_evict(score, cache, keep, recent=recent, lens=lens, out=spare)
            cache, spare = list(spare), cache
            for b in range(B):
                for g in range(Hkv):
                    at = [i for i in index[b, g].tolist() if i >= 0]
                    m = min(int(kept[b]), keep)
                    assert len(at) == m and at == sorted(set(at))
                    # what stays weighs no less than what goes, as far as the scores' errors let one tell
                    gone = [i for i in range(int(kept[b]) - recent) if i not in set(at)]
                    low = min((ref[b][g][i] for i in at if i < int(kept[b]) - recent), default=np.inf)
                    assert max((ref[b][g][i] for i in gone), default=0.0) <= low + 1e-3
                    held[b][g], ref[b][g] = [held[b][g][i] for i in at], [ref[b][g][i] for i in at]
        for b in range(B):
            for g in range(Hkv):
                m = int(lens[b])
                # T + 60 queries of G heads, each weight off by some 500 2^-23 at most
                assert len(held[b][g]) == m and np.abs(to64(score)[b, g, :m] - np.array(ref[b][g])).max() <= 1e-3
