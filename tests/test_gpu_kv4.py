"""The 4-bit cache on the GPU: rows in and out of it against the oracle, exactly, and single-token decode on it against the oracle
in 64 bits on the values that the cache stands for."""
import numpy as np
import pytest
import torch

from helpers import nan_bytes, to64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24            # half a step of fp32, relative


@pytest.fixture(scope="module")
def sb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2410_17980_amd import binding
    binding.load(build_if_missing=False)
    return binding


@pytest.fixture(scope="module")
def gen():
    from paper_2410_17980_amd import inputs
    return inputs


def empty_cache(B, Hkv, Tcap, d, fill=0xFF):
    """Codes and scales of nothing: every value a NaN."""
    new = lambda w: torch.full((B, Hkv, Tcap, w), fill, dtype=torch.uint8, device="cuda")
    return new(d // 2), new(d // 32), new(d // 2), new(d // 32)


def unpacked(codes):
    c = codes.cpu().numpy()
    return np.stack((c & 15, c >> 4), -1).reshape(c.shape[:-1] + (-1,))


def values(oracle, codes, scales):
    return oracle.kv4_values(unpacked(codes), scales.cpu().numpy())


def rows(B, Hkv, n, d, seed):
    """Values over many binades, with what rounds in a tie, exact powers of two, zeros and whole blocks of zeros among them."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, Hkv, n, d, generator=g) * torch.exp2(torch.randint(-20, 20, (B, Hkv, n, 1), generator=g).float())
    pick = torch.randint(0, 8, x.shape, generator=g)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])[torch.randint(0, 8, x.shape, generator=g)] * torch.where(x < 0, -1.0, 1.0)
    x = torch.where(pick == 0, 0.0, torch.where(pick == 1, ties, x))
    x[:, :, ::5, :32] = 0.0
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("B,Hkv,n,Tcap", [(1, 1, 1, 32), (2, 3, 7, 64), (3, 2, 300, 320), (1, 1, 96, 96)])
def test_store_and_load(sb, oracle, B, Hkv, n, Tcap, d):
    k, v = rows(B, Hkv, n, d, 1), rows(B, Hkv, n, d, 2)
    cache = empty_cache(B, Hkv, Tcap, d, fill=0x5A)
    sb.sb_attn_kv4_store(k.cuda(), v.cuda(), *cache)
    got = sb.sb_attn_kv4_load(*cache, n)
    torch.cuda.synchronize()
    for x, codes, scales, y in ((k, *cache[:2], got[0]), (v, *cache[2:], got[1])):
        want, byte = oracle.kv4(to64(x))
        assert np.array_equal(unpacked(codes)[:, :, :n], want)
        assert np.array_equal(scales.cpu().numpy()[:, :, :n], byte)
        assert np.array_equal(to64(y), oracle.kv4_values(want, byte))
        assert (codes[:, :, n:] == 0x5A).all() and (scales[:, :, n:] == 0x5A).all()


@pytest.mark.parametrize("d", [32, 128])
def test_positions(sb, oracle, d):
    """Rows of every entry at its own place; those outside the cache are left out, and read as zeros."""
    B, Hkv, n, Tcap = 5, 2, 20, 64
    pos = torch.tensor([0, 13, 44, 50, -7], dtype=torch.int32)
    k, v = rows(B, Hkv, n, d, 3), rows(B, Hkv, n, d, 4)
    cache = empty_cache(B, Hkv, Tcap, d, fill=0x7E)
    sb.sb_attn_kv4_store(k.cuda(), v.cuda(), *cache, pos=pos.cuda())
    got = sb.sb_attn_kv4_load(*cache, n, pos=pos.cuda())
    torch.cuda.synchronize()
    for x, codes, scales, y in ((k, *cache[:2], got[0]), (v, *cache[2:], got[1])):
        want, byte = oracle.kv4(to64(x))
        held = np.full((B, Hkv, Tcap, d // 2), 0x7E, dtype=np.uint8)
        back = np.zeros((B, Hkv, n, d))
        for b, p in enumerate(pos.tolist()):
            t = [i for i in range(n) if 0 <= p + i < Tcap]
            held[b, :, [p + i for i in t]] = (want[b, :, t, 0::2] + 16 * want[b, :, t, 1::2])
            back[b, :, t] = oracle.kv4_values(want, byte)[b, :, t]
        assert np.array_equal(codes.cpu().numpy(), held)
        assert np.array_equal(to64(y), back)


def test_far_positions_of_a_large_cache(sb):
    """Rows beyond byte 2^32 of the codes."""
    Tcap, d = 1 << 25, 128
    free, _ = torch.cuda.mem_get_info()
    if free < 6 * Tcap * (d // 2):
        pytest.skip("not enough memory")
    cache = [torch.zeros(3, 1, Tcap, w, dtype=torch.uint8, device="cuda") for w in (64, 4, 64, 4)]
    x = rows(3, 1, 8, d, 5).cuda()
    pos = torch.tensor([Tcap - 8] * 3, dtype=torch.int32, device="cuda")
    sb.sb_attn_kv4_store(x, x, *cache, pos=pos)
    k, v = sb.sb_attn_kv4_load(*cache, 8, pos=pos)
    assert torch.equal(k, v) and not torch.equal(k, torch.zeros_like(k))
    small = [torch.zeros(3, 1, 32, w, dtype=torch.uint8, device="cuda") for w in (64, 4, 64, 4)]
    sb.sb_attn_kv4_store(x, x, *small)
    for a, b in zip(cache, small):
        assert torch.equal(a[:, :, Tcap - 8:], b[:, :, :8])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_spoils_its_block(sb, bad):
    x = rows(1, 1, 4, 128, 6).cuda()
    clean = [torch.zeros(1, 1, 32, w, dtype=torch.uint8, device="cuda") for w in (64, 4, 64, 4)]
    spoilt = [t.clone() for t in clean]
    y = x.clone()
    y[0, 0, 2, 70] = bad
    sb.sb_attn_kv4_store(x, x, *clean)
    sb.sb_attn_kv4_store(y, x, *spoilt)
    (a, c), (b, e) = sb.sb_attn_kv4_load(*clean, 4), sb.sb_attn_kv4_load(*spoilt, 4)
    assert b[0, 0, 2, 64:96].isnan().all()
    b[0, 0, 2, 64:96] = a[0, 0, 2, 64:96]
    assert torch.equal(a, b) and torch.equal(c, e)


# ---- decode


def activations(gen, B, H, Hkv, T, d, seed, kind="mixed"):
    """By kv head in turn: N(0,1), k * 3, and logits around -6; "sharp": k * 40, "far": logits around -6 everywhere."""
    q, _, _ = gen.gaussian(B, H, 1, d, seed=seed, dtype="f32")
    _, k, v = gen.gaussian(B, Hkv, T, d, seed=seed + 1, dtype="f32")
    far = (6.0 * d ** 0.5) ** 0.5
    for h in range(Hkv):
        if kind == "sharp":
            k[:, h] *= 40.0
        elif kind == "far" or h % 3 == 2:
            k[:, h, :, d - 1] = -far
            q[:, h * (H // Hkv):(h + 1) * (H // Hkv), :, d - 1] = far
        elif h % 3 == 1:
            k[:, h] *= 3.0
    return tuple(t.to(torch.bfloat16) for t in (q[:, :, 0].contiguous(), k, v))


def check(sb, oracle, q, k, v, cap=None, T=None, lens=None, r=None, scores=True, want_m=False, given=None):
    """Bounds: a weight's exponent is off by what its logit is (d products and sums in fp32), by what the T factors 1 + e round, and by
    sums of at most T / 32 + 64 terms, of which those that matter are small where the weight is large: a relative error of
    rel = (T + 64) 2^-23 + 8 dz.  o: that and the 16 bits of a weight, times the largest value, and its own rounding (half a step, 2^-8)."""
    B, H, d = q.shape
    Hkv, n = k.shape[1], k.shape[2]
    cap = cap or (n + 31) // 32 * 32
    cache = empty_cache(B, Hkv, cap, d)
    sb.sb_attn_kv4_store(k.cuda(), v.cuda(), *cache)
    if lens is None and T is None:
        T = n
    ld = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens is not None else None
    at = [min(max(x, 0), cap if T is None else T) for x in lens] if lens is not None else [T] * B
    for b in range(B):                                   # what lies behind an entry's rows is anything at all
        for t in cache:
            t[b, :, at[b]:] = 0xFF
    was = torch.rand(B, Hkv, cap, generator=torch.Generator().manual_seed(9)).cuda() if given is None else given
    score = was.clone() if scores else None
    out = torch.full_like(was, -7.0) if scores else None
    ws = nan_bytes(sb.sb_attn_decode_kv4_workspace_bytes(B, H, Hkv, cap if T is None else T, cap, d, scores))
    got = sb.sb_attn_decode_kv4(q.cuda(), *cache, T=T, lens=ld, r=r.cuda() if r is not None else None, score=score, score_out=out,
                                want_m=want_m, workspace=ws)
    torch.cuda.synchronize()
    got = got if isinstance(got, tuple) else (got,)
    o, m = to64(got[0]), to64(got[1]) if want_m else None
    kv, vv = values(oracle, *cache[:2]), values(oracle, *cache[2:])
    G = H // Hkv
    worst = [0.0, 0.0]
    for b in range(B):
        for g in range(Hkv):
            kb, vb = kv[b, g, :at[b]], vv[b, g, :at[b]]
            total = np.zeros(at[b])
            rel = 0.0
            for h in range(g * G, (g + 1) * G):
                qh = to64(q)[b, h]
                A, left = oracle.row_weights(qh, kb)
                ref = A @ vb
                dz = d * U * (np.abs(kb) @ np.abs(qh)).max(initial=0.0) / np.sqrt(d)
                rel = max(rel, (at[b] + 64) * 2 * U + 8 * dz)
                top = np.abs(vb).max(initial=0.0)
                if r is not None:
                    ref = ref + left * to64(r)[h]
                    top = max(top, np.abs(to64(r)[h]).max())
                tol = 2.0 ** -8 * np.abs(ref) + top * (2.0 ** -16 + rel)
                err = np.abs(o[b, h] - ref)
                worst[0] = max(worst[0], float((err / (tol + 1e-300)).max()))
                assert (err <= tol).all(), (b, h, float((err - tol).max()))
                if want_m and left > 1e-290:
                    assert abs(m[b, h] - np.log(left)) <= 2e-3 + 2e-3 * abs(np.log(left)), (b, h)
                total += A
            if scores:
                s = to64(got[-1])[b, g]
                ref = to64(was)[b, g, :at[b]] + total
                err = np.abs(s[:at[b]] - ref)
                tol = G * rel + 2 * U * (G + 1) * ref
                worst[1] = max(worst[1], float((err / tol).max(initial=0.0)))
                assert (err <= tol).all(), (b, g, float((err - tol).max()))
                assert (s[at[b]:] == -7.0).all()
    if scores:
        # in place, and from nothing
        in_place = was.clone()
        sb.sb_attn_decode_kv4(q.cuda(), *cache, T=T, lens=ld, score=in_place)
        fresh = torch.zeros_like(was)
        sb.sb_attn_decode_kv4(q.cuda(), *cache, T=T, lens=ld, score_out=fresh)
        for b in range(B):
            assert want_m or torch.equal(in_place[b, :, :at[b]], got[-1][b, :, :at[b]])
            assert torch.equal(in_place[b, :, at[b]:], was[b, :, at[b]:])
            assert torch.allclose(in_place[b, :, :at[b]], was[b, :, :at[b]] + fresh[b, :, :at[b]], rtol=1e-6, atol=1e-6)
    print(f"o: {worst[0]:.3f} of the bound, scores: {worst[1]:.3f}")
    return got


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 64, 65, 255, 256, 257, 300, 1000, 1100, 2047, 2049, 2500, 5000])
def test_lengths(sb, oracle, gen, T, d):
    check(sb, oracle, *activations(gen, 2, 3, 3, T, d, seed=T + d))


@pytest.mark.parametrize("H,Hkv", [(4, 2), (12, 3), (5, 1), (32, 2), (34, 2), (50, 1)])
@pytest.mark.parametrize("T", [700, 3000])
def test_grouped_heads(sb, oracle, gen, H, Hkv, T):
    check(sb, oracle, *activations(gen, 2, H, Hkv, T, 64, seed=H + Hkv), r=gen.remainder_embedding(H, 64, seed=3))


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("want_m", [False, True])
def test_entries_of_different_lengths(sb, oracle, gen, d, want_m):
    """Empty entries, single keys, ends inside a tile, at its edge and inside the nearest keys, and lengths out of range."""
    lens = [0, 1, 31, 32, 33, 100, 256, 289, 2900, 3000, 4000, -5]
    check(sb, oracle, *activations(gen, len(lens), 4, 2, 3000, d, seed=d), T=3000, lens=lens, want_m=want_m, r=gen.remainder_embedding(4, d, seed=4))
    check(sb, oracle, *activations(gen, 5, 2, 2, 300, d, seed=d), T=300, lens=[0, 1, 40, 299, 300], want_m=want_m)


@pytest.mark.parametrize("kind", ["far", "sharp"])
@pytest.mark.parametrize("T", [500, 3000])
@pytest.mark.parametrize("want_m", [False, True])
def test_far_and_sharp_heads(sb, oracle, gen, kind, T, want_m):
    check(sb, oracle, *activations(gen, 1, 4, 2, T, 64, seed=7, kind=kind), r=gen.remainder_embedding(4, 64, seed=6), want_m=want_m)


@pytest.mark.parametrize("d", [64, 128])
def test_bound_below_the_capacity(sb, oracle, gen, d):
    q, k, v = activations(gen, 2, 3, 3, 400, d, seed=8)
    check(sb, oracle, q, k, v, cap=4096, T=400)
    check(sb, oracle, q, k, v, cap=416, T=77, scores=False)
    check(sb, oracle, q, k, v, cap=4096, lens=[400, 12])         # the bound is the capacity


def test_without_scores_nothing_else_changes(sb, gen):
    q, k, v = (t.cuda() for t in activations(gen, 2, 4, 2, 3000, 128, seed=11))
    cache = empty_cache(2, 2, 3008, 128)
    sb.sb_attn_kv4_store(k, v, *cache)
    o = sb.sb_attn_decode_kv4(q, *cache, T=3000)
    s = torch.zeros(2, 2, 3008, device="cuda")
    o2, s2 = sb.sb_attn_decode_kv4(q, *cache, T=3000, score=s)
    o3, m3 = sb.sb_attn_decode_kv4(q, *cache, T=3000, want_m=True)
    o4, m4, s4 = sb.sb_attn_decode_kv4(q, *cache, T=3000, want_m=True, score=torch.zeros_like(s))
    assert s2.data_ptr() == s.data_ptr() and torch.equal(o, o2) and torch.equal(o3, o4) and torch.equal(m3, m4)
    again = sb.sb_attn_decode_kv4(q, *cache, T=3000, score=torch.zeros_like(s))
    assert torch.equal(again[0], o) and torch.equal(again[1], s2)


def test_agrees_with_decode_on_the_values(sb, gen):
    """The bf16 decode of the rows as they come back: another kernel, the same numbers but for the weights' 16 bits."""
    q, k, v = (t.cuda() for t in activations(gen, 2, 6, 3, 2500, 128, seed=12))
    cache = empty_cache(2, 3, 2528, 128)
    sb.sb_attn_kv4_store(k, v, *cache)
    k4, v4 = sb.sb_attn_kv4_load(*cache, 2500)
    a, ma = sb.sb_attn_decode_kv4(q, *cache, T=2500, want_m=True)
    b, mb = sb.sb_attn_decode(q, k4, v4, want_m=True)
    # each is within half a step of a number that both are near to
    assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 2.0 ** -14 * v4.float().abs().max()).all()
    assert torch.allclose(ma, mb, rtol=1e-4, atol=1e-3)


@pytest.mark.parametrize("T", [300, 3000])
def test_nan_in_the_cache(sb, gen, T):
    """A NaN reaches every result that weighs it and no other head's."""
    q, k, v = (t.cuda() for t in activations(gen, 1, 3, 3, T, 64, seed=13))
    cap = (T + 31) // 32 * 32
    def run(k, v):
        cache = empty_cache(1, 3, cap, 64)
        sb.sb_attn_kv4_store(k, v, *cache)
        return sb.sb_attn_decode_kv4(q, *cache, T=T, score_out=torch.zeros(1, 3, cap, device="cuda"))
    o, s = run(k, v)
    vx = v.clone()
    vx[:, 2, T - 40, 5] = float("nan")                   # the head whose weights reach far
    ox, sx = run(k, vx)
    assert torch.equal(s, sx) and torch.equal(o[:, :2], ox[:, :2])
    assert ox[0, 2, :32].isnan().all() and torch.equal(o[0, 2, 32:], ox[0, 2, 32:])
    kx = k.clone()
    kx[:, 2, T - 40] = float("nan")
    ox, sx = run(kx, v)
    assert torch.equal(o[:, :2], ox[:, :2]) and torch.equal(s[:, :2], sx[:, :2])
    assert ox[0, 2].isnan().all() and sx[0, 2, T - 40].isnan() and torch.allclose(sx[0, 2, T - 39:], s[0, 2, T - 39:], rtol=1e-4, atol=1e-6)


@pytest.mark.parametrize("cap", [4096, 512])
def test_captured_with_lengths_that_grow(sb, gen, cap):
    """A captured step (append, decode, scores) follows lengths that change between replays."""
    B, H, Hkv, d = 3, 4, 2, 64
    q, k, v = (t.cuda() for t in activations(gen, B, H, Hkv, cap, d, seed=14))
    cache = empty_cache(B, Hkv, cap, d)
    lens = torch.tensor([0, cap // 2, cap - 70], dtype=torch.int32, device="cuda")
    first = lens.clone()
    nk, nv = k[:, :, :1].contiguous(), v[:, :, :1].contiguous()
    score = torch.zeros(B, Hkv, cap, device="cuda")
    out = torch.zeros_like(score)
    o = torch.empty(B, H, d, dtype=torch.bfloat16, device="cuda")
    ws = nan_bytes(sb.sb_attn_decode_kv4_workspace_bytes(B, H, Hkv, cap, cap, d, True))
    def step():
        sb.sb_attn_decode_kv4(q, *cache, lens=lens, score=score, score_out=out, o=o, workspace=ws)
        sb.sb_attn_kv4_store(nk, nv, *cache, pos=lens)
    def reset():
        sb.sb_attn_kv4_store(k, v, *cache)
        lens.copy_(first)
        score.zero_()
        out.zero_()
    def generate(step, n):
        reset()
        got = []
        for i in range(n):
            nk.copy_(k[:, :, 7 * i:7 * i + 1])
            nv.copy_(v[:, :, 7 * i:7 * i + 1])
            step()
            score.copy_(out)
            lens.add_(1)
            got.append((o.clone(), out.clone()))
        torch.cuda.synchronize()
        return got
    want = generate(step, 40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(2):
        ws.random_(0, 255)
        for (a, s), (b, t) in zip(generate(graph.replay, 40), want):
            assert torch.equal(a, b) and torch.equal(s, t)


def test_two_streams_at_once(sb, gen):
    """Calls with workspaces of their own on two streams."""
    B, H, Hkv, T, d = 4, 8, 2, 6000, 128
    sets = []
    for seed in (15, 16):
        q, k, v = (t.cuda() for t in activations(gen, B, H, Hkv, T, d, seed=seed))
        cache = empty_cache(B, Hkv, 6016, d)
        sb.sb_attn_kv4_store(k, v, *cache)
        sets.append((q, cache))
    want = [sb.sb_attn_decode_kv4(q, *c, T=T, score_out=torch.zeros(B, Hkv, 6016, device="cuda")) for q, c in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for _ in range(5):
        for (q, c), st in zip(sets, streams):
            with torch.cuda.stream(st):
                got.append(sb.sb_attn_decode_kv4(q, *c, T=T, score_out=torch.zeros(B, Hkv, 6016, device="cuda")))
    got += [sb.sb_attn_decode_kv4(q, *c, T=T, score_out=torch.zeros(B, Hkv, 6016, device="cuda"), stream=st) for (q, c), st in zip(sets, streams)]
    torch.cuda.synchronize()
    for i, (o, s) in enumerate(got):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(s, want[i % 2][1])


def test_refusals(sb):
    cache = empty_cache(2, 2, 64, 64)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    s = torch.zeros(2, 2, 64, device="cuda")
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    x = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16, device="cuda")
    for call, why in ((lambda: sb.sb_attn_decode_kv4(q.float(), *cache), "must be torch.bfloat16"), (lambda: sb.sb_attn_decode_kv4(q[:1], *cache), "has shape"),
                      (lambda: sb.sb_attn_decode_kv4(q[:, :3].contiguous(), *cache), "bad shape"), (lambda: sb.sb_attn_decode_kv4(q, *cache, T=65), "bad shape"),
                      (lambda: sb.sb_attn_decode_kv4(q, *cache, T=0), "bad shape"), (lambda: sb.sb_attn_decode_kv4(q, *cache, lens=lens.long()), "must be torch.int32"),
                      (lambda: sb.sb_attn_decode_kv4(q, *cache, lens=lens[:1]), "has shape"), (lambda: sb.sb_attn_decode_kv4(q, *cache, score=s[:, :, :63]), "must be contiguous"),
                      (lambda: sb.sb_attn_decode_kv4(q, *cache, score=s[:1]), "has shape"), (lambda: sb.sb_attn_decode_kv4(q, cache[0], *cache[:3]), "has shape"),
                      (lambda: sb.sb_attn_decode_kv4(q, *[t.short() for t in cache]), "must be torch.uint8"), (lambda: sb.sb_attn_decode_kv4(q, *[t[:, :, :33].contiguous() for t in cache]), "bad shape"),
                      (lambda: sb.sb_attn_decode_kv4(q, *cache, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda")), "workspace"),
                      (lambda: sb.sb_attn_decode_kv4(q, *cache, lens=lens.cpu()), "must live on the GPU"),
                      (lambda: sb.sb_attn_kv4_store(x, x[:, :, :2], *cache), "has shape|contiguous"), (lambda: sb.sb_attn_kv4_store(x, x.half(), *cache), "must be torch.bfloat16"),
                      (lambda: sb.sb_attn_kv4_load(*cache, 65), "expected 1 .. Tcap"), (lambda: sb.sb_attn_kv4_load(*cache, 0), "expected 1 .. Tcap"),
                      (lambda: sb.sb_attn_kv4_load(*cache, 3, k=x[:1]), "has shape"), (lambda: sb.sb_attn_kv4_load(*cache, 3, pos=lens.float()), "must be torch.int32")):
        with pytest.raises(sb.SbAttnError, match=why):
            call()
