"""The cache's, attention's and the 8-bit layers' calls refuse what they cannot take, on the host, before anything is launched (no GPU needed)."""
import ctypes
import os
import struct

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2504_02692_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2504_02692_amd import build
        build.build(verbose=False)
    return binding.load()


ONE, NULL = ctypes.c_void_p(256), ctypes.c_void_p(0)      # a non-null, aligned, never dereferenced address
ODD = ctypes.c_void_p(257)
NAN, INF = float("nan"), float("inf")
BIG = 1 << 40


def test_linear8_sizes(lib):
    up = lambda b: -(-b // 256) * 256
    size = lib.gptaq_linear8_weights_bytes
    assert size(64, 256) == up(4 * 2 * 2048 + 4 * 128 + 256 * 4)
    assert size(17, 130) == up(2 * 2 * 2048 + 2 * 128 + 130 * 4)
    ws = lib.gptaq_linear8_workspace_bytes
    for m, n, fits in ((1, 1, True), (1 << 20, 16384, True), (1 << 20, 16385, False), ((1 << 20) + 1, 64, False), (16, 65536, True), (16, 65537, False),
                       (0, 64, False), (64, 0, False), (-1, 64, False)):
        assert (size(m, n) > 0) == fits and (ws(1, m, n) > 0) == fits, (m, n)
        assert lib.gptaq_linear8_pack(ONE, max(n, 1), ONE, ONE, m, n, NULL, ctypes.c_void_p(264), BIG, ONE, NULL) == (-4 if fits else -2), (m, n)
    assert ws(0, 64, 64) == 0 and ws(-1, 64, 64) == 0 and ws((1 << 23) + 1, 64, 64) == 0
    for m, n in ((4096, 4096), (64, 300), (1000, 11008), (28672, 8192)):
        sizes = [ws(t, m, n) for t in [*range(1, 1500), 2048, 4096, 8192, 100000]]
        assert sizes == sorted(sizes)                     # the size for more tokens serves fewer


def test_linear8_refusals(lib):
    def pack(want, c=ONE, ldc=128, s=ONE, z=ONE, m=16, n=128, perm=NULL, w=ONE, wb=BIG, info=ONE):
        assert lib.gptaq_linear8_pack(c, ldc, s, z, m, n, perm, w, wb, info, NULL) == want

    for name in ("c", "s", "z", "w", "info"):
        pack(-1, **{name: NULL})
    pack(-2, ldc=127)
    for name in ("s", "z", "perm", "info"):
        pack(-2, **{name: ODD})
    pack(-4, w=ctypes.c_void_p(264))
    pack(-4, wb=lib.gptaq_linear8_weights_bytes(16, 128) - 1)

    def run(want, x=ONE, xs=ONE, tokens=4, ldx=128, w=ONE, wb=BIG, m=16, n=128, bias=NULL, y=ONE, ldy=16, f32=0, ws=ONE, nb=BIG):
        assert lib.gptaq_linear8_i8(x, xs, tokens, ldx, w, wb, m, n, bias, y, ldy, f32, ws, nb, NULL) == want

    for name in ("x", "xs", "w", "y", "ws"):
        run(-1, **{name: NULL})
    run(-2, tokens=-1)
    run(-2, tokens=(1 << 23) + 1)
    run(-2, ldx=127)
    run(-2, ldy=15)
    run(-2, m=0)
    run(-2, n=65537, ldx=65537)
    run(-2, w=ctypes.c_void_p(264))
    run(-2, y=ODD)
    run(-2, y=ctypes.c_void_p(258), f32=1)
    run(-2, xs=ODD)
    run(-2, bias=ODD)
    run(-4, ws=ctypes.c_void_p(264))
    run(-4, nb=256)
    run(-4, wb=lib.gptaq_linear8_weights_bytes(16, 128) - 1)
    run(-4, tokens=0, wb=0)
    run(0, tokens=0)
    run(0, tokens=0, x=NULL, xs=NULL, y=NULL, ws=NULL)


def test_quant_activations_refusals(lib):
    def run(want, x=ONE, tokens=4, n=64, ldx=64, clip=1.0, c=ctypes.c_void_p(4096), ldc=64, s=ONE):
        assert lib.gptaq_quant_activations_i8(x, tokens, n, ldx, clip, c, ldc, s, NULL) == want

    for name in ("x", "c", "s"):
        run(-1, **{name: NULL})
    run(-2, tokens=-1)
    run(-2, n=0)
    run(-2, n=(1 << 24) + 8, ldx=1 << 25, ldc=1 << 25)
    run(-2, ldx=63)
    run(-2, ldc=63)
    run(-2, x=ODD)
    run(-2, s=ODD)
    for clip in (0.0, -1.0, 1.5, NAN):
        run(-3, clip=clip)
    run(-3, c=ONE)                                        # codes where the input begins
    run(0, tokens=0)


def packed(pages=10, page=16, table=ONE, ld_table=5, table_pages=5, starts=ONE, lengths=ONE, seqs=2, kv_heads=2, d=64, keys=ONE, values=ONE):
    """A gptaq_cache."""
    return struct.pack("12q", *(v if isinstance(v, int) else v.value or 0 for v in (keys, values, pages, kv_heads, page, d, table, ld_table, table_pages, starts, lengths, seqs)))


def cache(want_append, want_attention, lib, tokens=3, heads=4, **more):
    d, kv_heads = more.get("d", 64), more.get("kv_heads", 2)
    far = ctypes.c_void_p(1 << 20)
    if want_append is not None:
        assert lib.gptaq_cache_append(ONE, heads * d, d, ONE, kv_heads * d, d, ONE, kv_heads * d, d, packed(**more), tokens, heads, ONE, 32, 0, far, heads * d, d,
                                      NULL) == want_append
    if want_attention is not None:
        assert lib.gptaq_attention(ONE, heads * d, d, packed(**more), tokens, heads, 0, 0, 0.125, far, heads * d, d, ONE, BIG, NULL) == want_attention


def test_cache_refusals(lib):
    for name in ("table", "starts", "lengths", "keys", "values"):
        cache(-1, -1, lib, **{name: NULL})
    for name in ("table", "starts", "lengths", "keys", "values"):
        cache(-2, -2, lib, **{name: ODD})
    cache(-2, -2, lib, keys=ctypes.c_void_p(264))         # 8-byte aligned
    for page in (0, 8, 24, 48, 512, -16):
        cache(-3, -3, lib, page=page)
    cache(-2, -2, lib, ld_table=4)
    cache(-2, -2, lib, table_pages=-1)
    cache(-2, -2, lib, table_pages=(1 << 26) + 1, ld_table=1 << 30)
    cache(-2, -2, lib, pages=-1)
    cache(-2, -2, lib, seqs=-1)
    cache(-2, -2, lib, seqs=(1 << 20) + 1)
    cache(-2, -2, lib, tokens=-1)
    cache(-2, -2, lib, tokens=(1 << 24) + 1)
    cache(-2, -2, lib, tokens=1 << 24, heads=128)         # 2^31 rows
    cache(-2, -2, lib, heads=5)
    cache(-2, -2, lib, heads=0)
    cache(-2, -2, lib, kv_heads=0)
    cache(-2, -2, lib, heads=8192, kv_heads=8192)
    cache(-3, -3, lib, d=72)
    cache(None, -3, lib, d=32)                            # (the cache takes it, attention has no kernel for it)
    cache(None, -3, lib, d=256)
    cache(-3, None, lib, d=272)
    assert lib.gptaq_attention(ONE, 256, 64, None, 3, 4, 0, 0, 0.125, ONE, 256, 64, ONE, BIG, NULL) == -1
    assert lib.gptaq_cache_append(ONE, 256, 64, ONE, 128, 64, ONE, 128, 64, None, 3, 4, ONE, 32, 0, ONE, 256, 64, NULL) == -1
    cache(0, 0, lib, tokens=0)
    cache(0, 0, lib, seqs=0)
    cache(0, 0, lib, tokens=0, table=NULL, starts=NULL, lengths=NULL, keys=NULL, values=NULL)


def test_append_refusals(lib):
    def run(want, q=ONE, k=ONE, v=ONE, ldq=256, hq=64, ldk=128, hk=64, ldv=128, hv=64, d=64, freqs=ONE, pairs=32, out=ctypes.c_void_p(1 << 20), ldo=256, ho=64, tokens=3):
        assert lib.gptaq_cache_append(q, ldq, hq, k, ldk, hk, v, ldv, hv, packed(d=d), tokens, 4, freqs, pairs, 0, out, ldo, ho, NULL) == want

    for name in ("q", "k", "v", "out", "freqs"):
        run(-1, **{name: NULL})
    for name in ("q", "k", "v", "out", "freqs"):
        run(-2, **{name: ODD})
    for pairs in (-8, 4, 12, 40):
        run(-3, pairs=pairs)
    for name in ("ldq", "hq", "ldk", "hk", "ldv", "hv", "ldo", "ho"):
        run(-2, **{name: -64})
    run(-2, ldo=255)                                      # rows of the output into each other
    run(-2, ho=63)
    run(-2, ldo=64, ho=128)
    run(-3, out=ONE, ldo=512)                             # the queries' own memory, in other places
    run(0, tokens=0, pairs=0, freqs=NULL)


def test_attention_refusals(lib):
    def run(want, q=ONE, ldq=256, hq=64, tokens=3, seqs=2, d=64, window=0, sinks=0, scale=0.125, out=ctypes.c_void_p(1 << 20), ldo=256, ho=64, ws=ONE, nb=BIG):
        assert lib.gptaq_attention(q, ldq, hq, packed(seqs=seqs, d=d), tokens, 4, window, sinks, scale, out, ldo, ho, ws, nb, NULL) == want

    for name in ("q", "out", "ws"):
        run(-1, **{name: NULL})
    for name in ("q", "out"):
        run(-2, **{name: ODD})
    for name in ("ldq", "hq", "ldo", "ho", "window", "sinks"):
        run(-2, **{name: -1})
    run(-2, ldo=255)
    for scale in (NAN, INF, -INF):
        run(-3, scale=scale)
    run(-4, ws=ctypes.c_void_p(264))
    run(-4, nb=lib.gptaq_attention_workspace_bytes(3, 2, 4, 2, 64) - 1)
    run(0, tokens=0)


def test_attention_refuses_scales_that_leave_fp32_as_exponents_of_two(lib):
    for scale, want in ((3e38, -3), (-2.4e38, -3), (2.3e38, 0), (0.0, 0)):
        rc = lib.gptaq_attention(ONE, 256, 64, packed(seqs=0), 3, 4, 0, 0, scale, ONE, 256, 64, ONE, BIG, NULL)
        assert rc == want, scale


def test_attention_workspace(lib):
    size = lib.gptaq_attention_workspace_bytes
    for bad in ((0, 1, 4, 2, 64), (1, 0, 4, 2, 64), (1, 1, 4, 3, 64), (1, 1, 4, 2, 72), (-1, 1, 4, 2, 64), (1, 1, 0, 1, 64), ((1 << 24) + 1, 1, 1, 1, 64)):
        assert size(*bad) == 0, bad
    for heads, kv_heads in ((32, 32), (64, 8), (1, 1), (24, 8)):
        for d in (64, 96, 128):
            for seqs in (1, 3, 64, 1000):
                sizes = [size(t, seqs, heads, kv_heads, d) for t in [*range(1, 600), 1000, 5000, 100000, 1 << 20]]
                assert sizes == sorted(sizes) and sizes[0] > 0
            assert len({size(100, seqs, heads, kv_heads, d) for seqs in (1, 2, 7, 100)}) == 1


def eight(m=48, n=128, **other):
    import torch
    from paper_2504_02692_amd import binding as B
    have = dict(data=torch.zeros(B.gptaq_linear8_weights_bytes(m, n), dtype=torch.uint8), bias=torch.zeros(m), info=torch.zeros(1, dtype=torch.int32))
    have.update(other)
    return B.Linear8Weights(m=m, n=n, **have)


@pytest.mark.parametrize("name,memory", [("bias", lambda t: t[:3]), ("bias", lambda t: t.double()), ("bias", lambda t: t[:1].expand(48)),
                                         ("data", lambda t: t.view(2, -1).t()), ("data", lambda t: t.short())])
def test_weights_whose_memory_became_another_are_refused(lib, name, memory):
    from paper_2504_02692_amd import binding as B
    w = eight()
    assert w._args(-1) == (w.data.data_ptr(), w.data.numel(), 48, 128, w.bias.data_ptr())
    t = getattr(w, name)
    t.data = memory(t.detach().clone())
    with pytest.raises(B.GptaqError, match=f"Linear8Weights.{name}"):
        w._args(-1)


def test_weights_are_fixed_copied_and_saved(lib, tmp_path):
    import copy
    import pickle
    import torch
    from paper_2504_02692_amd import binding as B
    w = eight(bias=torch.randn(48))
    torch.save({"layer": w}, tmp_path / "layer.pt")
    again = [copy.copy(w), copy.deepcopy(w), pickle.loads(pickle.dumps(w))]
    with torch.serialization.safe_globals([B.Linear8Weights]):
        again.append(torch.load(tmp_path / "layer.pt", weights_only=True)["layer"])
    for v in again:
        assert type(v) is B.Linear8Weights and (v.m, v.n) == (w.m, w.n)
        assert all(torch.equal(getattr(v, name), getattr(w, name)) for name in ("data", "bias", "info"))
        with pytest.raises(AttributeError, match="gptaq_linear8_pack"):
            v.bias = None
    assert copy.deepcopy(eight(bias=None)).bias is None


def test_the_binding_looks_at_shapes(lib, monkeypatch):
    """What the library cannot see: a tensor's type, its shape, and where it is."""
    import torch
    from paper_2504_02692_amd import binding as B
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)                 # host memory's own number
    monkeypatch.setattr(B, "_raw_stream", lambda device: 0)
    bf = torch.bfloat16
    good = dict(q=torch.zeros(3, 4, 64, dtype=bf), k=torch.zeros(3, 2, 64, dtype=bf), v=torch.zeros(3, 2, 64, dtype=bf), keys=torch.zeros(5, 2, 8, 16, 8, dtype=bf),
                values=torch.zeros(5, 2, 2, 64, 8, dtype=bf), table=torch.zeros(2, 3, dtype=torch.int32), starts=torch.zeros(3, dtype=torch.int32),
                lengths=torch.zeros(2, dtype=torch.int32), freqs=torch.zeros(32, dtype=torch.float64))
    ws = torch.zeros(256, dtype=torch.uint8)
    wrong = [("q", lambda t: t.float()), ("q", lambda t: t[0]), ("q", lambda t: t.transpose(1, 2)), ("keys", lambda t: t.float()), ("keys", lambda t: t[..., :4]),
             ("keys", lambda t: t.transpose(0, 1)), ("keys", lambda t: t[:, :, :4]), ("values", lambda t: t[:4]), ("values", lambda t: t[:, :1]), ("values", lambda t: t.half()),
             ("table", lambda t: t.long()), ("table", lambda t: t[:1]), ("table", lambda t: t[0]), ("table", lambda t: t.t().contiguous().t()), ("starts", lambda t: t[:2]),
             ("starts", lambda t: t.long()), ("lengths", lambda t: t.float()), ("lengths", lambda t: t[:1])]
    for name, f in wrong + [("k", lambda t: t[:2]), ("k", lambda t: t[:, :1]), ("v", lambda t: t[..., :32]), ("freqs", lambda t: t.float()), ("freqs", lambda t: t[::2])]:
        have = dict(good, **{name: f(good[name])})
        with pytest.raises(B.GptaqError):
            B.gptaq_cache_append(**have)
    for name, f in wrong:
        have = {k: v for k, v in dict(good, **{name: f(good[name])}).items() if k not in ("k", "v", "freqs")}
        with pytest.raises(B.GptaqError):
            B.gptaq_attention(**have, ws=ws)
    rest = {k: v for k, v in good.items() if k not in ("k", "v", "freqs")}
    with pytest.raises(B.GptaqError, match="out"):
        B.gptaq_attention(**rest, ws=ws, out=torch.zeros(3, 4, 32, dtype=bf))
    with pytest.raises(B.GptaqError, match="workspace"):
        B.gptaq_attention(**rest, ws=ws)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(B.GptaqError, match="cpu"):
        B.gptaq_attention(**rest, ws=ws)
    with pytest.raises(B.GptaqError, match="cpu"):
        B.gptaq_cache_append(**good)


class Calls:
    """In the library's place: what was called, and with how many arguments; every call succeeds."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        return lambda *args: self.made.append((name, len(args))) or 0


def test_products_tell_the_two_kinds_of_weights_apart(lib, monkeypatch):
    """On host memory, with nothing behind the calls: weights of the other kind are refused before the library is reached, those of the own kind reach it."""
    import torch
    from paper_2504_02692_amd import binding as B
    eight_bits = eight()
    four = B.LinearWeights(torch.zeros(B.gptaq_linear_weights_bytes(48, 128, 0), dtype=torch.uint8), 48, 128, 0, None, torch.zeros(48), torch.zeros(1, dtype=torch.int32))
    calls = Calls()
    monkeypatch.setattr(B, "load", lambda: calls)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)                 # host memory's own number
    monkeypatch.setattr(B, "_raw_stream", lambda device: 0)
    for check in ("_need", "_need_vec"):
        monkeypatch.setattr(B, check, lambda *args: None)
    codes, scales, x, ws = torch.zeros(4, 128, dtype=torch.int8), torch.ones(4), torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(256, dtype=torch.uint8)
    for name, args, own, other in (("gptaq_linear8_i8", (codes, scales), eight_bits, four), ("gptaq_linear_i8", (codes, scales), four, eight_bits), ("gptaq_linear", (x,), four, eight_bits)):
        with pytest.raises(B.GptaqError, match=f"{name}: weights: .*{type(own).__name__}"):
            getattr(B, name)(*args, other, ws)
        with pytest.raises(B.GptaqError, match=f"{name}: weights: "):
            getattr(B, name)(*args, other.data, ws)
        assert calls.made == []
        getattr(B, name)(*args, own, ws)
        assert calls.made == [(name, len(B._SIGS[name][1]))]
        calls.made.clear()


def test_an_mlp_with_a_layer_of_more_than_4_bits_refuses_bf16_activations(lib, monkeypatch):
    """Before anything runs, whichever of its layers it is."""
    import torch
    from paper_2504_02692_amd import binding as B
    from paper_2504_02692_amd import quantized_mlp as M
    calls = Calls()
    four = lambda m, n: B.LinearWeights(torch.zeros(B.gptaq_linear_weights_bytes(m, n, 0), dtype=torch.uint8), m, n, 0, None, None, torch.zeros(1, dtype=torch.int32))
    mlps = [M.QuantizedMLP(torch.ones(128), *layers) for layers in ((eight(96, 128), eight(128, 48)), (four(96, 128), eight(128, 48)), (eight(96, 128), four(128, 48)))]
    monkeypatch.setattr(B, "load", lambda: calls)
    for mlp in mlps:
        with pytest.raises(B.GptaqError, match="8-bit activations"):
            mlp(torch.zeros(4, 128), torch.zeros(4, 128), torch.zeros(256, dtype=torch.uint8), eight_bits=False)
    assert calls.made == []


def test_a_cache_that_is_full_stays_as_it_was(monkeypatch):
    """The example's cache, in host memory: a call that does not fit changes nothing, so other sequences and fewer tokens still do."""
    import torch
    from paper_2504_02692_amd import quantized_attention as A
    for name in ("zeros", "full"):
        monkeypatch.setattr(torch, name, lambda *a, make=getattr(torch, name), device=None, **more: make(*a, **more))
    cache = A.PagedCache(3, 6, 1, 64, 16, 64)                        # six pages, four a sequence at most

    def state():
        return [*cache.counts], [[*t] for t in cache.tables], [*cache.free], cache.table.tolist(), cache.starts.tolist(), cache.lengths.tolist()

    def consistent(counts):
        pages = [p for t in cache.tables for p in t] + cache.free
        assert sorted(pages) == list(range(6))
        for s, t in enumerate(cache.tables):
            assert len(t) == -(-cache.counts[s] // 16) and cache.table[s].tolist() == t + [-1] * (4 - len(t))
        assert cache.lengths.tolist() == cache.counts and cache.starts.tolist() == [0, counts[0], counts[0] + counts[1], sum(counts)]

    cache.grow([33, 5, 0])
    consistent([33, 5, 0])
    for counts in ([1, 1, 49], [32, 0, 0], [0, 60, 0], [20, 20, 20]):  # too many pages in all, or of one sequence
        before = state()
        with pytest.raises(RuntimeError, match="full"):
            cache.grow(counts)
        assert state() == before
    for counts in ([0, 0, 0], [15, 1, 0], [1, 26, 0], [15, 0, 0]):
        cache.grow(counts)
        consistent(counts)
    assert cache.counts == [64, 32, 0] and not cache.free
    for counts in ([0, 0], [0, 0, 0, 0], [0, -1, 0]):                # not a count for each sequence
        before = state()
        with pytest.raises(ValueError):
            cache.grow(counts)
        assert state() == before


def test_attention_over_the_queries_memory_in_other_places_is_refused(lib):
    own = -4                                              # (taken, as far as the workspace)
    for tokens, heads, ldo, ho, want in ((3, 4, 512, 64, -3), (3, 4, 256, 80, -2), (3, 4, 768, 192, -3), (3, 4, 256, 64, own), (1, 4, 512, 64, own), (1, 4, 512, 72, -3),
                                         (3, 2, 256, 64, own), (3, 2, 260, 64, -3)):
        assert lib.gptaq_attention(ONE, 256, 64, packed(), tokens, heads, 0, 0, 0.125, ONE, ldo, ho, ONE, 0, NULL) == want, (tokens, heads, ldo, ho)
    assert lib.gptaq_attention(ONE, 256, 64, packed(), 0, 4, 0, 0, 0.125, ONE, 512, 64, ONE, BIG, NULL) == 0
