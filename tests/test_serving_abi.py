"""The calls that run quantised layers refuse what they cannot take, on the host, before anything is launched (no GPU needed)."""
import ctypes
import os

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


def test_sizes(lib):
    tile = lambda m, n: -(-m // 16) * -(-n // 128)
    up = lambda b: -(-b // 256) * 256
    assert lib.gptaq_linear_weights_bytes(64, 256, 128) == up(tile(64, 256) * 1024 + 4 * 2 * 16 * 5)
    assert lib.gptaq_linear_weights_bytes(17, 96, 32) == up(tile(17, 96) * 1024 + 2 * 4 * 16 * 5)      # groups padded to whole tiles
    assert lib.gptaq_linear_weights_bytes(1, 1, 0) == up(1024 + 16 * 5)
    assert lib.gptaq_linear_weights_bytes(16, 1000, -1) == up(8 * 1024 + 16 * 5)
    for m, n, group in [(0, 128, 0), (16, 0, 0), (16, 130, 128), (16, 96, 48), (16, 64, 16), (1 << 21, 128, 0), (16, 1 << 21, 0)]:
        assert lib.gptaq_linear_weights_bytes(m, n, group) == 0
    size = lib.gptaq_linear_workspace_bytes
    assert size(0, 64, 64) == 0 and size(-1, 64, 64) == 0 and size(1, 0, 64) == 0 and size((1 << 23) + 1, 64, 64) == 0
    sizes = [size(t, 4096, 4096) for t in range(1, 3000)]
    assert sizes == sorted(sizes) and sizes[0] >= 4096 * 2      # the size for more tokens serves fewer


def test_pack_refusals(lib):
    f, big = lib.gptaq_linear_pack, 1 << 30
    assert f(NULL, 128, ONE, ONE, 16, 128, 128, ONE, big, ONE, NULL) == -1
    assert f(ONE, 128, NULL, ONE, 16, 128, 128, ONE, big, ONE, NULL) == -1
    assert f(ONE, 128, ONE, ONE, 16, 128, 128, ONE, big, NULL, NULL) == -1        # info required
    assert f(ONE, 127, ONE, ONE, 16, 128, 128, ONE, big, ONE, NULL) == -2         # ldc < n
    assert f(ONE, 128, ONE, ONE, 0, 128, 128, ONE, big, ONE, NULL) == -2
    assert f(ONE, 128, ONE, ODD, 16, 128, 128, ONE, big, ONE, NULL) == -2
    assert f(ONE, 128, ONE, ONE, 16, 128, 48, ONE, big, ONE, NULL) == -3
    assert f(ONE, 130, ONE, ONE, 16, 130, 128, ONE, big, ONE, NULL) == -3         # n % group
    assert f(ONE, 128, ONE, ONE, 16, 128, 128, ONE, 1024, ONE, NULL) == -4
    assert f(ONE, 128, ONE, ONE, 16, 128, 128, ctypes.c_void_p(264), big, ONE, NULL) == -4


def test_linear_refusals(lib):
    big = 1 << 30

    def both(want, x=ONE, xs=ONE, tokens=4, ldx=128, perm=NULL, w=ONE, wb=big, m=16, n=128, group=128, bias=NULL, y=ONE, ldy=16, f32=0, ws=ONE,
             nb=big):
        assert lib.gptaq_linear(x, tokens, ldx, perm, w, wb, m, n, group, bias, y, ldy, f32, ws, nb, NULL) == want
        assert lib.gptaq_linear_i8(x, xs, tokens, ldx, perm, w, wb, m, n, group, bias, y, ldy, f32, ws, nb, NULL) == want

    both(-1, x=NULL)
    both(-1, w=NULL)
    both(-1, y=NULL)
    both(-1, ws=NULL)
    assert lib.gptaq_linear_i8(ONE, NULL, 4, 128, NULL, ONE, big, 16, 128, 128, NULL, ONE, 16, 0, ONE, big, NULL) == -1
    both(-2, tokens=-1)
    both(-2, tokens=(1 << 23) + 1)
    both(-2, ldx=127)
    both(-2, ldy=15)
    both(-2, m=0)
    both(-2, n=1 << 21, ldx=1 << 21, group=0)
    both(-2, w=ctypes.c_void_p(264))
    both(-2, y=ODD)
    both(-2, y=ctypes.c_void_p(258), f32=1)
    both(-2, bias=ODD)
    both(-2, perm=ODD)
    both(-3, group=16)
    both(-3, n=120, group=32)
    both(-4, nb=512)
    both(-4, wb=lib.gptaq_linear_weights_bytes(16, 128, 128) - 1)                # weights of another size
    both(-4, wb=lib.gptaq_linear_weights_bytes(16, 128, 128), group=32)
    both(-4, tokens=0, wb=0)
    both(-4, ws=ctypes.c_void_p(264))
    both(0, tokens=0)                                                             # nothing to do
    assert lib.gptaq_linear(ODD, 4, 128, NULL, ONE, big, 16, 128, 128, NULL, ONE, 16, 0, ONE, big, NULL) == -2


def test_row_refusals(lib):
    def norm(want, x=ONE, r=NULL, w=NULL, tokens=4, n=64, ldx=64, ldr=64, eps=1e-5, s=NULL, lds=64, y=ONE, ldy=64):
        assert lib.gptaq_rms_norm(x, r, w, tokens, n, ldx, ldr, eps, s, lds, y, ldy, NULL) == want
        assert lib.gptaq_rms_norm_i8(x, r, w, tokens, n, ldx, ldr, eps, s, lds, 1.0, y, ldy, ONE, NULL) == want

    norm(-1, x=NULL)
    norm(-1, y=NULL)
    norm(-2, tokens=-1)
    norm(-2, n=0)
    norm(-2, ldx=63)
    norm(-2, ldy=63)
    norm(-2, r=ONE, ldr=63)
    norm(-2, s=ONE, lds=63)
    norm(-2, x=ODD)
    norm(-2, w=ODD)
    for eps in (-1.0, NAN, INF):
        norm(-3, eps=eps)
    norm(0, tokens=0)
    assert lib.gptaq_rms_norm(ONE, NULL, NULL, 4, 64, 64, 64, 1e-5, NULL, 64, ODD, 64, NULL) == -2
    assert lib.gptaq_rms_norm_i8(ONE, NULL, NULL, 4, 64, 64, 64, 1e-5, NULL, 64, 1.0, ONE, 64, NULL, NULL) == -1
    for clip in (0.0, -1.0, 1.5, NAN):
        assert lib.gptaq_rms_norm_i8(ONE, NULL, NULL, 4, 64, 64, 64, 1e-5, NULL, 64, clip, ONE, 64, ONE, NULL) == -3
        assert lib.gptaq_silu_mul_i8(ONE, ONE, 4, 64, 64, 64, clip, ONE, 64, ONE, NULL) == -3

    def gated(want, g=ONE, u=ONE, tokens=4, n=64, ldg=64, ldu=64, y=ONE, ldy=64):
        assert lib.gptaq_silu_mul(g, u, tokens, n, ldg, ldu, y, ldy, NULL) == want
        assert lib.gptaq_silu_mul_i8(g, u, tokens, n, ldg, ldu, 1.0, y, ldy, ONE, NULL) == want

    gated(-1, g=NULL)
    gated(-1, u=NULL)
    gated(-1, y=NULL)
    gated(-2, ldg=63)
    gated(-2, ldu=63)
    gated(-2, ldy=63)
    gated(-2, u=ODD)
    gated(-2, n=(1 << 24) + 8, ldg=1 << 25, ldu=1 << 25, ldy=1 << 25)
    gated(0, tokens=0)


def weights(m=48, n=128, **other):
    """LinearWeights as a program could have them, in host memory (device -1): what follows looks at them, and launches nothing."""
    import torch
    from paper_2504_02692_amd import binding as B
    have = dict(data=torch.zeros(B.gptaq_linear_weights_bytes(m, n, 0), dtype=torch.uint8), perm=torch.arange(n, dtype=torch.int32),
                bias=torch.zeros(m), info=torch.zeros(1, dtype=torch.int32))
    have.update(other)
    return B.LinearWeights(m=m, n=n, group=0, **have)


@pytest.mark.parametrize("name,memory", [("bias", lambda t: t[:3]), ("bias", lambda t: t.double()), ("bias", lambda t: t[:1].expand(48)),
                                         ("perm", lambda t: t[:100]), ("perm", lambda t: t.long()), ("perm", lambda t: t.repeat(2)[::2]),
                                         ("data", lambda t: t.view(2, -1).t()), ("data", lambda t: t.short())])
def test_weights_whose_memory_became_another_are_refused(lib, name, memory):
    """A layer's tensors are read where they are at the call, as many elements as the layer has: memory that holds fewer would be read past its end."""
    from paper_2504_02692_amd import binding as B
    w = weights()
    before = w._args(-1)
    assert before[0] == w.perm.data_ptr() and before[1:3] == (w.data.data_ptr(), w.data.numel()) and before[6] == w.bias.data_ptr()
    t = getattr(w, name)
    t.data = memory(t.detach().clone())
    with pytest.raises(B.GptaqError, match=name):
        w._args(-1)
    with pytest.raises(B.GptaqError, match=name):
        weights(**{name: memory(getattr(weights(), name))})._args(-1)


def test_weights_whose_memory_moved_are_read_there(lib):
    import torch
    w = weights()
    w.bias.data, w.perm.data = torch.ones(48), torch.zeros(128, dtype=torch.int32)
    args = w._args(-1)
    assert args[0] == w.perm.data_ptr() and args[6] == w.bias.data_ptr()


def test_memory_of_another_device_is_refused(lib, monkeypatch):
    """Addresses in host memory, or in that of a GPU other than the one the kernels run on, do not reach the library."""
    import torch
    from paper_2504_02692_amd import binding as B
    ws = torch.empty(1024, dtype=torch.uint8)
    for device in (0, 1):
        monkeypatch.setattr(torch.cuda, "current_device", lambda: device)
        for kept in ("perm", "bias", "data"):
            with pytest.raises(B.GptaqError, match="LinearWeights.perm" if kept == "perm" else "LinearWeights.data"):
                weights(**{k: None for k in ("perm", "bias") if k != kept})._args(device)
        with pytest.raises(B.GptaqError, match="ws"):
            B._ws(ws, device)
        with pytest.raises(B.GptaqError, match="cpu"):
            B._here(None, torch.empty(4))
    with pytest.raises(B.GptaqError, match="ws"):
        B._ws(ws)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)                 # host memory's own number
    assert B._ws(ws, -1) == ws.data_ptr() and B._here(ws, None) == -1
    with pytest.raises(B.GptaqError, match="ws"):
        B._ws(ws[:1].expand(1 << 20), -1)                                         # more bytes by its shape than it has


def test_workspaces_of_every_call_are_looked_at(lib, monkeypatch):
    """No call hands a workspace's address to the library unseen."""
    import inspect
    from paper_2504_02692_amd import binding as B
    for name, f in inspect.getmembers(B, inspect.isfunction):
        source = inspect.getsource(f)
        assert name == "_ws" or "ws.data_ptr()" not in source and "_ptr(ws)" not in source, name


def test_weights_are_copied_pickled_and_saved(lib, tmp_path):
    """A program that has laid a model out can store it and copy it; what comes back is as fixed as the weights it came from."""
    import copy
    import pickle
    import torch
    from paper_2504_02692_amd import binding as B
    w = weights(bias=torch.randn(48))
    torch.save({"layer": w}, tmp_path / "layer.pt")
    again = [copy.copy(w), copy.deepcopy(w), pickle.loads(pickle.dumps(w)), torch.load(tmp_path / "layer.pt", weights_only=False)["layer"]]
    with torch.serialization.safe_globals([B.LinearWeights]):
        again.append(torch.load(tmp_path / "layer.pt", weights_only=True)["layer"])
    for k, v in enumerate(again):
        assert type(v) is B.LinearWeights and (v.m, v.n, v.group) == (w.m, w.n, w.group)
        for name in ("data", "perm", "bias", "info"):
            assert torch.equal(getattr(v, name), getattr(w, name)) and (getattr(v, name) is getattr(w, name)) == (k == 0)
        with pytest.raises(AttributeError):
            v.bias = None
    assert copy.deepcopy(weights(perm=None, bias=None)).perm is None


def test_codes_in_the_inputs_memory_are_refused(lib):
    """One byte an element against two: rows of codes would lie where other rows' inputs are still read.  bf16 outputs may lie there."""
    other = [ctypes.c_void_p(4096 * k) for k in (1, 2, 3, 4)]
    for k in (0, 1, 3):                                                             # codes as x, residual, sum
        x, r, codes, s = other
        codes = (x, r, None, s)[k]
        assert lib.gptaq_rms_norm_i8(x, r, NULL, 4, 64, 64, 64, 1e-5, s, 64, 1.0, codes, 64, ONE, NULL) == -3
        assert lib.gptaq_rms_norm_i8(x, r, NULL, 0, 64, 64, 64, 1e-5, s, 64, 1.0, codes, 64, ONE, NULL) == 0
    for codes in other[:2]:
        assert lib.gptaq_silu_mul_i8(other[0], other[1], 4, 64, 64, 64, 1.0, codes, 64, ONE, NULL) == -3
        assert lib.gptaq_silu_mul_i8(other[0], other[1], 0, 64, 64, 64, 1.0, codes, 64, ONE, NULL) == 0


def test_sizes_are_those_that_pack_takes(lib):
    """A layer has a size of weights, and of a workspace, where gptaq_linear_pack and gptaq_linear take it, and only there."""
    k, off = 1 << 10, ctypes.c_void_p(264)                                          # (misaligned weights: what is refused last)
    for m, n, fits in ((128 * k, 128 * k, True), (128 * k + 1, 128 * k, False), (128 * k, 128 * k + 1, False), (k * k, k * k, False), (k * k, 16 * k, True),
                       (k * k, 16 * k + 1, False), (16 * k, k * k, True), (16 * k + 1, k * k, False), (1, k * k, True), (k * k, 1, True), (k * k + 1, 1, False),
                       (0, 1, False), (4096, 11008, True)):
        assert (lib.gptaq_linear_weights_bytes(m, n, 0) > 0) == fits and (lib.gptaq_linear_workspace_bytes(1, m, n) > 0) == fits, (m, n)
        assert lib.gptaq_linear_pack(ONE, n, ONE, ONE, m, n, 0, off, 1 << 62, ONE, NULL) == (-4 if fits else -2), (m, n)
        assert lib.gptaq_linear(ONE, 1, n, NULL, ONE, 1 << 62, m, n, 0, NULL, ONE, m, 0, off, 1 << 62, NULL) == (-4 if fits else -2), (m, n)
