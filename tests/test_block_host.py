"""What a residual block's operators refuse on the host (no GPU needed): every call below fails before anything is
enqueued, or has no array to touch."""
import ctypes
import os

import pytest

from paper_2609_37899_amd import soma

WS = ctypes.c_void_p(0x100000)         # none of these is ever dereferenced
BIG = 1 << 40


def ptr(k):
    """Arrays far apart from one another."""
    return ctypes.c_void_p(0x10000000000 * (k + 1))


def at(p, by):
    return ctypes.c_void_p(p.value + by)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(soma.LIB_PATH):
        from paper_2609_37899_amd import build
        build.build()
    return soma.load()


def passed(rc):
    """Past the checks: done, or nothing to run it on."""
    return rc in (soma.SOMA_OK, soma.SOMA_EDEVICE)


def la_cfg(**kw):
    c = soma.LinearAttentionConfig(1000, 2, 4, 2, 16, 24, 0, 0.25, 64, 32, 48)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


NAMES = ("q", "k", "v", "log_decay", "offsets", "s0", "do", "dsT", "dq", "dk", "dv", "ds0", "o", "sT")
A = {n: ptr(i) for i, n in enumerate(NAMES)}


def forward(lib, cfg, ws=WS, n=BIG, **kw):
    x = dict(A, **kw)
    return lib.soma_la_forward(cfg, *(x[k] for k in ("q", "k", "v", "log_decay", "offsets", "s0", "o", "sT")), ws, n, None)


def backward(lib, cfg, ws=WS, n=BIG, **kw):
    x = dict(A, **kw)
    return lib.soma_la_backward(cfg, *(x[k] for k in ("q", "k", "v", "log_decay", "offsets", "s0", "do", "dsT", "dq", "dk", "dv",
                                                      "ds0")), ws, n, None)


def step(lib, cfg, **kw):
    x = dict(A, **kw)
    return lib.soma_la_step(cfg, *(x[k] for k in ("q", "k", "v", "log_decay", "s0", "sT", "o")), None)


@pytest.mark.parametrize("field,value,code", [
    ("rows", -1, soma.SOMA_ESHAPE), ("rows", 2**30 + 1, soma.SOMA_ESHAPE), ("sequences", 0, soma.SOMA_ESHAPE),
    ("sequences", 65536, soma.SOMA_ESHAPE), ("heads", 0, soma.SOMA_ESHAPE), ("heads", 1025, soma.SOMA_ESHAPE),
    ("kv_heads", 0, soma.SOMA_ESHAPE), ("kv_heads", 3, soma.SOMA_ESHAPE), ("kv_heads", 8, soma.SOMA_ESHAPE),
    ("key_width", 0, soma.SOMA_ESHAPE), ("key_width", 257, soma.SOMA_ESHAPE), ("value_width", 0, soma.SOMA_ESHAPE),
    ("value_width", 257, soma.SOMA_ESHAPE), ("type", 2, soma.SOMA_EINVAL), ("type", -1, soma.SOMA_EINVAL),
    ("scale", float("nan"), soma.SOMA_EINVAL), ("scale", float("inf"), soma.SOMA_EINVAL), ("q_stride", 63, soma.SOMA_ESHAPE),
    ("k_stride", 31, soma.SOMA_ESHAPE), ("v_stride", 47, soma.SOMA_ESHAPE), ("q_stride", 2**33, soma.SOMA_ESHAPE),
    ("v_stride", 2**22 + 1, soma.SOMA_ESHAPE)])
def test_linear_attention_shapes(lib, field, value, code):
    c, out = la_cfg(**{field: value}), ctypes.c_size_t()
    assert lib.soma_la_workspace_size(c, 1, ctypes.byref(out)) == code
    for call in (forward, backward, step):
        assert call(lib, c) == code
    assert lib.soma_last_error()


def test_more_blocks_than_a_launch_has(lib):
    """2^24 blocks of 256 threads would be 2^32; dropout's elements are counted alike."""
    out = ctypes.c_size_t()
    for heads, width, code in ((256, 64, soma.SOMA_OK), (257, 64, soma.SOMA_ESHAPE), (128, 128, soma.SOMA_OK),
                               (129, 65, soma.SOMA_ESHAPE), (64, 256, soma.SOMA_OK), (65, 193, soma.SOMA_ESHAPE)):
        for kw in (dict(key_width=width, value_width=1), dict(key_width=1, value_width=width)):
            c = la_cfg(rows=65535, sequences=65535, heads=heads, kv_heads=heads, q_stride=2**22, k_stride=2**22, v_stride=2**22, **kw)
            assert lib.soma_la_workspace_size(c, 1, ctypes.byref(out)) == code, (heads, width)
            if code:
                assert forward(lib, c) == backward(lib, c) == step(lib, c) == code
    many = dict(width=2**10, x_stride=2**10, residual_stride=2**10)
    assert dropout(lib, dropout_cfg(rows=2**24 + 1, **many)) == soma.SOMA_ESHAPE


def test_linear_attention_arguments(lib):
    out, c = ctypes.c_size_t(), la_cfg()
    assert lib.soma_la_workspace_size(None, 0, ctypes.byref(out)) == soma.SOMA_EINVAL
    assert lib.soma_la_workspace_size(c, 0, None) == soma.SOMA_EINVAL
    need = []
    for grad in (0, 1):
        assert lib.soma_la_workspace_size(c, grad, ctypes.byref(out)) == soma.SOMA_OK
        need.append(out.value)
    assert 0 < need[0] < need[1]
    # blocks enough, or rows too few for pieces: no workspace
    for kw in (dict(sequences=500), dict(rows=512, type=1), dict(rows=256)):
        assert lib.soma_la_workspace_size(la_cfg(**kw), 0, ctypes.byref(out)) == soma.SOMA_OK and out.value == 0
    for call, names in ((forward, ("q", "k", "v", "log_decay", "o")), (backward, ("q", "k", "v", "log_decay", "do", "dq", "dk", "dv"))):
        for name in names:
            assert call(lib, c, **{name: None}) == soma.SOMA_EINVAL, name
    s = la_cfg(rows=2)
    for name in ("q", "k", "v", "log_decay", "sT", "o"):
        assert step(lib, s, **{name: None}) == soma.SOMA_EINVAL, name
    for call, cfg, names in ((forward, c, ("q", "k", "v", "log_decay", "offsets", "s0", "o", "sT")),
                             (backward, c, ("q", "k", "v", "log_decay", "offsets", "s0", "do", "dsT", "dq", "dk", "dv", "ds0")),
                             (step, s, ("q", "k", "v", "log_decay", "s0", "sT", "o"))):
        for name in names:
            assert call(lib, cfg, **{name: at(A[name], 2)}) == soma.SOMA_EINVAL, name
    assert step(lib, c) == soma.SOMA_ESHAPE                                # 1000 rows for 2 sequences
    for call, size in ((forward, need[0]), (backward, need[1])):
        assert call(lib, la_cfg(rows=1001), offsets=None) == soma.SOMA_ESHAPE   # no offsets: a multiple of the sequences
        for kw in (dict(ws=None), dict(ws=at(WS, 128)), dict(n=size - 1)):
            assert call(lib, c, **kw) == soma.SOMA_EWORKSPACE, kw
    # outputs that overlap: the last byte of 1000 rows of 64, 32 or 48 elements, or of 2 x 4 states
    ends = {"q": 256000, "k": 128000, "v": 192000, "do": 384000, "o": 384000, "s0": 12288, "sT": 12288, "log_decay": 16,
            "offsets": 12, "dsT": 12288, "dq": 256000, "dk": 128000, "dv": 192000, "ds0": 12288}
    for call, outs, ins in ((forward, ("o", "sT"), ("q", "k", "v", "log_decay", "offsets", "s0")),
                            (backward, ("dq", "dk", "dv", "ds0"), ("q", "k", "v", "log_decay", "offsets", "s0", "do", "dsT"))):
        for o in outs:
            for i in ins + tuple(x for x in outs if x != o):
                assert call(lib, c, **{o: at(A[i], ends[i] - 4)}) == soma.SOMA_EINVAL, (o, i)
                assert b"overlap" in lib.soma_last_error()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 1), (32, 8)])
def test_linear_attention_workspace_serves_fewer_rows(lib, dtype, heads, kv):
    out = ctypes.c_size_t()
    for S in (1, 3, 64, 65535):
        for dk, dv in ((1, 1), (64, 64), (45, 77), (256, 200), (30, 256)):
            for grad in (0, 1):
                last = 0
                for rows in (0, 1, 64, 256, 257, 768, 769, 10**4, 16384, 16385, 10**6, 2**30):
                    c = la_cfg(rows=rows, sequences=S, heads=heads, kv_heads=kv, key_width=dk, value_width=dv, type=dtype,
                               q_stride=heads * dk, k_stride=kv * dk, v_stride=kv * dv)
                    assert lib.soma_la_workspace_size(c, grad, ctypes.byref(out)) == soma.SOMA_OK
                    assert out.value >= last
                    last = out.value


@pytest.mark.parametrize("dtype", [0, 1])
def test_linear_attention_of_no_rows_is_no_error(lib, dtype):
    """Arrays of no rows have no address."""
    c = la_cfg(rows=0, type=dtype)
    none = dict.fromkeys(("q", "k", "v", "offsets", "s0", "do", "dsT", "dq", "dk", "dv", "ds0", "o", "sT"))
    assert passed(forward(lib, c, None, 0, **none)) and passed(backward(lib, c, None, 0, **none))


def drop(**kw):
    d = soma.Drop(0.1, 1, 2, None, 3, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return ctypes.byref(d)


DROPS = (dict(p=-0.1), dict(p=1.0), dict(p=float("nan")), dict(p=1 - 2.0**-18), dict(step_dev=0x1004), dict(reserved=1))


def dropout(lib, cfg, x=ptr(0), residual=ptr(1), d=None, y=ptr(2)):
    return lib.soma_dropout(cfg, x, residual, d if d is not None else drop(), y, None)


def dropout_cfg(**kw):
    c = soma.DropoutConfig(10, 20, 0, 0, 24, 20)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


@pytest.mark.parametrize("field,value,code", [
    ("rows", -1, soma.SOMA_ESHAPE), ("rows", 2**30 + 1, soma.SOMA_ESHAPE), ("width", 0, soma.SOMA_ESHAPE),
    ("width", 2**20 + 1, soma.SOMA_ESHAPE), ("type", 2, soma.SOMA_EINVAL), ("reserved", 1, soma.SOMA_EINVAL),
    ("x_stride", 19, soma.SOMA_ESHAPE), ("residual_stride", 19, soma.SOMA_ESHAPE), ("x_stride", 2**33, soma.SOMA_ESHAPE)])
def test_dropout_shapes(lib, field, value, code):
    assert dropout(lib, dropout_cfg(**{field: value})) == code and lib.soma_last_error()


def test_dropout_arguments(lib):
    c = dropout_cfg()
    assert lib.soma_dropout(None, ptr(0), None, None, ptr(1), None) == soma.SOMA_EINVAL
    for kw in (dict(x=None), dict(y=None), dict(x=at(ptr(0), 2)), dict(residual=at(ptr(0), 2)), dict(y=at(ptr(0), 2))):
        assert dropout(lib, c, **kw) == soma.SOMA_EINVAL, kw
    for kw in DROPS:
        assert dropout(lib, c, d=drop(**kw)) == soma.SOMA_EINVAL, kw
    # y over part of x, over strided x, over part of the residual, over the step
    for y in (at(ptr(0), 4 * (9 * 24 + 19)), ptr(0), at(ptr(1), 796), at(ptr(1), -796)):
        assert dropout(lib, c, y=y) == soma.SOMA_EINVAL and b"overlap" in lib.soma_last_error()
    assert dropout(lib, c, d=drop(step_dev=ptr(2).value + 8)) == soma.SOMA_EINVAL
    assert dropout(lib, dropout_cfg(rows=2**30, width=2**20, x_stride=2**20, residual_stride=2**20)) == soma.SOMA_ESHAPE
    assert passed(dropout(lib, c, y=ptr(1)))                      # in place of the residual
    assert lib.soma_dropout(dropout_cfg(rows=0), None, None, None, None, None) == soma.SOMA_OK


def norm_cfg(**kw):
    c = soma.NormConfig(10, 20, 1, 0, 1e-5, 0, 20, 20)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


N = {n: ptr(i) for i, n in enumerate(("x", "residual", "gain", "total", "y", "scales", "dy", "dtotal", "dresidual", "dx", "dgain"))}


def norm_forward(lib, cfg, d=None, **kw):
    x = dict(N, **kw)
    return lib.soma_norm_forward(cfg, x["x"], x["residual"], x["gain"], d, x["total"], x["y"], None)


def norm_codes(lib, cfg, d=None, **kw):
    x = dict(N, **kw)
    return lib.soma_norm_forward_codes(cfg, x["x"], x["residual"], x["gain"], d, x["total"], x["y"], x["scales"], None)


def norm_backward(lib, cfg, d=None, ws=WS, n=BIG, **kw):
    x = dict(N, **kw)
    return lib.soma_norm_backward(cfg, x["total"], x["gain"], x["dy"], x["dtotal"], d, x["dresidual"], x["dx"], x["dgain"], ws, n, None)


@pytest.mark.parametrize("field,value,code", [
    ("rows", -1, soma.SOMA_ESHAPE), ("rows", 2**30 + 1, soma.SOMA_ESHAPE), ("width", 0, soma.SOMA_ESHAPE),
    ("width", 2**14 + 1, soma.SOMA_ESHAPE), ("type", 2, soma.SOMA_EINVAL), ("sum_type", -1, soma.SOMA_EINVAL),
    ("reserved", 1, soma.SOMA_EINVAL), ("eps", -1e-5, soma.SOMA_EINVAL), ("eps", float("nan"), soma.SOMA_EINVAL),
    ("eps", float("inf"), soma.SOMA_EINVAL), ("x_stride", 19, soma.SOMA_ESHAPE), ("residual_stride", 19, soma.SOMA_ESHAPE),
    ("residual_stride", 2**33, soma.SOMA_ESHAPE)])
def test_norm_shapes(lib, field, value, code):
    c, out = norm_cfg(**{field: value}), ctypes.c_size_t()
    assert lib.soma_norm_workspace_size(c, ctypes.byref(out)) == code
    for call in (norm_forward, norm_codes, norm_backward):
        assert call(lib, c) == code and lib.soma_last_error()


def test_norm_arguments(lib):
    out, c = ctypes.c_size_t(), norm_cfg()
    assert lib.soma_norm_workspace_size(None, ctypes.byref(out)) == soma.SOMA_EINVAL
    assert lib.soma_norm_workspace_size(c, None) == soma.SOMA_EINVAL
    assert norm_forward(lib, norm_cfg(type=0, sum_type=1)) == soma.SOMA_EINVAL
    last = 0
    for rows in (0, 1, 3, 4, 5, 1000, 4096, 4097, 10**6, 2**30):
        assert lib.soma_norm_workspace_size(norm_cfg(rows=rows), ctypes.byref(out)) == soma.SOMA_OK
        assert out.value >= last
        last = out.value
    for call, names in ((norm_forward, ("x", "gain", "y")), (norm_codes, ("x", "gain", "y", "scales")), (norm_backward, ("total", "gain", "dy"))):
        for name in names:
            assert call(lib, c, **{name: None}) == soma.SOMA_EINVAL, name
        for kw in DROPS:
            assert call(lib, c, drop(**kw)) == soma.SOMA_EINVAL, kw
    assert norm_backward(lib, c, dresidual=None, dx=None, dgain=None) == soma.SOMA_EINVAL
    for call, names in ((norm_forward, ("x", "residual", "gain", "total", "y")), (norm_codes, ("x", "residual", "gain", "total", "scales")),
                        (norm_backward, ("total", "gain", "dy", "dtotal", "dresidual", "dx", "dgain"))):
        for name in names:
            assert call(lib, c, **{name: at(N[name], 1)}) == soma.SOMA_EINVAL, name
    # bytes of 10 x 20 elements of bf16 or fp32
    size = dict(x=400, residual=800, gain=80, total=800, y=400, scales=40, dy=400, dtotal=800, dresidual=800, dx=400, dgain=80)
    for call, outs, ins in ((norm_forward, ("total", "y"), ("x", "residual", "gain")),
                            (norm_codes, ("total", "scales"), ("x", "residual", "gain")),
                            (norm_backward, ("dresidual", "dx", "dgain"), ("total", "gain", "dy", "dtotal"))):
        for o in outs:
            for i in ins + tuple(x for x in outs if x != o):
                assert call(lib, c, **{o: at(N[i], size[i] - 4)}) == soma.SOMA_EINVAL, (o, i)
                assert b"overlap" in lib.soma_last_error()
    # in place of strided rows
    assert norm_forward(lib, norm_cfg(residual_stride=24), total=N["residual"]) == soma.SOMA_EINVAL
    assert passed(norm_forward(lib, c, total=N["residual"])) and passed(norm_backward(lib, c, dresidual=N["dtotal"]))
    assert lib.soma_norm_workspace_size(c, ctypes.byref(out)) == soma.SOMA_OK
    for kw in (dict(ws=None), dict(ws=at(WS, 128)), dict(n=out.value - 1)):
        assert norm_backward(lib, c, **kw) == soma.SOMA_EWORKSPACE, kw
    none = dict.fromkeys(("x", "residual", "total", "y", "scales"))
    assert norm_forward(lib, norm_cfg(rows=0), **none) == soma.SOMA_OK and norm_codes(lib, norm_cfg(rows=0), **none) == soma.SOMA_OK
    none = dict.fromkeys(("total", "dy", "dtotal", "dresidual", "dx"))
    assert passed(norm_backward(lib, norm_cfg(rows=0), **none))


def sample_cfg(**kw):
    c = soma.SampleConfig(10, 1000, 0, 0, 1000)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


SAMPLE = ("logits", "u", "temperature", "top_k", "top_p", "min_p", "tokens", "logprob")


def sample(lib, cfg, **kw):
    x = dict({n: ptr(i) for i, n in enumerate(SAMPLE)}, **kw)
    return lib.soma_sample(cfg, *(x[n] for n in SAMPLE), None)


@pytest.mark.parametrize("field,value,code", [
    ("rows", -1, soma.SOMA_ESHAPE), ("rows", 2**20 + 1, soma.SOMA_ESHAPE), ("vocab", 0, soma.SOMA_ESHAPE),
    ("vocab", 2**20 + 1, soma.SOMA_ESHAPE), ("type", 2, soma.SOMA_EINVAL), ("reserved", 1, soma.SOMA_EINVAL),
    ("logit_stride", 999, soma.SOMA_ESHAPE), ("logit_stride", 2**33, soma.SOMA_ESHAPE)])
def test_sample_shapes(lib, field, value, code):
    assert sample(lib, sample_cfg(**{field: value})) == code and lib.soma_last_error()


def test_sample_arguments(lib):
    c = sample_cfg()
    assert sample(lib, None) == soma.SOMA_EINVAL
    for name in ("logits", "u", "tokens"):
        assert sample(lib, c, **{name: None}) == soma.SOMA_EINVAL, name
    for i, name in enumerate(SAMPLE):
        assert sample(lib, c, **{name: at(ptr(i), 2)}) == soma.SOMA_EINVAL, name
    for o in ("tokens", "logprob"):
        for i, name in enumerate(SAMPLE):
            if name != o:
                assert sample(lib, c, **{o: at(ptr(i), 36)}) == soma.SOMA_EINVAL and b"overlap" in lib.soma_last_error()
    assert sample(lib, sample_cfg(rows=0), **dict.fromkeys(SAMPLE)) == soma.SOMA_OK


def test_classes_refuse_on_the_host():
    torch = pytest.importorskip("torch")
    soma.load()
    with pytest.raises(TypeError):
        soma.LinearAttention(10, 1, 2, 8, 8, torch.float16)
    with pytest.raises(TypeError):
        soma.LinearAttention(10, 1, 2, 8, 8, torch.float32, device="cpu")
    for bad in ((-1, 1, 2, 8, 8), (10, 1, -2, 8, 8), (10, 2**31, 2, 8, 8)):
        with pytest.raises(ValueError):
            soma.LinearAttention(*bad, torch.float32)
    for bad in ((10, 0, 2, 8, 8), (10, 1, 2, 0, 8), (10, 1, 2, 8, 300)):
        with pytest.raises(soma.SomaError):
            soma.LinearAttention(*bad, torch.float32)
    with pytest.raises(soma.SomaError):
        soma.LinearAttention(10, 1, 4, 8, 8, torch.float32, kv_heads=3)
    with pytest.raises(soma.SomaError):
        soma.LinearAttention(10, 1, 4, 8, 8, torch.float32, scale=float("nan"))
    for bad in (-0.1, 1.0, float("nan"), 1 - 2.0**-18):
        with pytest.raises(ValueError):
            soma.Dropout(10, 8, torch.float32, bad)
        with pytest.raises(ValueError):
            soma.RmsNorm(10, 8, torch.float32, drop=bad)
    with pytest.raises(TypeError):
        soma.Dropout(10, 8, torch.float16, 0.1)
    with pytest.raises(TypeError):
        soma.RmsNorm(10, 8, torch.bfloat16, torch.float16)
    with pytest.raises(soma.SomaError):
        soma.RmsNorm(10, 8, torch.float32, torch.bfloat16)
    with pytest.raises(soma.SomaError):
        soma.RmsNorm(10, 2**14 + 1, torch.float32)
    for make in (lambda: soma.Dropout(10, 8, torch.float32, 0.1, device="cpu"), lambda: soma.RmsNorm(10, 8, torch.float32, device="cpu"),
                 lambda: soma.Sampler(10, 8, torch.float32, device="cpu"), lambda: soma.Sampler(10, 8, torch.float16)):
        with pytest.raises(TypeError):
            make()
    for make in (lambda: soma.Sampler(-1, 8, torch.float32), lambda: soma.Dropout(10, -8, torch.float32, 0.1),
                 lambda: soma.RmsNorm(2**31, 8, torch.float32)):
        with pytest.raises(ValueError):
            make()
