"""The cache store, the attention and the log probabilities refuse bad arguments
on the host before any HIP call (no GPU needed), and their references against
values derived by hand."""
import ctypes
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
from paper_2609_20186_amd import binding as sd

OK, EINVAL, ESHAPE, EWORKSPACE = 0, -1, -2, -4
_buf = np.zeros(1 << 16, np.uint8)
P = (_buf.ctypes.data + 255) & ~255
INF = float("inf")


# ------------------------------------------------------------------ refusals

def store(**kw):
    a = dict(k=P, ks=256, v=P, vs=256, type=0, slots=P, n=4, count=None, Hkv=2, D=128, kc=P, vc=P,
             ctype=0, n_slots=64, k_scale=None, v_scale=None, stream=None)
    a.update(kw)
    return sd.lib.switchsd_store_cache(*a.values())


@pytest.mark.parametrize("kw,want", [
    (dict(type=2), EINVAL), (dict(type=3, ctype=3), EINVAL), (dict(ctype=1), EINVAL),
    (dict(ctype=2), EINVAL), (dict(n=-1), ESHAPE), (dict(Hkv=0), ESHAPE), (dict(Hkv=257), ESHAPE),
    (dict(D=96), ESHAPE), (dict(D=0), ESHAPE), (dict(n_slots=-1), ESHAPE),
    (dict(ks=255), ESHAPE), (dict(vs=248), ESHAPE), (dict(ks=-256), ESHAPE), (dict(ks=260), EINVAL),
    (dict(vs=2 ** 33), ESHAPE), (dict(n_slots=2 ** 41), ESHAPE),
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(slots=None), EINVAL),
    (dict(kc=None), EINVAL), (dict(vc=None), EINVAL), (dict(k=P + 2), EINVAL),
    (dict(vc=P + 8), EINVAL), (dict(slots=P + 4), EINVAL), (dict(k_scale=P), EINVAL),
    (dict(v_scale=P), EINVAL), (dict(n=0), OK), (dict(n_slots=0, kc=None, vc=None), OK),
])
def test_store_refusals(kw, want):
    assert store(**kw) == want


def attention_args(**kw):
    a = sd.AttentionArgs()
    a.B, a.R, a.rows, a.Hq, a.Hkv, a.D = 2, 8, 16, 8, 2, 128
    a.Lmax, a.page_size, a.max_pages, a.scale = 100, 16, 8, 0.1
    a.lengths = a.dn = a.table = a.held = P
    for k, v in kw.items():
        setattr(a, k, v)
    return a


CALL = dict(q=P, q_stride=1024, type=0, kc=P, vc=P, ctype=0, n_slots=64, ks=None, vs=None, out=P,
            lse=None, ws=P, bytes=1 << 40, stream=None)


def attend(args, **kw):
    return sd.lib.switchsd_paged_attention(ctypes.byref(args) if args else None,
                                           *{**CALL, **kw}.values())


@pytest.mark.parametrize("kw,want", [
    (dict(B=-1), ESHAPE), (dict(B=65537), ESHAPE), (dict(R=0), ESHAPE),
    (dict(R=2 ** 20 + 1), ESHAPE), (dict(rows=-1), ESHAPE), (dict(rows=17), ESHAPE),
    (dict(Hq=7), ESHAPE), (dict(Hq=0), ESHAPE), (dict(Hkv=0), ESHAPE), (dict(Hq=258), ESHAPE),
    (dict(D=32), ESHAPE), (dict(Lmax=0), ESHAPE), (dict(Lmax=2 ** 30 + 1), ESHAPE),
    (dict(page_size=0), ESHAPE), (dict(page_size=65537), ESHAPE), (dict(max_pages=0), ESHAPE),
    (dict(max_pages=2 ** 30), ESHAPE), (dict(scale=INF), EINVAL), (dict(scale=math.nan), EINVAL),
    (dict(lengths=None), EINVAL), (dict(dn=None), EINVAL), (dict(table=None), EINVAL),
    (dict(held=None), EINVAL), (dict(cu=P), EINVAL), (dict(B=0, rows=0), OK),
])
def test_attention_refusals(kw, want):
    assert attend(attention_args(**kw)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(type=2), EINVAL), (dict(type=3, ctype=3), EINVAL), (dict(ctype=1), EINVAL),
    (dict(n_slots=-1), ESHAPE), (dict(n_slots=2 ** 41), ESHAPE), (dict(q_stride=1016), ESHAPE),
    (dict(q_stride=1028), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL),
    (dict(kc=None), EINVAL), (dict(vc=None), EINVAL), (dict(q=P + 8), EINVAL),
    (dict(out=P + 4), EINVAL), (dict(kc=P + 2), EINVAL), (dict(ks=P), EINVAL), (dict(vs=P), EINVAL),
    (dict(ws=None), EWORKSPACE), (dict(ws=P + 64), EWORKSPACE), (dict(bytes=1000), EWORKSPACE),
])
def test_attention_call_refusals(kw, want):
    assert attend(attention_args(), **kw) == want
    assert attend(None) == EINVAL


def test_attention_workspace_bytes():
    size = sd.attention_workspace_bytes
    assert size(attention_args()) > 0
    assert size(attention_args(B=-1)) == 0 and size(attention_args(D=48)) == 0
    # what is read are sizes: no pointers, and rows that do not fit the batch
    assert size(attention_args(lengths=None, table=None)) == size(attention_args())
    # one work-group takes 32 or 128 rows of one head of the cache
    assert size(attention_args(R=8)) < size(attention_args(R=9, rows=18)) == \
        size(attention_args(R=17, rows=34)) == size(attention_args(R=1000, rows=2000))


def logprob_args(**kw):
    a = sd.LogprobArgs()
    a.logits, a.tokens, a.B, a.R, a.V, a.temperature = P, P, 2, 3, 50, 1.0
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def logprobs(args, logprob=P, lse=None, entropy=None, rank=None, n_top=0, ids=None, tops=None):
    return sd.lib.switchsd_token_logprobs(ctypes.byref(args), logprob, lse, entropy, rank, n_top,
                                          ids, tops, None)


BAD_LOGPROBS = [
    (dict(logits_type=3), EINVAL), (dict(logits_type=-1), EINVAL), (dict(temperature=0.0), EINVAL),
    (dict(temperature=-1.0), EINVAL), (dict(temperature=INF), EINVAL),
    (dict(temperature=math.nan), EINVAL), (dict(temperature=1e-40), EINVAL), (dict(B=-1), ESHAPE),
    (dict(B=1 << 24, R=1), ESHAPE), (dict(R=0), ESHAPE), (dict(R=1025), ESHAPE),
    (dict(V=0), ESHAPE), (dict(V=(1 << 26) + 1), ESHAPE), (dict(logits=None), EINVAL),
    (dict(logits=P + 1), EINVAL), (dict(logits=P + 2, logits_type=2), EINVAL),
    (dict(tokens=None), EINVAL), (dict(B=0, logits=None, tokens=None), OK),
]


@pytest.mark.parametrize("kw,want", BAD_LOGPROBS)
def test_logprob_refusals(kw, want):
    assert logprobs(logprob_args(**kw)) == want


def test_logprob_output_refusals():
    a = logprob_args()
    assert logprobs(a, n_top=-1, ids=P) == ESHAPE
    assert logprobs(a, n_top=65, ids=P) == ESHAPE
    assert logprobs(a, n_top=51, ids=P) == ESHAPE
    assert logprobs(a, n_top=5) == EINVAL and logprobs(a, ids=P) == EINVAL
    assert logprobs(a, logprob=None) == EINVAL
    assert logprobs(logprob_args(tokens=None), logprob=None, rank=P) == EINVAL


@pytest.mark.parametrize("kw,want", BAD_LOGPROBS)
def test_grad_refusals(kw, want):
    a = logprob_args(**kw)
    assert sd.lib.switchsd_token_logprobs_grad(ctypes.byref(a), P, None, P, None, P + 4096,
                                               None) == want


@pytest.mark.parametrize("args", [
    (None, None, P, None, P), (P, None, P, None, None), (P, None, None, None, P),
    (P, None, None, P, P), (P, None, P, None, P + 1),
    (P, None, P, None, P + 2), (P, None, P, None, P + 298),     # overlaps, but is not, the logits
])
def test_grad_argument_refusals(args):
    a = logprob_args()
    assert sd.lib.switchsd_token_logprobs_grad(ctypes.byref(a), *args, None) == EINVAL


# ------------------------------------------------------------------ binding

HUGE = 2 ** 32 + 16


@pytest.mark.parametrize("call", [
    lambda i: sd.build_attention_args(HUGE, 8, 8, 2, 128, 16, i(2, 4), i(2), 9, i(2), i(2)),
    lambda i: sd.build_attention_args(16, HUGE, 8, 2, 128, 16, i(2, 4), i(2), 9, i(2), i(2)),
    lambda i: sd.build_attention_args(16, 8, 8, 2, 128, HUGE, i(2, 4), i(2), 9, i(2), i(2)),
    lambda i: sd.build_attention_args(16, 8, 8, 2, 128, 16, i(2, 4), i(2), HUGE, i(2), i(2)),
    lambda i: sd.build_attention_args(16, 8, HUGE, 2, 128, 16, i(2, 4), i(2), 9, i(2), i(2)),
    lambda i: sd.build_logprob_args(torch.zeros(1, dtype=torch.float32).expand(1, 1, HUGE)),
])
def test_sizes_beyond_32_bits(call):
    with pytest.raises(ValueError, match="does not fit 32 bits"):
        call(lambda *s: torch.zeros(s, dtype=torch.int32))


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    s = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="keys must be a device tensor"):
        sd.switchsd_store_cache(x, x, s, x, x)
    with pytest.raises(ValueError, match="table must be"):
        sd.build_attention_args(4, 2, 2, 2, 128, 16, s, s, 9, s, s)
    with pytest.raises(ValueError, match="logits must be"):
        sd.build_logprob_args(x[0])
    with pytest.raises(ValueError, match="dpar comes with accept_node"):
        sd.build_logprob_args(x, dpar=s)


# ------------------------------------------------------------------ references

def test_e4m3_reference():
    vals = ref.e4m3_values()
    assert vals[1] == 2.0 ** -9 and vals[8] == 2.0 ** -6 and vals[126] == 448.0
    x = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(x, vals)
    # 17 lies between 16 and 18: the even fraction; 1e9 saturates
    got = ref.to_e4m3(np.array([17.0, -17.0, 19.0, 1e9, -INF, 0.0, -0.0, np.nan], np.float32))
    assert vals[got[0]] == 16 and got[1] == got[0] | 0x80 and vals[got[2]] == 20
    assert list(got[3:]) == [126, 254, 0, 128, 127]


def test_attention_reference_by_hand():
    """Two equal keys: the mean of their values; a third one twice as likely."""
    a = dict(rows=1, R=1, Lmax=8, Hq=1, Hkv=1, D=1, page=2, n_slots=8, scale=1.0, type="bf16",
             table=np.array([[1, 3]]), held=np.array([2]), lengths=np.array([3]),
             dn=np.array([1]))
    k, v = np.zeros((8, 1, 1)), np.zeros((8, 1, 1))
    k[6] = math.log(2.0)
    v[2], v[3], v[6], v[7] = 1.0, 3.0, 10.0, np.nan
    out, lse, _, _ = ref.attention(a, np.ones((1, 1, 1)), k, v)[0]
    assert out[0, 0] == pytest.approx((1 + 3 + 20) / 4) and lse[0] == pytest.approx(math.log(4))
    a["held"][:] = 1                                       # the second page is not there
    assert ref.attention(a, np.ones((1, 1, 1)), k, v)[0][0][0, 0] == pytest.approx(2.0)
    a["mask"] = np.array([[0]], np.uint32)
    a["lengths"][:] = 1
    out, lse, _, _ = ref.attention(a, np.ones((1, 1, 1)), k, v)[0]
    assert out[0, 0] == 0 and lse[0] == -INF


def test_logprob_reference_by_hand():
    lse, lp, h = ref.row_logprobs(np.array([0.0, math.log(3.0), np.nan, -INF]), 1.0)
    assert lse == pytest.approx(math.log(4)) and lp[1] == pytest.approx(math.log(0.75))
    assert lp[2] == lp[3] == -INF
    assert h == pytest.approx(-0.75 * math.log(0.75) - 0.25 * math.log(0.25))
    assert ref.order(np.array([0.0, 2.0, np.nan, 2.0, -INF])) == [1, 3, 0, 4, 2]
    assert ref.row_logprobs(np.array([np.nan, INF, INF]), 1.0)[1].tolist() == [-INF, 0.0, -INF]
    assert ref.row_logprobs(np.array([np.nan, np.nan]), 1.0)[1].tolist() == [0.0, -INF]


def test_grad_reference_against_differences():
    """Central differences of g log p_t + h H in 64 bits: their own error is of the
    order d^2 (third derivatives times the temperature's third power) + 2^-52 / d."""
    rng = np.random.default_rng(5)
    for T in (1.0, 0.6):
        x = rng.normal(size=9) * 2
        x[3] = -INF
        tok, g, ge, d = 4, 0.7, -0.3, 1e-5

        def loss(y):
            _, lp, h = ref.row_logprobs(y, T)
            return g * lp[tok] + ge * h
        lse, _, h = ref.row_logprobs(x, T)
        got = ref.grad_row(x, T, tok, lse, h, g, ge)
        for v in range(9):
            if v == 3:
                assert got[v] == 0
                continue
            e = np.zeros(9)
            e[v] = d
            assert got[v] == pytest.approx((loss(x + e) - loss(x - e)) / (2 * d), abs=1e-8)
