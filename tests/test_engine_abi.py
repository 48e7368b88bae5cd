"""The calls around the step reject bad arguments on the host before any HIP
call (no GPU needed), and the plain references of their tests agree with
hand-derived values."""
import ctypes

import numpy as np
import pytest
import torch

import engine_ref as ref
from paper_2609_20186_amd import binding as sd

OK, EINVAL, ESHAPE, EWORKSPACE = 0, -1, -2, -4

# Host buffers stand in for device pointers: every call below fails validation
# and never reaches HIP.
_buf = np.zeros(1 << 16, np.uint8)
P = (_buf.ctypes.data + 255) & ~255
FAR = P + (1 << 40)


def logits_args(**kw):
    a = sd.LogitsArgs()
    for f in ("logits", "dtok", "dpar", "dn", "tokens", "lengths", "prompt_lens", "repetition",
              "frequency", "presence", "bias_ids", "bias_vals", "allowed", "allowed_on"):
        setattr(a, f, P)
    a.logits_type, a.B, a.R, a.V, a.Lmax, a.n_bias = sd.BF16, 2, 8, 100, 16, 4
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_LOGITS = [
    (dict(B=-1), ESHAPE), (dict(R=0), ESHAPE), (dict(R=1025), ESHAPE), (dict(V=0), ESHAPE),
    (dict(V=(1 << 28) + 1), ESHAPE), (dict(Lmax=-1), ESHAPE), (dict(Lmax=1 << 21), ESHAPE),
    (dict(Lmax=0), ESHAPE), (dict(n_bias=-1), ESHAPE), (dict(n_bias=512), ESHAPE),
    (dict(logits_type=3), EINVAL), (dict(logits_type=-1), EINVAL), (dict(logits=None), EINVAL),
    (dict(logits=P + 1), EINVAL), (dict(logits=P + 2, logits_type=sd.F32), EINVAL),
    (dict(dtok=None), EINVAL), (dict(dn=None), EINVAL), (dict(tokens=None), EINVAL),
    (dict(lengths=None), EINVAL), (dict(bias_ids=None), EINVAL), (dict(bias_vals=None), EINVAL),
    (dict(tokens=None, repetition=None, presence=None), EINVAL),
]


@pytest.mark.parametrize("kw,code", BAD_LOGITS)
def test_logits_arguments(kw, code):
    a = logits_args(**kw)
    lib = sd.lib
    assert lib.switchsd_process_logits(ctypes.byref(a), FAR, sd.BF16, None) == code
    assert lib.switchsd_verify_processed(ctypes.byref(a), P, P, P, P, P, P, 1 << 15,
                                         None) == code


def test_process_rejects():
    lib = sd.lib
    call = lambda a, out, t: lib.switchsd_process_logits(ctypes.byref(a), out, t, None)
    assert lib.switchsd_process_logits(None, FAR, sd.BF16, None) == EINVAL
    a = logits_args()
    assert call(a, None, sd.BF16) == EINVAL
    assert call(a, FAR + 1, sd.BF16) == EINVAL
    assert call(a, FAR, sd.F32) == EINVAL               # bf16 logits, float output
    assert call(a, FAR, 7) == EINVAL
    f = logits_args(logits_type=sd.F32)
    assert call(f, FAR + 2, sd.F32) == EINVAL
    # a partial overlap in either direction, and one of different types
    n = 2 * 8 * 100
    assert call(a, P + 2, sd.BF16) == EINVAL
    assert call(a, P + 2 * n - 2, sd.BF16) == EINVAL
    assert call(logits_args(logits=P + 2 * n - 2), P, sd.BF16) == EINVAL
    assert call(f, P, sd.BF16) == EINVAL
    # an empty batch is a no-op
    assert call(logits_args(B=0, logits=None, dtok=None, tokens=None), None, sd.BF16) == OK
    # more work-groups than a launch takes
    assert call(logits_args(B=1 << 24, R=1024, V=1 << 28), FAR, sd.BF16) in (ESHAPE, EINVAL, -3)


def test_verify_rejects():
    lib = sd.lib
    a = logits_args()
    need = sd.workspace_bytes(2, 8)

    def call(outs=(P,) * 5, ws=P, n=need):
        return lib.switchsd_verify_processed(ctypes.byref(a), *outs, ws, n, None)
    for j in range(4):
        assert call(outs=tuple(None if i == j else P for i in range(5))) == EINVAL
    assert call(ws=None) == EWORKSPACE
    assert call(ws=P + 8) == EWORKSPACE
    assert call(n=need - 1) == EWORKSPACE
    assert lib.switchsd_verify_processed(None, P, P, P, P, P, P, need, None) == EINVAL
    z = logits_args(B=0)
    assert lib.switchsd_verify_processed(ctypes.byref(z), None, None, None, None, None, None, 0,
                                         None) == OK


def page_args(**kw):
    a = sd.PageArgs()
    for f in ("lengths", "dpar", "dn", "table", "held", "ring", "ring_state", "slots",
              "positions", "missing"):
        setattr(a, f, P)
    a.B, a.R, a.Lmax, a.page_size, a.max_pages, a.ring_pages = 2, 8, 100, 16, 7, 20
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), ESHAPE), (dict(B=65537), ESHAPE), (dict(R=0), ESHAPE), (dict(R=1025), ESHAPE),
    (dict(Lmax=0), ESHAPE), (dict(Lmax=(1 << 30) + 1), ESHAPE), (dict(page_size=0), ESHAPE),
    (dict(page_size=65537), ESHAPE), (dict(max_pages=0), ESHAPE), (dict(ring_pages=0), ESHAPE),
    (dict(max_pages=1 << 30), ESHAPE), (dict(B=65536, max_pages=32768, page_size=1), ESHAPE),
    (dict(lengths=None), EINVAL), (dict(dn=None), EINVAL), (dict(table=None), EINVAL),
    (dict(held=None), EINVAL), (dict(ring=None), EINVAL), (dict(ring_state=None), EINVAL),
    (dict(missing=None), EINVAL), (dict(slots=P + 4), EINVAL),
])
def test_plan_rejects(kw, code):
    a = page_args(**kw)
    assert sd.lib.switchsd_page_plan(ctypes.byref(a), P, 1 << 15, None) == code


def test_plan_workspace_and_empty():
    lib = sd.lib
    a = page_args()
    need = sd.workspace_bytes(2, 0)
    assert lib.switchsd_page_plan(None, P, need, None) == EINVAL
    assert lib.switchsd_page_plan(ctypes.byref(a), None, need, None) == EWORKSPACE
    assert lib.switchsd_page_plan(ctypes.byref(a), P + 8, need, None) == EWORKSPACE
    assert lib.switchsd_page_plan(ctypes.byref(a), P, need - 1, None) == EWORKSPACE
    assert lib.switchsd_page_plan(ctypes.byref(page_args(B=0, table=None)), None, 0, None) == OK


def test_spans_reject():
    def call(begin=P, end=P, tokens=P, table=P, held=P, B=2, Lmax=100, most=7, page=16, cu=P,
             slots=P, positions=P, packed=P, seq=P, cap=10):
        return sd.lib.switchsd_span_slots(begin, end, tokens, table, held, B, Lmax, most, page,
                                          cu, slots, positions, packed, seq, cap, None)
    for kw in (dict(B=-1), dict(B=65537), dict(Lmax=0), dict(Lmax=(1 << 30) + 1),
               dict(B=4, Lmax=1 << 29), dict(page=0), dict(page=65537), dict(cap=-1),
               dict(most=0), dict(B=4, most=1 << 29)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(begin=None), dict(end=None), dict(cu=None), dict(tokens=None),
               dict(table=None), dict(held=None), dict(slots=P + 4)):
        assert call(**kw) == EINVAL, kw
    assert call(B=0, begin=None, cu=None) == OK


def test_compact_rejects():
    def call(cache=P, planes=2, stride=4096, n=4, row=1024, slots=P, dpar=P, dn=P, node=P, B=2,
             R=8):
        return sd.lib.switchsd_compact_cache(cache, planes, stride, n, row, slots, dpar, dn, node,
                                             B, R, None)
    for kw in (dict(B=-1), dict(R=0), dict(R=1025), dict(planes=-1), dict(n=-1), dict(row=-4),
               dict(stride=4092), dict(n=1 << 60), dict(stride=-4096)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(row=1022), dict(stride=4098), dict(cache=None), dict(cache=P + 2),
               dict(slots=None), dict(slots=P + 4), dict(dn=None), dict(node=None)):
        assert call(**kw) == EINVAL, kw
    # nothing to move
    for kw in (dict(B=0), dict(planes=0), dict(n=0), dict(row=0), dict(dpar=None)):
        assert call(**kw) == OK, kw


def test_binding_checks_shapes():
    """Host tensors and wrong ranks are refused before the library is called."""
    t = torch.zeros((2, 3, 8))
    i = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError):
        sd.build_logits_args(t, i, None, i[:, 0])
    with pytest.raises(ValueError):
        sd.build_logits_args(t[0], i, None, i[:, 0])
    with pytest.raises(ValueError):
        sd.build_page_args(i[0], None, i[0], 9, 4, i, i[0], i[0], i[0], None, None, i[0])
    with pytest.raises(ValueError):
        sd.switchsd_compact_cache(t, i.long(), i, i[:, 0], i[:, 0])


# ------------------------------------------------------------------ the references

def _one(logits, **kw):
    V = len(logits)
    d = {"logits": torch.tensor(logits).view(1, 1, V), "dtok": np.full((1, 1), -1, np.int32),
         "dpar": None, "dn": np.array([1], np.int32), "tokens": np.zeros((1, 1), np.int32),
         "lengths": np.zeros(1, np.int32), "prompt_lens": None}
    for k in ("repetition", "frequency", "presence", "bias_ids", "bias_vals", "allowed",
              "allowed_on"):
        d[k] = None
    for k, v in kw.items():
        d[k] = np.array(v)
    return d


def test_reference_values():
    """Derived by hand: token 0 twice in the output, 1 in the prompt, 2 on the
    path, 3 untouched, 4 biased twice (the last entry holds), 5 masked."""
    d = _one([2.0, -2.0, 4.0, 1.0, 1.0, 9.0], tokens=[[1, 0, 0, 6, -1]], lengths=[5],
             prompt_lens=[1], repetition=np.array([2.0], np.float32),
             frequency=np.array([0.5], np.float32), presence=np.array([0.25], np.float32),
             bias_ids=[[4, 4, 6]], bias_vals=np.array([[7.0, -3.0, 5.0]], np.float32),
             allowed=np.array([[[0b011111]]], np.uint32))
    d["logits"] = d["logits"].repeat(1, 2, 1)
    d["dtok"], d["dn"] = np.array([[-1, 2]]), np.array([2])
    d["allowed"] = np.repeat(d["allowed"], 2, 1)
    for real in (np.float32, np.float64):
        y = ref.processed(d, real)
        # row 0: 2/2 - 1 - 0.25, -2 * 2, 4 and 1 untouched, 1 - 3, -inf
        assert y[0, 0][0].tolist() == [-0.25, -4.0, 4.0, 1.0, -2.0, -np.inf]
        assert y[0, 1][0].tolist() == [-0.25, -4.0, 1.25, 1.0, -2.0, -np.inf]
    g = ref.greedy(d, ref.processed(d, np.float32))
    assert g["amax"].tolist() == [[2, 2]] and g["accept_len"].tolist() == [1]
    assert g["out_tokens"].tolist() == [[2, 2]] and g["bonus"].tolist() == [2]


def test_reference_plan():
    """Two sequences of pages of 4, one finished; the second does not fit."""
    s = {"B": 3, "R": 2, "Lmax": 64, "page": 4, "dpar": None,
         "lengths": np.array([4, 0, 9]), "dn": np.array([2, 1, 2]),
         "table": np.array([[7, -1, -1], [5, 6, -1], [2, -1, -1]]), "held": np.array([1, 2, 1]),
         "ring": np.array([9, 8, 1, 3]), "ring_state": np.array([3, 2])}
    slots, positions, missing = ref.page_plan(s)
    # free pages: 3, 9; sequence 0 takes page 3, sequence 2 lacks two
    assert s["table"].tolist() == [[7, 3, -1], [-1, -1, -1], [2, -1, -1]]
    assert slots.tolist() == [[31, 12], [-1, -1], [-1, -1]]
    assert positions.tolist() == [[3, 4], [-1, -1], [8, 9]]
    assert missing.tolist() == [0, 0, 2]
    assert s["ring"].tolist() == [9, 5, 6, 3] and s["ring_state"].tolist() == [0, 3]


@pytest.mark.parametrize("t,blk", [(sd.BF16, 8), (sd.F16, 8), (sd.F32, 4)])
def test_logits_work_groups(t, blk):
    """2^24 work-groups or more are refused by the sizes alone, before any HIP
    call: a chunk holds 512 vectors and a work-group up to 64 rows."""
    lib = sd.lib
    size = 4 if t == sd.F32 else 2
    chunk = 512 * blk

    def both(B, R, V):
        a = logits_args(logits_type=t, B=B, R=R, V=V, logits=1 << 20)
        out = (1 << 20) + size * B * R * V + 4096
        need = sd.workspace_bytes(B, R)
        return (lib.switchsd_process_logits(ctypes.byref(a), out, t, None),
                lib.switchsd_verify_processed(ctypes.byref(a), P, P, P, P, P, P, need, None))
    assert both(1 << 24, 1, chunk) == (ESHAPE, ESHAPE)
    assert both(1 << 23, 1, chunk + 1) == (ESHAPE, ESHAPE)
    assert both(1 << 23, 65, chunk) == (ESHAPE, ESHAPE)
    assert both(1 << 16, 1024, chunk) == (ESHAPE, ESHAPE)   # 4 rows a work-group
    assert both(1 << 10, 1, 1 << 26) == (ESHAPE,) * 2       # 2^14 chunks (floats: 2^15)
    assert both(1 << 24, 1024, 1 << 26) == (ESHAPE, ESHAPE)


def test_logits_largest_vocabulary():
    """Offsets in a row are 32 bits wide: V up to 2^26 and no further."""
    lib = sd.lib
    for t in (sd.BF16, sd.F16, sd.F32):
        a = logits_args(logits_type=t, V=(1 << 26) + 1)
        assert lib.switchsd_process_logits(ctypes.byref(a), FAR, t, None) == ESHAPE
        assert lib.switchsd_verify_processed(ctypes.byref(a), P, P, P, P, P, P, 1 << 15,
                                             None) == ESHAPE
        # 2^26 itself: what is refused is a missing output
        a = logits_args(logits_type=t, V=1 << 26)
        assert lib.switchsd_process_logits(ctypes.byref(a), None, t, None) == EINVAL
        assert lib.switchsd_verify_processed(ctypes.byref(a), None, P, P, P, P, P, 1 << 15,
                                             None) == EINVAL


def test_compact_work_groups():
    """A work-group moves 256 pieces of 16 (else 4) bytes of a sequence: 2^24
    work-groups or more are refused."""
    def call(B, planes, row, cache):
        return sd.lib.switchsd_compact_cache(cache, planes, row, 1, row, P, P, P, P, B, 8, None)
    row = 1 << 20
    for size, at in ((16, P), (4, P + 4)):
        many = (1 << 24) // (row // size // 256)
        assert call(1, many, row, at) == ESHAPE
        assert call(many, 1, row, at) == ESHAPE
        assert call(1 << 24, 1, size, at) == ESHAPE
        assert call(1 << 24, 1 << 30, row, at) == ESHAPE
