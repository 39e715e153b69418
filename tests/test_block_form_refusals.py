"""Pointers that the calls beyond the causal Llama form have to refuse before anything is launched: without a GPU, on a context that no
call may get as far as using."""
import ctypes as C

import pytest
import torch

from paper_2603_22370_b200 import build as faar_build
from paper_2603_22370_b200 import faar

AT = 1 << 20                                                   # an address that is aligned to anything; never followed
ODD = AT + 2


@pytest.fixture(scope="module")
def refused():
    faar_build.build()
    lib = faar.lib()
    blank = C.create_string_buffer(b"\x7f" * 4096, 4096)      # no such device: a call that is not refused fails there

    def status(name, *args):
        return getattr(lib, name)(C.addressof(blank), *args)

    return status


def with_one_odd(args, which):
    return [ODD if i == which else a for i, a in enumerate(args)]


@pytest.mark.parametrize("name,args,words", [
    ("faar_layernorm", (4, 64, AT, 64, AT, AT, 1e-5, AT, 64, AT, AT), (9, 10)),
    ("faar_add_layernorm", (4, 64, AT, 64, AT, 64, AT, 64, AT, AT, 1e-5, AT, 64, AT, AT), (13, 14)),
    ("faar_layernorm_bwd", (4, 64, AT, 64, AT, 64, AT, AT, AT, None, 0, AT, 64, None, None, None, 0), (7, 8)),
    ("faar_rope_axes", (4, 1, 64, AT, 64, AT, "axes", 1e4, 0, AT, 64), (5,)),
    ("faar_attention_scored_fwd", (1, 8, 1, 1, 64, AT, 64, 2 * AT, 3 * AT, 64, "scores", 4 * AT, 64, AT), (13,)),
    ("faar_attention_scored_bwd", (1, 8, 1, 1, 64, AT, 64, 2 * AT, 3 * AT, 64, "scores", 4 * AT, 5 * AT, 64, AT, AT, 1 << 20, 6 * AT, 7 * AT, 8 * AT), (14,)),
    ("faar_attention_ranges", (1, 8, AT, 2 * AT, 3 * AT, 4 * AT), (2, 3, 4, 5))])
def test_words_that_are_not_aligned_are_refused(refused, name, args, words):
    structs = {"axes": faar.make_rope_axes([16, 8, 8]), "scores": faar.make_attention_scores()}
    args = [C.byref(structs[a]) if isinstance(a, str) else a for a in args]
    assert refused(name, *args) == faar.ERR_CUDA               # nothing else is wrong: it gets to the device that is not there
    for i in words:
        assert refused(name, *with_one_odd(args, i)) == faar.ERR_ALIGN, i


class DeviceTensor:
    """What the marshalling asks a tensor for."""
    is_cuda = True

    def __init__(self, dtype):
        self.dtype = dtype

    def data_ptr(self):
        return AT


INT_CALLS = [("faar_attention_ranges", (1, 8, "int", 2 * AT, 3 * AT, 4 * AT)), ("faar_attention_ranges", (1, 8, 2 * AT, "int", 3 * AT, 4 * AT)),
             ("faar_attention_ranges", (1, 8, None, None, 3 * AT, "int")), ("faar_rope_axes", (4, 1, 64, AT, 64, "int", "axes", 1e4, 0, AT, 64)),
             ("faar_rope", (4, 1, 64, AT, 64, "int", 1e4, 0, AT, 64)), ("faar_embedding", (4, 64, 100, AT, 64, "int", AT, 64))]


@pytest.mark.parametrize("name,args", INT_CALLS)
def test_ids_and_positions_of_another_type_are_refused(name, args):
    """64-bit ones would be read as twice as many of 32 bits."""
    faar_build.build()
    blank = C.create_string_buffer(b"\x7f" * 4096, 4096)

    def status(dtype):
        return getattr(faar._fast(), name)(C.addressof(blank), *({"int": DeviceTensor(dtype), "axes": faar.make_rope_axes([16, 8, 8])}.get(a, a)
                                                                 if isinstance(a, str) else a for a in args))

    assert status(torch.int32) == faar.ERR_CUDA                # nothing is wrong: it gets to the device that is not there
    for dtype in (torch.int64, torch.int16, torch.uint8, torch.bool, torch.float32):
        with pytest.raises(AssertionError):
            status(dtype)


MB = 1 << 20
FWD = dict(batch=1, seq=64, n_heads=2, n_kv_heads=1, head_dim=64, q=1 * MB, ldq=128, k=2 * MB, v=3 * MB, ldkv=64, scores={}, out=4 * MB, ldo=128, lse=5 * MB)
BWD = dict(batch=1, seq=64, n_heads=2, n_kv_heads=1, head_dim=64, q=1 * MB, ldq=128, k=2 * MB, v=3 * MB, ldkv=64, scores={}, out=4 * MB, dout=6 * MB, ldo=128,
           lse=5 * MB, scratch=7 * MB, scratch_bytes=64 * 2 * 4 + 16, dq=8 * MB, dk=9 * MB, dv=10 * MB)
INF, NAN = float("inf"), float("nan")
SHARED = [(dict(head_dim=32), faar.ERR_SHAPE), (dict(head_dim=256, ldq=512, ldo=512, ldkv=256), faar.ERR_SHAPE), (dict(n_heads=3, n_kv_heads=2, ldq=192, ldo=192, ldkv=128), faar.ERR_SHAPE),
          (dict(batch=0), faar.ERR_SHAPE), (dict(seq=0), faar.ERR_SHAPE), (dict(n_heads=0), faar.ERR_SHAPE), (dict(n_kv_heads=0), faar.ERR_SHAPE),
          (dict(batch=1 << 20, seq=1 << 20), faar.ERR_SHAPE), (dict(batch=1 << 29, seq=1), faar.ERR_SHAPE), (dict(seq=(1 << 30) + 1), faar.ERR_SHAPE),
          (dict(ldq=64), faar.ERR_SHAPE), (dict(ldo=64), faar.ERR_SHAPE), (dict(ldkv=56), faar.ERR_SHAPE), (dict(ldq=132), faar.ERR_ALIGN), (dict(ldo=132), faar.ERR_ALIGN),
          (dict(ldkv=68), faar.ERR_ALIGN)]
SHARED += [({p: None}, faar.ERR_INVALID_ARG) for p in ("q", "k", "v", "scores", "out", "lse")]
SHARED += [({p: FWD[p] + 8}, faar.ERR_ALIGN) for p in ("q", "k", "v", "out")]
SHARED += [(dict(scores=s), faar.ERR_INVALID_ARG) for s in (dict(scale=-1.0), dict(scale=INF), dict(scale=NAN), dict(softcap=-1.0), dict(softcap=INF), dict(softcap=NAN))]
SHARED += [(dict(scores={p: AT + 2}), faar.ERR_ALIGN) for p in ("slopes", "key_lo", "key_hi")]
OVER = [(dict(out=FWD[p] + 64 * shift), faar.ERR_INVALID_ARG) for p in ("q", "k", "v") for shift in (0, 1)]
BACK = [({p: None}, faar.ERR_INVALID_ARG) for p in ("dout", "dq", "dk", "dv")] + [({p: BWD[p] + 8}, faar.ERR_ALIGN) for p in ("dout", "dq", "dk", "dv")]
BACK += [(dict(scratch=None), faar.ERR_WORKSPACE), (dict(scratch=7 * MB + 8), faar.ERR_WORKSPACE), (dict(scratch_bytes=64 * 2 * 4 + 15), faar.ERR_WORKSPACE)]
BACK += [({p: BWD[o]}, faar.ERR_INVALID_ARG) for p in ("dq", "dk", "dv") for o in ("q", "k", "v", "dout")]
BACK += [(dict(dk=8 * MB), faar.ERR_INVALID_ARG), (dict(dv=8 * MB), faar.ERR_INVALID_ARG), (dict(dv=9 * MB), faar.ERR_INVALID_ARG)]


@pytest.mark.parametrize("name,base,changes", [("faar_attention_scored_fwd", FWD, SHARED + OVER), ("faar_attention_scored_bwd", BWD, SHARED + BACK)])
def test_attention_over_ranges_refuses_one_wrong_argument_at_a_time(refused, name, base, changes):
    """The call that is changed in one place is a good one: it gets as far as the device."""
    def status(**change):
        a = {**base, **change}
        if a["scores"] is not None:
            s = faar.AttentionScores(0.0, 0.0, None, None, None)
            for key, value in a["scores"].items():
                setattr(s, key, value)
            a["scores"] = C.byref(s)
        return refused(name, *a.values())

    assert status() == faar.ERR_CUDA
    assert status(scores=dict(scale=0.5, softcap=30.0, slopes=AT, key_lo=AT, key_hi=AT)) == faar.ERR_CUDA
    for change, want in changes:
        assert status(**change) == want, change


@pytest.mark.parametrize("name,base", [("faar_attention_scored_fwd", FWD), ("faar_attention_scored_bwd", BWD)])
def test_scales_and_caps_whose_factors_are_no_normal_floats_are_refused(refused, name, base):
    """scale log2(e), softcap log2(e) and scale / softcap are what the kernels multiply scores by: infinite, a score of 0 would be no number,
    and below the normal range they have no digits left."""
    least, most = 2.0 ** -126, (2 - 2.0 ** -23) * 2.0 ** 127
    LOG2E = 1.4426950408889634

    def status(scale, softcap):
        s = faar.AttentionScores(scale, softcap, None, None, None)
        return refused(name, *{**base, "scores": C.byref(s)}.values())

    for scale, softcap in [(most, 0.0), (0.7 * most, 0.0), (least / 2, 0.0), (0.0, most), (0.0, 0.7 * most), (0.0, least / 2), (0.0, 2.0 ** 123 * 1.01),
                           (2.0 ** 64, 2.0 ** -64), (2.0 ** -64, 2.0 ** 63), (0.0, 2.0 ** -131)]:
        assert status(scale, softcap) == faar.ERR_INVALID_ARG, (scale, softcap)
    for scale, softcap in [(0.69 * most, 0.0), (least, 0.0), (0.0, 2.0 ** 123), (2.0 ** 63, 2.0 ** -64), (2.0 ** -64, 2.0 ** 62), (0.0, 2.0 ** -126), (0.0, 50.0)]:
        assert status(scale, softcap) == faar.ERR_CUDA, (scale, softcap)
    assert 0.69 * LOG2E < 1 < 0.7 * LOG2E
