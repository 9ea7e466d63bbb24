"""Refusals of the operators around the loss pass: every mistake that the host can see becomes a status before a launch."""

import ctypes

import pytest
import torch

from paper_2605_17862_amd import binding as fb

P = ctypes.c_void_p


def test_mx4_sizes():
    # 64 rows and 256 entries: 8192 bytes of codes, 512 of scales
    assert fb.fopd_mx4_bytes(1, 1) == 8704
    assert fb.fopd_mx4_bytes(64, 256) == 8704
    assert fb.fopd_mx4_bytes(65, 257) == 4 * 8704
    assert fb.fopd_mx4_bytes(0, 64) == 0
    assert fb.fopd_mx4_bytes(151936, 4096) == 2374 * 16 * 8704
    assert fb.fopd_mx4_logits_workspace_bytes(45, 151936, 4096) >= 256 + fb.fopd_mx4_bytes(45, 4096)


def test_mx4_rejects_bad_arguments_before_launch():
    lib = fb.load_library()

    def quantize(x=4096, dt=1, R=8, d=64, ld=64, packed=8192, n=1 << 20):
        return lib.fopd_mx4_quantize(P(x), dt, R, d, ld, P(packed), n, None)

    def dequantize(packed=8192, n=1 << 20, R=8, d=64, out=4096, dt=1, ldo=64):
        return lib.fopd_mx4_dequantize(P(packed), n, R, d, P(out), dt, ldo, None)

    for call in (quantize, dequantize):
        assert call(packed=None) == 1
        assert call(packed=8192 + 8) == 3
        assert call(R=-1) == 2
        assert call(d=0) == 2
        assert call(d=(1 << 24) + 8, **{"ld" if call is quantize else "ldo": 1 << 25}) == 2
        assert call(dt=2) == 4
        assert call(n=fb.fopd_mx4_bytes(8, 64) - 1) == 5
        assert call(R=0) == 0
    assert quantize(x=None) == 1
    assert quantize(ld=56) == 2
    assert quantize(d=60, ld=60) == 3
    assert quantize(x=4096 + 4) == 3
    assert dequantize(out=None) == 1
    assert dequantize(ldo=60) == 2

    def logits(h=4096, dth=1, ldh=64, w=8192, wn=1 << 20, T=8, V=100, d=64, z=16384, dt=0, ld=100, ws=4096, wsn=1 << 20):
        return lib.fopd_mx4_logits(P(h), dth, ldh, P(w), wn, T, V, d, P(z), dt, ld, P(ws), wsn, None)

    assert logits(h=None) == 1
    assert logits(w=None) == 1
    assert logits(z=None) == 1
    assert logits(dth=7) == 4
    assert logits(dt=-1) == 4
    assert logits(T=-1) == 2
    assert logits(V=0) == 2
    assert logits(ldh=32) == 2
    assert logits(ld=96) == 2
    assert logits(ld=101) == 3
    assert logits(w=8192 + 4) == 3
    assert logits(V=(1 << 28) + 64, ld=(1 << 28) + 64, wn=1 << 62) == 2
    assert logits(wn=fb.fopd_mx4_bytes(100, 64) - 1) == 5
    assert logits(ws=None) == 5
    assert logits(ws=4096 + 16) == 5
    assert logits(wsn=fb.fopd_mx4_logits_workspace_bytes(8, 100, 64) - 1) == 5
    assert logits(T=0) == 0


def test_mx4_calls_without_rows_need_no_buffers():
    """Empty tensors have no address; sizes and types are looked at all the same."""
    lib = fb.load_library()

    def quantize(dt=1, d=64, ld=64):
        return lib.fopd_mx4_quantize(None, dt, 0, d, ld, None, 0, None)

    def dequantize(dt=1, d=64, ld=64):
        return lib.fopd_mx4_dequantize(None, 0, 0, d, None, dt, ld, None)

    def logits(dt=1, d=64, ld=64, dtz=0, V=100, ldz=100, w=8192, wn=1 << 20):
        return lib.fopd_mx4_logits(None, dt, ld, P(w), wn, 0, V, d, None, dtz, ldz, None, 0, None)

    for call in (quantize, dequantize, logits):
        assert call() == 0
        assert call(dt=2) == 4
        assert call(d=0) == 2
        assert call(ld=63) == 2
        assert call(d=(1 << 24) + 8, ld=1 << 25) == 2
    assert logits(dtz=7) == 4
    assert logits(V=0) == 2
    assert logits(ldz=99) == 2
    assert logits(V=(1 << 28) + 64, ldz=1 << 29) == 2


def _verify(lib, **kw):
    a = dict(z=4096, zd=8192, dt=1, R=8, V=64, ld=64, ldd=64, ids=4096, row=None, lens=None, B=2, K=3, tau=None, u=4096, e=4096,
             lde=64, n=4096, oi=4096, ol=4096, om=4096, ws=4096, wsn=1 << 22)
    a.update(kw)
    return lib.fopd_verify_draft(P(a["z"]), P(a["zd"]), a["dt"], a["R"], a["V"], a["ld"], a["ldd"], P(a["ids"]), P(a["row"]),
                                 P(a["lens"]), a["B"], a["K"], P(a["tau"]), P(a["u"]), P(a["e"]), a["lde"], P(a["n"]), P(a["oi"]),
                                 P(a["ol"]), P(a["om"]), P(a["ws"]), a["wsn"], None)


def test_verification_rejects_bad_arguments_before_launch():
    lib = fb.load_library()
    assert _verify(lib, z=None) == 1
    assert _verify(lib, ids=None) == 1
    assert _verify(lib, u=None) == 1                              # one of the two kinds of variates alone
    assert _verify(lib, e=None) == 1
    for out in ("n", "oi", "ol", "om"):
        assert _verify(lib, **{out: None}) == 1
    assert _verify(lib, dt=3) == 4
    assert _verify(lib, V=0) == 2
    assert _verify(lib, B=0) == 2
    assert _verify(lib, K=-1) == 2
    assert _verify(lib, K=1024, R=1 << 20) == 2
    assert _verify(lib, R=7) == 2                                 # a padded batch of 2 x 4 rows
    assert _verify(lib, R=0) == 2
    assert _verify(lib, B=1 << 19, K=2, R=1 << 22) == 2           # more than 2^20 places
    assert _verify(lib, ld=56) == 2
    assert _verify(lib, ldd=56) == 2
    assert _verify(lib, lde=60) == 2
    assert _verify(lib, lde=66) == 3
    assert _verify(lib, e=4096 + 4) == 3
    assert _verify(lib, zd=8192 + 2) == 3
    assert _verify(lib, ws=None) == 5
    assert _verify(lib, ws=4096 + 64) == 5
    need = fb.fopd_verify_workspace_bytes(8, 64, 2)
    assert need % 256 == 0 and _verify(lib, wsn=need - 1) == 5


@pytest.mark.parametrize("V", [1, 4095, 4096, 8191, 8192, 32000, 151936, 262144])
def test_a_workspace_for_a_verification_serves_every_smaller_one(V):
    """Around the row counts where a row is cut into half as many pieces, and over all sizes in between."""
    sizes = sorted({max(1, n + k) for n in [1 << e for e in range(17)] + [248, 1016, 1536] for k in (-1, 0, 1)})
    need = [fb.fopd_verify_workspace_bytes(R, V, 5) for R in sizes]
    assert need == sorted(need)
    need = [fb.fopd_verify_workspace_bytes(1000, V, B) for B in sizes]
    assert need == sorted(need)
    need = [fb.fopd_verify_workspace_bytes(R, v, 5) for R in (1, 2, 31, 33, 1023) for v in (V // 2 + 1, V, V + 1, 2 * V)]
    assert all(need[k:k + 4] == sorted(need[k:k + 4]) for k in range(0, len(need), 4))
    # a ragged batch of fewer samples, as the rollouts end
    assert max(fb.fopd_verify_workspace_bytes(8 * B, V, B) for B in range(1, 257)) == fb.fopd_verify_workspace_bytes(2048, V, 256)


def test_rows_whose_last_places_do_not_fit_32_bits_are_refused():
    """A workgroup forms the places behind a row's last vector, as many as it has lanes: they have to stay below 2^31."""
    lib = fb.load_library()
    most = (1 << 31) - 512
    for V in ((1 << 31) - 17, (1 << 31) - 256, most + 1):
        assert _verify(lib, V=V, ld=1 << 31, ldd=1 << 31, lde=1 << 31) == 2
        assert lib.fopd_token_logprobs(P(4096), 1, 1, V, 1 << 31, P(4096), None, P(4096), P(4096), None, None, P(4096), 0, None) == 2
        assert lib.fopd_mx4_dequantize(P(4096), 1 << 40, 1, V, P(4096), 1, 1 << 31, None) == 2
    assert _verify(lib, V=most, ld=1 << 31, ldd=1 << 31, lde=1 << 31, ws=None) == 5
    assert lib.fopd_token_logprobs(P(4096), 1, 1, most, 1 << 31, P(4096), None, P(4096), P(4096), None, None, P(4096), 0, None) == 5


def test_status_of_a_row_without_a_distribution():
    assert fb.fopd_flags_status(16) == 12
    assert fb.fopd_flags_status(17) == 6
    assert fb.fopd_status_string(12) != "unknown status"


def _entry(**kw):
    a = dict(grad=4096, out=4096, rows=1, cols=64, ld=64, ld_out=64, dt=0, dt_out=0)
    a.update(kw)
    return fb.GradTensor(*[a[k] for k, _ in fb.GradTensor._fields_])


def test_gradient_calls_reject_bad_arguments_before_launch():
    lib = fb.load_library()

    def norm(entries, n=None, s=4096, ws=4096, wsn=1 << 20):
        arr = (fb.GradTensor * len(entries))(*entries)
        return lib.fopd_grad_norm(ctypes.cast(arr, P), len(entries) if n is None else n, 0, P(s), None, P(ws), wsn, None)

    def clip(entries, n=None, s=4096, most=1.0, eps=1e-6):
        arr = (fb.GradTensor * len(entries))(*entries)
        return lib.fopd_grad_clip(ctypes.cast(arr, P), len(entries) if n is None else n, P(s), most, eps, None, None)

    good = _entry()
    for call in (norm, clip):
        assert call([good], n=-1) == 2
        assert call([good], s=None) == 1
        assert call([good, _entry(grad=None)]) == 1
        assert call([good, _entry(dt=2)]) == 4
        assert call([_entry(rows=2, ld=63)]) == 2
        assert call([_entry(rows=-1)]) == 2
        assert call([_entry(cols=1 << 41, ld=1 << 41)]) == 2
        assert call([_entry(rows=1 << 39, cols=1 << 39, ld=1 << 39)]) == 2
        assert call([_entry(rows=1 << 62, cols=4, ld=4)]) == 2
        assert call([_entry(grad=4096 + 2, out=8192)]) == 3
    assert lib.fopd_grad_norm(None, 1, 0, P(4096), None, P(4096), 1 << 20, None) == 1
    assert lib.fopd_grad_clip(None, 1, P(4096), 1.0, 0.0, None, None) == 1
    assert norm([good], ws=None) == 5
    assert norm([good], ws=4096 + 8) == 5
    assert norm([good], wsn=fb.fopd_grad_workspace_bytes() - 1) == 5
    assert clip([_entry(out=None)]) == 1
    assert clip([_entry(dt_out=5)]) == 4
    assert clip([_entry(dt_out=1)]) == 1                          # in place, of another type
    assert clip([_entry(rows=2, ld=64, ld_out=72)]) == 1          # in place, of another pitch
    assert clip([_entry(out=8192, rows=2, ld_out=60)]) == 2
    assert clip([_entry(out=8193, dt_out=1)]) == 3
    for bad in (-1.0, float("nan")):
        assert clip([good], most=bad) == 1
        assert clip([good], eps=bad) == 1


def test_gradient_list_refuses_what_it_cannot_describe():
    for grads, outs in (([torch.zeros(4)], None),                                       # host memory
                        ([torch.zeros(4, dtype=torch.float16)], None)):
        with pytest.raises(ValueError):
            fb.grad_tensors(grads, outs)
    with pytest.raises(ValueError):
        fb.grad_tensors([torch.zeros(4)], [])


class _OnDevice:
    """What the binding looks at of a tensor."""
    is_cuda = True

    def __init__(self, dtype, contiguous=True):
        self.dtype, self.contiguous = dtype, contiguous

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 4096

    def numel(self):
        return 1 << 20

    def element_size(self):
        return self.dtype.itemsize


def test_matrices_of_another_type_than_named_and_packed_ones_elsewhere_are_refused():
    """Read as the wider type a matrix would be run past; a packed weight in host memory is no address for the device."""
    f32, bf16, host = _OnDevice(torch.float32), _OnDevice(torch.bfloat16), torch.zeros(1 << 16, dtype=torch.uint8)
    packed, ws = _OnDevice(torch.uint8), (4096, 1 << 20)

    def verify(target, draft, dt):
        fb.fopd_verify_draft(target, draft, dt, 8, 64, 64, 64, 4096, None, None, 2, 3, None, 4096, 4096, 64, 4096, 4096, 4096, 4096, ws, stream=0)

    def logits(h, dth, w, z, dt):
        fb.fopd_mx4_logits(h, dth, 64, w, 8, 100, 64, z, dt, 104, ws, stream=0)

    for call in (lambda: verify(f32, bf16, fb.FOPD_F32), lambda: verify(f32, bf16, fb.FOPD_BF16), lambda: verify(bf16, None, fb.FOPD_F32),
                 lambda: fb.fopd_mx4_quantize(bf16, fb.FOPD_F32, 8, 64, 64, packed, stream=0),
                 lambda: fb.fopd_mx4_quantize(bf16, fb.FOPD_BF16, 8, 64, 64, host, stream=0),
                 lambda: fb.fopd_mx4_quantize(bf16, fb.FOPD_BF16, 8, 64, 64, _OnDevice(torch.uint8, False), stream=0),
                 lambda: fb.fopd_mx4_dequantize(packed, 8, 64, bf16, fb.FOPD_F32, 64, stream=0),
                 lambda: fb.fopd_mx4_dequantize(host, 8, 64, bf16, fb.FOPD_BF16, 64, stream=0),
                 lambda: logits(bf16, fb.FOPD_F32, packed, f32, fb.FOPD_F32), lambda: logits(bf16, fb.FOPD_BF16, packed, bf16, fb.FOPD_F32),
                 lambda: logits(bf16, fb.FOPD_BF16, host, f32, fb.FOPD_F32)):
        with pytest.raises(ValueError):
            call()
    # the library's own refusals are still reached: a type that does not exist, a missing matrix
    for call, status in ((lambda: verify(f32, f32, 5), 4), (lambda: verify(None, None, fb.FOPD_F32), 1)):
        with pytest.raises(fb.FopdError) as refused:
            call()
        assert refused.value.status == status
