"""Refusals of the operators on a served batch: what the calls check on the host, before any device is
touched.  Addresses are made up; nothing is read through them."""
import ctypes as C
import math
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20                       # an aligned address


@pytest.fixture(scope="module")
def td():
    from paper_2507_19017_b200 import build, binding
    build.build()
    return binding


def batch(td, **kw):
    v = dict(max_samples=4, cu_prompt=A, cu_response=A, result=None)
    v.update(kw)
    return C.pointer(td.TdBatch(v["max_samples"], 0, v["cu_prompt"], v["cu_response"], v["result"]))


def logits(td, **kw):
    v = dict(logits=A, logits_stride=100, dtype=td.BF16, vocab=100, n_rows=8, n_tokens=8, rows=td.ROWS_TOKEN,
             temperature=1.0, device=0, targets=A, batch=None)
    v.update({k: x for k, x in kw.items() if k in v})
    return v


def logprob(td, **kw):
    v = dict(logits(td, **kw), logprob=A, norm=A, entropy=A, entropy_bf16=A, status=A)
    v.update(kw)
    return td.lib().td_token_logprob(td.TdLogprobArgs(**v), None)


def logprob_grad(td, **kw):
    v = dict(logits(td, **kw), norm=A, entropy=A, grad_logprob=A, grad_entropy=A, grad_logits=2 * A, grad_stride=100, status=A)
    v.update(kw)
    return td.lib().td_token_logprob_grad(td.TdLogprobGradArgs(**v), None)


COMMON = [dict(dtype=0), dict(dtype=7), dict(vocab=0), dict(vocab=2 ** 31), dict(logits_stride=-1), dict(temperature=0.0),
          dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf), dict(temperature=1e-45),
          dict(rows=2), dict(n_rows=7), dict(rows=1), dict(logits=None), dict(targets=None), dict(logits=A + 1),
          dict(targets=A + 2), dict(status=A + 1), dict(n_tokens=2 ** 31, n_rows=2 ** 31 + 1)]


@pytest.mark.parametrize("bad", COMMON + [dict(logprob=None), dict(logprob=A + 2), dict(norm=A + 1), dict(entropy=A + 2), dict(entropy_bf16=A + 1)], ids=str)
def test_token_logprob_refuses(td, bad):
    assert logprob(td, **bad) == td.EINVAL


@pytest.mark.parametrize("bad", COMMON + [
    dict(grad_logits=None), dict(grad_logits=A + 1), dict(grad_stride=99), dict(grad_logits=A, grad_stride=104), dict(norm=None),
    dict(grad_logprob=None, grad_entropy=None), dict(entropy=None), dict(grad_logprob=A + 1), dict(grad_entropy=A + 2)], ids=str)
def test_token_logprob_grad_refuses(td, bad):
    assert logprob_grad(td, **bad) == td.EINVAL


@pytest.mark.parametrize("bad", [dict(cu_response=None), dict(cu_prompt=None), dict(cu_prompt=A + 2), dict(result=A + 4), dict(max_samples=2 ** 31)], ids=str)
def test_stream_rows_need_a_whole_batch(td, bad):
    assert logprob(td, rows=td.ROWS_STREAM, batch=batch(td, **bad)) == td.EINVAL
    assert logprob_grad(td, rows=td.ROWS_STREAM, batch=batch(td, **bad)) == td.EINVAL


def policy(td, **kw):
    v = dict(batch=batch(td), n_tokens=40, row_width=0, column_dtype=td.F32, kl_kind=td.KL_K3, reduction=td.MEAN_TOKENS, device=0,
             clip_low=0.2, clip_high=0.2, dual_clip=0.0, kl_coef=0.1, entropy_coef=0.1, norm=0.0, grad_scale=1.0, reserved=0, logprob=A,
             old_logprob=A, ref_logprob=A, entropy=A, mask=A, advantages=A, grad_logprob=A, grad_entropy=A, stats=A, workspace=A,
             workspace_bytes=td.lib().td_policy_loss_workspace_bytes(4))
    v.update(kw)
    return td.lib().td_policy_loss(td.TdPolicyArgs(**v), None)


@pytest.mark.parametrize("bad", [
    dict(batch=None), dict(n_tokens=2 ** 31), dict(row_width=9), dict(row_width=2 ** 31, n_tokens=2 ** 33), dict(column_dtype=0),
    dict(column_dtype=3), dict(kl_kind=0), dict(kl_kind=4), dict(reduction=2), dict(clip_low=-0.1), dict(clip_low=1.5),
    dict(clip_low=math.nan), dict(clip_high=-1.0), dict(dual_clip=0.5), dict(dual_clip=math.nan), dict(norm=-1.0), dict(norm=math.inf),
    dict(kl_coef=math.nan), dict(entropy_coef=math.inf), dict(grad_scale=math.nan), dict(stats=None), dict(logprob=None),
    dict(advantages=None), dict(grad_logprob=None), dict(logprob=A + 2), dict(old_logprob=A + 2), dict(ref_logprob=A + 1),
    dict(entropy=A + 1), dict(advantages=A + 1), dict(grad_logprob=A + 1), dict(grad_entropy=A + 2), dict(stats=A + 1)], ids=str)
def test_policy_loss_refuses(td, bad):
    assert policy(td, **bad) == td.EINVAL


def test_policy_loss_checks_its_batch_and_workspace(td):
    assert policy(td, batch=batch(td, cu_response=None)) == td.EINVAL
    need = td.lib().td_policy_loss_workspace_bytes(4)
    assert policy(td, workspace=None) == td.EWORKSPACE
    assert policy(td, workspace=A + 128) == td.EWORKSPACE
    assert policy(td, workspace_bytes=need - 1) == td.EWORKSPACE
    assert policy(td, batch=batch(td, max_samples=4096)) == td.EWORKSPACE
    assert td.lib().td_policy_loss_workspace_bytes(4096) > need


def embed(td, **kw):
    v = dict(ids=A, n_tokens=8, vocab=50, dim=16, dtype=td.BF16, table=A, table_stride=16, out=2 * A, out_stride=16, scale=1.0,
             tokens=td.TOKENS_SEQ, device=0, reserved=0, batch=None, status=A)
    v.update(kw)
    return td.lib().td_embed(td.TdEmbedArgs(**v), None)


def embed_grad(td, **kw):
    v = dict(ids=A, n_tokens=8, vocab=50, dim=16, dtype=td.BF16, grad_out=A, out_stride=16, grad_dtype=td.F32, accumulate=0,
             grad_table=2 * A, table_stride=16, scale=1.0, tokens=td.TOKENS_SEQ, device=0, reserved=0, batch=None, workspace=A,
             workspace_bytes=td.lib().td_embed_grad_workspace_bytes(8, 50, 16), status=A)
    v.update(kw)
    return td.lib().td_embed_grad(td.TdEmbedGradArgs(**v), None)


EMBED = [dict(dtype=0), dict(dtype=9), dict(vocab=0), dict(dim=0), dict(vocab=2 ** 31), dict(dim=2 ** 31), dict(n_tokens=2 ** 31),
         dict(table_stride=15), dict(ids=None), dict(ids=A + 2), dict(status=A + 2)]


@pytest.mark.parametrize("bad", EMBED + [dict(out_stride=15), dict(table=None), dict(out=None), dict(table=A + 1), dict(out=A + 1)], ids=str)
def test_embed_refuses(td, bad):
    assert embed(td, **bad) == td.EINVAL


@pytest.mark.parametrize("bad", EMBED + [dict(out_stride=-16), dict(grad_dtype=3), dict(accumulate=2),
                                         dict(grad_table=None), dict(grad_out=None), dict(grad_table=A + 2), dict(grad_out=A + 1)], ids=str)
def test_embed_grad_refuses(td, bad):
    assert embed_grad(td, **bad) == td.EINVAL


@pytest.mark.parametrize("call", [embed, embed_grad])
def test_embed_checks_its_batch(td, call):
    for tokens, b in ((0, {}), (4, {}), (td.TOKENS_PROMPT, dict(cu_prompt=None)), (td.TOKENS_RESPONSE, dict(cu_response=None)),
                      (td.TOKENS_SEQ, dict(cu_prompt=None)), (td.TOKENS_SEQ, dict(cu_response=A + 1))):
        assert call(td, tokens=tokens, batch=batch(td, **b)) == td.EINVAL


def test_embed_grad_checks_its_workspace(td):
    need = td.lib().td_embed_grad_workspace_bytes(8, 50, 16)
    assert embed_grad(td, workspace=None) == td.EWORKSPACE
    assert embed_grad(td, workspace=A + 64) == td.EWORKSPACE
    assert embed_grad(td, workspace_bytes=need - 1) == td.EWORKSPACE
    assert td.lib().td_embed_grad_workspace_bytes(10 ** 6, 50, 16) > td.lib().td_embed_grad_workspace_bytes(10 ** 5, 50, 16) > need > 0
    assert td.lib().td_embed_grad_workspace_bytes(2 ** 31, 50, 16) == 0


def test_null_arguments_and_empty_calls(td):
    L = td.lib()
    for name in ("td_token_logprob", "td_token_logprob_grad", "td_policy_loss", "td_embed", "td_embed_grad"):
        assert getattr(L, name)(None, None) == td.EINVAL
    assert logprob(td, n_tokens=0, n_rows=0, logits=None, targets=None, logprob=None) == td.OK       # nothing to do, no device needed
    assert logprob_grad(td, n_tokens=0, n_rows=0, logits=None, targets=None, grad_logits=None) == td.OK
    assert embed(td, n_tokens=0, ids=None, out=None) == td.OK


def test_a_call_without_a_device_says_so(td):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for call in (logprob, logprob_grad, policy, embed, embed_grad):
        assert call(td) == td.ECUDA


def test_operator_struct_layouts_match_the_header(td, tmp_path):
    names = {"td_batch": td.TdBatch, "td_logprob_args": td.TdLogprobArgs, "td_logprob_grad_args": td.TdLogprobGradArgs,
             "td_policy_args": td.TdPolicyArgs, "td_embed_args": td.TdEmbedArgs, "td_embed_grad_args": td.TdEmbedGradArgs}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "td.h"', "int main(void) {"]
    for n, s in names.items():
        lines.append(f'printf("%zu\\n", sizeof({n}));')
        lines += [f'printf("%zu\\n", offsetof({n}, {f[0]}));' for f in s._fields_]
    (tmp_path / "o.c").write_text("\n".join(lines + ["return 0; }"]))
    exe = tmp_path / "o"
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(tmp_path / "o.c")])
    got = list(map(int, subprocess.check_output([str(exe)]).split()))
    want = [v for s in names.values() for v in [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]]
    assert got == want


def test_binding_refuses_what_is_not_on_a_device(td):
    import torch
    x, y = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        td.token_logprob_grad(x, x, y, x, x)
    with pytest.raises(ValueError):
        td.embed(x, y, x)
    with pytest.raises(ValueError):
        td.embed_grad(x, y, x, None)
    with pytest.raises(ValueError):
        td.Batch(None, None)
    with pytest.raises(ValueError):
        td.Batch(None, y)


def test_operator_kernels_do_not_read_through_the_read_only_path():
    """That path (__ldg, ld.global.nc) is defined only for memory nothing writes while the kernel runs; these kernels
    are let in while the one ahead of them, which may write their operands, is still running."""
    csrc = os.path.join(ROOT, "paper_2507_19017_b200", "csrc")
    for name in ("td_ops.cu", "td_ops.cuh", "td_logprob.cuh", "td_policy.cuh", "td_embed.cuh"):
        with open(os.path.join(csrc, name)) as f:
            code = "\n".join(line.split("//")[0] for line in f)
        assert "__ldg" not in code and "global.nc" not in code and "tex." not in code, name


def thresholds(vocab, dim):
    """Numbers of positions around which the call's layout changes: chunks of the sums double, tiles of the sort grow."""
    slices = -(-dim // 256)
    at = {1, 8, 100, 2400, 8192, 2 ** 17, 2 ** 20, 3 * 10 ** 6}
    for r in (8, 16, 32, 64, 128, 256, 512):
        at.add(r * 148 * 64 // slices)
    return sorted({n + k for n in at for k in (-1, 0, 1, 2, 500) if n + k >= 0})


@pytest.mark.parametrize("vocab", [1, 511, 512, 32003, 129280, 2 ** 20])
def test_embed_grad_workspace_holds_for_every_smaller_call(td, vocab):
    """The size never falls as positions, vocabulary or columns grow."""
    size = td.lib().td_embed_grad_workspace_bytes
    dims = [1, 23, 255, 256, 257, 512, 1001, 1024, 2048, 4096, 5000, 8192, 70000]
    last = None
    for dim in dims:
        at = thresholds(vocab, dim)
        now = [size(n, vocab, dim) for n in at]
        assert all(a <= b for a, b in zip(now, now[1:])), dim
        assert all(size(n, v, dim) <= size(n, vocab, dim) for n in at[::7] for v in (1, 500, vocab // 2 + 1) if v <= vocab)
        common = [size(n, vocab, dim) for n in thresholds(vocab, 2048)]
        assert last is None or all(a <= b for a, b in zip(last, common)), dim
        last = common


def test_embed_grad_takes_a_larger_calls_workspace(td):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    room = td.lib().td_embed_grad_workspace_bytes(65536, 129280, 2048)
    for n in (37888, 37000, 9472, 8700, 20000, 65535, 1):
        assert embed_grad(td, n_tokens=n, vocab=129280, dim=2048, table_stride=2048, out_stride=2048, workspace_bytes=room) == td.ECUDA, n


class OnDevice:
    """What the binding asks of a tensor, for one that would be on a device."""

    def __init__(self, dtype, *shape, device=0):
        self.dtype, self.shape, self.device = dtype, shape, device

    def get_device(self):
        return self.device

    def stride(self):
        return (self.shape[1], 1) if len(self.shape) == 2 else (1,)

    def numel(self):
        return math.prod(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return A


def test_embed_grad_refuses_a_workspace_on_another_device(td):
    import torch
    ws = object.__new__(td.EmbedGradWorkspace)
    ws.device, ws.address, ws.nbytes = 1, A, td.lib().td_embed_grad_workspace_bytes(8, 50, 16)
    ids, grad, table = OnDevice(torch.int32, 8), OnDevice(torch.float32, 8, 16), OnDevice(torch.float32, 50, 16)
    with pytest.raises(ValueError, match="workspace"):
        td.embed_grad(table, ids, grad, ws, stream=0)
