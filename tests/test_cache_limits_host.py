"""What attention over a cache takes less of than the other calls on it is said where it is refused (no device is touched)."""
import pytest

from tests.test_cache_host import OnDevice, attend, some_cache, td  # noqa: F401


class Sized(OnDevice):
    def element_size(self):
        return 2


@pytest.mark.parametrize("dim", [0, 4, 12, 60, 250, 264, 576])
def test_buffers_of_a_head_size_that_attention_does_not_take(td, dim):
    import torch
    with pytest.raises(ValueError, match="multiple of 8 elements, 256 at most"):
        td.AttentionBuffers(3, 8, dim, torch.bfloat16, out=Sized(torch.bfloat16, 3, 8, dim))


@pytest.mark.parametrize("which", ["cache", "q", "out"])
def test_strides_that_attention_does_not_take(td, monkeypatch, which):
    import torch
    bf16, i32 = torch.bfloat16, torch.int32
    odd = dict(strides=(20 * 4160, 4160, 260, 65, 1)) if which == "cache" else {}
    cache = some_cache(td, monkeypatch, keys=Sized(bf16, 2, 20, 16, 4, 64, **odd), values=Sized(bf16, 2, 20, 16, 4, 64, **odd))
    odd = dict(strides=(8 * 68, 68, 1))
    out = td.AttentionBuffers(3, 8, 64, bf16, out=Sized(bf16, 3, 8, 64, **(odd if which == "out" else {})))
    q = Sized(bf16, 3, 8, 64, **(odd if which == "q" else {}))
    with pytest.raises(td.TdError, match="multiples of 16 bytes") as refused:
        td.cache_attention(out, cache, q, stream=0)
    assert refused.value.code == td.EINVAL
    fine = td.AttentionBuffers(3, 8, 64, bf16, out=Sized(bf16, 3, 8, 64))
    with pytest.raises(td.TdError) as refused:                        # another reason: no word of strides
        td.cache_attention(fine, some_cache(td, monkeypatch, keys=Sized(bf16, 2, 20, 16, 4, 64), values=Sized(bf16, 2, 20, 16, 4, 64)),
                           Sized(bf16, 3, 8, 64), layer=2, stream=0)
    assert "16 bytes" not in str(refused.value)


def test_scales_that_pass_floats_range_in_units_of_ln_2(td):
    import torch
    for scale in (2.4e38, -2.4e38, 3.4e38):
        assert attend(td, scale=scale) == td.EINVAL
    if not torch.cuda.is_available():
        assert attend(td, scale=2.3e38) == attend(td, scale=-2.3e38) == td.ECUDA


def test_a_cache_without_contents_is_refused_as_such(td, monkeypatch):
    """Tables only: the refusal is the call's own, and has no word of strides."""
    import torch
    tables = some_cache(td, monkeypatch, keys=None, values=None, page_size=16)
    tables.dim, tables.tag = 64, td.BF16
    out = td.AttentionBuffers(3, 8, 64, torch.bfloat16, out=Sized(torch.bfloat16, 3, 8, 64))
    with pytest.raises(td.TdError) as refused:
        td.cache_attention(out, tables, Sized(torch.bfloat16, 3, 8, 64), stream=0)
    assert refused.value.code == td.EINVAL and "16 bytes" not in str(refused.value)
