"""Tensors of calls on prompts whose shapes do not fit one another are refused before the library is called: kernels go by q's
sequences and elements, so k's, v's and everything shaped like them must have the same.  Tensors here lie on the host and say
that they do not; a call that got through would meet the library below."""
import pytest
import torch

from paper_2407_02328_amd import Q4Cache, binding, prompt_attention, prompt_attention_backward, prompt_scores


class OnGpu(torch.Tensor):
    """A host tensor that passes for one on the GPU."""

    @property
    def device(self):
        return torch.device("cuda", 0)

    def get_device(self):
        return 0


class Library:
    """Stands in for the library: no call may reach it."""

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_bytes"):
                return 256
            raise AssertionError(f"{name} was called")
        return call


@pytest.fixture(autouse=True)
def library(monkeypatch):
    empty = torch.empty
    monkeypatch.setattr(binding, "load_library", lambda: Library())
    monkeypatch.setattr(torch, "empty", lambda *args, device=None, **kw: empty(*args, **kw).as_subclass(OnGpu))


def on_gpu(shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


def refused(q_shape, k_shape, match, starts=None):
    """All three calls, with outputs that are the caller's and fit their inputs."""
    q, out, d_out, dq = (on_gpu(q_shape) for _ in range(4))
    k, v, dk, dv = (on_gpu(k_shape) for _ in range(4))
    packed = starts is not None
    at = dict(q_start=on_gpu((starts,), torch.int32), k_start=on_gpu((starts,), torch.int32)) if packed else {}
    value = lambda s: on_gpu((s[1], s[0]) if packed else s[:3], torch.float32)  # noqa: E731
    lse = value(q_shape)
    with pytest.raises(ValueError, match=match):
        prompt_attention(q, k, v, out=out, **at)
    with pytest.raises(ValueError, match=match):
        prompt_attention_backward(d_out, q, k, v, out, lse, dq=dq, dk=dk, dv=dv, **at)
    with pytest.raises(ValueError, match=match):
        prompt_scores(q, k, lse, scores=value(k_shape), **at)


@pytest.mark.parametrize("q_batch,k_batch", [(4, 2), (2, 4), (16, 1), (1, 16), (3, 0)])
def test_sequences_of_a_dense_batch(q_batch, k_batch):
    refused((q_batch, 8, 64, 128), (k_batch, 8, 64, 128), "^k: ")


@pytest.mark.parametrize("q_dim,k_dim", [(128, 64), (64, 128)])
def test_elements_of_a_head(q_dim, k_dim):
    refused((2, 8, 64, q_dim), (2, 4, 70, k_dim), "^k: ")
    refused((64, 8, q_dim), (70, 4, k_dim), "^k: ", starts=3)


def test_dimensions():
    refused((2, 8, 64, 128), (8, 64, 128), "^q, k: ")
    refused((64, 8, 128), (2, 8, 64, 128), "^q, k: ", starts=3)


def test_values_that_do_not_fit_the_keys():
    q, k, lse = on_gpu((2, 8, 64, 128)), on_gpu((2, 4, 70, 128)), on_gpu((2, 8, 64), torch.float32)
    for shape in ((1, 4, 70, 128), (2, 4, 70, 64), (2, 8, 70, 128), (2, 4, 64, 128)):
        with pytest.raises(ValueError, match="^v: "):
            prompt_attention(q, k, on_gpu(shape))
        with pytest.raises(ValueError, match="^v: "):
            prompt_attention_backward(q, q, k, on_gpu(shape), q, lse)


def test_prompts_that_do_not_fit_a_cache():
    cache = Q4Cache.__new__(Q4Cache)
    cache.cfg = binding.AdoreQ4Config(2, 8, 4, 128, 64, 8, binding.ADORE_BF16, 0.0)
    cache.device, cache.dtype, cache.lib = torch.device("cuda", 0), torch.bfloat16, Library()
    for k, v in (((1, 4, 70, 128), (1, 4, 70, 128)), ((2, 8, 70, 128), (2, 8, 70, 128)), ((2, 4, 70, 64), (2, 4, 70, 64))):
        with pytest.raises(ValueError, match="^k: "):
            cache.fill(on_gpu(k), on_gpu(v))
