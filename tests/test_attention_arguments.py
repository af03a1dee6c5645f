"""The attention side's binding refuses tensors that are not on the device that its kernels run on: none of their addresses reaches
the library.  Host only: tensors are stand-ins with the few members that the binding looks at, the library records its calls."""
import pytest
import torch

from paper_2509_15148_b200 import binding

GPU0, GPU1, HOST = torch.device("cuda", 0), torch.device("cuda", 1), torch.device("cpu")
BF, I32, F32, F64, U8 = torch.bfloat16, torch.int32, torch.float32, torch.float64, torch.uint8


class Tensor:
    def __init__(self, shape, dtype, device=GPU0, contiguous=True):
        self.shape, self.dtype, self.device, self.contiguous = torch.Size(shape), dtype, device, contiguous

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        st = [1]
        for n in self.shape[:0:-1]:
            st.insert(0, st[0] * n)
        return tuple(st) if i is None else st[i]

    def is_contiguous(self):
        return self.contiguous

    @property
    def is_cuda(self):
        return self.device.type == "cuda"

    def data_ptr(self):
        return 4096


@pytest.fixture
def calls(monkeypatch):
    """The calls that reached the library; the current device is cuda:0."""
    made = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or 0
    monkeypatch.setattr(binding, "load", lambda: Lib())
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    return made


def cache(device=GPU0):
    kv = (4, 16, 2, 64)
    return binding.PagedCache(Tensor(kv, BF, device), Tensor(kv, BF, device), Tensor((2, 2), I32, device))


def arguments(dev):
    """name -> (function, its arguments, all on `dev`)."""
    t = lambda *s, d=I32: Tensor(s, d, dev)  # noqa: E731
    q, kv, lens, cu, w = t(3, 4, 64, d=BF), t(3, 2, 64, d=BF), t(2), t(3), t(2, 2, 40, d=F32)
    c = cache(dev) if dev.type == "cuda" else None
    every = {
        "rope_append": (binding.rope_append, dict(q=q, k=kv, v=kv, positions=t(3), freqs=t(32, d=F64), cache=c, ctx_lens=lens, cu_tokens=cu,
                                                  max_tokens=2, q_out=q)),
        "tree_attention": (binding.tree_attention, dict(q=q, cache=c, ctx_lens=lens, cu_tokens=cu, pre=t(3), end=t(3), max_tokens=2, max_len=32, scale=0.1,
                                                        out=q, lse=t(3, 4, d=F32), workspace=t(4096, d=U8))),
        "cache_weights": (binding.cache_weights, dict(q=q, cache=c, lse=t(3, 4, d=F32), ctx_lens=lens, cu_tokens=cu, pre=t(3), end=t(3), max_tokens=2,
                                                      max_len=32, scale=0.1, weights_in=w, weights_out=w)),
        "cache_select": (binding.cache_select, dict(weights=w, lens=lens, budget=10, sinks=1, recent=2, kept=t(2, 2, 10), counts=lens)),
        "cache_gather": (binding.cache_gather, dict(src=c, kept=t(2, 2, 10), counts=lens, dst=c, weights_in=w, weights_out=t(2, 2, 10, d=F32))),
    }
    return every


NAMES = sorted(arguments(GPU0))


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_the_current_device_reach_the_library(calls, name):
    f, args = arguments(GPU0)[name]
    f(**args)
    assert calls == ["atts_" + name]


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device_than_the_current_one_are_refused(calls, name):
    f, args = arguments(GPU1)[name]
    with pytest.raises(ValueError):
        f(**args)
    assert calls == []


def test_host_tensors_are_refused(calls):
    f, args = arguments(HOST)["cache_select"]       # the only call without a cache, whose tensors are on a device
    with pytest.raises(ValueError):
        f(**args)
    assert calls == []


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("other", [GPU1, HOST])
def test_one_tensor_elsewhere_is_refused(calls, name, other):
    f, args = arguments(GPU0)[name]
    for key, x in args.items():
        if isinstance(x, Tensor):
            with pytest.raises(ValueError):
                f(**{**args, key: Tensor(x.shape, x.dtype, other)})
        elif isinstance(x, binding.PagedCache) and other.type == "cuda":
            with pytest.raises(ValueError):
                f(**{**args, key: cache(other)})
    assert calls == []


def test_a_workspace_with_gaps_is_refused(calls):
    f, args = arguments(GPU0)["tree_attention"]
    with pytest.raises(ValueError):
        f(**{**args, "workspace": Tensor((4096,), U8, contiguous=False)})
    assert calls == []


def test_tree_plan_refuses_device_tensors(calls):
    """(meta tensors stand for any that are not on the host)"""
    host = torch.tensor([-1, 0], dtype=I32), torch.tensor([0, 2], dtype=I32)
    binding.tree_plan(*host)
    assert calls == ["atts_tree_plan"]
    for bad in ((host[0].to("meta"), host[1]), (host[0], host[1].to("meta"))):
        with pytest.raises(ValueError):
            binding.tree_plan(*bad)
    assert calls == ["atts_tree_plan"]
