"""Tensors that say they are on a GPU that need not be there: for calls that refuse
them before they look at an address."""
import torch


class Elsewhere(torch.Tensor):
    @staticmethod
    def __new__(cls, gpu, *shape, dtype=torch.float32):
        return torch.Tensor._make_wrapper_subclass(cls, shape, dtype=dtype, device=f"cuda:{gpu}")

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise NotImplementedError(f"{func}: there is no such GPU")
