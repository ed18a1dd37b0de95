"""Objects that describe tensors on a GPU where there is none: what the native marshalling reads of a tensor (not a test module).
Calls with them are to be refused before anything would be launched."""
import math

import torch


class Described:
    def __init__(self, shape, dtype, at, device=0, stride=None, requires_grad=False):
        self.shape, self.dtype, self.at, self.device_index, self.requires_grad = torch.Size(shape), dtype, at, device, requires_grad
        self.by = stride or tuple(math.prod(shape[i + 1:]) for i in range(len(shape)))
        self.is_cuda = device >= 0

    def stride(self):
        return self.by

    def data_ptr(self):
        return self.at

    def numel(self):
        return math.prod(self.shape)

    def get_device(self):
        return self.device_index

    def is_contiguous(self):
        return self.by == tuple(math.prod(self.shape[i + 1:]) for i in range(len(self.shape)))

    @property
    def nbytes(self):
        return self.numel() * torch.empty(0, dtype=self.dtype).element_size()


class DescribedRouting:
    def __init__(self, tokens, choices, experts, at, device=0):
        self.tokens, self.choices, self.experts = tokens, choices, experts
        self.expert_ptr = Described((experts + 1,), torch.int32, at, device)
        self.slot_choice = Described((tokens * choices,), torch.int32, at + (1 << 24), device)
        self.choice_slot = Described((tokens, choices), torch.int32, at + (2 << 24), device)
