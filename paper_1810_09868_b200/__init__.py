"""VGG19 forward / backward pass for NVIDIA B200 (sm_100a) behind a C ABI.

`binding` mirrors include/vgg19_b200.h one to one.  `Net` is a small
convenience holder: it creates a handle and lets torch allocate the device
workspace (torch is used for device memory and streams only).
"""
from __future__ import annotations

from . import binding
from .binding import *  # noqa: F401,F403


class Net:
    """Owns a vgg19 handle and its torch-allocated workspace."""

    def __init__(self, height, width, batch_max, dtype, params=None, seed=0, flags=0, mode=binding.VGG19_MODE_BACKWARD,
                 host_io=False, device="cuda:0"):
        import torch
        self._torch = torch
        self.height, self.width, self.batch_max, self.dtype = height, width, batch_max, dtype
        self.device = torch.device(device)
        with torch.cuda.device(self.device):
            if params is None:
                self.handle = binding.vgg19_create(height, width, batch_max, dtype, seed, flags)
            else:
                self.handle = binding.vgg19_create_from_params(height, width, batch_max, dtype, params, flags)
        self.n_tensors, self.n_params = binding.vgg19_param_count(self.handle)
        nbytes = binding.vgg19_workspace_bytes(self.handle, batch_max, mode)
        if host_io:
            nbytes += binding.vgg19_io_bytes(self.handle, batch_max, mode)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        binding.vgg19_bind_workspace(self.handle, self.workspace, nbytes)

    @property
    def act_dtype(self):
        return self._torch.bfloat16 if self.dtype == binding.VGG19_BF16 else self._torch.float32

    def forward(self, images, logits=None, probs=None, stream=None):
        torch = self._torch
        B = images.shape[0]
        if logits is None:
            logits = torch.empty(B, 1000, dtype=torch.float32, device=self.device)
        stream = stream or torch.cuda.current_stream(self.device)
        binding.vgg19_forward(self.handle, images, B, logits, probs, stream)
        return logits

    def _allocating_for(self, stream):
        """What is allocated meanwhile belongs to `stream`: a torch stream, or its address."""
        torch = self._torch
        return torch.cuda.stream(torch.cuda.ExternalStream(stream, device=self.device) if isinstance(stream, int) else stream)

    def classify(self, images, top_k=5, stream=None):
        """The top_k classes of every image, most probable first: (ids int32, log probabilities fp32), [batch][top_k]."""
        torch = self._torch
        stream = stream or torch.cuda.current_stream(self.device)
        B = images.shape[0]
        with torch.cuda.device(self.device), self._allocating_for(stream):
            logits = self.forward(images, stream=stream)
            ids = torch.empty(B, top_k, dtype=torch.int32, device=self.device)
            logprob = torch.empty(B, top_k, dtype=torch.float32, device=self.device)
            binding.vgg19_logprobs(logits, top_id=ids, top_logprob=logprob, stream=stream)
        return ids, logprob

    def backward(self, images, labels, grads=None, loss=None, logits=None, stream=None):
        torch = self._torch
        B = images.shape[0]
        if grads is None:
            grads = torch.empty(self.n_params, dtype=torch.float32, device=self.device)
        if loss is None:
            loss = torch.empty(1, dtype=torch.float32, device=self.device)
        stream = stream or torch.cuda.current_stream(self.device)
        binding.vgg19_backward(self.handle, images, labels, B, grads, loss, logits, stream)
        return grads, loss

    def sgd_step(self, grads, lr, stream=None):
        """parameters <- parameters - lr * grads, on the device, with every derived filter copy rebuilt."""
        binding.vgg19_sgd_step(self.handle, grads, lr, stream or self._torch.cuda.current_stream(self.device))

    def muon_step(self, grads, momentum_buffer, lr, momentum=0.95, decay=0.0, bias_lr=None, steps=5, nesterov=True, stream=None):
        """The orthogonalised update of every weight tensor (biases: momentum and a plain step at bias_lr, lr if None).
        momentum_buffer: fp32, n_params elements, zeros at first; the workspace is allocated on the first call and kept."""
        torch = self._torch
        for name, t in (("grads", grads), ("momentum_buffer", momentum_buffer)):
            if t.dtype != torch.float32 or t.device != self.workspace.device or not t.is_contiguous() or t.numel() != self.n_params:
                raise binding.Vgg19Error(binding.VGG19_ERR_ARG, f"{name}: {self.n_params} dense float32 values on {self.device} are needed")
        stream = stream or torch.cuda.current_stream(self.device)
        with torch.cuda.device(self.device), self._allocating_for(stream):  # (memory that this stream may write to)
            if getattr(self, "muon_workspace", None) is None:
                self.muon_workspace = torch.empty(binding.vgg19_muon_step_bytes(self.handle), dtype=torch.uint8, device=self.device)
            binding.vgg19_muon_step(self.handle, grads, momentum_buffer, lr, momentum, decay, lr if bias_lr is None else bias_lr, steps,
                                    nesterov, self.muon_workspace, self.muon_workspace.numel(), stream)

    def set_dropout(self, rate, seed=0, first_pass=0):
        """Training passes drop the outputs of dense layers 1 and 2 at `rate` (0: none), each pass with masks of its own.  A mask goes by
        seed, pass and place in the batch: ranks that train on parts of a batch take seeds of their own."""
        with self._torch.cuda.device(self.device):
            binding.vgg19_set_dropout(self.handle, rate, seed, first_pass)

    def train_step(self, images, labels, lr, loss=None, stream=None):
        """Forward + backward + update as one recorded device program (workspace of VGG19_MODE_TRAIN)."""
        stream = stream or self._torch.cuda.current_stream(self.device)
        binding.vgg19_train_step(self.handle, images, labels, images.shape[0], lr, loss, stream)

    def saved_tensor(self, batch, mode, index):
        """View of a stored activation inside the workspace (no copy)."""
        off, dims = binding.vgg19_saved_tensor(self.handle, batch, mode, index)
        n = 1
        for d in dims:
            n *= d
        elt = 2 if self.dtype == binding.VGG19_BF16 else 4
        return self.workspace[off:off + n * elt].view(self.act_dtype).view(*dims)

    def param_slices(self):
        """[(offset, dims)] of the 38 tensors in the flat parameter buffer."""
        return [binding.vgg19_param_info(self.handle, i) for i in range(self.n_tensors)]

    def sync_status(self, stream=None):
        return binding.vgg19_sync_status(self.handle, stream or self._torch.cuda.current_stream(self.device))

    def close(self):
        if getattr(self, "handle", None):
            binding.vgg19_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
