"""A GPU cache whose rows are held in codes and its plain form, driven by the same calls."""
import numpy as np
import torch

from oracle import pages as OP
from pages_common import Both, i32


class BothCoded(Both):
    def __init__(self, ldr, bits, layers, hkv, d, page, n_pages, batch, max_pages, seed=0,
                 stream=None):
        self.g = ldr.Pages(layers, hkv, d, page, n_pages, batch, max_pages, codes=f"mxfp{bits}",
                           stream=stream).init()
        self.o = OP.CodedCache(bits, layers, hkv, d, page, n_pages, batch, max_pages)
        self.layers, self.dtype, self.batch = layers, torch.bfloat16, batch
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.g.pool.fill_(255)       # scales of NaN: a use of what free pages hold shows

    def check(self, contents=True):
        super().check(contents=False)
        if not contents or not max(self.o.rows):
            return
        K, V = self.g.read(i32([0] * self.batch), i32(self.o.rows), max(self.o.rows))
        K, V = K.double().cpu().numpy(), V.double().cpu().numpy()
        for layer in range(self.layers):
            for b, n in enumerate(self.o.rows):
                ok, ov = self.o.sequence(layer, b)
                assert np.array_equal(K[b, :n, layer], ok, equal_nan=True), (layer, b)
                assert np.array_equal(V[b, :n, layer], ov, equal_nan=True), (layer, b)
                assert not K[b, n:].any() and not V[b, n:].any(), b
