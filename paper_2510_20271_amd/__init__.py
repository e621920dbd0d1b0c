"""MI355X-native Euler Characteristic Curves (hard and soft) behind a C ABI.

``api`` binds the entry points of include/ecc.h; ``layer`` wraps the soft path as a
``torch.autograd.Function`` / ``nn.Module``; ``norm`` (group norm with an activation) and ``loss`` (cross entropy of a
linear head) are the layers on either side of it in a network; ``synth`` holds the seeded synthetic
inputs; ``build`` compiles the HIP sources for gfx950.
"""
__all__ = ["api", "layer", "norm", "loss", "synth", "build"]
