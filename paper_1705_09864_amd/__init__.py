"""MI355X-native binary-layer kernels (BMXNet hot path): thin Python binding over libbmx.

``paper_1705_09864_amd.binding`` marshals torch device tensors into the C ABI of
``include/bmx.h``; ``paper_1705_09864_amd.synth`` draws the seeded synthetic inputs;
``paper_1705_09864_amd.decoder_layer`` is a decoder layer's attention on 4-bit weights and a cache of 8 bits or 4;
``paper_1705_09864_amd.build`` compiles the HIP sources for gfx950.
"""
