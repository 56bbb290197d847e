"""OCS-expanded quantized layer for AMD MI355X: hand-written HIP behind a small C ABI.

`binding` holds the front end of libocs.so (ctypes, and an extension module for the calls of
generation), `build` compiles both, `layer` owns buffers and call order, `score` judges a quantized
output layer by perplexity, `workloads` draws the seeded synthetic layers.  Nothing is loaded at import time.
"""
