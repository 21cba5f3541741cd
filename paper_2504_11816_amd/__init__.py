"""Decode attention over a partly offloaded KV cache for one MI355X.

binding   ctypes layer over libokv.so (the C ABI declared in include/okv.h)
harness   device / pinned-host buffers and streams around a binding.Context
synth     seeded synthetic inputs (shared with the tests' CPU oracle)
cache8, cache16   paged KV caches in 8 bits, and in fp16 with several new tokens of a sequence at once
pages     taking, forking, shortening, freeing, compacting and copying pages
linear4, compressed   4-bit linear layers, and decoder layers made of them over either cache
sampling  probabilities of logits, verification of drafted tokens
build     hipcc driver that produces libokv.so next to this file
"""
