"""GaDei-style ASGD parameter server on one gfx950 GPU.

The server's hot path (push -> fused K-gradient apply -> pull fan-out) lives
in the HIP library built from csrc/ (libgadeips.so); `ps` is its thin ctypes
binding and `workloads` the seeded synthetic inputs. `learner` has what a
learner computes between a pull and a push (libgadeilearner.so): embeddings,
dropout and fully connected layers. Importing the package loads nothing: the
bindings load their library on first use and raise if it is not built.
"""
