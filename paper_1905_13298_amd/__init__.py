"""DeepShift shift operators (LinearShift, ConvShift) for AMD Instinct MI355X.

The compute path is the HIP library ``libdeepshift.so`` behind the C ABI in
``include/deepshift.h``; ``ops`` wraps it for PyTorch tensors and
``workloads`` generates seeded synthetic inputs. ``network`` runs a ResNet of shift
convolutions, ``decoder`` a language model's decoder on the 8-bit operators.
"""
