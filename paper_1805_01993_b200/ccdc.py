"""Python binding of the C-ABI library ``libccdc.so`` (declared in ``include/ccdc.h``).

Argument marshalling only: every step of the shuffle runs in the library's CUDA
kernels.  PyTorch supplies device memory and streams.  The function names are
those of the C ABI; ``Plan`` wraps a ``ccdc_plan_t`` and offers the same calls as
methods taking torch tensors.

There is no fallback: if the shared library has not been built (see
``paper_1805_01993_b200.build``) importing a symbol from here raises.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

_LIB_PATH = Path(__file__).resolve().parent / "libccdc.so"
_lib = None

I32, F32, BF16, F16 = 0, 1, 2, 3
ACTS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3}
NORMS = {"rms": 0, "layer": 1}
OK, EINVAL, ENOMEM, ECUDA, ESIZE, ESTATE = 0, -1, -2, -3, -4, -5
MAX_K = 32

_P, _I, _LL, _SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t
_ULL, _FL, _DB = ctypes.c_ulonglong, ctypes.c_float, ctypes.c_double
_PP = ctypes.POINTER(ctypes.c_void_p)

# name -> (restype, argtypes); mirrors include/ccdc.h
SIGNATURES = {
    "ccdc_plan": (_I, [_I, _I, _LL, _I, _LL, _I, _PP]),
    "ccdc_plan_jobs": (_I, [_I, _I, _LL, _I, _LL, _I, _PP]),
    "ccdc_plan_jobs_gamma": (_I, [_I, _I, _LL, _I, _LL, _I, _I, _PP]),
    "ccdc_plan_compression": (_I, [_I, _I, _LL, _I, _LL, _I, _PP]),
    "ccdc_plan_sharded": (_I, [_I, _I, _LL, _I, _LL, _I, _I, _I, _I, _PP]),
    "ccdc_plan_coded_row_position": (_LL, [_P, _LL, _I]),
    "ccdc_plan_node_is_local": (_I, [_P, _I]),
    "ccdc_coded_send_bytes": (_SZ, [_P]),
    "ccdc_plan_destroy": (None, [_P]),
    "ccdc_plan_upload": (_I, [_P]),
    "ccdc_plan_kernel_family": (_I, [_P]),
    "ccdc_plan_tune_family": (_I, [_P, _I]),
    "ccdc_shuffle_status": (_I, [_P]),
    "ccdc_plan_decode_threads": (_I, [_P]),
    "ccdc_plan_decode_chunks": (_I, [_P]),
    "ccdc_plan_decode_cluster": (_I, [_P]),
    "ccdc_plan_tune_decode": (_I, [_P, _I, _I]),
    "ccdc_plan_num_jobs": (_LL, [_P]),
    "ccdc_plan_num_batches": (_LL, [_P]),
    "ccdc_plan_num_groups": (_LL, [_P]),
    "ccdc_plan_files_per_batch": (_LL, [_P]),
    "ccdc_plan_batch_files": (_LL, [_P, _LL]),
    "ccdc_plan_packet_elems": (_LL, [_P]),
    "ccdc_plan_segment_elems": (_LL, [_P]),
    "ccdc_plan_coded_row_elems": (_LL, [_P]),
    "ccdc_plan_coded_bits": (_LL, [_P]),
    "ccdc_plan_batch_of_file": (_I, [_P, _LL, _P]),
    "ccdc_plan_batch": (_I, [_P, _LL, _P, _P, _P]),
    "ccdc_plan_group": (_I, [_P, _LL, _P]),
    "ccdc_plan_group_batches": (_I, [_P, _LL, _P]),
    "ccdc_plan_node_batches": (_LL, [_P, _I, _P]),
    "ccdc_partition_bytes": (_SZ, [_P, _I]),
    "ccdc_packets_bytes": (_SZ, [_P, _I]),
    "ccdc_decoded_bytes": (_SZ, [_P, _I]),
    "ccdc_coded_bytes": (_SZ, [_P]),
    "ccdc_out_bytes": (_SZ, [_P]),
    "ccdc_workspace_bytes": (_SZ, [_P]),
    "ccdc_map_workspace_bytes": (_SZ, [_P, _LL]),
    "ccdc_map": (_I, [_P, _PP, _PP, _P, _LL, _PP, _P, _P]),
    "ccdc_map_status": (_I, [_P, _LL, _P]),
    "ccdc_map_last_kernel": (ctypes.c_char_p, []),
    "ccdc_combine": (_I, [_P, _PP, _PP, _P]),
    "ccdc_encode": (_I, [_P, _PP, _P, _P]),
    "ccdc_decode": (_I, [_P, _PP, _P, _PP, _P]),
    "ccdc_reduce": (_I, [_P, _PP, _PP, _P, _P]),
    "ccdc_encode_fused": (_I, [_P, _PP, _P, _P]),
    "ccdc_decode_reduce": (_I, [_P, _PP, _P, _P, _P, _P]),
    "ccdc_encode_fused_peers": (_I, [_P, _PP, _PP, _P]),
    "ccdc_shuffle": (_I, [_P, _PP, _P, _P, _P, _P]),
    "ccdc_static_scratch_bytes": (_SZ, []),
    "ccdc_decode_reduce_static": (_I, [_P, _PP, _P, _P, _P]),
    "ccdc_compression_shuffle": (_I, [_P, _PP, _PP, _P, _P]),
    "ccdc_shuffle_host": (_I, [_P, _PP, _P, _PP, _P, _P, _P, _P]),
    "ccdc_shuffle_host_files": (_I, [_P, _P, _P, _PP, _P, _P, _P, _P]),
    "ccdc_job_host": (_I, [_P, _PP, _PP, _P, _LL, _P, _PP, _PP, _P, _PP, _P, _P, _P, _P, _P]),
    "ccdc_value_shard": (_I, [_I, _I, _I, _LL, _I, _I, ctypes.POINTER(ctypes.c_longlong)]),
    "ccdc_value_shard_position": (_LL, [_I, _I, _I, _LL, _I, _I, _LL]),
    "ccdc_value_shard_copy": (_I, [_I, _I, _I, _LL, _I, _I, _I, _P, _P, _LL, _P]),
    "ccdc_peer_buffer_create": (_I, [_SZ, _PP, _P]),
    "ccdc_peer_buffer_open": (_I, [_P, _PP]),
    "ccdc_peer_buffer_close": (_I, [_P]),
    "ccdc_peer_buffer_destroy": (_I, [_P]),
    "ccdc_peer_buffer_copy": (_I, [_P, _P, _SZ, _P]),
    "ccdc_dropout": (_I, [_LL, _LL, _I, _P, _LL, _P, _LL, _DB, _ULL, _ULL, _P]),
    "ccdc_residual_norm_forward": (_I, [_LL, _LL, _I, _I, _FL, _P, _LL, _P, _LL, _P, _P, _P, _LL, _FL, _DB, _ULL, _ULL,
                                        _P, _LL, _P, _LL, _P, _P]),
    "ccdc_residual_norm_workspace_bytes": (_SZ, [_LL, _LL]),
    "ccdc_residual_norm_backward": (_I, [_LL, _LL, _I, _I, _I, _P, _LL, _P, _LL, _P, _LL, _P, _LL, _P, _P, _P, _P, _LL,
                                         _FL, _DB, _ULL, _ULL, _P, _LL, _P, _LL, _P, _P, _P, _P, _SZ, _P]),
    "ccdc_ffn_saved_bytes": (_SZ, [_LL, _LL, _I]),
    "ccdc_ffn_workspace_bytes": (_SZ, [_LL, _LL, _LL, _I, _I, _I]),
    "ccdc_ffn_forward": (_I, [_LL, _LL, _LL, _I, _I, _P, _LL, _P, _P, _LL, _P, _LL, _P, _LL, _P, _P, _SZ, _P]),
    "ccdc_ffn_backward": (_I, [_LL, _LL, _LL, _I, _I, _I, _P, _LL, _P, _LL, _P, _P, _LL, _P, _LL, _P, _P, _LL, _P, _P,
                               _P, _P, _SZ, _P]),
    "ccdc_block_status": (_I, []),
    "ccdc_strerror": (ctypes.c_char_p, [_I]),
    "ccdc_last_cuda_error": (_I, []),
    "ccdc_num_kernel_launches": (_I, []),
    "ccdc_last_gather_kernel": (ctypes.c_char_p, []),
    "ccdc_last_decode_kernel": (ctypes.c_char_p, []),
}


class CcdcError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().ccdc_strerror(status).decode()
        if status == ECUDA:
            msg += f" [cudaError {lib().ccdc_last_cuda_error()}]"
        super().__init__(f"{where}: {msg} ({status})")


def lib():
    """The loaded shared library; raises if it is missing (there is no other path)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise ImportError(f"{_LIB_PATH} not built: run `python -m paper_1805_01993_b200.build`")
        L = ctypes.CDLL(str(_LIB_PATH))
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != OK:
        raise CcdcError(status, where)


def _ptr_array(tensors):
    arr = (ctypes.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = t.data_ptr() if t is not None and t.numel() > 0 else None
    return arr


PEER_HANDLE_BYTES = 64


class PeerBuffer:
    """Device memory that another process can open (``ccdc_peer_buffer_*``).  Quacks like a tensor
    for the step calls (``data_ptr`` / ``numel``).  ``PeerBuffer.create(nbytes)`` allocates on the
    current device and exposes ``handle`` (64 bytes to send to the other ranks);
    ``PeerBuffer.open(handle, nbytes)`` maps another process's buffer."""

    def __init__(self, ptr, nbytes, handle, owner):
        self.ptr, self.nbytes, self.handle, self.owner = ptr, nbytes, handle, owner

    @classmethod
    def create(cls, nbytes):
        ptr = ctypes.c_void_p()
        handle = (ctypes.c_ubyte * PEER_HANDLE_BYTES)()
        _check(lib().ccdc_peer_buffer_create(nbytes, ctypes.byref(ptr), handle), "ccdc_peer_buffer_create")
        return cls(ptr.value, nbytes, bytes(handle), True)

    @classmethod
    def open(cls, handle, nbytes):
        ptr = ctypes.c_void_p()
        buf = (ctypes.c_ubyte * PEER_HANDLE_BYTES).from_buffer_copy(handle)
        _check(lib().ccdc_peer_buffer_open(buf, ctypes.byref(ptr)), "ccdc_peer_buffer_open")
        return cls(ptr.value, nbytes, bytes(handle), False)

    def data_ptr(self):
        return self.ptr

    def numel(self):
        return self.nbytes // 4

    def copy_to(self, tensor, stream=None):
        """copies the buffer into a tensor (device or pinned host) of the same size."""
        _check(lib().ccdc_peer_buffer_copy(tensor.data_ptr(), self.ptr, self.nbytes, _stream_handle(stream)),
               "ccdc_peer_buffer_copy")

    def release(self):
        if self.ptr:
            fn = lib().ccdc_peer_buffer_destroy if self.owner else lib().ccdc_peer_buffer_close
            _check(fn(self.ptr), "ccdc_peer_buffer_release")
            self.ptr = None


def value_shard(K, r, Q, B, rank, world) -> int:
    """value length of rank's shard when every segment is cut into `world` sub-ranges."""
    out = ctypes.c_longlong()
    _check(lib().ccdc_value_shard(K, r, Q, B, rank, world, ctypes.byref(out)), "ccdc_value_shard")
    return out.value


def value_shard_position(K, r, Q, B, rank, world, local_pos) -> int:
    return lib().ccdc_value_shard_position(K, r, Q, B, rank, world, local_pos)


def value_shard_copy(K, r, Q, B, rank, world, to_local, src, dst, rows, stream=None):
    """device copy between the full layout [rows][Q][B] and the rank's [rows][Q][B_local]."""
    _check(lib().ccdc_value_shard_copy(K, r, Q, B, rank, world, int(to_local), src.data_ptr(), dst.data_ptr(), rows,
                                       _stream_handle(stream)), "ccdc_value_shard_copy")


def _stream_handle(stream):
    import torch

    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


class Plan:
    """``ccdc_plan`` / ``ccdc_plan_jobs`` plus the step calls on torch tensors."""

    def __init__(self, K, r, N, Q, B, dtype, jobs: bool = False, compression: bool = False, shard=None, gamma: int = 1):
        self.K, self.r, self.N, self.Q, self.B = K, r, N, Q, B
        self.dtype = {"int32": I32, "float32": F32, I32: I32, F32: F32}[dtype]
        self.jobs = jobs
        h = ctypes.c_void_p()
        fn = lib().ccdc_plan_compression if compression else lib().ccdc_plan_jobs if jobs else lib().ccdc_plan
        self._h = None
        self.shard = shard
        if shard is not None:           # (rank, world): this GPU's share of the logical nodes
            _check(lib().ccdc_plan_sharded(K, r, N, Q, B, self.dtype, int(jobs), shard[0], shard[1], ctypes.byref(h)),
                   "ccdc_plan_sharded")
        elif gamma != 1:
            if not jobs:
                raise ValueError("gamma > 1 belongs to the J-job scheme (jobs=True)")
            _check(lib().ccdc_plan_jobs_gamma(K, r, N, Q, B, self.dtype, gamma, ctypes.byref(h)), "ccdc_plan_jobs_gamma")
        else:
            _check(fn(K, r, N, Q, B, self.dtype, ctypes.byref(h)), "ccdc_plan")
        self._h = h
        L = lib()
        self.J = L.ccdc_plan_num_jobs(h)
        self.num_batches = L.ccdc_plan_num_batches(h)
        self.num_groups = L.ccdc_plan_num_groups(h)
        self.files_per_batch = L.ccdc_plan_files_per_batch(h)
        self.packet_elems = L.ccdc_plan_packet_elems(h)
        self.segment_elems = L.ccdc_plan_segment_elems(h)
        self.coded_row_elems = L.ccdc_plan_coded_row_elems(h)
        self.coded_bits = L.ccdc_plan_coded_bits(h)

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.ccdc_plan_destroy(self._h)
            self._h = None

    # ---- queries --------------------------------------------------------
    def batch_of_file(self, n):
        out = (ctypes.c_int * self.r)()
        _check(lib().ccdc_plan_batch_of_file(self._h, n, out), "ccdc_plan_batch_of_file")
        return [k for k in out if k >= 0]

    def batch(self, p):
        nodes = (ctypes.c_int * self.r)()
        f0, job = ctypes.c_longlong(), ctypes.c_longlong()
        _check(lib().ccdc_plan_batch(self._h, p, nodes, ctypes.byref(f0), ctypes.byref(job)), "ccdc_plan_batch")
        return [n for n in nodes if n >= 0], f0.value, job.value

    def group(self, g):
        out = (ctypes.c_int * (self.r + 1))()
        _check(lib().ccdc_plan_group(self._h, g, out), "ccdc_plan_group")
        return list(out)

    def group_batches(self, g):
        out = (ctypes.c_longlong * (self.r + 1))()
        _check(lib().ccdc_plan_group_batches(self._h, g, out), "ccdc_plan_group_batches")
        return list(out)

    def node_batches(self, k):
        n = lib().ccdc_plan_node_batches(self._h, k, None)
        out = (ctypes.c_longlong * max(n, 1))()
        lib().ccdc_plan_node_batches(self._h, k, out)
        return list(out)[:n]

    def partition_bytes(self, k):
        return lib().ccdc_partition_bytes(self._h, k)

    def packets_bytes(self, k):
        return lib().ccdc_packets_bytes(self._h, k)

    def decoded_bytes(self, k):
        return lib().ccdc_decoded_bytes(self._h, k)

    def node_is_local(self, k):
        return bool(lib().ccdc_plan_node_is_local(self._h, k))

    def coded_row_position(self, g, a):
        return lib().ccdc_plan_coded_row_position(self._h, g, a)

    @property
    def kernel_family(self):
        return lib().ccdc_plan_kernel_family(self._h)

    def tune_family(self, family):
        """0: loads through registers; 1: bulk-copy pipelines (before the tables are uploaded)."""
        _check(lib().ccdc_plan_tune_family(self._h, family), "ccdc_plan_tune_family")

    def shuffle_status(self):
        """after a synchronise: raises if a bounded wait inside a kernel ever ran out on this plan."""
        _check(lib().ccdc_shuffle_status(self._h), "ccdc_shuffle_status")

    @property
    def decode_threads(self):
        return lib().ccdc_plan_decode_threads(self._h)

    @property
    def decode_chunks(self):
        return lib().ccdc_plan_decode_chunks(self._h)

    @property
    def decode_cluster(self):
        return bool(lib().ccdc_plan_decode_cluster(self._h))

    def tune_decode(self, threads, chunks):
        """fixes the launch shape of the fused decode (before the tables are uploaded)."""
        _check(lib().ccdc_plan_tune_decode(self._h, threads, chunks), "ccdc_plan_tune_decode")

    @property
    def coded_send_bytes(self):
        return lib().ccdc_coded_send_bytes(self._h)

    @property
    def coded_bytes(self):
        return lib().ccdc_coded_bytes(self._h)

    @property
    def out_bytes(self):
        return lib().ccdc_out_bytes(self._h)

    @property
    def workspace_bytes(self):
        return lib().ccdc_workspace_bytes(self._h)

    def node_files(self, k):
        """global file ids in the order of node k's partition rows."""
        files = []
        for p in self.node_batches(k):
            _, f0, _ = self.batch(p)
            files.extend(range(f0, f0 + lib().ccdc_plan_batch_files(self._h, p)))
        return files

    # ---- device buffers (torch is the allocator) --------------------------
    @property
    def torch_dtype(self):
        import torch

        return torch.int32 if self.dtype == I32 else torch.float32

    def upload(self):
        _check(lib().ccdc_plan_upload(self._h), "ccdc_plan_upload")

    def alloc(self, nbytes, device="cuda"):
        import torch

        return torch.empty(max(nbytes // 4, 0), dtype=self.torch_dtype, device=device)

    def alloc_partitions(self, device="cuda"):
        """one buffer per node (empty for nodes that live on another GPU)."""
        return [self.alloc(self.partition_bytes(k) if self.node_is_local(k) else 0, device) for k in range(self.K)]

    def alloc_packets(self, device="cuda"):
        return [self.alloc(self.packets_bytes(k), device) for k in range(self.K)]

    def alloc_decoded(self, device="cuda"):
        return [self.alloc(self.decoded_bytes(k), device) for k in range(self.K)]

    def fill_partitions(self, part, values):
        """Copies Map outputs ``values`` [J*N][Q][B] (tensor on any device) into the
        node partitions: each node gets a replica of every file it stores."""
        import torch

        row = self.Q * self.B
        flat = values.reshape(-1, row)
        for k in range(self.K):
            if not self.node_is_local(k):
                continue
            idx = torch.as_tensor(self.node_files(k), dtype=torch.long, device=flat.device)
            if idx.numel():
                part[k].view(-1, row).copy_(flat.index_select(0, idx), non_blocking=False)

    def fill_partitions_streaming(self, part, file_iter, sample_index=None):
        """Places files one at a time: ``file_iter`` yields ``(n, tensor [Q][B])`` on
        the partitions' device; each is copied to the r nodes that store file n.
        With ``sample_index`` (1-D long tensor of element positions) also returns
        the sampled values ``[J*N][Q][len(sample_index)]`` on the host."""
        import torch

        row = self.Q * self.B
        where = [{n: i for i, n in enumerate(self.node_files(k))} for k in range(self.K)]
        sampled = None
        if sample_index is not None:
            sampled = torch.empty((self.J * self.N, self.Q, sample_index.numel()), dtype=self.torch_dtype)
        for n, t in file_iter:
            for k in self.batch_of_file(n):
                if not self.node_is_local(k):
                    continue
                i = where[k][n]
                part[k][i * row:(i + 1) * row].copy_(t.reshape(-1))
            if sampled is not None:
                sampled[n] = t.index_select(1, sample_index).cpu()
        return sampled

    # ---- steps ------------------------------------------------------------
    def map_workspace_bytes(self, rows):
        return lib().ccdc_map_workspace_bytes(self._h, rows)

    def map_status(self, rows, workspace):
        """after a synchronise: raises if a wait inside the Map kernel ran out."""
        _check(lib().ccdc_map_status(self._h, rows, workspace.data_ptr()), "ccdc_map_status")

    def map(self, files_x, files_y, w, rows, part, workspace, stream=None):
        """``files_x`` / ``files_y``: per node, bf16 ``[files][rows][Q*B]`` and fp32 ``[files][rows]``."""
        _check(lib().ccdc_map(self._h, _ptr_array(files_x), _ptr_array(files_y), w.data_ptr(), rows,
                              _ptr_array(part), workspace.data_ptr(), _stream_handle(stream)), "ccdc_map")

    def combine(self, part, packets, stream=None):
        _check(lib().ccdc_combine(self._h, _ptr_array(part), _ptr_array(packets), _stream_handle(stream)),
               "ccdc_combine")

    def encode(self, packets, coded, stream=None):
        _check(lib().ccdc_encode(self._h, _ptr_array(packets), coded.data_ptr(), _stream_handle(stream)),
               "ccdc_encode")

    def decode(self, packets, coded, decoded, stream=None):
        _check(lib().ccdc_decode(self._h, _ptr_array(packets), coded.data_ptr(), _ptr_array(decoded),
                                 _stream_handle(stream)), "ccdc_decode")

    def reduce(self, part, decoded, out, stream=None):
        _check(lib().ccdc_reduce(self._h, _ptr_array(part), _ptr_array(decoded), out.data_ptr(),
                                 _stream_handle(stream)), "ccdc_reduce")

    def encode_fused(self, part, coded, stream=None):
        _check(lib().ccdc_encode_fused(self._h, _ptr_array(part), coded.data_ptr(), _stream_handle(stream)),
               "ccdc_encode_fused")

    def encode_fused_peers(self, part, peer_coded, stream=None):
        """``peer_coded``: every rank's full coded buffer as addressable from this GPU."""
        _check(lib().ccdc_encode_fused_peers(self._h, _ptr_array(part), _ptr_array(peer_coded),
                                             _stream_handle(stream)), "ccdc_encode_fused_peers")

    def decode_reduce(self, part, coded, out, workspace=None, stream=None):
        ws = workspace.data_ptr() if workspace is not None and workspace.numel() else None
        _check(lib().ccdc_decode_reduce(self._h, _ptr_array(part), coded.data_ptr(), out.data_ptr(), ws,
                                        _stream_handle(stream)), "ccdc_decode_reduce")

    def compression_shuffle(self, part, recv, out, stream=None):
        _check(lib().ccdc_compression_shuffle(self._h, _ptr_array(part), _ptr_array(recv), out.data_ptr(),
                                              _stream_handle(stream)), "ccdc_compression_shuffle")

    def job_host(self, host_x, host_y, host_w, rows, host_out, dev_x, dev_y, dev_w, part, coded, out, map_workspace,
                 workspace=None, stream=None):
        """Map + shuffle from host tensors (pinned for asynchronous copies) through device staging buffers."""
        _check(lib().ccdc_job_host(self._h, _ptr_array(host_x), _ptr_array(host_y), host_w.data_ptr(), rows,
                                   host_out.data_ptr(), _ptr_array(dev_x), _ptr_array(dev_y), dev_w.data_ptr(),
                                   _ptr_array(part), coded.data_ptr(), out.data_ptr(), map_workspace.data_ptr(),
                                   workspace.data_ptr() if workspace is not None and workspace.numel() else None,
                                   _stream_handle(stream)), "ccdc_job_host")

    def shuffle_host(self, host_part, host_out, part, coded, out, workspace=None, stream=None):
        """``host_part`` / ``host_out``: CPU tensors (pinned for asynchronous copies)."""
        ws = workspace.data_ptr() if workspace is not None and workspace.numel() else None
        _check(lib().ccdc_shuffle_host(self._h, _ptr_array(host_part), host_out.data_ptr(), _ptr_array(part),
                                       coded.data_ptr(), out.data_ptr(), ws, _stream_handle(stream)),
               "ccdc_shuffle_host")

    def shuffle_host_files(self, host_values, host_out, part, coded, out, workspace=None, stream=None):
        """``host_values``: CPU tensor [J*N][Q][B], every file once (pinned for asynchronous copies)."""
        ws = workspace.data_ptr() if workspace is not None and workspace.numel() else None
        _check(lib().ccdc_shuffle_host_files(self._h, host_values.data_ptr(), host_out.data_ptr(), _ptr_array(part),
                                             coded.data_ptr(), out.data_ptr(), ws, _stream_handle(stream)),
               "ccdc_shuffle_host_files")

    def decode_reduce_static(self, part, coded, out, stream=None):
        """``ccdc_decode_reduce`` with the library's built-in scratch: no allocation."""
        _check(lib().ccdc_decode_reduce_static(self._h, _ptr_array(part), coded.data_ptr(), out.data_ptr(),
                                               _stream_handle(stream)), "ccdc_decode_reduce_static")

    def shuffle(self, part, coded, out, workspace=None, stream=None):
        ws = workspace.data_ptr() if workspace is not None and workspace.numel() else None
        _check(lib().ccdc_shuffle(self._h, _ptr_array(part), coded.data_ptr(), out.data_ptr(), ws,
                                  _stream_handle(stream)), "ccdc_shuffle")


# ---- block operators ------------------------------------------------------
# Tensors are 2-D [rows][columns] with contiguous columns and any row stride, all of one dtype (float32,
# bfloat16, float16) on one device.  Outputs and scratch that are not passed in come from torch's allocator,
# on the stream the call runs on.


# Small calls are bound by the host, so the checks compare plain integers and make no device or stream objects.


def _block_dtype(t):
    """type code of a tensor; raises for types the block operators do not take."""
    if not _BLOCK_TYPES:
        import torch

        _BLOCK_TYPES.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    code = _BLOCK_TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"float32, bfloat16 or float16 expected, got {t.dtype}")
    return code


_BLOCK_TYPES = {}


def _rows(t, name, like=None, shape=None):
    """row stride of a 2-D tensor; raises where it is not what the call takes."""
    strides, own = t.stride(), t.shape
    if len(strides) != 2 or (strides[1] != 1 and own[1] > 1):
        raise ValueError(f"{name}: a 2-D tensor with contiguous columns expected")
    if shape is not None and own != shape:
        raise ValueError(f"{name}: shape {tuple(shape)} expected, got {tuple(own)}")
    if like is None:
        if not t.is_cuda:
            raise ValueError(f"{name}: a CUDA tensor expected")
    elif t.dtype is not like.dtype or t.get_device() != like.get_device():
        raise ValueError(f"{name}: {like.dtype} on {like.device} expected, got {t.dtype} on {t.device}")
    return strides[0] if own[0] > 1 else own[1]


def _vector(t, name, like, n, dtype=None):
    """address of n contiguous values of like's (or the given) dtype."""
    if (t.numel() != n or not t.is_contiguous() or t.dtype is not (dtype or like.dtype)
            or t.get_device() != like.get_device()):
        raise ValueError(f"{name}: {n} contiguous {dtype or like.dtype} on {like.device} expected")
    return t.data_ptr()


def _buffer(t, name, like, need=0):
    """(address, bytes) of scratch or saved values that the caller brings: one piece of memory on like's device."""
    size = t.numel() * t.element_size()
    if t.get_device() != like.get_device() or not t.is_contiguous() or size < need:
        raise ValueError(f"{name}: a contiguous tensor{f' of {need} bytes' if need else ''} on {like.device} expected")
    return t.data_ptr(), size


def _elsewhere(x, stream):
    """a context that makes the call's stream and device torch's current ones, or None where they already are."""
    import torch

    if stream is not None:
        if stream.device != x.device:
            raise ValueError("the stream belongs to another device than the tensors")
        return torch.cuda.stream(stream)
    if x.is_cuda and x.get_device() != torch.cuda.current_device():
        return torch.cuda.device(x.device)
    return None


def _handle(x):
    """the current stream of x's device (which is the current device)."""
    import torch

    return torch._C._cuda_getCurrentRawStream(x.get_device())


def _empty_like(x):
    """a tensor of x's shape, type and device with contiguous rows (the cheapest call of torch's that makes one)."""
    import torch

    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


def dropout(x, p, seed, offset=0, out=None, stream=None):
    """``ccdc_dropout``: x with elements dropped by the counter-based mask of (seed, offset + element).
    The backward pass is the same call on the gradient.  ``out`` may be ``x``.  Elements are numbered modulo 2^64 (an
    ``offset`` of -8 is 2^64 - 8)."""
    ctx = _elsewhere(x, stream)
    if ctx is not None:
        with ctx:
            return dropout(x, p, seed, offset, out)
    ldx = _rows(x, "x")
    code = _block_dtype(x)
    rows, cols = x.shape
    if out is None:
        out, ldy = _empty_like(x), cols
    else:
        ldy = _rows(out, "out", x, x.shape)
    status = lib().ccdc_dropout(rows, cols, code, x.data_ptr(), ldx, out.data_ptr(), ldy, p, seed, offset, _handle(x))
    if status:
        _check(status, "ccdc_dropout")
    return out


def _norm_tensors(x, y, w_post, w_pre, gate, rows_per_gate):
    ldx = _rows(x, "x")
    M, D = x.shape
    ldy = D if y is None else _rows(y, "y", x, x.shape)
    pw = None if w_post is None else _vector(w_post, "w_post", x, D)
    pp = None if w_pre is None else _vector(w_pre, "w_pre", x, D)
    pg, per = None, 1
    if gate is not None:
        per = rows_per_gate
        if per is None:
            per = max(M, 1) if gate.numel() == D else 1
        if per < 1:
            raise ValueError("rows_per_gate must be at least 1")
        pg = _vector(gate, "gate", x, max(1, -(-M // per)) * D)
    return M, D, ldx, ldy, pw, pp, pg, per


def residual_norm_forward(x, y=None, *, w_post=None, w_pre=None, gate=None, rows_per_gate=None, alpha=1.0, p=0.0, seed=0,
                          offset=0, kind="rms", eps=1e-5, save=False, out=None, z=None, stream=None):
    """``ccdc_residual_norm_forward``: out = alpha*x + drop(gate * norm(y)*w_post), z = norm(out)*w_pre.
    Returns (out, z), or (out, z, stats) with ``save``; z is None without ``w_pre``.  ``stats`` is opaque and goes to
    ``residual_norm_backward``."""
    ctx = _elsewhere(x, stream)
    if ctx is not None:
        with ctx:
            return residual_norm_forward(x, y, w_post=w_post, w_pre=w_pre, gate=gate, rows_per_gate=rows_per_gate,
                                         alpha=alpha, p=p, seed=seed, offset=offset, kind=kind, eps=eps, save=save,
                                         out=out, z=z)
    M, D, ldx, ldy, pw, pp, pg, per = _norm_tensors(x, y, w_post, w_pre, gate, rows_per_gate)
    code = _block_dtype(x)
    if out is None:
        out, ldo = _empty_like(x), D
    else:
        ldo = _rows(out, "out", x, x.shape)
    pz, ldz, stats, ps = None, D, None, None
    if w_pre is None:
        if z is not None:
            raise ValueError("z needs w_pre")
    else:
        if z is None:
            z = _empty_like(x)
        else:
            ldz = _rows(z, "z", x, x.shape)
        pz = z.data_ptr()
    if save:
        import torch

        stats = x.new_empty(4 * M, dtype=torch.float32)
        ps = stats.data_ptr()
    status = lib().ccdc_residual_norm_forward(M, D, code, NORMS[kind], eps, x.data_ptr(), ldx,
                                              None if y is None else y.data_ptr(), ldy, pw, pp, pg, per, alpha, p, seed,
                                              offset, out.data_ptr(), ldo, pz, ldz, ps, _handle(x))
    if status:
        _check(status, "ccdc_residual_norm_forward")
    return (out, z, stats) if save else (out, z)


def residual_norm_backward(dout, dz, x, y, stats, *, w_post=None, w_pre=None, gate=None, rows_per_gate=None, alpha=1.0,
                           p=0.0, seed=0, offset=0, kind="rms", eps=None, grad_dtype=None, dx=None, dy=None,
                           dw_post=None, dw_pre=None, dgate=None, workspace=None, stream=None):
    """``ccdc_residual_norm_backward``: (dx, dy, dw_post, dw_pre, dgate), None for what the forward call lacked.
    ``dz`` comes with ``w_pre``, and only then; ``dout`` may be None (zero) beside it.  ``eps`` is accepted for symmetry; the forward's is in ``stats``."""
    import torch

    ctx = _elsewhere(x, stream)
    if ctx is not None:
        with ctx:
            return residual_norm_backward(dout, dz, x, y, stats, w_post=w_post, w_pre=w_pre, gate=gate,
                                          rows_per_gate=rows_per_gate, alpha=alpha, p=p, seed=seed, offset=offset,
                                          kind=kind, grad_dtype=grad_dtype, dx=dx, dy=dy, dw_post=dw_post, dw_pre=dw_pre,
                                          dgate=dgate, workspace=workspace)
    M, D, ldx, ldy, pw, pp, pg, per = _norm_tensors(x, y, w_post, w_pre, gate, rows_per_gate)
    code = _block_dtype(x)
    gt = x.dtype if grad_dtype is None else grad_dtype
    if gt != x.dtype and gt != torch.float32:
        raise TypeError("grad_dtype is the tensors' dtype or float32")
    ps = _vector(stats, "stats (of residual_norm_forward with save)", x, 4 * M, torch.float32)

    def given(t, name):
        return (None, D) if t is None else (t.data_ptr(), _rows(t, name, x, x.shape))

    def rows_out(t, name):
        if t is None:
            t = _empty_like(x)
            return t, t.data_ptr(), D
        return t, t.data_ptr(), _rows(t, name, x, x.shape)

    def param_out(t, of, name):
        if of is None:
            if t is not None:
                raise ValueError(f"{name}: the forward call has no such input")
            return None, None
        if t is None:
            t = torch.empty_like(of, dtype=gt)
            return t, t.data_ptr()
        return t, _vector(t, name, x, of.numel(), gt)

    po, ldo = given(dout, "dout")
    pz, ldz = given(dz, "dz")
    dx, pdx, lddx = rows_out(dx, "dx")
    if y is None:
        if dy is not None:
            raise ValueError("dy: the forward call has no such input")
        pdy, lddy = None, D
    else:
        dy, pdy, lddy = rows_out(dy, "dy")
    dw_post, p1 = param_out(dw_post, w_post, "dw_post")
    dw_pre, p2 = param_out(dw_pre, w_pre, "dw_pre")
    dgate, p3 = param_out(dgate, gate, "dgate")
    L = lib()
    if workspace is None:
        ws_bytes = L.ccdc_residual_norm_workspace_bytes(M, D)
        workspace = x.new_empty(ws_bytes, dtype=torch.uint8)
        pws = workspace.data_ptr()
    else:
        pws, ws_bytes = _buffer(workspace, "workspace", x)
    status = L.ccdc_residual_norm_backward(
        M, D, code, F32 if gt == torch.float32 else code, NORMS[kind], po, ldo, pz, ldz, x.data_ptr(), ldx,
        None if y is None else y.data_ptr(), ldy, ps, pw, pp, pg, per, alpha, p, seed, offset, pdx, lddx, pdy, lddy,
        p1, p2, p3, pws, ws_bytes, _handle(x))
    if status:
        _check(status, "ccdc_residual_norm_backward")
    return dx, dy, dw_post, dw_pre, dgate


def _ffn_tensors(x, w_gate, w_up, w_down):
    M, D = x.shape if x.dim() == 2 else (0, 0)
    F = w_gate.shape[0]
    ldx = _rows(x, "x")
    ldw = _rows(w_gate, "w_gate", x, (F, D))
    if _rows(w_up, "w_up", x, (F, D)) != ldw:
        raise ValueError("w_gate and w_up need one row stride")
    return M, D, F, ldx, ldw, _rows(w_down, "w_down", x, (D, F))


def _ffn_aligned(size, *values):
    """whether these addresses (given in bytes) and lengths (given in elements) are multiples of 16 bytes"""
    addresses, lengths = 0, 0
    for address, length in values:
        addresses |= address
        lengths |= length
    return int(addresses % 16 == 0 and lengths * size % 16 == 0)


def ffn_forward(x, w_gate, w_up, w_down, act="silu", save=False, out=None, saved=None, workspace=None, stream=None):
    """``ccdc_ffn_forward``: (act(x w_gate^T) * (x w_up^T)) w_down^T.  Returns y, or (y, saved) with ``save``;
    ``saved`` is opaque and goes to ``ffn_backward``."""
    import torch

    ctx = _elsewhere(x, stream)
    if ctx is not None:
        with ctx:
            return ffn_forward(x, w_gate, w_up, w_down, act, save, out, saved, workspace)
    M, D, F, ldx, ldw, ldd = _ffn_tensors(x, w_gate, w_up, w_down)
    code, L = _block_dtype(x), lib()
    if out is None:
        out, ldy = _empty_like(x), D
    else:
        ldy = _rows(out, "out", x, x.shape)
    ptrs = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), out.data_ptr()
    psaved = None
    if save:
        need = L.ccdc_ffn_saved_bytes(M, F, code)
        if saved is None:
            saved = x.new_empty(need, dtype=torch.uint8)
        psaved = _buffer(saved, "saved", x, need)[0]
    if workspace is None:
        aligned = _ffn_aligned(x.element_size(), *zip(ptrs, (ldx, ldw, D, ldd, ldy)), (0, F))
        ws_bytes = L.ccdc_ffn_workspace_bytes(M, D, F, code, 0, aligned)
        workspace = x.new_empty(ws_bytes, dtype=torch.uint8)
        pws = workspace.data_ptr()
    else:
        pws, ws_bytes = _buffer(workspace, "workspace", x)
    status = L.ccdc_ffn_forward(M, D, F, code, ACTS[act], ptrs[0], ldx, ptrs[1], ptrs[2], ldw, ptrs[3], ldd, ptrs[4], ldy,
                                psaved, pws, ws_bytes, _handle(x))
    if status:
        _check(status, "ccdc_ffn_forward")
    return (out, saved) if save else out


def ffn_backward(dy, x, w_gate, w_up, w_down, saved, act="silu", grad_dtype=None, dx=None, dw_gate=None, dw_up=None,
                 dw_down=None, workspace=None, stream=None):
    """``ccdc_ffn_backward``: (dx, dw_gate, dw_up, dw_down).  Gradients may be passed in (contiguous, e.g. slices of
    a partition row); with ``grad_dtype`` float32 the sums are not rounded to the tensors' type, as their factors a, dh
    and du are."""
    import torch

    ctx = _elsewhere(x, stream)
    if ctx is not None:
        with ctx:
            return ffn_backward(dy, x, w_gate, w_up, w_down, saved, act, grad_dtype, dx, dw_gate, dw_up, dw_down, workspace)
    M, D, F, ldx, ldw, ldd = _ffn_tensors(x, w_gate, w_up, w_down)
    code, L = _block_dtype(x), lib()
    gt = x.dtype if grad_dtype is None else grad_dtype
    if gt != x.dtype and gt != torch.float32:
        raise TypeError("grad_dtype is the tensors' dtype or float32")
    lddy = _rows(dy, "dy", x, x.shape)
    psaved = _buffer(saved, "saved (of ffn_forward with save)", x, L.ccdc_ffn_saved_bytes(M, F, code))[0]
    if dx is None:
        dx, lddx = _empty_like(x), D
    else:
        lddx = _rows(dx, "dx", x, x.shape)
    grads, at = [], []
    for t, shape, name in ((dw_gate, (F, D), "dw_gate"), (dw_up, (F, D), "dw_up"), (dw_down, (D, F), "dw_down")):
        if t is None:
            t = x.new_empty(shape, dtype=gt)
            at.append(t.data_ptr())
        else:
            at.append(_vector(t, name, x, D * F, gt))
        grads.append(t)
    ptrs = dy.data_ptr(), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), dx.data_ptr()
    if workspace is None:
        aligned = _ffn_aligned(x.element_size(), *zip(ptrs, (lddy, ldx, ldw, D, ldd, lddx)), (0, F))
        ws_bytes = L.ccdc_ffn_workspace_bytes(M, D, F, code, 1, aligned)
        workspace = x.new_empty(ws_bytes, dtype=torch.uint8)
        pws = workspace.data_ptr()
    else:
        pws, ws_bytes = _buffer(workspace, "workspace", x)
    status = L.ccdc_ffn_backward(M, D, F, code, F32 if gt == torch.float32 else code, ACTS[act], ptrs[0], lddy, ptrs[1], ldx,
                                 ptrs[2], ptrs[3], ldw, ptrs[4], ldd, psaved, ptrs[5], lddx, *at,
                                 pws, ws_bytes, _handle(x))
    if status:
        _check(status, "ccdc_ffn_backward")
    return dx, *grads


def block_status():
    """after a synchronise: raises if a bounded wait inside a feed-forward kernel ever ran out on this device."""
    _check(lib().ccdc_block_status(), "ccdc_block_status")


def num_kernel_launches() -> int:
    return lib().ccdc_num_kernel_launches()


def last_gather_kernel() -> str:
    """Kernel form of this thread's most recent gather launch (combine, encode, decode, fused encode)."""
    return lib().ccdc_last_gather_kernel().decode()


def last_decode_kernel() -> str:
    """Kernel form of this thread's most recent fused decode launch."""
    return lib().ccdc_last_decode_kernel().decode()


def map_last_kernel() -> str:
    """Name of the kernel the most recent ``Plan.map`` launched."""
    return lib().ccdc_map_last_kernel().decode()
